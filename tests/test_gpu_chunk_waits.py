"""Waits of attention of chunks under a short limit."""
import pytest
import torch

from paper_2607_06601_gb300 import trr

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def test_a_long_run_under_a_short_limit():
    """Runs of some 200 tiles (about 200 us) under a limit of 100 us: every wait is for something that comes sooner, or
    behind copies that go on."""
    tokens, new, heads, d = 40_000, 2048, 8, 128
    c = trr.Cache(1, 1, heads, heads, d, 64, 64, tokens, [1, 1, 1, tokens // 64], max_append=1000, max_queries=1)
    g = torch.Generator("cuda").manual_seed(1)
    ints = lambda x: torch.as_tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rows = lambda n: torch.randn(n, heads, d, generator=g, device="cuda").bfloat16()  # noqa: E731
    full, wide = (torch.full((1000,), x, dtype=torch.uint8, device="cuda") for x in (2, 16))
    for at in range(0, tokens, 1000):
        c.append(0, ints([0] * 1000), ints(range(at, at + 1000)), rows(1000), rows(1000), wide, full)
    args = (0, ints([0]), ints([tokens - new]), ints([0, new]), rows(new), torch.full((new,), 2, dtype=torch.uint8, device="cuda"))
    workspace = c.chunk_workspace(1, new, tokens)
    want = c.chunk_attn(*args, workspace=workspace)
    assert c.status() == 0
    for _ in range(5):
        c.set_wait_limit(100_000)
        got = c.chunk_attn(*args, workspace=workspace)
        assert c.status() == 0 and torch.equal(got, want)
