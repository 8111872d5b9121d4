"""Arguments of attention of chunks that the host refuses before anything is enqueued."""
import numpy as np
import pytest
import torch

from paper_2607_06601_gb300 import trr
from test_gpu_chunk import LAYOUTS, fill, holder

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def test_rows_over_their_queries():
    """Queries are read after the first rows are written, so the two may not overlap."""
    rng = np.random.default_rng(1)
    h = holder(LAYOUTS[0])
    fill(h, rng, 0, 0, 60)
    n = 20
    both = torch.randn(2 * n, h.Hq, h.d, device="cuda").bfloat16()
    before = both.clone()
    args = (0, h.ints([0]), h.ints([40]), h.ints([0, n]))
    modes = torch.full((n,), 2, dtype=torch.uint8, device="cuda")
    for q, out in ((both[:n], both[:n]), (both[:n], both[1:n + 1]), (both[n - 1:2 * n - 1], both[:n])):
        with pytest.raises(trr.TrrError):
            h.gpu.chunk_attn(*args, q, modes, out=out)
    assert torch.equal(both, before) and h.gpu.status() == 0
    want = h.gpu.chunk_attn(*args, both[:n], modes)
    assert torch.equal(h.gpu.chunk_attn(*args, both[:n], modes, out=both[n:]), want)


def test_logarithms_off_their_alignment():
    h = holder(LAYOUTS[0])
    q = torch.zeros(4, h.Hq, h.d, dtype=torch.bfloat16, device="cuda")
    out, workspace = torch.zeros_like(q), h.gpu.chunk_workspace(1, 4)
    ids, offsets, modes = h.ints([0]), h.ints([0, 4]), torch.zeros(4, dtype=torch.uint8, device="cuda")
    space = torch.zeros(4 * h.Hq * 4 + 16, dtype=torch.uint8, device="cuda")
    for off, code in ((2, 1), (4, 0)):
        got = trr.load().trr_chunk_attn(h.gpu.handle, 0, 1, ids.data_ptr(), ids.data_ptr(), offsets.data_ptr(), 4, q.data_ptr(), modes.data_ptr(), None, 1, 0,
                                        0.0, out.data_ptr(), space.data_ptr() + off, workspace.data_ptr(), workspace.numel(), None)
        assert got == code
    assert h.gpu.status() == 0
