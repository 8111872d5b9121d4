"""Calls that follow one another without a wait: every kernel of a call sees its own call's plan
and what the calls before it left in the tables, the pages and the rows, on whichever SM it runs."""
import numpy as np
import pytest
import torch

from _parity import dev
from paper_2607_06601_gb300 import workloads as wl
from test_gpu_group_attn import LAYOUTS, family

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("lay,members", [(LAYOUTS[1], 12), (LAYOUTS[2], 12), (LAYOUTS[3], 40)])
def test_rows_are_those_of_the_same_calls_waited_for(lay, members):
    """A beam search in small: forks, releases and compactions that move pages, rows computed by a
    kernel of the stream just before each call, and calls whose plans differ, once with the GPU
    waited for after each call and three times without: the same bits."""
    rng = np.random.default_rng([1, members])
    h, kids = family(rng, lay, 2, members, 330, 12)
    n = 2 * members
    turns = []
    for _ in range(24):
        m = int(rng.integers(2, n + 1))
        gone = rng.choice(kids, 3, replace=False)
        cut = rng.integers(100, 331, 3)
        modes = rng.choice(3, m, p=(0.1, 0.3, 0.6))
        offsets = np.sort(rng.integers(0, m + 1, int(rng.integers(2, 6))))
        offsets[0], offsets[-1] = 0, m
        turns.append(dict(gone=h.ints(gone), src=h.ints(rng.integers(0, 2, 3)), cut=h.ints(cut), seqs=h.ints(rng.permutation(kids)[:m]),
                          ts=h.ints(rng.integers(90, 345, m)), modes=dev(modes.astype(np.uint8), torch.uint8), offsets=h.ints(offsets),
                          windows=h.ints(rng.choice([3, 60, 400], m)), sinks=int(rng.integers(0, 20)),
                          q=dev(wl.bf16_bits(rng.standard_normal((m, h.Hq, h.d), dtype=np.float32)), torch.bfloat16)))
    q = torch.empty((n, h.Hq, h.d), dtype=torch.bfloat16, device="cuda")

    def go(wait):
        rows = []
        after = torch.cuda.synchronize if wait else lambda: None
        for t in turns:
            m = t["seqs"].numel()
            h.gpu.free(t["gone"])
            after()
            h.gpu.fork(t["src"], t["gone"], t["cut"])
            after()
            h.gpu.compact()
            after()
            torch.mul(t["q"], 1, out=q[:m])
            after()
            rows.append(h.gpu.decode_attn_shared(0, t["seqs"], t["ts"], q[:m], t["modes"], t["offsets"], windows=t["windows"], sinks=t["sinks"]))
            after()
        assert h.gpu.status() == 0
        return rows

    go(True)  # the tables of the first turn then hold what the last one left, each time
    truth = go(True)
    assert all(torch.isfinite(r.float()).all() for r in truth) and sum(bool((r != 0).any()) for r in truth) > 20
    for _ in range(3):
        for i, (a, b) in enumerate(zip(truth, go(False))):
            assert torch.equal(a, b), f"turn {i}"
