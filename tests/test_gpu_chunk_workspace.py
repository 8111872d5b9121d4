"""How large the workspace of attention of chunks is, by default and at most."""
import numpy as np
import pytest
import torch

from _shared import Holder
from paper_2607_06601_gb300 import trr
from test_gpu_chunk import call, check

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def test_no_more_than_the_pools_hold():
    """Contexts far longer than the pools: the workspace is one for what the pools hold, for each chunk, and does for a sequence
    that has all of it."""
    h = Holder(1, 3, 4, 2, 64, 32, 16, 200_000, [10, 20, 30, 15], archive=2, max_queries=1)
    slots = 75 * 16
    least = trr.trr_chunk_workspace_bytes(h.gpu.handle, 3, 100, 0)
    held = trr.trr_chunk_workspace_bytes(h.gpu.handle, 3, 100, 3 * slots)
    assert trr.trr_chunk_workspace_bytes(h.gpu.handle, 3, 100, 3 * 200_000) == held <= least + 2 * (3 * slots + 96) * 2 * 64 * 2
    assert h.gpu.chunk_workspace(3, 100).numel() == held
    rng = np.random.default_rng(1)
    widths = np.repeat([2, 4, 8, 16], [160, 320, 480, 240])
    rng.shuffle(widths)
    for at in range(0, slots, 600):
        h.append(rng, 0, 1, np.arange(at, at + 600), bits=widths[at:at + 600], p_skip=0.0)
    check(h, rng, [1, 1, 1], [slots - 40, 500, 100_000], [40, 50, 10], [2] * 100, [1] * 100)
    call(h, rng, [1, 1, 1], [slots - 40, slots - 40, slots - 40], [40, 30, 30], [2] * 100, [1] * 100)
