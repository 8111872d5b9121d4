"""The few-row kernel's bounded waits: one that runs out is reported, and the cache serves on."""
import numpy as np
import pytest
import torch

from _parity import dev
from paper_2607_06601_gb300 import workloads as wl
from test_gpu_group_attn import LAYOUTS, check, family, last_of

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


# in groups two of the first layout's queries are few rows as well: the tensor kernel, whose waits would run out too, has no segment
@pytest.mark.parametrize("lay,groups", [(LAYOUTS[0], False), (LAYOUTS[2], False), (LAYOUTS[0], True)])
def test_few_rows_whose_wait_runs_out(lay, groups):
    """A limit of a nanosecond against copies from memory that no cache holds: a warp looks for its
    first block, and gives up, within the microsecond that the block takes.  Every try may find its
    blocks there all the same; of ten with hundreds of warps each, one must not."""
    rng = np.random.default_rng([1, int(groups)])
    h, kids = family(rng, lay, 8, 2, 400, 30)
    ts, n = last_of(h, kids), len(kids)
    offsets = [0, 2, 4, 6, 8] if groups else None  # the other queries stand alone
    check(h, rng, kids, ts, [2] * n, [1] * n, 0, offsets)
    q = dev(wl.bf16_bits(rng.standard_normal((n, h.Hq, h.d), dtype=np.float32)), torch.bfloat16)
    modes = dev(np.full(n, 2, np.uint8), torch.uint8)
    cold = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")  # twice L2
    found = []
    for i in range(10):
        cold.fill_(i)
        h.gpu.set_wait_limit(1)
        if groups:
            h.gpu.decode_attn_shared(0, h.ints(kids), h.ints(ts), q, modes, h.ints(offsets))
        else:
            h.gpu.decode_attn_sinks(0, h.ints(kids), h.ints(ts), q, modes, 0)
        found.append(h.gpu.status())
        h.gpu.set_wait_limit(0)
        check(h, rng, kids, ts, [2] * n, [1] * n, 0, offsets)
    assert set(found) <= {0, 8} and 8 in found, found
