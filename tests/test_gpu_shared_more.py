"""Shared prompts: the example run whole, bounded waits, calls that follow one another on one
cache, and groups of a size at which the kernels change."""
import os
import sys

import numpy as np
import pytest
import torch

from _parity import check_attention, dev
from paper_2607_06601_gb300 import trr, workloads as wl
from test_gpu_group_attn import LAYOUTS, check, family, last_of

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def test_the_example_runs():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import shared_prompt
    got = shared_prompt.main(quiet=True)
    assert torch.isfinite(got["rows"].float()).all()
    # a window and the sinks: the number of pages stops growing
    assert all(sum(a) <= sum(got["pages"][2]) + 8 for a in got["pages"][2:])


@pytest.mark.parametrize("members", [2, 40])  # few rows, and the tensor kernel
def test_a_wait_that_runs_out_is_reported_and_the_cache_serves_on(members):
    rng = np.random.default_rng([30, members])
    h, kids = family(rng, LAYOUTS[0], 1, members, 300, 20)
    ts = last_of(h, kids)
    check(h, rng, kids, ts, [2] * members, [1] * members, 0, [0, members])
    q = dev(wl.bf16_bits(rng.standard_normal((members, h.Hq, h.d), dtype=np.float32)), torch.bfloat16)
    modes = dev(np.full(members, 2, np.uint8), torch.uint8)
    for _ in range(3):
        h.gpu.set_wait_limit(1)
        h.gpu.decode_attn_shared(0, h.ints(kids), h.ints(ts), q, modes, h.ints([0, members]))
        # (the few-row kernel's only waits are for its copies, which may be there at its first look)
        assert h.gpu.status() in ((0, 8) if members == 2 else (8,))
        h.gpu.set_wait_limit(0)
        check(h, rng, kids, ts, [2] * members, [1] * members, 0, [0, members])


@pytest.mark.parametrize("lay", LAYOUTS)
@pytest.mark.parametrize("members", [3, 4, 8, 11, 12, 16, 17])
def test_group_sizes_at_which_the_kernel_changes(lay, members):
    """Rows of a group around 8 / groups (few rows), 32, 64 and 128 (copies in the tensor kernel)."""
    rng = np.random.default_rng([31, members])
    h, kids = family(rng, lay, 1, members, 180, 9)
    check(h, rng, kids, last_of(h, kids), [2] * members, [1] * members, 0, [0, members])


def test_calls_in_a_row_with_other_shapes():
    """One workspace, calls of changing size without a wait between: each finds its own plan."""
    rng = np.random.default_rng(32)
    h, kids = family(rng, LAYOUTS[1], 2, 20, 260, 30)
    ts = last_of(h, kids)
    calls = []
    for n, offsets, sinks in ((40, [0, 20, 40], 0), (3, [0, 3], 2), (40, None, 7), (1, None, 0), (25, [0, 20], 0)) * 3:
        modes = rng.choice(3, n)
        windows = rng.choice([3, 50, 400], n)
        q = wl.bf16_bits(rng.standard_normal((n, h.Hq, h.d), dtype=np.float32))
        args = (0, h.ints(kids[:n]), h.ints(ts[:n]), dev(q, torch.bfloat16), dev(modes.astype(np.uint8), torch.uint8))
        kw = dict(windows=h.ints(windows))
        out = h.gpu.decode_attn_sinks(*args, sinks, **kw) if offsets is None else h.gpu.decode_attn_shared(*args, h.ints(offsets), sinks=sinks, **kw)
        calls.append((out, n, q, modes, windows, sinks))
    assert h.gpu.status() == 0
    for out, n, q, modes, windows, sinks in calls:
        check_attention(out.double().cpu().numpy(), h.attend(0, kids[:n], ts[:n], q, modes, windows, sinks), modes)


def test_attention_between_appends_and_forks():
    """Every call sees what the calls before it on the stream did."""
    rng = np.random.default_rng(33)
    h, kids = family(rng, LAYOUTS[0], 1, 4, 120, 6, archive=16)
    for turn in range(4):
        ts = last_of(h, kids)
        for s, t in zip(kids, ts):
            h.append(rng, 0, s, [t + 1], p_skip=0.0)
        check(h, rng, kids, [t + 1 for t in ts], [2, 1, 2, 2], [40] * 4, 3, [0, 4])
        h.fork([kids[turn]] * 3, [k for k in kids if k != kids[turn]], [ts[turn] + 2] * 3)
        ts = last_of(h, kids)
        check(h, rng, kids, ts, [2] * 4, [1] * 4, 0, [0, 4])
    h.gpu.compact()
    check(h, rng, kids, ts, [2] * 4, [1] * 4, 0, [0, 4])


def test_offsets_past_32_bits():
    """A pool of more than 4 GB: pages at its far end are forked, moved and attended."""
    rng = np.random.default_rng(34)
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GB")
    from _shared import Holder
    pages = (4 << 30) // (128 + 2 * 64 * 128 * 4) + 300  # of 16 bits: 64 slots x 2 KV heads x 512 bytes
    h = Holder(1, 6, 4, 2, 128, 64, 64, 1024, [64, 64, 64, pages], archive=8)
    # the pages handed out next lie behind 4 GB
    h.gpu.region("next_page").view(torch.int32)[3] = pages - 200
    n = 500
    for s in (0, 1):
        k, v = (wl.bf16_bits(rng.standard_normal((n, 2, 128), dtype=np.float32)) for _ in range(2))
        h.append(rng, 0, s, np.arange(n), k=k, v=v, bits=np.full(n, 16), p_skip=0.0)
    h.fork([0, 0, 1], [2, 3, 4], [n, 450, 33])
    seqs, ts = [0, 2, 3, 4], [n - 1, n - 1, 449, 32]
    check(h, rng, seqs, ts, [2] * 4, [1] * 4, 0, [0, 3])
    check(h, rng, seqs, ts, [1] * 4, [100] * 4, 20)
    h.free([1])
    h.gpu.compact()  # from the far end to the front
    assert int(h.gpu.region("next_page").view(torch.int32)[3]) < 64
    check(h, rng, seqs, ts, [2] * 4, [1] * 4, 0, [0, 3])
