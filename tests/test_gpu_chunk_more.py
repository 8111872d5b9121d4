"""Attention of chunks where its kernels' rules change: references that move, values that binary16 does
not hold, long runs cut between CTAs, waits that run out, pools past 4 GB.

Bounds: tests/test_gpu_chunk.py.  Where scores are large, their own error (2^-11 of scale sum |q k|, from
keys in binary16) bounds weights and rows as `rows_within` says."""
import numpy as np
import pytest
import torch

from _parity import check_attention, dev
from _shared import Holder
from paper_2607_06601_gb300 import trr, workloads as wl
from test_gpu_chunk import LAYOUTS, call, check, fill, holder, truth

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def rows_within(got, ref, off):
    """A score's error e moves its weight by a factor up to exp(e), so a row by at most 2 (exp(e) - 1) of the largest value
    that it joins; beside it stand the output's rounding (2^-8 of the value) and the library's 2e-2."""
    most = np.abs(ref).max(-1, keepdims=True)
    bound = 2 * np.expm1(off)[:, :, None] * np.maximum(most, 4.0) + 2.0 ** -8 * np.abs(ref) + 2e-2
    assert (np.abs(got.double().cpu().numpy() - ref) <= bound).all()


@pytest.mark.parametrize("lay", [LAYOUTS[0], LAYOUTS[2]])
@pytest.mark.parametrize("shape", ["up", "down", "spike", "steps", "last"])
def test_scores_that_grow_and_fall_along_the_past(lay, shape):
    """A row's reference comes from its first tile; scores that rise above it by far more than binary16's range, all
    along, in one token of a tile, or at its very end, have to move it, and with it what was summed before."""
    rng = np.random.default_rng([1, len(shape), ord(shape[0])])
    h = holder(lay)
    n, new = 700, 140
    at = np.arange(n)
    size = {"up": at / 8.0, "down": (n - at) / 8.0, "spike": np.where(at == 333, 60.0, 1.0), "steps": np.where(at % 200 < 100, 1.0, 1.0 + at / 10.0),
            "last": np.where(at == 95, 80.0, np.where(at == 479, 95.0, 0.5))}[shape]
    unit = rng.standard_normal(h.d).astype(np.float32)
    unit /= np.sqrt((unit ** 2).sum())
    k = size[:, None, None] * unit + 0.05 * rng.standard_normal((n, h.Hkv, h.d))
    q = 6.0 * unit + 0.05 * rng.standard_normal((new, h.Hq, h.d))
    h.append(rng, 0, 1, at, k=wl.bf16_bits(k.astype(np.float32)), bits=rng.choice([8, 16], n), p_skip=0.1)
    modes, windows = rng.choice(3, new, p=[0.1, 0.4, 0.5]), rng.integers(1, 500, new)
    q_bits = wl.bf16_bits(q.astype(np.float32))
    out, lse, _, modes, windows = call(h, rng, [1], [n - new], [new], modes, windows, 3, q_bits=q_bits, scale=1.0)
    ref, ref_lse, off = truth(h, 0, [1], [n - new], [new], q_bits, modes, windows, 3, 1.0)
    assert np.nanmax(ref_lse[np.isfinite(ref_lse)]) > 100
    rows_within(out, ref, off)
    seen = np.isfinite(ref_lse)
    assert (np.abs(lse.double().cpu().numpy()[seen] - ref_lse[seen]) <= off[seen] + 2.0 ** -20 * np.abs(ref_lse[seen])).all()


@pytest.mark.parametrize("lay", [LAYOUTS[1], LAYOUTS[5]])
@pytest.mark.parametrize("kind", ["tiny v", "tiny k", "huge v", "huge k", "wide v"])
def test_values_of_16_bits_that_binary16_does_not_hold(lay, kind):
    rng = np.random.default_rng([2, len(kind), ord(kind[-1])])
    h = holder(lay)
    n, new = 260, 90
    k, v = (rng.standard_normal((n, h.Hkv, h.d)) for _ in range(2))
    scale = 0.0
    if kind == "tiny v":
        v *= 2.0 ** -30
    elif kind == "tiny k":
        k *= 2.0 ** -34
        scale = 2.0 ** 31
    elif kind == "huge v":
        v[:, 0] *= 2.0 ** 40
    elif kind == "huge k":
        k[:, :, 0] = 2.0 ** 17 * np.sign(k[:, :, 0])
        scale = 2.0 ** -18
    else:
        v *= 2.0 ** rng.integers(-40, 10, (n, 1, 1))
    h.append(rng, 0, 0, np.arange(n), k=wl.bf16_bits(k.astype(np.float32)), v=wl.bf16_bits(v.astype(np.float32)), bits=np.full(n, 16), p_skip=0.0)
    modes, windows = rng.choice([1, 2], new), rng.integers(1, 40, new)
    out, _, q_bits, modes, windows = call(h, rng, [0], [n - new], [new], modes, windows, 2, scale=scale)
    ref = truth(h, 0, [0], [n - new], [new], q_bits, modes, windows, 2, scale if scale else None)[0]
    got = out.double().cpu().numpy()
    # Half a bf16 step of the value (2^-8), and the weights' half step of binary16, 2^-11 of each, in the heads whose values
    # it holds: at most 2^-11 sum w |v|; 2^-12 of the same for sums in binary32.  (Keys: 16-bit ones are exact there.)
    h.values, values = (lambda *a: [np.abs(x) if i == 2 else x for i, x in enumerate(values(*a))]), h.values
    spread = truth(h, 0, [0], [n - new], [new], q_bits, modes, windows, 2, scale if scale else None)[0]
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -12) * spread).all()


@pytest.mark.parametrize("lay", [dict(Hq=4, Hkv=4, d=64, G=32, P=32), dict(Hq=8, Hkv=2, d=128, G=64, P=64), dict(Hq=2, Hkv=2, d=128, G=128, P=32)])
@pytest.mark.parametrize("bits", [2, 4, 8, 16])
def test_long_pasts(lay, bits):
    """Over 12,000 tokens of each width: runs of dozens of tiles, cut between CTAs and joined.  Rows are held to 1.1 times
    the root mean square of the output's own rounding: keys (2^-12 in the mean) and weights (2^-12 each, averaged over
    thousands) add less than a tenth to the 2^-9 of bf16."""
    rng = np.random.default_rng([3, bits])
    tokens, new = 12000, 200
    h = Holder(1, 1, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], tokens, [tokens // lay["P"] + 4] * 4, archive=16)
    for at in range(0, tokens, 1000):
        h.append(rng, 0, 0, np.arange(at, at + 1000), bits=np.full(1000, bits), p_skip=0.0)
    out, _, q_bits, modes, windows = call(h, rng, [0], [tokens - new], [new], [2] * new, [1] * new)
    ref = truth(h, 0, [0], [tokens - new], [new], q_bits, modes, windows, 0)[0]
    rounding = np.sqrt(((torch.from_numpy(ref).bfloat16().double().numpy() - ref) ** 2).mean())
    error = np.sqrt(((out.double().cpu().numpy() - ref) ** 2).mean())
    assert error <= 1.1 * rounding, f"{error / rounding:.3f} times the rounding of the output"


def test_many_blocks_of_both_modes():
    """A chunk of 1000 queries of a layout with 7 heads for its KV head: dozens of blocks of rows, whose edges lie inside
    a query's heads; windows that every block sees another part of."""
    rng = np.random.default_rng(4)
    h = holder(LAYOUTS[4], maxctx=1800, caps=500)
    fill(h, rng, 0, 0, 1700)
    n = 1000
    check(h, rng, [0], [700], [n], rng.choice(3, n, p=[0.1, 0.6, 0.3]), np.where(rng.random(n) < 0.5, 40, rng.integers(1, 900, n)), 11)


@pytest.mark.parametrize("lay", [LAYOUTS[0], LAYOUTS[2]])
def test_calls_in_a_row_with_other_shapes(lay):
    """One workspace, calls of changing size without a wait between: each finds its own plan."""
    rng = np.random.default_rng(5)
    h = holder(lay, S=3)
    for s in range(3):
        fill(h, rng, 0, s, 500 + 100 * s)
    workspace = h.gpu.chunk_workspace(3, 700)
    calls = []
    for seqs, starts, lens, sinks in (([0, 1, 2], [400, 0, 650], [100, 600, 50], 0), ([1], [599], [1], 3), ([2, 0], [300, 490], [400, 10], 0), ([0], [0], [500], 1)) * 3:
        n = sum(lens)
        modes, windows = rng.choice(3, n).astype(np.uint8), rng.integers(1, 300, n).astype(np.int32)
        q = dev(wl.bf16_bits(rng.standard_normal((n, h.Hq, h.d), dtype=np.float32)), torch.bfloat16)
        calls.append((0, h.ints(seqs), h.ints(starts), h.ints(np.append(0, np.cumsum(lens))), q, dev(modes, torch.uint8), dev(windows, torch.int32), 0, sinks))
    want = []
    for c in calls:
        want.append(h.gpu.chunk_attn(*c))
        torch.cuda.synchronize()
    got = [h.gpu.chunk_attn(*c, workspace=workspace) for c in calls]
    assert h.gpu.status() == 0 and all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_wait_that_runs_out():
    rng = np.random.default_rng(6)
    h = holder(LAYOUTS[2])
    fill(h, rng, 0, 0, 900)
    n = 150
    q = dev(wl.bf16_bits(rng.standard_normal((n, h.Hq, h.d), dtype=np.float32)), torch.bfloat16)
    modes = torch.full((n,), 2, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        h.gpu.set_wait_limit(1)
        h.gpu.chunk_attn(0, h.ints([0]), h.ints([750]), h.ints([0, n]), q, modes)
        assert h.gpu.status() == 8
        h.gpu.set_wait_limit(0)
        check(h, rng, [0], [750], [n], [2] * n, [1] * n)


def test_offsets_past_32_bits():
    """A pool of more than 4 GB: pages at its far end are attended and read back."""
    rng = np.random.default_rng(7)
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GB")
    pages = (4 << 30) // (128 + 2 * 64 * 128 * 4) + 300  # of 16 bits: 64 slots x 2 KV heads x 512 bytes
    h = Holder(1, 2, 4, 2, 128, 64, 64, 1024, [64, 64, 64, pages], archive=8)
    h.gpu.region("next_page").view(torch.int32)[3] = pages - 200  # the pages handed out next lie behind 4 GB
    n = 500
    h.append(rng, 0, 1, np.arange(n), bits=np.full(n, 16), p_skip=0.0)
    check(h, rng, [1], [300], [200], rng.choice(3, 200), [100] * 200, 5)
    k, v, bits = h.gpu.read(0, h.ints([1]), h.ints([0]), h.ints([0, n]), n, dtype=torch.float32)
    pos, kk, vv = h.values(0, 1, 1)
    assert len(pos) == n and np.array_equal(k[:, 1].cpu().numpy(), kk.astype(np.float32)) and np.array_equal(v[:, 1].cpu().numpy(), vv.astype(np.float32))
    assert (bits == 16).all()


def test_outputs_past_32_bits():
    """More than 2^31 elements read back, at a stride: the far rows of a tensor of 5 GB."""
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GB")
    rng = np.random.default_rng(8)
    h = holder(LAYOUTS[0])
    h.append(rng, 0, 0, np.arange(300))
    rows, wide = 2_200_000, 4 * 64
    big = torch.full((rows, 4, wide), 7.0, dtype=torch.bfloat16, device="cuda")
    k, v = big[:, 1].view(rows, 4, 64), big[:, 3].view(rows, 4, 64)
    bits = torch.full((rows, 4), 9, dtype=torch.uint8, device="cuda")
    h.gpu.read(0, h.ints([0, 0]), h.ints([0, 100]), h.ints([7, 107, 107]), rows, k=k, v=v, bits=bits)
    h.gpu.read(0, h.ints([0]), h.ints([100]), h.ints([rows - 200, rows]), rows, k=k, v=v, bits=bits)
    assert h.gpu.status() == 0
    one = h.gpu.read(0, h.ints([0]), h.ints([0]), h.ints([0, 300]), 300)
    for a, b in zip((k, v, bits), one):
        assert torch.equal(a[7:107], b[:100]) and torch.equal(a[rows - 200:], b[100:])
    assert (big[:, 0] == 7).all() and (k[107:rows - 200] == 7).all() and (bits[107:rows - 200] == 9).all()


@pytest.mark.parametrize("lay,new", [(dict(Hq=32, Hkv=8, d=128, G=64, P=32), 30), (dict(Hq=8, Hkv=8, d=128, G=64, P=16), 9), (dict(Hq=16, Hkv=8, d=64, G=64, P=32), 20)])
def test_short_blocks_whose_tiles_come_in_any_order(lay, new):
    """Many blocks of few rows, whose tiles the two halves of a CTA take in turn: a tile may land before the one ahead of
    it.  Bit for bit the same rows over calls with the tiles in memory, and held to the definition."""
    rng = np.random.default_rng([9, new])
    S, total = 24, 1500
    h = holder(lay, S=S, maxctx=total + new, caps=S * (total + new) // (2 * lay["P"]) + 4 * S, archive=2 * S + 4)
    for s in range(S):
        fill(h, rng, 0, s, total + new, bits=None)
    n = S * new
    modes, windows = rng.choice(3, n, p=[0.1, 0.4, 0.5]), np.full(n, 300)
    q_bits = wl.bf16_bits(rng.standard_normal((n, h.Hq, h.d), dtype=np.float32))
    args = ([*range(S)], [total] * S, [new] * S, modes, windows, 4)
    out, lse = check(h, rng, *args, q_bits=q_bits)
    cold = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")  # twice L2
    call_args = (0, h.ints(args[0]), h.ints(args[1]), h.ints(np.arange(S + 1) * new), dev(q_bits, torch.bfloat16), dev(modes.astype(np.uint8), torch.uint8))
    for i in range(60):
        if i % 2:
            cold.fill_(i)
        assert torch.equal(h.gpu.chunk_attn(*call_args, window_scalar=300, sinks=4), out), i
    assert h.gpu.status() == 0


def test_more_rows_than_32_bits_count_are_refused():
    c = trr.Cache(1, 1, 2048, 1, 64, 64, 16, 64, [4] * 4, max_append=16, max_queries=1)
    with pytest.raises(trr.TrrError):
        trr.trr_chunk_workspace_bytes(c.handle, 1, 1 << 20, 64)
    assert trr.trr_chunk_workspace_bytes(c.handle, 1, (1 << 20) - 1, 64) > 0
