"""Attention of chunks of new tokens (trr_chunk_attn) against the definition in 64 bits.

Rows are held to the library's bounds for attention (tests/_parity.py: 5e-3 of a row's largest value
and 2e-2 on top of the output's own rounding).  The logarithm of a softmax sum is off by no more than
its scores are: keys become binary16 (half a step: 2^-11 of a value), so a score by at most
2^-11 scale sum |q k|; 2^-16 stands for the exponentials and the sums in binary32."""
import numpy as np
import pytest
import torch

from _parity import ROW_RTOL, check_attention, dev
from _shared import Holder
from paper_2607_06601_gb300 import trr, workloads as wl

pytestmark = pytest.mark.gpu

LAYOUTS = [dict(Hq=4, Hkv=4, d=64, G=32, P=16), dict(Hq=12, Hkv=4, d=64, G=64, P=32), dict(Hq=8, Hkv=2, d=128, G=64, P=16),
           dict(Hq=4, Hkv=2, d=64, G=32, P=64), dict(Hq=7, Hkv=1, d=128, G=128, P=32), dict(Hq=6, Hkv=6, d=128, G=32, P=64)]


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def holder(lay, S=3, maxctx=1024, caps=400, L=1, **kw):
    return Holder(L, S, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], maxctx, [caps] * 4, **kw)


def fill(h, rng, layer, seq, n, **kw):
    for at in range(0, n, 1000):
        h.append(rng, layer, seq, np.arange(at, min(n, at + 1000)), **kw)


def truth(h, layer, seqs, starts, lens, q_bits, modes, windows, sinks, scale=None):
    """Rows and logarithms of sums in 64 bits, and how far the latter may be off."""
    q = wl.bf16_to_f32(q_bits).astype(np.float64)
    n, g = len(q), h.Hq // h.Hkv
    scale = 1 / np.sqrt(h.d) if scale is None else scale
    out, lse, off = np.zeros((n, h.Hq, h.d)), np.full((n, h.Hq), -np.inf), np.zeros((n, h.Hq))
    row, kept = 0, {}
    for s, start, count in zip(seqs, starts, lens):
        if count == 0:
            continue
        at = slice(row, row + count)
        t, m, w = np.arange(start, start + count)[:, None], modes[at, None], windows[at, None]
        for kvh in range(h.Hkv):
            if (s, kvh) not in kept:
                kept[s, kvh] = h.values(layer, s, kvh)
            pos, k, v = kept[s, kvh]
            see = (pos <= t) & ((m == 2) | ((m == 1) & ((pos > t - w) | (pos < sinks))))
            any_ = see.any(1)
            for head in range(kvh * g, kvh * g + g):
                if not any_.any():
                    continue
                x = np.where(see, scale * (q[at, head] @ k.T), -np.inf)
                top = np.where(any_, x.max(1, initial=-np.inf), 0.0)[:, None]
                p = np.exp(x - top)
                total = p.sum(1)
                out[at, head] = np.where(any_[:, None], p @ v / np.where(any_, total, 1.0)[:, None], 0.0)
                with np.errstate(divide="ignore"):
                    lse[at, head] = np.where(any_, np.log(total) + top[:, 0], -np.inf)
                off[at, head] = np.where(see, scale * (np.abs(q[at, head]) @ np.abs(k).T), 0.0).max(1) * 2.0 ** -11 + 2.0 ** -16
        row += count
    return out, lse, off


def call(h, rng, seqs, starts, lens, modes, windows, sinks=0, layer=0, scale=0.0, expect=0, loud=1.0, q_bits=None, **kw):
    n, offsets = int(sum(lens)), np.append(0, np.cumsum(lens))
    q_bits = wl.bf16_bits(loud * rng.standard_normal((n, h.Hq, h.d), dtype=np.float32)) if q_bits is None else q_bits
    modes, windows = np.asarray(modes, np.uint8), np.asarray(windows, np.int32)
    out, lse = h.gpu.chunk_attn(layer, h.ints(seqs), h.ints(starts), h.ints(offsets), dev(q_bits, torch.bfloat16), dev(modes, torch.uint8),
                                windows=dev(windows, torch.int32), sinks=sinks, softmax_scale=scale, with_lse=True, **kw)
    assert h.gpu.status() == expect
    return out, lse, q_bits, modes, windows


def check(h, rng, seqs, starts, lens, modes, windows, sinks=0, layer=0, scale=0.0, **kw):
    out, lse, q_bits, modes, windows = call(h, rng, seqs, starts, lens, modes, windows, sinks, layer, scale, **kw)
    ref, ref_lse, off = truth(h, layer, seqs, starts, lens, q_bits, modes, windows, sinks, scale if scale > 0 else None)
    check_attention(out.double().cpu().numpy(), ref, modes)
    lse = lse.double().cpu().numpy()
    empty = np.isneginf(ref_lse)
    assert np.isneginf(lse[empty]).all() and (np.abs(lse[~empty] - ref_lse[~empty]) <= off[~empty]).all()
    return out, lse


@pytest.mark.parametrize("lay", LAYOUTS)
@pytest.mark.parametrize("past,new", [(0, 1), (1, 1), (0, 17), (60, 5), (127, 1), (128, 130), (300, 64), (40, 333)])
def test_one_chunk_all_full(lay, past, new):
    rng = np.random.default_rng([1, past, new])
    h = holder(lay)
    fill(h, rng, 0, 1, past + new)
    check(h, rng, [1], [past], [new], [2] * new, [1] * new)


@pytest.mark.parametrize("lay", LAYOUTS)
@pytest.mark.parametrize("sinks", [0, 1, 5, 200])
def test_routed_chunks_of_odd_lengths(lay, sinks):
    """Every mode, windows from one token to past the start, chunks of a token and of none, a
    sequence that stores nothing, one named twice."""
    rng = np.random.default_rng([2, sinks])
    h = holder(lay, S=5, maxctx=900)
    total, lens = [700, 129, 64, 1, 0], [150, 129, 1, 1, 0]
    for s, n in enumerate(total):
        fill(h, rng, 0, s, n)
    seqs, starts = [0, 1, 2, 3, 4, 4, 0], [550, 0, 63, 0, 0, 7, 20]
    lens = lens + [3, 77]
    n = sum(lens)
    windows = np.exp(rng.uniform(0, np.log(1200), n)).astype(np.int32)
    check(h, rng, seqs, starts, lens, rng.choice(3, n), windows, sinks)


@pytest.mark.parametrize("lay", LAYOUTS[:4])
@pytest.mark.parametrize("window,sinks", [(1, 0), (30, 4), (100, 64), (257, 0), (2 ** 31 - 1, 3)])
def test_local_chunks_far_into_a_sequence(lay, window, sinks):
    rng = np.random.default_rng([3, window % 1000, sinks])
    h = holder(lay, maxctx=2200, caps=600)
    fill(h, rng, 0, 0, 2000)
    fill(h, rng, 0, 2, 1500)
    n = 130
    check(h, rng, [0, 2], [1890, 1480], [110, 20], [1] * n, [window] * n, sinks)


@pytest.mark.parametrize("bits", [2, 4, 8, 16])
@pytest.mark.parametrize("lay", LAYOUTS)
def test_one_width(lay, bits):
    rng = np.random.default_rng([4, bits])
    h = holder(lay)
    fill(h, rng, 0, 0, 400, bits=np.full(400, bits), p_skip=0.0)
    check(h, rng, [0], [260], [140], rng.choice(3, 140), [50] * 140, 2)


@pytest.mark.parametrize("lay", [LAYOUTS[0], LAYOUTS[2]])
def test_nothing_stored_in_sight(lay):
    """Skip tokens alone, windows over a gap, and queries before the first stored token."""
    rng = np.random.default_rng(5)
    h = holder(lay)
    h.append(rng, 0, 0, np.arange(50), p_skip=1.0)
    h.append(rng, 0, 1, np.concatenate([np.arange(40, 60), np.arange(300, 303)]), p_skip=0.0)
    n = 300
    out, lse = check(h, rng, [0, 1], [0, 3], [50, 250], [2] * 50 + [1] * 250, [10] * n)
    assert (out[:87] == 0).all() and np.isneginf(lse[:87]).all() and np.isneginf(lse[150:]).all()


def test_scores_far_apart_and_scales():
    rng = np.random.default_rng(6)
    for lay in (LAYOUTS[1], LAYOUTS[5]):
        h = holder(lay)
        fill(h, rng, 0, 0, 700, k=None)
        for scale, loud in ((0.0, 30.0), (1e-3, 1.0), (0.5, 2.0), (0.0, 1e-20)):
            n = 200
            out, lse, q, modes, windows = call(h, rng, [0], [500], [n], [2] * n, [1] * n, scale=scale, loud=loud)
            ref, ref_lse, off = truth(h, 0, [0], [500], [n], q, modes, windows, 0, scale if scale > 0 else None)
            assert (np.abs(lse.double().cpu().numpy() - ref_lse) <= off + 2.0 ** -22 * np.abs(ref_lse)).all()
            # weights are off by the scores' error, rows by that much of the largest value
            row = 4 * off.max(1)[:, None, None] * np.abs(ref).max() + 2.0 ** -8 * np.abs(ref) + 2e-2
            assert (np.abs(out.double().cpu().numpy() - ref) <= row).all()


@pytest.mark.parametrize("lay", [LAYOUTS[0], LAYOUTS[2]])
def test_values_out_of_sight_do_not_matter(lay):
    """Infinities and NaN in K and V of 16 bits: rows that do not see them are as if they were not there."""
    rng = np.random.default_rng(7)
    h = holder(lay)
    n, new = 330, 150
    k, v = (wl.bf16_bits(rng.standard_normal((n, h.Hkv, h.d), dtype=np.float32)) for _ in range(2))
    bits = rng.choice([2, 8, 16], n)
    odd = [10, 220, 260]
    bits[odd] = 16
    clean = [x.copy() for x in (k, v)]
    k[odd[1], 0, 3], v[odd[0], :, 5], v[odd[2], 0, :] = 0x7F80, 0x7FC0, 0xFF80
    h.append(rng, 0, 0, np.arange(n), k=clean[0], v=clean[1], bits=bits, p_skip=0.0)
    h.append(rng, 0, 1, np.arange(n), k=k, v=v, bits=bits, p_skip=0.0)
    modes, windows = rng.choice(3, new, p=[.1, .6, .3]), rng.integers(1, 100, new)
    q_bits = wl.bf16_bits(rng.standard_normal((new, h.Hq, h.d), dtype=np.float32))
    start = n - new
    a = call(h, rng, [0], [start], [new], modes, windows, 4, q_bits=q_bits)[0].double().cpu().numpy()
    b = call(h, rng, [1], [start], [new], modes, windows, 4, q_bits=q_bits)[0].double().cpu().numpy()
    t = start + np.arange(new)
    sees = np.zeros(new, bool)
    for p in odd:
        sees |= (p <= t) & ((modes == 2) | ((modes == 1) & (p > t - windows)))
    assert (~sees).sum() > 20 and sees.sum() > 20
    assert np.isfinite(b[~sees]).all()
    check_attention(b[~sees], truth(h, 0, [0], [start], [new], q_bits, modes.astype(np.uint8), windows, 4)[0][~sees])
    full = (modes == 2) & sees
    assert np.isnan(b[full][:, :, 5]).all()  # NaN in V at position 10, in every KV head
    heads = h.Hq // h.Hkv
    local = (modes == 1) & (260 <= t) & (260 > t - windows) & ~((220 > t - windows) & (220 <= t))
    assert not np.isfinite(b[local][:, :heads]).any() and np.isfinite(b[local][:, heads:]).all()


def test_queries_not_finite_stay_in_their_rows():
    rng = np.random.default_rng(8)
    h = holder(LAYOUTS[2])
    fill(h, rng, 0, 0, 300)
    n = 100
    q_bits = wl.bf16_bits(rng.standard_normal((n, h.Hq, h.d), dtype=np.float32))
    want = call(h, rng, [0], [200], [n], [2] * n, [1] * n, q_bits=q_bits)[0]
    dirty = q_bits.copy()
    dirty[7, 3, 0], dirty[50, 0, 9] = 0x7FC0, 0x7F80
    got = call(h, rng, [0], [200], [n], [2] * n, [1] * n, q_bits=dirty)[0]
    same = torch.ones(n, h.Hq, dtype=torch.bool)
    same[7, 3] = same[50, 0] = False
    assert torch.equal(got.cpu()[same], want.cpu()[same]) and torch.isnan(got[7, 3]).all()


def test_rows_outside_every_chunk_stay():
    rng = np.random.default_rng(9)
    h = holder(LAYOUTS[1])
    fill(h, rng, 0, 0, 100)
    q = dev(wl.bf16_bits(rng.standard_normal((90, h.Hq, h.d), dtype=np.float32)), torch.bfloat16)
    out = torch.full((90, h.Hq, h.d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((90, h.Hq), 7.0, device="cuda")
    modes = torch.full((90,), 2, dtype=torch.uint8, device="cuda")
    h.gpu.chunk_attn(0, h.ints([0, 0]), h.ints([30, 60]), h.ints([11, 41, 80]), q, modes, out=out, lse=lse)
    assert h.gpu.status() == 0
    for t in (out, lse):
        assert (t[:11] == 7).all() and (t[80:] == 7).all() and not (t[11:80] == 7).any()


def test_errors_on_the_device():
    rng = np.random.default_rng(10)
    h = holder(LAYOUTS[0], S=3, maxctx=300)
    for s in range(3):
        fill(h, rng, 0, s, 200)
    seqs, starts, lens = [0, 9, 1, 2], [150, 0, 290, 150], [50, 10, 20, 50]
    n = sum(lens)
    modes, windows = np.full(n, 2), np.full(n, 5)
    modes[3], modes[90], modes[91] = 3, 1, 7
    windows[90] = 0
    bad = np.zeros(n, bool)
    bad[[3, 90, 91]] = True
    bad[50:80] = True
    out, lse, q_bits, m, w = call(h, rng, seqs, starts, lens, modes, windows, expect=1)
    assert h.gpu.status() == 0
    assert (out[torch.from_numpy(bad)] == 0).all() and torch.isneginf(lse[torch.from_numpy(bad)]).all()
    ref = truth(h, 0, [0, 2], [150, 150], [50, 50], np.delete(q_bits, np.s_[50:80], 0), np.delete(np.where(m > 2, 0, m), np.s_[50:80]),
                np.delete(w, np.s_[50:80]), 0)[0]
    keep = np.delete(~bad, np.s_[50:80])
    check_attention(np.delete(out.double().cpu().numpy(), np.s_[50:80], 0)[keep], ref[keep])
    call(h, rng, [1], [290], [20], [2] * 20, [1] * 20, expect=4)
    call(h, rng, [1], [-1], [20], [2] * 20, [1] * 20, expect=4)
    q = dev(q_bits, torch.bfloat16)
    for offsets in ([0, 40, 30], [-1, 5, 9], [0, 5, 400]):
        out = h.gpu.chunk_attn(0, h.ints([0, 1]), h.ints([0, 0]), h.ints(offsets), q, dev(np.full(n, 2, np.uint8), torch.uint8))
        assert h.gpu.status() == 1 and (out == 0).all()


def test_a_workspace_too_small_for_what_is_stored():
    rng = np.random.default_rng(11)
    h = holder(LAYOUTS[0])
    fill(h, rng, 0, 0, 900, p_skip=0.0)
    out, lse, *_ = call(h, rng, [0], [800], [100], [2] * 100, [1] * 100, expect=2, max_keys=200)
    assert (out == 0).all() and torch.isneginf(lse).all()
    check(h, rng, [0], [800], [100], [1] * 100, [90] * 100, max_keys=200)  # windows reach over 189 positions
    with pytest.raises(trr.TrrError):
        call(h, rng, [0], [800], [100], [2] * 100, [1] * 100, workspace=torch.empty(4096, dtype=torch.uint8, device="cuda"))


def near(a, b):
    """Two results that are each within ROW_RTOL of a row's largest value of the truth (what check_attention asks)
    are within twice that of one another: both are bf16, and two neighbours of one truth are 2^-7 = 7.8e-3 apart
    where each is half a step, 3.9e-3, off."""
    a, b = (x.double().cpu().numpy() for x in (a, b))
    most = np.abs(b).max(-1)
    assert (np.abs(a - b).max(-1) <= 2 * ROW_RTOL * most).all()


def test_the_same_rows_as_decode_attention():
    """Chunks against the same queries one by one, and prefixes of a chunk against the whole."""
    rng = np.random.default_rng(12)
    h = holder(LAYOUTS[2], S=2)
    fill(h, rng, 0, 1, 500)
    n = 140
    modes, windows = rng.choice(3, n).astype(np.uint8), np.full(n, 60, np.int32)
    out, _, q_bits, *_ = call(h, rng, [1], [360], [n], modes, windows, 3)
    one = h.gpu.decode_attn_sinks(0, h.ints([1] * n), h.ints(np.arange(360, 500)), dev(q_bits, torch.bfloat16), dev(modes, torch.uint8), 3,
                                  window_scalar=60)
    near(out, one)
    few = call(h, rng, [1], [360], [30], modes[:30], windows[:30], 3, q_bits=q_bits[:30])[0]
    near(few, out[:30])


def test_streams_graphs_and_repeats():
    """Bit for bit the same: again, on another stream, captured and replayed over other rows."""
    rng = np.random.default_rng(13)
    h = holder(LAYOUTS[0], S=4)
    for s in range(4):
        fill(h, rng, 0, s, 600 + 37 * s)
    seqs, starts, lens = [0, 1, 2, 3], [500, 600, 0, 710], [100, 37, 674, 1]
    n = sum(lens)
    modes, windows = rng.choice(3, n).astype(np.uint8), rng.integers(1, 400, n)
    want, want_lse, q_bits, m, w = call(h, rng, seqs, starts, lens, modes, windows, 4)
    args = (0, h.ints(seqs), h.ints(starts), h.ints(np.append(0, np.cumsum(lens))), dev(q_bits, torch.bfloat16), dev(m, torch.uint8))
    kw = dict(windows=dev(w, torch.int32), sinks=4)
    for _ in range(3):
        assert torch.equal(h.gpu.chunk_attn(*args, **kw), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = h.gpu.chunk_attn(*args, stream=side, **kw)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    q = args[4].clone()
    workspace = h.gpu.chunk_workspace(4, n)
    out, lse = torch.empty_like(want), torch.empty_like(want_lse)
    graphs = []
    for _ in range(2):  # two graphs that share the workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            h.gpu.chunk_attn(*args[:4], q, args[5], out=out, lse=lse, workspace=workspace, **kw)
        graphs.append(graph)
    for graph in graphs * 2:
        q.copy_(torch.randn(q.shape, device="cuda"))
        graph.replay()
        assert not torch.equal(out, want)
        q.copy_(args[4])
        graph.replay()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert h.gpu.status() == 0


def test_prompt_by_chunks_then_decode_then_read():
    """A prompt appended and attended chunk by chunk, a decode step on it, and all of it read back."""
    rng = np.random.default_rng(14)
    h = holder(LAYOUTS[3], S=2, L=2, maxctx=600)
    at = 0
    for new in (200, 1, 130, 77):
        for layer in range(2):
            h.append(rng, layer, 1, np.arange(at, at + new))
            check(h, rng, [1], [at], [new], rng.choice(3, new), rng.integers(1, 300, new), 2, layer=layer)
        at += new
    for layer in range(2):
        h.append(rng, layer, 1, [at], p_skip=0.0)
        q = wl.bf16_bits(rng.standard_normal((1, h.Hq, h.d), dtype=np.float32))
        got = h.gpu.decode_attn(layer, h.ints([1]), h.ints([at]), dev(q, torch.bfloat16), dev(np.array([2], np.uint8), torch.uint8))
        check_attention(got.double().cpu().numpy(), h.attend(layer, [1], [at], q, [2], [1]))
        k, v, bits = h.gpu.read(layer, h.ints([1]), h.ints([0]), h.ints([0, at + 1]), at + 1, dtype=torch.float32)
        pos, kk, vv = h.values(layer, 1, 1)
        assert np.array_equal(np.nonzero(bits[:, 1].cpu().numpy())[0], pos)
        assert np.array_equal(k[:, 1].cpu().numpy()[pos], kk.astype(np.float32)) and np.array_equal(v[:, 1].cpu().numpy()[pos], vv.astype(np.float32))


def test_many_chunks_and_forked_sequences():
    rng = np.random.default_rng(15)
    lay = LAYOUTS[1]
    h = holder(lay, S=130, maxctx=400, caps=900, archive=140)
    fill(h, rng, 0, 0, 210)
    kids = list(range(1, 129))
    h.fork([0] * 128, kids, [int(x) for x in rng.integers(0, 211, 128)])
    lens = rng.integers(0, 6, 128).tolist()
    starts = []
    for s, n in zip(kids, lens):
        last = int(h.gpu.region("last_pos").view(torch.int32)[s].item())
        h.append(rng, 0, s, np.arange(last + 1, last + 1 + n))
        starts.append(last + 1)
    n = sum(lens)
    check(h, rng, kids, starts, lens, rng.choice(3, n), rng.integers(1, 250, n), 1)


def test_refusals():
    h = holder(LAYOUTS[0])
    q = torch.zeros(8, 4, 64, dtype=torch.bfloat16, device="cuda")
    modes = torch.zeros(8, dtype=torch.uint8, device="cuda")
    ids, starts, offsets = h.ints([0]), h.ints([0]), h.ints([0, 8])
    for bad in (dict(starts=h.ints([0, 1])), dict(offsets=h.ints([0, 4, 8])), dict(q=q[:7]), dict(q=q.float()), dict(modes=modes.int()),
                dict(windows=h.ints([1])), dict(out=q[:5]), dict(lse=torch.zeros(8, device="cuda")), dict(q=q.transpose(0, 1).contiguous().transpose(0, 1))):
        kw = dict(seq_ids=ids, starts=starts, offsets=offsets, q=q, modes=modes, window_scalar=5)
        kw.update(bad)
        with pytest.raises(ValueError):
            h.gpu.chunk_attn(0, **kw)
    for kw in (dict(sinks=-1), dict(layer=1), dict(layer=-1)):
        with pytest.raises(trr.TrrError):
            h.gpu.chunk_attn(kw.pop("layer", 0), ids, starts, offsets, q, modes, window_scalar=5, **kw)
    out = h.gpu.chunk_attn(0, h.ints([]), h.ints([]), h.ints([0]), q[:0], modes[:0])
    assert out.shape == (0, 4, 64) and h.gpu.status() == 0
    heads = Holder(1, 2, 4, 4, 64, 32, 16, 256, [64] * 4, head_modes=1)
    with pytest.raises(trr.TrrError):
        heads.gpu.chunk_attn(0, ids, starts, offsets, q, modes, workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
