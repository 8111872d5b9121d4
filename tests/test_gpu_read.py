"""Stretches of a cache read back (trr_kv_read) against the CPU oracle's values.

z + c*s is exact in 64 bits, so the one rounding to binary32 is known: the float32 rows have to be
equal to it, and the bf16 rows to that value rounded once more."""
import numpy as np
import pytest
import torch

from _parity import dev
from _shared import Holder
from paper_2607_06601_gb300 import trr, workloads as wl

pytestmark = pytest.mark.gpu

LAYOUTS = [dict(Hq=4, Hkv=4, d=64, G=32, P=16), dict(Hq=12, Hkv=4, d=64, G=64, P=32), dict(Hq=8, Hkv=2, d=128, G=64, P=16),
           dict(Hq=6, Hkv=6, d=64, G=32, P=64), dict(Hq=3, Hkv=1, d=128, G=128, P=32), dict(Hq=5, Hkv=5, d=128, G=32, P=64)]


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def holder(lay, S=3, maxctx=512, caps=200, L=1, **kw):
    return Holder(L, S, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], maxctx, [caps] * 4, **kw)


def truth(h, layer, seqs, starts, lens):
    """Rows in 64 bits and widths."""
    k, v, bits = np.zeros((sum(lens), h.Hkv, h.d)), np.zeros((sum(lens), h.Hkv, h.d)), np.zeros((sum(lens), h.Hkv), np.uint8)
    row = 0
    for s, start, n in zip(seqs, starts, lens):
        for i in range(n):
            at = h.tokens[layer][s].get(start + i)
            for head in range(h.Hkv) if at else ():
                c, kk, vv = h.orc.dequant_token(layer, at[0], at[1], head)
                if c >= 0:
                    k[row + i, head], v[row + i, head], bits[row + i, head] = kk, vv, (2, 4, 8, 16)[c]
        row += n
    return k, v, bits


def check(h, layer, seqs, starts, lens, expect=0):
    offsets = np.append(0, np.cumsum(lens))
    args = (layer, h.ints(seqs), h.ints(starts), h.ints(offsets), int(offsets[-1]))
    want = truth(h, layer, seqs, starts, lens)
    for dtype in (torch.float32, torch.bfloat16):
        k, v, bits = h.gpu.read(*args, dtype=dtype)
        assert h.gpu.status() == expect
        assert np.array_equal(bits.cpu().numpy(), want[2])
        for got, ref in ((k, want[0]), (v, want[1])):
            ref = ref.astype(np.float32)
            if dtype == torch.bfloat16:
                ref = wl.bf16_to_f32(wl.bf16_bits(ref))
            assert got.dtype == dtype and np.array_equal(got.float().cpu().numpy(), ref)
    return want


@pytest.mark.parametrize("lay", LAYOUTS)
@pytest.mark.parametrize("n", [1, 17, 64, 301])
def test_whole_sequence(lay, n):
    rng = np.random.default_rng([1, n])
    h = holder(lay)
    h.append(rng, 0, 1, np.arange(n))
    check(h, 0, [1], [0], [n])


@pytest.mark.parametrize("bits", [2, 4, 8, 16])
@pytest.mark.parametrize("lay", LAYOUTS[:3])
def test_one_width(lay, bits):
    rng = np.random.default_rng([2, bits])
    h = holder(lay)
    h.append(rng, 0, 0, np.arange(5, 150), bits=np.full(145, bits), p_skip=0.0)
    check(h, 0, [0, 0], [0, 149], [200, 1])


def test_stretches_of_every_kind():
    """Ragged, empty, overlapping, repeated, past the last token, in the second layer; sequences that
    hold nothing; empty stretches whose ids and starts mean nothing."""
    rng = np.random.default_rng(3)
    h = holder(LAYOUTS[3], S=6, L=2, maxctx=700)
    for s, n in ((0, 300), (2, 1), (3, 700)):
        h.append(rng, 1, s, np.arange(n))
    h.append(rng, 0, 0, np.arange(40))
    seqs, starts, lens = [0, 1, 3, 77, 3, 2, 0, 3, -5], [280, 0, 650, -9, 600, 0, 0, 0, 3], [60, 33, 50, 0, 64, 5, 1, 129, 0]
    check(h, 1, seqs, starts, lens)
    check(h, 0, [0, 3], [3, 0], [100, 10])


def test_gaps_forks_and_evictions():
    rng = np.random.default_rng(4)
    h = holder(LAYOUTS[0], S=4, caps=120)
    h.append(rng, 0, 0, np.sort(rng.choice(400, 180, replace=False)))
    h.fork([0], [2], [215])
    h.append(rng, 0, 2, np.arange(230, 300))
    check(h, 0, [2, 0], [0, 100], [310, 300])
    before = truth(h, 0, [2], [0], [310])
    h.gpu.evict(h.ints([2]), h.ints([180]), 3)
    h.gpu.compact()
    k, v, bits = h.gpu.read(0, h.ints([2]), h.ints([0]), h.ints([0, 310]), 310, dtype=torch.float32)
    bits = bits.cpu().numpy()
    assert (bits[180:] == before[2][180:]).all() and (bits[:3] == before[2][:3]).all() and (bits[3:180] != before[2][3:180]).any()
    kept = bits > 0
    assert np.array_equal(k.cpu().numpy()[kept], before[0].astype(np.float32)[kept])
    assert (k.cpu().numpy()[~kept] == 0).all() and (v.cpu().numpy()[~kept] == 0).all()


def test_per_head_modes():
    rng = np.random.default_rng(5)
    h = holder(LAYOUTS[3], head_modes=1)
    h.append(rng, 0, 1, np.arange(200), p_skip=0.5)
    want = check(h, 0, [1], [0], [210])
    assert (want[2] > 0).any(1).sum() > (want[2] > 0).all(1).sum()


def test_many_stretches_of_one_position():
    rng = np.random.default_rng(6)
    h = holder(LAYOUTS[2], S=2, maxctx=3000, caps=400)
    for at in range(0, 3000, 1000):
        h.append(rng, 0, 1, np.arange(at, at + 1000))
    starts = rng.integers(0, 3000, 900).tolist()
    check(h, 0, [1] * 900, starts, [1] * 900)


@pytest.mark.parametrize("lay", LAYOUTS[1:4:2])
def test_many_rows(lay):
    """As many rows as make units of 48 to 64 positions and one, two and more of them a CTA; the same rows all along."""
    rng = np.random.default_rng(8)
    h = holder(lay, S=1)
    h.append(rng, 0, 0, np.arange(131), p_skip=0.2)
    want = truth(h, 0, [0], [0], [131])
    for times in (220, 250, 280, 297, 430, 600):
        n = 131 * times
        k, v, bits = h.gpu.read(0, h.ints([0] * times), h.ints([0] * times), h.ints(np.arange(times + 1) * 131), n, dtype=torch.float32)
        assert h.gpu.status() == 0
        for got, ref in ((k, want[0]), (v, want[1]), (bits, want[2])):
            ref = torch.from_numpy(ref.astype(np.uint8 if got is bits else np.float32)).cuda()
            assert torch.equal(got.view(times, 131, *got.shape[1:]), ref.expand(times, *ref.shape))


def test_values_far_apart_and_not_finite():
    """Scales from binary16's smallest to its largest; 16-bit rows that hold infinities and NaN."""
    rng = np.random.default_rng(7)
    h = holder(LAYOUTS[1])
    n = 128
    k = rng.standard_normal((n, 4, 64)).astype(np.float32) * (2.0 ** rng.integers(-24, 16, (n, 4, 1)))
    k = np.clip(k, -65000, 65000).astype(np.float32)
    k[3, 0, :32], k[3, 0, 5] = -65000.0, 65000.0
    h.append(rng, 0, 0, np.arange(n), k=wl.bf16_bits(k), p_skip=0.0)
    check(h, 0, [0], [0], [n])
    x = wl.bf16_bits(rng.standard_normal((4, 4, 64), dtype=np.float32))
    x[0, 0, :3] = [0x7F80, 0xFF80, 0x7FC1]
    h.append(rng, 0, 1, np.arange(4), k=x, v=x, bits=[16] * 4, p_skip=0.0)
    got, _, _ = h.gpu.read(0, h.ints([1]), h.ints([0]), h.ints([0, 4]), 4)
    assert np.array_equal(got.view(torch.int16).cpu().numpy().view(np.uint16)[1:], x[1:])
    row = got[0, 0, :3].float().cpu().numpy()
    assert np.isposinf(row[0]) and np.isneginf(row[1]) and np.isnan(row[2])


def test_strided_outputs_and_rows_outside_every_stretch():
    """K and V into one tensor of pairs; rows before the first and behind the last stretch stay."""
    rng = np.random.default_rng(8)
    h = holder(LAYOUTS[0])
    h.append(rng, 0, 1, np.arange(100))
    both = torch.full((130, 2, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    bits = torch.full((130, 4), 9, dtype=torch.uint8, device="cuda")
    h.gpu.read(0, h.ints([1]), h.ints([10]), h.ints([20, 110]), 130, k=both[:, 0], v=both[:, 1], bits=bits)
    assert h.gpu.status() == 0
    want = truth(h, 0, [1], [10], [90])
    for i in range(2):
        assert np.array_equal(both[20:110, i].float().cpu().numpy(), wl.bf16_to_f32(wl.bf16_bits(want[i].astype(np.float32))))
    assert np.array_equal(bits[20:110].cpu().numpy(), want[2])
    assert (both[:20] == 7).all() and (both[110:] == 7).all() and (bits[:20] == 9).all() and (bits[110:] == 9).all()


def test_errors_on_the_device():
    rng = np.random.default_rng(9)
    h = holder(LAYOUTS[0])
    h.append(rng, 0, 0, np.arange(100))
    h.append(rng, 0, 1, np.arange(100))
    args = (h.ints([0, 3, 1, 0]), h.ints([0, 0, 500, 0]), h.ints([0, 50, 100, 150, 200]))
    k, v, bits = h.gpu.read(0, *args, 200)
    assert h.gpu.status() == 1 and h.gpu.status() == 0  # the sequence that is not there, before the stretch past the end
    want = truth(h, 0, [0], [0], [50])[2]
    assert np.array_equal(bits[:50].cpu().numpy(), want) and np.array_equal(bits[150:].cpu().numpy(), want)
    assert (k[50:150] == 0).all() and (v[50:150] == 0).all() and (bits[50:150] == 0).all()
    h.gpu.read(0, h.ints([1]), h.ints([-1]), h.ints([0, 5]), 5)
    assert h.gpu.status() == 4
    for offsets in ([0, 40, 30], [-1, 5, 9], [0, 5, 201]):
        k, v, bits = h.gpu.read(0, h.ints([0, 1]), h.ints([0, 0]), h.ints(offsets), 200)
        assert h.gpu.status() == 1 and (k == 0).all() and (v == 0).all() and (bits == 0).all()


def test_another_stream_and_a_graph():
    rng = np.random.default_rng(10)
    h = holder(LAYOUTS[5])
    h.append(rng, 0, 0, np.arange(300))
    args = (0, h.ints([0]), h.ints([0]), h.ints([0, 300]), 300)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    k, v, bits = h.gpu.read(*args, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    want = [x.clone() for x in (k, v, bits)]
    assert np.array_equal(want[2].cpu().numpy(), truth(h, 0, [0], [0], [300])[2])
    graph = torch.cuda.CUDAGraph()
    for t in (k, v, bits):
        t.zero_()
    with torch.cuda.graph(graph):
        h.gpu.read(*args, k=k, v=v, bits=bits)
    for _ in range(3):
        graph.replay()
    assert h.gpu.status() == 0 and all(torch.equal(a, b) for a, b in zip((k, v, bits), want))


def test_refusals():
    h = holder(LAYOUTS[0])
    ids, starts, offsets = h.ints([0]), h.ints([0]), h.ints([0, 8])
    with pytest.raises(ValueError):
        h.gpu.read(0, ids, starts, h.ints([0]), 8)
    with pytest.raises(ValueError):
        h.gpu.read(0, ids, starts, offsets, 8, dtype=torch.float16)
    with pytest.raises(ValueError):
        h.gpu.read(0, ids, starts, offsets, 8, k=torch.empty(7, 4, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        h.gpu.read(0, ids, starts, offsets, 8, k=torch.empty(8, 64, 4, dtype=torch.bfloat16, device="cuda").transpose(1, 2))
    with pytest.raises(ValueError):
        h.gpu.read(0, ids, starts, offsets, 8, bits=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(trr.TrrError):
        h.gpu.read(1, ids, starts, offsets, 8)
    with pytest.raises(trr.TrrError):  # rows that do not start at 16 bytes
        h.gpu.read(0, ids, starts, offsets, 8, k=torch.empty(8 * 256 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(8, 4, 64))
    k, v, bits = h.gpu.read(0, h.ints([]), h.ints([]), h.ints([0]), 0)
    assert k.shape == (0, 4, 64) and h.gpu.status() == 0
