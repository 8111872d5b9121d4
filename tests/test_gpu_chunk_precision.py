"""How near rows and logarithms of attention of chunks come to the definition.

Scores here are exact: K has one channel that is not zero, q is 1 there, both are numbers that binary16 holds, so that
only weights, V and sums are rounded.  Then an element of a row is off by
  2^-8 of itself: half a step of bf16;
  2^-11 sum w |v|: half a step of binary16 of each weight; V of 16 bits is exact unless it lies below 2^-14;
  2^-33 w_top sum |v|, w_top the row's largest weight: half of binary16's smallest step, 2^-25, where a weight lies below
  2^-14 of a reference that stands at 2^-8 of some weight of the row;
  2^-12 sum w |v|: binary32 sums and exponentials."""
import numpy as np
import pytest
import torch

from _parity import dev
from _shared import Holder
from paper_2607_06601_gb300 import workloads as wl
from test_gpu_chunk import call

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


WIDE = [dict(Hq=4, Hkv=4, d=64, G=32, P=16), dict(Hq=8, Hkv=2, d=128, G=64, P=32)]


def one_channel(n, heads, d, size):
    """[n][heads][d] rows, `size` in channel 0 and zeros, as bf16 bits."""
    x = np.zeros((n, heads, d), np.float32)
    x[:, :, 0] = np.asarray(size, np.float32).reshape(-1, 1)
    bits = wl.bf16_bits(x)
    assert np.array_equal(wl.bf16_to_f32(bits), x)
    return bits


def exact_rows(h, scores, v, starts_at, new):
    """Rows of full queries at positions starts_at .. over scores[n] (the same for all queries and heads) and v [n][Hkv][d];
    what the weights add up |v| to, and w_top sum |v|."""
    x, w = np.repeat(v, h.Hq // h.Hkv, axis=1), np.exp(scores - scores.max())
    rows, total = np.s_[starts_at:starts_at + new], w.cumsum()
    over = lambda y: y.cumsum(0)[rows] / total[rows, None, None]  # noqa: E731
    top = np.maximum.accumulate(w)[rows] / total[rows]
    return over(w[:, None, None] * x), over(w[:, None, None] * np.abs(x)), top[:, None, None] * np.abs(x).cumsum(0)[rows]


def within(got, ref, spread, most, extra=0.0):
    off = np.abs(got.double().cpu().numpy() - ref)
    bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -12) * spread + 2.0 ** -33 * most + extra
    assert (off <= bound).all(), f"{(off / np.maximum(bound, 1e-300)).max():.2f} times the bound"


@pytest.mark.parametrize("top", [8, 12, 15, 17, 18, 20])
@pytest.mark.parametrize("lay,n,new", [(WIDE[0], 250, 20), (WIDE[0], 270, 200), (WIDE[1], 230, 10), (WIDE[1], 220, 150),
                                       (dict(Hq=32, Hkv=8, d=64, G=64, P=32), 3000, 1000)])
def test_weights_far_below_a_first_token_that_adds_nothing(lay, n, new, top):
    """A first token that draws most of each row's weight and has V = 0, `top` nats above all others: the rows are what the
    others' weights leave of them, in one run and over long ones."""
    rng = np.random.default_rng([1, n, top])
    h = Holder(1, 1, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], n, [n // lay["P"] + 2] * 4, archive=4)
    scores = np.zeros(n)
    scores[0] = top
    v_bits = wl.bf16_bits((1.0 + 0.5 * rng.standard_normal((n, h.Hkv, h.d))).astype(np.float32))
    v_bits[0] = 0
    k_bits = one_channel(n, h.Hkv, h.d, scores)
    for at in range(0, n, 1000):
        part = slice(at, min(n, at + 1000))
        h.append(rng, 0, 0, np.arange(n)[part], k=k_bits[part], v=v_bits[part], bits=np.full(n, 16)[part], p_skip=0.0)
    q_bits = one_channel(new, h.Hq, h.d, np.ones(new))
    out, lse, *_ = call(h, rng, [0], [n - new], [new], [2] * new, [1] * new, scale=1.0, q_bits=q_bits)
    ref, spread, most = exact_rows(h, scores, wl.bf16_to_f32(v_bits).astype(np.float64), n - new, new)
    within(out, ref, spread, most)
    total = np.log(np.exp(scores - top).cumsum())[n - new:, None] + top
    assert (np.abs(lse.double().cpu().numpy() - total) <= 2.0 ** -16).all()


@pytest.mark.parametrize("top", [12, 17, 20, 60])
@pytest.mark.parametrize("lay,n,new,at,window,sinks", [
    (WIDE[0], 700, 20, [350], 0, 0), (WIDE[0], 700, 200, [1, 349, 520], 0, 0), (WIDE[1], 500, 150, [0, 260], 0, 0), (WIDE[0], 700, 150, [0], 150, 1),
    (WIDE[1], 600, 20, [0], 170, 1), (dict(Hq=16, Hkv=4, d=128, G=64, P=64), 4000, 1000, [0, 2000], 0, 0)])
def test_tokens_that_add_nothing_anywhere(lay, n, new, at, window, sinks, top):
    """The same with such tokens within runs, with two of them, and with one that is kept in sight before a window."""
    rng = np.random.default_rng([2, n, new, top])
    h = Holder(1, 1, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], n, [n // lay["P"] + 2] * 4, archive=5)
    scores = np.zeros(n)
    scores[at] = top
    v_bits = wl.bf16_bits((1.0 + 0.5 * rng.standard_normal((n, h.Hkv, h.d))).astype(np.float32))
    v_bits[at] = 0
    k_bits = one_channel(n, h.Hkv, h.d, scores)
    for a in range(0, n, 1000):
        part = slice(a, min(n, a + 1000))
        h.append(rng, 0, 0, np.arange(n)[part], k=k_bits[part], v=v_bits[part], bits=np.full(n, 16)[part], p_skip=0.0)
    q_bits = one_channel(new, h.Hq, h.d, np.ones(new))
    out, lse, *_ = call(h, rng, [0], [n - new], [new], [1 if window else 2] * new, [max(1, window)] * new, sinks, scale=1.0, q_bits=q_bits)
    v, w = wl.bf16_to_f32(v_bits).astype(np.float64), np.exp(scores - top)
    t, pos = np.arange(n - new, n)[:, None], np.arange(n)
    w = np.where((pos <= t) & ((window == 0) | (pos > t - window) | (pos < sinks)), w, 0.0)
    total = w.sum(1)
    over = lambda y: np.repeat(np.einsum("qt,thd->qhd", w / total[:, None], y, optimize=True), h.Hq // h.Hkv, axis=1)  # noqa: E731
    # weights below 2^-14 of a reference: 2^-33 of the row's largest, or 2^-11 of the mean weight of its tile's other tokens,
    # all of which weigh alike here, so that the bound on weights holds that too
    seen = np.repeat(np.einsum("qt,thd->qhd", (w > 0).astype(float), np.abs(v), optimize=True), h.Hq // h.Hkv, axis=1)
    within(out, over(v), over(np.abs(v)), (w.max(1) / total)[:, None, None] * seen)
    assert (np.abs(lse.double().cpu().numpy() - (np.log(total) + top)[:, None]) <= 2.0 ** -16 + 2.0 ** -22 * top).all()


@pytest.mark.parametrize("shape", ["up", "down", "up and down", "two steps"])
@pytest.mark.parametrize("lay,new", [(WIDE[0], 20), (WIDE[0], 200), (WIDE[1], 20), (WIDE[1], 150)])
def test_references_that_move_with_every_tile(lay, new, shape):
    """Scores in steps of 24 every 40 tokens: each tile's weights are taken twice.  Bit for bit the same over calls, with the
    tiles in memory and not."""
    rng = np.random.default_rng([3, new])
    n = 400
    h = Holder(1, 1, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], n, [n // lay["P"] + 2] * 4, archive=2)
    stair = np.arange(n) // 40
    scores = 24.0 * {"up": stair, "down": 9 - stair, "up and down": np.minimum(stair, 9 - stair), "two steps": 4 * (stair % 2)}[shape]
    v_bits = wl.bf16_bits(rng.standard_normal((n, h.Hkv, h.d), dtype=np.float32))
    h.append(rng, 0, 0, np.arange(n), k=one_channel(n, h.Hkv, h.d, scores), v=v_bits, bits=np.full(n, 16), p_skip=0.0)
    q_bits = one_channel(new, h.Hq, h.d, np.ones(new))
    out, lse, *_ = call(h, rng, [0], [n - new], [new], [2] * new, [1] * new, scale=1.0, q_bits=q_bits)
    ref, spread, most = exact_rows(h, scores, wl.bf16_to_f32(v_bits).astype(np.float64), n - new, new)
    within(out, ref, spread, most)
    cold = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")  # twice L2
    for i in range(6):
        if i % 2:
            cold.fill_(i)
        again = call(h, rng, [0], [n - new], [new], [2] * new, [1] * new, scale=1.0, q_bits=q_bits)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("size", [-14, -20, -27])
@pytest.mark.parametrize("lay", WIDE)
def test_small_elements_of_queries_before_large_keys(lay, size):
    """Query rows with one element of 1 and others far below it, over keys that are 0 at the one and large at the others: scores
    as near as sum |scale q k| lets them be (half a step of binary16: 2^-11 of it).  A token in sight each, so that the
    logarithm is the score; 2^-16 stands for exponentials and sums."""
    rng = np.random.default_rng([4, -size])
    n = 160
    h = Holder(1, 1, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], n, [n // lay["P"] + 2] * 4, archive=2)
    k, q = rng.standard_normal((n, h.Hkv, h.d)) * 2.0 ** 12, rng.standard_normal((n, h.Hq, h.d)) * 2.0 ** size
    k[:, :, 5], q[:, :, 5] = 0.0, 1.0
    k_bits, q_bits = wl.bf16_bits(k.astype(np.float32)), wl.bf16_bits(q.astype(np.float32))
    h.append(rng, 0, 0, np.arange(n), k=k_bits, bits=np.full(n, 16), p_skip=0.0)
    scale = 2.0 ** (-8 - size)
    _, lse, *_ = call(h, rng, [0], [0], [n], [1] * n, [1] * n, scale=scale, q_bits=q_bits)
    q, k = (wl.bf16_to_f32(x).astype(np.float64) for x in (q_bits, k_bits))
    k = np.repeat(k, h.Hq // h.Hkv, axis=1)
    off = np.abs(lse.double().cpu().numpy() - scale * (q * k).sum(-1))
    assert (off <= 2.0 ** -11 * scale * np.abs(q * k).sum(-1) + 2.0 ** -16).all()


@pytest.mark.parametrize("lay,n,new", [(WIDE[0], 300, 20), (WIDE[0], 300, 160), (WIDE[1], 260, 100), (dict(Hq=4, Hkv=2, d=64, G=32, P=16), 3000, 30),
                                       (dict(Hq=2, Hkv=2, d=128, G=64, P=16), 2500, 40)])
def test_channels_far_apart(lay, n, new):
    """V of 16 bits whose channels are 2^0 to 2^-70 in size, one of them zeros: each channel as near as its own values are.  (Binary16's steps are 2^-16 of what a channel's samples are scaled to, 2^-8: less than the 2^-12 of sums.)"""
    rng = np.random.default_rng([5, n, new])
    h = Holder(1, 1, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], n, [n // lay["P"] + 2] * 4, archive=4)
    v = rng.standard_normal((n, h.Hkv, h.d)) * 2.0 ** (-7.0 * (np.arange(h.d) % 11))
    v[:, 0, 20] = 0.0
    v_bits = wl.bf16_bits(v.astype(np.float32))
    scores = rng.integers(-8, 8, n) / 4.0
    k_bits = one_channel(n, h.Hkv, h.d, scores)
    for at in range(0, n, 1000):
        part = slice(at, min(n, at + 1000))
        h.append(rng, 0, 0, np.arange(n)[part], k=k_bits[part], v=v_bits[part], bits=np.full(n, 16)[part], p_skip=0.0)
    out, *_ = call(h, rng, [0], [n - new], [new], [2] * new, [1] * new, scale=1.0, q_bits=one_channel(new, h.Hq, h.d, np.ones(new)))
    ref, spread, _ = exact_rows(h, scores, wl.bf16_to_f32(v_bits).astype(np.float64), n - new, new)
    within(out, ref, spread, 0.0)


def test_channels_that_are_small_but_for_one_token():
    """Scaled by what the others need, one value is more than binary16 holds; and beside it tokens of fewer bits."""
    rng = np.random.default_rng(6)
    lay, n, new = WIDE[0], 400, 140
    h = Holder(1, 2, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], n, [2 * n // lay["P"] + 2] * 4, archive=4)
    scores = rng.integers(-16, 1, n) / 4.0  # (their groups' least value, which is stored as it is)
    for seq, bits in ((0, np.full(n, 16)), (1, rng.choice([8, 16], n))):
        v = rng.standard_normal((n, h.Hkv, h.d)) * 2.0 ** -20
        if seq == 0:
            v[37, 1, 3], v[200, 3, 60] = 3000.0, -5.0
        h.append(rng, 0, seq, np.arange(n), k=one_channel(n, h.Hkv, h.d, scores), v=wl.bf16_bits(v.astype(np.float32)), bits=bits, p_skip=0.0)
    for seq in (0, 1):
        out, *_ = call(h, rng, [seq], [n - new], [new], [2] * new, [1] * new, scale=1.0, q_bits=one_channel(new, h.Hq, h.d, np.ones(new)))
        v = np.stack([h.values(0, seq, head)[2] for head in range(h.Hkv)], 1)
        k = np.stack([h.values(0, seq, head)[1][:, 0] for head in range(h.Hkv)], 1)
        assert np.array_equal(k, np.repeat(scores[:, None], h.Hkv, 1))
        ref, spread, most = exact_rows(h, scores, v, n - new, new)
        within(out, ref, spread, most)
