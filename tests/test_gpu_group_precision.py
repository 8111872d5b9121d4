"""How near the rows of attention over groups and sinks come to the definition.

On 16-bit pages K, V and q are what was appended, bit for bit, and only the kernels' own arithmetic
is left.  The bound there: half a unit in the last place of the bf16 output, and 2^-14 of sum_j w_j |v_j| for
everything before it.  A weight is off by at most 2^-17 (a sum of two bf16 numbers), 2^-21 (its
exponential) and 2^-16 (sums in binary32 of scores up to some 50 in size); numerator and
denominator both carry it: twice their sum, 2^-15 and a half, is below 2^-14.

Over long runs of quantised pages it is the size of all errors together that tells.  Rounding exact
rows to bf16 leaves a relative error of 1.7e-3 (root mean square); weights in binary16 add 2^-11 / sqrt 3
of a value's distance from its range's middle, 2.8e-4 of a row, K and V in binary16 (in groups) as
much again: squares add up to 1.73e-3 at most.  The bound: 1.1 times the rounding's own."""
import numpy as np
import pytest
import torch

from _parity import dev
from _shared import Holder
from paper_2607_06601_gb300 import workloads as wl
from test_gpu_group_attn import LAYOUTS, family, last_of

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def beyond(h, got, seqs, ts, q_bits, lows, sinks):
    """By how much the largest error passes the bound, in units of the bound, over all rows."""
    q, worst, kept = wl.bf16_to_f32(q_bits).astype(np.float64), 0.0, {}
    for i, (s, t, lo) in enumerate(zip(seqs, ts, lows)):
        for head in range(h.Hq):
            kvh = head // (h.Hq // h.Hkv)
            if (s, kvh) not in kept:
                kept[s, kvh] = h.values(0, s, kvh)
            pos, k, v = kept[s, kvh]
            see = (pos <= t) & ((pos >= lo) | (pos < sinks))
            x = k[see] @ q[i, head] / np.sqrt(h.d)
            w = np.exp(x - x.max())
            w /= w.sum()
            ref = w @ v[see]
            half_unit = np.exp2(np.floor(np.log2(np.abs(ref) + 1e-30)) - 8)
            worst = max(worst, (np.abs(got[i, head] - ref) / (half_unit + 2.0 ** -14 * (w @ np.abs(v[see])))).max())
    return worst


@pytest.mark.parametrize("loud", [1.0, 4.0])
@pytest.mark.parametrize("lay,members", [(LAYOUTS[0], 5), (LAYOUTS[0], 40), (LAYOUTS[0], 70), (LAYOUTS[2], 2), (LAYOUTS[2], 12), (LAYOUTS[2], 40),
                                         (LAYOUTS[5], 1), (LAYOUTS[5], 6)])
def test_weights_on_16_bit_pages(lay, members, loud):
    """Groups of one, two and four copies of their rows, segments of more than one tile: weights
    that a later tile raises over the first one's, rows that one token takes and rows spread wide."""
    rng = np.random.default_rng([1, members, int(loud)])
    h, kids = family(rng, lay, 1, members, 260, 20, mix=(0, 0, 0, 1), p_skip=0.0)
    ts = last_of(h, kids)
    q = wl.bf16_bits(loud * rng.standard_normal((members, h.Hq, h.d), dtype=np.float32))
    full = dev(np.full(members, 2, np.uint8), torch.uint8)
    got = h.gpu.decode_attn_shared(0, h.ints(kids), h.ints(ts), dev(q, torch.bfloat16), full, h.ints([0, members]))
    assert h.gpu.status() == 0
    assert beyond(h, got.double().cpu().numpy(), kids, ts, q, [-1] * members, 0) <= 1.0
    local = dev(np.full(members, 1, np.uint8), torch.uint8)
    got = h.gpu.decode_attn_sinks(0, h.ints(kids), h.ints(ts), dev(q, torch.bfloat16), local, 20, window_scalar=100)
    assert h.gpu.status() == 0
    assert beyond(h, got.double().cpu().numpy(), kids, ts, q, [t - 99 for t in ts], 20) <= 1.0


@pytest.mark.parametrize("bits", [2, 4, 8, 16])
@pytest.mark.parametrize("lay", [LAYOUTS[0], LAYOUTS[4]])
def test_errors_do_not_grow_with_a_run(lay, bits):
    """12,000 tokens of one width, and so many queries that a warp takes hundreds of blocks of one
    segment: what a run adds up loses nothing on the way."""
    rng = np.random.default_rng([2, bits])
    tokens, n = 12_000, 256 * 4 // lay["Hkv"]
    h = Holder(1, 1, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], tokens, [tokens // lay["P"] + 1] * 4, archive=14, max_queries=n)
    for at in range(0, tokens, 1000):
        h.append(rng, 0, 0, np.arange(at, at + 1000), bits=np.full(1000, bits), p_skip=0.0)
    q_bits = wl.bf16_bits(rng.standard_normal((n, h.Hq, h.d), dtype=np.float32))
    q, heads = wl.bf16_to_f32(q_bits).astype(np.float64), h.Hq // h.Hkv
    ref = np.zeros(q.shape)
    for kvh in range(h.Hkv):
        _, k, v = h.values(0, 0, kvh)
        mine = slice(kvh * heads, (kvh + 1) * heads)
        x = np.einsum("qhd,kd->qhk", q[:, mine], k, optimize=True) / np.sqrt(h.d)
        p = np.exp(x - x.max(-1, keepdims=True))
        ref[:, mine] = p @ v / p.sum(-1, keepdims=True)
    rounding = np.sqrt(((torch.from_numpy(ref).bfloat16().double().numpy() - ref) ** 2).mean())
    args = (0, h.ints([0] * n), h.ints([tokens - 1] * n), dev(q_bits, torch.bfloat16), dev(np.full(n, 2, np.uint8), torch.uint8))
    for got in (h.gpu.decode_attn_sinks(*args, 0), h.gpu.decode_attn_shared(*args, h.ints([0, n // 2, n]))):
        assert h.gpu.status() == 0
        error = np.sqrt(((got.double().cpu().numpy() - ref) ** 2).mean())
        assert error <= 1.1 * rounding, f"{error / rounding:.2f} times the rounding of the output"
