"""Attention over groups and sinks where every CTA and every warp has a long run: rings, records
and barriers used many times over, segments and jobs that follow one another within a run, batches
of page addresses renewed inside it, changes of class, SMs left to the few rows.

Few sequences and many queries that name them again make such calls small to check.  A test that
has to reach a state reads it off the call's plan: the workspace begins with four 64-bit numbers,
work and share of the tensor kernel's CTAs (2 a tile, 2 a segment), work and share of the few-row
kernel's warps (1 a block, 1 a segment)."""
import numpy as np
import pytest
import torch

from _parity import check_attention, dev
from _shared import Holder
from paper_2607_06601_gb300 import workloads as wl

pytestmark = pytest.mark.gpu

EVEN, NATIVE = (0.25,) * 4, (0, 0, 0, 1)


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def holder(rng, lay, lengths, mix):
    Hq, Hkv, d, G, P = lay
    most = max(lengths)
    h = Holder(1, len(lengths), Hq, Hkv, d, G, P, most, [sum(-(-n // P) + 1 for n in lengths)] * 4, archive=len(lengths) * -(-most // 1024) + 4,
               max_queries=1024)
    for s, n in enumerate(lengths):
        for at in range(0, n, 1024):
            h.append(rng, 0, s, np.arange(at, min(n, at + 1024)), mix)
    return h


def truth(h, seqs, ts, q_bits, modes, windows, sinks):
    """The definition in 64 bits, a sequence's queries at once."""
    q = wl.bf16_to_f32(q_bits).astype(np.float64)
    seqs, ts, modes, windows = (np.asarray(x, np.int64) for x in (seqs, ts, modes, windows))
    heads, out = h.Hq // h.Hkv, np.zeros((len(seqs), h.Hq, h.d))
    for s in np.unique(seqs):
        mine = np.flatnonzero((seqs == s) & (modes > 0))
        if mine.size == 0:
            continue
        for kvh in range(h.Hkv):
            pos, k, v = h.values(0, int(s), kvh)
            see = pos[None] <= ts[mine, None]
            see &= (modes[mine, None] == 2) | (pos[None] > (ts - windows)[mine, None]) | (pos[None] < sinks)
            x = np.einsum("qhd,kd->qhk", q[mine, kvh * heads:(kvh + 1) * heads], k, optimize=True) / np.sqrt(h.d)
            x = np.where(see[:, None], x, -np.inf)
            top = x.max(-1, keepdims=True)
            p = np.exp(x - np.where(np.isfinite(top), top, 0))
            total = p.sum(-1, keepdims=True)
            out[mine, kvh * heads:(kvh + 1) * heads] = p @ v / np.where(total > 0, total, 1)
    return out


def check(h, rng, seqs, ts, modes, windows, sinks, offsets=None):
    """Runs the call, compares its rows, returns its plan's (work, share, few work, few share)."""
    q = wl.bf16_bits(rng.standard_normal((len(seqs), h.Hq, h.d), dtype=np.float32))
    args = (0, h.ints(seqs), h.ints(ts), dev(q, torch.bfloat16), dev(np.asarray(modes, np.uint8), torch.uint8))
    if offsets is None:
        got = h.gpu.decode_attn_sinks(*args, sinks, windows=h.ints(windows))
    else:
        got = h.gpu.decode_attn_shared(*args, h.ints(offsets), windows=h.ints(windows), sinks=sinks)
    assert h.gpu.status() == 0
    check_attention(got.double().cpu().numpy(), truth(h, seqs, ts, q, modes, windows, sinks), np.asarray(modes))
    return h.gpu.workspace()[:32].view(torch.int64).tolist()


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


# (query heads, KV heads, d, group, page): plain and permuted rows, one, two and four groups of a row
WIDE = [(4, 4, 64, 32, 16), (12, 4, 64, 64, 32), (4, 2, 64, 32, 64), (8, 2, 128, 64, 16), (6, 1, 128, 128, 32), (8, 1, 128, 32, 64)]
FEW = [(4, 4, 64, 32, 16), (12, 4, 64, 64, 32), (4, 2, 64, 32, 64), (8, 2, 128, 64, 16), (6, 1, 128, 128, 32), (4, 2, 128, 32, 32)]


@pytest.mark.parametrize("mix", [EVEN, NATIVE, (0.5, 0.45, 0.05, 0)])
@pytest.mark.parametrize("lay", WIDE)
def test_many_tiles_for_every_cta(lay, mix):
    """Groups of 32 to 200 rows (and one or two of a KV head) over prompts of thousands of tokens."""
    rng = np.random.default_rng([1, *lay])
    lengths = [10_005, 7555, 9301]
    h = holder(rng, lay, lengths, mix)
    heads = lay[0] // lay[1]
    sizes = [max(2, rows // heads) for rows in (32, 70, 200, 130, 40, 9, 64, 33)]
    offsets, seqs = [0], []
    tiles = sum(-(-5000 * m // (128 if c < 3 else 64)) for c, m in enumerate(mix))  # of one segment, roughly
    need = 24 * sms() / tiles / lay[1]
    i = 0
    while need > 0 and offsets[-1] + sizes[i % len(sizes)] <= 1000:
        m = sizes[i % len(sizes)]
        seqs += [i % 3] * m
        offsets.append(offsets[-1] + m)
        need -= -(-m * heads // 128)
        i += 1
    ts = [lengths[s] - 1 - int(rng.integers(0, 60)) for s in seqs]
    n = len(seqs)
    work, per, few_work, few_per = check(h, rng, seqs, ts, [2] * n, [1] * n, 0, offsets)
    assert per >= 2 * 20
    modes = rng.choice(3, n, p=(0.1, 0.2, 0.7))
    check(h, rng, seqs, ts, modes, rng.choice([5, 300, 2000], n), 33, offsets)


@pytest.mark.parametrize("mix", [EVEN, NATIVE])
@pytest.mark.parametrize("lay", [WIDE[0], WIDE[1], (16, 4, 128, 64, 32)])
def test_many_segments_for_every_cta(lay, mix):
    """Short prompts by the hundred: a CTA's run holds whole segments, and more than it announces ahead."""
    rng = np.random.default_rng([2, *lay])
    lengths = [300, 131, 64, 260, 17, 205]
    h = holder(rng, lay, lengths, mix)
    members = 5
    groups = 200
    seqs = [g % 6 for g in range(groups) for _ in range(members)]
    ts = [lengths[s] - 1 for s in seqs]
    n = len(seqs)
    work, per, few_work, few_per = check(h, rng, seqs, ts, [2] * n, [1] * n, 0, list(range(0, n + 1, members)))
    segments = 4 * sum(lengths[g % 6] >= 60 for g in range(groups))
    assert segments / sms() > 3 and per >= 15
    odd = np.sort(rng.choice(n + 1, 190, replace=False)).tolist()
    check(h, rng, seqs, ts, rng.choice(3, n), rng.choice([1, 20, 100], n), 4, odd)  # groups across prompts


@pytest.mark.parametrize("mix", [EVEN, NATIVE, (0, 0, 1, 0), (0.5, 0.5, 0, 0)])
@pytest.mark.parametrize("lay", FEW)
def test_many_blocks_for_every_warp(lay, mix):
    """A thousand single queries at positions all over sequences of thousands of tokens."""
    rng = np.random.default_rng([3, *lay])
    lengths = [4001, 3333]
    h = holder(rng, lay, lengths, mix)
    n = 1000
    seqs = rng.integers(0, 2, n)
    ts = [int(rng.integers(lengths[s] * 3 // 4, lengths[s])) for s in seqs]
    modes = rng.choice([1, 2], n, p=(0.2, 0.8))
    work, per, few_work, few_per = check(h, rng, seqs, ts, modes, rng.choice([1500, 2900], n), 100)
    assert few_per >= (40 if lay[1] > 1 else 25)
    # windows that leave every run many short segments, and queries that see nothing or are skipped
    ts = [int(rng.integers(0, lengths[s])) for s in seqs]
    check(h, rng, seqs, ts, rng.choice(3, n), rng.choice([1, 17, 40, 600], n), 20)


def test_sms_left_to_the_few_rows():
    """The plan's rule that reserves SMs for the few rows beside a long share of tiles."""
    rng = np.random.default_rng(4)
    lay = WIDE[0]
    h = holder(rng, lay, [4001], EVEN)
    members, n = 5, 60
    for last in (4000, 3990):
        work, per, few_work, few_per = check(h, rng, [0] * n, [last] * n, [2] * n, [1] * n, 0, list(range(0, n + 1, members)))
        # shares of 20 and more, and runs of more than 6 blocks on few SMs' warps (16 each): not on all of them
        assert per >= 20 and few_per > 6 and few_work <= few_per * 16 * (sms() // 16)
