"""Attention with sinks and over shared prompts (trr_decode_attn_sinks, trr_decode_attn_shared)
against the definition in 64 bits, at the sizes and masks where such kernels go wrong.

The bounds are those of the library's attention (tests/_parity.py): 5e-3 of a row's largest
value and 2e-2 on top of the output's own rounding."""
import numpy as np
import pytest
import torch

from _parity import check_attention, dev
from _shared import Holder
from paper_2607_06601_gb300 import trr, workloads as wl

pytestmark = pytest.mark.gpu

LAYOUTS = [dict(Hq=4, Hkv=4, d=64, G=32, P=16), dict(Hq=12, Hkv=4, d=64, G=64, P=32), dict(Hq=8, Hkv=2, d=128, G=64, P=16),
           dict(Hq=4, Hkv=2, d=64, G=32, P=64), dict(Hq=6, Hkv=1, d=128, G=128, P=32), dict(Hq=8, Hkv=1, d=128, G=32, P=64)]


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def family(rng, lay, prompts, members, prefix, suffix, mix=(0.25,) * 4, p_skip=0.2, maxctx=1024, archive=0):
    """`prompts` sequences of `prefix` tokens, each forked `members` times; the forks go on."""
    S = prompts * (1 + members)
    caps = [prompts * (prefix // lay["P"] + 2) + S * (2 + -(-suffix // lay["P"])) + S] * 4
    h = Holder(1, S, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], maxctx, caps, archive=2 * S + 8 + archive)
    for s in range(prompts):
        h.append(rng, 0, s, np.arange(prefix), mix, p_skip)
    kids = list(range(prompts, S))
    if kids:
        h.fork([(s - prompts) // members for s in kids], kids, [prefix] * len(kids))
        for s in kids:
            n = int(rng.integers(max(1, suffix // 2), suffix + 1))
            h.append(rng, 0, s, np.arange(prefix, prefix + n), mix, p_skip)
    return h, kids


def last_of(h, seqs):
    last = h.gpu.region("last_pos").cpu().numpy().view(np.int32)
    return [int(last[s]) for s in seqs]


def run(h, rng, seqs, ts, modes, windows, sinks=0, offsets=None, scale=0.0, expect=0, stream=None, loud=1.0):
    q = wl.bf16_bits(loud * rng.standard_normal((len(seqs), h.Hq, h.d), dtype=np.float32))
    args = (0, h.ints(seqs), h.ints(ts), dev(q, torch.bfloat16), dev(np.asarray(modes, np.uint8), torch.uint8))
    out = torch.full((len(seqs), h.Hq, h.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    if offsets is None:
        h.gpu.decode_attn_sinks(*args, sinks, windows=h.ints(windows), softmax_scale=scale, out=out, stream=stream)
    else:
        h.gpu.decode_attn_shared(*args, h.ints(offsets), windows=h.ints(windows), sinks=sinks, softmax_scale=scale, out=out, stream=stream)
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    assert h.gpu.status() == expect
    return out.double().cpu().numpy(), q


def check(h, rng, seqs, ts, modes, windows, sinks=0, offsets=None, scale=0.0, **kw):
    got, q = run(h, rng, seqs, ts, modes, windows, sinks, offsets, scale, **kw)
    check_attention(got, h.attend(0, seqs, ts, q, modes, windows, sinks, scale if scale > 0 else None), modes)
    return got


@pytest.mark.parametrize("lay", LAYOUTS)
@pytest.mark.parametrize("prefix,suffix", [(1, 1), (15, 3), (64, 1), (333, 40)])
def test_shared_prompt_all_full(lay, prefix, suffix):
    rng = np.random.default_rng([1, prefix])
    h, kids = family(rng, lay, 1, 5, prefix, suffix)
    check(h, rng, kids, last_of(h, kids), [2] * 5, [1] * 5, 0, [0, 5])


@pytest.mark.parametrize("lay", LAYOUTS)
def test_several_prompts_routed(lay):
    """Groups of every mode, windows from one token to past the start, sinks; queries outside
    the groups; empty groups."""
    rng = np.random.default_rng(2)
    h, kids = family(rng, lay, 3, 6, 200, 50)
    ts = last_of(h, kids)
    modes = rng.choice(3, len(kids))
    windows = rng.choice([1, 7, 64, 150, 1000], len(kids))
    for sinks in (0, 1, 20, 64):
        check(h, rng, kids, ts, modes, windows, sinks, [0, 6, 12, 18])
    check(h, rng, kids, ts, modes, windows, 4, [2, 2, 6, 6, 11])
    check(h, rng, kids, ts, modes, windows, 4, [0])
    check(h, rng, kids, ts, modes, windows, 4, [0, 18])  # groups of sequences with no page in common
    check(h, rng, kids, ts, modes, windows, 4)


@pytest.mark.parametrize("lay", LAYOUTS[:4])
@pytest.mark.parametrize("members", [1, 2, 9, 33, 70])
def test_rows_of_a_group(lay, members):
    """From one row for a KV head to more than a tile of 128."""
    rng = np.random.default_rng([3, members])
    h, kids = family(rng, lay, 1, members, 150, 5)
    check(h, rng, kids, last_of(h, kids), [2] * members, [1] * members, 0, [0, members])


@pytest.mark.parametrize("mix", [(1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (0, 0.5, 0, 0.5)])
@pytest.mark.parametrize("lay", LAYOUTS[:3])
def test_each_width(lay, mix):
    rng = np.random.default_rng([4, int(10 * mix[0]), int(10 * mix[3])])
    h, kids = family(rng, lay, 2, 4, 260, 30, mix=mix, p_skip=0.0)
    ts = last_of(h, kids)
    check(h, rng, kids, ts, [2] * 8, [1] * 8, 0, [0, 4, 8])
    check(h, rng, kids, ts, [1] * 8, [40] * 8, 10)


@pytest.mark.parametrize("lay", LAYOUTS)
def test_window_and_sinks(lay):
    """The two ranges apart, touching, overlapping, in one page, and either of them empty."""
    rng = np.random.default_rng(5)
    h, _ = family(rng, lay, 2, 0, 300, 0)
    n = 12
    seqs = [0, 1] * 6
    ts = [299] * 6 + [0, 1, 15, 16, 63, 130]
    for sinks in (0, 1, 16, 17, 100, 290, 5000):
        check(h, rng, seqs, ts, [1] * n, [1, 2, 16, 17, 200, 1 << 30] * 2, sinks)
    check(h, rng, seqs, ts, [2, 1, 0] * 4, [33] * n, 5)


def test_without_sinks_the_rows_are_those_of_decode_attn():
    """Both calls' rows are the definition's; each is rounded to bf16 by itself, so they may
    differ from one another by a unit in the last place."""
    rng = np.random.default_rng(6)
    h, kids = family(rng, LAYOUTS[0], 2, 4, 300, 40)
    ts, modes, windows = last_of(h, kids), [2, 1, 2, 1, 0, 2, 1, 2], [64] * 8
    got, q = run(h, np.random.default_rng(61), kids, ts, modes, windows, 0, [0, 4, 8])
    ref = h.gpu.decode_attn(0, h.ints(kids), h.ints(ts), dev(q, torch.bfloat16), dev(np.asarray(modes, np.uint8), torch.uint8),
                            windows=h.ints(windows))
    truth = h.attend(0, kids, ts, q, modes, windows)
    check_attention(got, truth, modes)
    check_attention(ref.double().cpu().numpy(), truth, modes)


def test_positions_inside_the_shared_past():
    """Queries of a group at positions before the fork, one sequence named several times."""
    rng = np.random.default_rng(7)
    h, kids = family(rng, LAYOUTS[1], 1, 4, 200, 30)
    seqs = kids + [kids[0], kids[1], 0, 0]
    ts = last_of(h, kids) + [150, 10, 199, 0]
    check(h, rng, seqs, ts, [2] * 8, [1] * 8, 0, [0, 8])
    check(h, rng, seqs, ts, [1, 2] * 4, [60] * 8, 3, [0, 4, 8])


def test_rows_that_see_nothing():
    rng = np.random.default_rng(8)
    h = Holder(1, 4, 4, 2, 64, 32, 16, 600, [60] * 4)
    h.append(rng, 0, 0, np.arange(100), p_skip=0.0)
    h.append(rng, 0, 1, np.arange(300, 340), p_skip=0.0)
    h.append(rng, 0, 2, np.arange(50), p_skip=1.0)
    seqs, ts = [0, 1, 1, 2, 3, 0], [500, 200, 320, 49, 10, 599]
    got = check(h, rng, seqs, ts, [1, 2, 1, 2, 2, 1], [50, 1, 400, 1, 1, 20], 0, [0, 6])
    assert (got[[0, 1, 3, 4, 5]] == 0).all() and (got[2] != 0).any()
    got = check(h, rng, seqs, ts, [1, 2, 1, 2, 2, 1], [50, 1, 400, 1, 1, 20], 8)
    assert (got[0] != 0).any() and (got[3] == 0).all()


def test_pages_after_an_eviction():
    """What eviction leaves is what a query with those sinks and that window sees."""
    rng = np.random.default_rng(9)
    h, kids = family(rng, LAYOUTS[0], 1, 3, 400, 20)
    ts, windows = last_of(h, kids), [64, 90, 33]
    before, q = run(h, np.random.default_rng(91), kids, ts, [1] * 3, windows, 10)
    h.gpu.evict(h.ints(kids), h.ints([t - w + 1 for t, w in zip(ts, windows)]), 10)
    after, _ = run(h, np.random.default_rng(91), kids, ts, [1] * 3, windows, 10)
    check_attention(before, h.attend(0, kids, ts, q, [1] * 3, windows, 10))
    check_attention(after, h.attend(0, kids, ts, q, [1] * 3, windows, 10))


@pytest.mark.parametrize("lay", [LAYOUTS[0], LAYOUTS[2]])
def test_nan_and_infinity_out_of_sight(lay):
    """16-bit rows may hold anything: what a row does not see does not reach it, and a row
    that sees it is not finite."""
    rng = np.random.default_rng(11)
    P = lay["P"]
    h = Holder(1, 4, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], P, 400, [80] * 4)
    k, v = (wl.bf16_bits(rng.standard_normal((200, lay["Hkv"], lay["d"]), dtype=np.float32)) for _ in range(2))
    for p, bad in ((30, 0x7FC0), (31, 0x7F80), (120, 0xFF80)):
        k[p], v[p] = bad, bad
    h.append(rng, 0, 0, np.arange(200), k=k, v=v, bits=np.full(200, 16), p_skip=0.0)
    h.fork([0, 0], [1, 2], [200, 200])
    for s in (1, 2):
        h.append(rng, 0, s, np.arange(200, 210), p_skip=0.0)
    check(h, rng, [1, 2, 0, 0], [209, 205, 119, 29], [1, 1, 1, 2], [80, 30, 88, 1], 30, [0, 2])
    got, _ = run(h, rng, [1, 2, 0], [209, 209, 29], [2, 1, 2], [1, 20, 1], 5, [0, 3])
    assert not np.isfinite(got[0]).any() and np.isfinite(got[1:]).all()


def test_large_scores_and_values():
    """Scores far apart (one key takes all), values near the ends of binary16, tiny ones."""
    rng = np.random.default_rng(12)
    lay = LAYOUTS[1]
    for scale in (1e-4, 60000.0):
        h = Holder(1, 3, lay["Hq"], lay["Hkv"], lay["d"], lay["G"], lay["P"], 400, [60] * 4)
        k = wl.bf16_bits(rng.standard_normal((300, lay["Hkv"], lay["d"]), dtype=np.float32))
        v = wl.bf16_bits(scale * rng.uniform(-1, 1, (300, lay["Hkv"], lay["d"])).astype(np.float32))
        h.append(rng, 0, 0, np.arange(300), k=k, v=v)
        h.fork([0], [1], [300])
        got, q = run(h, rng, [0, 1], [299, 299], [2, 2], [1, 1], 0, [0, 2], loud=8.0)
        ref = h.attend(0, [0, 1], [299, 299], q, [2, 2], [1, 1])
        # relative to the values' size: the absolute bound of check_attention is for values near one
        assert np.abs(got - ref).max() <= 5e-3 * np.abs(ref).max()
    h, kids = family(rng, lay, 1, 3, 300, 20)
    check(h, rng, kids, last_of(h, kids), [2] * 3, [1] * 3, 0, [0, 3], scale=2.0)
    check(h, rng, kids, last_of(h, kids), [2] * 3, [1] * 3, 0, [0, 3], scale=1e-6)


def test_queries_of_any_size():
    """Query rows far outside binary16's range, and zero ones."""
    rng = np.random.default_rng(13)
    h, kids = family(rng, LAYOUTS[0], 1, 3, 130, 9)
    for loud in (1e-30, 0.0, 1e12):
        check(h, rng, kids, last_of(h, kids), [2] * 3, [1] * 3, 0, [0, 3], scale=1.0 / max(loud, 1.0), loud=loud)


def test_long_context():
    """A prompt of many tiles in the wide-group layout, and windows deep inside it."""
    rng = np.random.default_rng(14)
    lay = LAYOUTS[2]
    h, kids = family(rng, lay, 1, 6, 1000, 60, maxctx=4096)
    for s in kids[:2]:
        h.append(rng, 0, s, np.arange(1100, 2100))
    ts = last_of(h, kids)
    check(h, rng, kids, ts, [2] * 6, [1] * 6, 0, [0, 6])
    check(h, rng, kids, ts, [1, 2, 1, 2, 1, 1], [700, 1, 300, 1, 64, 999], 64, [0, 6])


def test_other_stream_and_graph():
    rng = np.random.default_rng(15)
    h, kids = family(rng, LAYOUTS[0], 2, 4, 150, 20)
    ts = last_of(h, kids)
    s = torch.cuda.Stream()
    check(h, rng, kids, ts, [2, 1, 2, 0] * 2, [30] * 8, 4, [0, 4, 8], stream=s)
    q = wl.bf16_bits(rng.standard_normal((8, h.Hq, h.d), dtype=np.float32))
    out = torch.empty((8, h.Hq, h.d), dtype=torch.bfloat16, device="cuda")
    args = (0, h.ints(kids), h.ints(ts), dev(q, torch.bfloat16), dev(np.full(8, 2, np.uint8), torch.uint8), h.ints([0, 4, 8]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.gpu.decode_attn_shared(*args, out=out)
    for _ in range(2):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        check_attention(out.double().cpu().numpy(), h.attend(0, kids, ts, q, [2] * 8, [1] * 8))
    assert h.gpu.status() == 0


def test_the_same_call_gives_the_same_bits():
    rng = np.random.default_rng(16)
    h, kids = family(rng, LAYOUTS[2], 2, 8, 700, 60)
    ts = last_of(h, kids)
    rows = [run(h, np.random.default_rng(17), kids, ts, [2] * 16, [1] * 16, 0, [0, 8, 16])[0] for _ in range(4)]
    assert all(np.array_equal(rows[0], r) for r in rows[1:])


def test_errors_zero_the_query_and_keep_the_rest():
    rng = np.random.default_rng(18)
    h, kids = family(rng, LAYOUTS[0], 1, 6, 100, 10)
    ts = last_of(h, kids)
    seqs, modes, windows = list(kids), [2, 1, 2, 2, 1, 2], [5] * 6
    for change, code in (((seqs, 3, 99), 1), ((ts, 2, -1), 4), ((ts, 2, 1024), 4), ((modes, 5, 3), 1), ((windows, 4, 0), 1)):
        lists = [list(x) for x in (seqs, ts, modes, windows)]
        at = [seqs, ts, modes, windows].index(change[0])
        lists[at][change[1]] = change[2]
        for offsets in (None, [0, 6]):
            got, q = run(h, rng, *lists, 2, offsets, expect=code)
            ok = [i for i in range(6) if i != change[1]]
            ref = h.attend(0, [seqs[i] for i in ok], [ts[i] for i in ok], q[ok], [modes[i] for i in ok], [windows[i] for i in ok], 2)
            check_attention(got[ok], ref)
            assert (got[change[1]] == 0).all()
    # two errors: the lowest query's counts
    got, _ = run(h, rng, [99] + seqs[1:], ts[:1] + [-5] + ts[2:], modes, windows, 0, [0, 6], expect=1)
    got, _ = run(h, rng, seqs[:1] + [99] + seqs[2:], [5000] + ts[1:], modes, windows, 0, [0, 6], expect=4)
    for offsets in ([0, 7], [-1, 3], [4, 2], [0, 6, 3]):
        got, _ = run(h, rng, seqs, ts, modes, windows, 0, offsets, expect=1)
        assert (got == 0).all()


def test_refusals_and_empty_calls():
    rng = np.random.default_rng(19)
    h, kids = family(rng, LAYOUTS[0], 1, 2, 50, 5)
    c, n = h.gpu, 2
    ids, ts, modes, off = h.ints(kids), h.ints(last_of(h, kids)), dev(np.full(2, 2, np.uint8), torch.uint8), h.ints([0, 2])
    q = torch.zeros((n, h.Hq, h.d), dtype=torch.bfloat16, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    empty = c.decode_attn_shared(0, none, none, q[:0], modes[:0], h.ints([0]))
    assert empty.shape == (0, h.Hq, h.d) and c.launches() == 0
    long = torch.zeros(4000, dtype=torch.int32, device="cuda")
    qs = torch.zeros((4000, h.Hq, h.d), dtype=torch.bfloat16, device="cuda")
    for call, code in ((lambda: c.decode_attn_sinks(1, ids, ts, q, modes, 0), 1), (lambda: c.decode_attn_sinks(-1, ids, ts, q, modes, 0), 1),
                       (lambda: c.decode_attn_sinks(0, ids, ts, q, modes, -1), 1),
                       (lambda: c.decode_attn_shared(0, ids, ts, q, modes, h.ints([0, 1, 1, 2])), 1),
                       (lambda: c.decode_attn_sinks(0, long, long, qs, long.to(torch.uint8), 0), 1)):
        with pytest.raises(trr.TrrError) as e:
            call()
        assert e.value.code == code
    room = torch.zeros(n * h.Hq * h.d + 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(trr.TrrError) as e:
        c.decode_attn_sinks(0, ids, ts, room[1:1 + q.numel()].view(q.shape), modes, 0)  # rows off their 16 bytes
    assert e.value.code == 1
    with pytest.raises(trr.TrrError) as e:
        trr.trr_decode_attn_sinks(c.handle, 0, ids, ts, q, modes, None, 1, 0, 0.0, torch.empty_like(q), c.workspace()[:-1])
    assert e.value.code == 2
    for call in (lambda: c.decode_attn_sinks(0, ids, ts[:1], q, modes, 0), lambda: c.decode_attn_sinks(0, ids, ts, q[:1], modes, 0),
                 lambda: c.decode_attn_sinks(0, ids, ts, q, modes, 0, windows=ts[:1]), lambda: c.decode_attn_sinks(0, ids, ts, q.float(), modes, 0),
                 lambda: c.decode_attn_shared(0, ids, ts, q, modes, none), lambda: c.decode_attn_shared(0, ids, ts, q.transpose(0, 1), modes, off),
                 lambda: c.decode_attn_sinks(0, ids, ts, q, modes, 0, out=q[:1])):
        with pytest.raises(ValueError):
            call()
    heads = Holder(1, 2, 4, 2, 64, 32, 16, 100, [20] * 4, head_modes=1)
    with pytest.raises(trr.TrrError) as e:
        heads.gpu.decode_attn_sinks(0, h.ints([0]), h.ints([5]), q[:1], dev(np.full(1, 2, np.uint8), torch.uint8), 0)
    assert e.value.code == 6
    assert c.status() == 0
