"""Page operations (trr_fork, trr_evict, trr_free_seqs, trr_compact) on the GPU against the
plain model of tests/_shared.py: metadata and every byte of the pools equal, and attention
and appends afterwards over the tokens that each sequence should hold."""
import numpy as np
import pytest
import torch

from _parity import check_attention, dev
from _shared import META, Holder, model_compact, model_evict, model_fork, model_free, same, snapshot
from paper_2607_06601_gb300 import trr, workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def holder(rng, L=2, S=10, Hq=4, Hkv=2, d=64, G=32, P=16, n=300, caps=(400,) * 4, seqs=3, **kw):
    h = Holder(L, S, Hq, Hkv, d, G, P, n + 200, list(caps), **kw)
    for layer in range(L):
        for s in range(seqs):
            h.append(rng, layer, s, np.arange(n - 7 * s))
    return h


def check_rows(h, rng, seqs):
    """Every mode's attention of the sequences' last positions, by the library's existing call."""
    if h.head_modes:
        return
    for layer in range(h.L):
        held = [s for s in seqs if h.tokens[layer][s]]
        if not held:
            continue
        ts = [max(h.tokens[layer][s]) for s in held]
        q = wl.bf16_bits(rng.standard_normal((len(held), h.Hq, h.d), dtype=np.float32))
        for mode in (1, 2):
            got = h.gpu.decode_attn(layer, h.ints(held), h.ints(ts), dev(q, torch.bfloat16),
                                    dev(np.full(len(held), mode, np.uint8), torch.uint8), window_scalar=50)
            assert h.gpu.status() == 0
            check_attention(got.double().cpu().numpy(), h.attend(layer, held, ts, q, [mode] * len(held), [50] * len(held)))


@pytest.mark.parametrize("kw", [dict(), dict(Hq=8, Hkv=2, d=128, G=64, P=32, L=1), dict(Hq=3, Hkv=3, P=64, G=64),
                                dict(Hq=4, Hkv=2, head_modes=1), dict(Hq=6, Hkv=3, d=128, G=128, head_modes=1, P=64)])
def test_every_operation_in_turn(kw):
    rng = np.random.default_rng(10)
    h = holder(rng, **kw)
    m = snapshot(h)
    # lengths: everything, a cut inside pages, on a page border, one token, none, past the end
    src, dst, lengths = [0, 0, 1, 2, 0, 1], [3, 4, 5, 6, 7, 8], [300, 123, 64, 1, 0, 10_000]
    h.fork(src, dst, lengths)
    model_fork(m, h, src, dst, lengths)
    same(snapshot(h), m, "fork")
    check_rows(h, rng, range(9))
    # the forks go on by themselves: neither the source nor a sister sees it
    for layer in range(h.L):
        for s in (3, 4, 6, 7):
            at = max(h.tokens[layer][s], default=-1) + 1
            last = int(m["last_pos"][layer, s])
            h.append(rng, layer, s, np.arange(max(at, last + 1), max(at, last + 1) + 40))
    check_rows(h, rng, range(9))
    m = snapshot(h)
    seqs, keep = [0, 3, 5, 6], [200, 310, 64, 41]
    h.gpu.evict(h.ints(seqs), h.ints(keep), 20)
    for (layer, s), gone in model_evict(m, h, seqs, keep, 20).items():
        for p in gone:
            del h.tokens[layer][s][p]
    same(snapshot(h), m, "evict")
    check_rows(h, rng, range(9))
    h.free([1, 4, 7])
    model_free(m, [1, 4, 7])
    same(snapshot(h), m, "free")
    h.gpu.compact()
    model_compact(m, h)
    same(snapshot(h), m, "compact")
    check_rows(h, rng, range(9))
    h.fork([0, 3], [0, 4], [150, 300])  # a sequence cut back in place, and a fork of what was evicted
    model_fork(m, h, [0, 3], [0, 4], [150, 300])
    same(snapshot(h), m, "cut back")
    for layer in range(h.L):
        h.append(rng, layer, 0, np.arange(160, 200))
        h.append(rng, layer, 1, np.arange(5, 60))  # a freed sequence starts anew
    check_rows(h, rng, range(9))
    m = snapshot(h)
    h.gpu.compact()
    model_compact(m, h)
    same(snapshot(h), m, "compact again")
    assert h.gpu.status() == 0
    check_rows(h, rng, range(9))


@pytest.mark.parametrize("seed", range(4))
def test_random_turns(seed):
    """Longer runs of random operations, sequences of all lengths."""
    rng = np.random.default_rng([seed, 20])
    h = holder(rng, L=1, S=12, n=[5, 200, 333, 64][seed], P=[16, 16, 32, 64][seed], seqs=2 + seed % 2, caps=(600,) * 4, archive=96)
    for turn in range(10):
        m = snapshot(h)
        perm = rng.permutation(h.S)
        k = int(rng.integers(1, 5))
        src, dst = rng.choice(perm[:4], k), perm[4:4 + k]
        lengths = rng.integers(0, 420, k)
        h.fork(src.tolist(), dst.tolist(), lengths.tolist())
        model_fork(m, h, src.tolist(), dst.tolist(), lengths.tolist())
        seqs = rng.choice(h.S, 3, replace=False).tolist()
        keep, sinks = rng.integers(0, 400, 3).tolist(), int(rng.integers(0, 70))
        h.gpu.evict(h.ints(seqs), h.ints(keep), sinks)
        for (layer, s), gone in model_evict(m, h, seqs, keep, sinks).items():
            for p in gone:
                del h.tokens[layer][s][p]
        out = rng.choice(h.S, 2, replace=False).tolist()
        h.free(out)
        model_free(m, out)
        if turn % 2:
            h.gpu.compact()
            model_compact(m, h)
        same(snapshot(h), m, f"turn {turn}")
        assert h.gpu.status() == 0
        for s in rng.choice(h.S, 3, replace=False):
            at = int(snapshot(h)["last_pos"][0, s]) + 1
            if at + 30 < 500:
                h.append(rng, 0, int(s), np.arange(at, at + int(rng.integers(1, 30))))
    check_rows(h, rng, range(h.S))


def test_decode_step_right_after_each_operation():
    """The decode step reads a settled layer's state early: not right after these calls."""
    rng = np.random.default_rng(30)
    h = holder(rng, L=4, S=6, n=120, seqs=2)
    last = 119
    for turn in range(3):
        h.fork([0, 0], [2, 3], [120 + turn, 100])
        if turn:
            h.free([4])
            h.gpu.compact()
        last += 1
        for layer in range(h.L):
            k, v, q = (wl.bf16_bits(rng.standard_normal((2, x, h.d), dtype=np.float32)) for x in (h.Hkv, h.Hkv, h.Hq))
            seqs, pos = [0, 2], [last, last]
            bits = np.array([4, 16], np.uint8)
            out = h.gpu.decode_step(layer, h.ints(seqs), h.ints(pos), dev(k, torch.bfloat16), dev(v, torch.bfloat16),
                                    dev(bits, torch.uint8), dev(np.full(2, 2, np.uint8), torch.uint8), dev(q, torch.bfloat16))
            for i, s in enumerate(seqs):
                assert h.orc.append(layer, np.array([h.used + i], np.int32), np.array([last], np.int32), k[i:i + 1], v[i:i + 1],
                                    bits[i:i + 1], np.array([2], np.uint8)) == 0
                h.tokens[layer][s][last] = (h.used + i, last)
            check_attention(out.double().cpu().numpy(), h.attend(layer, seqs, pos, q, [2, 2], [0, 0]))
        h.used += 2
        assert h.gpu.status() == 0


def test_a_fork_in_error_changes_nothing():
    rng = np.random.default_rng(40)
    h = holder(rng, caps=(60,) * 4)
    m = snapshot(h)
    bad = [([0, 1], [3, 3], [10, 10]), ([0, 3], [3, 4], [10, 10]), ([0, 10], [3, 4], [5, 5]), ([0, -1], [3, 4], [5, 5]),
           ([0, 0], [3, 10], [5, 5]), ([0, 0], [3, 4], [5, -1]), ([0, 0], [0, 3], [5, 5])]
    for src, dst, lengths in bad:
        h.gpu.fork(h.ints(src), h.ints(dst), h.ints(lengths))
        assert h.gpu.status() == 1
        same(snapshot(h), m, f"{src} {dst}")
    full = next_free = int(m["next_page"].max())
    while next_free < 60:  # forks of a cut page fill the pools, then one more does not fit
        h.gpu.fork(h.ints([0] * 7), h.ints(range(3, 10)), h.ints([201] * 7))
        st = h.gpu.status()
        now = snapshot(h)
        if st:
            assert st == 3
            same(now, m, "out of pages")
            break
        m, next_free = now, int(now["next_page"].max())
    else:
        pytest.fail("the pool never ran out")
    assert full < 60
    h.gpu.free(h.ints(range(3, 10)))
    h.gpu.compact()
    h.gpu.fork(h.ints([0]), h.ints([3]), h.ints([201]))
    assert h.gpu.status() == 0


def test_entries_in_error_of_evict_and_free():
    rng = np.random.default_rng(41)
    h = holder(rng)
    m = snapshot(h)
    h.gpu.evict(h.ints([0, 10, 1, 0, -1]), h.ints([200, 200, 150, 290, 5]), 4)
    assert h.gpu.status() == 1
    model_evict(m, h, [0, 1], [200, 150], 4)
    same(snapshot(h), m, "evict")
    h.gpu.free(h.ints([2, 77, 2]))
    assert h.gpu.status() == 1
    model_free(m, [2])
    same(snapshot(h), m, "free")


def test_refusals_and_empty_calls():
    rng = np.random.default_rng(42)
    h = holder(rng)
    m = snapshot(h)
    c, none = h.gpu, torch.zeros(0, dtype=torch.int32, device="cuda")
    c.fork(none, none, none)
    c.evict(none, none, 3)
    c.free(none)
    too_many = torch.zeros(h.S + 1, dtype=torch.int32, device="cuda")
    for call in (lambda: c.fork(too_many, too_many, too_many), lambda: c.evict(too_many, too_many), lambda: c.free(too_many),
                 lambda: c.evict(h.ints([0]), h.ints([5]), -1)):
        with pytest.raises(trr.TrrError) as e:
            call()
        assert e.value.code == 1
    small = torch.empty(c.workspace().numel() - 1, dtype=torch.uint8, device="cuda")
    odd = torch.empty(c.workspace().numel() + 256, dtype=torch.uint8, device="cuda")[16:]
    for ws in (small, odd):
        for call in (lambda: trr.trr_compact(c.handle, ws), lambda: trr.trr_fork(c.handle, h.ints([0]), h.ints([3]), h.ints([9]), ws)):
            with pytest.raises(trr.TrrError) as e:
                call()
            assert e.value.code == 2
    for call in (lambda: c.fork(h.ints([0, 1]), h.ints([3]), h.ints([5, 5])), lambda: c.evict(h.ints([0]), h.ints([5, 6])),
                 lambda: c.free(torch.zeros(1, dtype=torch.int64, device="cuda")), lambda: c.free(torch.zeros(1, dtype=torch.int32)),
                 lambda: c.free(h.ints([1, 2, 3, 4])[::2])):
        with pytest.raises(ValueError):
            call()
    assert c.status() == 0
    same(snapshot(h), m, "refused calls")


def test_in_a_graph_on_another_stream():
    """A turn of a beam search captured once and replayed: each replay gives the same state."""
    rng = np.random.default_rng(43)
    h = holder(rng)
    src, a, b = h.ints([0, 1, 0]), h.ints([3, 4, 5]), h.ints([6, 7, 8])
    lengths, keep = h.ints([250, 200, 77]), h.ints([150, 0, 70])
    h.gpu.workspace()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        h.gpu.fork(src, b, lengths)
        h.gpu.evict(b, keep, 4)
        h.gpu.free(a)
        h.gpu.compact()
        h.gpu.fork(b, a, lengths)
        h.gpu.free(b)
        h.gpu.compact()
    graph.replay()
    first = snapshot(h)
    for _ in range(3):
        graph.replay()
    now = snapshot(h)
    for n in META:
        assert np.array_equal(first[n], now[n]), n
    assert h.gpu.status() == 0 and (now["ntok"][:, 3:6].sum(-1) > 0).all() and (now["ntok"][:, 6:] == 0).all()
