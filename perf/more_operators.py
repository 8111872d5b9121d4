"""Prompts that enter a mixed-precision paged KV cache by chunks, and what a cache holds read back, as
cases to be run and timed.

Two kinds of case:

  chunk  attention of the new tokens of a batch of sequences, some tokens for each, over everything
         that the sequences have stored, the new tokens included (Cache.chunk_attn)
  read   K and V of stretches of positions, dequantised and in order of position, with the width of
         each token (Cache.read)

`prepare` lays the cache out byte for byte as the library documents it (include/trr.h), so both
forms read the same pages.  With `own` false, `run` computes with elementary torch operations in
32 bits; with `own` true it makes the library's calls.
"""
import math

import numpy as np
import torch

own = False

BITS = (2, 4, 8, 16)
# shares of tokens stored at 2, 4, 8 and 16 bits, as the repository's workloads mix them
MIXES = {"even": (0.25, 0.25, 0.25, 0.25), "decoder": (0.20, 0.40, 0.30, 0.10), "ragged": (0.25, 0.45, 0.25, 0.05),
         "long": (0.50, 0.45, 0.0, 0.05), "native": (0.0, 0.0, 0.0, 1.0), "four": (0.0, 1.0, 0.0, 0.0)}
STORED = 0.8           # share of tokens that are not skip tokens and so store their K and V
ROUTED = (0.2, 0.5, 0.3)  # shares of skip, local and full queries of a routed batch
SKIP, LOCAL, FULL = 0, 1, 2


def listed():
    return [
        # the last five tokens of one short prompt: the smallest call, all latency
        dict(name="chunk-tiny", kind="chunk", seqs=1, lo=67, hi=67, new_lo=5, new_hi=5, modes="full", window=32, sinks=0, hq=4, hkv=2, d=64, gs=32,
             page=16, mix="even"),
        # eight drafted tokens for each of 32 sequences of the small decoder, to be verified in one call
        dict(name="chunk-draft", kind="chunk", seqs=32, lo=2048, hi=2048, new_lo=8, new_hi=8, modes="full", window=256, sinks=0, hq=12, hkv=12, d=64,
             gs=32, page=32, mix="decoder"),
        # the last 512 tokens of one prompt of the small decoder, every token with its router's mode
        dict(name="chunk-160m-routed", kind="chunk", seqs=1, lo=2048, hi=2048, new_lo=512, new_hi=512, modes="routed", window=256, sinks=0, hq=12, hkv=12,
             d=64, gs=32, page=32, mix="decoder"),
        # a batch of prompts of odd lengths, chunks from one token to about a thousand, routed, first tokens kept in sight
        dict(name="chunk-ragged", kind="chunk", seqs=16, lo=1024, hi=8192, new_lo=1, new_hi=1021, modes="routed", window=511, sinks=4, hq=32, hkv=32, d=64,
             gs=32, page=32, mix="ragged"),
        # a whole prompt at once in a cache that stores everything at 16 bits
        dict(name="chunk-native", kind="chunk", seqs=1, lo=4096, hi=4096, new_lo=4096, new_hi=4096, modes="full", window=512, sinks=0, hq=32, hkv=32, d=64,
             gs=32, page=32, mix="native"),
        # streams whose new tokens see a window and the first tokens only, query groups of 4
        dict(name="chunk-stream", kind="chunk", seqs=8, lo=8192, hi=16384, new_lo=256, new_hi=700, modes="local", window=1024, sinks=64, hq=32, hkv=8,
             d=128, gs=64, page=32, mix="long"),
        # 2048 tokens at the end of a long document, query groups of 4: the largest call
        dict(name="chunk-gqa-long", kind="chunk", seqs=1, lo=32768, hi=32768, new_lo=2048, new_hi=2048, modes="full", window=1024, sinks=0, hq=32, hkv=8,
             d=128, gs=64, page=64, mix="long"),
        # one short sequence, whole, rounded to bf16
        dict(name="read-tiny", kind="read", seqs=1, lo=130, hi=130, share=1.0, dtype="bf16", hq=4, hkv=2, d=64, gs=32, page=16, mix="even"),
        # a layer of a batch of the small decoder, whole, to be handed to another worker
        dict(name="read-160m", kind="read", seqs=32, lo=2048, hi=2048, share=1.0, dtype="bf16", hq=12, hkv=12, d=64, gs=32, page=32, mix="decoder"),
        # the middle of ragged sequences in 32 bits, as a study of what quantisation costs takes it
        dict(name="read-ragged", kind="read", seqs=24, lo=1024, hi=8192, share=0.37, dtype="f32", hq=32, hkv=32, d=64, gs=32, page=32, mix="ragged"),
        # long documents, few wide KV heads
        dict(name="read-gqa-long", kind="read", seqs=4, lo=32768, hi=32768, share=1.0, dtype="bf16", hq=32, hkv=8, d=128, gs=64, page=32, mix="long"),
    ]


def draw(rng):
    def spread(lo, hi):  # whole numbers spread over their logarithm
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    hq, hkv, d, gs = rng.choice([(12, 12, 64, 32), (32, 32, 64, 32), (32, 8, 128, 64), (4, 2, 64, 32), (12, 4, 64, 64), (8, 2, 128, 32), (16, 2, 64, 64),
                                 (7, 1, 128, 128)])
    case = dict(hq=hq, hkv=hkv, d=d, gs=gs, page=rng.choice([16, 32, 64]), mix=rng.choice(sorted(MIXES)))
    if rng.random() < 0.35:
        seqs = spread(1, 32)
        hi = min(spread(40, 32768), max(40, 32 * 2048 * 18 * 64 // (seqs * hkv * d)))
        return dict(case, kind="read", seqs=seqs, lo=max(1, hi // rng.choice([1, 2, 8])), hi=hi, share=rng.choice([1.0, 0.6, 0.1]),
                    dtype=rng.choice(["bf16", "f32"]))
    seqs = spread(1, 32)
    hi = min(spread(40, 32768), max(40, 32 * 2048 * 32 * 64 // (seqs * hkv * d)))
    new = spread(1, max(1, min(hi, 2048, 2 ** 36 // (seqs * hi * hq * d) + 1)))
    return dict(case, kind="chunk", seqs=seqs, lo=max(1, new, hi // rng.choice([1, 2, 8])), hi=max(hi, new), new_lo=max(1, new // rng.choice([1, 3, 16])),
                new_hi=new, modes=rng.choice(["full", "routed", "routed", "local"]), window=spread(1, 1024), sinks=rng.choice([0, 1, 4, 64]))


# ------------------------------------------------------------------------------ inputs --


def up(x, a):
    return -(-x // a) * a


class Layout:
    """Sizes of the documented page layout for one case."""

    def __init__(self, case):
        self.hq, self.hkv, self.d, self.gs, self.P = case["hq"], case["hkv"], case["d"], case["gs"], case["page"]
        self.ng = self.d // self.gs
        g = self.hq // self.hkv
        self.permuted = not (g >= 2 and g * self.ng <= 8)  # 8- and 16-bit rows keep each line's chunks in a permuted order
        self.hdr = up(4 * self.P, 128)
        self.row = [self.d * b // 8 for b in BITS]         # bytes of one K or V row
        self.slice = [self.P * (2 * self.row[c] + (2 * self.ng * 4 if c < 3 else 0)) for c in range(4)]
        self.page = [up(self.hdr + self.hkv * s, 128) for s in self.slice]


def lengths(case):
    """Tokens of each sequence: the case's own, whatever the seed, so that outputs have one shape."""
    return np.random.default_rng(11).integers(case["lo"], case["hi"] + 1, case["seqs"])


def build(case, seed):
    """Which tokens each sequence stores at which width, and its tables.  Token i of a class, over all
    sequences in order, is row i of that class's K and V."""
    r = np.random.default_rng([seed, 1])
    P, S = case["page"], case["seqs"]
    lens = lengths(case)
    MP, W32 = -(-int(lens.max()) // P), -(-int(lens.max()) // 32)
    t = dict(last_pos=(lens - 1).astype(np.int32)[None], ntok=np.zeros((1, S, 4), np.int32), presence=np.zeros((1, S, W32), np.uint32))
    t.update({n: np.full((1, S, 4, MP), -1, np.int32) for n in ("page_table", "page_first", "page_last")})
    slots, rows, tokens = [[] for _ in BITS], [0] * 4, []
    for s in range(S):
        cls, has, at = r.choice(4, size=lens[s], p=MIXES[case["mix"]]), r.random(lens[s]) < STORED, np.arange(lens[s])
        mine = []
        for c in range(4):
            pos = at[has & (cls == c)]
            k, first = -(-len(pos) // P), sum(len(x) for x in slots[c])
            fill = np.full((k * P, 2), -1, np.int64)
            fill[:len(pos), 0], fill[:len(pos), 1] = pos, rows[c] + np.arange(len(pos))
            slots[c].append(fill.reshape(k, P, 2))
            t["page_table"][0, s, c, :k] = first + np.arange(k)
            t["page_first"][0, s, c, :k] = pos[::P]
            t["page_last"][0, s, c, :k] = [pos[min(len(pos), (i + 1) * P) - 1] for i in range(k)]
            t["ntok"][0, s, c] = len(pos)
            np.bitwise_or.at(t["presence"][0, s], pos // 32, np.uint32(1) << (pos % 32).astype(np.uint32))
            mine.append((pos, rows[c]))
            rows[c] += len(pos)
        tokens.append(mine)
    slots = [np.concatenate(x) for x in slots]
    # pages of a running cache lie in no order
    for c in range(4):
        order = r.permutation(len(slots[c]))
        slots[c] = slots[c][np.argsort(order)]
        table = t["page_table"][0, :, c]
        table[table >= 0] = order[table[table >= 0]]
    t["next_page"] = np.array([len(x) for x in slots], np.int32)
    return dict(tables=t, slots=slots, rows=rows, tokens=tokens, lens=lens, MP=MP, rng=r)


def rows_of(lay, counts, seed):
    """K and V of every stored token, by class: codes with scale and zero for each group, or bf16 rows."""
    g = torch.Generator("cuda").manual_seed(seed)
    loud = torch.ones(lay.hkv * lay.d, device="cuda")
    loud[torch.randperm(lay.hkv * lay.d, generator=g, device="cuda")[:-(-lay.hkv * lay.d // 100)]] = 8.0  # a few outlier channels
    found = []
    for c, b in enumerate(BITS):
        both = []
        for _ in range(2):
            x = (torch.randn(counts[c], lay.hkv * lay.d, generator=g, device="cuda") * loud).bfloat16().view(-1, lay.hkv, lay.ng, lay.gs)
            if b == 16:
                both.append(x.flatten(2))
                continue
            x = x.float()
            lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
            z, s = lo.half(), ((hi - lo) / (2 ** b - 1)).half()
            code = ((x - z.float()) / s.float()).round_().clamp_(0, 2 ** b - 1).to(torch.uint8)
            both.append((code.flatten(2), s.squeeze(-1), z.squeeze(-1)))
        found.append(both)
    return found


def permute_chunks(x, lay, c):
    """[.., slice bytes] with the 16-byte chunks of each 128-byte line of the code rows in the stored order, or back."""
    if not (lay.permuted and c >= 2):
        return x
    n = 2 * lay.P * lay.row[c]
    line = torch.arange(n // 128, device="cuda")[:, None]
    at = ((torch.arange(8, device="cuda") ^ (line % 8)) + 8 * line).flatten()
    lead = x.shape[:-1]
    codes = x[..., :n].reshape(*lead, n // 16, 16)[..., at, :].reshape(*lead, n)
    return torch.cat([codes, x[..., n:]], -1)


def page_bytes(lay, c, slots, rows):
    """[pages, page bytes] of one class: slot positions, then each KV head's slice."""
    pos = torch.from_numpy(slots[..., 0].astype(np.int32)).cuda().clamp_min(0)
    at = torch.from_numpy(slots[..., 1]).cuda().clamp_min(0)  # a slot that holds nothing keeps some other token's bytes
    n, P = at.shape
    out = torch.zeros(n, lay.page[c], dtype=torch.uint8, device="cuda")
    if n == 0:
        return out
    out[:, :4 * P] = pos.view(torch.uint8).view(n, 4 * P)
    parts = []
    for which in range(2):
        x = rows[which] if BITS[c] == 16 else rows[which][0]
        if BITS[c] == 16:
            x = x.view(torch.uint8).view(-1, lay.hkv, lay.row[c])
        elif BITS[c] < 8:
            per = 8 // BITS[c]
            x = x.view(-1, lay.hkv, lay.row[c], per)
            x = sum(x[..., i] << (BITS[c] * i) for i in range(per))
        parts.append(x[at].transpose(1, 2).reshape(n, lay.hkv, -1))
    if BITS[c] < 16:
        for which in range(2):
            sz = torch.stack(rows[which][1:], -1).view(torch.uint8).view(-1, lay.hkv, 4 * lay.ng)
            parts.append(sz[at].transpose(1, 2).reshape(n, lay.hkv, -1))
    out[:, lay.hdr:lay.hdr + lay.hkv * lay.slice[c]] = permute_chunks(torch.cat(parts, -1), lay, c).reshape(n, -1)
    return out


def stretches(case):
    """First position and number of positions of what a call asks of each sequence."""
    r, lens = np.random.default_rng(12), lengths(case)
    if case["kind"] == "chunk":  # the last tokens of each
        count = np.minimum(r.integers(case["new_lo"], case["new_hi"] + 1, len(lens)), lens)
        return lens - count, count
    count = np.maximum(1, (case["share"] * lens).astype(np.int64))
    return (lens - count) // 2, count


def modes_of(case, n, seed):
    r = np.random.default_rng([seed, 3])
    if case["modes"] == "routed":
        return r.choice(3, size=n, p=ROUTED).astype(np.uint8)
    return np.full(n, FULL if case["modes"] == "full" else LOCAL, np.uint8)


def query_rows(case, n, seed):
    g = torch.Generator("cuda").manual_seed(seed + 7)
    return torch.randn(n, case["hq"], case["d"], generator=g, device="cuda").bfloat16()


def prepare(case, seed):
    b, lay = build(case, seed), Layout(case)
    caps = [len(x) + 1 for x in b["slots"]]
    starts, count = stretches(case)
    state = dict(case=case, lay=lay)
    if own:
        from paper_2607_06601_gb300 import trr
        state["cache"] = cache = trr.Cache(1, case["seqs"], lay.hq, lay.hkv, lay.d, lay.gs, lay.P, int(b["lens"].max()), caps, max_append=64,
                                           max_queries=64)
        regions = {n: cache.region(n) for n in b["tables"]}
        pools = [cache.region("pool%d" % x).view(caps[c], lay.page[c]) for c, x in enumerate(BITS)]
    else:
        regions = {n: torch.empty(x.nbytes, dtype=torch.uint8, device="cuda") for n, x in b["tables"].items()}
        pools = [torch.empty(caps[c], lay.page[c], dtype=torch.uint8, device="cuda") for c in range(4)]
    for n, x in b["tables"].items():
        regions[n].copy_(torch.from_numpy(np.ascontiguousarray(x).reshape(-1).view(np.uint8)))
        state[n] = regions[n].view(torch.int32).view(x.shape)
    state["pools"] = pools
    rows = rows_of(lay, b["rows"], seed)
    for c in range(4):
        pools[c].zero_()
        pools[c][:len(b["slots"][c])] = page_bytes(lay, c, b["slots"][c], rows[c])
    ints = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    state.update(seq_ids=ints(np.arange(case["seqs"])), starts=ints(starts), offsets=ints(np.append(0, np.cumsum(count))))
    # what a program's own bookkeeping knows without asking the GPU
    state.update(ntok=b["tables"]["ntok"][0].tolist(), first=starts.tolist(), count=count.tolist(), keys=int((starts + count).sum()))
    if case["kind"] == "chunk":
        n = int(count.sum())
        state.update(q=query_rows(case, n, seed), modes=torch.from_numpy(modes_of(case, n, seed)).cuda())
    return state


# -------------------------------------------------------------------------- plain forms --


def read_class(state, s, c):
    """K, V in 32 bits and positions of the tokens of class c of sequence s, in order of position."""
    lay, b, n = state["lay"], BITS[c], state["ntok"][s][c]
    P, hkv = lay.P, lay.hkv
    ids = state["page_table"][0, s, c, :-(-n // P)].long()
    raw = state["pools"][c][ids]
    pos = raw[:, :4 * P].contiguous().view(torch.int32).flatten()[:n].long()
    x = permute_chunks(raw[:, lay.hdr:lay.hdr + hkv * lay.slice[c]].reshape(len(ids), hkv, lay.slice[c]), lay, c)
    found = []
    for which in range(2):
        m = P * lay.row[c]
        codes = x[..., which * m:(which + 1) * m].reshape(len(ids), hkv, P, lay.row[c])
        if b == 16:
            v = codes.contiguous().view(torch.bfloat16).float()
        else:
            per = 8 // b
            v = torch.stack([(codes >> (b * i)) & (2 ** b - 1) for i in range(per)], -1).flatten(-2).float()
            w = 4 * lay.ng * P
            sz = x[..., 2 * m + which * w:2 * m + (which + 1) * w].contiguous().view(torch.float16).view(len(ids), hkv, P, lay.ng, 2).float()
            v = (sz[..., 1:] + v.view(len(ids), hkv, P, lay.ng, lay.gs) * sz[..., :1]).flatten(-2)
        found.append(v.transpose(1, 2).reshape(-1, hkv, lay.d)[:n])
    return found[0], found[1], pos


def plain_chunk(state):
    case, lay, outs, row = state["case"], state["lay"], [], 0
    g = lay.hq // lay.hkv
    for s, (first, count) in enumerate(zip(state["first"], state["count"])):
        k, v, pos = (torch.cat(x) for x in zip(*[read_class(state, s, c) for c in range(4)]))
        q = state["q"][row:row + count].float().view(count, lay.hkv, g, lay.d)
        mode = state["modes"][row:row + count, None]
        t = torch.arange(first, first + count, device="cuda")[:, None]
        seen = (pos <= t) & ((mode == FULL) | ((mode == LOCAL) & ((pos > t - case["window"]) | (pos < case["sinks"]))))
        rows = []
        for h in range(lay.hkv):
            x = (torch.einsum("qrd,td->qrt", q[:, h], k[:, h]) / math.sqrt(lay.d)).masked_fill_(~seen[:, None], -math.inf)
            top = x.amax(-1, keepdim=True) if len(pos) else x.new_full((count, g, 1), -math.inf)
            w = x.sub_(torch.where(top.isfinite(), top, 0.0)).exp_()
            total = w.sum(-1, keepdim=True)
            rows.append(torch.where(total > 0, torch.einsum("qrt,td->qrd", w, v[:, h]) / total, 0.0))
        outs.append(torch.stack(rows, 1).view(count, lay.hq, lay.d).bfloat16())
        row += count
    return torch.cat(outs)


def plain_read(state):
    case, lay = state["case"], state["lay"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    n, row = sum(state["count"]), 0
    k, v = (torch.zeros(n, lay.hkv, lay.d, dtype=dtype, device="cuda") for _ in range(2))
    bits = torch.zeros(n, lay.hkv, dtype=torch.uint8, device="cuda")
    for s, (first, count) in enumerate(zip(state["first"], state["count"])):
        for c, b in enumerate(BITS):
            kc, vc, pos = read_class(state, s, c)
            keep = (pos >= first) & (pos < first + count)
            at = pos[keep] - first + row
            k[at], v[at], bits[at] = kc[keep].to(dtype), vc[keep].to(dtype), b
        row += count
    return {"k": k, "v": v, "bits": bits}


def run(state):
    case = state["case"]
    if not own:
        return plain_chunk(state) if case["kind"] == "chunk" else plain_read(state)
    cache = state["cache"]
    if case["kind"] == "chunk":
        return cache.chunk_attn(0, state["seq_ids"], state["starts"], state["offsets"], state["q"], state["modes"], window_scalar=case["window"],
                                sinks=case["sinks"], max_keys=state["keys"])
    k, v, bits = cache.read(0, state["seq_ids"], state["starts"], state["offsets"], sum(state["count"]),
                            dtype=torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
    return {"k": k, "v": v, "bits": bits}


# ----------------------------------------------------------------------- work and truth --


def token_bytes(case):
    """Bytes of one stored token's K and V for one KV head, scales and zeros among them, over the mix."""
    d, ng = case["d"], case["d"] // case["gs"]
    return sum(p * (2 * d * b // 8 + (8 * ng if b < 16 else 0)) for p, b in zip(MIXES[case["mix"]], BITS))


def work(case):
    """Of the sizes that the case's ranges have on average."""
    per = case["hkv"] * token_bytes(case) + 4  # all heads of a token, and its position
    length = (case["lo"] + case["hi"]) / 2
    if case["kind"] == "read":
        n = case["seqs"] * max(1.0, case["share"] * length)
        return {"bytes": n * (STORED * per + case["hkv"] * (2 * case["d"] * (2 if case["dtype"] == "bf16" else 4) + 1)), "flops": 0}
    new = min((case["new_lo"] + case["new_hi"]) / 2, length)
    skip, near, full = {"routed": ROUTED, "full": (0, 0, 1), "local": (0, 1, 0)}[case["modes"]]
    sight = min(case["window"] + case["sinks"], length - new / 2)     # positions that a local query sees
    reach = length if full * new >= 1 else min(length, new + sight)   # positions that a chunk's queries see between them
    pairs = case["seqs"] * new * STORED * (full * (length - new / 2) + near * sight)
    rows = case["seqs"] * new * case["hq"]
    return {"bytes": case["seqs"] * STORED * reach * per + rows * 2 * (2 - skip) * case["d"], "flops": 4 * case["hq"] * case["d"] * pairs}


def exact(case, seed):
    """From the stored codes and not from pages, in 64 bits: attention query group by query group, values one class at a time."""
    b, lay = build(case, seed), Layout(case)
    made = rows_of(lay, b["rows"], seed)
    starts, count = stretches(case)

    def values(c, which, rows):
        if BITS[c] == 16:
            return made[c][which][rows].double()
        code, scale, zero = (y[rows].double() for y in made[c][which])
        return zero.repeat_interleave(lay.gs, -1) + code * scale.repeat_interleave(lay.gs, -1)

    if case["kind"] == "read":
        ks, vs, bits = [], [], []
        for s in range(case["seqs"]):
            k, v = (torch.zeros(count[s], lay.hkv, lay.d, dtype=torch.float64, device="cuda") for _ in range(2))
            width = torch.zeros(count[s], lay.hkv, dtype=torch.uint8, device="cuda")
            for c in range(4):
                pos, base = b["tokens"][s][c]
                i, j = np.searchsorted(pos, [starts[s], starts[s] + count[s]])
                at = torch.from_numpy(pos[i:j] - starts[s]).cuda()
                k[at], v[at] = (values(c, which, slice(base + i, base + j)) for which in range(2))
                width[at] = BITS[c]
            ks.append(k), vs.append(v), bits.append(width)
        return {"k": torch.cat(ks), "v": torch.cat(vs), "bits": torch.cat(bits)}

    n, g = int(count.sum()), lay.hq // lay.hkv
    q = query_rows(case, n, seed).double()
    modes = modes_of(case, n, seed)
    out = torch.zeros(n, lay.hq, lay.d, dtype=torch.float64, device="cuda")
    row = 0
    for s in range(case["seqs"]):
        pos = torch.from_numpy(np.concatenate([x[0] for x in b["tokens"][s]])).cuda()
        k, v = (torch.cat([values(c, which, slice(x[1], x[1] + len(x[0]))) for c, x in enumerate(b["tokens"][s])]) for which in range(2))
        here = np.arange(count[s])
        for mode, kept in ((FULL, 0), (LOCAL, case["sinks"])):  # queries of one mode, some at a time
            mine = here[modes[row:row + count[s]] == mode]
            for part in np.array_split(mine, max(1, -(-len(mine) * len(pos) // 2 ** 24))):
                if not len(part) or not len(pos):
                    continue
                t = torch.from_numpy(starts[s] + part).cuda()
                since = torch.zeros_like(t) if mode == FULL else t - (case["window"] - 1)
                hidden = (pos[None] > t[:, None]) | ((pos[None] < since[:, None]) & (pos[None] >= kept))
                at = torch.from_numpy(row + part).cuda()
                for h in range(lay.hq):
                    x = q[at, h] @ k[:, h // g].T * lay.d ** -0.5
                    x[hidden] = -math.inf
                    total = torch.logsumexp(x, -1)
                    out[at, h] = torch.exp(x - torch.where(total.isfinite(), total, 0.0)[:, None]) @ v[:, h // g]
        row += int(count[s])
    return out
