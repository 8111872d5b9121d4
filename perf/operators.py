"""Operators on a mixed-precision paged KV cache that sequences share, as cases to be run and timed.

Three kinds of case:

  shared  one decode step's attention for a batch whose sequences were forked from a few long
          prompts: the pages that a group of sequences has in common are read once for the group
          (Cache.decode_attn_shared)
  sinks   decode attention of queries that see a sliding window and the first few tokens
          (Cache.decode_attn_sinks)
  pages   one turn of a beam search over forked sequences: Cache.fork, Cache.evict, Cache.free and
          Cache.compact on the page tables and pages of every layer

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
        # two continuations of one short prompt: the smallest call, all latency
        dict(name="shared-tiny", kind="shared", groups=1, members=2, prefix=64, suffix=8, hq=4, hkv=2, d=64, gs=32, page=16,
             mix="even", routed=False, window=32, sinks=0),
        # a batch of 32 samples of one system prompt, small decoder with a KV head per query head
        dict(name="shared-160m", kind="shared", groups=1, members=32, prefix=2048, suffix=64, hq=12, hkv=12, d=64, gs=32, page=32,
             mix="decoder", routed=False, window=256, sinks=0),
        # several prompts, odd sizes, routed modes: local queries keep a window and the sinks, skip queries read nothing
        dict(name="shared-routed-odd", kind="shared", groups=7, members=9, prefix=4099, suffix=131, hq=32, hkv=32, d=64, gs=32, page=32,
             mix="ragged", routed=True, window=256, sinks=4),
        # 16 answers to one long document, query groups of 4
        dict(name="shared-gqa-long", kind="shared", groups=1, members=16, prefix=32768, suffix=256, hq=32, hkv=8, d=128, gs=64, page=32,
             mix="long", routed=False, window=1024, sinks=0),
        # many samples of one long document: products with 256 rows for a KV head
        dict(name="shared-gqa-wide", kind="shared", groups=1, members=64, prefix=32768, suffix=256, hq=32, hkv=8, d=128, gs=64, page=64,
             mix="long", routed=False, window=1024, sinks=0),
        # one streaming sequence just past its window
        dict(name="sinks-tiny", kind="sinks", seqs=1, lo=130, hi=130, window=32, sinks=4, hq=4, hkv=2, d=64, gs=32, page=16, mix="even"),
        # a batch of streaming sequences of the small decoder
        dict(name="sinks-160m", kind="sinks", seqs=32, lo=2048, hi=2048, window=256, sinks=4, hq=12, hkv=12, d=64, gs=32, page=32,
             mix="decoder"),
        # ragged contexts, a KV head per query head, an odd window
        dict(name="sinks-1p3b-ragged", kind="sinks", seqs=64, lo=1024, hi=8192, window=511, sinks=16, hq=32, hkv=32, d=64, gs=32, page=32,
             mix="ragged"),
        # a large batch with query groups, wide window, many sinks
        dict(name="sinks-gqa-wide", kind="sinks", seqs=128, lo=4096, hi=8192, window=1024, sinks=64, hq=32, hkv=8, d=128, gs=64, page=32,
             mix="long"),
        # two beams of one short sequence
        dict(name="pages-tiny", kind="pages", layers=1, parents=1, children=2, prefix=130, hkv=2, d=64, gs=32, page=16, mix="even",
             window=32, sinks=4),
        # 32 beams over 4 prompts, every layer of the small decoder
        dict(name="pages-160m", kind="pages", layers=12, parents=4, children=32, prefix=2048, hkv=12, d=64, gs=32, page=32, mix="decoder",
             window=256, sinks=4),
        # the same over 24 layers of 32 KV heads, longer prompts: page copies dominate
        dict(name="pages-24-layers", kind="pages", layers=24, parents=4, children=32, prefix=4096, hkv=32, d=64, gs=32, page=32, mix="decoder",
             window=256, sinks=4),
    ]


def draw(rng):
    def spread(lo, hi):  # whole numbers spread over their logarithm
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["shared", "shared", "sinks", "sinks", "pages"])
    hq, hkv, d, gs = rng.choice([(12, 12, 64, 32), (32, 32, 64, 32), (32, 8, 128, 64), (4, 2, 64, 32), (12, 4, 64, 64), (8, 2, 128, 32), (16, 2, 64, 64)])
    page, mix = rng.choice([16, 32, 64]), rng.choice(sorted(MIXES))
    if kind == "shared":
        groups, members = spread(1, 8), spread(1, 48)
        prefix = spread(40, max(41, min(32768, 1_000_000 // (groups * members + 8), 200_000_000 // (groups * hkv * d * 8))))
        return dict(kind=kind, groups=groups, members=members, prefix=prefix, suffix=spread(1, 256), hq=hq, hkv=hkv, d=d, gs=gs, page=page,
                    mix=mix, routed=rng.random() < 0.5, window=spread(1, 1024), sinks=rng.choice([0, 1, 4, 64]))
    if kind == "sinks":
        seqs, hi = spread(1, 96), spread(60, 8192)
        hi = min(hi, max(60, 64 * 8192 * 32 // (seqs * hkv * d // 64)))
        return dict(kind=kind, seqs=seqs, lo=max(1, hi // rng.choice([1, 2, 8])), hi=hi, window=spread(1, 1024), sinks=rng.choice([0, 1, 4, 16, 64, 100]),
                    hq=hq, hkv=hkv, d=d, gs=gs, page=page, mix=mix)
    layers, parents = spread(1, 12), spread(1, 4)
    return dict(kind=kind, layers=layers, parents=parents, children=spread(1, 32), prefix=spread(40, 2048), hkv=min(hkv, 12), d=d, gs=gs, page=page,
                mix=mix, window=spread(1, 512), sinks=rng.choice([0, 1, 4, 64]))


# ------------------------------------------------------------------------------ inputs --


def up(x, a):
    return -(-x // a) * a


class Layout:
    """Sizes of the documented page layout for one case."""

    def __init__(self, case, hq):
        self.hq, self.hkv, self.d, self.gs, self.P = hq, case["hkv"], case["d"], case["gs"], case["page"]
        self.ng = self.d // self.gs
        g = self.hq // self.hkv
        self.permuted = not (g >= 2 and g * self.ng <= 8)  # 8- and 16-bit rows keep each line's chunks in a permuted order
        self.hdr = up(4 * self.P, 128)
        self.row = [self.d * b // 8 for b in BITS]         # bytes of one K or V row
        self.slice = [self.P * (2 * self.row[c] + (2 * self.ng * 4 if c < 3 else 0)) for c in range(4)]
        self.page = [up(self.hdr + self.hkv * s, 128) for s in self.slice]


def paged(lists, P, pages):
    """Tables of new pages for one (sequence, class): positions and contents cut into pages of P."""
    pos, con = lists
    k = -(-len(pos) // P)
    first, fill = len(pages), np.full((2, k * P), -1, np.int64)
    fill[0, :len(pos)], fill[1, :len(pos)] = pos, con
    pages += list(fill.reshape(2, k, P).swapaxes(0, 1))
    return list(range(first, first + k))


def build(case, seed):
    """Page tables of the case, and what each slot holds: `content` indexes that class's K and V rows."""
    r = np.random.default_rng([seed, 1])
    P, mix = case["page"], MIXES[case["mix"]]
    layers = case.get("layers", 1)
    if case["kind"] == "shared":
        groups, members = case["groups"], case["members"]
        lens = [case["prefix"]] * groups + list(case["prefix"] + r.integers(max(1, case["suffix"] // 2), case["suffix"] + 1, groups * members))
        parent = [-1] * groups + [i // members for i in range(groups * members)]
    elif case["kind"] == "sinks":
        lens = list(r.integers(case["lo"], case["hi"] + 1, case["seqs"]))
        parent = [-1] * case["seqs"]
    else:
        lens = [case["prefix"]] * case["parents"] + [0] * (2 * case["children"])
        parent = [-1] * len(lens)
    S, most = len(lens), int(max(lens)) + 1
    MP, W32 = -(-most // P), -(-most // 32)
    t = dict(last_pos=np.full((layers, S), -1, np.int32), ntok=np.zeros((layers, S, 4), np.int32), presence=np.zeros((layers, S, W32), np.uint32))
    t.update({n: np.full((layers, S, 4, MP), -1, np.int32) for n in ("page_table", "page_first", "page_last")})
    pages, contents = [[] for _ in BITS], [0] * 4
    tokens = {}  # (layer, sequence): (positions, contents) by class
    for layer in range(layers):
        for s in range(S):
            n, start = int(lens[s]), 0
            if n == 0:
                continue
            base = tokens.get((layer, parent[s])) if parent[s] >= 0 else None
            start = int(lens[parent[s]]) if base else 0
            cls = r.choice(4, size=n - start, p=mix)
            at = np.arange(start, n)
            has = r.random(n - start) < STORED
            mine = []
            for c in range(4):
                pos = at[has & (cls == c)]
                con = contents[c] + np.arange(len(pos))
                contents[c] += len(pos)
                ids = []
                if base:
                    keep = len(base[c][0]) // P  # full pages are the parent's own, a partly filled one is copied
                    ids = list(t["page_table"][layer, parent[s], c, :keep])
                    pos, con = np.concatenate([base[c][0], pos]), np.concatenate([base[c][1], con])
                    ids += paged((pos[keep * P:], con[keep * P:]), P, pages[c])
                else:
                    ids = paged((pos, con), P, pages[c])
                t["page_table"][layer, s, c, :len(ids)] = ids
                t["page_first"][layer, s, c, :len(ids)] = pos[::P]
                t["page_last"][layer, s, c, :len(ids)] = np.append(pos[P - 1::P], pos[len(pos) - 1:])[:len(ids)] if len(pos) % P else pos[P - 1::P]
                t["ntok"][layer, s, c] = len(pos)
                np.bitwise_or.at(t["presence"][layer, s], pos // 32, np.uint32(1) << (pos % 32).astype(np.uint32))
                mine.append((pos, con))
            tokens[layer, s] = mine
            t["last_pos"][layer, s] = n - 1
    t["next_page"] = np.array([len(p) for p in pages], np.int32)
    slots = [np.array(p, np.int64).reshape(-1, 2, P) for p in pages]
    return dict(tables=t, slots=slots, contents=contents, tokens=tokens, lens=lens, parent=parent, S=S, most=most, MP=MP, rng=r)


def rows_of(case, lay, counts, seed):
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


def chunk_order(lines):
    return torch.arange(8, device="cuda")[None, :] ^ (torch.arange(lines, device="cuda") % 8)[:, None]


def permute_chunks(x, lay, c):
    """[.., slice bytes] with the 16-byte chunks of each 128-byte line of the code rows in the stored order, or back."""
    if not (lay.permuted and c >= 2):
        return x
    n = 2 * lay.P * lay.row[c]
    at = (chunk_order(n // 128) + 8 * torch.arange(n // 128, device="cuda")[:, None]).flatten()
    lead = x.shape[:-1]
    codes = x[..., :n].reshape(*lead, n // 16, 16)[..., at, :].reshape(*lead, n)
    return torch.cat([codes, x[..., n:]], -1)


def page_bytes(lay, c, slots, rows):
    """[pages, page bytes] of one class: slot positions, then each KV head's slice."""
    pos = torch.from_numpy(slots[:, 0].astype(np.int32)).cuda().clamp_min(0)
    at = torch.from_numpy(slots[:, 1]).cuda().clamp_min(0)  # a slot that holds nothing keeps some other token's bytes
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


def queries_of(case, b, seed):
    """Sequences, positions and modes of the call's queries, one for each sequence that decodes."""
    r = np.random.default_rng([seed, 2])
    seqs = np.arange(case["groups"], b["S"]) if case["kind"] == "shared" else np.arange(b["S"])
    pos = np.array([int(b["lens"][s]) - 1 for s in seqs])
    if case["kind"] == "sinks":
        modes = np.where(r.random(len(seqs)) < ROUTED[0], SKIP, LOCAL)
        modes[0] = LOCAL  # a call has some work
    else:
        modes = r.choice(3, size=len(seqs), p=ROUTED) if case["routed"] else np.full(len(seqs), FULL)
        modes[0] = FULL
    return seqs, pos, modes


def query_rows(case, n, seed):
    g = torch.Generator("cuda").manual_seed(seed + 7)
    return torch.randn(n, case["hq"], case["d"], generator=g, device="cuda").bfloat16()


def prepare(case, seed):
    b = build(case, seed)
    hq = case.get("hq", case["hkv"])
    lay = Layout(case, hq)
    caps = [int(n) + 1 for n in b["tables"]["next_page"]]
    if case["kind"] == "pages":  # the pools are outputs: their sizes go by the case alone
        lists = case["layers"] * case["parents"]
        held = [lists * case["prefix"] * STORED * p for p in MIXES[case["mix"]]]
        caps = [int((x + 6 * math.sqrt(x)) / lay.P) + lists + 2 * case["layers"] * case["children"] for x in held]
    state = dict(case=case, lay=lay, MP=b["MP"], S=b["S"], caps=caps)
    if own:
        from paper_2607_06601_gb300 import trr
        state["cache"] = cache = trr.Cache(case.get("layers", 1), b["S"], hq, lay.hkv, lay.d, lay.gs, lay.P, b["most"], caps, max_append=64,
                                           max_queries=max(16, b["S"]))
        regions = {n: cache.region(n) for n in b["tables"]}
        pools = [cache.region("pool%d" % x).view(caps[c], lay.page[c]) for c, x in enumerate(BITS)]
    else:
        regions = {n: torch.empty(x.nbytes, dtype=torch.uint8, device="cuda") for n, x in b["tables"].items()}
        pools = [torch.empty(caps[c], lay.page[c], dtype=torch.uint8, device="cuda") for c in range(4)]
    for n, x in b["tables"].items():
        regions[n].copy_(torch.from_numpy(x.reshape(-1).view(np.uint8)))
        state[n] = regions[n].view(torch.int32).view(x.shape)
    state["pools"] = pools
    if case["kind"] == "pages":
        # the values of K and V play no part in moving pages: any bytes, under the slots' true positions
        g = torch.Generator("cuda").manual_seed(seed)
        for c in range(4):
            words = pools[c].view(torch.int32)
            words.copy_(torch.randint(-2 ** 31, 2 ** 31, words.shape, generator=g, device="cuda", dtype=torch.int32))
            n = len(b["slots"][c])
            words[:n, :lay.P] = torch.from_numpy(b["slots"][c][:, 0].astype(np.int32)).cuda().clamp_min(0)
        r, kids = np.random.default_rng([seed, 3]), case["children"]
        lengths = r.integers(max(1, case["prefix"] // 2), case["prefix"] + 1, kids)
        ints = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
        state.update(parents=ints(r.integers(0, case["parents"], kids)), lengths=ints(lengths), keep_from=ints(np.maximum(0, lengths - case["window"])),
                     bank_a=ints(case["parents"] + np.arange(kids)), bank_b=ints(case["parents"] + kids + np.arange(kids)))
        return state
    rows = rows_of(case, lay, b["contents"], seed)
    for c in range(4):
        pools[c].zero_()
        pools[c][:len(b["slots"][c])] = page_bytes(lay, c, b["slots"][c], rows[c])
    seqs, pos, modes = queries_of(case, b, seed)
    state.update(seq_ids=torch.from_numpy(seqs.astype(np.int32)).cuda(), q_positions=torch.from_numpy(pos.astype(np.int32)).cuda(),
                 modes=torch.from_numpy(modes.astype(np.uint8)).cuda(), q=query_rows(case, len(seqs), seed))
    pt, ntok = b["tables"]["page_table"][0], b["tables"]["ntok"][0]
    if case["kind"] == "shared":
        shared = ntok[:case["groups"]] // lay.P
        state["group_offsets"] = torch.arange(0, len(seqs) + 1, case["members"], dtype=torch.int32, device="cuda")
        # widths of the gathers of the plain form: most shared pages of a group, most pages of a sequence past them
        state["wide"] = [int(x) for x in shared.max(0)]
        state["wide_own"] = [int(x) for x in (-(-ntok[seqs] // lay.P) - shared[[b["parent"][s] for s in seqs]]).max(0)]
    else:
        first, last = b["tables"]["page_first"][0], b["tables"]["page_last"][0]
        there = pt >= 0
        state["wide"] = [int(x) for x in (there & (first < case["sinks"])).sum(-1).max(0)]
        state["wide_own"] = [int(x) for x in (there & (last >= (pos - case["window"] + 1)[:, None, None])).sum(-1).max(0)]
    return state


# -------------------------------------------------------------------------- plain forms --


def read_pages(state, c, ids):
    """K, V in 32 bits and slot positions of the pages `ids` [.., pages]: [.., pages * P, Hkv, d] and [.., pages * P]."""
    lay, b = state["lay"], BITS[c]
    lead, P, hkv = ids.shape[:-1], lay.P, lay.hkv
    raw = state["pools"][c][ids.long().clamp_min(0)]
    pos = raw[..., :4 * P].contiguous().view(torch.int32).flatten(-2)
    x = permute_chunks(raw[..., lay.hdr:lay.hdr + hkv * lay.slice[c]].reshape(*ids.shape, hkv, lay.slice[c]), lay, c)
    found = []
    for which in range(2):
        n = P * lay.row[c]
        codes = x[..., which * n:(which + 1) * n].reshape(*ids.shape, hkv, P, lay.row[c])
        if b == 16:
            v = codes.contiguous().view(torch.bfloat16).float()
        else:
            per = 8 // b
            v = torch.stack([(codes >> (b * i)) & (2 ** b - 1) for i in range(per)], -1).flatten(-2).float()
            m = 4 * lay.ng * P
            sz = x[..., 2 * n + which * m:2 * n + (which + 1) * m].contiguous().view(torch.float16).view(*ids.shape, hkv, P, lay.ng, 2).float()
            v = (sz[..., 1:] + v.view(*v.shape[:-1], lay.ng, lay.gs) * sz[..., :1]).flatten(-2)
        found.append(v.transpose(-3, -2).reshape(*lead, -1, hkv, lay.d))
    return found[0], found[1], pos


def gather(state, tables, counts, index, good):
    """K, V, slot positions and which slots count, over all classes; tables [r, 4, MP], counts [r, 4], index and good per class [r, pages]."""
    P, parts = state["lay"].P, []
    for c in range(4):
        ids = tables[:, c].gather(1, index[c].clamp(0, state["MP"] - 1))
        k, v, pos = read_pages(state, c, ids)
        slot = index[c][..., None] * P + torch.arange(P, device="cuda")
        parts.append((k, v, pos, ((slot < counts[:, c, None, None]) & good[c][..., None]).flatten(1)))
    return [torch.cat(x, 1) for x in zip(*parts)]


def in_sight(state, pos, t, modes):
    """Which stored positions [.., tokens] the queries at t with these modes see."""
    case = state["case"]
    near = (pos > t - case["window"]) | (pos < case["sinks"])
    return (pos <= t) & ((modes == FULL) | ((modes == LOCAL) & near))


def softmax_parts(scores, seen):
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    w = torch.exp(scores - torch.where(top.isfinite(), top, 0.0))
    total = w.sum(-1, keepdim=True)
    return torch.where(total > 0, w / total, 0.0)


def plain_shared(state):
    case, lay = state["case"], state["lay"]
    groups, members, g = case["groups"], case["members"], lay.hq // lay.hkv
    seq, t, modes = state["seq_ids"].long(), state["q_positions"], state["modes"]
    n = len(seq)
    tables, counts = state["page_table"][0, seq], state["ntok"][0, seq]
    lead = tables.view(groups, members, 4, -1)[:, :1]
    same = ((tables.view(groups, members, 4, -1) == lead) & (lead >= 0)).long().cumprod(-1).sum(-1)  # pages in common with the group's first
    common = torch.minimum(same.amin(1), torch.tensor(state["wide"], device="cuda"))
    q = state["q"].float().view(groups, members, lay.hkv, g, lay.d) / math.sqrt(lay.d)
    steps = [torch.arange(w, device="cuda").expand(groups, w) for w in state["wide"]]
    k, v, pos, good = gather(state, tables.view(groups, members, 4, -1)[:, 0], counts.view(groups, members, 4)[:, 0], steps,
                             [s < common[:, c, None] for c, s in enumerate(steps)])
    seen = good[:, None] & in_sight(state, pos[:, None], t.view(groups, members, 1), modes.view(groups, members, 1))
    scores = torch.einsum("gmhrd,gthd->gmhrt", q, k).reshape(n, lay.hkv, g, -1)
    start = common.repeat_interleave(members, 0)
    steps = [start[:, c, None] + torch.arange(w, device="cuda") for c, w in enumerate(state["wide_own"])]
    k2, v2, pos2, good2 = gather(state, tables, counts, steps, [torch.ones_like(s, dtype=torch.bool) for s in steps])
    seen2 = good2 & in_sight(state, pos2, t[:, None], modes[:, None])
    scores2 = torch.einsum("nhrd,nthd->nhrt", q.flatten(0, 1), k2)
    w = softmax_parts(torch.cat([scores, scores2], -1), torch.cat([seen.flatten(0, 1), seen2], -1)[:, None, None])
    cut = scores.shape[-1]
    out = torch.einsum("gmhrt,gthd->gmhrd", w[..., :cut].reshape(groups, members, lay.hkv, g, -1), v).flatten(0, 1)
    return (out + torch.einsum("nhrt,nthd->nhrd", w[..., cut:], v2)).reshape(n, lay.hq, lay.d).bfloat16()


def plain_sinks(state):
    case, lay = state["case"], state["lay"]
    seq, t, modes = state["seq_ids"].long(), state["q_positions"], state["modes"]
    tables, counts = state["page_table"][0, seq], state["ntok"][0, seq]
    first, last = state["page_first"][0, seq], state["page_last"][0, seq]
    index, good = [], []
    for c in range(4):
        there = tables[:, c] >= 0
        head = (there & (first[:, c] < case["sinks"])).sum(-1, keepdim=True)
        near = torch.maximum(head, (there & (last[:, c] <= t[:, None] - case["window"])).sum(-1, keepdim=True))
        a = torch.arange(state["wide"][c], device="cuda").expand(len(seq), -1)
        index.append(torch.cat([a, near + torch.arange(state["wide_own"][c], device="cuda")], 1))
        good.append(torch.cat([a < head, torch.ones(len(seq), state["wide_own"][c], dtype=torch.bool, device="cuda")], 1))
    k, v, pos, there = gather(state, tables, counts, index, good)
    q = state["q"].float().view(len(seq), lay.hkv, -1, lay.d) / math.sqrt(lay.d)
    w = softmax_parts(torch.einsum("nhrd,nthd->nhrt", q, k), (there & in_sight(state, pos, t[:, None], modes[:, None]))[:, None, None])
    return torch.einsum("nhrt,nthd->nhrd", w, v).reshape(len(seq), lay.hq, lay.d).bfloat16()


def plain_free(state, seqs):
    seqs = seqs.long()
    state["last_pos"][:, seqs] = -1
    state["ntok"][:, seqs] = 0
    state["presence"][:, seqs] = 0
    for name in ("page_table", "page_first", "page_last"):
        state[name][:, seqs] = -1


def plain_fork(state, src, dst, lengths):
    P, src, dst, length = state["lay"].P, src.long(), dst.long(), lengths.long()
    at = torch.arange(state["MP"], device="cuda")
    for c in range(4):
        pt, pf, pl = (state[n][:, src, c].clone() for n in ("page_table", "page_first", "page_last"))
        ntok = state["ntok"][:, src, c].long()
        take = ((at < -(-ntok // P)[..., None]) & (pf < length[:, None])).sum(-1)
        end = (take - 1).clamp_min(0)[..., None]
        page = pt.gather(-1, end).squeeze(-1)
        words = state["pools"][c].view(torch.int32)
        pos = words[page.long().clamp_min(0), :P]
        held = (end * P + torch.arange(P, device="cuda") < ntok[..., None]) & (pos < length[:, None]) & (take[..., None] > 0)
        kept = held.sum(-1)
        part = (take > 0) & (kept < P)
        rank = part.flatten().long().cumsum(0).view(part.shape)
        new = torch.where(part, state["next_page"][c] + rank - 1, page).int()
        state["next_page"][c] += part.sum().int()
        words[new[part].long()] = words[page[part].long()]
        pt.scatter_(-1, end, new[..., None])
        pl.scatter_(-1, end, torch.where(part, torch.where(held, pos, -1).amax(-1), pl.gather(-1, end).squeeze(-1))[..., None])
        gone = at >= take[..., None]
        for name, x in (("page_table", pt), ("page_first", pf), ("page_last", pl)):
            state[name][:, dst, c] = x.masked_fill(gone, -1)
        state["ntok"][:, dst, c] = torch.where(take > 0, (take - 1) * P + kept, 0).int()
    left = (length[:, None] - 32 * torch.arange(state["presence"].shape[-1], device="cuda")).clamp(0, 32)
    state["presence"][:, dst] = (state["presence"][:, src].long() & ((1 << left) - 1)).int()
    state["last_pos"][:, dst] = torch.minimum(state["last_pos"][:, src], (length - 1).int())


def plain_evict(state, seqs, keep_from, sinks):
    P, seqs = state["lay"].P, seqs.long()
    at = torch.arange(state["MP"], device="cuda")
    gone_bits = torch.zeros_like(state["presence"][:, seqs], dtype=torch.int64)
    for c in range(4):
        pt, pf, pl = (state[n][:, seqs, c] for n in ("page_table", "page_first", "page_last"))
        ntok = state["ntok"][:, seqs, c].long()
        gone = ((at + 1) * P <= ntok[..., None]) & (pf >= sinks) & (pl < keep_from[:, None])
        pos = state["pools"][c].view(torch.int32)[pt.long().clamp_min(0), :P].long().masked_fill(~gone[..., None], 0).flatten(-2)
        gone_bits.scatter_add_(-1, pos // 32, (1 << (pos % 32)) * gone.repeat_interleave(P, -1).long())
        there = at < -(-ntok // P)[..., None]
        order = torch.sort((gone | ~there).int(), dim=-1, stable=True).indices
        left = (there & ~gone).sum(-1, keepdim=True)
        for name, x in (("page_table", pt), ("page_first", pf), ("page_last", pl)):
            state[name][:, seqs, c] = x.gather(-1, order).masked_fill(at >= left, -1)
        state["ntok"][:, seqs, c] = (ntok - P * gone.sum(-1)).int()
    state["presence"][:, seqs] = (state["presence"][:, seqs].long() & ~gone_bits).int()


def plain_compact(state):
    P, at = state["lay"].P, torch.arange(state["MP"], device="cuda")
    for c in range(4):
        pt = state["page_table"][:, :, c]
        there = at < -(-state["ntok"][:, :, c].long() // P)[..., None]
        live = torch.zeros(state["caps"][c], dtype=torch.bool, device="cuda")
        live[pt[there].long()] = True
        count = live.sum()
        at_page = torch.arange(state["caps"][c], device="cuda")
        holes, movers = torch.nonzero(~live & (at_page < count)).flatten(), torch.nonzero(live & (at_page >= count)).flatten()
        to = at_page.int()
        to[movers] = holes.int()
        state["pools"][c].view(torch.int32)[holes] = state["pools"][c].view(torch.int32)[movers]
        state["page_table"][:, :, c] = torch.where(there, to[pt.long().clamp_min(0)], pt)
        state["next_page"][c] = count.int()


def run(state):
    case = state["case"]
    if case["kind"] == "shared":
        if own:
            return state["cache"].decode_attn_shared(0, state["seq_ids"], state["q_positions"], state["q"], state["modes"], state["group_offsets"],
                                                     window_scalar=case["window"], sinks=case["sinks"])
        return plain_shared(state)
    if case["kind"] == "sinks":
        if own:
            return state["cache"].decode_attn_sinks(0, state["seq_ids"], state["q_positions"], state["q"], state["modes"], case["sinks"],
                                                    window_scalar=case["window"])
        return plain_sinks(state)
    # bank B takes the parents' beams and forgets the middle of their past, bank A goes; then A takes B's and B goes: the state after a
    # pass is the one before it
    a, b = state["bank_a"], state["bank_b"]
    if own:
        cache = state["cache"]
        cache.fork(state["parents"], b, state["lengths"])
        cache.evict(b, state["keep_from"], case["sinks"])
        cache.free(a)
        cache.compact()
        cache.fork(b, a, state["lengths"])
        cache.free(b)
        cache.compact()
    else:
        plain_fork(state, state["parents"], b, state["lengths"])
        plain_evict(state, b, state["keep_from"], case["sinks"])
        plain_free(state, a)
        plain_compact(state)
        plain_fork(state, b, a, state["lengths"])
        plain_free(state, b)
        plain_compact(state)
    names = ("last_pos", "ntok", "presence", "page_table", "page_first", "page_last", "next_page")
    return {**{n: state[n] for n in names}, "pages": [p.view(torch.int32) for p in state["pools"]]}


# ----------------------------------------------------------------------- work and truth --


def token_bytes(case):
    """Bytes of one stored token's K and V for one KV head, scales and zeros among them, over the mix."""
    d, ng = case["d"], case["d"] // case["gs"]
    return sum(p * (2 * d * b // 8 + (8 * ng if b < 16 else 0)) for p, b in zip(MIXES[case["mix"]], BITS))


def work(case):
    per = case["hkv"] * token_bytes(case) + 4  # all heads of a token, and its position
    if case["kind"] == "pages":
        lay = Layout(case, case["hkv"])
        pages = case["layers"] * case["children"] * sum(lay.page[c] for c in range(4) if MIXES[case["mix"]][c] > 0)
        length = 0.75 * case["prefix"]
        rows = case["layers"] * case["children"] * (STORED * length / case["page"] * 12 + length / 8 + 20)
        # two forks copy each child's partly filled pages, two compactions move them; tables are read and written by the forks, the eviction
        # and the release
        return {"bytes": 4 * 2 * pages + 6 * rows, "flops": 0}
    row = 2 * case["hq"] * case["d"] * 2  # a query's row and its output
    key = 4 * case["hq"] * case["d"]      # both products, all query heads
    if case["kind"] == "sinks":
        n = case["seqs"] * ((1 - ROUTED[0]) if case["seqs"] > 1 else 1)
        ctx = (case["lo"] + case["hi"]) / 2
        keys = STORED * min(ctx, case["window"] + case["sinks"])
        return {"bytes": n * keys * per + case["seqs"] * row, "flops": n * keys * key}
    n, tail = case["groups"] * case["members"], 0.75 * case["suffix"] + 0.5
    full = n * ROUTED[2] if case["routed"] else n
    near = n * ROUTED[1] * STORED * min(case["prefix"] + tail, case["window"] + case["sinks"]) if case["routed"] else 0.0
    return {"bytes": (STORED * (case["groups"] * min(1.0, full) * case["prefix"] + full * tail) + near) * per + n * row,
            "flops": (STORED * full * (case["prefix"] + tail) + near) * key}


def exact(case, seed):
    """Attention of each query over the tokens that it sees, in 64 bits, from the stored codes and not from pages."""
    if case["kind"] == "pages":
        return None  # whole numbers: the plain form says what they are
    b = build(case, seed)
    lay = Layout(case, case["hq"])
    rows = rows_of(case, lay, b["contents"], seed)
    seqs, ts, modes = queries_of(case, b, seed)
    q = query_rows(case, len(seqs), seed).double()
    out = torch.zeros_like(q)
    for i, (s, t, mode) in enumerate(zip(seqs, ts, modes)):
        ks, vs = [], []
        for c in range(4):
            pos, con = b["tokens"][0, int(s)][c]
            see = pos <= t
            if mode == LOCAL:
                see = see & ((pos >= t - case["window"] + 1) | (pos < case["sinks"]))
            con = torch.from_numpy(con[see & (mode != SKIP)]).cuda()
            for which, to in ((0, ks), (1, vs)):
                x = rows[c][which]
                if BITS[c] < 16:
                    code, scale, zero = (y[con].double() for y in x)
                    to.append(zero.repeat_interleave(lay.gs, -1) + code * scale.repeat_interleave(lay.gs, -1))
                else:
                    to.append(x[con].double())
        k, v = torch.cat(ks).repeat_interleave(lay.hq // lay.hkv, 1), torch.cat(vs).repeat_interleave(lay.hq // lay.hkv, 1)
        if len(k):
            out[i] = torch.einsum("ht,thd->hd", torch.softmax(torch.einsum("hd,thd->ht", q[i], k) / math.sqrt(lay.d), -1), v)
    return out
