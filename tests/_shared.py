"""Helpers of the tests of shared pages: a plain model of the page operations on copies of a
cache's metadata, and attention in 64 bits over the tokens that a sequence holds."""
from __future__ import annotations

import numpy as np
import torch

import oracle
from _parity import dev
from paper_2607_06601_gb300 import trr, workloads as wl

META = ("last_pos", "ntok", "presence", "page_table", "page_first", "page_last", "next_page")
BITS = (2, 4, 8, 16)


class Holder:
    """A GPU cache together with the tokens that each of its sequences should hold.

    `tokens[layer][seq]` maps a position to (an archive sequence of a CPU oracle cache,
    position there): the oracle quantised the same rows, so its values are the truth."""

    def __init__(self, L, S, Hq, Hkv, d, G, P, maxctx, caps, head_modes=0, archive=64, fill=0xFF, max_queries=256):
        self.L, self.S, self.Hq, self.Hkv, self.d, self.P, self.head_modes = L, S, Hq, Hkv, d, P, head_modes
        self.gpu = trr.Cache(L, S, Hq, Hkv, d, G, P, maxctx, caps, max_append=1024, max_queries=max_queries, head_modes=head_modes)
        for b in BITS:  # what no token was written to holds NaN scales and positions of -1
            self.gpu.region(f"pool{b}").fill_(fill)
        need = [archive * L * (-(-maxctx // P) + 1)] * 4
        self.orc = oracle.OracleCache(L, archive, Hq, Hkv, d, G, P, maxctx, need, head_modes=head_modes)
        self.tokens = [[{} for _ in range(S)] for _ in range(L)]
        self.used = 0

    def append(self, rng, layer, seq, positions, mix=(0.25, 0.25, 0.25, 0.25), p_skip=0.2, k=None, v=None, bits=None):
        """Random tokens at `positions`, to the GPU and to a fresh archive sequence."""
        n = len(positions)
        if n == 0:
            return
        pos = np.asarray(positions, np.int32)
        bits = np.asarray(BITS, np.uint8)[rng.choice(4, size=n, p=mix)] if bits is None else np.asarray(bits, np.uint8)
        shape = (n, self.Hq) if self.head_modes else n
        modes = np.where(rng.random(shape) < p_skip, 0, 2).astype(np.uint8)
        rows = [wl.bf16_bits(rng.standard_normal((n, self.Hkv, self.d), dtype=np.float32)) if x is None else x for x in (k, v)]
        self.gpu.append(layer, dev(np.full(n, seq, np.int32), torch.int32), dev(pos, torch.int32), dev(rows[0], torch.bfloat16),
                        dev(rows[1], torch.bfloat16), dev(bits, torch.uint8), dev(modes, torch.uint8))
        assert self.gpu.status() == 0
        assert self.orc.append(layer, np.full(n, self.used, np.int32), pos, rows[0], rows[1], bits, modes) == 0
        stores = modes.reshape(n, -1).max(1) > 0
        for p in pos[stores]:
            self.tokens[layer][seq][int(p)] = (self.used, int(p))
        self.used += 1

    def ints(self, x):
        return dev(np.asarray(x, np.int32), torch.int32)

    def fork(self, src, dst, lengths):
        self.gpu.fork(self.ints(src), self.ints(dst), self.ints(lengths))
        for layer in range(self.L):
            new = [{p: x for p, x in self.tokens[layer][s].items() if p < n} for s, n in zip(src, lengths)]
            for d, x in zip(dst, new):
                self.tokens[layer][d] = x

    def free(self, seqs):
        self.gpu.free(self.ints(seqs))
        for layer in range(self.L):
            for s in seqs:
                self.tokens[layer][s] = {}

    def values(self, layer, seq, head):
        """Positions, K and V (64 bits) of one KV head of what the sequence holds."""
        held = sorted(self.tokens[layer][seq].items())
        kv = [self.orc.dequant_token(layer, a, p, head) for _, (a, p) in held]
        pos = np.array([p for p, _ in held], np.int64)
        return pos, np.array([x[1] for x in kv]).reshape(-1, self.d), np.array([x[2] for x in kv]).reshape(-1, self.d)

    def attend(self, layer, seqs, ts, q_bits, modes, windows, sinks=0, scale=None):
        """The definition: softmax over the tokens in sight, in 64 bits; [n][Hq][d]."""
        q = wl.bf16_to_f32(q_bits).astype(np.float64)
        scale = 1 / np.sqrt(self.d) if scale is None else scale
        out = np.zeros((len(seqs), self.Hq, self.d))
        kept = {}
        for i, (s, t, m, w) in enumerate(zip(seqs, ts, modes, windows)):
            if m == 0:
                continue
            for h in range(self.Hq):
                kvh = h // (self.Hq // self.Hkv)
                if (s, kvh) not in kept:
                    kept[s, kvh] = self.values(layer, s, kvh)
                pos, k, v = kept[s, kvh]
                see = pos <= t
                if m == 1:
                    see &= (pos >= t - w + 1) | (pos < sinks)
                if see.any():
                    x = scale * (k[see] @ q[i, h])
                    p = np.exp(x - x.max())
                    out[i, h] = p @ v[see] / p.sum()
        return out


def snapshot(h: Holder):
    torch.cuda.synchronize()
    m = {n: h.gpu.region(n).cpu().numpy().view(np.uint32 if n == "presence" else np.int32).copy() for n in META}
    L, S = h.L, h.S
    MP = m["page_table"].size // (L * S * 4)
    m["last_pos"] = m["last_pos"].reshape(L, S)
    m["ntok"] = m["ntok"].reshape(L, S, 4)
    m["presence"] = m["presence"].reshape(L, S, -1)
    for n in ("page_table", "page_first", "page_last"):
        m[n] = m[n].reshape(L, S, 4, MP)
    m["pools"] = [h.gpu.region(f"pool{b}").cpu().numpy().reshape(-1, h.orc.page_bytes(c)).copy() for c, b in enumerate(BITS)]
    return m


def same(a, b, what=""):
    for n in META:
        assert np.array_equal(a[n], b[n]), f"{what}: {n} differs at {np.argwhere(a[n] != b[n])[:4].tolist()}"
    for c in range(4):
        bad = np.argwhere(a["pools"][c] != b["pools"][c])
        assert bad.size == 0, f"{what}: pool of {BITS[c]} bits differs at {bad[:4].tolist()}"


def positions_of(m, P, c, page):
    return m["pools"][c][page, :4 * P].copy().view(np.int32)


def model_fork(m, h, src, dst, lengths):
    """trr_fork on a snapshot, entry by entry."""
    P, old = h.P, {n: m[n].copy() for n in META}
    for layer in range(h.L):
        for s, d, length in zip(src, dst, lengths):
            for c in range(4):
                nt = int(old["ntok"][layer, s, c])
                lists = {n: [] for n in ("page_table", "page_first", "page_last")}
                count = 0
                for k in range(-(-nt // P)):
                    page = int(old["page_table"][layer, s, c, k])
                    pos = positions_of(m, P, c, page)[:min(P, nt - k * P)]
                    keep = pos[pos < length]
                    if keep.size == 0:
                        break
                    if keep.size < P:
                        new = int(m["next_page"][c])
                        m["next_page"][c] += 1
                        m["pools"][c][new] = m["pools"][c][page]
                        if h.head_modes:
                            for j in range(h.Hkv):
                                at = h.orc.hdr_bytes + (j + 1) * h.orc.slice_bytes(c) - 16
                                w = m["pools"][c][new, at:at + 8].view(np.uint64)
                                w &= np.uint64((1 << keep.size) - 1)
                        page = new
                    lists["page_table"].append(page)
                    lists["page_first"].append(int(keep[0]))
                    lists["page_last"].append(int(keep[-1]))
                    count += keep.size
                for n, x in lists.items():
                    m[n][layer, d, c] = -1
                    m[n][layer, d, c, :len(x)] = x
                m["ntok"][layer, d, c] = count
            bits = np.unpackbits(old["presence"][layer, s].view(np.uint8), bitorder="little")
            bits[max(0, length):] = 0
            m["presence"][layer, d] = np.packbits(bits, bitorder="little").view(np.uint32)
            m["last_pos"][layer, d] = min(int(old["last_pos"][layer, s]), length - 1)


def model_evict(m, h, seqs, keep_from, sinks):
    """trr_evict on a snapshot; returns the forgotten positions of every (layer, sequence)."""
    P, gone = h.P, {}
    for layer in range(h.L):
        for s, lo in zip(seqs, keep_from):
            for c in range(4):
                nt = int(m["ntok"][layer, s, c])
                np_ = -(-nt // P)
                keep = []
                for k in range(np_):
                    pos = positions_of(m, P, c, int(m["page_table"][layer, s, c, k]))[:min(P, nt - k * P)]
                    if pos.size == P and pos.min() >= sinks and pos.max() < lo:
                        gone.setdefault((layer, s), []).extend(pos.tolist())
                        for p in pos:
                            m["presence"][layer, s, p // 32] &= ~np.uint32(1 << (p % 32))
                    else:
                        keep.append(k)
                for n in ("page_table", "page_first", "page_last"):
                    x = m[n][layer, s, c, keep].copy()
                    m[n][layer, s, c, :np_] = -1
                    m[n][layer, s, c, :len(keep)] = x
                m["ntok"][layer, s, c] = nt - P * (np_ - len(keep))
    return gone


def model_free(m, seqs):
    for s in seqs:
        m["last_pos"][:, s] = -1
        m["ntok"][:, s] = 0
        m["presence"][:, s] = 0
        for n in ("page_table", "page_first", "page_last"):
            m[n][:, s] = -1


def model_compact(m, h):
    for c in range(4):
        rows = [(layer, s, k) for layer in range(h.L) for s in range(h.S) for k in range(-(-int(m["ntok"][layer, s, c]) // h.P))]
        used = {int(m["page_table"][layer, s, c, k]) for layer, s, k in rows}
        n = len(used)
        holes, movers = sorted(set(range(n)) - used), sorted(p for p in used if p >= n)
        to = dict(zip(movers, holes))
        for a, b in to.items():
            m["pools"][c][b] = m["pools"][c][a]
        for layer, s, k in rows:
            page = int(m["page_table"][layer, s, c, k])
            m["page_table"][layer, s, c, k] = to.get(page, page)
        m["next_page"][c] = n
