"""Several samples of one prompt, then one of them streamed past its window.

    python examples/shared_prompt.py [--layers L] [--samples N] [--prompt T] [--steps K]

One prompt is stored once and forked into samples that share its pages.  Each step appends a
token to every sample and attends with all of them at once, the prompt's pages read once for the
group.  Every few steps the better half of the samples goes on in two copies each (a beam
search): forks into the other bank of sequences, the old bank freed, the pages compacted.  Then
the first sample streams on alone: its local queries keep the first tokens (sinks) in sight, and
what neither they nor the window reads is evicted, so that its pages stop growing in number.

Rows and scores are random numbers in place of a model's.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_06601_gb300 import trr  # noqa: E402

BITS = torch.tensor([2, 4, 8, 16], dtype=torch.uint8)


class Model:
    """Stands for a decoder: K, V and Q rows of new tokens, their widths and modes."""

    def __init__(self, cache, seed=0):
        self.cache, self.g = cache, torch.Generator("cuda").manual_seed(seed)

    def rows(self, n, heads):
        return torch.randn(n, heads, self.cache.d, generator=self.g, device="cuda").bfloat16()

    def widths(self, n):
        pick = torch.multinomial(torch.tensor([0.2, 0.4, 0.3, 0.1], device="cuda"), n, replacement=True, generator=self.g)
        return BITS.cuda()[pick]

    def append(self, seq_ids, positions):
        """New tokens of every layer; returns how many were appended."""
        c, n = self.cache, seq_ids.numel()
        modes = torch.full((n,), trr.MODE_FULL, dtype=torch.uint8, device="cuda")
        for layer in range(c.L):
            c.append(layer, seq_ids, positions, self.rows(n, c.Hkv), self.rows(n, c.Hkv), self.widths(n), modes)
        return n


def ints(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def pages_in_use(cache):
    return cache.region("next_page").view(torch.int32).cpu().tolist()


def main(layers=2, samples=8, prompt=500, steps=24, window=64, sinks=4, turn=8, quiet=False):
    say = (lambda *a: None) if quiet else print
    # sequence 0 is the prompt, then two banks of samples
    seqs, most = 1 + 2 * samples, prompt + steps + 4 * window
    pages = layers * (prompt // 16 + 8 + 2 * samples * (steps // 16 + 3))
    cache = trr.Cache(layers, seqs, 12, 12, 64, 32, 16, most, [pages] * 4, max_append=1024, max_queries=max(16, samples))
    model = Model(cache)
    for start in range(0, prompt, 1024):
        at = torch.arange(start, min(start + 1024, prompt), dtype=torch.int32, device="cuda")
        model.append(torch.zeros_like(at), at)
    say("the prompt's pages of 2, 4, 8 and 16 bits:", pages_in_use(cache))

    banks = [ints(range(1, 1 + samples)), ints(range(1 + samples, seqs))]
    now = 0
    cache.fork(torch.zeros_like(banks[0]), banks[0], torch.full_like(banks[0], prompt))
    say(f"with {samples} samples that share them:", pages_in_use(cache))
    group = ints([0, samples])
    modes = torch.full((samples,), trr.MODE_FULL, dtype=torch.uint8, device="cuda")
    for step in range(steps):
        seq_ids, positions = banks[now], torch.full((samples,), prompt + step, dtype=torch.int32, device="cuda")
        model.append(seq_ids, positions)
        for layer in range(layers):
            out = cache.decode_attn_shared(layer, seq_ids, positions, model.rows(samples, cache.Hq), modes, group)
        if (step + 1) % turn == 0:  # the better half goes on, twice each
            scores = out.float().sum((1, 2))
            best = banks[now][scores.argsort(descending=True)[:(samples + 1) // 2]]
            parents = best.repeat_interleave(2)[:samples].contiguous()
            cache.fork(parents, banks[1 - now], torch.full_like(parents, prompt + step + 1))
            cache.free(banks[now])
            cache.compact()
            now = 1 - now
            say(f"step {step + 1}, beams turned:", pages_in_use(cache))

    seq, at = banks[now][:1].contiguous(), prompt + steps
    cache.free(ints([s for s in range(seqs) if s != int(seq)]))
    local = torch.full((1,), trr.MODE_LOCAL, dtype=torch.uint8, device="cuda")
    used = []
    for step in range(3 * window):
        position = ints([at + step])
        model.append(seq, position)
        for layer in range(layers):
            out = cache.decode_attn_sinks(layer, seq, position, model.rows(1, cache.Hq), local, sinks, window_scalar=window)
        if (step + 1) % (window // 2) == 0:
            cache.evict(seq, ints([at + step + 1 - window]), sinks)
            cache.compact()
            used.append(pages_in_use(cache))
            say(f"streamed {step + 1} tokens:", used[-1])
    assert cache.status() == 0
    return {"rows": out, "pages": used}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 2), ("samples", 8), ("prompt", 500), ("steps", 24), ("window", 64), ("sinks", 4)):
        ap.add_argument("--" + name, type=int, default=value)
    main(**vars(ap.parse_args()))
