"""Decode steps of a serving batch over paged record caches.

Prompts of different lengths are encoded into the pages of each layer's pools, the boxes of
their keys beside them.  Every decode step then appends one token a sequence (records and
boxes), chooses `budget` pages a KV head by the box bound and attends over them; the same
queries over all pages show what the choice left out.

    python examples/paged_decode.py [--tokens 20000] [--budget 64] [--steps 4]

Keys follow a theme that changes from stretch to stretch of the text, queries look for one of
the themes: attention is concentrated, as it is where choosing pages makes sense.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import torch

import paper_2603_27467_gb300 as tac

HEADS, GROUP, D, PAGE = 8, 4, 128, 64


class Layer:
    """One layer's pools, boxes and codebooks (K: 8-bit linear norms, V: 4-bit in log space)."""

    def __init__(self, index: int, pages: int):
        k = tac.layer_cfg(D, 64, 8, tac.NORM_LINEAR, 0, index, 0)
        v = tac.layer_cfg(D, 64, 4, tac.NORM_LOG, 0, index, 1)
        self.cache = tac.PagedCache.empty(k, v, pages, HEADS, PAGE)
        self.bounds = tac.PageBounds.empty(pages, HEADS, D, PAGE)

    def write(self, keys, values, table, start, first, seq, pos):
        """Keys and values [rows, HEADS, D] of tokens at positions `pos` of the sequences `seq`."""
        slot = self.cache.slots(table, pos, seq)
        tac.encode_multi([tac.EncodeJob(self.cache.k.cfg, keys.reshape(-1, D), self.cache.k, slot),
                          tac.EncodeJob(self.cache.v.cfg, values.reshape(-1, D), self.cache.v, slot)])
        tac.page_bounds(self.bounds, keys, table, start, first)


def run(lengths, budget: int, steps: int = 2, layers: int = 2, seed: int = 0) -> dict:
    """Prefill, then `steps` decode steps.  Returns the share of the cached tokens that the chosen
    pages hold, and the relative error (2-norm) that reading only them leaves in the outputs."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    seqs, ends = len(lengths), [n + steps for n in lengths]
    per = [-(-n // PAGE) for n in ends]
    pages = sum(per)
    table = torch.full((seqs, max(per)), -1, dtype=torch.int32, device="cuda")
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)   # pages as they were free
    at = 0
    for s, n in enumerate(per):
        table[s, :n] = order[at: at + n]
        at += n
    seq = torch.cat([torch.full((n,), s, device="cuda") for s, n in enumerate(lengths)])
    pos = torch.cat([torch.arange(n, device="cuda") for n in lengths])
    first = i32([0] + [sum(lengths[: s + 1]) for s in range(seqs)])
    themes = 2.0 * torch.randn((32, HEADS, D), generator=g, device="cuda")

    def rows(which):
        x = torch.randn((len(which), HEADS, D), generator=g, device="cuda")
        return (x + themes[which]).to(torch.bfloat16), torch.randn((len(which), HEADS, D), generator=g, device="cuda").to(torch.bfloat16)

    stack = [Layer(i, pages) for i in range(layers)]
    for layer in stack:
        layer.write(*rows(pos // 512 * 7 % 32), table, i32([0] * seqs), first, seq, pos)
    now, one = list(lengths), torch.arange(seqs, device="cuda")
    left, total, read, held = 0.0, 0.0, 0, 0
    for _ in range(steps):
        start = i32(now)
        lens = start + 1                             # the new token sees itself
        for layer in stack:
            layer.write(*rows(torch.randint(0, 32, (seqs,), generator=g, device="cuda")), table, start, None, one, start)
            look = themes[torch.randint(0, 8, (seqs,), generator=g, device="cuda")]
            q = 0.5 * look[:, :, None] + torch.randn((seqs, HEADS, GROUP, D), generator=g, device="cuda")
            q = q.reshape(seqs, HEADS * GROUP, D).to(torch.bfloat16)
            chosen, count = tac.select_pages(q, layer.bounds, table, lens, budget)
            out = tac.attend_pages(q, layer.cache, table, lens, 1.0 / math.sqrt(D), chosen, count)
            whole = tac.attend_pages(q, layer.cache, table, lens, 1.0 / math.sqrt(D))
            left += float((out.double() - whole.double()).square().sum())
            total += float(whole.double().square().sum())
            read += int(torch.minimum(count * PAGE, lens[:, None]).sum())
            held += int(lens.sum()) * HEADS
        now = [n + 1 for n in now]
    return {"share_read": read / held, "relative_error": math.sqrt(left / total)}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=20000)
    ap.add_argument("--budget", type=int, default=64)
    ap.add_argument("--steps", type=int, default=4)
    a = ap.parse_args()
    lengths = [a.tokens, a.tokens // 3, a.tokens // 7, max(1, a.tokens // 50)]
    got = run(lengths, a.budget, a.steps)
    print(f"{len(lengths)} sequences of {lengths} tokens, {a.budget} pages of {PAGE} tokens a KV head: "
          f"{100 * got['share_read']:.0f} % of the cache read, outputs {100 * got['relative_error']:.2f} % off those of the whole cache")


if __name__ == "__main__":
    main()
