"""Drafted tokens over a cache in pages, for sequences of unequal lengths.

A pool of pages holds the keys and values of all sequences, rotated by their
positions, in 16 bits or in 8- or 4-bit codes.  Every step drafts a tree of tokens a
sequence: its queries and keys are rotated by the nodes' depths, the queries
attend to the sequence's pages and, by the tree's mask, to the drafted rows, and the
rows on the accepted path go into the pages.  Rejected rows never enter the cache, so
nothing has to be compacted.  A denoising block is the draft whose rows all see each
other, one token the draft of one node.

    python examples/drafted_tokens.py [--sequences 8] [--prompt 4096] [--steps 4] [--codes mxfp8|mxfp4]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_00724_gb300 import wf  # noqa: E402

FORMATS = {"mxfp8": wf.WF_MXFP8, "mxfp4": wf.WF_MXFP4}


class PagedCache:
    """Keys and values of one layer (bf16 rows of H heads), in pages that sequences take as they grow."""

    def __init__(self, sequences: int, heads: int, d: int, pages: int, page_rows: int, longest: int, codes: str | None):
        self.fmt, self.page_rows = FORMATS.get(codes), page_rows
        kind = torch.bfloat16 if codes is None else torch.uint8
        width = d // 2 if codes == "mxfp4" else d
        self.K, self.V = (torch.zeros(pages, heads, page_rows, width, dtype=kind, device="cuda") for _ in "KV")
        self.Ks = self.Vs = None
        if codes is not None:
            self.Ks, self.Vs = (torch.zeros(wf.wf_scales_bytes(self.K, self.fmt), dtype=torch.uint8, device="cuda")
                                for _ in "KV")
        self.free = list(range(pages))
        self.owned = [0] * sequences  # pages of each sequence
        self.table = torch.full((sequences, -(-longest // page_rows)), -1, dtype=torch.int32, device="cuda")
        self.length = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.lengths = [0] * sequences  # the same on the host, where pages are handed out
        freq = torch.exp(torch.arange(d // 2, dtype=torch.float64) * (-math.log(10000.0) / (d // 2)))
        self.plan = wf.wf_rotary_plan(freq).cuda()
        self.ws = torch.zeros(256, dtype=torch.uint8, device="cuda")

    def _reserve(self, more: list[int]) -> None:
        """Pages for so many rows more of each sequence."""
        for b, rows in enumerate(more):
            need = -(-(self.lengths[b] + rows) // self.page_rows)
            if need > self.table.shape[1]:
                raise ValueError(f"sequence {b} outgrows its table")
            while self.owned[b] < need:
                self.table[b, self.owned[b]] = self.free.pop()
                self.owned[b] += 1

    def append(self, K, V, counts: list[int], rows=None, rotated: bool = False) -> None:
        """The first counts[b] new rows of each sequence, or of the rows [B, m] of them."""
        if len(counts) != K.shape[0] or min(counts) < 0 or max(counts) > (K.shape[2] if rows is None else rows.shape[1]):
            raise ValueError("counts of rows that are not there")
        self._reserve(counts)
        count = torch.tensor(counts, dtype=torch.int32, device="cuda")
        wf.wf_paged_append(K, V, self.K, self.V, self.table, self.length, Ks=self.Ks, Vs=self.Vs, fmt=self.fmt, rows=rows,
                           count=count, plan=None if rotated else self.plan)
        self.length += count
        self.lengths = [n + c for n, c in zip(self.lengths, counts)]

    def attend(self, Q, K, V, depth, mask=None):
        """Q [B, Hq, q, d] over the pages and the drafted K, V [B, H, q, d]; Q and K are rotated in place by depth [B, q]
        past the sequence."""
        pos = (self.length[:, None] + depth)[None].to(torch.int32).contiguous()
        wf.wf_rotary_apply(Q, K, self.plan, pos, Q, K)
        n, O = max(self.lengths), torch.empty_like(Q)
        size = wf.wf_tree_attn_workspace_bytes(Q, self.K, n, K.shape[2], fmt=self.fmt)
        if size > self.ws.nbytes:  # the word in which a call reports a wait that gave up goes along
            larger = torch.zeros(size, dtype=torch.uint8, device="cuda")
            larger[:4] = self.ws[:4]
            self.ws = larger
        wf.wf_tree_attn(Q, self.K, self.V, self.table, n, K, V, O, self.ws, cache_len=self.length, mask=mask, Ks=self.Ks,
                        Vs=self.Vs, fmt=self.fmt)
        return O


def draft_tree(parents: list[int]):
    """(depth of each node, mask words [q, words] int32) of a tree whose node i hangs below parents[i] (-1: a root)."""
    depth, seen = [], []
    for i, p in enumerate(parents):
        depth.append(0 if p < 0 else depth[p] + 1)
        seen.append((0 if p < 0 else seen[p]) | 1 << i)
    words = -(-len(parents) // 32)
    signed = [[(s >> 32 * w & 0xffffffff) - ((s >> 32 * w + 31 & 1) << 32) for w in range(words)] for s in seen]
    return depth, torch.tensor(signed, dtype=torch.int32)


def path_to(parents: list[int], node: int) -> list[int]:
    path = []
    while node >= 0:
        path.append(node)
        node = parents[node]
    return path[::-1]


def main(argv=None) -> dict:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--sequences", type=int, default=8)
    p.add_argument("--prompt", type=int, default=4096)
    p.add_argument("--steps", type=int, default=4)
    p.add_argument("--heads", type=int, default=8)
    p.add_argument("--group", type=int, default=4)
    p.add_argument("--page-rows", type=int, default=16)
    p.add_argument("--codes", choices=sorted(FORMATS))
    a = p.parse_args(argv)
    B, H, d = a.sequences, a.heads, 128
    parents = [-1, 0, 0, 1, 1, 2, 3, 6]  # what a drafter proposes: two branches, the first one longer
    q = len(parents)
    depth, words = draft_tree(parents)
    depth = torch.tensor(depth, device="cuda").expand(B, q)
    mask = words.cuda().expand(B, -1, -1).contiguous()
    longest = a.prompt + a.steps * q
    cache = PagedCache(B, H, d, B * -(-longest // a.page_rows), a.page_rows, longest, a.codes)
    g = torch.Generator(device="cuda").manual_seed(0)

    def draw(*shape):
        return torch.randn(*shape, generator=g, device="cuda").bfloat16()
    prompts = [max(1, a.prompt - 37 * b) for b in range(B)]
    K, V = draw(B, H, a.prompt, d), draw(B, H, a.prompt, d)
    cache.append(K, V, prompts)
    record = []
    for step in range(a.steps):
        Q, Kt, Vt = draw(B, H * a.group, q, d), draw(B, H, q, d), draw(B, H, q, d)
        before = list(cache.lengths)
        O = cache.attend(Q, Kt, Vt, depth, mask)
        took = [path_to(parents, (3 * b + step) % q) for b in range(B)]  # what a verifier would accept
        rows = torch.zeros(B, q, dtype=torch.int32)
        for b, path in enumerate(took):
            rows[b, :len(path)] = torch.tensor(path)
        cache.append(Kt, Vt, [len(path) for path in took], rows=rows.cuda(), rotated=True)
        record.append(dict(Q=Q, K=Kt, V=Vt, O=O, lengths=before, took=took))
    wf.wf_workspace_status(cache.ws)
    print(f"{B} sequences of {min(cache.lengths)} to {max(cache.lengths)} tokens in {sum(cache.owned)} pages of "
          f"{a.page_rows} rows, {2 * cache.K.nbytes / 1e6:.1f} MB; {a.steps} drafts of {q} tokens")
    return {"cache": cache, "K": K, "V": V, "prompts": prompts, "steps": record, "parents": parents}


if __name__ == "__main__":
    main()
