"""Several answers to one long prompt, from an 8-bit or 4-bit cache.

A prompt's keys and values are turned into the filter's pyramid and a quantised
cache once, and the 16-bit tensors can go.  Every denoising step then selects
prompt rows for all answers together (their query blocks form one group a key
head, so the selection is one row list a head) and attends each answer's block
to the selected rows of the quantised cache, read once for all, and to the
answer's own rows.  A stretch of the prompt that changed is quantised into its
place, and the pyramid over it is rebuilt.

One selection serves at most 256 query rows of a key head (wf_filter's limit),
eight answers' blocks of 32; more answers are attended in groups, each with a
selection of its own.  Every query head has a key head here: with grouped heads
the two calls want the queries in different orders.

    python examples/shared_prompt.py [--tokens 32768] [--answers 4] [--heads 32] [--four-bit]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_00724_gb300 import wf  # noqa: E402


class SharedPrompt:
    """One prompt's keys and values [H, n, d] (bf16), kept quantised with the pyramid of its keys."""

    MAX_ROWS = 256  # query rows a selection: wf_filter's limit a key head

    def __init__(self, K: torch.Tensor, V: torch.Tensor, levels: int, kept: int, fmt: int):
        H, n, d = K.shape
        self.levels, self.fmt = levels, fmt
        self.keep = wf.wf_default_schedule(n, levels, kept)
        if self.keep[0] != 2 * self.keep[1]:
            raise ValueError("an odd count would score raw keys, which are not kept")
        self.pyramid = torch.empty(H, n - (n >> levels), d, dtype=K.dtype, device=K.device)
        wf.wf_dwt_build(K[None], levels, self.pyramid)
        width = d // 2 if fmt == wf.WF_MXFP4 else d
        self.Kc, self.Vc = (torch.empty(1, H, n, width, dtype=torch.uint8, device=K.device) for _ in range(2))
        self.Ks, self.Vs = (torch.empty(wf.wf_scales_bytes(self.Kc, fmt), dtype=torch.uint8, device=K.device)
                            for _ in range(2))
        wf.wf_cache_quantize(K[None], V[None], self.Kc, self.Ks, self.Vc, self.Vs, fmt, 0)
        # The filter takes the keys for their shape; with every kept pair of tokens selected it reads the pyramid
        # alone, so one head's worth of memory stands for all of them.
        self.shape = K.new_empty(1, 1, n, d).expand(1, H, n, d)
        self.idx = torch.empty(H, self.keep[0], dtype=torch.int32, device=K.device)
        self.ws, self.attn_ws = (torch.zeros(256, dtype=torch.uint8, device=K.device) for _ in range(2))

    def write(self, K: torch.Tensor, V: torch.Tensor, pos: int) -> None:
        """Rows [pos, pos + count) of the prompt from K, V [H, count, d]: into the cache, and into the pyramid's
        coefficients over the blocks of 2^levels tokens that hold them.  The blocks' other rows are read back out of
        the cache, the only place where they still are."""
        H, count, d = K.shape
        if count == 0:
            return
        wf.wf_cache_quantize(K[None], V[None], self.Kc, self.Ks, self.Vc, self.Vs, self.fmt, pos)
        n, L = self.Kc.shape[2], self.levels
        lo, hi = pos >> L << L, -(-(pos + count) >> L) << L
        rows = torch.empty(1, H, hi - lo, d, dtype=K.dtype, device=K.device)
        wf.wf_cache_dequantize(self.Kc, self.Ks, None, None, self.fmt, rows, None, lo)
        rows[0, :, pos - lo:pos - lo + count] = K
        stretch = torch.empty(H, (hi - lo) - (hi - lo >> L), d, dtype=K.dtype, device=K.device)
        wf.wf_dwt_build(rows, L, stretch)
        for level in range(1, L + 1):  # n / 2^level rows from n - n / 2^(level - 1) on
            to, at, m = n - (n >> level - 1), (hi - lo) - (hi - lo >> level - 1), hi - lo >> level
            self.pyramid[:, to + (lo >> level):to + (hi >> level)] = stretch[:, at:at + m]

    @staticmethod
    def _at_least(ws: torch.Tensor, size: int) -> torch.Tensor:
        """ws, or a larger workspace in its place where a step has more answers or longer ones; the word in which
        the calls report a wait that gave up goes along."""
        if ws.nbytes >= size:
            return ws
        larger = torch.zeros(size, dtype=torch.uint8, device=ws.device)
        larger[:4] = ws[:4]
        return larger

    def attend(self, Q: torch.Tensor, Kg: torch.Tensor, Vg: torch.Tensor, gen_len=None) -> torch.Tensor:
        """Q [H, B, q, d]: the query blocks of B answers, head by head; Kg, Vg [B, H, ng, d] the answers' own rows,
        of which the first gen_len[b] count.  The answers' outputs, [H, B, q, d]."""
        H, B, q, d = Q.shape
        if H != self.Kc.shape[1]:
            raise ValueError("a query head a key head")
        if B * q > self.MAX_ROWS:
            raise ValueError(f"one selection serves at most {self.MAX_ROWS} query rows: attend in groups of answers")
        grouped, by_answer = Q.view(1, H * B, q, d), Q.transpose(0, 1)
        O = torch.empty_like(Q)
        self.ws = self._at_least(self.ws, wf.wf_filter_workspace_bytes(grouped, self.shape, self.levels, self.keep))
        self.attn_ws = self._at_least(self.attn_ws, wf.wf_prefix_attn_workspace_bytes(
            by_answer, self.Kc, self.keep[0], Kg.shape[2], fmt=self.fmt))
        wf.wf_filter(grouped, self.pyramid, self.shape, self.levels, self.keep, self.idx, self.ws)
        wf.wf_prefix_attn(by_answer, self.Kc, self.Vc, self.keep[0], Kg, Vg, O.transpose(0, 1), self.attn_ws,
                          idx=self.idx, gen_len=gen_len, Ks=self.Ks, Vs=self.Vs, fmt=self.fmt)
        return O


def main(argv=None) -> dict:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--tokens", type=int, default=32768)
    p.add_argument("--answers", type=int, default=4)
    p.add_argument("--heads", type=int, default=32)
    p.add_argument("--steps", type=int, default=3)
    p.add_argument("--four-bit", action="store_true")
    a = p.parse_args(argv)
    n, B, H, q, d, levels = a.tokens, a.answers, a.heads, 32, 128, 4
    fmt = wf.WF_MXFP4 if a.four_bit else wf.WF_MXFP8
    g = torch.Generator(device="cuda").manual_seed(0)

    def draw(*shape):
        return torch.randn(*shape, generator=g, device="cuda").bfloat16()
    K, V = draw(H, n, d), draw(H, n, d)
    prompt = SharedPrompt(K, V, levels, n // 16, fmt)
    Kg, Vg = draw(B, H, q, d), draw(B, H, q, d)
    gen_len = torch.tensor([q - b % 3 for b in range(B)], dtype=torch.int32, device="cuda")
    for _ in range(a.steps):
        Q = draw(H, B, q, d)
        O = prompt.attend(Q, Kg, Vg, gen_len)
    wf.wf_workspace_status(prompt.ws)
    wf.wf_workspace_status(prompt.attn_ws)
    cache, pyramid = 2 * (prompt.Kc.nbytes + prompt.Ks.nbytes), prompt.pyramid.nbytes
    result = {"cache_bytes": cache, "pyramid_bytes": pyramid, "bf16_bytes": K.nbytes + V.nbytes,
              "rows": prompt.keep[0], "Q": Q, "O": O, "K": K, "V": V, "Kg": Kg, "Vg": Vg, "gen_len": gen_len,
              "prompt": prompt}
    print(f"{n} tokens, {H} heads, with a pyramid of {pyramid / 1e6:.1f} MB in bf16: "
          f"{(cache + pyramid) / 1e6:.1f} MB with keys and values quantised, "
          f"{(result['bf16_bytes'] + pyramid) / 1e6:.1f} MB with them in bf16; "
          f"{B} answers attend to {prompt.keep[0]} rows a head")
    return result


if __name__ == "__main__":
    main()
