"""examples/drafted_tokens.py: the cache holds what was accepted, and every step's
attention is that of the definition over it (bf16; with codes, what the codes stand for)."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import mx

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import drafted_tokens  # noqa: E402


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("codes,page_rows", [(None, 16), ("mxfp8", 24), ("mxfp4", 16)])
def test_drafted_tokens(codes, page_rows):
    args = ["--sequences", "3", "--prompt", "90", "--steps", "3", "--heads", "2", "--group", "2", "--page-rows", str(page_rows)]
    r = drafted_tokens.main(args + (["--codes", codes] if codes else []))
    cache, parents = r["cache"], r["parents"]
    table, d = cache.table.cpu().numpy(), 128
    values = {}
    for x in "KV":
        t = getattr(cache, x).cpu()
        values[x] = mx.values(t.numpy(), getattr(cache, x + "s").cpu().numpy().reshape(*t.shape[:3], d // 32), codes) \
            if codes else f64(t)
    assert cache.lengths == [p + sum(len(s["took"][b]) for s in r["steps"]) for b, p in enumerate(r["prompts"])]
    for b in range(3):
        j = np.arange(cache.lengths[b])
        page, at = table[b, j // page_rows], j % page_rows
        assert (page >= 0).all()
        K, V = (values[x][page, :, at].transpose(1, 0, 2) for x in "KV")  # [H, rows, d]
        rows = f64(r["V"])[b, :, :r["prompts"][b]]
        accepted = [f64(s["V"])[b][:, s["took"][b]] for s in r["steps"]]
        want = np.concatenate([rows, *accepted], 1)
        if codes:
            want = mx.values(*[mx.pack(c, codes) if i == 0 else c for i, c in enumerate(mx.quantize(want, codes))], codes)
        assert np.array_equal(V, want)
        for s in r["steps"]:
            n = s["lengths"][b]
            for hq in range(4):
                for i in range(len(parents)):
                    seen = drafted_tokens.path_to(parents, i)
                    k = np.concatenate([K[hq // 2, :n], f64(s["K"])[b, hq // 2, seen]])
                    v = np.concatenate([V[hq // 2, :n], f64(s["V"])[b, hq // 2, seen]])
                    o = mx.attention(f64(s["Q"])[b, hq, i:i + 1], k, v)[0]
                    A = mx.attention(f64(s["Q"])[b, hq, i:i + 1], k, np.abs(v))[0]
                    # The output's rounding and the weights' (2^-8 each), and fp32's share.
                    assert (np.abs(f64(s["O"])[b, hq, i] - o) <= 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.0 ** -11) * A).all()


def test_draft_tree():
    depth, words = drafted_tokens.draft_tree([-1] + list(range(39)))
    assert depth == list(range(40)) and words.shape == (40, 2)
    assert words[31].tolist() == [-1, 0] and words[39].tolist() == [-1, 255]
    assert drafted_tokens.path_to([-1, 0, 0, 1], 3) == [0, 1, 3]
