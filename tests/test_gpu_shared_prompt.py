"""The example of several answers to one prompt: the selection is the oracle's
for the grouped query blocks, the outputs are the float64 attention over the
quantised cache's selected rows and each answer's own rows, and a rewritten
stretch is read back."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle
from helpers import assert_close_out, eps_valid, f64
from oracle import mx
from paper_2606_00724_gb300 import wf

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import shared_prompt  # noqa: E402


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
def test_example(fmt):
    args = ["--tokens", "2048", "--answers", "4", "--heads", "3", "--steps", "2"]
    r = shared_prompt.main(args + (["--four-bit"] if fmt == "mxfp4" else []))
    prompt, Q, H, B = r["prompt"], r["Q"], 3, 4
    # The quantised cache holds the rounded keys and values.
    values = {}
    for name, codes, scales, want in (("K", prompt.Kc, prompt.Ks, r["K"]), ("V", prompt.Vc, prompt.Vs, r["V"])):
        c, s = mx.quantize(f64(want), fmt)
        assert np.array_equal(codes[0].cpu().numpy(), mx.pack(c, fmt))
        values[name] = mx.values(mx.pack(c, fmt), s, fmt)
    # Every head's selection is a Top-K for the blocks of all answers together.
    keep, L = prompt.keep, prompt.levels
    for h in range(H):
        K64 = f64(r["K"][h])
        pyr = oracle.haar_pyramid_spec32(K64.astype(np.float32), L, True)
        sets = torch.empty(H, sum(keep), dtype=torch.int32, device="cuda")
        wf.wf_filter(Q.view(1, H * B, 32, 128), prompt.pyramid, prompt.shape, L, keep, prompt.idx, prompt.ws, sets)
        got = oracle.split_level_sets(sets[h].cpu().numpy(), L, keep)
        eps_valid(f64(Q[h]).reshape(-1, 128), pyr, K64, 2048, L, keep, got)
        assert np.array_equal(prompt.idx[h].cpu().numpy(), got[0])
    want = mx.prefix_attention(f64(Q).transpose(1, 0, 2, 3), values["K"][None], values["V"][None], f64(r["Kg"]),
                               f64(r["Vg"]), keep[0], prompt.idx.cpu().numpy(), None, r["gen_len"].cpu().numpy())
    assert_close_out(f64(r["O"]).transpose(1, 0, 2, 3), want, torch.bfloat16)
    # A stretch of the prompt changes.
    new = torch.randn(H, 17, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    prompt.write(new, -new, 100)
    out = torch.empty(2, 1, H, 19, 128, dtype=torch.bfloat16, device="cuda")
    wf.wf_cache_dequantize(prompt.Kc, prompt.Ks, prompt.Vc, prompt.Vs, prompt.fmt, out[0], out[1], 99)
    c, s = mx.quantize(f64(new), fmt)
    rounded = mx.values(mx.pack(c, fmt), s, fmt)
    assert np.array_equal(f64(out[0, 0, :, 1:18]), rounded) and np.array_equal(f64(out[1, 0, :, 1:18]), -rounded)
    assert np.array_equal(f64(out[0, 0, :, [0, 18]]), values["K"][:, [99, 117]])
