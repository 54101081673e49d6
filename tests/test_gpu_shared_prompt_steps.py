"""The example of several answers to one prompt over a program's steps: more and
longer answers as it goes, rewritten stretches of the prompt, what it reports
and what it refuses."""
import os
import sys

import pytest
import torch

from paper_2606_00724_gb300 import wf

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from shared_prompt import SharedPrompt  # noqa: E402

H, N, D, LEVELS, KEPT = 3, 2048, 128, 4, 128


def rn(g, *shape, by=1.0):
    return (by * torch.randn(*shape, generator=g)).bfloat16().cuda()


def prompt_of(seed, fmt=wf.WF_MXFP8):
    g = torch.Generator().manual_seed(seed)
    K, V = rn(g, H, N, D), rn(g, H, N, D)
    return g, K, V, SharedPrompt(K, V, LEVELS, KEPT, fmt)


def test_answers_and_generations_grow():
    g, K, V, prompt = prompt_of(0)
    for B, q, ng in ((1, 1, 1), (2, 8, 4), (6, 32, 40), (1, 4, 300), (8, 32, 90)):
        Q, Kg, Vg = rn(g, H, B, q, D), rn(g, B, H, ng, D), rn(g, B, H, ng, D)
        O = prompt.attend(Q, Kg, Vg)
        wf.wf_workspace_status(prompt.ws)
        wf.wf_workspace_status(prompt.attn_ws)
        fresh = SharedPrompt(K, V, LEVELS, KEPT, wf.WF_MXFP8).attend(Q, Kg, Vg)
        assert torch.equal(O, fresh) and torch.isfinite(O).all()


@pytest.mark.parametrize("fmt", [wf.WF_MXFP8, wf.WF_MXFP4])
@pytest.mark.parametrize("pos,count", [(100, 17), (0, 16), (2031, 17), (1024, 1), (5, 2000)])
def test_rewritten_stretch_is_selected_by(pos, count, fmt):
    # The pyramid after a write is that of the rows that the prompt now has: the new ones as given, in the blocks of
    # 16 tokens around them the others as the cache holds them, and the first ones elsewhere.
    g, K, V, prompt = prompt_of(1, fmt)
    new = rn(g, H, count, D)
    prompt.write(new, -new, pos)
    kept = torch.empty(1, H, N, D, dtype=torch.bfloat16, device="cuda")
    wf.wf_cache_dequantize(prompt.Kc, prompt.Ks, None, None, fmt, kept, None)
    now = K.clone()
    lo, hi = pos // 16 * 16, -(-(pos + count) // 16) * 16
    now[:, lo:hi] = kept[0, :, lo:hi]
    now[:, pos:pos + count] = new
    want = torch.empty_like(prompt.pyramid)
    wf.wf_dwt_build(now[None], LEVELS, want)
    assert torch.equal(prompt.pyramid, want)


def test_rewritten_rows_are_found():
    # Rows that answer the queries much better than all others are written over: the next step selects them.
    g, K, V, prompt = prompt_of(2)
    Q, Kg, Vg = rn(g, H, 2, 8, D), rn(g, 2, H, 8, D), rn(g, 2, H, 8, D)
    Q[:] = Q[:, :1, :1]
    prompt.attend(Q, Kg, Vg)
    stretch = torch.arange(640, 672, device="cuda")
    assert not torch.isin(stretch, prompt.idx[0]).all()
    new = Q[:, 0, :1].expand(H, 32, D).contiguous()
    prompt.write(new, new, 640)
    prompt.attend(Q, Kg, Vg)
    for h in range(H):
        assert torch.isin(stretch, prompt.idx[h]).all()


def test_bytes_that_are_reported(capsys):
    # The pyramid stays in 16 bits and counts on both sides: 15/16 of the keys at four levels.
    import shared_prompt
    r = shared_prompt.main(["--tokens", "2048", "--answers", "2", "--heads", "2", "--steps", "1"])
    keys = 2 * 2048 * 128
    assert r["cache_bytes"] == 2 * (keys + keys // 32) and r["pyramid_bytes"] == 2 * keys * 15 // 16
    said = capsys.readouterr().out
    kept = r["cache_bytes"] + r["pyramid_bytes"]
    assert f"{kept / 1e6:.1f} MB with keys and values quantised" in said
    assert f"{(2 * 2 * keys + r['pyramid_bytes']) / 1e6:.1f} MB with them in bf16" in said


def test_answers_of_one_selection():
    # 256 rows a key head are one selection; more are refused with what to do about it, and groups of them work.
    g, K, V, prompt = prompt_of(3)
    Q, Kg, Vg = rn(g, H, 16, 32, D), rn(g, 16, H, 32, D), rn(g, 16, H, 32, D)
    with pytest.raises(ValueError, match="groups"):
        prompt.attend(Q, Kg, Vg)
    for at in (slice(0, 8), slice(8, 16)):
        O = prompt.attend(Q[:, at].contiguous(), Kg[at], Vg[at])
        assert O.shape == (H, 8, 32, D) and torch.isfinite(O).all()
    with pytest.raises(ValueError, match="key head"):
        prompt.attend(rn(g, 2 * H, 1, 32, D), Kg[:1], Vg[:1])


def test_selection_reads_no_keys():
    g, K, V, prompt = prompt_of(4)
    Q, Kg, Vg = rn(g, H, 4, 32, D), rn(g, 4, H, 32, D), rn(g, 4, H, 32, D)
    before = prompt.attend(Q, Kg, Vg), prompt.idx.clone()
    prompt.shape[0, 0].fill_(float("nan"))  # the memory that stands in for the keys, in the filter's arguments alone
    assert torch.equal(prompt.attend(Q, Kg, Vg), before[0]) and torch.equal(prompt.idx, before[1])
