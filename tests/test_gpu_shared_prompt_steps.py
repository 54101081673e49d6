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
