"""The plan of a wf_prefix_attn call, on the host: no call writes past the
workspace that it asks for, and the parts and tiles cover the keys."""
import random

import pytest

from paper_2606_00724_gb300 import build as wf_build
from paper_2606_00724_gb300 import wf


@pytest.fixture(scope="module", autouse=True)
def lib():
    wf_build.build()
    return wf.lib()


@pytest.mark.parametrize("dtype", [wf.WF_BF16, wf.WF_F32])
def test_what_a_call_writes_fits(dtype):
    r = random.Random(1)
    for _ in range(3000):
        P = r.choice([1, 1, 2, 3, 30])
        B, H, G = P * r.choice([1, 2, 5, 24, 100]), r.choice([1, 2, 8, 51]), r.choice([1, 2, 7])
        d, q, n = r.choice([64, 128]), r.choice([1, 4, 32, 100]), r.choice([1, 100, 2000, 40000, 1 << 20])
        k, n_g = r.choice([n, r.randint(0, n)]), r.choice([0, 1, 40, 300, 2000])
        q_desc, kv = (wf.wf_tensor(b, h, s, d, h * s * d, s * d, d, dtype) for b, h, s in ((B, H * G, q), (P, H, n)))
        p = wf.wf_testing_prefix_plan(q_desc, kv, k, n_g)
        rows, parts = B * H * G * q, p.prompt_parts + p.own_parts
        if parts > 1 or p.joined:
            assert p.workspace_used >= 256 + parts * rows * (8 + 4 * d)
        assert p.workspace_used <= wf.lib().wf_prefix_attn_workspace_bytes(q_desc, kv, k, n_g)
        assert (p.prompt_parts > 0) == (k > 0 and not p.direct)
        assert p.prompt_parts <= -(-k // p.key_tile)
        assert not p.joined or (dtype == wf.WF_BF16 and p.own_parts == 0 and 4 <= p.join_rows <= 64)
        # The joining kernel's shared memory: query rows, two stages of K and V, the parts' weights.
        if p.joined:
            assert 64 * d * 2 + 4 * 64 * d * 2 + 4 * 64 * 4 + p.join_rows * (p.prompt_parts + 4) * 8 <= 232448
