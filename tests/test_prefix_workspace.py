"""A wf_prefix_attn workspace serves every call with no more keys, own rows and
query rows than the one it was sized for; host only."""
import random

import pytest

from paper_2606_00724_gb300 import build as wf_build
from paper_2606_00724_gb300 import wf


@pytest.fixture(scope="module", autouse=True)
def lib():
    wf_build.build()
    return wf.lib()


def size(B, P, H, G, q, d, n, k, n_g, dtype):
    def desc(B, H, S):
        return wf.wf_tensor(B, H, S, d, H * S * d, S * d, d, dtype)
    return wf.lib().wf_prefix_attn_workspace_bytes(desc(B, H * G, q), desc(P, H, n), k, n_g)


@pytest.mark.parametrize("dtype", [wf.WF_BF16, wf.WF_F32])
@pytest.mark.parametrize("B,H,G,q,n_g", [(16, 4, 7, 1, 65), (4, 32, 1, 32, 32), (1, 1, 1, 1, 0), (8, 8, 4, 1, 33),
                                         (64, 1, 1, 1, 700), (3, 50, 1, 100, 0)])
def test_fewer_keys_fit(B, H, G, q, n_g, dtype):
    n = 32768
    whole = size(B, 1, H, G, q, 128, n, n, n_g, dtype)
    last = 0
    for k in list(range(0, 3000, 67)) + list(range(3000, n, 509)) + [9721, 32128, n]:
        now = size(B, 1, H, G, q, 128, n, k, n_g, dtype)
        assert 0 < now <= whole, k
        if k != 9721 and k != 32128:
            assert now >= last, k
            last = now
    last = 0
    for g in range(0, 1500, 13):
        now = size(B, 1, H, G, q, 128, n, 5000, g, dtype)
        assert now >= last, g
        last = now


@pytest.mark.parametrize("dtype", [wf.WF_BF16, wf.WF_F32])
@pytest.mark.parametrize("d", [64, 128])
def test_smaller_calls_of_any_shape_fit(d, dtype):
    r = random.Random(0)
    for _ in range(300):
        P = r.choice([1, 1, 2, 3])
        B, H, G = P * r.randint(1, 24), r.choice([1, 2, 8, 40]), r.choice([1, 2, 7])
        q, n = r.choice([1, 4, 32, 100]), r.choice([100, 2000, 40000])
        k, n_g = r.randint(0, n), r.choice([0, 1, 40, 300, 2000])
        most = size(B, P, H, G, q, d, n, k, n_g, dtype)
        # Fewer answers to each prompt, fewer prompts, shorter blocks, fewer keys.
        p = r.randint(1, P)
        assert size(p * r.randint(1, B // P), p, H, G, r.randint(1, q), d, n, r.randint(0, k), r.randint(0, n_g),
                    dtype) <= most
