"""wf_prefix_attn where a CTA walks many key tiles, and where the own rows meet
the parts of a long prompt in the joining kernel, against the float64
definition.  Every case states what it has to reach and checks that the call is
planned so, so that another split cannot empty it."""
import numpy as np
import pytest
import torch

from helpers import assert_close_out
from paper_2606_00724_gb300 import wf
from test_gpu_prefix_attn import Case, f64

pytestmark = pytest.mark.gpu


def plan(c):
    kv = wf.code_desc(c.K, c.fmt) if c.fmt is not None else wf.desc(c.K)
    p = wf.wf_testing_prefix_plan(wf.desc(c.Q), kv, c.k, c.ng)
    p.tiles = -(-c.k // p.key_tile)
    p.per = -(-p.tiles // p.prompt_parts) if p.prompt_parts else 0  # key tiles a CTA
    return p


LONG = [  # B, P, H, G, q, n, ng, key tiles a CTA at least
    (1, 1, 152, 1, 1, 1500, 0, 12),   # one query row, one part: an even number of tiles
    (1, 1, 150, 1, 1, 1411, 0, 11),
    (1, 1, 150, 1, 2, 1295, 0, 11),   # an odd number
    (1, 1, 40, 1, 3, 3000, 300, 8),   # own rows as units
    (2, 2, 38, 2, 7, 2000, 0, 8),
    (2, 1, 76, 1, 100, 900, 0, 8),    # 200 query rows: both row tiles of a CTA
    (3, 1, 50, 1, 100, 1290, 0, 11),  # 256 and 44
    (2, 1, 150, 1, 64, 1100, 0, 9),   # 128: one full row tile
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cache", [None, "mxfp8", "mxfp4"])
@pytest.mark.parametrize("shape", LONG)
def test_many_tiles_a_cta(shape, cache, d):
    B, P, H, G, q, n, ng, per = shape
    c = Case(B, P, H, G, q, d, n, ng, "bf16", cache, seed=n)
    assert plan(c).per >= per and not plan(c).joined
    c.check()


@pytest.mark.parametrize("cache", [None, "mxfp8", "mxfp4"])
@pytest.mark.parametrize("q", [1, 140])
def test_many_tiles_of_selected_rows_and_unequal_lengths(q, cache):
    c = Case(2, 2, 76, 1, q, 128, 1600, 0, "bf16", cache, k=1444, select=True, plen=[1444, 1283], seed=18)
    assert plan(c).per >= 11
    c.check()
    c = Case(3, 3, 50, 1, q, 64, 1500, 0, "bf16", cache, plen=[0, 1, 1409], seed=19, layout="bshd")
    assert plan(c).per >= 11
    O = c.check()
    assert (O[0] == 0).all() and (O[1] != 0).any()  # one 4-bit row holds zeros too


@pytest.mark.parametrize("cache", [None, "mxfp8"])
@pytest.mark.parametrize("shape", [(1, 152, 1, 128, 700, 5), (1, 152, 40, 128, 330, 3), (2, 76, 50, 64, 450, 4),
                                   (2, 76, 100, 64, 330, 6)])
def test_many_tiles_a_cta_in_fp32(shape, cache):
    B, H, q, d, n, per = shape
    c = Case(B, 1, H, 1, q, d, n, 20 if q == 100 else 0, "f32", cache, seed=n)
    assert plan(c).per >= per
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 60, 200])
def test_maximum_rises_from_tile_to_tile_of_a_cta(q, dtype):
    # Logits along each head's first query go from about 3 to 82 over one CTA's tiles, slowly and then by more than 8
    # (log2) a tile; the rows' other parts set them apart.  Values of half the usual size: at such peaked rows O is a
    # value row up to 2.4, whose rounding (2^-7) and that of its weight (2.4 x 2^-9) stay below 2e-2 together.
    c = Case(1, 1, 150, 1, q, 128, 1300, 0, dtype, seed=20)
    assert plan(c).per >= 5
    first = c.Q[:, :, :1].float()
    c.Q.copy_(first + 0.3 * c.Q.float() * (torch.arange(q, device="cuda") > 0)[:, None])
    rise = torch.linspace(0, 1, 1300, device="cuda").pow(3)[:, None] * 7 + 0.3
    c.K.copy_(first / first.norm(dim=-1, keepdim=True) * 11.3 * rise + 0.05 * c.K.float())
    c.V.mul_(0.5)
    c.K64, c.V64 = f64(c.K), f64(c.V)
    c.check()


JOINED = [  # B, P, H, G, q, d, n, ng, parts, query rows a CTA of the joining kernel
    (64, 1, 1, 1, 1, 128, 3000, 9, 24, 4),
    (64, 1, 1, 1, 1, 64, 3000, 9, 24, 4),
    (16, 2, 8, 7, 1, 128, 1900, 30, 8, 4),
    (32, 2, 2, 1, 24, 64, 2100, 17, 9, 4),
    (8, 1, 8, 1, 40, 64, 2500, 20, 7, 8),
    (8, 1, 8, 1, 40, 128, 2500, 20, 7, 8),
    (640, 2, 1, 1, 1, 64, 1500, 11, 12, 16),
    (32, 2, 8, 1, 32, 128, 1500, 32, 3, 16),
    (32, 2, 5, 1, 64, 64, 1200, 20, 2, 32),
    (32, 2, 5, 1, 64, 128, 1200, 20, 2, 32),
    (16, 1, 10, 1, 64, 128, 1200, 200, 2, 64),
    (16, 1, 10, 1, 64, 64, 1200, 200, 2, 64),
    (16, 2, 10, 2, 50, 128, 1100, 210, 1, 64),  # blocks of 64 and 36 rows
]


@pytest.mark.parametrize("cache", [None, "mxfp4"])
@pytest.mark.parametrize("shape", JOINED)
def test_own_rows_joined_with_parts(shape, cache):
    B, P, H, G, q, d, n, ng, parts, rows = shape
    r = np.random.default_rng(n + ng)
    glen = r.integers(0, ng + 1, B).tolist()
    glen[:4] = [0, 1, ng, -1]
    plen = [n - 77] * P
    plen[-1] = 0 if P > 1 else n - 130
    for lens in (dict(), dict(plen=plen, glen=glen)):
        c = Case(B, P, H, G, q, d, n, ng, "bf16", cache, seed=21, **lens)
        p = plan(c)
        assert p.joined and not p.direct and (p.prompt_parts, p.join_rows) == (parts, rows)
        O = c.check()
        if lens and P > 1:
            empty = [b for b in range(B // P * (P - 1), B) if glen[b] <= 0]
            assert (O[empty] == 0).all()


DIRECT = [  # B, P, H, G, q, d, n, ng, rows
    (40, 1, 3, 1, 1, 128, 127, 128, 16),
    (6, 2, 16, 1, 60, 64, 70, 30, 32),
    (8, 4, 16, 1, 24, 128, 60, 0, 16),
    (20, 1, 16, 1, 32, 64, 100, 20, 32),
    (20, 1, 16, 2, 32, 128, 64, 70, 64),
]


@pytest.mark.parametrize("select", [False, True])
@pytest.mark.parametrize("shape", DIRECT)
def test_few_prompt_rows_attended_with_the_own_rows(shape, select):
    B, P, H, G, q, d, n, ng, rows = shape
    glen = [(7 * b) % (ng + 1) for b in range(B)] if ng else None
    c = Case(B, P, H, G, q, d, n, ng, "bf16", select=select, plen=[n - 3 * p for p in range(P)], glen=glen, seed=22)
    p = plan(c)
    assert p.direct and p.join_rows == rows
    c.check()


@pytest.mark.parametrize("shape", [(64, 2, 2, 1, 1, 128, 1500, 50), (16, 2, 10, 1, 64, 64, 1200, 200)])
def test_nan_and_infinity_stay_with_their_rows_when_joined(shape):
    c = Case(*shape, "bf16", plen=[1200, 1100], glen=[50, 20, 50, 0] + [40] * (shape[0] - 4), seed=23)
    assert plan(c).joined and plan(c).prompt_parts > 1
    before = c.run()
    nan = float("nan")
    c.Vg[0, 0, 3] = nan
    c.Kg[2, 1, 49] = nan
    c.Vg[4, 0, 7] = float("inf")
    c.K[1, 1, 1100:] = nan           # past the length of prompt 1
    c.V[0, 1, 1200:] = float("inf")  # and of prompt 0
    c.Kg[1, :, 20:] = nan
    c.Vg[3] = nan
    after = c.run()
    touched = torch.zeros(after.shape[:2], dtype=torch.bool)
    touched[0, 0] = touched[2, 1] = touched[4, 0] = True
    assert torch.equal(after[~touched], before[~touched])
    assert torch.isnan(after[0, 0]).all() and torch.isnan(after[2, 1]).all()
    assert (~torch.isfinite(after[4, 0])).all()
    c.V[1, 0, 700] = nan             # a row of prompt 1, key head 0
    last = c.run()
    half = shape[0] // 2
    assert torch.isnan(last[half:, 0]).all()
    assert torch.equal(last[half:, 1:], after[half:, 1:])
