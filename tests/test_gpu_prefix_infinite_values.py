"""wf_prefix_attn where every logit of a query row is -inf: O is 0 whatever the
value rows hold, infinities and NaN among them, on every route."""
import pytest
import torch

from test_gpu_prefix_attn import Case

pytestmark = pytest.mark.gpu

SHAPES = [  # B, P, H, G, q, d, n, ng
    (2, 1, 2, 1, 4, 64, 64, 20),       # the prompt's rows where the own rows are: blocks of 16 query rows
    (40, 1, 3, 1, 1, 128, 127, 128),
    (3, 1, 16, 2, 5, 128, 90, 0),      # no own rows
    (64, 1, 1, 1, 1, 128, 1500, 9),    # own rows where the prompt's parts are joined: blocks of 4, 16 and 64 query rows
    (16, 1, 4, 1, 32, 128, 3000, 40),
    (4, 1, 16, 1, 64, 64, 1100, 70),
    (16, 1, 10, 1, 64, 128, 1200, 200),
    (2, 1, 1, 1, 4, 64, 300, 70),      # own rows as units of the prompt's kernel
    (2, 1, 1, 1, 200, 64, 300, 70),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_infinite_values_under_no_weight(shape, dtype):
    c = Case(*shape, dtype, seed=17)
    c.Q[..., 0] = 1.0
    c.K[..., 0] = -float("inf")
    c.V[:, :, 0] = float("inf")
    c.V[:, :, -1, 3] = float("nan")
    if c.ng:
        c.Kg[..., 0] = -float("inf")
        c.Vg[:, :, 0] = -float("inf")
        c.Vg[:, :, -1, 5] = float("nan")
    assert (c.run() == 0).all()
