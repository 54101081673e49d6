"""Values of seen rows that are not finite reach the query rows that see them, however small the row's weight is, with
a mask and without one, in both types; rows that a mask hides touch nothing."""
import pytest
import torch

from test_gpu_tree_attn import Case, words

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)


def run(c, mask):
    O, ws, args = torch.full_like(c.Q, 7.0), c.workspace(), {**c.args(), "mask": mask}
    from paper_2606_00724_gb300 import wf
    wf.wf_tree_attn(c.Q, c.K, c.V, c.pages.cuda(), c.n, c.Kt, c.Vt, O, ws, **args)
    wf.wf_workspace_status(ws)
    return O


def low_logits(c, j):
    """Logits of -500 or less of drafted row j: its weight is 0 in either type."""
    c.Q[..., 0] = 8.0
    c.Kt[:, :, j] = 0
    c.Kt[:, :, j, 0] = -64.0 * c.Q.shape[3] ** 0.5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cache", [None, "mxfp8"])
@pytest.mark.parametrize("q,G", [(2, 1), (5, 2), (20, 1), (40, 4), (70, 1)])
def test_a_weight_that_underflows_does_not_hide_a_value(q, G, cache, dtype):
    c = Case(2, 2, G, q, 128, 90, 16, q, dtype, cache, shape="block", seed=41)
    j = q // 2
    low_logits(c, j)
    all_of_them = torch.ones(2, q, q, dtype=torch.bool).numpy()
    before = run(c, None)
    assert torch.isfinite(before).all()
    c.Vt[0, 1, j, 3], c.Vt[0, 1, j, 70], c.Vt[0, 1, j, 127] = float("inf"), -float("inf"), float("nan")
    bad = torch.zeros(128, dtype=torch.bool)
    bad[[3, 70, 127]] = True
    for mask in (None, words(all_of_them)):
        O = run(c, mask)
        assert not torch.isfinite(O[0, G:, :, bad]).any()
        assert torch.equal(O[0, G:, :, ~bad], before[0, G:, :, ~bad])
        assert torch.equal(O[1], before[1]) and torch.equal(O[0, :G], before[0, :G])
    # Hidden from all but the last row.
    all_of_them[0, :-1, j] = False
    O = run(c, words(all_of_them))
    assert torch.isfinite(O[:, :, :-1]).all() and not torch.isfinite(O[0, G:, -1][:, bad]).any()
    assert torch.isfinite(O[0, G:, -1][:, ~bad]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [3, 24])
def test_a_mask_that_hides_nothing_and_none_at_all(q, dtype):
    # The same rows in the same order: the same bits.
    c = Case(3, 2, 2, q, 128, 200, 16, q, dtype, shape="block", seed=42, tlen=[q, 1, 0])
    ones = torch.ones(3, q, q, dtype=torch.bool).numpy()
    assert torch.equal(run(c, None), run(c, words(ones)))
