"""Drafted values that are not finite behind a mask, where the tensor-core kernel of wf_tree_attn brings its rows by
chunks: pages that have no 8 rows or more in common with a tile.  Such values are taken out of a tile after it has
arrived, so the products must wait for that as they wait for the rows."""
import pytest
import torch

from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ps", [1, 4, 100])
@pytest.mark.parametrize("q,G", [(20, 1), (40, 2), (70, 2), (150, 2)])
def test_what_a_masked_drafted_row_holds_does_not_matter(q, G, ps, d):
    # 20 to 300 query rows a key head: one row tile of half or of whole height, and two.
    c = Case(2, 2, G, q, d, 90, ps, q, seed=31)
    hidden = q // 2
    c.sees[0, :, hidden] = False
    c.sees[0, -1, hidden] = True      # one row sees it
    before = c.check()
    c.Vt[0, :, hidden, ::3] = float("nan")
    c.Vt[0, :, hidden, 1::3] = float("inf")
    for _ in range(5):
        after = c.run()
        assert torch.equal(after[1], before[1]) and torch.equal(after[0, :, :-1], before[0, :, :-1])
        last = after[0, :, -1]
        assert torch.isnan(last[:, ::3]).all() and (last[:, 1::3] == float("inf")).all()
        assert torch.isfinite(last[:, 2::3]).all()


@pytest.mark.parametrize("ps", [1, 100])
@pytest.mark.parametrize("q", [19, 70])
def test_masked_values_in_any_part_of_a_long_draft(q, ps):
    # Rows that nothing sees but the last query row, in tiles that different ranges have.
    c = Case(1, 1, 2, q + 1, 128, 600, ps, 280, seed=32)
    hidden = [3, 70, 129, 200, 279]
    c.sees[:, :, hidden] = False
    before = c.check()
    for j in hidden:
        c.Vt[0, 0, j, j % 128] = float("nan")
        c.Vt[0, 0, j, (j + 1) % 128] = -float("inf")
    assert torch.equal(c.run(), before)
    c.sees[:, -1, hidden] = True
    after = c.run()
    assert torch.equal(after[:, :, :-1], before[:, :, :-1])
    for j in hidden:
        assert torch.isnan(after[0, :, -1, j % 128]).all()
