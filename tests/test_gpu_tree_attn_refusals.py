"""What the binding of wf_tree_attn refuses, where it would be dropped without a word."""
import pytest
import torch

from paper_2606_00724_gb300 import wf
from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)


@pytest.mark.parametrize("drop", ["Kt", "Vt"])
def test_drafted_keys_and_values_go_together(drop):
    c = Case(1, 1, 1, 2, 64, 20, 16, 2, shape="block", seed=71)
    rows = {"Kt": c.Kt, "Vt": c.Vt, drop: None}
    O, ws = torch.empty_like(c.Q), c.workspace()
    with pytest.raises(ValueError, match="together"):
        wf.wf_tree_attn(c.Q, c.K, c.V, c.pages.cuda(), c.n, rows["Kt"], rows["Vt"], O, ws)
