"""What examples/drafted_tokens.py refuses before it changes anything."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import drafted_tokens  # noqa: E402


@pytest.mark.parametrize("counts,rows", [([3, 5], None), ([-1, 2], None), ([2, 3], [[0, 1], [1, 2]]), ([2], None)])
def test_the_example_refuses_counts_that_its_rows_do_not_have(counts, rows):
    cache = drafted_tokens.PagedCache(2, 1, 128, 4, 16, 32, None)
    x = torch.zeros(2, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    rows = None if rows is None else torch.tensor(rows, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        cache.append(x, x, counts, rows=rows)
    assert cache.lengths == [0, 0] and cache.owned == [0, 0] and len(cache.free) == 4
    cache.append(x, x, [4, 0])
    assert cache.lengths == [4, 0] and cache.length.tolist() == [4, 0]
