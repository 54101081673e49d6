"""The first key tiles of a range, of which the second may arrive before the first: a cached tile that is widened
from codes, or looked up in many pages, followed by drafted tiles that come straight from memory.  Half a tile of
query rows, so that two warps take every other key tile.  The same bits every time, those of the definition, and
values of drafted rows that nothing sees never come through."""
import pytest
import torch

from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)


@pytest.mark.parametrize("cache", ["mxfp8", "mxfp4", None])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,n_t", [(92, 131), (92, 300), (128, 129), (1, 500), (200, 400), (1500, 131), (0, 400)])
def test_a_cached_tile_before_drafted_ones(n, n_t, d, cache):
    c = Case(2, 3, 1, 64, d, n, 39, n_t, "bf16", cache, shape="chain", layout="bshd", seed=91)
    before = c.check()
    c.sees[:, :, 1::7] = False
    hidden = c.check()
    c.Vt[:, :, 1::7, 5] = float("nan")
    c.Vt[:, :, 1::7, d - 1] = float("inf")
    for _ in range(40):
        assert torch.equal(c.run(), hidden)
    assert torch.isfinite(before).all()


@pytest.mark.parametrize("cache", ["mxfp8", "mxfp4", None])
@pytest.mark.parametrize("ps", [16, 128])
def test_ranges_of_a_few_tiles(ps, cache):
    c = Case(9, 4, 2, 33, 128, 700, ps, 40, "bf16", cache, clen=[700, 130, 257, 1, 0, 385, 513, 640, 129], seed=92)
    first = c.check()
    for _ in range(40):
        assert torch.equal(c.run(), first)
