"""Codes in pages with an odd number of rows: two scale bytes of a 64-wide row then begin at either half of a word, and
a tile crosses many pages.  Several hundred cached rows of unequal lengths, against the float64 definition."""
import pytest
import torch

from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cache", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("ps", [1, 7, 25, 127])
@pytest.mark.parametrize("q,G", [(3, 2), (16, 1), (20, 1), (40, 2), (70, 2), (150, 2)])
def test_pages_of_an_odd_number_of_rows(q, G, ps, cache, d):
    # 6 to 300 query rows a key head: the kernel for few rows, and row tiles of half height, whole height, and two.
    Case(3, 2, G, q, d, 700, ps, q, "bf16", cache, clen=[700, 333, 130], seed=51).check()


@pytest.mark.parametrize("cache", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("ps", [2, 6, 66])
@pytest.mark.parametrize("q", [4, 24])
def test_pages_of_an_even_number_of_rows_that_divide_nothing(q, ps, cache):
    Case(3, 3, 2, q, 64, 500, ps, q, "bf16", cache, clen=[499, 66, 257], seed=52).check()


@pytest.mark.parametrize("cache", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("ps", [1, 25])
def test_fp32_queries(ps, cache):
    Case(3, 2, 2, 9, 64, 300, ps, 9, "f32", cache, clen=[300, 77, 25], seed=53).check()
