"""wf_prefix_attn refuses key counts that its kernels' 32-bit key numbers (a
range's end, rounded up to tiles) do not take; host only."""
import ctypes

import pytest
import torch

from paper_2606_00724_gb300 import build as wf_build
from paper_2606_00724_gb300 import wf

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="placeholder pointers: host-only check")
UNSUPPORTED = -8


@pytest.fixture(scope="module")
def lib():
    wf_build.build()
    return wf.lib()


def desc(B, H, S, D, dtype=wf.WF_BF16):
    return wf.wf_tensor(B, H, S, D, H * S * D, S * D, D, dtype)


def P(x):
    return ctypes.c_void_p(x)


@no_gpu
@pytest.mark.parametrize("dtype", [wf.WF_BF16, wf.WF_F32])
def test_key_counts_past_the_kernels_numbers(lib, dtype):
    q, n = desc(1, 1, 1, 64, dtype), 2 ** 31 - 1
    kv, scales = desc(1, 1, n, 64, wf.WF_MXFP4), (P(0x100000), P(0x200000))

    def call(k, g=None, kg=None):
        return lib.wf_prefix_attn(P(0x10000), q, P(0x20000), P(0x30000), kv, *scales, None, k, None, kg, kg, g, None,
                                  P(0x40000), q, 0.0, P(0x50000), 1 << 60, None)
    for k in (2 ** 30, 2 ** 31 - 128, n):
        assert lib.wf_prefix_attn_workspace_bytes(q, kv, k, 0) == 0
        assert call(k) == UNSUPPORTED
        # The same number of own rows.
        assert lib.wf_prefix_attn_workspace_bytes(q, kv, 5, k) == 0
        assert call(5, desc(1, 1, k, 64, dtype), P(0x60000)) == UNSUPPORTED
    # A cache of that length is no obstacle, and a count below is served.
    assert lib.wf_prefix_attn_workspace_bytes(q, kv, 2 ** 30 - 1, 0) > 0
    assert lib.wf_prefix_attn_workspace_bytes(q, kv, 64, 2 ** 30 - 1) > 0
