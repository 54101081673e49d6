"""Refusals and sizes of the quantised cache and of the attention over shared
prompts, through the C ABI, without a GPU: every argument is checked on the
host before anything is launched."""
import ctypes

import pytest
import torch

from paper_2606_00724_gb300 import build as wf_build
from paper_2606_00724_gb300 import wf

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="placeholder pointers: host-only check")


@pytest.fixture(scope="module")
def lib():
    wf_build.build()
    return wf.lib()


def _desc(B, H, S, D, dtype=wf.WF_BF16, sb=None, sh=None, ss=None):
    ss = D if ss is None else ss
    sh = S * ss if sh is None else sh
    sb = H * sh if sb is None else sb
    return wf.wf_tensor(B, H, S, D, sb, sh, ss, dtype)


def P(x):
    return ctypes.c_void_p(x)


INVALID, SHAPE, DTYPE, ALIGN, SPACE, UNSUPPORTED = -1, -2, -3, -4, -5, -8
FP8, FP4 = wf.WF_MXFP8, wf.WF_MXFP4


def test_scales_bytes(lib):
    assert lib.wf_scales_bytes(_desc(2, 3, 10, 128, FP8)) == 2 * 3 * 10 * 4
    assert lib.wf_scales_bytes(_desc(2, 3, 10, 64, FP4)) == 2 * 3 * 10 * 2
    assert lib.wf_scales_bytes(_desc(2, 3, 10, 128)) == 0         # not a quantised cache
    assert lib.wf_scales_bytes(_desc(2, 3, 10, 96, FP8)) == 0
    assert lib.wf_scales_bytes(_desc(2, 3, 10, 64, FP4, ss=80)) == 0   # 40-byte rows


@no_gpu
def test_quantize_rejects(lib):
    nt, kv = _desc(1, 2, 5, 128), _desc(1, 2, 64, 128, FP8)
    need = lib.wf_scales_bytes(kv)

    def call(Kn=P(0x1000), Vn=P(0x2000), nt=nt, Kc=P(0x3000), Ks=P(0x4000), Vc=P(0x5000), Vs=P(0x6000), kv=kv,
             size=need, pos=0):
        return lib.wf_cache_quantize(Kn, Vn, nt, Kc, Ks, Vc, Vs, kv, size, pos, None)
    assert call(Kn=None) == INVALID and call(Kc=None) == INVALID and call(Ks=None) == INVALID
    assert call(Vn=None) == INVALID and call(Vc=None) == INVALID and call(Vs=None) == INVALID
    assert call(pos=-1) == INVALID and call(pos=60) == INVALID and call(pos=2 ** 62) == INVALID
    assert call(size=need - 1) == SPACE
    assert call(kv=_desc(1, 2, 64, 128)) == DTYPE                       # a bf16 cache
    assert call(nt=_desc(1, 2, 5, 128, FP8)) == DTYPE                   # codes as new rows
    assert call(nt=_desc(1, 3, 5, 128)) == SHAPE and call(nt=_desc(1, 2, 5, 64)) == SHAPE
    assert call(kv=_desc(1, 2, 64, 128, FP8, ss=136)) == ALIGN
    assert call(kv=_desc(1, 2, 64, 128, FP4, ss=144), size=10 ** 9) == ALIGN   # 72-byte rows
    assert call(kv=_desc(1, 2, 64, 128, FP8, ss=64), size=10 ** 9) == SHAPE    # rows overlap
    assert call(Kn=P(0x1008)) == ALIGN and call(Vc=P(0x5008)) == ALIGN and call(Ks=P(0x4002)) == ALIGN
    assert lib.wf_cache_quantize(P(0x1000), None, None, P(0x3000), P(0x4000), None, None, kv, need, 0, None) == INVALID
    assert call(nt=_desc(1, 2, 0, 128), pos=64) == 0                    # no rows: nothing to do


@no_gpu
def test_dequantize_rejects(lib):
    out, kv = _desc(1, 2, 5, 128, wf.WF_F32), _desc(1, 2, 64, 128, FP4)
    need = lib.wf_scales_bytes(kv)

    def call(Kc=P(0x1000), Ks=P(0x2000), Vc=P(0x3000), Vs=P(0x4000), kv=kv, size=need, idx=None, pos=0, Ko=P(0x5000),
             Vo=P(0x6000), out=out):
        return lib.wf_cache_dequantize(Kc, Ks, Vc, Vs, kv, size, idx, pos, Ko, Vo, out, None)
    assert call(Kc=None) == INVALID and call(Ko=None) == INVALID and call(Vo=None) == INVALID
    assert call(Vs=None) == INVALID and call(pos=60) == INVALID
    assert call(idx=P(0x7000), pos=1) == INVALID                        # a selection has no position
    assert call(idx=P(0x7002)) == ALIGN and call(Ko=P(0x5004)) == ALIGN
    assert call(size=0) == SPACE
    assert call(out=_desc(1, 2, 5, 128, FP4)) == DTYPE and call(kv=_desc(1, 2, 64, 128, 9)) == DTYPE
    assert call(out=_desc(2, 2, 5, 128)) == SHAPE
    assert call(out=_desc(1, 2, 0, 128)) == 0


@no_gpu
def test_prefix_attn_rejects(lib):
    q, kv, g = _desc(4, 6, 3, 128), _desc(2, 2, 64, 128), _desc(4, 2, 7, 128)
    need = lib.wf_prefix_attn_workspace_bytes(q, kv, 64, 7)
    assert need > 256

    def call(Q=P(0x10000), q=q, K=P(0x20000), V=P(0x30000), kv=kv, Ks=None, Vs=None, idx=None, k=64, plen=None,
             Kg=P(0x40000), Vg=P(0x50000), g=g, glen=None, O=P(0x60000), o=q, scale=0.0, ws=P(0x70000), size=need):
        return lib.wf_prefix_attn(Q, q, K, V, kv, Ks, Vs, idx, k, plen, Kg, Vg, g, glen, O, o, scale, ws, size, None)
    assert call(size=need - 1) == SPACE
    for name in ("Q", "K", "V", "Kg", "Vg", "O", "ws"):
        assert call(**{name: None}) == INVALID, name
    for name in ("Q", "K", "V", "Kg", "Vg", "O"):
        assert call(**{name: P(0x10008)}) == ALIGN, name
    for name in ("idx", "plen", "glen"):
        assert call(**{name: P(0x10002)}) == ALIGN, name
    assert call(ws=P(0x70010)) == ALIGN
    assert call(k=-1) == INVALID and call(k=65) == INVALID
    assert call(scale=-1.0) == INVALID and call(scale=float("inf")) == INVALID and call(scale=float("nan")) == INVALID
    assert call(kv=_desc(3, 2, 64, 128)) == SHAPE                       # 4 sequences on 3 prompts
    assert call(kv=_desc(2, 4, 64, 128)) == SHAPE                       # 6 query heads on 4
    assert call(kv=_desc(2, 2, 64, 64)) == SHAPE
    assert call(kv=_desc(2, 2, 64, 128, wf.WF_F32)) == DTYPE
    assert call(g=_desc(2, 2, 7, 128)) == SHAPE and call(g=_desc(4, 6, 7, 128)) == SHAPE
    assert call(g=_desc(4, 2, 7, 128, FP8)) == DTYPE
    assert call(o=_desc(4, 6, 2, 128)) == SHAPE and call(o=_desc(4, 6, 3, 128, wf.WF_F32)) == DTYPE
    assert call(kv=_desc(2, 2, 64, 128, FP8), size=10 ** 9) == INVALID         # no scales
    assert call(Ks=P(0x80000), Vs=P(0x90000)) == INVALID                # scales of a bf16 prompt
    assert call(kv=_desc(2, 2, 64, 128, FP8), Ks=P(0x80001), Vs=P(0x90000), size=10 ** 9) == ALIGN
    assert call(q=_desc(1 << 15, 1 << 10, 64, 128, sb=0, sh=0), kv=_desc(1, 1, 64, 128)) == UNSUPPORTED


def test_prefix_attn_workspace(lib):
    q = _desc(4, 6, 3, 128)
    assert lib.wf_prefix_attn_workspace_bytes(q, _desc(2, 2, 64, 128), 65, 0) == 0
    assert lib.wf_prefix_attn_workspace_bytes(q, _desc(2, 2, 64, 128), 64, -1) == 0
    assert lib.wf_prefix_attn_workspace_bytes(q, _desc(3, 2, 64, 128), 64, 0) == 0
    assert lib.wf_prefix_attn_workspace_bytes(q, _desc(2, 2, 64, 128, FP4), 64, 0) >= 256


@no_gpu
def test_other_calls_refuse_quantised_caches(lib):
    kv = _desc(1, 2, 64, 128, FP8)
    assert lib.wf_coeffs_bytes(kv, 2) == 0
    assert lib.wf_dwt_build(P(0x1000), None, kv, 2, P(0x2000), 10 ** 9, None) == DTYPE
    q = _desc(1, 2, 8, 128)
    assert lib.wf_sparse_attn(P(0x1000), q, P(0x2000), P(0x3000), kv, P(0x4000), 8, None, None, None, P(0x5000), q, 0.0,
                              P(0x10000), 10 ** 9, None) == DTYPE


def test_binding_refuses_what_it_cannot_describe():
    K = torch.zeros(1, 2, 8, 128, dtype=torch.bfloat16)
    codes, scales = torch.zeros(1, 2, 8, 128, dtype=torch.uint8), torch.zeros(1, 2, 8, 4, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        wf.wf_cache_quantize(K, None, codes, scales, None, None, FP8, 0)
    with pytest.raises(ValueError, match="unknown format"):
        wf.wf_scales_bytes(codes, wf.WF_BF16)
    with pytest.raises(ValueError, match="8-bit"):
        wf.wf_scales_bytes(K, FP8)
    assert wf.code_desc(codes[..., :64], FP4).head_dim == 128
