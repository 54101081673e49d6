"""Plans, refusals and sizes of the cache in pages, through the C ABI, without a
GPU: every argument is checked on the host before anything is launched."""
import ctypes
import math
import random
from fractions import Fraction

import pytest
import torch

from oracle.paged import PI
from paper_2606_00724_gb300 import build as wf_build
from paper_2606_00724_gb300 import wf

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="placeholder pointers: host-only check")
INVALID, SHAPE, DTYPE, ALIGN, SPACE, UNSUPPORTED = -1, -2, -3, -4, -5, -8
FP8, FP4 = wf.WF_MXFP8, wf.WF_MXFP4


@pytest.fixture(scope="module", autouse=True)
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


def test_plan_is_the_nearest_turn():
    r = random.Random(0)
    freq = [0.0, 1.0, -1.0, 2.0 ** -40, 5e-324, 4294967295.9] + [r.choice([1, -1]) * 2.0 ** r.uniform(-70, 31.9)
                                                                for _ in range(300)]
    plan = wf.wf_rotary_plan(torch.tensor(freq, dtype=torch.float64), torch.arange(306, dtype=torch.int32) % 64)
    for f, (turn, axis), i in zip(freq, plan.tolist(), range(306)):
        want = Fraction(f) * 2 ** 64 / (2 * PI)
        # pi to 60 digits leaves 2^64 2^32 / 10^59 of it open, far below the half that rounding may take.
        off = (turn - want) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= Fraction(1, 2) + Fraction(1, 10 ** 20), f
        assert axis == i % 64


def test_plan_refuses():
    def plan(freq, axis=None):
        a = None if axis is None else torch.tensor(axis, dtype=torch.int32)
        return wf.wf_rotary_plan(torch.tensor(freq, dtype=torch.float64), a)
    for bad in ([], [math.nan], [math.inf], [2.0 ** 32], [1.0, -2.0 ** 33]):
        with pytest.raises(wf.WfError):
            plan(bad)
    for axis in ([-1], [64]):
        with pytest.raises(wf.WfError):
            plan([1.0], axis)
    with pytest.raises(ValueError):
        plan([1.0], [0, 1])
    with pytest.raises(ValueError):
        wf.wf_rotary_plan(torch.ones(4))


@no_gpu
def test_rotary_rejects(lib):
    q, k = _desc(2, 6, 5, 128), _desc(2, 2, 5, 128)

    def call(Q=P(0x1000), q=q, K=P(0x2000), k=k, plan=P(0x3000), pairs=64, pos=P(0x4000), axes=1, Qo=P(0x5000), qo=None,
             Ko=P(0x6000), ko=None):
        return lib.wf_rotary_apply(Q, q, K, k, plan, pairs, 0, pos, axes, Qo, qo or q, Ko, ko or k, None)
    for name in ("Q", "K", "plan", "pos", "Qo", "Ko"):
        assert call(**{name: None}) == INVALID, name
    for name in ("Q", "K", "plan", "Qo", "Ko"):
        assert call(**{name: P(0x7008)}) == ALIGN, name
    assert call(pos=P(0x7002)) == ALIGN
    assert call(pairs=0) == SHAPE and call(pairs=72) == SHAPE and call(pairs=12) == SHAPE
    assert call(axes=0) == INVALID
    assert call(qo=_desc(2, 6, 4, 128)) == SHAPE and call(ko=_desc(2, 3, 5, 128)) == SHAPE
    assert call(k=_desc(3, 2, 5, 128)) == SHAPE and call(k=_desc(2, 2, 4, 128)) == SHAPE
    assert call(k=_desc(2, 2, 5, 64)) == SHAPE
    assert call(qo=_desc(2, 6, 5, 128, wf.WF_F32)) == DTYPE and call(k=_desc(2, 2, 5, 128, wf.WF_F32)) == DTYPE
    assert call(q=_desc(2, 6, 5, 128, FP8)) == DTYPE
    assert call(q=_desc(2, 6, 5, 128, ss=132)) == ALIGN
    assert call(q=_desc(1 << 14, 1 << 12, 1 << 8, 128, sb=0, sh=0), K=None, Ko=None) == UNSUPPORTED
    empty, none = _desc(2, 6, 0, 128), _desc(2, 2, 0, 128)
    assert call(Q=None, q=empty, K=P(0x2000), k=none, Qo=None, pos=None) == 0


@no_gpu
def test_append_rejects(lib):
    nt, pool = _desc(3, 2, 5, 128), _desc(40, 2, 16, 128)

    def call(Kn=P(0x1000), Vn=P(0x2000), nt=nt, at=None, m=5, start=P(0x3000), count=None, plan=None, pairs=0, pos=None,
             axes=0, K=P(0x4000), V=P(0x5000), Ks=None, Vs=None, pool=pool, size=0, pages=P(0x6000), table=8):
        return lib.wf_paged_append(Kn, Vn, nt, at, m, start, count, plan, pairs, 0, pos, axes, K, V, Ks, Vs, pool, size,
                                   pages, table, None)
    for name in ("Kn", "Vn", "start", "K", "V", "pages"):
        assert call(**{name: None}) == INVALID, name
    for name in ("Kn", "Vn", "K", "V"):
        assert call(**{name: P(0x7008)}) == ALIGN, name
    for name in ("start", "count", "pages"):
        assert call(**{name: P(0x7002)}) == ALIGN, name
    assert call(at=P(0x7001), m=3) == ALIGN and call(plan=P(0x7008), pairs=64) == ALIGN
    assert call(m=4) == INVALID and call(m=-1, at=P(0x7000)) == INVALID
    assert call(table=0) == INVALID and call(table=1 << 27) == UNSUPPORTED
    assert call(plan=P(0x7000), pairs=65) == SHAPE and call(plan=P(0x7000), pairs=64, pos=P(0x8000)) == INVALID
    assert call(nt=_desc(3, 4, 5, 128)) == SHAPE and call(nt=_desc(3, 2, 5, 64)) == SHAPE
    assert call(nt=_desc(3, 2, 5, 128, wf.WF_F32)) == DTYPE and call(nt=_desc(3, 2, 5, 128, FP8)) == DTYPE
    assert call(pool=_desc(40, 2, 0, 128)) == SHAPE
    assert call(pool=_desc(1 << 20, 2, 1 << 11, 128)) == UNSUPPORTED
    codes = _desc(40, 2, 16, 128, FP4)
    need = lib.wf_scales_bytes(codes)
    scales = dict(Ks=P(0x8000), Vs=P(0x9000), size=need)
    assert call(pool=codes, **{**scales, "size": need - 1}) == SPACE
    assert call(pool=codes, **{**scales, "Ks": None}) == INVALID and call(pool=codes, **{**scales, "Vs": None}) == INVALID
    assert call(pool=codes, **{**scales, "Ks": P(0x8002)}) == ALIGN
    assert call(Ks=P(0x8000), Vs=P(0x9000)) == INVALID             # scales of rows that have none
    assert call(nt=_desc(3, 2, 0, 128), m=0) == 0                  # no rows: nothing to do
    assert call(nt=_desc(3, 2, 0, 128), m=2, at=P(0x7000)) == INVALID


@no_gpu
def test_tree_attn_rejects(lib):
    q, pool, t = _desc(4, 6, 3, 128), _desc(40, 2, 16, 128), _desc(4, 2, 7, 128)
    need = lib.wf_tree_attn_workspace_bytes(q, pool, 120, 7)
    assert need > 256

    def call(Q=P(0x10000), q=q, K=P(0x20000), V=P(0x30000), pool=pool, Ks=None, Vs=None, pages=P(0x80000), table=8, n=120,
             clen=None, Kt=P(0x40000), Vt=P(0x50000), t=t, tlen=None, mask=None, O=P(0x60000), o=q, scale=0.0,
             ws=P(0x70000), size=need):
        return lib.wf_tree_attn(Q, q, K, V, pool, Ks, Vs, pages, table, n, clen, Kt, Vt, t, tlen, mask, O, o, scale, ws,
                                size, None)
    assert call(size=need - 1) == SPACE
    for name in ("Q", "K", "V", "Kt", "Vt", "O", "ws", "pages"):
        assert call(**{name: None}) == INVALID, name
    for name in ("Q", "K", "V", "Kt", "Vt", "O"):
        assert call(**{name: P(0x10008)}) == ALIGN, name
    for name in ("pages", "clen", "tlen", "mask"):
        assert call(**{name: P(0x10002)}) == ALIGN, name
    assert call(ws=P(0x70010)) == ALIGN
    assert call(n=-1) == INVALID and call(n=129) == INVALID and call(table=0) == INVALID
    assert call(scale=-1.0) == INVALID and call(scale=float("inf")) == INVALID and call(scale=float("nan")) == INVALID
    assert call(pool=_desc(40, 4, 16, 128)) == SHAPE               # 6 query heads on 4
    assert call(pool=_desc(40, 2, 16, 64)) == SHAPE
    assert call(pool=_desc(40, 2, 16, 128, wf.WF_F32)) == DTYPE
    assert call(t=_desc(2, 2, 7, 128)) == SHAPE and call(t=_desc(4, 6, 7, 128)) == SHAPE
    assert call(t=_desc(4, 2, 7, 128, FP8)) == DTYPE
    assert call(o=_desc(4, 6, 2, 128)) == SHAPE and call(o=_desc(4, 6, 3, 128, wf.WF_F32)) == DTYPE
    assert call(pool=_desc(40, 2, 16, 128, FP8), size=10 ** 9) == INVALID
    assert call(Ks=P(0x90000), Vs=P(0xa0000)) == INVALID
    assert call(q=_desc(1 << 15, 1 << 10, 64, 128, sb=0, sh=0), pool=_desc(1, 1, 64, 128)) == UNSUPPORTED
    assert call(q=_desc(1 << 9, 4, 64, 128, sb=0, sh=0), o=_desc(1 << 9, 4, 64, 128, sb=0, sh=0), t=None, Kt=None,
                Vt=None, pool=_desc(1, 2, 1 << 28, 128, sb=0, sh=0), n=1 << 28) == UNSUPPORTED   # too many tiles
    assert lib.wf_tree_attn_workspace_bytes(q, pool, -1, 0) == 0
    assert lib.wf_tree_attn_workspace_bytes(q, pool, 0, 0) >= 256


@pytest.mark.parametrize("dtype", [wf.WF_BF16, wf.WF_F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cache", ["rows", FP8])
def test_workspace_of_the_largest_call_serves_smaller_ones(lib, d, dtype, cache):
    def size(B, H, G, q, n, n_t):
        pool = _desc(7, H, 16, d, dtype if cache == "rows" else cache)
        return lib.wf_tree_attn_workspace_bytes(_desc(B, H * G, q, d, dtype), pool, n, n_t)
    r = random.Random(1)
    for _ in range(400):
        B, H, G, q = r.randint(1, 40), r.choice([1, 2, 8, 40]), r.choice([1, 2, 7]), r.choice([1, 4, 32, 100])
        n, n_t = r.choice([100, 2000, 40000, 200000]), r.choice([0, 1, 40, 300])
        assert 0 < size(r.randint(1, B), H, r.randint(1, G), r.randint(1, q), r.randint(0, n), r.randint(0, n_t)) <= \
            size(B, H, G, q, n, n_t)


def test_binding_refuses_what_it_cannot_describe():
    x = torch.zeros(2, 4, 3, 64)
    plan = wf.wf_rotary_plan(torch.ones(32, dtype=torch.float64))
    pages, pos = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(1, 2, 3, dtype=torch.int32)
    pool = torch.zeros(5, 4, 16, 64)
    with pytest.raises(ValueError, match="GPU"):
        wf.wf_rotary_apply(x, None, plan, pos, x, None)
    with pytest.raises(ValueError, match="GPU"):
        wf.wf_paged_append(x, x, pool, pool, pages, pages[:, 0])
    with pytest.raises(ValueError, match="GPU"):
        wf.wf_tree_attn(x, pool, pool, pages, 8, None, None, x, x)
