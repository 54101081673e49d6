"""The quantised cache on the GPU against its definition: codes and scales are
equal to the bit, rows read back are code times scale, and rows around a
written window keep what they held."""
import numpy as np
import pytest
import torch

from oracle import mx
from paper_2606_00724_gb300 import wf

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

FMT = {"mxfp8": wf.WF_MXFP8, "mxfp4": wf.WF_MXFP4}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def lay(B, H, n, w, dtype, layout):
    if layout == "bshd":
        return torch.zeros(B, n, H, w, dtype=dtype, device="cuda").transpose(1, 2)
    if layout == "wide":  # rows of a larger buffer: strides above the packed ones
        return torch.zeros(B, H, n + 3, 2 * w, dtype=dtype, device="cuda")[:, :, 2:n + 2, :w]
    return torch.zeros(B, H, n, w, dtype=dtype, device="cuda")


def cache(B, H, n, d, fmt, layout):
    codes = [lay(B, H, n, d if fmt == "mxfp8" else d // 2, torch.uint8, layout) for _ in range(2)]
    for c in codes:
        c.fill_(0x5a)
    return codes, [torch.full((B, H, n, d // 32), 99, dtype=torch.uint8, device="cuda") for _ in range(2)]


def rows(r, B, H, m, d, dtype, layout):
    x = r.standard_normal((B, H, m, d)) * np.exp2(r.integers(-6, 6, (B, H, m, 1)))
    t = lay(B, H, m, d, DT[dtype], layout)
    t.copy_(torch.from_numpy(x))
    return t


def f64(t):
    return t.double().cpu().numpy()


CASES = [  # B, H, d, n, rows, pos, layout
    (1, 1, 64, 1, 1, 0, "bhsd"), (2, 3, 128, 40, 1, 39, "bshd"), (2, 3, 64, 77, 33, 5, "wide"),
    (1, 4, 128, 300, 300, 0, "bhsd"), (3, 2, 128, 50, 0, 50, "bhsd"), (2, 16, 128, 1200, 1111, 17, "bshd"),
    (1, 32, 64, 2048, 2048, 0, "bhsd"), (4, 32, 128, 600, 599, 1, "wide"),
]


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,d,n,m,pos,layout", CASES)
def test_write_and_read_back(B, H, d, n, m, pos, layout, dtype, fmt):
    r = np.random.default_rng(n + m)
    Kn, Vn = rows(r, B, H, m, d, dtype, layout), rows(r, B, H, m, d, dtype, layout)
    (Kc, Vc), (Ks, Vs) = cache(B, H, n, d, fmt, layout)
    wf.wf_cache_quantize(Kn, Vn, Kc, Ks, Vc, Vs, FMT[fmt], pos)
    at = slice(pos, pos + m)
    for new, c, s in ((Kn, Kc, Ks), (Vn, Vc, Vs)):
        codes, scales = mx.quantize(f64(new), fmt)
        want_c, want_s = np.full(c.shape, 0x5a, np.uint8), np.full(s.shape, 99, np.uint8)
        want_c[:, :, at], want_s[:, :, at] = mx.pack(codes, fmt), scales
        assert np.array_equal(c.cpu().numpy(), want_c)
        assert np.array_equal(s.cpu().numpy(), want_s)
    Ko, Vo = (lay(B, H, m, d, DT[dtype], layout) for _ in range(2))
    wf.wf_cache_dequantize(Kc, Ks, Vc, Vs, FMT[fmt], Ko, Vo, pos)
    for out, c, s in ((Ko, Kc, Ks), (Vo, Vc, Vs)):
        want = mx.values(c.cpu().numpy()[:, :, at], s.cpu().numpy()[:, :, at], fmt)
        assert np.array_equal(f64(out), want)  # 4 digits and a power of two: exact in bf16 too


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_alone_and_selected_rows(dtype, fmt):
    B, H, d, n, m = 2, 3, 128, 100, 37
    r = np.random.default_rng(5)
    Kn = rows(r, B, H, n, d, dtype, "bhsd")
    (Kc, Vc), (Ks, Vs) = cache(B, H, n, d, fmt, "bshd")
    wf.wf_cache_quantize(Kn, None, Kc, Ks, None, None, FMT[fmt], 0)
    assert (Vc == 0x5a).all() and (Vs == 99).all()
    idx = r.integers(-20, n + 20, (B * H, m)).astype(np.int32)  # any order, repeats, some out of range
    out = lay(B, H, m, d, DT[dtype], "bhsd")
    wf.wf_cache_dequantize(Kc, Ks, None, None, FMT[fmt], out, None, idx=torch.from_numpy(idx).cuda())
    all_rows = mx.values(Kc.cpu().numpy(), Ks.cpu().numpy(), fmt).reshape(B * H, n, d)
    want = np.stack([all_rows[u][idx[u].clip(0, n - 1)] for u in range(B * H)]).reshape(B, H, m, d)
    assert np.array_equal(f64(out), want)


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_blocks(dtype, fmt):
    # Zeros, subnormals, the largest values, exact limits of a scale and the next value, signed zeros, NaN and
    # infinities beside ordinary blocks.
    top = 448.0 if fmt == "mxfp8" else 6.0
    big = torch.finfo(DT[dtype]).max
    x = torch.randn(8, 128, generator=torch.Generator().manual_seed(6), dtype=torch.float64)
    x[0, :32] = 0
    x[0, 32:64] = -0.0
    x[1] *= 2.0 ** -133   # below the smallest normal number
    x[2] = x[2].clamp(-3, 3) / 3 * big
    x[2, 5] = big
    x[3, :32], x[3, 32:64] = top, top * (1 + 2.0 ** -7)
    x[4, 40], x[5, 127], x[6, 0] = float("nan"), float("inf"), -float("inf")
    x[7, :32] = torch.arange(32) * top / 62  # ties
    Kn = x.to(DT[dtype]).view(1, 1, 8, 128).cuda()
    (Kc, _), (Ks, _) = cache(1, 1, 8, 128, fmt, "bhsd")
    wf.wf_cache_quantize(Kn, None, Kc, Ks, None, None, FMT[fmt], 0)
    codes, scales = mx.quantize(f64(Kn), fmt)
    assert np.array_equal(Ks.cpu().numpy(), scales)
    assert np.array_equal(Kc.cpu().numpy(), mx.pack(codes, fmt))
    out = torch.empty(1, 1, 8, 128, dtype=torch.float32, device="cuda")
    wf.wf_cache_dequantize(Kc, Ks, None, None, FMT[fmt], out, None)
    want = mx.values(mx.pack(codes, fmt), scales, fmt)
    assert np.array_equal(f64(out), want.astype(np.float32).astype(float), equal_nan=True)
    assert np.isnan(want).sum() == 96


def test_rows_past_32_bits():
    # 2^25 + 40 rows of 128 codes: byte offsets beyond 2^32, a selection at both ends.
    n, d, m = (1 << 25) + 40, 128, 40
    Kc = torch.zeros(1, 1, n, d, dtype=torch.uint8, device="cuda")
    Ks = torch.zeros(1, 1, n, d // 32, dtype=torch.uint8, device="cuda")
    new = rows(np.random.default_rng(7), 1, 1, m, d, "bf16", "bhsd")
    wf.wf_cache_quantize(new, None, Kc, Ks, None, None, wf.WF_MXFP8, n - m)
    idx = torch.tensor([[n - 1, 0, n - m, n - 2]], dtype=torch.int32, device="cuda")
    out = torch.empty(1, 1, 4, d, dtype=torch.float32, device="cuda")
    wf.wf_cache_dequantize(Kc, Ks, None, None, wf.WF_MXFP8, out, None, idx=idx)
    codes, scales = mx.quantize(f64(new), "mxfp8")
    want = mx.values(codes, scales, "mxfp8")[0, 0]
    assert np.array_equal(f64(out)[0, 0], np.stack([want[-1], 0 * want[0], want[0], want[-2]]))
    assert int(Kc.view(-1)[: (n - m) * d].amax()) == 0


def test_on_a_stream_of_its_own():
    side = torch.cuda.Stream()
    r = np.random.default_rng(8)
    Kn = rows(r, 1, 4, 600, 128, "f32", "bhsd")
    (Kc, _), (Ks, _) = cache(1, 4, 600, 128, "mxfp8", "bhsd")
    out = torch.empty(1, 4, 600, 128, dtype=torch.float32, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    wf.wf_cache_quantize(Kn, None, Kc, Ks, None, None, wf.WF_MXFP8, 0, stream=side)
    with torch.cuda.stream(side):
        wf.wf_cache_dequantize(Kc, Ks, None, None, wf.WF_MXFP8, out, None)
    side.synchronize()
    codes, scales = mx.quantize(f64(Kn), "mxfp8")
    assert np.array_equal(f64(out), mx.values(codes, scales, "mxfp8"))
