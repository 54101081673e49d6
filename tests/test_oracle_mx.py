"""The CPU definitions of the quantised cache and of the attention over shared
prompts, pinned by facts that do not come from them: torch's float8 casts and
float8_e4m3fn values, rounding ties worked out by hand, the bound on a
rounding, and torch's float64 softmax."""
import numpy as np
import pytest
import torch

from oracle import mx


def test_e4m3_magnitudes_are_torchs():
    codes = torch.arange(127, dtype=torch.uint8)
    assert np.array_equal(mx.magnitudes("mxfp8"), codes.view(torch.float8_e4m3fn).double().numpy())


def test_e4m3_codes_are_torchs():
    # The block's largest value is 448, so the scale is 1 and the codes are those of the plain cast.
    r = np.random.default_rng(0)
    x = (r.standard_normal((64, 32)) * np.exp(r.uniform(-8, 4, (64, 1)))).clip(-448, 448).astype(np.float32)
    x[:, 7] = 448
    codes, scales = mx.quantize(x.astype(np.float64), "mxfp8")
    assert (scales == 127).all()
    assert np.array_equal(codes, torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_e2m1_ties_go_to_the_even_code():
    x = np.zeros((1, 32))
    x[0, :12] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -2.5, -5, 2.51]
    codes, scales = mx.quantize(x, "mxfp4")
    assert scales[0, 0] == 127
    want = [6, 0, 1, 1, 2, 2, 4, 4, 0, -2, -4, 3]
    assert mx.values(mx.pack(codes, "mxfp4"), scales, "mxfp4")[0, :12].tolist() == want


@pytest.mark.parametrize("fmt,top,digits", [("mxfp8", 448.0, 4), ("mxfp4", 6.0, 2)])
def test_scale_is_the_least_that_covers_the_block(fmt, top, digits):
    r = np.random.default_rng(1)
    x = r.standard_normal((200, 64)) * np.exp2(r.integers(-120, 110, (200, 1)).astype(float))
    x[0] = 0
    x[1, :32] = top                    # exactly covered by scale 1
    x[2, :32] = np.nextafter(top, 1e9)  # just not
    codes, scales = mx.quantize(x, fmt)
    assert scales[0].tolist() == [0, 0] and scales[1, 0] == 127 and scales[2, 0] == 128
    s = np.repeat(np.exp2(scales.astype(float) - 127), 32, -1)
    assert (np.abs(x) <= top * s).all()
    least = scales > 0
    assert (np.abs(x).reshape(200, 2, 32).max(-1)[least] > top * s[:, ::32][least] / 2).all()
    # The rounding: half a unit of the last of `digits` binary digits, or half the smallest magnitude.
    err = np.abs(mx.values(mx.pack(codes, fmt), scales, fmt) - x)
    smallest = mx.magnitudes(fmt)[1]
    assert (err <= np.maximum(np.abs(x) * 2.0 ** -digits, smallest * s / 2)).all()


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
def test_blocks_with_nan_or_infinity(fmt):
    x = np.ones((2, 96))
    x[0, 40], x[1, 95] = np.nan, -np.inf
    codes, scales = mx.quantize(x, fmt)
    v = mx.values(mx.pack(codes, fmt), scales, fmt)
    assert np.isnan(v[0, 32:64]).all() and np.isnan(v[1, 64:]).all()
    assert (v[0, :32] == 1).all() and (v[0, 64:] == 1).all() and (v[1, :64] == 1).all()


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
def test_quantising_its_own_values_changes_nothing(fmt):
    x = np.random.default_rng(2).standard_normal((50, 64))
    c, s = mx.quantize(x, fmt)
    v = mx.values(mx.pack(c, fmt), s, fmt)
    c2, s2 = mx.quantize(v, fmt)
    assert np.array_equal(v, mx.values(mx.pack(c2, fmt), s2, fmt))


def test_attention_is_torchs():
    g = torch.Generator().manual_seed(3)
    Q, K, V = (torch.randn(r, 16, generator=g, dtype=torch.float64) for r in (5, 40, 40))
    want = torch.softmax(Q @ K.T / 4, 1) @ V
    assert np.abs(mx.attention(Q.numpy(), K.numpy(), V.numpy()) - want.numpy()).max() < 1e-14
    assert (mx.attention(Q.numpy(), K[:0].numpy(), V[:0].numpy()) == 0).all()


def test_prefix_attention_is_attention_over_each_sequences_rows():
    g = torch.Generator().manual_seed(4)
    B, P, H, G, q, d, n, ng = 4, 2, 2, 3, 2, 8, 20, 5

    def t(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64).numpy()
    Q, K, V, Kg, Vg = t(B, H * G, q, d), t(P, H, n, d), t(P, H, n, d), t(B, H, ng, d), t(B, H, ng, d)
    idx = np.array([[3, 30, 0], [1, 1, 2], [5, -4, 7], [19, 18, 17]])
    got = mx.prefix_attention(Q, K, V, Kg, Vg, 3, idx, prefix_len=[2, 9], gen_len=[0, 5, 1, -2])
    # Sequence 1 (prompt 0, two rows), query head 4 (key head 1), all own rows.
    want = mx.attention(Q[1, 4], np.concatenate([K[0, 1, [1, 1]], Kg[1, 1]]), np.concatenate([V[0, 1, [1, 1]], Vg[1, 1]]))
    assert np.array_equal(got[1, 4], want)
    # Sequence 3 (prompt 1), query head 0: three clamped rows, no own row.
    want = mx.attention(Q[3, 0], K[1, 0, [5, 0, 7]], V[1, 0, [5, 0, 7]])
    assert np.array_equal(got[3, 0], want)
