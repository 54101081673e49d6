"""wf_rotary_apply against the float64 definition: both types, head_dims, orders
of channels and memory, part of the channels, axes, far and negative positions,
in place, other streams and graphs.

Tolerances.  fp32: cosine and sine are those of an angle that is off by 2^-32 of a
turn (1.5e-9) and rounded to fp32 as a fraction (2^-25), by a function that is off
by a unit in the last place (2^-24 at most): below 2^-22.9 of (|x| + |y|) with the
rounding of one product; the sum's rounding adds half a step.  bf16: the
special-function unit is 2^-20.5 off, half a step of the output 2^-8 of it."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2606_00724_gb300 import wf

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def lay(t, layout):
    """[B, H, rows, d] in another order, or inside a wider tensor of NaN."""
    if layout == "bshd":
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "wide":
        B, H, S, d = t.shape
        view = torch.full((B, S + 1, H + 2, 2 * d), float("nan"), dtype=t.dtype, device=t.device)
        view = view.transpose(1, 2)[:, 1:H + 1, 1:, :d]
        view.copy_(t)
        return view
    return t.contiguous()


def tolerance(x, want, pairs, adjacent, dtype):
    """Per element, from the magnitudes of a pair."""
    if adjacent:
        a = np.abs(x[..., :2 * pairs]).reshape(*x.shape[:-1], pairs, 2).sum(-1).repeat(2, -1)
    else:
        a = np.tile(np.abs(x[..., :pairs]) + np.abs(x[..., pairs:2 * pairs]), 2)
    tol = np.zeros(x.shape)
    tol[..., :2 * pairs] = a * (2.0 ** -22 if dtype == "f32" else 2.0 ** -19)
    turned = np.abs(want) + tol
    turned[..., 2 * pairs:] = 0  # not rounded at all
    return tol + turned * (2.0 ** -24 if dtype == "f32" else 2.0 ** -8)


def inputs(B, rows, Hq, Hk, d, dtype, layout, axes, pairs, seed, lo=0, hi=5000):
    g = torch.Generator().manual_seed(seed)
    Q, K = (lay(torch.randn(B, H, rows, d, generator=g).to(DT[dtype]).cuda(), layout) for H in (Hq, Hk))
    pos = torch.randint(lo, hi, (axes, B, rows), generator=g).to(torch.int32)
    freq = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
    axis = (torch.arange(pairs) % axes).to(torch.int32)
    return Q, K, pos, freq, axis


def check(got, x, pos, freq, axis, adjacent, dtype):
    x = x.double().cpu().numpy()
    got = got.double().cpu().numpy()
    for b in range(x.shape[0]):
        want = paged.rotate(x[b], pos[:, b].numpy(), freq.tolist(), axis.tolist(), adjacent)
        assert (np.abs(got[b] - want) <= tolerance(x[b], want, len(freq), adjacent, dtype)).all()


SHAPES = [  # B, rows, Hq, Hk, d, pairs, axes
    (1, 1, 1, 1, 64, 8, 1),
    (32, 1, 32, 8, 128, 64, 1),
    (3, 37, 7, 1, 128, 32, 2),
    (2, 130, 28, 4, 64, 32, 3),
    (1, 3000, 5, 2, 128, 64, 3),
    (2, 1500, 40, 8, 128, 16, 1),
    (5, 11, 3, 3, 64, 24, 4),
]


@pytest.mark.parametrize("layout", ["bhsd", "bshd", "wide"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype, adjacent, layout):
    B, rows, Hq, Hk, d, pairs, axes = shape
    Q, K, pos, freq, axis = inputs(B, rows, Hq, Hk, d, dtype, layout, axes, pairs, seed=rows)
    Qo, Ko = (lay(torch.full_like(x, float("nan")), layout) for x in (Q, K))
    wf.wf_rotary_apply(Q, K, wf.wf_rotary_plan(freq, axis).cuda(), pos.cuda(), Qo, Ko, adjacent=adjacent)
    some = slice(0, None, max(1, rows // 60))  # the definition is slow
    for x, y in ((Q, Qo), (K, Ko)):
        assert not torch.isnan(y).any()
        check(y[:, :3, some], x[:, :3, some], pos[:, :, some], freq, axis, adjacent, dtype)
        check(y[:, -1:, -40:], x[:, -1:, -40:], pos[:, :, -40:], freq, axis, adjacent, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions(dtype):
    Q, K, pos, freq, axis = inputs(2, 60, 2, 1, 128, dtype, "bhsd", 1, 64, seed=1, lo=-2 ** 31, hi=2 ** 31)
    pos[0, 0, :6] = torch.tensor([2 ** 31 - 1, -2 ** 31, 0, 1, -1, 1 << 20])
    freq[0], freq[1] = 3.5, -1e6  # more than a turn a position, and backwards
    Qo, Ko = torch.empty_like(Q), torch.empty_like(K)
    wf.wf_rotary_apply(Q, K, wf.wf_rotary_plan(freq).cuda(), pos.cuda(), Qo, Ko)
    check(Qo, Q, pos, freq, axis, False, dtype)
    check(Ko, K, pos, freq, axis, False, dtype)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_queries_alone_and_back(dtype, adjacent):
    Q, K, pos, freq, axis = inputs(2, 333, 9, 2, 128, dtype, "bshd", 2, 32, seed=2)
    plan, pos_d = wf.wf_rotary_plan(freq, axis).cuda(), pos.cuda()
    Qo, Ko = torch.empty_like(Q), torch.empty_like(K)
    wf.wf_rotary_apply(Q, K, plan, pos_d, Qo, Ko, adjacent=adjacent)
    alone = torch.empty_like(Q)
    wf.wf_rotary_apply(Q, None, plan, pos_d, alone, None, adjacent=adjacent)
    assert torch.equal(alone, Qo)
    q, k = Q.clone(), K.clone()
    wf.wf_rotary_apply(q, k, plan, pos_d, q, k, adjacent=adjacent)
    assert torch.equal(q, Qo) and torch.equal(k, Ko)
    if dtype == "f32":  # by -p: back, to two rotations' errors of a vector no longer than the first
        wf.wf_rotary_apply(q, k, plan, -pos_d, q, k, adjacent=adjacent)
        long = Q.abs().max().item()
        assert (q - Q).abs().max().item() <= 2 * 2 * 1.5 * long * (2.0 ** -22 + 2.0 ** -24)


def test_gradient_is_the_rotation_back():
    # d/dx of <g, R x> is R^T g: against differences of the definition, which is linear, so a unit step is exact.
    Q, _, pos, freq, axis = inputs(1, 4, 1, 1, 64, "f32", "bhsd", 1, 16, seed=3)
    g = torch.randn(Q.shape, generator=torch.Generator().manual_seed(4)).cuda()
    out = torch.empty_like(g)
    wf.wf_rotary_apply(g, None, wf.wf_rotary_plan(freq, axis).cuda(), (-pos).cuda(), out, None)
    x, gn = Q[0].double().cpu().numpy(), g[0].double().cpu().numpy()
    base = (gn * paged.rotate(x, pos[:, 0].numpy(), freq.tolist(), axis.tolist())).sum((0, 2))
    for c in range(64):
        step = x.copy()
        step[..., c] += 1
        d = (gn * paged.rotate(step, pos[:, 0].numpy(), freq.tolist(), axis.tolist())).sum((0, 2)) - base
        assert (np.abs(out[0, 0, :, c].double().cpu().numpy() - d) <= 2.0 ** -20 * np.abs(gn).max()).all()


def test_a_nan_or_an_infinity_stays_with_its_pair():
    Q, K, pos, freq, axis = inputs(1, 50, 2, 2, 128, "bf16", "bhsd", 1, 32, seed=5)
    plan = wf.wf_rotary_plan(freq, axis).cuda()
    a, b = torch.empty_like(Q), torch.empty_like(Q)
    wf.wf_rotary_apply(Q, None, plan, pos.cuda(), a, None)
    Q[0, 1, 7, 3], Q[0, 0, 9, 100] = float("nan"), float("inf")
    wf.wf_rotary_apply(Q, None, plan, pos.cuda(), b, None)
    same = torch.ones_like(Q, dtype=torch.bool)
    same[0, 1, 7, [3, 35]] = same[0, 0, 9, 100] = False
    assert torch.equal(a[same], b[same])
    assert torch.isnan(b[0, 1, 7, [3, 35]]).all() and b[0, 0, 9, 100] == float("inf")


def test_an_axis_that_positions_lack_is_the_last():
    Q, K, pos, freq, axis = inputs(1, 20, 1, 1, 64, "f32", "bhsd", 1, 16, seed=6)
    a, b = torch.empty_like(Q), torch.empty_like(Q)
    wf.wf_rotary_apply(Q, None, wf.wf_rotary_plan(freq, axis + 5).cuda(), pos.cuda(), a, None)
    wf.wf_rotary_apply(Q, None, wf.wf_rotary_plan(freq).cuda(), pos.cuda(), b, None)
    assert torch.equal(a, b)


def test_no_rows_another_stream_and_a_graph():
    Q, K, pos, freq, axis = inputs(2, 100, 4, 2, 128, "bf16", "bhsd", 1, 64, seed=7)
    plan, pos = wf.wf_rotary_plan(freq, axis).cuda(), pos.cuda()
    wf.wf_rotary_apply(Q[:, :, :0], K[:, :, :0], plan, pos[:, :, :0].contiguous(), Q[:, :, :0], K[:, :, :0])
    want, got, Ko = torch.empty_like(Q), torch.zeros_like(Q), torch.zeros_like(K)
    wf.wf_rotary_apply(Q, None, plan, pos, want, None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    wf.wf_rotary_apply(Q, K, plan, pos, got, Ko, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    got.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wf.wf_rotary_apply(Q, K, plan, pos, got, Ko)
    pos.add_(1)  # a replay reads what is there then
    wf.wf_rotary_apply(Q, None, plan, pos, want, None)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_rows_past_32_bits():
    # 2^31 elements and more between the first and the last row.
    rows, d = (1 << 25) + 3, 64
    Q = torch.zeros(1, 1, rows, d, dtype=torch.bfloat16, device="cuda")
    x = torch.randn(1, 1, 5, d, generator=torch.Generator().manual_seed(8)).bfloat16()
    Q[:, :, -5:] = x.cuda()
    freq = 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda").view(1, 1, rows)
    wf.wf_rotary_apply(Q, None, wf.wf_rotary_plan(freq).cuda(), pos, Q, None)
    check(Q[:, :, -5:], x, pos[:, :, -5:].cpu(), freq, torch.zeros(32, dtype=torch.int32), False, "bf16")
    assert not Q[:, :, :-5].any()
