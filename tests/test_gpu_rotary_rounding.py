"""How far a rotation is off before it is rounded: the same for both types, since both go through one fp32 series.

An angle beyond its nearest quarter turn is x, |x| <= pi / 4: a whole number rounded to fp32, times a rounded constant,
rounded, so 3 2^-24 of x, which moves a cosine or a sine by at most 3 2^-24 x cos x < 1.67 2^-24 (x cos x and x sin x
are below 0.556); the turn that the whole number leaves out is 2^-32, 2^-29.3 of an angle.  The series' own rounding is
half a step of numbers up to 1, 2^-25, and below 2^-26 of what is added to it.  So cosine and sine are off by less than
2.5 2^-24, the product that is rounded by 2^-24 more, together below 2^-22 of |x| + |y|.  The sum's rounding is 2^-24 of
it, and for bf16 the output's 2^-8."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2606_00724_gb300 import wf
from test_gpu_rotary import DT

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cancel", [False, True])
def test_rounded_once_from_fp32(cancel, dtype, adjacent):
    rows, d, pairs = 400, 128, 64
    g = torch.Generator().manual_seed(61)
    x = torch.randn(1, 1, rows, d, generator=g, dtype=torch.float64).to(DT[dtype])
    freq = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
    pos = torch.randint(1, 1 << 20, (1, 1, rows), generator=g).to(torch.int32)
    a, b = (slice(0, d, 2), slice(1, d, 2)) if adjacent else (slice(0, pairs), slice(pairs, d))
    if cancel:  # the first channel of a pair all but cancels
        angle = np.array([[paged.angle(f, p) for f in freq.tolist()] for p in pos[0, 0].tolist()])
        tan = torch.from_numpy(np.tan(angle))
        x[0, 0, :, a] = (x[0, 0, :, b].double() * tan).clamp(-1e4, 1e4).to(DT[dtype])
    out = torch.empty_like(x, device="cuda")
    wf.wf_rotary_apply(x.cuda(), None, wf.wf_rotary_plan(freq).cuda(), pos.cuda(), out, None, adjacent=adjacent)
    x, got = x[0].double().numpy(), out[0].double().cpu().numpy()
    want = paged.rotate(x, pos[:, 0].numpy(), freq.tolist(), [0] * pairs, adjacent)
    sums = np.abs(x[..., a]) + np.abs(x[..., b])
    tol = np.zeros(x.shape)
    tol[..., a] = tol[..., b] = sums * 2.0 ** -22
    step = 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    err, bound = np.abs(got - want), tol + (np.abs(want) + tol) * step
    assert (err <= bound).all(), (err / bound).max()
