"""Cosine and sine of a rotation as the outputs of the rows (1, 0): off by less than a step of 2^-24.

A turn is cut at 2^-32 (0.025 of 2^-24 as an angle).  An angle is held in two fp32 numbers, which leave nothing that
counts.  Of the sine, what is added to x is below 0.081 and off by 0.11 (its product), 0.06 (1/6), 0.065 (x^2) and 0.06
(its sum) of 2^-24 at most, and the first term left out is 0.03; the sum's rounding is half a step, 0.5.  Of the cosine
what 1 - x^2 / 2 rounds off is added back, and the rest is below 0.016, so less than 0.1 with the rounding of the sum, 0.5.
Together below 0.9."""
import math

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2606_00724_gb300 import wf

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_cosine_and_sine(d, adjacent):
    rows, pairs = 6000, d // 2
    freq = torch.cat([10000.0 ** (-torch.arange(pairs // 2, dtype=torch.float64) / (pairs // 2)),
                      2 * math.pi * torch.arange(1, pairs // 2 + 1, dtype=torch.float64) / rows])  # whole turns as well
    g = torch.Generator().manual_seed(101)
    pos = torch.cat([torch.arange(rows // 2), torch.randint(-(1 << 31), 1 << 31, (rows // 2,), generator=g)])
    pos = pos.to(torch.int32).view(1, 1, rows)
    a, b = (slice(0, d, 2), slice(1, d, 2)) if adjacent else (slice(0, pairs), slice(pairs, d))
    x = torch.zeros(1, 1, rows, d, device="cuda")
    x[..., a] = 1.0
    out = torch.empty_like(x)
    wf.wf_rotary_apply(x, None, wf.wf_rotary_plan(freq).cuda(), pos.cuda(), out, None, adjacent=adjacent)
    angle = np.array([[paged.angle(f, p) for f in freq.tolist()] for p in pos[0, 0].tolist()])
    out = out[0, 0].double().cpu().numpy()
    worst = max(np.abs(out[:, a] - np.cos(angle)).max(), np.abs(out[:, b] - np.sin(angle)).max()) * 2.0 ** 24
    assert worst <= 1.0, worst
