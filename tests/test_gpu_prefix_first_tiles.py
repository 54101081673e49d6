"""wf_prefix_attn from codes, few key tiles and at most 128 stacked query rows: two warps take every other tile out of
four stages, and the first tiles of either may arrive before the other's.  The same bits every time."""
import pytest
import torch

from paper_2606_00724_gb300 import wf

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

FMT = {"mxfp8": wf.WF_MXFP8, "mxfp4": wf.WF_MXFP4}


@pytest.mark.parametrize("cache", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("k", [300, 385, 640, 5000])
def test_the_same_bits_every_time(k, cache):
    B, H, G, q, d = 4, 40, 2, 12, 128
    g = torch.Generator(device="cuda").manual_seed(93)
    draw = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    Q, K, V, Kg, Vg = draw(B, H * G, q, d), draw(1, H, k, d), draw(1, H, k, d), draw(B, H, q, d), draw(B, H, q, d)
    codes = [torch.zeros(1, H, k, d if cache == "mxfp8" else d // 2, dtype=torch.uint8, device="cuda") for _ in "KV"]
    scales = [torch.zeros(1, H, k, d // 32, dtype=torch.uint8, device="cuda") for _ in "KV"]
    wf.wf_cache_quantize(K, V, codes[0], scales[0], codes[1], scales[1], FMT[cache], 0)
    # What the codes stand for, attended to in 64 bits.
    wf.wf_cache_dequantize(codes[0], scales[0], codes[1], scales[1], FMT[cache], K, V)
    keys, values = (torch.cat([a.double().expand(B, -1, -1, -1), b.double()], 2).repeat_interleave(G, 1)
                    for a, b in ((K, Kg), (V, Vg)))
    p = torch.softmax(Q.double() @ keys.transpose(2, 3) / d ** 0.5, -1)
    want, A = p @ values, p @ values.abs()
    ws = torch.zeros(wf.wf_prefix_attn_workspace_bytes(Q, codes[0], k, q, fmt=FMT[cache]), dtype=torch.uint8, device="cuda")
    first = None
    for _ in range(40):
        O = torch.full_like(Q, float("nan"))
        wf.wf_prefix_attn(Q, codes[0], codes[1], k, Kg, Vg, O, ws, Ks=scales[0], Vs=scales[1], fmt=FMT[cache])
        first = O if first is None else first
        assert torch.equal(O, first)
    wf.wf_workspace_status(ws)
    # The output's rounding, the weights' and fp32's share of logits and sums, as wf_tree_attn's tests derive them.
    assert ((first.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -11) * A).all()
