"""wf_prefix_attn against the float64 definition: both types and head_dims,
prompts in 32 and 16 bits and quantised, whole and selected, shared by one to
many sequences, one to many query rows, lengths of zero and one, and what must
not cross from one sequence to another."""
import numpy as np
import pytest
import torch

from helpers import assert_close_out
from oracle import mx
from paper_2606_00724_gb300 import wf

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

FMT = {"mxfp8": wf.WF_MXFP8, "mxfp4": wf.WF_MXFP4}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.double().cpu().numpy()


def lay(t, layout):
    t = t.cuda()
    if layout == "bshd":
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "wide":
        wide = torch.full((*t.shape[:2], t.shape[2] + 3, 2 * t.shape[3]), float("nan")).to(t.dtype).cuda()
        view = wide[:, :, 1:t.shape[2] + 1, :t.shape[3]]
        view.copy_(t)
        return view
    return t


class Case:
    def __init__(self, B, P, H, G, q, d, n, ng, dtype="bf16", cache=None, k=None, select=False, layout="bhsd",
                 plen=None, glen=None, seed=0, spread=1.0, scale=0.0):
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]

        def draw(*shape, by=1.0):
            return (torch.randn(*shape, generator=g, dtype=torch.float64) * by).to(dt)
        self.scale = scale
        self.Q = lay(draw(B, H * G, q, d, by=spread), layout)
        K, V = draw(P, H, n, d), draw(P, H, n, d)
        self.Kg = self.Vg = None
        if ng:
            self.Kg, self.Vg = lay(draw(B, H, ng, d), layout), lay(draw(B, H, ng, d), layout)
        self.Ks = self.Vs = self.fmt = None
        if cache:
            self.fmt = FMT[cache]
            (kc, ks), (vc, vs) = mx.quantize(f64(K), cache), mx.quantize(f64(V), cache)
            kc, vc = mx.pack(kc, cache), mx.pack(vc, cache)
            self.K64, self.V64 = mx.values(kc, ks, cache), mx.values(vc, vs, cache)
            self.K, self.V = (lay(torch.from_numpy(c), layout if layout != "wide" else "bshd") for c in (kc, vc))
            self.Ks, self.Vs = (torch.from_numpy(s).cuda() for s in (ks, vs))
        else:
            self.K64, self.V64 = f64(K), f64(V)
            self.K, self.V = lay(K, layout), lay(V, layout)
        self.k = n if k is None else k
        self.idx = None
        if select:
            r = np.random.default_rng(seed)
            self.idx = torch.from_numpy(r.integers(-3, n + 3, (P * H, self.k)).astype(np.int32)).cuda()
        self.plen = None if plen is None else torch.tensor(plen, dtype=torch.int32).cuda()
        self.glen = None if glen is None else torch.tensor(glen, dtype=torch.int32).cuda()
        self.ng = ng

    def run(self, stream=None):
        size = wf.wf_prefix_attn_workspace_bytes(self.Q, self.K, self.k, self.ng, fmt=self.fmt)
        ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")  # scratch may hold anything
        ws[:4] = 0
        O = torch.full_like(self.Q, float("nan"))
        torch.cuda.synchronize()
        wf.wf_prefix_attn(self.Q, self.K, self.V, self.k, self.Kg, self.Vg, O, ws, idx=self.idx, prefix_len=self.plen,
                          gen_len=self.glen, Ks=self.Ks, Vs=self.Vs, fmt=self.fmt, scale=self.scale, stream=stream)
        wf.wf_workspace_status(ws, stream)
        return O

    def want(self):
        at = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        return mx.prefix_attention(f64(self.Q), self.K64, self.V64, None if self.Kg is None else f64(self.Kg),
                                   None if self.Vg is None else f64(self.Vg), self.k, at(self.idx), at(self.plen),
                                   at(self.glen), self.scale or None)

    def check(self):
        O = self.run()
        assert_close_out(f64(O), self.want(), self.Q.dtype)
        return O


SHAPES = [  # B, P, H, G, q, n, ng
    (1, 1, 1, 1, 1, 1, 0),        # one token, one key
    (1, 1, 2, 1, 1, 0 + 5, 1),
    (3, 3, 2, 1, 1, 129, 2),      # every sequence a prompt of its own
    (4, 1, 4, 1, 1, 1001, 7),
    (5, 1, 2, 3, 1, 300, 65),     # grouped heads, 15 rows
    (2, 2, 2, 7, 1, 700, 0),
    (6, 2, 3, 1, 24, 515, 17),    # 72 rows
    (4, 1, 2, 1, 32, 1024, 32),   # 128 rows
    (9, 3, 1, 2, 33, 250, 40),    # 198 rows
    (8, 1, 2, 1, 64, 640, 130),   # 512 rows
    (5, 1, 1, 7, 11, 2500, 64),   # 385 rows
    (1, 1, 1, 1, 300, 200, 300),  # a long block of one sequence
    (40, 1, 3, 1, 1, 127, 128),
    (2, 1, 40, 1, 4, 64, 3),
    (3, 1, 2, 1, 1, 90, 1300),    # long generations
    (2, 1, 2, 2, 20, 260, 700),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype, d):
    B, P, H, G, q, n, ng = shape
    Case(B, P, H, G, q, d, n, ng, dtype, seed=n + q).check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cache", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("shape", [SHAPES[i] for i in (0, 3, 5, 6, 9, 10)])
def test_quantised_prompts(shape, cache, dtype, d):
    B, P, H, G, q, n, ng = shape
    Case(B, P, H, G, q, d, n, ng, dtype, cache, seed=n, layout="bshd").check()


@pytest.mark.parametrize("cache", [None, "mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bhsd", "bshd", "wide"])
def test_selected_rows(layout, dtype, cache):
    Case(4, 2, 3, 2, 5, 128, 400, 9, dtype, cache, k=333, select=True, layout=layout, seed=1).check()
    Case(6, 1, 2, 1, 32, 64, 300, 0, dtype, cache, k=1, select=True, layout=layout, seed=2).check()


@pytest.mark.parametrize("cache", [None, "mxfp8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 32])
def test_lengths(q, dtype, cache):
    # Lengths of zero, one, below zero and beyond the end; rows with nothing to attend to are 0.
    c = Case(8, 4, 2, 2, q, 128, 700, 40, dtype, cache, k=650, plen=[0, 1, 130, 9999],
             glen=[0, 3, 1, 40, -5, 77, 12, 0], seed=3)
    O = c.check()
    assert (O[0] == 0).all() and not (O[1] == 0).any()
    c = Case(4, 2, 2, 1, q, 64, 300, 5, dtype, cache, plen=[0, 0], glen=[0, 0, 0, 5], seed=4)
    O = c.check()
    assert (O[:3] == 0).all() and not (O[3] == 0).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_prompt_rows_at_all(dtype):
    Case(4, 2, 2, 1, 3, 128, 10, 12, dtype, k=0, seed=5).check()
    O = Case(4, 2, 2, 1, 3, 128, 10, 0, dtype, k=0, seed=5).check()
    assert (O == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 40])
def test_steep_softmax_and_scale(q, dtype):
    # Logits of a spread of about 30, and an explicit scale.
    Case(4, 1, 2, 2, q, 128, 1500, 33, dtype, seed=6, spread=30.0).check()
    Case(4, 1, 2, 2, q, 64, 500, 33, dtype, seed=7, scale=0.5).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 20, 64])
def test_nan_and_infinity_stay_with_their_rows(q, dtype):
    c = Case(8, 2, 2, 2, q, 128, 400, 50, dtype, plen=[400, 390], glen=[50, 20, 50, 0, 50, 50, 1, 50], seed=8)
    before = c.run()
    nan = float("nan")
    c.Vg[0, 0, 3] = nan           # sequence 0, key head 0
    c.Kg[2, 1, 49] = nan          # sequence 2, key head 1
    c.Vg[4, 0, 7] = float("inf")  # sequence 4, key head 0
    c.K[1, 1, 391:] = nan         # past the length of prompt 1
    c.V[1, 1, 390:] = float("inf")
    c.Kg[1, :, 20:] = nan         # past the length of sequence 1
    c.Vg[3] = nan
    after = c.run()
    touched = torch.zeros(8, 4, dtype=torch.bool)
    touched[0, :2] = touched[2, 2:] = touched[4, :2] = True
    assert torch.equal(after[~touched], before[~touched])
    assert torch.isnan(after[0, :2, :, :]).all() and torch.isnan(after[2, 2:]).all()
    assert (~torch.isfinite(after[4, :2])).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_in_one_prompt_stays_with_its_sequences(dtype):
    c = Case(6, 3, 2, 1, 9, 64, 200, 4, dtype, seed=9)
    before = c.run()
    c.V[1, 0, 77] = float("nan")
    after = c.run()
    assert torch.isnan(after[2:4, 0]).all()
    assert torch.equal(after[[0, 1, 4, 5]], before[[0, 1, 4, 5]]) and torch.equal(after[2:4, 1], before[2:4, 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_of_minus_infinity_add_nothing(dtype):
    c = Case(2, 1, 1, 1, 4, 64, 300, 70, dtype, seed=10)
    c.Q[..., 0] = 1.0
    c.K[0, 0, :200, 0] = -float("inf")      # the first tiles, keys in between
    c.Kg[0, 0, 3, 0] = -float("inf")
    c.K64, c.V64 = f64(c.K), f64(c.V)
    c.check()
    c.K[..., 0] = c.Kg[..., 0] = -float("inf")   # nothing else left
    assert (c.run() == 0).all()


@pytest.mark.parametrize("cache", [None, "mxfp4"])
def test_same_bits_again_and_on_another_stream(cache):
    c = Case(16, 1, 4, 1, 32, 128, 3000, 40, "bf16", cache, seed=11)
    first = c.run()
    assert torch.equal(c.run(), first)
    side = torch.cuda.Stream()
    assert torch.equal(c.run(stream=side), first)
    with torch.cuda.stream(side):
        again = c.run()
        side.synchronize()
    assert torch.equal(again, first)


def test_long_prompt_past_32_bits():
    # 2^25 rows of 128 codes: byte offsets beyond 2^32; rows at both ends selected.
    n, d = (1 << 25) + 64, 128
    codes = torch.zeros(1, 1, n, d, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(1, 1, n, d // 32, dtype=torch.uint8, device="cuda")
    g = torch.Generator().manual_seed(12)
    x = torch.randn(1, 1, 50, d, generator=g)
    c, s = mx.quantize(x.double().numpy(), "mxfp8")
    codes[:, :, -50:], scales[:, :, -50:] = torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()
    v = mx.values(c, s, "mxfp8")[0, 0]
    idx = torch.arange(n - 50, n, dtype=torch.int32, device="cuda").view(1, 50)
    for dtype in ("bf16", "f32"):
        Q = torch.randn(2, 1, 3, d, generator=g).to(DT[dtype]).cuda()
        O = torch.empty_like(Q)
        ws = torch.zeros(wf.wf_prefix_attn_workspace_bytes(Q, codes, 50, 0, fmt=wf.WF_MXFP8), dtype=torch.uint8,
                         device="cuda")
        wf.wf_prefix_attn(Q, codes, codes, 50, None, None, O, ws, idx=idx, Ks=scales, Vs=scales, fmt=wf.WF_MXFP8)
        want = np.stack([mx.attention(f64(Q)[b, 0], v, v) for b in range(2)])[:, None]
        assert_close_out(f64(O), want, Q.dtype)


def test_captured_in_a_graph():
    c = Case(4, 1, 2, 1, 16, 128, 2000, 20, "bf16", seed=13)
    want = c.run()
    ws = torch.zeros(wf.wf_prefix_attn_workspace_bytes(c.Q, c.K, c.k, c.ng), dtype=torch.uint8, device="cuda")
    O = torch.zeros_like(c.Q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wf.wf_prefix_attn(c.Q, c.K, c.V, c.k, c.Kg, c.Vg, O, ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, want)


@pytest.mark.parametrize("cache", [None, "mxfp8"])
@pytest.mark.parametrize("B", [2, 12])
def test_a_wait_that_gives_up_is_reported(B, cache):
    # The first wait of every CTA is on a barrier that nothing completes: the call ends, the status word is set, and
    # the next call works.
    c = Case(B, 1, 2, 1, 32, 128, 700, 20, "bf16", cache, seed=14)
    want = c.run()
    wf.wf_testing_set_wait_failure(True, 20000)
    try:
        with pytest.raises(wf.WfError) as e:
            c.run()
        assert e.value.status == -7
    finally:
        wf.wf_testing_set_wait_failure(False, 0)
    assert torch.equal(c.run(), want)


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_code_and_scale_is_read_exactly(dtype, fmt):
    # One prompt row a unit: the weight is 1, so O is the value row, to the bit.  Unit h holds every code, the scale
    # bytes go through 0 (2^-127) to 254; bf16 rounds what lies below its smallest normal number to nearest even.
    d, H = 128, 255
    codes = np.concatenate([np.arange(127), [0], np.arange(128, 255), [0]]).astype(np.uint8)
    V = np.zeros((1, H, 1, d if fmt == "mxfp8" else d // 2), np.uint8)
    for h in range(H):
        V[0, h, 0] = np.roll(codes, 37 * h)[:d] if fmt == "mxfp8" else (np.arange(d // 2) * 7 + h) % 256
    S = np.repeat(np.arange(H, dtype=np.uint8)[None, :, None, None], 4, axis=3)
    want = torch.from_numpy(mx.values(V, S, fmt))[:, :, 0]
    K = np.zeros_like(V)
    one = np.full_like(S, 127)
    Q = torch.ones(1, H, 1, d, dtype=DT[dtype], device="cuda")
    K, V, one, S = (torch.from_numpy(x).cuda() for x in (K, V, one, S))
    O = torch.empty_like(Q)
    ws = torch.zeros(wf.wf_prefix_attn_workspace_bytes(Q, K, 1, 0, fmt=FMT[fmt]), dtype=torch.uint8, device="cuda")
    wf.wf_prefix_attn(Q, K, V, 1, None, None, O, ws, Ks=one, Vs=S, fmt=FMT[fmt])
    normal = (want == 0) | ((want.abs() >= 2.0 ** -126) & (want.abs() <= torch.finfo(DT[dtype]).max))
    got = O.double().cpu()[:, :, 0]
    assert torch.equal(got[normal], want[normal])
    assert normal.double().mean() > 0.9


@pytest.mark.parametrize("cache", [None, "mxfp8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [2, 8])
def test_nan_key_reaches_every_row_that_attends_to_it(B, dtype, cache):
    # A key row with a NaN (a NaN scale in a quantised prompt) makes every query row of its key head NaN and no other.
    c = Case(B, 2, 2, 1, 32, 128, 500, 10, dtype, cache, seed=15)
    before = c.run()
    if cache:
        c.Ks[0, 1, 300, 2] = 255
    else:
        c.K[0, 1, 300, 70] = float("nan")
    after = c.run()
    assert torch.isnan(after[:B // 2, 1]).all()
    assert torch.equal(after[B // 2:], before[B // 2:]) and torch.equal(after[:, 0], before[:, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rising_logits(dtype):
    # Keys ordered so that a row's maximum rises from tile to tile, by little and by much, up to logits of about 80.
    c = Case(3, 1, 1, 1, 64, 128, 1100, 100, dtype, seed=16)
    rise = torch.linspace(0, 1, 1100).pow(3) * 7 + 0.3
    c.K[0, 0] = (f := c.Q[0, 0, 0].float())[None] / f.norm() * 11.3 * rise.cuda()[:, None] + 0.05 * c.K[0, 0].float()
    c.K64 = f64(c.K)
    c.check()
