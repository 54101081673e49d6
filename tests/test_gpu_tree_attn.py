"""wf_tree_attn against the float64 definition: both types and head_dims, pages of
any size in any order, caches in 32 and 16 bits and quantised, trees, chains and
blocks, lengths of zero and one, rows that see nothing, and what must not cross
from one row or sequence to another.  Pages that no sequence has and rows behind a
length hold NaN throughout.

Tolerances, with A the same weights' mean of |V|.  bf16: the output is rounded
(2^-8 of it), and so is each weight (2^-8 of A); products of up to 128 channels
summed in fp32 move a logit of such inputs by less than 2^-13, and so a weight and
the sum of weights, together 2^-12 of A, doubled for what else is fp32.  fp32: sums
of n weights and products, n 2^-24 of A at most, and as much as 128 of them for the
logits."""
import numpy as np
import pytest
import torch

from oracle import mx, paged
from paper_2606_00724_gb300 import wf
from test_gpu_rotary import DT, lay

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

FMT = {"mxfp8": wf.WF_MXFP8, "mxfp4": wf.WF_MXFP4}


def f64(t):
    return t.double().cpu().numpy()


def words(sees):
    """[B, q, n_t] truth values as [B, q, words] int32."""
    B, q, n = sees.shape
    bits = np.zeros((B, q, -(-n // 32) * 32), np.uint32)
    bits[..., :n] = sees
    w = (bits.reshape(B, q, -1, 32) << np.arange(32, dtype=np.uint32)).sum(-1).astype(np.uint32)
    return torch.from_numpy(w.view(np.int32)).cuda()


def tree_mask(r, B, q, n_t, shape):
    """Trees or chains of n_t nodes, of which the q query rows are the first (or see what node i % n_t sees)."""
    if shape == "block":
        return None
    sees = np.zeros((B, n_t, n_t), bool)
    for b in range(B):
        for i in range(n_t):
            if i:
                sees[b, i] = sees[b, i - 1 if shape == "chain" else int(r.integers(0, i))]
            sees[b, i, i] = True
    return sees[:, np.arange(q) % n_t]


class Case:
    def __init__(self, B, H, G, q, d, n, ps, n_t, dtype="bf16", cache=None, shape="tree", layout="bhsd", clen=None,
                 tlen=None, seed=0, spread=1.0, scale=0.0):
        r, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        dt = DT[dtype]

        def draw(*s, by=1.0):
            return (torch.randn(*s, generator=g, dtype=torch.float64) * by).to(dt)
        self.scale, self.n, self.n_t, self.cache, self.fmt = scale, n, n_t, cache, FMT.get(cache)
        self.Q = lay(draw(B, H * G, q, d, by=spread).cuda(), layout)
        entries = -(-n // ps) + 2
        pool = B * entries + 2
        self.pages = torch.randperm(pool, generator=g)[:B * entries].view(B, entries).to(torch.int32)
        self.clen, self.tlen = clen, tlen
        lens = [n if clen is None else min(n, max(0, c)) for c in (clen or [0] * B)]
        K, V = draw(pool, H, ps, d), draw(pool, H, ps, d)
        used = torch.zeros(pool, ps, dtype=torch.bool)
        for b in range(B):
            j = torch.arange(lens[b])
            used[self.pages[b, j // ps].long(), j % ps] = True
            self.pages[b, -(-lens[b] // ps):] = torch.tensor([-1, 2 ** 31 - 1, pool])[b % 3]
        self.Ks = self.Vs = None
        if cache:
            (kc, ks), (vc, vs) = mx.quantize(f64(K), cache), mx.quantize(f64(V), cache)
            kc, vc = mx.pack(kc, cache), mx.pack(vc, cache)
            self.K64, self.V64 = mx.values(kc, ks, cache), mx.values(vc, vs, cache)
            self.K, self.V = (lay(torch.from_numpy(c).cuda(), "bshd" if layout == "bshd" else "bhsd") for c in (kc, vc))
            self.Ks, self.Vs = (torch.from_numpy(s).cuda() for s in (ks, vs))
            for s in (self.Ks, self.Vs):
                s.transpose(1, 2)[~used.cuda()] = 255  # NaN
        else:
            self.K64, self.V64 = f64(K), f64(V)
            for t in (K, V):
                t.transpose(1, 2)[~used] = float("nan")
            self.K, self.V = lay(K.cuda(), layout), lay(V.cuda(), layout)
        self.Kt = self.Vt = self.sees = None
        if n_t:
            self.Kt, self.Vt = draw(B, H, n_t, d), draw(B, H, n_t, d)
            for b in range(B):
                if tlen is not None:
                    self.Kt[b, :, max(0, tlen[b]):] = self.Vt[b, :, max(0, tlen[b]):] = float("nan")
            self.Kt, self.Vt = lay(self.Kt.cuda(), layout), lay(self.Vt.cuda(), layout)
            self.sees = tree_mask(r, B, q, n_t, shape)

    def args(self):
        ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
        return dict(cache_len=ints(self.clen), tree_len=ints(self.tlen),
                    mask=None if self.sees is None else words(self.sees), Ks=self.Ks, Vs=self.Vs, fmt=self.fmt,
                    scale=self.scale)

    def workspace(self):
        size = wf.wf_tree_attn_workspace_bytes(self.Q, self.K, self.n, self.n_t, fmt=self.fmt)
        ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")  # scratch may hold anything
        ws[:4] = 0
        return ws

    def run(self, stream=None):
        ws, O, args, pages = self.workspace(), torch.full_like(self.Q, float("nan")), self.args(), self.pages.cuda()
        torch.cuda.synchronize()
        wf.wf_tree_attn(self.Q, self.K, self.V, pages, self.n, self.Kt, self.Vt, O, ws, stream=stream, **args)
        wf.wf_workspace_status(ws, stream)
        return O

    def want(self, absolute=False):
        return paged.tree_attention(f64(self.Q), self.K64, self.V64, self.pages.numpy(), self.n,
                                    None if self.Kt is None else f64(self.Kt), None if self.Vt is None else f64(self.Vt),
                                    self.clen, self.tlen, self.sees, self.scale or None, absolute)

    def check(self):
        O = self.run()
        want, A = self.want(), self.want(True)
        err = np.abs(f64(O) - want)
        if self.Q.dtype == torch.bfloat16:
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -11) * A
        else:
            tol = 2.0 ** -24 * np.abs(want) + (self.n + self.n_t + 256) * 2.0 ** -24 * A
        assert (err <= tol + 1e-30).all(), f"{(err / (tol + 1e-30)).max():.3g} of the tolerance"
        return O


SHAPES = [  # B, H, G, q, n, ps, n_t
    (1, 1, 1, 1, 0, 1, 1),          # one token, nothing but itself
    (1, 1, 1, 1, 1, 1, 0),          # one token, one key
    (3, 2, 1, 1, 130, 1, 1),        # pages of one row
    (2, 2, 4, 1, 515, 16, 1),
    (4, 1, 7, 1, 1001, 24, 1),      # pages that end inside a tile
    (2, 2, 2, 7, 300, 100, 7),
    (5, 3, 1, 16, 129, 128, 16),
    (2, 1, 4, 5, 2050, 64, 5),      # 20 rows a key head
    (2, 1, 7, 26, 700, 64, 26),     # 182
    (1, 2, 4, 64, 1100, 32, 64),    # 256
    (2, 2, 1, 80, 333, 16, 80),
    (3, 1, 5, 33, 64, 24, 33),      # 165, one word and a bit of the mask
    (1, 1, 1, 300, 257, 16, 300),
    (40, 2, 4, 1, 70, 16, 1),
    (2, 1, 4, 4, 0, 16, 90),        # no cache
    (2, 1, 2, 3, 200, 16, 9),       # more drafted rows than queries
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype, d):
    B, H, G, q, n, ps, n_t = shape
    Case(B, H, G, q, d, n, ps, n_t, dtype, seed=n + q).check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cache", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("shape", [SHAPES[i] for i in (1, 2, 3, 4, 6, 7, 8, 9)])
def test_quantised_caches(shape, cache, dtype, d):
    B, H, G, q, n, ps, n_t = shape
    Case(B, H, G, q, d, n, ps, n_t, dtype, cache, layout="bshd", seed=n).check()


@pytest.mark.parametrize("shape", ["chain", "block", "tree"])
@pytest.mark.parametrize("layout", ["bshd", "wide"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layouts_and_drafts(dtype, layout, shape):
    Case(3, 2, 4, 9, 128, 250, 16, 9, dtype, shape=shape, layout=layout, seed=1).check()
    Case(2, 2, 1, 40, 64, 100, 24, 40, dtype, shape=shape, layout=layout, seed=2).check()


@pytest.mark.parametrize("cache", [None, "mxfp8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 5, 40])
def test_lengths(q, dtype, cache):
    # Of zero, one, below zero and beyond the end.
    Case(8, 2, 2, q, 128, 700, 24, q, dtype, cache, clen=[0, 1, 130, 9999, 24, 25, -7, 699],
         tlen=[q, 1, q, q // 2, q + 9, 1, q, 0], seed=3).check()
    c = Case(4, 2, 1, q, 64, 300, 16, q, dtype, cache, clen=[0, 0, -1, 5], tlen=[0, -3, 1, 0], seed=4)
    O = c.check()
    assert (O[:2] == 0).all() and not (O[3] == 0).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q,G", [(3, 1), (20, 4), (70, 1)])
def test_rows_whose_mask_leaves_nothing(q, G, dtype):
    c = Case(2, 2, G, q, 128, 100, 16, q, dtype, clen=[0, 100], seed=5)
    c.sees[:, 1] = False
    O = c.check()
    assert (O[0, :, 1] == 0).all() and not (O[1, :, 1] == 0).any() and not (O[0, :, 2] == 0).any()
    c.sees[:] = False
    assert (c.check()[0] == 0).all()


def test_bits_behind_the_last_drafted_row_are_not_looked_at():
    c = Case(2, 2, 2, 5, 128, 50, 16, 5, seed=6)
    want = c.run()
    full = torch.full_like(words(c.sees), -1) << 5
    mask = words(c.sees) | full
    O, ws = torch.empty_like(c.Q), c.workspace()
    wf.wf_tree_attn(c.Q, c.K, c.V, c.pages.cuda(), c.n, c.Kt, c.Vt, O, ws, **{**c.args(), "mask": mask})
    assert torch.equal(O, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q,G", [(2, 1), (8, 2), (40, 1), (70, 2)])
def test_what_a_masked_drafted_row_holds_does_not_matter(q, G, dtype):
    c = Case(2, 2, G, q, 128, 90, 16, q, dtype, seed=7)
    hidden = q // 2
    c.sees[0, :, hidden] = False
    c.sees[0, -1, hidden] = True      # one row sees it
    before = c.run()
    c.Vt[0, :, hidden, ::3] = float("nan")
    c.Vt[0, :, hidden, 1::3] = float("inf")
    after = c.run()
    assert torch.equal(after[1], before[1]) and torch.equal(after[0, :, :-1], before[0, :, :-1])
    last = after[0, :, -1]
    assert torch.isnan(last[:, ::3]).all() and (last[:, 1::3] == float("inf")).all()
    assert torch.isfinite(last[:, 2::3]).all()
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(DT[dtype]).min):
        c.Vt[0, :, hidden] = 0
        c.Kt[0, :, hidden] = bad
        assert torch.equal(c.run()[0, :, :-1], before[0, :, :-1]), bad


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 20, 64])
def test_a_nan_in_one_sequence_stays_there(q, dtype):
    c = Case(4, 2, 2, q, 128, 400, 24, q, dtype, seed=8)
    before = c.run()
    c.V[c.pages[1, 3], 1, 5] = float("nan")
    after = c.run()
    assert torch.equal(after[[0, 2, 3]], before[[0, 2, 3]]) and torch.equal(after[1, :2], before[1, :2])
    assert torch.isnan(after[1, 2:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sequences_that_share_pages(dtype):
    c = Case(6, 2, 2, 3, 128, 200, 16, 3, dtype, seed=9)
    c.pages[1:4, :10] = c.pages[0, :10]
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 6, 40])
def test_steep_softmax_scale_and_logits_of_minus_infinity(q, dtype):
    c = Case(2, 2, 2, q, 128, 600, 16, q, dtype, seed=10, scale=0.5)
    c.check()
    c = Case(2, 1, 1, q, 64, 300, 16, q, dtype, shape="block", seed=11)
    c.Q[..., 0] = 1.0
    rows = torch.zeros(c.K.shape[:3], dtype=torch.bool)
    for b in range(2):
        rows[c.pages[b, :12].long()] = True      # the first 192 keys
    c.K[..., 0][rows.cuda()] = -float("inf")
    c.Kt[:, :, 0, 0] = -float("inf")
    c.K64 = f64(c.K)
    c.check()
    c.K[..., 0] = c.Kt[..., 0] = -float("inf")
    assert (c.run() == 0).all()


@pytest.mark.parametrize("cache", [None, "mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q,n", [(1, 9000), (16, 5000), (64, 20000)])
def test_long_caches(q, n, dtype, cache):
    if dtype == "f32":
        n //= 4
    Case(3, 1, 4, q, 128, n, 64, q, dtype, cache, clen=[n, n // 3, n - 17], seed=12).check()


@pytest.mark.parametrize("cache", [None, "mxfp4"])
@pytest.mark.parametrize("q", [1, 32])
def test_same_bits_again_on_another_stream_and_beside_another_call(q, cache):
    c = Case(6, 2, 4, q, 128, 3000, 16, q, "bf16", cache, clen=[3000, 10, 1700, 2999, 0, 64], seed=13)
    first = c.run()
    assert torch.equal(c.run(), first)
    side = torch.cuda.Stream()
    assert torch.equal(c.run(stream=side), first)
    # Two calls at once, each with a workspace of its own.
    outs, args, pages = [], c.args(), c.pages.cuda()
    torch.cuda.synchronize()
    for s in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(s):
            outs.append((torch.zeros_like(c.Q), c.workspace()))
    torch.cuda.synchronize()
    for _ in range(5):
        for (O, ws), s in zip(outs, (None, side)):
            wf.wf_tree_attn(c.Q, c.K, c.V, pages, c.n, c.Kt, c.Vt, O, ws, stream=s, **args)
    torch.cuda.synchronize()
    for O, ws in outs:
        assert torch.equal(O, first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 24])
def test_two_graphs_that_share_a_workspace(q, dtype):
    a = Case(3, 2, 2, q, 128, 900, 16, q, dtype, seed=14)
    b = Case(2, 2, 4, q, 128, 500, 24, q, dtype, "mxfp8", seed=15)
    want = [a.run(), b.run()]
    ws = max((a.workspace(), b.workspace()), key=lambda t: t.nbytes)
    outs, graphs, keep = [], [], []
    for c in (a, b):
        O, args, pages = torch.zeros_like(c.Q), c.args(), c.pages.cuda()
        keep.append((args, pages))
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            wf.wf_tree_attn(c.Q, c.K, c.V, pages, c.n, c.Kt, c.Vt, O, ws, **args)
        outs.append(O)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for O, w in zip(outs, want):
        assert torch.equal(O, w)


def test_lengths_change_between_replays():
    c = Case(3, 2, 4, 2, 128, 2000, 16, 2, clen=[2000, 1500, 900], seed=16)
    args, pages, O, ws = c.args(), c.pages.cuda(), torch.zeros_like(c.Q), c.workspace()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        wf.wf_tree_attn(c.Q, c.K, c.V, pages, c.n, c.Kt, c.Vt, O, ws, **args)
    for clen in ([2000, 1500, 900], [3, 0, 899], [1999, 16, 17]):
        args["cache_len"].copy_(torch.tensor(clen))
        g.replay()
        torch.cuda.synchronize()
        c.clen = clen
        assert torch.equal(O, c.run())


@pytest.mark.parametrize("cache", [None, "mxfp8"])
def test_a_wait_that_gives_up_is_reported(cache):
    c = Case(2, 2, 4, 40, 128, 700, 16, 40, "bf16", cache, seed=17)
    want = c.run()
    wf.wf_testing_set_wait_failure(True, 20000)
    try:
        with pytest.raises(wf.WfError) as e:
            c.run()
        assert e.value.status == -7
    finally:
        wf.wf_testing_set_wait_failure(False, 0)
    assert torch.equal(c.run(), want)


@pytest.mark.parametrize("dtype,fmt", [("bf16", None), ("bf16", "mxfp8"), ("f32", "mxfp8"), ("f32", None)])
@pytest.mark.parametrize("q", [1, 40])
def test_a_pool_past_32_bits(q, dtype, fmt):
    # The sequence's last page starts behind 2^32 bytes.
    d, ps = 128, 16
    size = {None: DT[dtype].itemsize, "mxfp8": 1}[fmt]
    pool = (1 << 32) // (ps * d * size) + 3
    x = torch.randn(1, 1, 40, d, generator=torch.Generator().manual_seed(18)).to(DT[dtype])
    at = [pool - 1, 5, pool - 2]
    v = f64(x)[0, 0]
    K = torch.zeros(pool, 1, ps, d, dtype=torch.uint8 if fmt else DT[dtype], device="cuda")
    Ks = None
    if fmt:
        codes, byte = mx.quantize(v, fmt)
        v = mx.values(codes, byte, fmt)
        Ks = torch.zeros(pool, 1, ps, d // 32, dtype=torch.uint8, device="cuda")
    for i, p in enumerate(at):
        rows = slice(16 * i, min(40, 16 * i + 16))
        m = rows.stop - rows.start
        K[p, 0, :m] = torch.from_numpy(codes[rows]).cuda() if fmt else x[0, 0, rows].cuda()
        if fmt:
            Ks[p, 0, :m] = torch.from_numpy(byte[rows]).cuda()
    pages = torch.tensor([at], dtype=torch.int32, device="cuda")
    Q = torch.randn(1, 2, q, d, generator=torch.Generator().manual_seed(19)).to(DT[dtype]).cuda()
    O = torch.empty_like(Q)
    f = FMT.get(fmt)
    ws = torch.zeros(wf.wf_tree_attn_workspace_bytes(Q, K, 40, 0, fmt=f), dtype=torch.uint8, device="cuda")
    wf.wf_tree_attn(Q, K, K, pages, 40, None, None, O, ws, Ks=Ks, Vs=Ks, fmt=f)
    want = np.stack([mx.attention(f64(Q)[0, h], v, v) for h in range(2)])[None]
    A = np.stack([mx.attention(f64(Q)[0, h], v, np.abs(v)) for h in range(2)])[None]
    tol = 2.0 ** -7 * A + 2.0 ** -11 * A if dtype == "bf16" else 300 * 2.0 ** -24 * A
    assert (np.abs(f64(O) - want) <= tol).all()


def test_as_they_are_used_together():
    # Two rounds of drafting: rotate queries and drafted keys, attend, take the accepted rows into the pages.
    B, H, G, q, d, ps, entries = 3, 2, 2, 6, 128, 16, 6
    r, g = np.random.default_rng(20), torch.Generator().manual_seed(20)
    freq = 10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)
    plan = wf.wf_rotary_plan(freq).cuda()
    K, V = (torch.zeros(B * entries, H, ps, d, dtype=torch.bfloat16, device="cuda") for _ in "KV")
    pages = torch.randperm(B * entries, generator=g).view(B, entries).to(torch.int32).cuda()
    length = torch.zeros(B, dtype=torch.int32, device="cuda")
    draw = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
    # A prompt of unequal lengths.
    Kp, Vp, count = draw(B, H, 40, d), draw(B, H, 40, d), torch.tensor([40, 17, 0], dtype=torch.int32, device="cuda")
    wf.wf_paged_append(Kp, Vp, K, V, pages, length, count=count, plan=plan)
    length += count
    line = [([], []) for _ in range(B)]
    for b in range(B):
        m = int(count[b])
        x = torch.empty_like(Kp)
        wf.wf_rotary_apply(Kp, None, plan, torch.arange(40, dtype=torch.int32, device="cuda").expand(1, B, 40)
                           .contiguous(), x, None)
        line[b][0].append(f64(x)[b, :, :m])
        line[b][1].append(f64(Vp)[b, :, :m])
    for step in range(2):
        sees = tree_mask(r, B, q, q, "tree")
        depth = torch.from_numpy(sees.sum(-1) - 1).to(torch.int32).cuda()
        pos = (length[:, None] + depth)[None].contiguous()
        Q, Kt, Vt = draw(B, H * G, q, d), draw(B, H, q, d), draw(B, H, q, d)
        wf.wf_rotary_apply(Q, Kt, plan, pos, Q, Kt)
        O, n = torch.empty_like(Q), int(length.max())
        ws = torch.zeros(wf.wf_tree_attn_workspace_bytes(Q, K, n, q), dtype=torch.uint8, device="cuda")
        wf.wf_tree_attn(Q, K, V, pages, n, Kt, Vt, O, ws, cache_len=length, mask=words(sees))
        for b in range(B):
            k, v = (np.concatenate(x, 1) for x in line[b])
            for hq in range(H * G):
                for i in range(q):
                    at = np.flatnonzero(sees[b, i])
                    kk = np.concatenate([k[hq // G], f64(Kt)[b, hq // G, at]])
                    vv = np.concatenate([v[hq // G], f64(Vt)[b, hq // G, at]])
                    want = mx.attention(f64(Q)[b, hq, i:i + 1], kk, vv)[0]
                    A = mx.attention(f64(Q)[b, hq, i:i + 1], kk, np.abs(vv))[0]
                    assert (np.abs(f64(O)[b, hq, i] - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -11) * A).all()
        # The path to the deepest node is accepted; it is already rotated.
        last = sees.sum(-1).argmax(1)
        took = [np.flatnonzero(sees[b, last[b]]) for b in range(B)]
        rows = torch.zeros(B, q, dtype=torch.int32)
        for b in range(B):
            rows[b, :len(took[b])] = torch.from_numpy(took[b])
            line[b][0].append(f64(Kt)[b, :, took[b]].transpose(1, 0, 2))
            line[b][1].append(f64(Vt)[b, :, took[b]].transpose(1, 0, 2))
        count = torch.tensor([len(t) for t in took], dtype=torch.int32, device="cuda")
        wf.wf_paged_append(Kt, Vt, K, V, pages, length, rows=rows.cuda(), count=count)
        length += count


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype,q", [("bf16", 1), ("bf16", 20), ("f32", 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_every_code_and_scale_is_read_exactly(d, dtype, q, fmt):
    # One cached row a sequence: the weight is 1, so O is the value row, to the bit.  Page h holds other codes; the
    # scale bytes go through 0 (2^-127) to 254.  What bf16 rounds below its smallest normal number is left out.
    B = 255
    codes = np.concatenate([np.arange(127), [0], np.arange(128, 255), [0]]).astype(np.uint8)
    V = np.zeros((B, 1, 1, d if fmt == "mxfp8" else d // 2), np.uint8)
    for h in range(B):
        V[h, 0, 0] = np.roll(codes, 37 * h)[:d] if fmt == "mxfp8" else (np.arange(d // 2) * 7 + h) % 256
    S = np.repeat(np.arange(B, dtype=np.uint8)[:, None, None, None], d // 32, axis=3)
    want = torch.from_numpy(mx.values(V, S, fmt))[:, 0, 0]
    K, one = np.zeros_like(V), np.full_like(S, 127)
    Q = torch.ones(B, 1, q, d, dtype=DT[dtype], device="cuda")
    K, V, one, S = (torch.from_numpy(x).cuda() for x in (K, V, one, S))
    pages = torch.arange(B, dtype=torch.int32, device="cuda").view(B, 1)
    O = torch.empty_like(Q)
    ws = torch.zeros(wf.wf_tree_attn_workspace_bytes(Q, K, 1, 0, fmt=FMT[fmt]), dtype=torch.uint8, device="cuda")
    wf.wf_tree_attn(Q, K, V, pages, 1, None, None, O, ws, Ks=one, Vs=S, fmt=FMT[fmt])
    wf.wf_workspace_status(ws)
    normal = (want == 0) | ((want.abs() >= 2.0 ** -126) & (want.abs() <= torch.finfo(DT[dtype]).max))
    for i in (0, q - 1):
        assert torch.equal(O[:, 0, i].double().cpu()[normal], want[normal])
    assert normal.double().mean() > 0.9


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,G,q,n,ps,n_t", [
    (70, 1, 1, 20, 150, 16, 20),      # more sequences than a warp has lanes
    (70, 1, 1, 2, 150, 8, 2),
    (3, 2, 1, 40, 1500, 100, 40),     # pages without common parts of 8 rows
    (3, 1, 4, 2, 1500, 100, 2),
    (2, 1, 4, 2, 700, 48, 300),       # long drafts
    (2, 1, 2, 400, 260, 16, 150),     # several row tiles, of which the last is short
])
def test_walks_and_tiles(B, H, G, q, n, ps, n_t, dtype):
    r = np.random.default_rng(21)
    clen = [int(x) for x in r.integers(0, n + 1, B)]
    tlen = [int(x) for x in r.integers(0, n_t + 1, B)]
    Case(B, H, G, q, 128, n, ps, n_t, dtype, clen=clen, tlen=tlen, seed=22).check()


@pytest.mark.parametrize("q", [1, 40])
def test_masked_values_in_any_part_of_a_long_draft(q):
    # Drafted rows that nothing sees but the last query row hold NaN, in tiles that different ranges have.
    c = Case(1, 1, 2, q + 1, 128, 600, 16, 280, seed=23)
    hidden = [3, 70, 129, 200, 279]
    c.sees[:, :, hidden] = False
    before = c.run()
    for j in hidden:
        c.Vt[0, 0, j, j % 128] = float("nan")
        c.Vt[0, 0, j, (j + 1) % 128] = -float("inf")
    assert torch.equal(c.run(), before)
    c.sees[:, -1, hidden] = True
    after = c.run()
    assert torch.equal(after[:, :, :-1], before[:, :, :-1])
    for j in hidden:
        assert torch.isnan(after[0, :, -1, j % 128]).all()


@pytest.mark.parametrize("q", [1, 24])
def test_heads_that_share_their_rows(q):
    # A pool whose key heads have a stride of 0: all of them are the same rows.
    c = Case(2, 1, 3, q, 128, 300, 16, q, "bf16", seed=24)
    want, A = c.check(), c.want(True)
    c.K, c.V = (t.expand(-1, 3, -1, -1) for t in (c.K, c.V))
    c.Kt, c.Vt = (t.expand(-1, 3, -1, -1) for t in (c.Kt, c.Vt))
    assert c.K.stride(1) == 0
    got = c.run()     # three query heads on three key heads
    # Each is within its tolerance of the definition.
    assert (np.abs(f64(got) - f64(want)) <= 2 * (2.0 ** -8 * np.abs(f64(want)) + (2.0 ** -8 + 2.0 ** -10) * A)).all()


def test_smaller_calls_leave_the_rest_alone():
    # Outputs inside a wider tensor, and rows of the workspace of a larger call.
    c = Case(3, 2, 2, 5, 128, 400, 16, 5, seed=25)
    want = c.run()
    wide = torch.full((3, 4, 9, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    O, args = wide[:, :, 2:7, :128], c.args()
    ws = torch.full((wf.wf_tree_attn_workspace_bytes(c.Q, c.K, 100000, 300) + 512,), 0x7f, dtype=torch.uint8, device="cuda")
    ws[:4] = 0
    wf.wf_tree_attn(c.Q, c.K, c.V, c.pages.cuda(), c.n, c.Kt, c.Vt, O, ws, **args)
    assert torch.equal(O, want)
    O.fill_(7.0)
    assert (wide == 7.0).all()
    assert (ws[-512:] == 0x7f).all()
