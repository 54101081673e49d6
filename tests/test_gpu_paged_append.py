"""wf_paged_append against the definition: rows in 32 and 16 bits and quantised,
rotated on the way or as they are, page sizes that divide nothing, unequal counts,
accepted rows of a draft, tables that end, and pages that nothing may touch.

What is not rotated has to be equal to the bit.  Rotated rows are as far off as
wf_rotary_apply's (the tolerance is its tests'); where they are quantised, a code is
the nearest to a value that is as far off, so half a step of the format more: 2^-4
(E4M3) or 2^-2 (E2M1) of the value, or half the smallest step, 2^-10 or 2^-2 of a
scale that is below 2 max / 448 (2 max / 6)."""
import numpy as np
import pytest
import torch

from oracle import mx, paged
from paper_2606_00724_gb300 import wf
from test_gpu_rotary import DT, lay, tolerance

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

FMT = {"mxfp8": wf.WF_MXFP8, "mxfp4": wf.WF_MXFP4}
FILL = 0x55  # what pools hold before


class Case:
    def __init__(self, B, H, rows, d, ps, entries, dtype="bf16", cache=None, layout="bhsd", pool_layout="bhsd", pairs=0,
                 axes=0, adjacent=False, accept=None, count=None, start=None, keys_alone=False, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.cache, self.fmt, self.adjacent = dtype, cache, FMT.get(cache), adjacent
        self.Kn, self.Vn = (lay(torch.randn(B, H, rows, d, generator=g).to(DT[dtype]).cuda(), layout) for _ in "KV")
        pool = B * entries + 3
        self.pages = torch.randperm(pool, generator=g)[:B * entries].view(B, entries).to(torch.int32)
        m = rows if accept is None else accept
        self.m = m
        most = entries * ps
        self.start = torch.tensor(start, dtype=torch.int32) if start is not None else \
            torch.randint(0, max(1, most - m + 1), (B,), generator=g).to(torch.int32)
        self.count = None if count is None else torch.tensor(count, dtype=torch.int32)
        self.rows = None if accept is None else torch.randint(0, rows, (B, m), generator=g).to(torch.int32)
        self.plan = self.pos = None
        if pairs:
            self.freq = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
            self.axis = (torch.arange(pairs) % max(1, axes)).to(torch.int32)
            self.plan = wf.wf_rotary_plan(self.freq, self.axis).cuda()
            if axes:
                self.pos = torch.randint(-100, 40000, (axes, B, rows), generator=g).to(torch.int32)
        dt = torch.uint8 if cache else DT[dtype]
        width = d // 2 if cache == "mxfp4" else d

        def make():
            t = torch.full((pool, H, ps, width * dt.itemsize), FILL, dtype=torch.uint8, device="cuda").view(dt)
            return t if pool_layout == "bhsd" else t.transpose(1, 2).contiguous().transpose(1, 2)
        self.K, self.V = make(), make()
        self.Ks = self.Vs = None
        if cache:
            self.Ks, self.Vs = (torch.full((pool, H, ps, d // 32), FILL, dtype=torch.uint8, device="cuda") for _ in "KV")
        if keys_alone:
            self.Vn = self.V = self.Vs = None

    def run(self, stream=None):
        at = lambda t: None if t is None else t.cuda()  # noqa: E731
        args = [at(t) for t in (self.pages, self.start, self.rows, self.count, self.pos)]
        torch.cuda.synchronize()
        wf.wf_paged_append(self.Kn, self.Vn, self.K, self.V, args[0], args[1], Ks=self.Ks, Vs=self.Vs, fmt=self.fmt,
                           rows=args[2], count=args[3], plan=self.plan, pos=args[4], adjacent=self.adjacent,
                           stream=stream)
        torch.cuda.synchronize()
        return self

    def check(self):
        pool, H, ps = self.K.shape[:3]
        put = paged.places(self.pages.numpy(), ps, pool, self.start.tolist(), self.m,
                           None if self.count is None else self.count.tolist())
        for new, held, scales, name in ((self.Kn, self.K, self.Ks, "K"), (self.Vn, self.V, self.Vs, "V")):
            if new is None:
                continue
            untouched = torch.ones(pool, ps, dtype=torch.bool)
            held, new = held.cpu(), new.cpu()
            scales = None if scales is None else scales.cpu()
            for b, i, page, at in put:
                untouched[page, at] = False
                row = i if self.rows is None else int(self.rows[b, i])
                x = new[b, :, row].double().numpy()
                got = held[page, :, at]
                if name == "K" and self.plan is not None:
                    pos = np.full((64, 1), int(self.start[b]) + i) if self.pos is None else \
                        self.pos[:, b, row:row + 1].numpy()
                    want = paged.rotate(x[:, None], pos, self.freq.tolist(), self.axis.tolist(), self.adjacent)[:, 0]
                    tol = tolerance(x, want, len(self.freq), self.adjacent, self.dtype)
                    if self.cache:
                        got = mx.values(got.numpy(), scales[page, :, at].numpy(), self.cache)
                        top = (np.abs(want) + tol).reshape(H, -1, 32).max(-1).repeat(32, -1)
                        near, least = (2.0 ** -4, 2.0 ** -10 * 2 / 448) if self.cache == "mxfp8" else (0.25, 0.25 * 2 / 6)
                        tol = 2 * tol + near * (np.abs(want) + tol) + least * top
                    else:
                        got = got.double().numpy()
                    assert (np.abs(got - want) <= tol).all(), (b, i)
                elif self.cache:
                    codes, byte = mx.quantize(x, self.cache)
                    assert np.array_equal(got.numpy(), mx.pack(codes, self.cache)), (b, i)
                    assert np.array_equal(scales[page, :, at].numpy(), byte), (b, i)
                else:
                    assert torch.equal(got, new[b, :, row]), (b, i)
            bytes_ = held.contiguous().view(torch.uint8).transpose(1, 2)
            assert (bytes_[untouched] == FILL).all()
            if scales is not None:
                assert (scales.transpose(1, 2)[untouched] == FILL).all()
        return len(put)


SHAPES = [  # B, H, rows, d, ps, entries
    (1, 1, 1, 64, 1, 1),
    (32, 8, 1, 128, 16, 5),
    (3, 4, 70, 128, 24, 4),
    (2, 6, 33, 64, 100, 2),
    (2, 3, 129, 128, 7, 30),
    (4, 40, 9, 64, 128, 1),
]


@pytest.mark.parametrize("pool_layout", ["bhsd", "bshd"])
@pytest.mark.parametrize("cache", [None, "mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_rows_as_they_are(shape, dtype, cache, pool_layout):
    c = Case(*shape, dtype, cache, layout="bshd" if pool_layout == "bhsd" else "wide", pool_layout=pool_layout, seed=1)
    assert c.run().check() == shape[0] * shape[2]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("pairs,axes", [(8, 0), (32, 0), (32, 3), (16, 2)])
@pytest.mark.parametrize("cache", [None, "mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotated_on_the_way(dtype, cache, pairs, axes, adjacent):
    Case(3, 2, 21, 128, 24, 3, dtype, cache, pairs=pairs, axes=axes, adjacent=adjacent, seed=2).run().check()
    Case(2, 5, 8, 64, 16, 3, dtype, cache, "bshd", "bshd", pairs=pairs, axes=axes, adjacent=adjacent, seed=3).run().check()


def test_many_rows_a_thread():
    # Enough rows that a thread takes several heads.
    Case(2, 36, 2100, 64, 64, 40, "bf16", pairs=32, layout="bshd", seed=4).run().check()
    Case(1, 33, 2100, 64, 64, 40, "bf16", "mxfp8", seed=5).run().check()


@pytest.mark.parametrize("cache", [None, "mxfp4"])
def test_counts_starts_and_tables_that_end(cache):
    c = Case(8, 2, 12, 128, 5, 4, "bf16", cache, start=[0, 1, 19, 20, 30, -3, 15, 2 ** 31 - 1],
             count=[0, 1, 5, 12, 3, 12, -4, 99], seed=6)
    c.pages[1, 0], c.pages[0, 1] = -1, 2 ** 31 - 1
    assert c.run().check() == 0 + 0 + 1 + 0 + 0 + 9 + 0 + 0
    c = Case(3, 2, 12, 128, 5, 4, "bf16", cache, start=[0, 8, 3], count=[12, 7, 99], seed=7)
    c.pages[2, 1] = c.K.shape[0]
    assert c.run().check() == 12 + 7 + 12 - 5


@pytest.mark.parametrize("cache", [None, "mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accepted_rows_of_a_draft(dtype, cache):
    c = Case(5, 3, 48, 128, 16, 4, dtype, cache, accept=9, count=[9, 0, 4, 1, 7], seed=8)
    c.rows[0, 2], c.rows[2, 1] = 99, -1  # clamped
    assert c.run().rows is not None
    c.rows.clamp_(0, 47)
    assert c.check() == 21
    c = Case(2, 2, 30, 64, 3, 9, dtype, cache, accept=11, pairs=32, axes=2, seed=9)  # rotated by the new row's position
    assert c.run().check() == 22
    c = Case(2, 2, 30, 64, 3, 9, dtype, cache, accept=11, pairs=32, seed=10)         # or by the place
    assert c.run().check() == 22


@pytest.mark.parametrize("cache", [None, "mxfp8"])
def test_keys_alone_and_nothing_at_all(cache):
    assert Case(2, 3, 5, 128, 16, 2, "bf16", cache, pairs=64, keys_alone=True, seed=11).run().check() == 10
    c = Case(2, 3, 0, 128, 16, 2, "bf16", cache, seed=12)
    assert c.run().check() == 0


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_codes_as_the_contiguous_cache(dtype, fmt):
    c = Case(1, 4, 96, 128, 16, 6, dtype, fmt, start=[0], seed=13)
    c.Kn[0, 1, 5, 40], c.Kn[0, 2, 6, 3] = float("nan"), float("inf")
    c.run()
    K = torch.zeros(1, 4, 96, c.K.shape[3], dtype=torch.uint8, device="cuda")
    Ks = torch.zeros(1, 4, 96, 4, dtype=torch.uint8, device="cuda")
    V, Vs = K.clone(), Ks.clone()
    wf.wf_cache_quantize(c.Kn, c.Vn, K, Ks, V, Vs, c.fmt, 0)
    order = c.pages[0].long().cuda()
    for pool, line in ((c.K, K), (c.Ks, Ks), (c.V, V), (c.Vs, Vs)):
        assert torch.equal(pool[order].transpose(0, 1).reshape(line.shape[1:]), line[0])
    # A pool reads back as a cache does.
    out, back = torch.empty(*c.K.shape[:3], 128, dtype=DT[dtype], device="cuda"), torch.empty_like(c.Kn)
    wf.wf_cache_dequantize(c.K, c.Ks, None, None, c.fmt, out, None)
    wf.wf_cache_dequantize(K, Ks, None, None, c.fmt, back, None)
    assert torch.equal(out[order].transpose(0, 1).reshape(back.shape[1:]).nan_to_num(7), back[0].nan_to_num(7))


def test_another_stream_and_a_graph():
    c = Case(3, 2, 4, 128, 16, 3, pairs=64, start=[0, 5, 30], seed=14).run()
    d = Case(3, 2, 4, 128, 16, 3, pairs=64, start=[0, 5, 30], seed=14).run(stream=torch.cuda.Stream())
    assert torch.equal(c.K, d.K) and torch.equal(c.V, d.V)
    start, pages = c.start.cuda(), c.pages.cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wf.wf_paged_append(c.Kn, c.Vn, c.K, c.V, pages, start, plan=c.plan)
    start.add_(4)  # the next rows, without a new capture
    graph.replay()
    torch.cuda.synchronize()
    d.start += 4
    d.run()
    assert torch.equal(c.K, d.K) and torch.equal(c.V, d.V)


def test_a_pool_past_32_bits():
    # The last page starts behind 2^32 bytes and 2^31 elements.
    pages = (1 << 20) + 2
    K = torch.zeros(pages, 1, 16, 128, dtype=torch.bfloat16, device="cuda")
    x = torch.randn(1, 1, 3, 128, generator=torch.Generator().manual_seed(15)).bfloat16().cuda()
    table = torch.tensor([[pages - 1, 0]], dtype=torch.int32, device="cuda")
    start = torch.tensor([14], dtype=torch.int32, device="cuda")
    wf.wf_paged_append(x, None, K, None, table, start)
    assert torch.equal(K[-1, 0, 14:], x[0, 0, :2]) and torch.equal(K[0, 0, 0], x[0, 0, 2])
    assert torch.count_nonzero(K[-1, 0, :14]) == 0 and torch.count_nonzero(K[1:-1]) == 0
