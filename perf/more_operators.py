"""The operators of a paged cache for drafted tokens, as they are timed.

rotate: positions of one or several axes rotated into query and key rows (wf_rotary_apply).
append: new rows of several sequences, or the drafted rows that were accepted, written into the pages of a cache with
    the rotation on the way, in 32 or 16 bits or quantised (wf_paged_append).
tree:   attention of each sequence's drafted tokens over its pages and, by a mask, over the drafted rows (wf_tree_attn);
    one token a sequence is a draft of one node.

Rows are [batch, heads, rows, head_dim] in that memory order ("bhsd") or with the rows before the heads ("bshd"); pages
are [pages, heads, page rows, head_dim] in the same two orders.
"""
from __future__ import annotations

import math

import torch

own = False  # True: the library's calls; False: their plain form

DEVICE = "cuda"
BLOCK = 32  # elements that share a scale
EXACT_FLOPS = 4e11  # work of a case that exact() takes on
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4.0, "bf16": 2.0, "mxfp8": 1 + 1 / BLOCK, "mxfp4": 0.5 + 1 / BLOCK}  # bytes an element


def _rotate(B, rows, Hq, Hk, d, pairs, far, axes=1, adjacent=False, dtype="bf16", layout="bshd", name=None):
    """far: the first token's position is drawn below it."""
    c = dict(op="rotate", B=B, rows=rows, Hq=Hq, Hk=Hk, d=d, pairs=pairs, far=far, axes=axes, adjacent=adjacent,
             dtype=dtype, layout=layout)
    return dict(c, name=name) if name else c


def _append(B, rows, H, d, n, ps, cache, pairs=0, axes=1, adjacent=False, accept=0, lens=False, dtype="bf16",
            layout="bshd", name=None):
    """n: rows that a sequence's table has room for; accept: rows are drafts, of which at most so many go in;
    lens: unequal numbers of rows go in.  Pages of 4-bit codes are read back (wf_cache_dequantize takes a pool of pages
    as it takes a cache), by a program that goes on with the values that later steps will see."""
    c = dict(op="append", B=B, rows=rows, H=H, d=d, n=n, ps=ps, cache=cache, pairs=pairs, axes=axes, adjacent=adjacent,
             accept=accept, lens=lens, dtype=dtype, layout=layout)
    return dict(c, name=name) if name else c


def _tree(B, H, G, d, n, ps, q, cache="bf16", shape="tree", lens=False, dtype="bf16", layout="bhsd", name=None):
    """shape: "tree" and "chain" (each node sees its ancestors and itself) or "block" (every node sees all);
    lens: caches and trees of unequal sizes."""
    c = dict(op="tree", B=B, H=H, G=G, d=d, n=n, ps=ps, q=q, cache=cache, shape=shape, lens=lens, dtype=dtype,
             layout=layout)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The next token of 32 sequences, queries and keys as the projection leaves them: latency.
        _rotate(32, 1, 32, 8, 128, 64, 32768, name="rotate_token"),
        # A prompt with a picture in it (time, height, width), 28 query heads on 4, an odd length: bandwidth.
        _rotate(1, 24999, 28, 4, 128, 64, 1, axes=3, name="rotate_image_prompt"),
        # A batch of fp32 rows of 64-wide heads, neighbouring channels in pairs, half of the channels rotated.
        _rotate(3, 2001, 16, 16, 64, 16, 100000, adjacent=True, dtype="f32", layout="bhsd", name="rotate_f32_part"),
        # The next token of 32 sequences into pages of 16: latency.
        _append(32, 1, 8, 128, 8192, 16, "bf16", 64, name="append_token"),
        # Prompts of up to 8K tokens of unequal lengths, 32 heads, pages of 64: bandwidth.
        _append(4, 8192, 32, 128, 8192, 64, "bf16", 64, lens=True, name="append_prompts"),
        # Two prompts of 8K into pages of 8-bit codes.
        _append(2, 8192, 32, 128, 8192, 128, "mxfp8", 64, name="append_fp8_prompts"),
        # What was accepted of 16 sequences' 48 drafted rows (already rotated), into 4-bit pages, and those read back.
        _append(16, 48, 8, 128, 512, 32, "mxfp4", accept=9, lens=True, layout="bhsd", name="append_fp4_accepted"),
        # Seven drafted tokens each of four short fp32 sequences: the smallest call.
        _tree(4, 4, 1, 64, 1001, 16, 7, "f32", lens=True, dtype="f32", name="tree_f32_1k"),
        # One token each of 32 sequences of up to 8K, 32 query heads on 8: bandwidth.
        _tree(32, 8, 4, 128, 8192, 16, 1, lens=True, layout="bshd", name="tree_token_8k"),
        # Trees of 26 nodes of 8 sequences, 28 query heads on 4: 182 query rows a key head.
        _tree(8, 4, 7, 128, 16384, 64, 26, lens=True, name="tree_26_16k"),
        # Blocks of 64 drafted rows that see each other, 32 query heads on 8, long caches: the tensor cores' rate.
        _tree(4, 8, 4, 128, 32768, 64, 64, shape="block", name="tree_block_32k"),
        # Trees of 16 nodes of two sequences of 128K in 8 bits.
        _tree(2, 8, 4, 128, 131072, 128, 16, "mxfp8", name="tree_fp8_128k"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choices(["rotate", "append", "tree"], [2, 3, 5])[0]
    d = rng.choice([64, 128, 128])
    layout = rng.choice(["bhsd", "bshd"])
    dtype = rng.choices(["bf16", "f32"], [3, 1])[0]
    fmt = rng.choice(["mxfp8", "mxfp4"])
    pairs = rng.choice([d // 2, d // 2, d // 4, 8])
    axes, adjacent = rng.choice([1, 1, 2, 3]), rng.random() < 0.3
    ps = rng.choice([1, 16, 16, 32, 64, 128, 24, 100])
    if op == "rotate":
        Hk, G, B = rng.choice([1, 4, 6, 8, 16]), rng.choice([1, 2, 4, 7]), rng.choice([1, 1, 2, 3, 32])
        most = (1 << 26 if dtype == "bf16" else 1 << 25) // (B * Hk * (1 + G) * d)
        return _rotate(B, log(1, min(32768, most)), Hk * G, Hk, d, pairs, log(1, 1 << 20), axes, adjacent, dtype, layout)
    cache = rng.choices([dtype, fmt], [1, 1])[0]
    if op == "append":
        B, H = rng.choice([1, 2, 3, 8, 32]), rng.choice([1, 4, 6, 8, 32])
        most = min(32768, (1 << 26 if dtype == "bf16" else 1 << 25) // (B * H * d))
        if rng.random() < 0.3:
            rows = rng.randint(1, 64)
            return _append(B, rows, H, d, max(ps, rows, min(most, 512 if cache == "mxfp4" else 4096)), ps, cache, 0, 1,
                           False, rng.randint(1, rows), rng.random() < 0.5, dtype, layout)
        rows = log(1, most)
        n = rows if cache == "mxfp4" else max(rows, min(most, log(64, 32768)))
        return _append(B, rows, H, d, n, ps, cache, rng.choice([0, pairs, pairs]), axes, adjacent, 0,
                       rng.random() < 0.5, dtype, layout)
    B, H, G = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([1, 4, 6, 8, 16]), rng.choice([1, 1, 2, 4, 7])
    q = rng.choice([1, 1, 5, 16, 32, rng.randint(2, 80)])

    def cap():  # operations and cached elements at or below those of the largest listed cases of the type
        most, cells = (1.3e11, 1 << 27) if dtype == "bf16" else (1.7e10, 1 << 26)
        return min(131072, cells // (B * H * d), int(most / (4 * d * B * H * G * q)) - q)

    while cap() < 256:
        if B > 1:
            B //= 2
        elif q > 1:
            q = (q + 1) // 2
        else:
            H = max(1, H // 2)
    return _tree(B, H, G, d, log(64, cap()), ps, q, cache, rng.choice(["tree", "tree", "chain", "block"]),
                 rng.random() < 0.5, dtype, layout)


# ---------------------------------------------------------------------------
# Inputs.
# ---------------------------------------------------------------------------
def _empty(case, B, H, rows, width, dtype):
    """[B, H, rows, width] in the case's memory order."""
    if case["layout"] == "bshd":
        return torch.empty(B, rows, H, width, dtype=dtype, device=DEVICE).transpose(1, 2)
    return torch.empty(B, H, rows, width, dtype=dtype, device=DEVICE)


def _normal(case, g, B, H, rows, d, dtype):
    t = _empty(case, B, H, rows, d, dtype)
    t.copy_(torch.randn(B, H, rows, d, generator=g, device=DEVICE))
    return t


def _keys(case, g, B, H, rows, d, dtype):
    """Keys as models have them: a few channels of each head larger than the rest, tokens of unequal norms."""
    t = _empty(case, B, H, rows, d, dtype)
    channel = torch.exp(0.5 * torch.randn(1, H, 1, d, generator=g, device=DEVICE))
    token = torch.exp(0.25 * torch.randn(B, H, rows, 1, generator=g, device=DEVICE))
    t.copy_(torch.randn(B, H, rows, d, generator=g, device=DEVICE) * channel * token)
    return t


def _frequencies(case):
    """Radians a position of each pair, and its axis: contiguous groups of pairs, the first axis a smaller one."""
    pairs, axes = case["pairs"], case["axes"]
    freq = torch.arange(pairs, dtype=torch.float64).mul_(-1.0 / pairs).mul_(math.log(10000.0)).exp_()
    first = pairs // 4 if axes == 3 else pairs // axes
    rest = max(1, axes - 1)
    axis = [0 if i < first or axes == 1 else min(axes - 1, 1 + (i - first) * rest // (pairs - first))
            for i in range(pairs)]
    return freq, torch.tensor(axis, dtype=torch.int32)


def _positions(case, g, B, rows, first):
    """[axes, B, rows] int32: a third of text, a picture of rows x columns in the next third, text again."""
    i = torch.arange(rows, device=DEVICE).expand(B, rows)
    at, end = rows // 3, rows // 3 + rows // 3
    width = max(1, math.isqrt(end - at))
    picture = (i >= at) & (i < end)
    after = i - end + at + width
    axes = [torch.where(i < at, i, torch.where(picture, torch.full_like(i, at), after)),
            torch.where(i < at, i, torch.where(picture, at + (i - at) // width, after)),
            torch.where(i < at, i, torch.where(picture, at + (i - at) % width, after))]
    if case["axes"] == 1:
        axes = [i]
    return torch.stack([first.view(B, 1) + a for a in axes[:case["axes"]]]).to(torch.int32).contiguous()


def _tables(case, g, B, n, spare):
    """(pages of the pool, [B, pages a sequence] int32): pages in a random order, as a pool in use has them."""
    each = -(-n // case["ps"])
    order = torch.randperm(B * each, generator=g, device=DEVICE).view(B, each).to(torch.int32)
    return B * each + spare, order.contiguous()


def _pool(case, pages, H, d, cache):
    """An empty pool of pages: rows or codes, and scales."""
    if cache in _DT:
        return _empty(case, pages, H, case["ps"], d, _DT[cache]).zero_(), None
    codes = _empty(case, pages, H, case["ps"], d if cache == "mxfp8" else d // 2, torch.uint8).zero_()
    return codes, torch.zeros(pages, H, case["ps"], d // BLOCK, dtype=torch.uint8, device=DEVICE)


def _mask(case, g, sizes):
    """[B, q, words] int32: bit j of row i: node i sees drafted row j.  Nodes past a tree's size see none."""
    B, q = case["B"], case["q"]
    chance = torch.rand(B, q, generator=g, device=DEVICE).cpu()
    node = torch.arange(q)
    parent = node - 1 if case["shape"] == "chain" else (chance * node).floor().long().minimum(node - 1)
    parent = parent.expand(B, q)
    sees = torch.zeros(B, q, 32 * (-(-q // 32)), dtype=torch.bool)
    for i in range(q):
        if i:
            sees[:, i] = sees[torch.arange(B), parent[:, i]]
        sees[:, i, i] = True
    sees &= (node.view(1, q, 1) < sizes.cpu().view(B, 1, 1))
    weight = (1 << torch.arange(32)).view(1, 1, 1, 32)
    words = (sees.view(B, q, -1, 32) * weight).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).to(DEVICE).contiguous()


def _inputs(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    s = dict(case)
    op, B, d, dt = case["op"], case["B"], case["d"], _DT[case["dtype"]]
    if op == "rotate":
        s["Q"], s["K"] = _normal(case, g, B, case["Hq"], case["rows"], d, dt), _keys(case, g, B, case["Hk"], case["rows"], d, dt)
        s["Qo"], s["Ko"] = torch.empty_like(s["Q"]), torch.empty_like(s["K"])
        first = torch.randint(0, case["far"], (B,), generator=g, device=DEVICE)
        s["pos"] = _positions(case, g, B, case["rows"], first)
        s["freq"], s["axis"] = _frequencies(case)
        return s
    H, n, ps, cache = case["H"], case["n"], case["ps"], case["cache"]
    if op == "append":
        rows, m = case["rows"], case["accept"] or case["rows"]
        # Longer tables than the rows: the sequences have some already.
        pages, s["pages"] = _tables(case, g, B, n, 1)  # the last page is no sequence's
        s["Kn"], s["Vn"] = _keys(case, g, B, H, rows, d, dt), _normal(case, g, B, H, rows, d, dt)
        s["start"] = torch.randint(0, max(1, n - m + 1), (B,), generator=g, device=DEVICE).to(torch.int32)
        s["count"] = s["rows_at"] = s["pos"] = None
        if case["lens"]:
            s["count"] = torch.randint((m + 1) // 2, m + 1, (B,), generator=g, device=DEVICE).to(torch.int32)
        if case["accept"]:
            order = torch.rand(B, rows, generator=g, device=DEVICE).argsort(1)[:, :m]
            s["rows_at"] = order.sort(1).values.to(torch.int32).contiguous()
        if case["pairs"]:
            s["freq"], s["axis"] = _frequencies(case)
            if case["axes"] > 1:
                s["pos"] = _positions(case, g, B, rows, s["start"])
        for x in "KV":
            s[x], s[x + "s"] = _pool(case, pages, H, d, cache)
            if cache == "mxfp4":
                s[x + "o"] = torch.empty(pages, H, ps, d, dtype=dt, device=DEVICE)
        return s
    G, q = case["G"], case["q"]
    pages, s["pages"] = _tables(case, g, B, n, 0)
    for x, make in (("K", _keys), ("V", _normal)):
        s[x], s[x + "s"] = _pool(case, pages, H, d, cache)
        each = max(1, (1 << 26) // (H * ps * d))
        for i in range(0, pages, each):  # some pages at a time
            k = min(each, pages - i)
            part = make(dict(case, layout="bhsd"), g, k, H, ps, d, torch.float32)
            if cache in _DT:
                s[x][i:i + k].copy_(part)
            else:
                c, e = _quantise(part, cache)
                s[x][i:i + k].copy_(c)
                s[x + "s"][i:i + k].copy_(e)
    s["Q"] = _normal(case, g, B, H * G, q, d, dt)
    s["O"] = torch.empty_like(s["Q"])
    s["Kt"], s["Vt"] = _keys(case, g, B, H, q, d, dt), _normal(case, g, B, H, q, d, dt)
    s["len"] = torch.full((B,), n, dtype=torch.int32, device=DEVICE)
    sizes = torch.full((B,), q, dtype=torch.int32, device=DEVICE)
    if case["lens"]:
        s["len"] = torch.randint(n // 2, n + 1, (B,), generator=g, device=DEVICE).to(torch.int32)
        sizes = torch.randint((q + 1) // 2, q + 1, (B,), generator=g, device=DEVICE).to(torch.int32)
        used = -(-s["len"] // ps)
        past = torch.arange(s["pages"].shape[1], device=DEVICE) >= used.view(B, 1)
        s["pages"] = s["pages"].masked_fill(past, -1)  # pages that a sequence does not have yet
    s["tree_len"] = sizes
    s["mask"] = None if case["shape"] == "block" else _mask(case, g, sizes)
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# ---------------------------------------------------------------------------
# One pass.
# ---------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2606_00724_gb300 import wf
    op = s["op"]
    if op != "tree" and s["pairs"] and "plan" not in s:
        s["plan"] = wf.wf_rotary_plan(s["freq"], s["axis"]).to(DEVICE)
    if op == "rotate":
        wf.wf_rotary_apply(s["Q"], s["K"], s["plan"], s["pos"], s["Qo"], s["Ko"], adjacent=s["adjacent"])
        return {"Q": s["Qo"], "K": s["Ko"]}
    fmt = {"mxfp8": wf.WF_MXFP8, "mxfp4": wf.WF_MXFP4}.get(s["cache"])
    if op == "append":
        wf.wf_paged_append(s["Kn"], s["Vn"], s["K"], s["V"], s["pages"], s["start"], Ks=s["Ks"], Vs=s["Vs"], fmt=fmt,
                           rows=s["rows_at"], count=s["count"], plan=s.get("plan"), pos=s["pos"],
                           adjacent=s["adjacent"])
        if s["cache"] == "mxfp4":
            wf.wf_cache_dequantize(s["K"], s["Ks"], s["V"], s["Vs"], fmt, s["Ko"], s["Vo"])
        return _held(s)
    if "ws" not in s:
        size = wf.wf_tree_attn_workspace_bytes(s["Q"], s["K"], s["n"], s["q"], fmt=fmt)
        s["ws"] = torch.zeros(size, dtype=torch.uint8, device=DEVICE)
    wf.wf_tree_attn(s["Q"], s["K"], s["V"], s["pages"], s["n"], s["Kt"], s["Vt"], s["O"], s["ws"], cache_len=s["len"],
                    tree_len=s["tree_len"], mask=s["mask"], Ks=s["Ks"], Vs=s["Vs"], fmt=fmt)
    return s["O"]


def _held(s):
    """The sequences' pages as the values that they hold."""
    if s["cache"] != "mxfp8":
        return {x: (s[x + "o"] if s["cache"] == "mxfp4" else s[x])[:-1] for x in "KV"}
    return {"K": s["K"][:-1].view(torch.float8_e4m3fn), "Ks": s["Ks"][:-1].view(torch.float8_e8m0fnu),
            "V": s["V"][:-1].view(torch.float8_e4m3fn), "Vs": s["Vs"][:-1].view(torch.float8_e8m0fnu)}


def _fp4_values(codes):
    """What two E2M1 codes a byte stand for, without their scales."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    table = torch.cat([table, -table])
    return torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], -1).flatten(-2)


def _quantise(x, fmt):
    """Codes and scale bytes of the rows x ([..., d] fp32)."""
    v = x.unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(v.abs().amax(-1, keepdim=True))  # m 2^e with m in [1/2, 1)
    # The least power of two whose multiple by the format's largest value (448 or 6) covers the block.
    e = e - 9 + (m > 0.875) if fmt == "mxfp8" else e - 3 + (m > 0.75)
    e = torch.where(m > 0, e, -127).clamp(-127, 127)
    y = torch.ldexp(v, -e).flatten(-2)
    scale = (e.squeeze(-1) + 127).to(torch.uint8)
    if fmt == "mxfp8":
        return y.to(torch.float8_e4m3fn).view(torch.uint8), scale
    a = y.abs()
    i = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4))
    code = i.to(torch.uint8) | ((y < 0).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def _values(codes, scale, fmt):
    """The fp32 rows that codes and scale bytes stand for."""
    v = codes.view(torch.float8_e4m3fn).float() if fmt == "mxfp8" else _fp4_values(codes)
    e = scale.to(torch.int32) - 127
    return torch.ldexp(v.unflatten(-1, (-1, BLOCK)), e.unsqueeze(-1)).flatten(-2)


def _turned(s, x, pos):
    """The rows x ([B, H, rows, d]) rotated by the positions pos ([axes, B, rows]), in fp32.  Angles of far positions
    do not fit 32 bits; their cosines and sines do."""
    freq, axis = s["freq"].to(DEVICE), s["axis"].to(DEVICE).long()
    angle = pos[axis].permute(1, 2, 0).double() * freq  # [B, rows, pairs]
    c, w = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)
    x, pairs = x.float(), s["pairs"]
    if s["adjacent"]:
        a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
        turned = torch.stack([a * c - b * w, b * c + a * w], -1).flatten(-2)
    else:
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
        turned = torch.cat([a * c - b * w, b * c + a * w], -1)
    return torch.cat([turned, x[..., 2 * pairs:]], -1)


def _run_plain(s):
    op = s["op"]
    if op == "rotate":
        s["Qo"].copy_(_turned(s, s["Q"], s["pos"]))
        s["Ko"].copy_(_turned(s, s["K"], s["pos"]))
        return {"Q": s["Qo"], "K": s["Ko"]}
    if op == "tree":
        return _attention(s)
    B, H, d, ps, rows = s["B"], s["H"], s["d"], s["ps"], s["rows"]
    new = {"K": s["Kn"], "V": s["Vn"]}
    if s["pairs"]:
        pos = s["pos"] if s["pos"] is not None else s["start"].view(1, B, 1) + torch.arange(rows, device=DEVICE)
        new["K"] = _turned(s, s["Kn"], pos)
    if s["rows_at"] is not None:
        at = s["rows_at"].long().view(B, 1, -1, 1).expand(-1, H, -1, d)
        new = {x: t.gather(2, at) for x, t in new.items()}
    m = new["K"].shape[2]
    i = torch.arange(m, device=DEVICE)
    place = s["start"].view(B, 1).long() + i
    page = s["pages"].long().gather(1, (place // ps).clamp_max(s["pages"].shape[1] - 1))
    if s["count"] is not None:  # rows past a count go to the page that no sequence has
        page = torch.where(i < s["count"].view(B, 1), page, s["K"].shape[0] - 1)
    for x, t in new.items():
        if s["cache"] in _DT:
            s[x][page, :, place % ps] = t.transpose(1, 2).to(s[x].dtype)
        else:
            codes, scale = _quantise(t.float(), s["cache"])
            s[x][page, :, place % ps] = codes.transpose(1, 2)
            s[x + "s"][page, :, place % ps] = scale.transpose(1, 2)
        if s["cache"] == "mxfp4":
            s[x + "o"].copy_(_values(s[x], s[x + "s"], "mxfp4"))
    return _held(s)


def _attention(s):
    B, H, G, q, d, n = (s[x] for x in ("B", "H", "G", "q", "d", "n"))
    rows = (s["Q"].float() / math.sqrt(d)).reshape(B, H, G * q, d)
    table = s["pages"].long().clamp_min(0)

    def cached(x):  # [B, H, pages x rows, d]
        t = s[x][table].transpose(1, 2).flatten(2, 3)
        if s["cache"] in _DT:
            return t.float()
        return _values(t, s[x + "s"][table].transpose(1, 2).flatten(2, 3), s["cache"])

    K = cached("K")
    logits = rows @ K.transpose(2, 3)
    logits.masked_fill_(torch.arange(K.shape[2], device=DEVICE) >= s["len"].view(B, 1, 1, 1), -math.inf)
    del K
    last = (rows @ s["Kt"].float().transpose(2, 3)).view(B, H, G, q, q)
    j = torch.arange(q, device=DEVICE)
    seen = (j < s["tree_len"].view(B, 1, 1)).expand(B, q, q)
    if s["mask"] is not None:
        seen = seen & ((s["mask"][..., j // 32] >> (j % 32)) & 1).bool()
    last = last.masked_fill(~seen.view(B, 1, 1, q, q), -math.inf).view(B, H, G * q, q)
    top = torch.maximum(logits.amax(-1, keepdim=True), last.amax(-1, keepdim=True))
    top = top.clamp_min(torch.finfo(torch.float32).min)  # a row without keys
    p, pt = logits.sub_(top).exp_(), (last - top).exp_()
    total = p.sum(-1, keepdim=True) + pt.sum(-1, keepdim=True)
    out = p @ cached("V") + pt @ s["Vt"].float()
    s["O"].copy_(torch.where(total > 0, out / total, 0.0).view(B, H * G, q, d))
    return s["O"]


# ---------------------------------------------------------------------------
# What a pass cannot do without.
# ---------------------------------------------------------------------------
def work(case):
    op, B, d = case["op"], case["B"], case["d"]
    es = _SIZE[case["dtype"]]
    if op == "rotate":
        cells = B * case["rows"] * (case["Hq"] + case["Hk"]) * d
        return {"bytes": int(2 * cells * es + 4 * case["axes"] * B * case["rows"]), "flops": 3 * cells}
    H = case["H"]
    if op == "append":
        part = 0.75 if case["lens"] else 1.0  # mean of the drawn counts, of their most
        cells = 2 * B * H * part * (case["accept"] or case["rows"]) * d
        moved = cells * (es + _SIZE[case["cache"]])
        if case["cache"] == "mxfp4":  # the pages read back
            moved += 2 * B * H * -(-case["n"] // case["ps"]) * case["ps"] * d * (es + _SIZE["mxfp4"])
        return {"bytes": int(moved), "flops": int(2 * cells)}
    G, q, n = case["G"], case["q"], case["n"]
    share = 0.75 if case["lens"] else 1.0
    moved = 2 * B * H * share * n * d * _SIZE[case["cache"]] + 2 * B * H * share * q * d * es + 2 * B * H * G * q * d * es
    return {"bytes": int(moved), "flops": int(4 * B * H * G * q * d * share * (n + q))}


# ---------------------------------------------------------------------------
# The definitions in 64 bits, apart from the plain form.
# ---------------------------------------------------------------------------
def _levels(fmt):
    """The magnitudes of a format, ascending; the place of one in the list is its code."""
    if fmt == "mxfp4":
        return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEVICE)
    return torch.tensor([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10)
                         for c in range(127)], dtype=torch.float64, device=DEVICE)


def _nearest(x, fmt):
    """(value in units of the scale, scale) of every element of x: the nearest magnitude of the format, a tie to the
    even code."""
    levels = _levels(fmt)
    v = x.unflatten(-1, (-1, BLOCK))
    most = v.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, -127.0)
    for _ in range(2):  # once more where the rounding of log2 put the first answer one too low
        first = torch.ceil(torch.log2((most / levels[-1]).clamp_min(2.0 ** -127)))
        e = torch.maximum(e, first)
        e = torch.where(levels[-1] * torch.exp2(e - 1) >= most, (e - 1).clamp_min(-127), e)
        e = torch.where(levels[-1] * torch.exp2(e) < most, e + 1, e)
    y = v.abs() / torch.exp2(e)
    hi = torch.searchsorted(levels, y.contiguous()).clamp(1, levels.numel() - 1)
    lo = hi - 1
    below, above = y - levels[lo], levels[hi] - y
    code = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return (levels[code] * torch.sign(v)).flatten(-2), torch.exp2(e).squeeze(-1)


def _rotation(s, x, pos):
    """x ([H, rows, d]) as complex numbers times e^(i angle), pos [axes, rows], in 64 bits."""
    x = x.double()
    pairs = s["pairs"]
    turn = torch.stack([pos[int(s["axis"][i])].double() * float(s["freq"][i]) for i in range(pairs)], -1)
    phase = torch.polar(torch.ones_like(turn), turn)
    re = slice(0, 2 * pairs, 2) if s["adjacent"] else slice(0, pairs)
    im = slice(1, 2 * pairs, 2) if s["adjacent"] else slice(pairs, 2 * pairs)
    z = torch.complex(x[..., re], x[..., im]) * phase
    out = x.clone()
    out[..., re], out[..., im] = z.real, z.imag
    return out


def exact(case, seed):
    op, B = case["op"], case["B"]
    if op == "tree" and work(case)["flops"] > EXACT_FLOPS:
        return None
    s = _inputs(case, seed)
    if op == "rotate":
        return {x: torch.stack([_rotation(s, s[x][b], s["pos"][:, b]) for b in range(B)]) for x in "QK"}
    if op == "append":
        out = {}
        for x in "KV":
            out[x] = torch.zeros(*s[x].shape[:3], case["d"], dtype=torch.float64, device=DEVICE)
            if case["cache"] == "mxfp8":
                out[x + "s"] = torch.full(s[x + "s"].shape, 2.0 ** -127, dtype=torch.float64, device=DEVICE)
            for b in range(B):
                start, table = int(s["start"][b]), s["pages"][b].long()
                rows = s[x + "n"][b].double()
                if x == "K" and case["pairs"]:
                    line = torch.arange(start, start + case["rows"], device=DEVICE).expand(case["axes"], -1)
                    rows = _rotation(s, rows, line if s["pos"] is None else s["pos"][:, b])
                if s["rows_at"] is not None:
                    rows = rows[:, s["rows_at"][b].long()]
                if s["count"] is not None:
                    rows = rows[:, :int(s["count"][b])]
                at = torch.arange(start, start + rows.shape[1], device=DEVICE)
                to = (table[at // case["ps"]], slice(None), at % case["ps"])
                if s[x + "s"] is None:
                    out[x][to] = rows.transpose(0, 1)
                else:
                    value, scale = _nearest(rows, case["cache"])
                    if case["cache"] == "mxfp4":
                        value = value * scale.repeat_interleave(BLOCK, -1)
                    else:
                        out[x + "s"][to] = scale.transpose(0, 1)
                    out[x][to] = value.transpose(0, 1)
        return {name: t[:-1] for name, t in out.items()}
    G, q, H, ps, d = (case[x] for x in ("G", "q", "H", "ps", "d"))
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEVICE)
    for b in range(B):
        n, t = int(s["len"][b]), int(s["tree_len"][b])
        table = s["pages"][b, :-(-n // ps)].long()
        sees = torch.ones(q, t, dtype=torch.bool, device=DEVICE)
        if s["mask"] is not None:
            for j in range(t):
                sees[:, j] = (s["mask"][b, :, j // 32].long() >> (j % 32)) % 2 == 1
        allowed = torch.cat([torch.ones(q, n, dtype=torch.bool, device=DEVICE), sees], 1).repeat(G, 1)
        for h in range(H):
            K, V = (_cached64(s, x, table, h)[:n] for x in "KV")
            K, V = torch.cat([K, s["Kt"][b, h, :t].double()]), torch.cat([V, s["Vt"][b, h, :t].double()])
            Q = s["Q"][b, h * G:(h + 1) * G].double().flatten(0, 1)
            w = (Q @ K.T / math.sqrt(d)).masked_fill(~allowed, -math.inf)
            w = torch.where(allowed.any(1, keepdim=True), torch.softmax(w, 1), 0.0)
            out[b, h * G:(h + 1) * G] = (w @ V).view(G, q, d)
    return out


def _cached64(s, x, table, h):
    """The rows of one key head on the pages of a table, in 64 bits."""
    t = s[x][table, h].flatten(0, 1)
    fmt = s["cache"]
    if fmt in _DT:
        return t.double()
    if fmt == "mxfp4":
        t = torch.stack([t % 16, t // 16], -1).flatten(-2)
    sign = 128 if fmt == "mxfp8" else 8
    v = _levels(fmt)[(t % sign).long()] * torch.where(t >= sign, -1.0, 1.0)
    e = s[x + "s"][table, h].flatten(0, 1).double() - 127
    return v * torch.exp2(e).repeat_interleave(BLOCK, -1)
