"""The operators of the quantised cache and of prompts that several sequences share, as they are timed.

store: rows of keys and values written into a cache of 8-bit or 4-bit floating-point codes with one power-of-two
    scale per 32 elements (wf_cache_quantize).
fetch: rows of such a cache read back, a range or a selection (wf_cache_dequantize).
attn:  attention of B sequences over P cached prompts, B / P sequences a prompt, whole or at selected rows, kept in
    32 or 16 bits or quantised, and over each sequence's own generation rows (wf_prefix_attn).

Layouts are the library's: [batch, heads, rows, head_dim], in that memory order ("bhsd") or with the rows before the
heads ("bshd").
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


def _store(B, H, d, n, rows, pos, fmt, dtype="bf16", layout="bhsd", back=False, name=None):
    c = dict(op="store", B=B, H=H, d=d, n=n, rows=rows, pos=pos, fmt=fmt, dtype=dtype, layout=layout, back=back)
    return dict(c, name=name) if name else c


def _fetch(B, H, d, n, rows, pos, fmt, dtype="bf16", layout="bhsd", select=False, name=None):
    c = dict(op="fetch", B=B, H=H, d=d, n=n, rows=rows, pos=pos, fmt=fmt, dtype=dtype, layout=layout, select=select)
    return dict(c, name=name) if name else c


def _attn(B, P, H, G, d, n, q, ng, cache="bf16", dtype="bf16", layout="bhsd", k=0, lens=False, name=None):
    """k: selected rows of the prompt (0: all of them); lens: prompts and generations of unequal lengths."""
    c = dict(op="attn", B=B, P=P, H=H, G=G, d=d, n=n, q=q, ng=ng, cache=cache, dtype=dtype, layout=layout, k=k,
             lens=lens)
    return dict(c, name=name) if name else c


def listed():
    return [
        # A denoising block's 32 new rows a head into a cache of 32K tokens, at an unaligned place: latency.
        _store(2, 32, 128, 32768, 32, 12340, "mxfp8", name="store_fp8_block"),
        # A whole prompt of 32K tokens, once a prompt: bandwidth.
        _store(1, 32, 128, 32768, 32768, 0, "mxfp8", name="store_fp8_prompt"),
        # A ragged stretch of an fp32 cache with 64-wide heads into 4 bits, and the same rows read back (a program that
        # goes on with the values that later steps will see).
        _store(2, 16, 64, 8200, 5001, 129, "mxfp4", "f32", "bshd", True, name="store_fp4_f32_ragged"),
        # The rows that a filter selected, 2048 a head, for attention in 16 bits.
        _fetch(2, 32, 128, 32768, 2048, 0, "mxfp8", select=True, name="fetch_fp8_selected"),
        # A whole prompt of 32K tokens out of 4 bits (a pyramid rebuilt after the 16-bit keys were dropped).
        _fetch(1, 32, 128, 32768, 32768, 0, "mxfp4", name="fetch_fp4_prompt"),
        # One new token each of four short fp32 sequences on one short prompt of an odd length: the smallest call.
        _attn(4, 1, 4, 1, 64, 1001, 1, 7, "f32", "f32", name="attn_f32_token_1k"),
        # fp32 denoising blocks of four sequences on a prompt of 8K.
        _attn(4, 1, 16, 1, 128, 8192, 32, 32, "f32", "f32", name="attn_f32_block_8k"),
        # One new token each of 16 sequences (28 query heads on 4) on one prompt of 32K, generations of unequal
        # lengths: bandwidth of the prompt, read once for all.
        _attn(16, 1, 4, 7, 128, 32768, 1, 65, lens=True, name="attn_bf16_token_32k"),
        # Denoising blocks of 16 sequences on one prompt of 32K, 32 heads: the tensor cores' rate.
        _attn(16, 1, 32, 1, 128, 32768, 32, 32, name="attn_bf16_block_32k"),
        # 64-wide heads, two prompts of unequal ragged lengths, caches in [B, rows, H, d] order.
        _attn(6, 2, 16, 1, 64, 8200, 24, 17, layout="bshd", lens=True, name="attn_bf16_d64_8k"),
        # One new token each of 8 sequences (32 query heads on 8) on a prompt of 128K in 8 bits.
        _attn(8, 1, 8, 4, 128, 131072, 1, 33, "mxfp8", name="attn_fp8_token_128k"),
        # Denoising blocks of 4 sequences a prompt at the rows that a filter selected, out of 4 bits.
        _attn(8, 2, 32, 1, 128, 32768, 32, 32, "mxfp4", k=2048, name="attn_fp4_selected_32k"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choices(["store", "fetch", "attn"], [2, 2, 5])[0]
    d = rng.choice([64, 128, 128])
    layout = rng.choice(["bhsd", "bshd"])
    dtype = rng.choices(["bf16", "f32"], [3, 1])[0]
    fmt = rng.choice(["mxfp8", "mxfp4"])
    if op != "attn":
        B, H = rng.choice([1, 1, 2, 3, 4]), rng.choice([1, 4, 6, 8, 16, 32])
        n = log(64, min(131072, (1 << (26 if dtype == "bf16" else 25)) // (B * H * d)))
        rows = min(n, log(1, n)) if rng.random() < 0.8 else n
        pos = rng.randint(0, n - rows)
        if op == "store":
            back = fmt == "mxfp4"
            return _store(B, H, d, n, rows, pos, fmt, dtype, layout, back)
        select = rng.random() < 0.5
        return _fetch(B, H, d, n, rows, 0 if select else pos, fmt, dtype, layout, select)
    P = rng.choice([1, 1, 1, 2, 3])
    B = P * rng.choice([1, 2, 3, 4, 8, 16, 24])
    H, G = rng.choice([1, 4, 6, 8, 16, 32]), rng.choice([1, 1, 1, 2, 4, 7])
    q = rng.choice([1, 1, 32, rng.randint(2, 64)])
    cache = rng.choices([dtype, fmt], [3, 2])[0]
    lo = 64

    def cap_of():  # operations and prompt elements at or below those of the largest listed case of the type
        most, cells = (2.7e11, 1 << 27) if dtype == "bf16" else (1.7e10, 1 << 26)
        return min(131072, cells // (P * H * d), int(most / (4 * d * B * H * G * q)) - 300)

    while cap_of() < 4 * lo:
        if B > P:
            B = P
        elif q > 1:
            q = (q + 1) // 2
        elif G > 1:
            G = 1
        else:
            H = max(1, H // 2)
    n = log(lo, cap_of())
    ng = rng.choice([0, 1, 32, rng.randint(2, 300)])
    k = log(16, n) if rng.random() < 0.3 else 0
    return _attn(B, P, H, G, d, n, q, ng, cache, dtype, layout, k, rng.random() < 0.4)


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
    """Keys as caches have them: a few channels of each head larger than the rest, tokens of unequal norms."""
    t = _empty(case, B, H, rows, d, dtype)
    channel = torch.exp(0.5 * torch.randn(1, H, 1, d, generator=g, device=DEVICE))
    token = torch.exp(0.25 * torch.randn(B, H, rows, 1, generator=g, device=DEVICE))
    t.copy_(torch.randn(B, H, rows, d, generator=g, device=DEVICE) * channel * token)
    return t


def _codes(case, B, H, n, d, fmt):
    codes = _empty(case, B, H, n, d if fmt == "mxfp8" else d // 2, torch.uint8)
    return codes.zero_(), torch.zeros(B, H, n, d // BLOCK, dtype=torch.uint8, device=DEVICE)


def _inputs(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    s = dict(case)
    op, B, H, d, n = (case[x] for x in ("op", "B", "H", "d", "n"))
    dt = _DT[case["dtype"]]
    if op == "store":
        s["Kn"] = _keys(case, g, B, H, case["rows"], d, dt)
        s["Vn"] = _normal(case, g, B, H, case["rows"], d, dt)
        (s["Kc"], s["Ks"]), (s["Vc"], s["Vs"]) = (_codes(case, B, H, n, d, case["fmt"]) for _ in range(2))
        return s
    P = case.get("P", B)
    fmt = case["fmt"] if op == "fetch" else case["cache"]
    if fmt in _DT:
        s["K"], s["V"] = _keys(case, g, P, H, n, d, dt), _normal(case, g, P, H, n, d, dt)
    else:
        for x, make in (("K", _keys), ("V", _normal)):
            codes, scales = _codes(case, P, H, n, d, fmt)
            for i in range(P):  # a prompt at a time
                rows = make(dict(case, layout="bhsd"), g, 1, H, n, d, torch.float32)
                c, e = _quantise(rows, fmt)
                codes[i:i + 1].copy_(c)
                scales[i:i + 1].copy_(e)
            s[x + "c"], s[x + "s"] = codes, scales
    count = case["rows"] if op == "fetch" and case["select"] else case.get("k", 0)
    s["idx"] = None
    if count:
        order = torch.rand(P * H, n, generator=g, device=DEVICE).argsort(1)[:, :count]
        s["idx"] = order.sort(1).values.to(torch.int32).contiguous()
    if op == "fetch":
        s["Ko"], s["Vo"] = (_empty(case, B, H, case["rows"], d, dt) for _ in range(2))
        return s
    G, q, ng = case["G"], case["q"], case["ng"]
    s["Q"] = _normal(case, g, B, H * G, q, d, dt)
    s["O"] = torch.empty_like(s["Q"])
    s["Kg"] = s["Vg"] = s["prefix_len"] = s["gen_len"] = None
    if ng:
        s["Kg"], s["Vg"] = _keys(case, g, B, H, ng, d, dt), _normal(case, g, B, H, ng, d, dt)
    if case["lens"]:
        most = case["k"] or n
        s["prefix_len"] = torch.randint(max(1, most // 2), most + 1, (P,), generator=g, device=DEVICE).int()
        if ng:
            s["gen_len"] = torch.randint(0, ng + 1, (B,), generator=g, device=DEVICE).int()
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
    formats = {"mxfp8": wf.WF_MXFP8, "mxfp4": wf.WF_MXFP4}
    if op == "store":
        fmt, pos = formats[s["fmt"]], s["pos"]
        wf.wf_cache_quantize(s["Kn"], s["Vn"], s["Kc"], s["Ks"], s["Vc"], s["Vs"], fmt, pos)
        if not s["back"]:
            return _stored(s)
        if "Ko" not in s:
            s["Ko"], s["Vo"] = torch.empty_like(s["Kn"]), torch.empty_like(s["Vn"])
        wf.wf_cache_dequantize(s["Kc"], s["Ks"], s["Vc"], s["Vs"], fmt, s["Ko"], s["Vo"], pos)
        return {"K": s["Ko"], "V": s["Vo"]}
    if op == "fetch":
        wf.wf_cache_dequantize(s["Kc"], s["Ks"], s["Vc"], s["Vs"], formats[s["fmt"]], s["Ko"], s["Vo"], s["pos"],
                               idx=s["idx"])
        return {"K": s["Ko"], "V": s["Vo"]}
    fmt = formats.get(s["cache"])
    K, V, Ks, Vs = (s["K"], s["V"], None, None) if fmt is None else (s["Kc"], s["Vc"], s["Ks"], s["Vs"])
    k = s["k"] or s["n"]
    if "ws" not in s:
        size = wf.wf_prefix_attn_workspace_bytes(s["Q"], K, k, s["ng"], fmt=fmt)
        s["ws"] = torch.zeros(size, dtype=torch.uint8, device=DEVICE)
    wf.wf_prefix_attn(s["Q"], K, V, k, s["Kg"], s["Vg"], s["O"], s["ws"], idx=s["idx"], prefix_len=s["prefix_len"],
                      gen_len=s["gen_len"], Ks=Ks, Vs=Vs, fmt=fmt)
    return s["O"]


def _stored(s):
    """The 8-bit caches as the values that they hold."""
    return {"K": s["Kc"].view(torch.float8_e4m3fn), "Ks": s["Ks"].view(torch.float8_e8m0fnu),
            "V": s["Vc"].view(torch.float8_e4m3fn), "Vs": s["Vs"].view(torch.float8_e8m0fnu)}


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
    if fmt == "mxfp8":
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
        table = torch.cat([table, -table])
        v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], -1).flatten(-2)
    e = scale.to(torch.int32) - 127
    return torch.ldexp(v.unflatten(-1, (-1, BLOCK)), e.unsqueeze(-1)).flatten(-2)


def _at(t, idx):
    """Rows idx ([P*H, k]) of t ([P, H, n, w])."""
    rows = idx.long().view(*t.shape[:2], -1, 1)
    return t.gather(2, rows.expand(-1, -1, -1, t.shape[3]))


def _run_plain(s):
    op = s["op"]
    if op == "store":
        at = slice(s["pos"], s["pos"] + s["rows"])
        out = {}
        for x in "KV":
            codes, scale = _quantise(s[x + "n"].float(), s["fmt"])
            s[x + "c"][:, :, at] = codes
            s[x + "s"][:, :, at] = scale
            if s["back"]:
                out[x] = _values(codes, scale, s["fmt"]).to(s[x + "n"].dtype)
        return out if s["back"] else _stored(s)
    if op == "fetch":
        out = {}
        for x in "KV":
            codes, scale = s[x + "c"], s[x + "s"]
            if s["idx"] is not None:
                codes, scale = _at(codes, s["idx"]), _at(scale, s["idx"])
            else:
                at = slice(s["pos"], s["pos"] + s["rows"])
                codes, scale = codes[:, :, at], scale[:, :, at]
            s[x + "o"].copy_(_values(codes, scale, s["fmt"]))
            out[x] = s[x + "o"]
        return out
    return _attention(s)


def _prompt(s, x):
    """The prompt rows that are attended, in fp32."""
    if s["cache"] in _DT:
        return (s[x] if s["idx"] is None else _at(s[x], s["idx"])).float()
    codes, scale = s[x + "c"], s[x + "s"]
    if s["idx"] is not None:
        codes, scale = _at(codes, s["idx"]), _at(scale, s["idx"])
    return _values(codes, scale, s["cache"])


def _attention(s):
    B, P, H, G, q, d, ng = (s[x] for x in ("B", "P", "H", "G", "q", "d", "ng"))
    Q = s["Q"].float() / math.sqrt(d)
    # The query rows of a prompt's key head: its B / P sequences, their G heads, q rows each.
    rows = Q.reshape(P, B // P, H, G * q, d)
    stacked = rows.transpose(1, 2).reshape(P, H, -1, d)
    K, V = _prompt(s, "K"), _prompt(s, "V")
    logits = stacked @ K.transpose(2, 3)
    if s["prefix_len"] is not None:
        past = torch.arange(K.shape[2], device=K.device) >= s["prefix_len"].view(P, 1, 1, 1)
        logits.masked_fill_(past, -math.inf)
    top = logits.amax(-1, keepdim=True)
    if ng:
        Kg, Vg = s["Kg"].float(), s["Vg"].float()
        last = rows.reshape(B, H, G * q, d) @ Kg.transpose(2, 3)
        if s["gen_len"] is not None:
            past = torch.arange(ng, device=Kg.device) >= s["gen_len"].view(B, 1, 1, 1)
            last.masked_fill_(past, -math.inf)
        top = torch.maximum(top, _stack(last.amax(-1, keepdim=True), P))
    top = top.clamp_min(torch.finfo(torch.float32).min)  # a row without keys
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = p @ V
    if ng:
        p = (last - _unstack(top, B)).exp_()
        total = total + _stack(p.sum(-1, keepdim=True), P)
        out = out + _stack(p @ Vg, P)
    out = torch.where(total > 0, out / total, 0.0)
    s["O"].copy_(_unstack(out, B).reshape(B, H * G, q, d))
    return s["O"]


def _stack(t, P):
    """[B, H, r, w] -> [P, H, B / P * r, w]."""
    B, H, r, w = t.shape
    return t.view(P, B // P, H, r, w).transpose(1, 2).reshape(P, H, -1, w)


def _unstack(t, B):
    """[P, H, B / P * r, w] -> [B, H, r, w]."""
    P, H, _, w = t.shape
    return t.view(P, H, B // P, -1, w).transpose(1, 2).reshape(B, H, -1, w)


# ---------------------------------------------------------------------------
# What a pass cannot do without.
# ---------------------------------------------------------------------------
def work(case):
    op, B, H, d = (case[x] for x in ("op", "B", "H", "d"))
    es = _SIZE[case["dtype"]]
    if op in ("store", "fetch"):
        cells = 2 * B * H * case["rows"] * d
        moved = cells * (es + _SIZE[case["fmt"]])
        if op == "store" and case["back"]:
            moved += cells * es  # the values read back
        if op == "fetch" and case["select"]:
            moved += 4 * B * H * case["rows"]
        return {"bytes": int(moved), "flops": 2 * cells}
    P, G, q, ng, k = case["P"], case["G"], case["q"], case["ng"], case["k"] or case["n"]
    share = 0.75 if case["lens"] else 1.0  # mean of the drawn prompt lengths, of their most
    part = 0.5 if case["lens"] else 1.0
    moved = 2 * P * H * share * k * d * _SIZE[case["cache"]] + 2 * B * H * part * ng * d * es + 2 * B * H * G * q * d * es
    if case["k"]:
        moved += 4 * P * H * share * k
    return {"bytes": int(moved), "flops": int(4 * B * H * G * q * d * (share * k + part * ng))}


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
    """(value, scale) of every element of x: the nearest magnitude of the format times its block's scale, a tie to
    the even code."""
    levels = _levels(fmt)
    v = x.double().unflatten(-1, (-1, BLOCK))
    most = v.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, -127.0)
    for _ in range(2):  # once more where the rounding of log2 put the first answer one too low
        first = torch.ceil(torch.log2((most / levels[-1]).clamp_min(2.0 ** -127)))
        e = torch.maximum(e, first)
        e = torch.where(levels[-1] * torch.exp2(e - 1) >= most, (e - 1).clamp_min(-127), e)
        e = torch.where(levels[-1] * torch.exp2(e) < most, e + 1, e)
    scale = torch.exp2(e)
    y = v.abs() / scale
    hi = torch.searchsorted(levels, y.contiguous()).clamp(1, levels.numel() - 1)
    lo = hi - 1
    below, above = y - levels[lo], levels[hi] - y
    code = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return (levels[code] * torch.sign(v)).flatten(-2), scale.squeeze(-1)


def exact(case, seed):
    op = case["op"]
    if op == "attn" and work(case)["flops"] > EXACT_FLOPS:
        return None
    s = _inputs(case, seed)
    if op == "store":
        out = {}
        at = slice(case["pos"], case["pos"] + case["rows"])
        for x in "KV":
            value = torch.empty(s[x + "n"].shape, dtype=torch.float64, device=DEVICE)
            scale = torch.empty(*s[x + "n"].shape[:3], case["d"] // BLOCK, dtype=torch.float64, device=DEVICE)
            for b in range(case["B"]):
                for h in range(case["H"]):
                    value[b, h], scale[b, h] = _nearest(s[x + "n"][b, h], case["fmt"])
            if case["back"]:
                out[x] = value * scale.repeat_interleave(BLOCK, -1)
                continue
            out[x] = torch.zeros(s[x + "c"].shape, dtype=torch.float64, device=DEVICE)
            out[x][:, :, at] = value
            out[x + "s"] = torch.full(s[x + "s"].shape, 2.0 ** -127, dtype=torch.float64, device=DEVICE)
            out[x + "s"][:, :, at] = scale
        return out

    def rows(x, p, h, fmt):
        if fmt in _DT:
            t = s[x][p, h].double()
        else:
            levels = _levels(fmt)
            c = s[x + "c"][p, h]
            if fmt == "mxfp4":
                c = torch.stack([c % 16, c // 16], -1).flatten(-2)
            sign_bit = 128 if fmt == "mxfp8" else 8
            t = levels[(c % sign_bit).long()] * torch.where(c >= sign_bit, -1.0, 1.0)
            t = t * torch.exp2(s[x + "s"][p, h].double() - 127).repeat_interleave(BLOCK, -1)
        return t if s["idx"] is None else t[s["idx"][p * case["H"] + h].long()]

    if op == "fetch":
        out = {x: torch.empty(s[x + "o"].shape, dtype=torch.float64, device=DEVICE) for x in "KV"}
        at = slice(None) if case["select"] else slice(case["pos"], case["pos"] + case["rows"])
        for x in "KV":
            for b in range(case["B"]):
                for h in range(case["H"]):
                    out[x][b, h] = rows(x, b, h, case["fmt"])[at]
        return out
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEVICE)
    G, each = case["G"], case["B"] // case["P"]
    prompt = [case["k"] or case["n"]] * case["P"] if s["prefix_len"] is None else s["prefix_len"].tolist()
    gen = [case["ng"]] * case["B"] if s["gen_len"] is None else s["gen_len"].tolist()
    for p in range(case["P"]):
        for h in range(case["H"]):
            K, V = (rows(x, p, h, case["cache"])[:prompt[p]] for x in "KV")
            for b in range(p * each, (p + 1) * each):
                Kb, Vb = K, V
                if gen[b]:
                    Kb = torch.cat([K, s["Kg"][b, h, :gen[b]].double()])
                    Vb = torch.cat([V, s["Vg"][b, h, :gen[b]].double()])
                if not len(Kb):
                    continue
                Q = s["Q"][b, h * G:(h + 1) * G].double().flatten(0, 1)
                out[b, h * G:(h + 1) * G] = (torch.softmax(Q @ Kb.T / math.sqrt(case["d"]), 1) @ Vb).view(G, -1, case["d"])
    return out
