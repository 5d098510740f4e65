"""Cases of the operators of a quantised decoder: microscaled 4-bit products, and an 8-bit key/value cache with its attention.

`run` computes a case either in plain tensor operations (in 32 bits, `own` false) or by the calls a program makes of the library (`own` true).

Formats, as both sides of `run` take them:

* 4-bit matrices [rows][cols]: e2m1 codes, two to a byte (even column in the low half), rows padded with zeros to a multiple of 32 columns; one
  scale byte for each block of 32 ("mx": a power of two, e8m0) or 16 ("nv": e4m3, times an fp32 scale of the whole matrix) columns.  The scales are
  stored in tiles of 128 rows x 4 blocks, 512 bytes each: row r, block j of a tile at byte 16 (r % 32) + 4 (r / 32) + j.
* the cache: [pages][heads][page tokens][dim] of int8 or e4m3 codes for keys and for values, one bf16 scale for every 16 tokens and head, and a table
  of page numbers [requests][pages of a request].  A request has `lens` tokens in the cache, the last `starts[i + 1] - starts[i]` of which are new.
"""
import math
import random

import numpy as np
import torch

own = False

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = {"mx": 32, "nv": 16}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
QMAX = {"int8": 127.0, "e4m3": 448.0}
TOKENS = 16          # tokens that share a scale of the cache


# ---- cases ---------------------------------------------------------------------------------------------------------

def listed():
    return [
        # a decode batch's activations on their way to a projection
        {"name": "round trip nv 16x4096", "op": "round_trip", "fmt": "nv", "rows": 16, "cols": 4096, "kind": "activations"},
        # an MLP weight converted once
        {"name": "round trip mx 14336x4096", "op": "round_trip", "fmt": "mx", "rows": 14336, "cols": 4096, "kind": "weights"},
        # one token through the query projection: latency
        {"name": "linear nv 1x4096x4096", "op": "linear", "fmt": "nv", "tokens": 1, "inner": 4096, "outer": 4096},
        # a decode batch through the gate projection
        {"name": "linear mx 24x4096x14336", "op": "linear", "fmt": "mx", "tokens": 24, "inner": 4096, "outer": 14336},
        # a chunk of a prompt, of no round length, through the down projection
        {"name": "linear nv 500x14336x4096", "op": "linear", "fmt": "nv", "tokens": 500, "inner": 14336, "outer": 4096},
        # whole prompts through the up projection
        {"name": "linear nv 8192x4096x14336", "op": "linear", "fmt": "nv", "tokens": 8192, "inner": 4096, "outer": 14336},
        # one step of a decode batch: one token each into blocks that are partly filled
        {"name": "append int8 64x1", "op": "append", "type": "int8", "heads": 8, "dim": 128, "page": 64, "requests": 64, "new": 1,
         "past_min": 0, "past_max": 4096, "seed": 1, "idle": False},
        # prompts of different lengths
        {"name": "append e4m3 6x2048", "op": "append", "type": "e4m3", "heads": 8, "dim": 128, "page": 16, "requests": 6, "new": 2048,
         "past_min": 0, "past_max": 500, "seed": 2, "idle": False},
        # one conversation with a long history
        {"name": "attention int8 1x1 in 100000", "op": "attention", "type": "int8", "heads": 8, "group": 4, "dim": 128, "page": 64, "requests": 1,
         "new": 1, "past_min": 100000, "past_max": 100000, "window": 0, "seed": 3, "idle": False},
        # a decode batch of ragged lengths
        {"name": "attention e4m3 64x1 in 8192", "op": "attention", "type": "e4m3", "heads": 8, "group": 4, "dim": 128, "page": 16, "requests": 64,
         "new": 1, "past_min": 100, "past_max": 8192, "window": 0, "seed": 4, "idle": False},
        # drafted tokens checked at once, with a sliding window; one request has nothing new
        {"name": "attention int8 16x5 window 4096", "op": "attention", "type": "int8", "heads": 8, "group": 4, "dim": 128, "page": 48, "requests": 16,
         "new": 5, "past_min": 0, "past_max": 20000, "window": 4096, "seed": 5, "idle": True},
        # chunks of prompts behind what the cache already holds
        {"name": "attention e4m3 4x1024 in 8192", "op": "attention", "type": "e4m3", "heads": 8, "group": 4, "dim": 128, "page": 32, "requests": 4,
         "new": 1024, "past_min": 0, "past_max": 8192, "window": 0, "seed": 6, "idle": False},
    ]


def draw(rng):
    def spread(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    while True:
        op = rng.choice(("round_trip", "linear", "linear", "append", "attention", "attention", "attention"))
        if op == "round_trip":
            c = {"op": op, "fmt": rng.choice(("mx", "nv")), "rows": spread(1, 16384), "cols": spread(64, 16384), "kind": rng.choice(("weights", "activations"))}
            fits = 4096 <= c["rows"] * c["cols"] <= 14336 * 4096
        elif op == "linear":
            c = {"op": op, "fmt": rng.choice(("mx", "nv")), "tokens": spread(1, 8192), "inner": spread(128, 14336), "outer": spread(64, 14336)}
            fits = c["tokens"] * c["inner"] * c["outer"] <= 8192 * 4096 * 14336
        else:
            step = rng.random() < 0.6                               # a step of a decode batch, or prompts
            c = {"op": op, "type": rng.choice(("int8", "e4m3")), "heads": rng.choice((1, 2, 4, 8)), "dim": rng.choice((64, 80, 96, 128, 128, 256)),
                 "page": rng.choice((16, 32, 48, 64, 128)), "requests": spread(1, 128) if step else spread(1, 8),
                 "new": spread(1, 8) if step else spread(9, 2048 if op == "append" else 1024), "past_min": 0,
                 "past_max": spread(1, 4096 if op == "append" else 32768), "seed": rng.randrange(1 << 30), "idle": rng.random() < 0.1}
            if op == "attention":
                c["group"] = rng.choice((1, 2, 3, 4, 4, 5, 7, 8, 8, 12))
                c["window"] = rng.choice((0, 0, 0, spread(16, 8192)))
                most = c["past_max"] + c["new"]
                fits = (c["requests"] * c["heads"] * c["group"] * c["new"] * most * max(128, c["dim"]) <= 4 * 32 * 1024 * 9216 * 128
                        and c["requests"] * c["heads"] * most * c["dim"] <= 64 * 8 * 8192 * 128)
            else:
                fits = c["requests"] * c["heads"] * c["dim"] * c["new"] <= 6 * 8 * 128 * 2048
        if fits and 3072 not in c.values():
            return c


def lengths(case):
    """[(tokens already in the cache, new tokens)] of the requests."""
    r = random.Random(case["seed"])
    got = [(r.randint(case["past_min"], case["past_max"]), r.randint((case["new"] + 1) // 2, case["new"])) for _ in range(case["requests"])]
    if case["idle"] and len(got) > 1:
        got[-1] = (got[-1][0], 0)
    return got


def work(case):
    if case["op"] == "round_trip":
        n = case["rows"] * case["cols"]
        held = n * (0.5 + 1 / BLOCK[case["fmt"]])
        return {"bytes": 2 * n + held + held + 2 * n, "flops": 2 * n}
    if case["op"] == "linear":
        t, i, o = case["tokens"], case["inner"], case["outer"]
        return {"bytes": 2 * t * i + o * i * (0.5 + 1 / BLOCK[case["fmt"]]) + 2 * t * o, "flops": 2 * t * i * o}
    h, d = case["heads"], case["dim"]
    if case["op"] == "append":
        new = sum(n for _, n in lengths(case))
        held = sum(p % TOKENS for p, n in lengths(case) if n)
        back = new + held
        return {"bytes": 2 * h * d * (2 * new + held + new + back + 2 * back), "flops": 4 * h * d * new}
    w, n_q, seen, pairs = case["window"], 0, 0, 0
    for past, new in lengths(case):
        n_q += new
        first = max(0, past - w + 1) if w else 0
        seen += past + new - first if new else 0
        pairs += sum(min(past + i + 1, w) if w else past + i + 1 for i in range(new))
    hq = h * case["group"]
    return {"bytes": seen * h * (2 * d + 4 / TOKENS) + n_q * hq * (4 * d + 4), "flops": 4 * d * hq * pairs}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _activations(rows, cols, g, dev):
    """Gaussian with channels of very different size, rows 16-byte aligned."""
    x = torch.empty(rows, -(-cols // 8) * 8, dtype=torch.bfloat16, device=dev)[:, :cols]
    x.copy_(torch.randn(rows, cols, generator=g, device=dev) * torch.randn(cols, generator=g, device=dev).mul(0.7).exp())
    return x


def _weights(rows, cols, g, dev):
    x = torch.empty(rows, -(-cols // 8) * 8, dtype=torch.bfloat16, device=dev)[:, :cols]
    w = torch.randn(rows, cols, generator=g, device=dev) * 0.02
    x.copy_(torch.where(torch.rand(rows, cols, generator=g, device=dev) < 1e-3, w * 20, w))
    return x


def _tensor_scale(x, fmt):
    """The whole matrix's scale: the power of two under which its largest block scale still fits e4m3."""
    if fmt == "mx":
        return None
    return torch.exp2(torch.ceil(torch.log2(x.float().abs().amax() / (6 * 448)))).reshape(1)


def _fp4_buffers(rows, cols, fmt, dev):
    tiles = -(-rows // 128) * -(-(-(-cols // 32) * 32 // BLOCK[fmt]) // 4)
    return torch.empty(rows, -(-cols // 32) * 16, dtype=torch.uint8, device=dev), torch.empty(tiles * 512, dtype=torch.uint8, device=dev)


def _ints(values, dev):
    return torch.tensor(values, dtype=torch.int32).to(dev)


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    s = dict(case)
    if case["op"] == "round_trip":
        rows, cols = case["rows"], case["cols"]
        s["x"] = (_weights if case["kind"] == "weights" else _activations)(rows, cols, g, dev)
        s["tensor_scale"] = _tensor_scale(s["x"], case["fmt"])
        s["codes"], s["scales"] = _fp4_buffers(rows, cols, case["fmt"], dev)
        s["out"] = torch.empty(rows, cols, dtype=torch.bfloat16, device=dev)
        return s
    if case["op"] == "linear":
        s["x"] = _activations(case["tokens"], case["inner"], g, dev)
        s["x_scale"] = _tensor_scale(s["x"], case["fmt"])
        w = _weights(case["outer"], case["inner"], g, dev)
        s["w_scale"] = _tensor_scale(w, case["fmt"])
        # the weights are kept quantised, in the layout of the format
        q, scale = _quantise(w, case["fmt"], s["w_scale"])
        s["w_codes"], s["w_scales"] = _pack(q), _tiled(scale)
        s["x_codes"], s["x_scales"] = _fp4_buffers(case["tokens"], case["inner"], case["fmt"], dev)
        s["out"] = torch.empty(case["tokens"], case["outer"], dtype=torch.bfloat16, device=dev)
        return s
    # requests in a cache whose pages are handed out in no order; tokens past a request's end hold whatever was there
    h, d, page, n = case["heads"], case["dim"], case["page"], lengths(case)
    per = max(1, max(-(-(p + m) // page) for p, m in n))
    need = sum(-(-(p + m) // page) for p, m in n)
    pages = need + 8
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    rows, at = np.zeros((len(n), per), dtype=np.int64), 0
    for i, (p, m) in enumerate(n):
        k = -(-(p + m) // page)
        rows[i, :k] = np.arange(at, at + k)
        at += k
    s["table"] = order[torch.from_numpy(rows).to(dev)].contiguous()
    s["lens"] = _ints([p + m for p, m in n], dev)
    s["starts"] = _ints([0] + list(np.cumsum([m for _, m in n])), dev)
    s["total"], s["max_new"], s["max_len"] = sum(m for _, m in n), max(m for _, m in n), max(p + m for p, m in n)
    for name in ("k", "v"):
        # codes as an append leaves them: the largest of every 16 tokens near the end of the range
        x = torch.randn(pages, h, page, d, generator=g, device=dev, dtype=torch.bfloat16)
        s[name] = (x * 32).round_().clamp_(-127, 127).to(torch.int8) if case["type"] == "int8" else (x * 100).clamp_(-448, 448).to(CODES["e4m3"])
        size = 1 / 32 if case["type"] == "int8" else 1 / 100
        s[name + "_scale"] = (torch.rand(pages, h, page // TOKENS, generator=g, device=dev).add(0.5) * size).to(torch.bfloat16)
    hq = h if case["op"] == "append" else h * case["group"]
    x = torch.randn(s["total"], (hq + 2 * h) * d, generator=g, device=dev).to(torch.bfloat16)      # one token's q, k and v side by side
    s["q"] = x[:, :hq * d].view(-1, hq, d)
    s["k_new"], s["v_new"] = x[:, hq * d:(hq + h) * d].view(-1, h, d), x[:, (hq + h) * d:].view(-1, h, d)
    if case["op"] == "append":
        # what is read back: the blocks of 16 tokens that the new ones share
        back = [m + p % TOKENS if m else 0 for p, m in n]
        s["back"], s["back_total"], s["max_back"] = _ints([0] + list(np.cumsum(back)), dev), sum(back), max(back)
        s["k_out"] = torch.empty(sum(back), h, d, dtype=torch.bfloat16, device=dev)
        s["v_out"] = torch.empty_like(s["k_out"])
    else:
        s["out"] = torch.empty(s["total"], hq, d, dtype=torch.bfloat16, device=dev)
        s["lse"] = torch.empty(s["total"], hq, dtype=torch.float32, device=dev)
    return s


# ---- a pass --------------------------------------------------------------------------------------------------------

_contexts = {}


def _library():
    """The library's context of the current stream, made once as a program does."""
    from paper_2602_17698_b200 import binding
    stream = torch.cuda.current_stream()
    key = stream.cuda_stream
    if key not in _contexts:
        _contexts[key] = binding.Context(stream=stream)
    return _contexts[key], binding


def run(s):
    if own:
        ctx, lib = _library()
        if s["op"] == "round_trip":
            m = lib.Fp4Matrix(s["codes"], s["scales"], s["rows"], s["cols"], s["fmt"], s["tensor_scale"])
            ctx.fp4_quantize(s["x"], m)
            return ctx.fp4_dequantize(m, out=s["out"])
        if s["op"] == "linear":
            x = lib.Fp4Matrix(s["x_codes"], s["x_scales"], s["tokens"], s["inner"], s["fmt"], s["x_scale"])
            w = lib.Fp4Matrix(s["w_codes"], s["w_scales"], s["outer"], s["inner"], s["fmt"], s["w_scale"])
            return ctx.fp4_gemm(ctx.fp4_quantize(s["x"], x), w, out=s["out"])
        cache = lib.Kv8Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"])
        if s["op"] == "append":
            ctx.kv8_append(cache, s["k_new"], s["v_new"], s["starts"], s["lens"], s["max_new"])
            k, v = ctx.kv8_read(cache, s["back"], s["lens"], s["max_back"], out=(s["k_out"], s["v_out"]))
            return {"k": k, "v": v, "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
        out, lse = ctx.kv8_attention(cache, s["q"], s["starts"], s["lens"], s["max_new"], s["max_len"], window=s["window"], out=s["out"], lse=s["lse"])
        return {"out": out, "lse": lse}
    if s["op"] == "round_trip":
        q, scale = _quantise(s["x"], s["fmt"], s["tensor_scale"])
        s["codes"].copy_(_pack(q))
        s["scales"].copy_(_tiled(scale))
        return _values(s["codes"], s["scales"], s["rows"], s["cols"], s["fmt"], s["tensor_scale"]).to(torch.bfloat16)
    if s["op"] == "linear":
        q, scale = _quantise(s["x"], s["fmt"], s["x_scale"])
        x = _values(_pack(q), _tiled(scale), s["tokens"], s["inner"], s["fmt"], s["x_scale"])
        w = _values(s["w_codes"], s["w_scales"], s["outer"], s["inner"], s["fmt"], s["w_scale"])
        return torch.matmul(x, w.t()).to(torch.bfloat16)
    if s["op"] == "append":
        _append(s, s["k"], s["k_scale"], s["k_new"])
        _append(s, s["v"], s["v_scale"], s["v_new"])
        return {"k": _read(s, s["k"], s["k_scale"]), "v": _read(s, s["v"], s["v_scale"]), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    return _attention(s)


# ---- the plain forms -----------------------------------------------------------------------------------------------
# (a quotient by a number is taken by a tensor of that number: torch would multiply by the rounded reciprocal)

def _quantise(x, fmt, tensor_scale):
    """Codes as whole numbers 0..15 [rows][cols padded to 32] and the scale bytes [rows][blocks]."""
    rows, cols = x.shape
    b = BLOCK[fmt]
    v = torch.zeros(rows, -(-cols // 32) * 32, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, -1, b)
    amax = v.abs().amax(-1)
    if fmt == "mx":
        e = (torch.frexp(amax).exponent - 3).clamp(-127, 127)          # floor(log2 amax) - 2
        e = torch.where(amax == 0, -127, e)
        scale, d = (e + 127).to(torch.uint8), _power(e)
    else:
        held = ((amax / torch.full_like(amax, 6)) / tensor_scale).clamp(max=448.0).to(torch.float8_e4m3fn)
        scale, d = held.view(torch.uint8), held.float() * tensor_scale
    r = torch.where(d[..., None] > 0, v / d[..., None], 0.0)
    a = r.abs()
    # the midpoints between neighbouring values; a tie goes to the even code
    q = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    return (q + torch.signbit(r).to(torch.uint8) * 8).view(rows, -1), scale


def _power(e):
    """2^e for whole e from -127 to 127, exact."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _pack(q):
    q = q.view(q.shape[0], -1, 2)
    return q[..., 0] | (q[..., 1] << 4)


def _tiled(scale):
    rows, n = scale.shape
    t = torch.zeros(-(-rows // 128) * 128, -(-n // 4) * 4, dtype=torch.uint8, device=scale.device)
    t[:rows, :n] = scale
    return t.view(t.shape[0] // 128, 4, 32, t.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1)


def _values(codes, scales, rows, cols, fmt, tensor_scale):
    """The 32-bit values that a 4-bit matrix stands for."""
    b = BLOCK[fmt]
    n = -(-cols // 32) * 32 // b
    t = scales.view(-(-rows // 128), -(-n // 4), 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-(-rows // 128) * 128, -(-n // 4) * 4)[:rows, :n].contiguous()
    s = _power(t.to(torch.int32) - 127) if fmt == "mx" else t.view(torch.float8_e4m3fn).float() * tensor_scale
    q = torch.stack((codes & 15, codes >> 4), -1).view(rows, -1)
    v = torch.tensor(E2M1 + tuple(-e for e in E2M1), device=codes.device)[q.to(torch.int32)]
    return (v.view(rows, n, b) * s[..., None]).view(rows, -1)[:, :cols]


def _up(x):
    """The smallest bf16 that is not below x."""
    b = x.to(torch.bfloat16)
    return torch.where(b.float() < x, (b.view(torch.int16) + 1).view(torch.bfloat16), b)


def _append(s, codes, scales, x):
    page, dev = s["page"], x.device
    lens, new = s["lens"].long(), (s["starts"][1:] - s["starts"][:-1]).long()
    past = lens - new
    block = past[:, None] // TOKENS + torch.arange(s["max_new"] // TOKENS + 2, device=dev)            # the blocks of 16 tokens that get new ones
    b, j = torch.nonzero((block * TOKENS < lens[:, None]) & (new > 0)[:, None], as_tuple=True)
    block = block[b, j]
    p = block[:, None] * TOKENS + torch.arange(TOKENS, device=dev)                                    # [blocks][16] positions
    old, fresh = p < past[b][:, None], (p >= past[b][:, None]) & (p < lens[b][:, None])
    where = s["table"][b, block * TOKENS // page].long()
    slot, group = p % page, block * TOKENS % page // TOKENS
    held = codes[where[:, None], :, slot].float() * old[..., None, None]                              # [blocks][16][heads][dim]
    coming = x[(s["starts"][b].long()[:, None] + p - past[b][:, None]).clamp(0, x.shape[0] - 1)].float() * fresh[..., None, None]
    before = scales[where, :, group].float() * old.any(1)[:, None]
    top = coming.abs().amax((1, 3))
    after = torch.maximum(before, _up(top / torch.full_like(top, QMAX[s["type"]])).float())
    at = after[:, None, :, None]
    q = torch.where(at > 0, (held * before[:, None, :, None] + coming) / at, 0.0)
    q = q.round().to(torch.int8) if s["type"] == "int8" else q.to(torch.float8_e4m3fn)
    i, t = torch.nonzero(old | fresh, as_tuple=True)
    codes.view(torch.uint8)[where[i], :, slot[i, t]] = q.view(torch.uint8)[i, t]
    scales[where, :, group] = after.to(torch.bfloat16)


def _read(s, codes, scales):
    page = s["page"]
    n = (s["back"][1:] - s["back"][:-1]).long()
    b = torch.repeat_interleave(torch.arange(len(n), device=n.device), n, output_size=s["back_total"])
    p = s["lens"][b].long() - n[b] + torch.arange(s["back_total"], device=n.device) - s["back"][b].long()
    where, slot = s["table"][b, p // page].long(), p % page
    return (codes[where, :, slot].float() * scales[where, :, slot // TOKENS].float()[..., None]).to(torch.bfloat16)


def _attention(s):
    h, g, d, page, dev = s["heads"], s["group"], s["dim"], s["page"], s["q"].device
    n, most, queries = len(s["lens"]), s["max_len"], s["max_new"]
    lens, new = s["lens"].long(), (s["starts"][1:] - s["starts"][:-1]).long()
    # every request padded to the longest
    p = torch.arange(most, device=dev)
    where, slot = s["table"][:, p // page].long(), (p % page).expand(n, -1)
    k = (s["k"][where, :, slot].float() * s["k_scale"][where, :, slot // TOKENS].float()[..., None]).transpose(1, 2)       # [n][heads][most][dim]
    v = (s["v"][where, :, slot].float() * s["v_scale"][where, :, slot // TOKENS].float()[..., None]).transpose(1, 2)
    i = torch.arange(queries, device=dev)
    row = (s["starts"][:-1].long()[:, None] + i).clamp(max=s["total"] - 1)
    q = s["q"][row].float().view(n, queries, h, g, d).permute(0, 2, 3, 1, 4).reshape(n, h, g * queries, d)
    at = (lens - new)[:, None, None] + i[:, None]                                                                          # the queries' positions
    seen = (p <= at) & (i < new[:, None])[..., None]
    seen = seen & (p > at - s["window"]) if s["window"] else seen
    x = torch.matmul(q, k.transpose(2, 3)).mul_(d ** -0.5).view(n, h, g, queries, most)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    e = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = e.sum(-1, keepdim=True)
    v = torch.where((p < lens[:, None])[:, None, :, None], v, 0.0)
    o = torch.matmul(e.view(n, h, g * queries, most), v).view(n, h, g, queries, d) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).squeeze(-1)
    b, j = torch.nonzero(i < new[:, None], as_tuple=True)
    return {"out": o.permute(0, 3, 1, 2, 4)[b, j].reshape(-1, h * g, d).to(torch.bfloat16), "lse": lse.permute(0, 3, 1, 2)[b, j].reshape(-1, h * g)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    dev = s["table"].device if "table" in s else s["x"].device
    grid = torch.tensor(E2M1, dtype=torch.float64, device=dev)

    def four_bits(x, fmt, scale):
        """What a matrix stands for once it is held in 4 bits."""
        rows, cols = x.shape
        b = BLOCK[fmt]
        v = torch.nn.functional.pad(x.double(), (0, -cols % b)).view(rows, -1, b)
        m = v.abs().amax(-1, keepdim=True)
        if fmt == "mx":
            d = torch.exp2((torch.frexp(m).exponent.double() - 1).clamp(-125, 129) - 2)     # frexp: m = f 2^e with f in [1/2, 1)
        else:
            m = m / 6 / scale.double()
            ulp = torch.exp2(torch.frexp(m.clamp(min=2.0 ** -6)).exponent.double() - 4)       # e4m3: three bits behind the leading one
            d = (torch.round(m / ulp) * ulp).clamp(max=448.0) * scale.double()
        r = torch.where(d > 0, v.abs() / d, 0.0).clamp(max=6.0)
        low = torch.bucketize(r, grid, right=True) - 1                                   # the grid point at or below r
        high = (low + 1).clamp(max=7)
        half = (grid[low] + grid[high]) / 2
        pick = torch.where((r > half) | ((r == half) & (low % 2 == 1)), high, low)
        return (torch.where(low == 7, 6.0, grid[pick]) * v.sign() * d).view(rows, -1)[:, :cols]

    def eight_bits(x, kind):
        if kind == "int8":
            return torch.round(x)
        ulp = torch.exp2(torch.frexp(x.abs().clamp(min=2.0 ** -6)).exponent.double() - 4)
        return torch.round(x / ulp) * ulp

    if case["op"] == "round_trip":
        return four_bits(s["x"], case["fmt"], s["tensor_scale"])
    if case["op"] == "linear":
        b, rows, cols = BLOCK[case["fmt"]], case["outer"], case["inner"]
        n = -(-cols // 32) * 32 // b
        r, j = torch.arange(rows, device=dev)[:, None], torch.arange(n, device=dev)
        byte = s["w_scales"][((r // 128) * -(-n // 4) + j // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + j % 4]
        scale = torch.exp2(byte.double() - 127) if case["fmt"] == "mx" else byte.view(torch.float8_e4m3fn).double() * s["w_scale"].double()
        c = torch.arange(cols, device=dev)
        q = (s["w_codes"][:, c // 2] >> (c % 2 * 4).to(torch.uint8)) & 15
        w = grid[(q & 7).long()] * torch.where(q > 7, -1.0, 1.0) * scale[:, c // b]
        return four_bits(s["x"], case["fmt"], s["x_scale"]) @ w.t()
    page, n = case["page"], lengths(case)
    if case["op"] == "append":
        got = {"k_scale": s["k_scale"].double(), "v_scale": s["v_scale"].double(), "k": [], "v": []}
        table = s["table"].long().cpu()
        at = 0
        for i, (past, new) in enumerate(n):
            for name in ("k", "v"):
                if not new:
                    continue
                first = past // TOKENS * TOKENS
                pos = torch.arange(first, past + new)
                where, slot, group = table[i][pos // page].to(dev), (pos % page).to(dev), (pos % page // TOKENS).to(dev)
                blk = ((pos - first) // TOKENS).to(dev)
                count = int(blk[-1]) + 1
                held = past - first
                x = s[name + "_new"][at:at + new].double()
                top = torch.zeros(count, case["heads"], dtype=torch.float64, device=dev)
                top.index_reduce_(0, blk[held:], x.abs().amax(-1), "amax")
                need = top / QMAX[case["type"]]
                ulp = torch.exp2(torch.frexp(need).exponent.double() - 8)                # bf16: seven bits behind the leading one, rounded up
                scale = torch.where(need > 0, torch.ceil(need / ulp) * ulp, 0.0)
                old = got[name + "_scale"][where[0], :, group[0]].clone()
                if held:
                    scale[0] = torch.maximum(scale[0], old)
                values = torch.cat((s[name][where[:held], :, slot[:held]].double() * old[..., None], x))
                q = eight_bits(values / scale[blk][..., None], case["type"])
                got[name].append(torch.nan_to_num(q * scale[blk][..., None]))
                got[name + "_scale"][where, :, group] = scale[blk]
            at += new
        empty = torch.zeros(0, case["heads"], case["dim"], dtype=torch.float64, device=dev)
        return {k: torch.cat(v) if isinstance(v, list) and v else empty if isinstance(v, list) else v for k, v in got.items()}
    outs, lses, at = [], [], 0
    h, g, d = case["heads"], case["group"], case["dim"]
    for i, (past, new) in enumerate(n):
        if not new:
            continue
        pos = torch.arange(past + new, device=dev)
        where, slot = s["table"][i].long()[pos // page], pos % page
        k = (s["k"][where, :, slot].double() * s["k_scale"][where, :, slot // TOKENS].double()[..., None]).transpose(0, 1)     # [heads][keys][dim]
        v = (s["v"][where, :, slot].double() * s["v_scale"][where, :, slot // TOKENS].double()[..., None]).transpose(0, 1)
        t = torch.arange(past, past + new, device=dev)[:, None]
        mask = (pos <= t) & (pos > t - case["window"]) if case["window"] else pos <= t
        q = s["q"][at:at + new].double().view(new, h, g, d)
        o, l = torch.empty_like(q), torch.empty(new, h, g, dtype=torch.float64, device=dev)
        for j in range(g):
            x = torch.where(mask, torch.matmul(q[:, :, j].transpose(0, 1), k.transpose(1, 2)) / math.sqrt(d), -math.inf)     # [heads][new][keys]
            l[:, :, j] = torch.logsumexp(x, -1).t()
            o[:, :, j] = torch.matmul(torch.softmax(x, -1), v).transpose(0, 1)
        outs.append(o.view(new, h * g, d))
        lses.append(l.view(new, h * g))
        at += new
    if not outs:
        return {"out": torch.zeros(0, h * g, d, dtype=torch.float64, device=dev), "lse": torch.zeros(0, h * g, dtype=torch.float64, device=dev)}
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
