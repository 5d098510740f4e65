"""Cases of the operators around the attention of a quantised decoder: rotary positions, a key/value cache held in 4 bits with its attention, and
low-rank adapters of many requests beside a shared projection.

`run` computes a case either in plain tensor operations (in 32 bits, angles in 64; `own` false) or by the calls a program makes of the library (`own` true).

What both sides of `run` take:

* requests: request i has `lens` tokens by now, the last `starts[i + 1] - starts[i]` of which are the call's rows `starts[i] ..`.
* rotary positions: a table of frequencies, fp32 [rotated / 2], in radians per position; pairs of a head are (i, i + rotated / 2) ("half") or
  (2 i, 2 i + 1) ("interleaved"), elements from `rotated` on stay as they are.
* the cache: [pages][heads][page tokens] rows of e2m1 codes, two to a byte (even element in the low half), padded with zeros to a multiple of 32
  elements; an e4m3 scale byte for every 16 elements of a row, rows of scales padded to a multiple of 4; one fp32 scale for every head of the keys and of
  the values; a table of page numbers [requests][pages of a request].
* adapters: a [adapters][rank][in] and b [adapters][out][rank] in bf16, an fp32 scale each; the adapter of every request, -1 for none.
"""
import math
import random

import numpy as np
import torch

own = False

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = 16           # elements that share a scale of the cache


# ---- cases ---------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one step of a decode batch: queries and keys side by side in the projection's result
        {"name": "rotary half 64x1", "op": "rotary", "pairs": "half", "heads": 8, "group": 4, "dim": 128, "rotated": 128, "stretch": 1.0, "requests": 64,
         "new": 1, "past_min": 0, "past_max": 8192, "seed": 11, "back": False},
        # prompts of different lengths, frequencies scaled for a long context
        {"name": "rotary half 6x2048", "op": "rotary", "pairs": "half", "heads": 8, "group": 4, "dim": 128, "rotated": 128, "stretch": 8.0, "requests": 6,
         "new": 2048, "past_min": 0, "past_max": 100000, "seed": 12, "back": False},
        # a quarter of the head in neighbouring pairs, as gradients come back through it
        {"name": "rotary interleaved back 8x700", "op": "rotary", "pairs": "interleaved", "heads": 16, "group": 1, "dim": 80, "rotated": 20, "stretch": 1.0,
         "requests": 8, "new": 700, "past_min": 0, "past_max": 0, "seed": 13, "back": True},
        # one step of a decode batch into the cache
        {"name": "append 64x1", "op": "append", "heads": 8, "dim": 128, "page": 64, "requests": 64, "new": 1, "past_min": 0, "past_max": 4096, "seed": 1,
         "idle": False},
        # prompts of different lengths into the cache
        {"name": "append 6x2048", "op": "append", "heads": 8, "dim": 128, "page": 16, "requests": 6, "new": 2048, "past_min": 0, "past_max": 500, "seed": 2,
         "idle": False},
        # one conversation with a long history
        {"name": "attention 1x1 in 100000", "op": "attention", "heads": 8, "group": 4, "dim": 128, "page": 64, "requests": 1, "new": 1,
         "past_min": 100000, "past_max": 100000, "window": 0, "seed": 3, "idle": False},
        # a decode batch of ragged lengths
        {"name": "attention 64x1 in 8192", "op": "attention", "heads": 8, "group": 4, "dim": 128, "page": 16, "requests": 64, "new": 1, "past_min": 100,
         "past_max": 8192, "window": 0, "seed": 4, "idle": False},
        # drafted tokens checked at once, with a sliding window; one request has nothing new
        {"name": "attention 16x5 window 4096", "op": "attention", "heads": 8, "group": 4, "dim": 128, "page": 48, "requests": 16, "new": 5, "past_min": 0,
         "past_max": 20000, "window": 4096, "seed": 5, "idle": True},
        # chunks of prompts behind what the cache already holds
        {"name": "attention 4x1024 in 8192", "op": "attention", "heads": 8, "group": 4, "dim": 128, "page": 32, "requests": 4, "new": 1024, "past_min": 0,
         "past_max": 8192, "window": 0, "seed": 6, "idle": False},
        # one token of one request beside the output projection: latency
        {"name": "adapters 1x1 rank 16 4096x4096", "op": "adapters", "requests": 1, "new": 1, "inner": 4096, "outer": 4096, "rank": 16, "adapters": 4,
         "f32": False, "seed": 7, "idle": False},
        # a decode batch whose requests have an adapter each, beside the query, key and value projection
        {"name": "adapters 64x1 rank 16 4096x6144", "op": "adapters", "requests": 64, "new": 1, "inner": 4096, "outer": 6144, "rank": 16, "adapters": 64,
         "f32": False, "seed": 8, "idle": False},
        # prompts of different lengths beside the same projection, some without an adapter
        {"name": "adapters 6x2048 rank 64 4096x6144", "op": "adapters", "requests": 6, "new": 2048, "inner": 4096, "outer": 6144, "rank": 64, "adapters": 4,
         "f32": False, "seed": 9, "idle": True},
    ]


def draw(rng):
    def spread(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    while True:
        op = rng.choice(("rotary", "append", "attention", "attention", "attention", "adapters", "adapters"))
        step = rng.random() < 0.6                                   # a step of a decode batch, or prompts
        c = {"op": op, "requests": spread(1, 128) if step else spread(1, 8), "seed": rng.randrange(1 << 30), "idle": rng.random() < 0.1,
             "new": spread(1, 8) if step else spread(9, 1024 if op == "attention" else 2048)}
        if op == "adapters":
            c["inner"], c["rank"], c["adapters"] = 8 * spread(16, 1792), rng.choice((8, 16, 16, 32, 64, 128)), spread(1, 64)
            c["outer"] = 8 * spread(8, 1792) if rng.random() < 0.8 else spread(64, 14336)
            c["f32"] = rng.random() < 0.25
            rows = c["requests"] * c["new"]
            fits = rows * (c["inner"] + 2 * c["outer"]) <= 6 * 2048 * (4096 + 2 * 6144) and rows * c["rank"] * (c["inner"] + c["outer"]) <= 6 * 2048 * 64 * 10240 \
                and c["adapters"] * c["rank"] * (c["inner"] + c["outer"]) <= 64 * 64 * 10240
        else:
            c["heads"], c["dim"] = rng.choice((1, 2, 4, 8)), rng.choice((64, 80, 96, 128, 128, 256))
            c["past_min"], c["past_max"] = 0, spread(1, 4096 if op == "append" else 32768)
            if op == "rotary":
                del c["idle"]
                c["group"], c["pairs"], c["back"] = rng.choice((1, 2, 4, 5, 8)), rng.choice(("half", "interleaved")), rng.random() < 0.3
                c["rotated"], c["stretch"] = rng.choice((c["dim"], c["dim"], c["dim"] // 2, c["dim"] // 4)), rng.choice((1.0, 4.0, 8.0, 32.0))
                fits = c["requests"] * c["new"] * c["heads"] * (c["group"] + 1) * c["dim"] <= 6 * 2048 * 40 * 128
            else:
                c["page"] = rng.choice((16, 32, 48, 64, 128))
            if op == "attention":
                c["group"] = rng.choice((1, 2, 3, 4, 4, 5, 7, 8, 8, 12))
                c["window"] = rng.choice((0, 0, 0, spread(16, 8192)))
                most = c["past_max"] + c["new"]
                fits = (c["requests"] * c["heads"] * c["group"] * c["new"] * most * max(128, c["dim"]) <= 4 * 32 * 1024 * 9216 * 128
                        and c["requests"] * c["heads"] * most * c["dim"] <= 64 * 8 * 8192 * 128)
            elif op == "append":
                fits = c["requests"] * c["heads"] * c["dim"] * c["new"] <= 6 * 8 * 128 * 2048
        if fits:
            return c


def lengths(case):
    """[(tokens a request had before, its new tokens)]."""
    r = random.Random(case["seed"])
    got = [(r.randint(case.get("past_min", 0), case.get("past_max", 0)), r.randint((case["new"] + 1) // 2, case["new"])) for _ in range(case["requests"])]
    if case.get("idle") and len(got) > 1:
        got[-1] = (got[-1][0], 0)
    return got


def adapter_ids(case):
    """The requests' adapters: each its own where there are as many, else any of them, and for some none."""
    r = random.Random(case["seed"] + 1)
    if case["adapters"] == case["requests"]:
        return r.sample(range(case["adapters"]), case["requests"])
    return [-1 if r.random() < 0.1 and i else r.randrange(case["adapters"]) for i in range(case["requests"])]


def work(case):
    n = lengths(case)
    new = sum(m for _, m in n)
    if case["op"] == "rotary":
        heads = case["heads"] * (case["group"] + 1)
        return {"bytes": new * heads * 4 * case["dim"], "flops": new * heads * 3 * case["rotated"]}
    if case["op"] == "adapters":
        ids, i, o, r = adapter_ids(case), case["inner"], case["outer"], case["rank"]
        has = sum(m for (_, m), a in zip(n, ids) if a >= 0)
        used = len({a for (_, m), a in zip(n, ids) if a >= 0 and m})
        size = 4 if case["f32"] else 2
        return {"bytes": 2 * has * i + 2 * size * new * o + 2 * used * r * (i + o), "flops": 2 * has * r * (i + o)}
    h, d = case["heads"], case["dim"]
    row = d / 2 + d / BLOCK
    if case["op"] == "append":
        return {"bytes": 2 * h * new * (2 * d + row + row + 2 * d), "flops": 4 * h * d * new}
    w, seen, pairs = case["window"], 0, 0
    for past, m in n:
        first = max(0, past - w + 1) if w else 0
        seen += past + m - first if m else 0
        pairs += sum(min(past + i + 1, w) if w else past + i + 1 for i in range(m))
    hq = h * case["group"]
    return {"bytes": seen * h * 2 * row + new * hq * (4 * d + 4), "flops": 4 * d * hq * pairs}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _ints(values, dev):
    return torch.tensor(values, dtype=torch.int32).to(dev)


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    s, n = dict(case), lengths(case)
    s["lens"], s["starts"] = _ints([p + m for p, m in n], dev), _ints([0] + list(np.cumsum([m for _, m in n])), dev)
    s["total"], s["max_new"], s["max_len"] = sum(m for _, m in n), max(m for _, m in n), max(p + m for p, m in n)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.bfloat16)

    if case["op"] == "adapters":
        t, i, o, r = s["total"], case["inner"], case["outer"], case["rank"]
        # activations with channels of very different size; the shared projection's result is there already
        s["x"] = (normal(t, i) * torch.randn(i, generator=g, device=dev).mul(0.7).exp()).to(torch.bfloat16)
        s["base"] = normal(t, o).float() if case["f32"] else normal(t, o)
        s["a"] = normal(case["adapters"], r, i) * i ** -0.5
        s["b"] = normal(case["adapters"], o, r) * 0.05
        s["scale"] = torch.rand(case["adapters"], generator=g, device=dev) + 0.5
        s["ids"] = _ints(adapter_ids(case), dev)
        s["out"] = torch.empty_like(s["base"])
        return s
    h, d = case["heads"], case["dim"]
    hq = h * case.get("group", 1)
    x = normal(s["total"], (hq + 2 * h) * d)                                       # one token's q, k and v side by side
    s["q"], s["k_new"], s["v_new"] = (t.view(-1, t.shape[1] // d, d) for t in x.split((hq * d, h * d, h * d), 1))
    if case["op"] == "rotary":
        half = case["rotated"] // 2
        f = 10000.0 ** (-np.arange(half) / half)
        # slow pairs, which turn less than once in 8192 positions, are stretched
        s["freq"] = torch.from_numpy(np.where(f * 8192 < 2 * math.pi, f / case["stretch"], f).astype(np.float32)).to(dev)
        s["factor"] = 0.1 * math.log(case["stretch"]) + 1.0
        s["out"] = (torch.empty(s["total"], hq, d, dtype=torch.bfloat16, device=dev), torch.empty(s["total"], h, d, dtype=torch.bfloat16, device=dev))
        return s
    # requests in a cache whose pages are handed out in no order; what no request holds is whatever was there
    page = case["page"]
    need = [-(-(p + m) // page) for p, m in n]
    pages = sum(need) + 8
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    rows, at = np.zeros((len(n), max(1, max(need))), dtype=np.int64), 0
    for i, k in enumerate(need):
        rows[i, :k] = np.arange(at, at + k)
        at += k
    s["table"] = order[torch.from_numpy(rows).to(dev)].contiguous()
    for name in ("k", "v"):
        # a program calibrates one scale for every head
        s[name + "_head"] = torch.exp2(torch.randint(-2, 2, (h,), generator=g, device=dev).float())
        s[name] = torch.empty(pages, h, page, -(-d // 32) * 16, dtype=torch.uint8, device=dev)
        s[name + "_scale"] = torch.empty(pages, h, page, -(-d // 64) * 4, dtype=torch.uint8, device=dev)
        for p in range(0, pages, 2048):
            part = slice(p, min(pages, p + 2048))
            s[name][part], s[name + "_scale"][part] = _quantise(normal(part.stop - p, h, page, d).transpose(1, 2), s[name + "_head"], True)
    if case["op"] == "append":
        s["k_out"] = torch.empty(s["total"], h, d, dtype=torch.bfloat16, device=dev)
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
    key = stream.device_index, stream.cuda_stream
    if key not in _contexts:
        _contexts[key] = binding.Context(stream=stream)
    return _contexts[key], binding


def run(s):
    if own:
        ctx, lib = _library()
        if s["op"] == "rotary":
            table = lib.RotaryTable(s["freq"], interleaved=s["pairs"] == "interleaved", factor=s["factor"])
            q, k = ctx.rotary(table, s["q"], s["k_new"], starts=s["starts"], lens=s["lens"], max_new=s["max_new"], inverse=s["back"], out=s["out"])
            return {"q": q, "k": k}
        if s["op"] == "adapters":
            adapters = lib.LoraAdapters(s["a"], s["b"], s["scale"])
            return ctx.lora_add(adapters, s["x"], s["base"], s["ids"], s["starts"], s["max_new"], out=s["out"])
        cache = lib.Kv4Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], s["dim"], s["k_head"], s["v_head"])
        if s["op"] == "append":
            ctx.kv4_append(cache, s["k_new"], s["v_new"], s["starts"], s["lens"], s["max_new"])
            k, v = ctx.kv4_read(cache, s["starts"], s["lens"], s["max_new"], out=(s["k_out"], s["v_out"]))
            return {"k": k, "v": v}
        out, lse = ctx.kv4_attention(cache, s["q"], s["starts"], s["lens"], s["max_new"], s["max_len"], window=s["window"], out=s["out"], lse=s["lse"])
        return {"out": out, "lse": lse}
    if s["op"] == "rotary":
        b, p = _positions(s)
        angle = p.double()[:, None] * s["freq"].double() * (-1.0 if s["back"] else 1.0)
        c, z = ((t * s["factor"]).float()[:, None] for t in (angle.cos(), angle.sin()))
        return {name: _turned(x, c, z, s["pairs"]) for name, x in (("q", s["q"]), ("k", s["k_new"]))}
    if s["op"] == "adapters":
        a = s["ids"][_request_of(s)].long()
        x = torch.matmul(s["x"].float(), s["a"].float().flatten(0, 1).t()).view(len(a), -1, s["rank"])
        x *= torch.where(torch.arange(s["adapters"], device=a.device) == a[:, None], s["scale"], 0.0)[..., None]
        y = torch.matmul(x.flatten(1), s["b"].float().transpose(1, 2).flatten(0, 1)).add_(s["base"])
        return y.to(s["base"].dtype)
    if s["op"] == "append":
        b, p = _positions(s)
        page = s["table"][b, p // s["page"]].long()
        got = {}
        for name in ("k", "v"):
            codes, scales = _quantise(s[name + "_new"], s[name + "_head"])
            s[name][page, :, p % s["page"]] = codes
            s[name + "_scale"][page, :, p % s["page"]] = scales
            got[name] = (_values(s[name][page, :, p % s["page"]], s[name + "_scale"][page, :, p % s["page"]], s["dim"])
                         * s[name + "_head"][:, None]).to(torch.bfloat16)
        return got
    return _attention(s)


# ---- the plain forms -----------------------------------------------------------------------------------------------
# (a quotient by a number is taken by a tensor of that number: torch would multiply by the rounded reciprocal)

def _request_of(s):
    n = (s["starts"][1:] - s["starts"][:-1]).long()
    return torch.repeat_interleave(torch.arange(len(n), device=n.device), n, output_size=s["total"])


def _positions(s):
    """Request and position of every row."""
    b = _request_of(s)
    return b, s["lens"][b].long() - s["starts"][b + 1].long() + torch.arange(s["total"], device=b.device)


def _turned(x, c, z, pairs):
    half = c.shape[-1]
    v = x[..., :2 * half].float()
    i, j = (v[..., :half], v[..., half:]) if pairs == "half" else (v[..., ::2], v[..., 1::2])
    i, j = i * c - j * z, j * c + i * z
    v = torch.cat((i, j), -1) if pairs == "half" else torch.stack((i, j), -1).flatten(-2)
    return torch.cat((v.to(x.dtype), x[..., 2 * half:]), -1)


def _quantise(x, head, pages=False):
    """Code bytes and scale bytes of [tokens][heads][dim]; pages: [pages][page tokens][heads][dim] as pages hold them."""
    x = x.float()
    head = head[:, None]
    if pages:
        x, head = x.transpose(1, 2), head[:, None]
    dim = x.shape[-1]
    v = torch.nn.functional.pad(x, (0, -dim % 32)).unflatten(-1, (-1, BLOCK))
    top = v.abs().amax(-1)
    scale = ((top / torch.full_like(top, 6)) / head).clamp(max=448.0).to(torch.float8_e4m3fn)
    d = (scale.float() * head)[..., None]
    r = torch.where(d > 0, v / d, 0.0).flatten(-2)
    a = r.abs()
    # the midpoints between neighbouring values; a tie goes to the even code
    q = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    q = q + torch.signbit(r).to(torch.uint8) * 8
    held = -(-dim // 64) * 4
    return q[..., ::2] | (q[..., 1::2] << 4), torch.nn.functional.pad(scale.view(torch.uint8), (0, 4))[..., :held]


def _values(codes, scales, dim):
    """32-bit values of rows of the cache, before their head's scale."""
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()
    v = torch.tensor(E2M1 + tuple(-e for e in E2M1), device=codes.device)[q]
    blocks = v.shape[-1] // BLOCK
    scale = torch.nn.functional.pad(scales, (0, 2))[..., :blocks].contiguous().view(torch.float8_e4m3fn).float()
    return (v.unflatten(-1, (-1, BLOCK)) * scale[..., None]).flatten(-2)[..., :dim]


def _attention(s):
    h, g, d, page, dev = s["heads"], s["group"], s["dim"], s["page"], s["q"].device
    n, most, queries = len(s["lens"]), s["max_len"], s["max_new"]
    lens, new = s["lens"].long(), (s["starts"][1:] - s["starts"][:-1]).long()
    # every request padded to the longest
    p = torch.arange(most, device=dev)
    where, slot = s["table"][:, p // page].long(), (p % page).expand(n, -1)
    k, v = ((_values(s[x][where, :, slot], s[x + "_scale"][where, :, slot], d) * s[x + "_head"][:, None]).transpose(1, 2) for x in ("k", "v"))
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
    dev, n = s["starts"].device, lengths(case)
    if case["op"] == "rotary":
        half, at = case["rotated"] // 2, 0
        pick = torch.arange(half, device=dev)
        i, j = (pick, pick + half) if case["pairs"] == "half" else (2 * pick, 2 * pick + 1)
        got = {"q": s["q"].double(), "k": s["k_new"].double()}
        for past, new in n:
            for p in range(new):
                angle = (past + p) * s["freq"].double()
                turn = torch.polar(torch.full_like(angle, s["factor"]), -angle if case["back"] else angle)
                for x in got.values():
                    z = torch.complex(x[at, :, i], x[at, :, j]) * turn
                    x[at, :, i], x[at, :, j] = z.real, z.imag
                at += 1
        return got
    if case["op"] == "adapters":
        y, at = s["base"].double(), 0
        for (_, new), a in zip(n, adapter_ids(case)):
            if a >= 0 and new:
                y[at:at + new] += s["scale"][a].double() * ((s["x"][at:at + new].double() @ s["a"][a].double().t()) @ s["b"][a].double().t())
            at += new
        return y
    grid = torch.tensor(E2M1, dtype=torch.float64, device=dev)
    if case["op"] == "append":
        got = {}
        for name in ("k", "v"):
            x, g = s[name + "_new"].double(), s[name + "_head"].double()[:, None, None]
            x = x.unflatten(-1, (-1, BLOCK))
            m = x.abs().amax(-1, keepdim=True) / 6 / g
            ulp = torch.exp2(torch.frexp(m.clamp(min=2.0 ** -6)).exponent.double() - 4)           # e4m3: three bits behind the leading one
            d = (torch.round(m / ulp) * ulp).clamp(max=448.0) * g
            r = torch.where(d > 0, x.abs() / d, 0.0).clamp(max=6.0)
            low = torch.bucketize(r, grid, right=True) - 1                                        # the grid point at or below r
            high = (low + 1).clamp(max=7)
            half = (grid[low] + grid[high]) / 2
            up = (r > half) | ((r == half) & (low % 2 == 1))
            got[name] = (torch.where(up, grid[high], grid[low]) * x.sign() * d).flatten(-2)
        return got
    h, g, d, page = case["heads"], case["group"], case["dim"], case["page"]

    def rows(name, i, upto):
        """Values of a request's tokens [heads][upto][dim]."""
        pos, c = torch.arange(upto, device=dev), torch.arange(d, device=dev)
        where, slot = s["table"][i].long()[pos // page], pos % page
        q = (s[name][where, :, slot][..., c // 2] >> (c % 2 * 4).to(torch.uint8)) & 15
        scale = s[name + "_scale"][where, :, slot].view(torch.float8_e4m3fn).double()[..., c // BLOCK] * s[name + "_head"].double()[:, None]
        return (grid[(q & 7).long()] * torch.where(q > 7, -1.0, 1.0) * scale).transpose(0, 1)

    out, lse, at = torch.zeros(s["total"], h, g, d, dtype=torch.float64, device=dev), torch.zeros(s["total"], h, g, dtype=torch.float64, device=dev), 0
    for i, (past, new) in enumerate(n):
        if not new:
            continue
        k, v, pos = rows("k", i, past + new), rows("v", i, past + new), torch.arange(past + new, device=dev)
        t = torch.arange(past, past + new, device=dev)[:, None]
        mask = (pos <= t) & (pos > t - case["window"]) if case["window"] else pos <= t
        q = s["q"][at:at + new].double().view(new, h, g, d)
        for j in range(g):
            x = torch.where(mask, torch.matmul(q[:, :, j].transpose(0, 1), k.transpose(1, 2)) / math.sqrt(d), -math.inf)         # [heads][new][keys]
            lse[at:at + new, :, j] = torch.logsumexp(x, -1).t()
            out[at:at + new, :, j] = torch.matmul(torch.softmax(x, -1), v).transpose(0, 1)
        at += new
    return {"out": out.view(-1, h * g, d), "lse": lse.view(-1, h * g)}
