"""Workloads of the serving operators: few-token products with MX-packed weights, appending rotated keys and values to an
MX-packed paged cache, and the attention of one new token over that cache.

`listed()` names the fixed cases, `draw()` makes more of the same ranges, `prepare()` the inputs of one, `run()` makes one
pass: with `own` the library's calls, without it the same operators in elementary torch operations on 32-bit values.
`work()` counts the bytes and operations a pass cannot do without, `exact()` gives the results in 64 bits.

All packed tensors are line-major planes (shared exponents, microexponents, codes) with 16-byte pitches, as the library's
pack call writes them: a weight row is a line of K elements; a cache line is one token's n_kv * head_dim elements.
"""
import math
import random

import torch

own = False

MANTISSA = {"mx4": 2, "mx6": 4, "mx9": 7}          # magnitude bits; a code has one more (the sign)
BITS = {"mx4": 4.0, "mx6": 6.0, "mx9": 9.0}        # bits per element with both scale levels
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ------------------------------------------------------------------------------------------------------------------

def gemv(name, fmt, tokens, n, k, dtype, out=None):
    return {"name": name, "op": "gemv", "fmt": fmt, "tokens": tokens, "n": n, "k": k, "dtype": dtype, "out": out or dtype}


def append(name, fmt_k, fmt_v, tokens, n_q, n_kv, head_dim, dtype, rot_dim, interleaved=False, padding=0, page=16):
    return {"name": name, "op": "append", "fmt_k": fmt_k, "fmt_v": fmt_v, "tokens": tokens, "n_q": n_q, "n_kv": n_kv,
            "head_dim": head_dim, "dtype": dtype, "rot_dim": rot_dim, "interleaved": interleaved, "padding": padding, "page": page}


def attend(name, fmt_k, fmt_v, batch, shortest, longest, n_q, n_kv, head_dim, dtype, page=16, window=0):
    return {"name": name, "op": "attend", "fmt_k": fmt_k, "fmt_v": fmt_v, "batch": batch, "shortest": shortest, "longest": longest,
            "n_q": n_q, "n_kv": n_kv, "head_dim": head_dim, "dtype": dtype, "page": page, "window": window}


def listed():
    return [
        # a projection of one decoded token: the smallest product of a serving step, where the launch counts
        gemv("gemv mx4 1x4096x4096", "mx4", 1, 4096, 4096, "bf16"),
        # the widening linear layer of the library's training benchmark, one token
        gemv("gemv mx6 1x16384x4096", "mx6", 1, 16384, 4096, "bf16"),
        # a large layer and a batch of sixteen streams, logits-like 32-bit output
        gemv("gemv mx9 16x16384x8192", "mx9", 16, 16384, 8192, "bf16", "f32"),
        # nothing a multiple of anything: short last block, odd rows, 32-bit activations
        gemv("gemv mx6 3x5003x2063 f32", "mx6", 3, 5003, 2063, "f32"),
        # one stream, one new token
        append("append mx9 1 token", "mx9", "mx9", 1, 32, 8, 128, "bf16", 128),
        # a prompt of 16384 tokens with grouped heads
        append("append mx9 16384 tokens", "mx9", "mx9", 16384, 32, 8, 128, "bf16", 128),
        # mixed formats, part of the head rotated in neighbouring pairs, ragged batch padded with empty slots
        append("append mx6/mx4 1003 f32", "mx6", "mx4", 1003, 20, 4, 80, "f32", 32, interleaved=True, padding=61, page=24),
        # one short conversation
        attend("attend mx9 1x777", "mx9", "mx9", 1, 777, 777, 32, 8, 128, "bf16"),
        # a serving batch of many lengths
        attend("attend mx6 64x2k-8k", "mx6", "mx6", 64, 2048, 8192, 32, 8, 128, "bf16"),
        # one long document, the cache in four bits
        attend("attend mx4 1x131072", "mx4", "mx4", 1, 131072, 131072, 64, 8, 128, "bf16", page=64),
        # a chat batch with the widest format
        attend("attend mx9 16x500-4k", "mx9", "mx9", 16, 500, 4096, 32, 8, 128, "bf16", page=32),
        # odd head size and page, an empty sequence, a sliding window, mixed formats, 32-bit queries
        attend("attend mx9/mx4 7 f32 window", "mx9", "mx4", 7, 0, 3001, 20, 4, 80, "f32", page=24, window=1024),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("gemv", "append", "attend"))
    fmt = [rng.choice(("mx4", "mx6", "mx9")) for _ in range(2)]
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "gemv":
        n = _log(rng, 300, 32768)
        k = _log(rng, 300, min(16384, (1 << 27) // n))
        if rng.random() < 0.6:
            n, k = -(-n // 640) * 640, -(-k // 1280) * 1280
        while n * k > 1 << 27:
            n -= 640
        n = max(n, 300)
        c = gemv("", fmt[0], _log(rng, 1, 16), n, k, dtype, rng.choice(("bf16", "f32")))
    else:
        head_dim = rng.choice((64, 80, 112, 128, 128, 128, 256))
        n_kv = rng.choice((1, 2, 4, 5, 8, 8, 16))
        n_q = n_kv * rng.choice([g for g in (1, 2, 4, 5, 7, 8, 16) if g * n_kv <= 64])
        page = rng.choice((16, 16, 24, 32, 64, 128))
        if op == "append":
            most = min(16384, (1 << 26) // ((n_q + 2 * n_kv) * head_dim))
            c = append("", fmt[0], fmt[1], _log(rng, 1, most), n_q, n_kv, head_dim, dtype,
                       rng.choice((head_dim, head_dim, head_dim // 2, 32)), rng.random() < 0.3, page=page)
        else:
            batch = _log(rng, 1, 64)
            longest = _log(rng, 16, min(131072, (1 << 28) // (batch * n_kv * head_dim)))
            c = attend("", fmt[0], fmt[1], batch, rng.randint(0, longest), longest, n_q, n_kv, head_dim, dtype, page,
                       rng.choice((0, 0, 0, max(1, longest // 3))))
    del c["name"]
    return c


def lengths(case):
    """Sequence lengths of an attention case, from its shortest to its longest in a mixed order."""
    b, lo, hi = case["batch"], case["shortest"], case["longest"]
    lens = [hi - (hi - lo) * i // max(1, b - 1) for i in range(b)]
    random.Random(b * 1000003 + hi).shuffle(lens)
    return lens


# ---- the format in elementary operations ------------------------------------------------------------------------------------

def _quantize(x, m):
    """Block exponents [rows, nb], shifts [rows, nb, 8], signed magnitudes and the values of fp32 x [rows, 16 nb]."""
    rows = x.shape[0]
    b = x.view(torch.int32).reshape(rows, -1, 8, 2)
    e = (b >> 23) & 255
    sub = e.amax(-1)
    F = sub.amax(-1)
    tau = (F[..., None] - sub).clamp(max=1)
    p = (F[..., None] - tau - (m - 1)).clamp(min=1)                        # exponent field of one unit
    unit = (p << 23).view(torch.float32)[..., None]
    inverse = ((254 - p) << 23).view(torch.float32)[..., None]
    x4 = x.reshape(rows, -1, 8, 2)
    q = (x4.abs() * inverse).round().clamp(max=2 ** m - 1)
    return F, tau, torch.signbit(x4), q, (torch.copysign(q * unit, x4)).reshape(rows, -1)


def _packed(x, m):
    """The three planes of fp32 x [rows, cols] and its quantized values; cols is padded to whole blocks."""
    rows, cols = x.shape
    full = torch.nn.functional.pad(x, (0, -cols % 16)).contiguous()
    F, tau, sign, q, values = _quantize(full, m)
    nb, bits = F.shape[1], m + 1
    two = torch.arange(8, device=x.device)
    micro = (tau << two).sum(-1)
    code = ((sign.to(torch.int64) << m) | q.to(torch.int64)).reshape(rows, 2 * nb, 8)
    word = (code << (bits * two)).sum(-1)                                  # eight codes in m + 1 bytes
    elems = ((word[..., None] >> (8 * torch.arange(bits, device=x.device))) & 255).reshape(rows, -1)
    pad = lambda t: torch.nn.functional.pad(t.to(torch.uint8), (0, -t.shape[1] % 16))  # noqa: E731
    return [pad(F), pad(micro), pad(elems)], values[:, :cols]


def _values(planes, m, cols):
    """fp32 values [..., cols] of packed lines."""
    exps, micro, elems = planes
    nb, bits = -(-cols // 16), m + 1
    eight = torch.arange(8, device=exps.device, dtype=torch.int32)
    e = elems[..., :2 * nb * bits].reshape(*elems.shape[:-1], 2 * nb, bits).to(torch.int64)
    word = (e << (8 * torch.arange(bits, device=e.device))).sum(-1)
    code = ((word[..., None] >> (bits * eight)) & (2 * 2 ** m - 1)).to(torch.int32)
    code = code.reshape(*elems.shape[:-1], nb, 8, 2)
    tau = (micro[..., :nb, None].to(torch.int32) >> eight) & 1
    p = (exps[..., :nb, None].to(torch.int32) - tau - (m - 1)).clamp(min=0)
    unit = (p << 23).view(torch.float32)[..., None]
    value = (code & (2 ** m - 1)).to(torch.float32) * unit
    return torch.where(code >> m > 0, -value, value).reshape(*elems.shape[:-1], 16 * nb)[..., :cols]


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def _handle(fmt_or_fmts, planes, **cache):
    """The library's view of packed tensors that a program keeps."""
    from paper_2302_08007_b200 import binding as bdr
    cfg = {"mx4": bdr.MX4, "mx6": bdr.MX6, "mx9": bdr.MX9}
    if not cache:
        return cfg[fmt_or_fmts], bdr.Planes(*planes)
    return bdr.KVCache(cfg[fmt_or_fmts[0]], cfg[fmt_or_fmts[1]], bdr.Planes(*planes[0]), bdr.Planes(*planes[1]), **cache)


def _rotation(n_pos, rot_dim, device):
    """cos and sin of position * 10000^(-2 i / rot_dim)."""
    angle = torch.arange(n_pos, device=device, dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(0, rot_dim, 2, device=device, dtype=torch.float64) / rot_dim)
    return torch.cos(angle).float(), torch.sin(angle).float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    s = {"case": case}
    if case["op"] == "gemv":
        n, k, t = case["n"], case["k"], case["tokens"]
        m = MANTISSA[case["fmt"]]
        s["w"] = _packed(randn(n, k) * k ** -0.5, m)[0]
        gain = torch.where(torch.rand(k, device="cuda", generator=gen) < 0.01, 20.0, 1.0)      # outlier channels
        s["x"] = (randn(t, k) * gain).to(DTYPE[case["dtype"]])
        if own:
            s["cfg"], s["planes"] = _handle(case["fmt"], s["w"])
        return s
    n_kv, d, page = case["n_kv"], case["head_dim"], case["page"]
    m = MANTISSA[case["fmt_k"]], MANTISSA[case["fmt_v"]]
    if case["op"] == "append":
        t = case["tokens"]
        n_pages = -(-t // page) + 8
        n_slots = n_pages * page
        qkv = randn(t, case["n_q"] + 2 * n_kv, d)                          # what a fused projection leaves: one row per token
        qkv[:, :, ::17] *= 6.0
        qkv = qkv.to(DTYPE[case["dtype"]])
        s["q"], s["k"], s["v"] = qkv.split((case["n_q"], n_kv, n_kv), 1)
        start = torch.randint(0, 4096, (1,), device="cuda", generator=gen)
        s["positions"] = start + torch.arange(t, device="cuda")
        s["cos"], s["sin"] = _rotation(4096 + t, case["rot_dim"], "cuda")
        pages = torch.randperm(n_pages, device="cuda", generator=gen)
        at = torch.arange(t, device="cuda")
        slots = pages[at // page] * page + at % page
        if case["padding"]:
            slots[torch.randperm(t, device="cuda", generator=gen)[:case["padding"]]] = -1
        s["slots"] = slots
        empty = lambda w: torch.zeros((n_slots, -(-w // 16) * 16), dtype=torch.uint8, device="cuda")  # noqa: E731
        c = n_kv * d
        s["kp"], s["vp"] = ([empty(c // 16), empty(c // 16), empty(c * (mm + 1) // 8)] for mm in m)
        s["q_out"] = torch.empty((t, case["n_q"], d), dtype=qkv.dtype, device="cuda")
        s["k_dq"], s["v_dq"] = (torch.empty((t, n_kv, d), dtype=qkv.dtype, device="cuda") for _ in range(2))
    else:
        b, lens = case["batch"], lengths(case)
        need = [-(-x // page) for x in lens]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
        table = torch.full((b, max(1, max(need))), -1, dtype=torch.int32, device="cuda")
        first = 0
        for i, x in enumerate(need):
            table[i, :x] = order[first:first + x]
            first += x
        s["table"], s["lengths"] = table, torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["q"] = randn(b, case["n_q"], d).to(DTYPE[case["dtype"]])
        keys = randn(n_pages * page, n_kv * d)
        keys[:, ::29] *= 4.0
        s["kp"] = _packed(keys, m[0])[0]
        del keys
        s["vp"] = _packed(randn(n_pages * page, n_kv * d), m[1])[0]
    if own:
        s["cache"] = _handle((case["fmt_k"], case["fmt_v"]), (s["kp"], s["vp"]), n_pages=n_pages, page_size=page, n_kv=n_kv, head_dim=d)
        if case["op"] == "attend":
            from paper_2302_08007_b200 import binding as bdr
            size = bdr.mx_attn_decode_workspace_bytes(s["cache"], case["batch"], case["n_q"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return {"gemv": _gemv_own, "append": _append_own, "attend": _attend_own}[case["op"]](case, state)
    return {"gemv": _gemv_plain, "append": _append_plain, "attend": _attend_plain}[case["op"]](case, state)


def _gemv_own(case, s):
    from paper_2302_08007_b200 import binding as bdr
    y = torch.empty((case["tokens"], case["n"]), dtype=DTYPE[case["out"]], device="cuda")
    return bdr.mx_gemv(s["cfg"], s["planes"], case["n"], case["k"], s["x"], y)


def _append_own(case, s):
    from paper_2302_08007_b200 import binding as bdr
    bdr.mx_kv_append(s["cache"], s["k"], s["v"], s["slots"], s["positions"], s["cos"], s["sin"], interleaved=case["interleaved"],
                     q=s["q"], q_out=s["q_out"], k_dq=s["k_dq"], v_dq=s["v_dq"])
    return {"q": s["q_out"], "k": s["k_dq"], "v": s["v_dq"], "k planes": s["kp"], "v planes": s["vp"]}


def _attend_own(case, s):
    from paper_2302_08007_b200 import binding as bdr
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    bdr.mx_attn_decode(s["cache"], s["q"], s["table"], s["lengths"], out, s["workspace"], scale=case["head_dim"] ** -0.5,
                       window=case["window"], lse=lse)
    return {"out": out, "lse": lse}


def _gemv_plain(case, s):
    w = _values(s["w"], MANTISSA[case["fmt"]], case["k"])
    return (s["x"].float() @ w.T).to(DTYPE[case["out"]])


def _rotate(x, c, s, rot, interleaved):
    """x [T, heads, d] in 32 bits; c, s [T, 1, rot / 2]; every product and sum rounded once."""
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * c - b * s, b * c + a * s
    y = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((y, x[..., rot:]), -1)


def _append_plain(case, s):
    dtype, t = DTYPE[case["dtype"]], case["tokens"]
    c, sn = s["cos"][s["positions"]][:, None], s["sin"][s["positions"]][:, None]
    turn = lambda x: _rotate(x.float(), c, sn, case["rot_dim"], case["interleaved"])  # noqa: E731
    s["q_out"].copy_(turn(s["q"]))
    kept = s["slots"] >= 0
    at = s["slots"][kept]
    kp, kd = _packed(turn(s["k"]).reshape(t, -1), MANTISSA[case["fmt_k"]])
    vp, vd = _packed(s["v"].float().reshape(t, -1), MANTISSA[case["fmt_v"]])
    s["kp"][0][at], s["kp"][1][at], s["kp"][2][at] = kp[0][kept], kp[1][kept], kp[2][kept]
    s["vp"][0][at], s["vp"][1][at], s["vp"][2][at] = vp[0][kept], vp[1][kept], vp[2][kept]
    return {"q": s["q_out"], "k": kd.reshape(t, -1, case["head_dim"]).to(dtype), "v": vd.reshape(t, -1, case["head_dim"]).to(dtype),
            "k planes": s["kp"], "v planes": s["vp"]}


def _attend_plain(case, s):
    b, n_q, d = s["q"].shape
    n_kv, page = case["n_kv"], case["page"]
    t = torch.arange(max(1, case["longest"]), device="cuda")
    slots = s["table"].clamp(min=0).long()[:, t // page] * page + t % page                      # [batch, tokens]
    keys = _values([p[slots] for p in s["kp"]], MANTISSA[case["fmt_k"]], n_kv * d).reshape(b, -1, n_kv, d)
    q = s["q"].float().reshape(b, n_kv, -1, d)
    score = torch.einsum("bhgd,blhd->bhgl", q, keys) * case["head_dim"] ** -0.5
    del keys
    n = s["lengths"][:, None]
    seen = (t < n) & (t >= n - case["window"]) if case["window"] else t < n
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    weight = torch.exp(score - top)
    total = weight.sum(-1, keepdim=True)
    values = _values([p[slots] for p in s["vp"]], MANTISSA[case["fmt_v"]], n_kv * d).reshape(b, -1, n_kv, d)
    out = torch.einsum("bhgl,blhd->bhgd", weight, values) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).reshape(b, n_q)
    return {"out": out.reshape(b, n_q, d).to(s["q"].dtype), "lse": lse}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------

def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] == "gemv":
        t, n, k = case["tokens"], case["n"], case["k"]
        return {"bytes": n * k * BITS[case["fmt"]] / 8 + t * k * size[case["dtype"]] + t * n * size[case["out"]], "flops": 2 * t * n * k}
    c, b = case["n_kv"] * case["head_dim"], size[case["dtype"]]
    both = (BITS[case["fmt_k"]] + BITS[case["fmt_v"]]) / 8
    if case["op"] == "append":
        # q, k and v in; rotated q, both quantized tensors and the cache lines out
        t, q = case["tokens"], case["n_q"] * case["head_dim"]
        return {"bytes": t * (2 * (q + 2 * c) * b + 8 * 2 + 4 * case["rot_dim"]) + (t - case["padding"]) * c * both,
                "flops": t * (3 * (case["n_q"] + case["n_kv"]) * case["rot_dim"] + 8 * c)}
    seen = sum(min(x, case["window"]) if case["window"] else x for x in lengths(case))
    q = case["n_q"] * case["head_dim"]
    return {"bytes": seen * c * both + case["batch"] * (2 * q * b + 4 * case["n_q"]), "flops": 4 * seen * q}


# ---- the same in 64 bits ----------------------------------------------------------------------------------------------------

def _bits(line, count, width):
    """`count` little-endian fields of `width` bits from uint8 lines."""
    bit = (line[..., None] >> torch.arange(8, device=line.device, dtype=torch.uint8)) & 1
    bit = bit.flatten(-2)[..., :count * width].reshape(*line.shape[:-1], count, width)
    field = bit[..., 0].to(torch.int16)
    for i in range(1, width):
        field += bit[..., i].to(torch.int16) << i
    return field


def _decode64(planes, m, cols):
    nb = -(-cols // 16)
    code = _bits(planes[2], 16 * nb, m + 1)
    tau = _bits(planes[1], 8 * nb, 1).repeat_interleave(2, -1)
    power = planes[0][..., :nb].to(torch.int32).repeat_interleave(16, -1) - 127 - tau - (m - 1)
    value = torch.ldexp((code & (2 ** m - 1)).double(), power)
    return torch.where(code >= 2 ** m, -value, value)[..., :cols]


def _turn64(x, cos, sin, rot, interleaved):
    y = x.clone()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = cos[:, i, None], sin[:, i, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def _nearest64(x, m):
    """Every value of x [..., multiple of 16] in the format, by the format's definition."""
    blocks = x.reshape(*x.shape[:-1], -1, 8, 2)
    high = torch.frexp(blocks.abs())[1] - 1
    high = torch.where(blocks == 0, -127, high.clamp(min=-127))
    pair = high.amax(-1, keepdim=True)
    block = pair.amax(-2, keepdim=True)
    step = torch.ldexp(torch.ones_like(blocks[..., :1]), block - (block - pair).clamp(max=1) - (m - 1))
    q = (blocks.abs() / step).round().clamp(max=2 ** m - 1)
    return (torch.sign(blocks) * q * step).reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "gemv":
        x, m = s["x"].double(), MANTISSA[case["fmt"]]
        return torch.cat([x @ _decode64([p[i:i + 2048] for p in s["w"]], m, case["k"]).T for i in range(0, case["n"], 2048)], 1)
    n_kv, d = case["n_kv"], case["head_dim"]
    m = MANTISSA[case["fmt_k"]], MANTISSA[case["fmt_v"]]
    if case["op"] == "append":
        cos, sin = s["cos"][s["positions"]].double(), s["sin"][s["positions"]].double()
        q, k = (_turn64(s[x].double(), cos, sin, case["rot_dim"], case["interleaved"]) for x in "qk")
        flat = lambda x, mm: _nearest64(x.reshape(x.shape[0], -1), mm).reshape(x.shape)  # noqa: E731
        return {"q": q, "k": flat(k, m[0]), "v": flat(s["v"].double(), m[1]), "k planes": None, "v planes": None}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for i, n in enumerate(lengths(case)):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == 0:
            continue
        t = torch.arange(first, n, device="cuda")
        at = s["table"][i].long()[torch.div(t, case["page"], rounding_mode="floor")] * case["page"] + t % case["page"]
        q = s["q"][i].double().reshape(n_kv, -1, d)
        score = []
        for j in range(0, len(at), 8192):
            key = _decode64([p[at[j:j + 8192]] for p in s["kp"]], m[0], n_kv * d).reshape(-1, n_kv, d)
            score.append(torch.matmul(q, key.permute(1, 2, 0)) / math.sqrt(d))
        score = torch.cat(score, -1)
        lse[i] = torch.logsumexp(score, -1).reshape(-1)
        weight = torch.softmax(score, -1)
        for j in range(0, len(at), 8192):
            value = _decode64([p[at[j:j + 8192]] for p in s["vp"]], m[1], n_kv * d).reshape(-1, n_kv, d)
            out[i] += torch.matmul(weight[..., j:j + 8192], value.permute(1, 0, 2)).reshape(-1, d)
    return {"out": out, "lse": lse}
