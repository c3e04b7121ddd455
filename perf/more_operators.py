"""Workloads of the operators around the linear layers of a language model, on MX-packed operands: the gated feed-forward layer
(both projections, the activation and the product; its gradients; its form for a few tokens) and the softmax cross entropy over a
vocabulary whose logits are never kept (with its gradients).

`listed()` names the fixed cases, `draw()` makes more of the same ranges, `prepare()` the inputs of one, `run()` makes one
pass: with `own` the library's calls, without it the same operators in elementary torch operations on 32-bit values.
`work()` counts the bytes and operations a pass cannot do without, `exact()` gives the results in 64 bits.

All packed tensors are line-major planes (shared exponents, microexponents, codes) with 16-byte pitches, as the library's
pack call writes them: a line is a row of K elements.  The weights of a gated layer are one tensor of 2 N lines, first the N of
the gate, then the N of the other projection.
"""
import math

import torch

own = False

MANTISSA = {"mx4": 2, "mx6": 4, "mx9": 7}          # magnitude bits; a code has one more (the sign)
BITS = {"mx4": 4.0, "mx6": 6.0, "mx9": 9.0}        # bits per element with both scale levels
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("silu", "gelu", "gelu_tanh", "relu")


# ---- cases ------------------------------------------------------------------------------------------------------------------

def gated(name, fmt_a, fmt_w, m, n, k, dtype, act="silu", save=True):
    """Forward: h = act(a Wg^T) * (a Wu^T), with both products kept for the backward pass where `save`."""
    return {"name": name, "op": "gated", "fmt_a": fmt_a, "fmt_w": fmt_w, "m": m, "n": n, "k": k, "dtype": dtype, "act": act, "save": save}


def gated_grad(name, fmt_a, fmt_w, m, n, k, dtype, act="silu", save=True):
    """Gradients of a and of both weights from that of h; the products come from the forward pass, or again from the operands."""
    return {"name": name, "op": "gated_grad", "fmt_a": fmt_a, "fmt_w": fmt_w, "m": m, "n": n, "k": k, "dtype": dtype, "act": act, "save": save}


def gated_few(name, fmt_w, tokens, n, k, dtype, act="silu"):
    """A few tokens through both projections, activations unpacked."""
    return {"name": name, "op": "gated_few", "fmt_w": fmt_w, "m": tokens, "n": n, "k": k, "dtype": dtype, "act": act}


def entropy(name, fmt_a, fmt_w, m, v, k):
    """Loss and log of the sum of exponentials of every row."""
    return {"name": name, "op": "entropy", "fmt_a": fmt_a, "fmt_w": fmt_w, "m": m, "n": v, "k": k}


def entropy_step(name, fmt_a, fmt_w, m, v, k, dtype):
    """The loss and its gradients with regard to hidden states and vocabulary weights."""
    return {"name": name, "op": "entropy_step", "fmt_a": fmt_a, "fmt_w": fmt_w, "m": m, "n": v, "k": k, "dtype": dtype}


def listed():
    return [
        # the widening half of a training step's feed-forward layer: tokens and widths of the library's linear-layer benchmark
        gated("gated mx6 8192x8192x4096", "mx6", "mx6", 8192, 8192, 4096, "bf16"),
        # nothing a multiple of anything, mixed formats, 32-bit results, inference (nothing kept)
        gated("gated mx9/mx4 1003x2747x1500 f32", "mx9", "mx4", 1003, 2747, 1500, "f32", "gelu", False),
        # the same layer's gradients
        gated_grad("gated grad mx6 8192x8192x4096", "mx6", "mx6", 8192, 8192, 4096, "bf16"),
        # odd sizes, the products computed again because nothing was kept
        gated_grad("gated grad mx4/mx9 517x1401x1111 f32", "mx4", "mx9", 517, 1401, 1111, "f32", "gelu_tanh", False),
        # the widening half for one decoded token, where the launch counts
        gated_few("gated few mx4 1x8192x4096", "mx4", 1, 8192, 4096, "bf16"),
        # a wide layer and a batch of sixteen streams
        gated_few("gated few mx9 16x16384x4096", "mx9", 16, 16384, 4096, "bf16"),
        # ragged everything, 32-bit activations
        gated_few("gated few mx6 3x2503x2063 f32", "mx6", 3, 2503, 2063, "f32", "relu"),
        # scoring a batch of tokens
        entropy("entropy mx9 4096x32000x4096", "mx9", "mx9", 4096, 32000, 4096),
        # scoring one token: the weights count
        entropy("entropy mx6 1x32000x4096", "mx6", "mx6", 1, 32000, 4096),
        # a small ragged vocabulary
        entropy("entropy mx4 777x10007x1003", "mx4", "mx4", 777, 10007, 1003),
        # the head of a training step
        entropy_step("entropy step mx6 4096x32000x4096", "mx6", "mx6", 4096, 32000, 4096, "bf16"),
        # a small ragged step with 32-bit gradients
        entropy_step("entropy step mx9/mx6 301x5003x1037 f32", "mx9", "mx6", 301, 5003, 1037, "f32"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("gated", "gated_grad", "gated_few", "entropy", "entropy_step"))
    fmt = [rng.choice(("mx4", "mx6", "mx9")) for _ in range(2)]
    if rng.random() < 0.6:
        fmt[1] = fmt[0]
    dtype = rng.choice(("bf16", "bf16", "f32"))
    act = rng.choice(("silu", "silu", "gelu", "gelu_tanh", "relu"))
    whole = rng.random() < 0.5
    even = lambda x, to: -(-x // to) * to if whole else x  # noqa: E731
    if op == "gated_few":
        n = even(_log(rng, 150, 16384), 128)
        k = even(_log(rng, 300, min(16384, (1 << 26) // n)), 256)
        while n * k > 1 << 26:
            n -= 128
        c = gated_few("", fmt[0], _log(rng, 1, 16), n, k, dtype, act)
    elif op in ("gated", "gated_grad"):
        k = even(_log(rng, 64, 8192), 256)
        n = even(_log(rng, 100, min(16384, (1 << 26) // k)), 256)
        m = even(_log(rng, 1, min(8192, (1 << 37) // (n * k))), 256)
        c = (gated if op == "gated" else gated_grad)("", *fmt, m, n, k, dtype, act, rng.random() < 0.6)
    else:
        k = even(_log(rng, 64, 8192), 256)
        v = even(_log(rng, 300, min(131072, (1 << 27) // k)), 256)
        m = even(_log(rng, 1, min(8192, (1 << 38) // (v * k), (1 << 28) // v)), 256)
        c = entropy("", *fmt, m, v, k) if op == "entropy" else entropy_step("", *fmt, m, v, k, dtype)
    del c["name"]
    return c


# ---- the format in elementary operations ------------------------------------------------------------------------------------

def _pack_rows(x, m):
    rows, cols = x.shape
    full = torch.nn.functional.pad(x, (0, -cols % 16)).contiguous()
    e = (full.view(torch.int32).reshape(rows, -1, 8, 2) >> 23) & 255
    sub = e.amax(-1)
    F = sub.amax(-1)
    tau = (F[..., None] - sub).clamp(max=1)
    p = (F[..., None] - tau - (m - 1)).clamp(min=1)                        # exponent field of one unit
    x4 = full.reshape(rows, -1, 8, 2)
    q = (x4.abs() * ((254 - p) << 23).view(torch.float32)[..., None]).round().clamp(max=2 ** m - 1)
    nb, bits = F.shape[1], m + 1
    eight = torch.arange(8, device=x.device)
    micro = (tau << eight).sum(-1)
    code = ((torch.signbit(x4).to(torch.int64) << m) | q.to(torch.int64)).reshape(rows, 2 * nb, 8)
    word = (code << (bits * eight)).sum(-1)                                # eight codes in m + 1 bytes
    elems = ((word[..., None] >> (8 * torch.arange(bits, device=x.device))) & 255).reshape(rows, -1)
    pad = lambda t: torch.nn.functional.pad(t.to(torch.uint8), (0, -t.shape[1] % 16))  # noqa: E731
    return [pad(F), pad(micro), pad(elems)]


def _packed(x, m):
    """The three planes of fp32 x [rows, cols], some rows at a time."""
    step = max(1, (1 << 25) // x.shape[1])
    parts = [_pack_rows(x[i:i + step], m) for i in range(0, x.shape[0], step)]
    return [torch.cat(p) for p in zip(*parts)]


def _values(planes, m, cols):
    """fp32 values [rows, cols] of packed lines."""
    exps, micro, elems = planes
    nb, bits = -(-cols // 16), m + 1
    eight = torch.arange(8, device=exps.device, dtype=torch.int32)
    e = elems[:, :2 * nb * bits].reshape(elems.shape[0], 2 * nb, bits).to(torch.int64)
    word = (e << (8 * torch.arange(bits, device=e.device))).sum(-1)
    code = ((word[..., None] >> (bits * eight)) & (2 * 2 ** m - 1)).to(torch.int32).reshape(elems.shape[0], nb, 8, 2)
    tau = (micro[:, :nb, None].to(torch.int32) >> eight) & 1
    p = (exps[:, :nb, None].to(torch.int32) - tau - (m - 1)).clamp(min=0)
    value = (code & (2 ** m - 1)).to(torch.float32) * (p << 23).view(torch.float32)[..., None]
    return torch.where(code >> m > 0, -value, value).reshape(elems.shape[0], 16 * nb)[:, :cols]


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    op, m, n, k = case["op"], case["m"], case["n"], case["k"]
    s = {"case": case}
    gain = torch.where(torch.rand(k, device="cuda", generator=gen) < 0.01, 8.0, 1.0)           # outlier channels
    lines = n if op.startswith("entropy") else 2 * n
    w = randn(lines, k) * k ** -0.5
    if op == "gated_few":
        s["x"] = (randn(m, k) * gain).to(DTYPE[case["dtype"]])
    elif op.startswith("gated"):
        a = randn(m, k) * gain
        if op == "gated_grad":
            s["dh"] = (randn(m, n) * 1e-3).to(DTYPE[case["dtype"]])
    else:
        # hidden states that know the next token more often than not; one token in twenty is padding or part of a prompt
        a = 1.5 * randn(m, k)
        s["targets"] = torch.randint(0, n, (m,), device="cuda", generator=gen)
        sure = torch.rand(m, 1, device="cuda", generator=gen) < 0.6
        a += torch.where(sure, 8.0, 0.0) * w[s["targets"]]
        s["targets"][torch.rand(m, device="cuda", generator=gen) < 0.05] = -100
        if op == "entropy_step":
            counted = s["targets"] >= 0
            s["dloss"] = counted.float() / counted.sum().clamp(min=1)                          # of the mean over those that count
    s["w"] = _packed(w, MANTISSA[case["fmt_w"]])
    del w
    if op != "gated_few":
        s["a"] = _packed(a, MANTISSA[case["fmt_a"]])
        del a
    if op == "gated_grad" and case["save"]:
        # what the forward pass left
        s["gate_up"] = (_values(s["a"], MANTISSA[case["fmt_a"]], k) @ _values(s["w"], MANTISSA[case["fmt_w"]], k).T).to(DTYPE[case["dtype"]])
    if own:
        from paper_2302_08007_b200 import binding as bdr
        cfg = {"mx4": bdr.MX4, "mx6": bdr.MX6, "mx9": bdr.MX9}
        s["cfg_w"], s["pw"] = cfg[case["fmt_w"]], bdr.Planes(*s["w"])
        if op != "gated_few":
            s["cfg_a"], s["pa"] = cfg[case["fmt_a"]], bdr.Planes(*s["a"])
        size = 0
        if op == "gated":
            size = bdr.mx_gated_gemm_workspace_bytes(m, n, k)
        elif op == "gated_grad":
            size = bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k, DTYPE[case["dtype"]])
        elif op == "entropy":
            size = bdr.mx_cross_entropy_workspace_bytes(m, n, k)
        elif op == "entropy_step":
            size = max(bdr.mx_cross_entropy_workspace_bytes(m, n, k), bdr.mx_cross_entropy_bwd_workspace_bytes(m, n, k, DTYPE[case["dtype"]]))
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        s["act"] = {"silu": bdr.ACT_SILU, "gelu": bdr.ACT_GELU, "gelu_tanh": bdr.ACT_GELU_TANH, "relu": bdr.ACT_RELU}[case.get("act", "silu")]
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return {"gated": _gated_own, "gated_grad": _gated_grad_own, "gated_few": _gated_few_own, "entropy": _entropy_own,
                "entropy_step": _entropy_step_own}[case["op"]](case, state)
    return {"gated": _gated_plain, "gated_grad": _gated_grad_plain, "gated_few": _gated_few_plain, "entropy": _entropy_plain,
            "entropy_step": _entropy_step_plain}[case["op"]](case, state)


def _new(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _operands(s):
    return s["cfg_a"], s["pa"], s["cfg_w"], s["pw"], s["case"]["m"], s["case"]["n"], s["case"]["k"]


def _gated_own(case, s):
    from paper_2302_08007_b200 import binding as bdr
    dtype = DTYPE[case["dtype"]]
    h = _new(case["m"], case["n"], dtype=dtype)
    gate_up = _new(case["m"], 2 * case["n"], dtype=dtype) if case["save"] else None
    bdr.mx_gated_gemm(*_operands(s), h, s["workspace"], act=s["act"], gate_up=gate_up)
    return {"h": h, "gate_up": gate_up} if case["save"] else {"h": h}


def _gated_grad_own(case, s):
    from paper_2302_08007_b200 import binding as bdr
    dtype = DTYPE[case["dtype"]]
    da, dw = _new(case["m"], case["k"], dtype=dtype), _new(2 * case["n"], case["k"], dtype=dtype)
    bdr.mx_gated_gemm_bwd(*_operands(s), s["dh"], da, dw, s["workspace"], act=s["act"], gate_up=s.get("gate_up"))
    return {"da": da, "dw": dw}


def _gated_few_own(case, s):
    from paper_2302_08007_b200 import binding as bdr
    h = _new(case["m"], case["n"], dtype=DTYPE[case["dtype"]])
    return bdr.mx_gated_gemv(s["cfg_w"], s["pw"], case["n"], case["k"], s["x"], h, act=s["act"])


def _entropy_own(case, s):
    from paper_2302_08007_b200 import binding as bdr
    loss, lse = _new(case["m"]), _new(case["m"])
    bdr.mx_cross_entropy(*_operands(s), s["targets"], loss, lse, s["workspace"])
    return {"loss": loss, "lse": lse}


def _entropy_step_own(case, s):
    from paper_2302_08007_b200 import binding as bdr
    dtype = DTYPE[case["dtype"]]
    loss, lse = _new(case["m"]), _new(case["m"])
    da, dw = _new(case["m"], case["k"], dtype=dtype), _new(case["n"], case["k"], dtype=dtype)
    bdr.mx_cross_entropy(*_operands(s), s["targets"], loss, lse, s["workspace"])
    bdr.mx_cross_entropy_bwd(*_operands(s), s["targets"], lse, s["dloss"], da, dw, s["workspace"])
    return {"loss": loss, "lse": lse, "da": da, "dw": dw}


def _act(g, name):
    if name == "silu":
        return g / (1 + torch.exp(-g))
    if name == "gelu":
        return 0.5 * g * (1 + torch.erf(g * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g)))
    return g.clamp(min=0)


def _act_grad(g, name):
    if name == "silu":
        p = 1 / (1 + torch.exp(-g))
        return p * (1 + g * (1 - p))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(g * math.sqrt(0.5))) + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g))
        return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)
    return (g > 0).to(g.dtype)


def _both(case, s):
    return _values(s["a"], MANTISSA[case["fmt_a"]], case["k"]), _values(s["w"], MANTISSA[case["fmt_w"]], case["k"])


def _gated_plain(case, s):
    a, w = _both(case, s)
    gate_up = a @ w.T
    g, u = gate_up.split(case["n"], 1)
    h = (_act(g, case["act"]) * u).to(DTYPE[case["dtype"]])
    return {"h": h, "gate_up": gate_up.to(DTYPE[case["dtype"]])} if case["save"] else {"h": h}


def _gated_grad_plain(case, s):
    a, w = _both(case, s)
    gate_up = s["gate_up"].float() if case["save"] else a @ w.T
    g, u = gate_up.split(case["n"], 1)
    dh = s["dh"].float()
    d = torch.cat((dh * u * _act_grad(g, case["act"]), dh * _act(g, case["act"])), 1)
    return {"da": (d @ w).to(s["dh"].dtype), "dw": (d.T @ a).to(s["dh"].dtype)}


def _gated_few_plain(case, s):
    g, u = (s["x"].float() @ _values(s["w"], MANTISSA[case["fmt_w"]], case["k"]).T).split(case["n"], 1)
    return (_act(g, case["act"]) * u).to(s["x"].dtype)


def _loss_plain(logits, targets):
    top = logits.amax(1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(logits - top).sum(1))
    there = targets >= 0
    hit = logits.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    return torch.where(there, lse - hit, 0.0), lse


def _entropy_plain(case, s):
    a, w = _both(case, s)
    loss, lse = _loss_plain(a @ w.T, s["targets"])
    return {"loss": loss, "lse": lse}


def _entropy_step_plain(case, s):
    a, w = _both(case, s)
    logits = a @ w.T
    loss, lse = _loss_plain(logits, s["targets"])
    there = s["targets"] >= 0
    d = logits.sub_(lse[:, None]).exp_()
    d[torch.arange(case["m"], device="cuda"), s["targets"].clamp(min=0)] -= there.float()
    d *= torch.where(there, s["dloss"], 0.0)[:, None]
    dtype = DTYPE[case["dtype"]]
    return {"loss": loss, "lse": lse, "da": (d @ w).to(dtype), "dw": (d.T @ a).to(dtype)}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------

def work(case):
    size = {"bf16": 2, "f32": 4}
    op, m, n, k = case["op"], case["m"], case["n"], case["k"]
    b = size[case.get("dtype", "f32")]
    if op == "gated_few":
        return {"bytes": 2 * n * k * BITS[case["fmt_w"]] / 8 + m * (n + k) * b, "flops": 4 * m * n * k}
    packed = (m * k * BITS[case["fmt_a"]] + (n if op.startswith("entropy") else 2 * n) * k * BITS[case["fmt_w"]]) / 8
    if op == "gated":
        return {"bytes": packed + m * n * b * (3 if case["save"] else 1), "flops": 4 * m * n * k}
    if op == "gated_grad":
        return {"bytes": packed + m * n * b * (3 if case["save"] else 1) + (m + 2 * n) * k * b, "flops": (8 if case["save"] else 12) * m * n * k}
    if op == "entropy":
        return {"bytes": packed + 16 * m, "flops": 2 * m * n * k}
    # the logits once, and a product for each gradient
    return {"bytes": packed + 20 * m + (m + n) * k * b, "flops": 6 * m * n * k}


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
    """Values in 64 bits by the format's definition: sign, magnitude, times 2^(exponent - shift - (m - 1))."""
    nb = -(-cols // 16)
    out = torch.empty((planes[0].shape[0], cols), dtype=torch.float64, device=planes[0].device)
    for i in range(0, out.shape[0], 2048):
        exps, micro, elems = (p[i:i + 2048] for p in planes)
        code = _bits(elems, 16 * nb, m + 1)
        tau = _bits(micro, 8 * nb, 1).repeat_interleave(2, -1)
        power = exps[:, :nb].to(torch.int32).repeat_interleave(16, -1) - 127 - tau - (m - 1)
        value = torch.ldexp((code & (2 ** m - 1)).double(), power)
        out[i:i + 2048] = torch.where(code >= 2 ** m, -value, value)[:, :cols]
    return out


def _gate64(g, name):
    """Activation and its derivative."""
    if name == "silu":
        p = torch.special.expit(g)
        return g * p, p + g * p * torch.special.expit(-g)
    if name == "gelu":
        below = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * below, below + g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        p = torch.special.expit(2 * c * (g + 0.044715 * g ** 3))            # (1 + tanh x) / 2
        return g * p, p + g * p * (1 - p) * 2 * c * (1 + 0.134145 * g ** 2)
    return torch.relu(g), torch.heaviside(g, torch.zeros_like(g))


def exact(case, seed):
    s = prepare(case, seed)
    op, n, k = case["op"], case["n"], case["k"]
    w = _decode64(s["w"], MANTISSA[case["fmt_w"]], k)
    a = s["x"].double() if op == "gated_few" else _decode64(s["a"], MANTISSA[case["fmt_a"]], k)
    if op == "gated_grad" and case["save"]:
        g, u = s["gate_up"][:, :n].double(), s["gate_up"][:, n:].double()
    elif op.startswith("gated"):
        g, u = torch.mm(a, w[:n].t()), torch.mm(a, w[n:].t())
    if op.startswith("gated"):
        y, slope = _gate64(g, case["act"])
        if op == "gated_few":
            return y * u
        if op == "gated":
            return {"h": y * u, "gate_up": torch.cat((g, u), 1)} if case["save"] else {"h": y * u}
        dh = s["dh"].double()
        dg, du = dh * u * slope, dh * y
        return {"da": torch.mm(dg, w[:n]) + torch.mm(du, w[n:]), "dw": torch.cat((torch.mm(dg.t(), a), torch.mm(du.t(), a)))}
    logits = torch.mm(a, w.t())
    lse = torch.logsumexp(logits, 1)
    rows = torch.nonzero(s["targets"] >= 0)[:, 0]
    loss = torch.zeros_like(lse)
    loss[rows] = lse[rows] - logits[rows, s["targets"][rows]]
    if op == "entropy":
        return {"loss": loss, "lse": lse}
    d = torch.softmax(logits, 1)
    d[rows, s["targets"][rows]] -= 1
    scale = torch.zeros_like(lse)
    scale[rows] = s["dloss"][rows].double()
    d *= scale[:, None]
    return {"loss": loss, "lse": lse, "da": torch.mm(d, w), "dw": torch.mm(d.t(), a)}
