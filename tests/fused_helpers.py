"""Plain 64-bit forms of the gated feed-forward layer and of the cross entropy, and bounds on what fp32 arithmetic may leave."""
import math

import torch

from paper_2302_08007_b200 import binding as bdr

CFG = {"mx4": bdr.MX4, "mx6": bdr.MX6, "mx9": bdr.MX9}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # finfo.eps / 2, relative to the value
ACTS = {"silu": bdr.ACT_SILU, "gelu": bdr.ACT_GELU, "gelu_tanh": bdr.ACT_GELU_TANH, "relu": bdr.ACT_RELU}


def packed(cfg, x):
    """Planes of x along its rows and the values they stand for, in 64 bits."""
    p = bdr.bdr_pack(cfg, x, bdr.alloc_planes(cfg, *x.shape))
    y = bdr.bdr_unpack(cfg, p, torch.empty_like(x, dtype=torch.float32))
    return p, y.double()


def workspace(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda").fill_(0xFF)   # NaN wherever it is read before it is written


def gate(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        p = torch.special.expit(g)
        return g * p, p + g * p * torch.special.expit(-g)
    if act == "gelu":
        below = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * below, below + g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        p = torch.special.expit(2 * c * (g + 0.044715 * g ** 3))
        return g * p, p + g * p * (1 - p) * 2 * c * (1 + 0.134145 * g ** 2)
    return torch.where(g < 0, 0.0, g), (g > 0).double()


def sum_bound(n, size):
    """Error of a sum of n products accumulated in fp32, sixteen at a time, cut off rather than rounded: every addition is off by at most
    2^-23 of the sum of the magnitudes `size`, and so are the sixteen terms of each."""
    return (n / 16 + 17) * 2.0 ** -23 * size


def gated(a, w, n, act):
    """h, the two products, and the bounds of all three in fp32."""
    gu = a @ w.T
    e = sum_bound(a.shape[1], a.abs() @ w.abs().T)
    g, u, eg, eu = gu[:, :n], gu[:, n:], e[:, :n], e[:, n:]
    y, _ = gate(g, act)
    # slopes are below 1.2; the activation itself is within 2^-20 of |g| (exponential, quotient, and for the tanh form the argument's
    # own rounding, whose effect is largest where the sigmoid is not yet small)
    eh = 1.2 * eg * (u.abs() + eu) + y.abs() * eu + 2.0 ** -20 * (g * u).abs()
    return y * u, gu, eh, e


def gated_grads(a, w, n, act, dh, gu, egu, dtype):
    """da, dw and their bounds.  gu: the products, egu: how far the kernel's may be from them."""
    g, u, eg, eu = gu[:, :n], gu[:, n:], egu[:, :n], egu[:, n:]
    y, slope = gate(g, act)
    d = torch.cat((dh * u * slope, dh * y), 1)
    es = 1.0 * eg + 2.0 ** -20 * (1 + g.abs())                       # second derivatives are below 1
    if act == "relu":
        es = es + (g.abs() <= eg).double() * (eg > 0)
    ed = torch.cat((dh.abs() * (eu * (slope.abs() + es) + u.abs() * es), dh.abs() * (1.2 * eg + 2.0 ** -20 * g.abs())), 1)
    return products(d, ed, a, w, dtype)


def products(d, ed, a, w, dtype):
    """d w, d^T a with bounds: d itself is off by ed, rounded to the type (three parts: 24 bits, at least 2^-134 apart from zero)."""
    ed = ed + HALF_STEP[dtype] * (d.abs() + ed) + 2.0 ** -133
    da, dw = d @ w, d.T @ a
    size_a, size_w = (d.abs() + ed) @ w.abs(), (d.abs() + ed).T @ a.abs()
    parts = 3 if dtype == torch.float32 else 1
    ea = ed @ w.abs() + sum_bound(parts * d.shape[1], size_a) + HALF_STEP[dtype] * (da.abs() + ed @ w.abs())
    ew = ed.T @ a.abs() + sum_bound(parts * d.shape[0], size_w) + HALF_STEP[dtype] * (dw.abs() + ed.T @ a.abs())
    return da, dw, ea, ew


def entropy(a, w, targets):
    """loss, lse, logits and the bounds of the three."""
    logits = a @ w.T
    e = sum_bound(a.shape[1], a.abs() @ w.abs().T)
    lse = torch.logsumexp(logits, 1)
    there = (targets >= 0) & (targets < w.shape[0])
    at = targets.clamp(0, w.shape[0] - 1)[:, None]
    hit, ehit = logits.gather(1, at)[:, 0], e.gather(1, at)[:, 0]
    # the log of a sum of exponentials moves no further than its terms' exponents; the exponentials are within 2^-21, their arguments, up
    # to the spread of the row, within 2^-23 of themselves, the sum of V positive terms joined in pieces within (128 + V / 128) half steps
    spread = (logits.amax(1) - logits.amin(1))
    elog = e.amax(1) + 2.0 ** -21 + spread * 2.0 ** -22 + (160 + w.shape[0] / 128) * 2.0 ** -24 + 4 * 2.0 ** -24 * lse.abs() + 2.0 ** -23
    loss = torch.where(there, lse - hit, 0.0)
    return loss, lse, logits, elog + ehit + 2.0 ** -24 * loss.abs(), elog, e


def entropy_grads(a, w, targets, lse, dloss, dtype, elog=0.0):
    logits = a @ w.T
    e = sum_bound(a.shape[1], a.abs() @ w.abs().T)
    p = torch.exp(logits - lse[:, None])
    there = (targets >= 0) & (targets < w.shape[0])
    rows = torch.nonzero(there)[:, 0]
    d = p.clone()
    d[rows, targets[rows]] -= 1
    scale = torch.where(there, dloss, torch.zeros_like(dloss))[:, None]
    ep = p * (torch.expm1(e + elog + 2.0 ** -22 * (logits - lse[:, None]).abs() + 2.0 ** -21)) + 2.0 ** -23 * d.abs() + 2.0 ** -126
    return products(d * scale, ep * scale.abs(), a, w, dtype)


def check(got, want, bound, what):
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), "%s: %d of %d off; largest error %g of bound %g" % (
        what, int(bad.sum()), bad.numel(), float((got - want).abs()[bad].max()), float(bound.expand_as(want)[bad].max()))
