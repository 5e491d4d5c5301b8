"""The norms around a block and their gradients in 64 bits, and how far fp32 arithmetic may be from them."""
import numpy as np

U32 = 2.0 ** -24
# A row's sum: chains of at most 32 terms a lane, then 6 additions across lanes and 8 across wavefronts.
CHAIN = 48


def norm(x, kind, weight=None, bias=None, eps=1e-6, off=0.0):
    """(y, bound): the norm of rows x, each element of which may be `off` away, and its fp32 error.

    centred elements: the mean is off by CHAIN U32 mean|x| + mean(off), a subtraction rounds once.  Call that d.  The mean
    square's root: relative error d / root + CHAIN U32 / 2 + the root's 2^-22.  Three more roundings."""
    if kind == "none":
        return x, np.zeros_like(x) + off
    off = np.zeros_like(x) + off
    d, xm = off, x
    if kind == "layer":
        mean = x.mean(1, keepdims=True)
        xm = x - mean
        d = off + off.mean(1, keepdims=True) + CHAIN * U32 * np.abs(x).mean(1, keepdims=True) + U32 * (np.abs(x) + np.abs(mean))
    r = 1 / np.sqrt((xm * xm).mean(1, keepdims=True) + eps)
    rel = r * np.sqrt((d * d).mean(1, keepdims=True)) + CHAIN * U32 / 2 + 2.0 ** -22
    y, e = xm * r, d * r * (1 + rel) + np.abs(xm * r) * (rel + U32)
    if weight is not None:
        y, e = y * weight, e * np.abs(weight)
    if bias is not None:
        y = y + bias
    return y, e + 3 * U32 * (np.abs(y) + (0 if bias is None else np.abs(bias)))


def forward(S, B, post, pre, v, alpha, beta, eps=1e-6):
    """((S', bound), (U, bound) or None); v: dict of the vectors."""
    total, e = beta * S, U32 * np.abs(beta * S)
    if B is not None:
        b, eb = norm(B, post, v.get("post_weight"), v.get("post_bias"), eps)
        f = alpha * (1.0 if v.get("gate") is None else v["gate"])
        total = total + f * b
        e = e + np.abs(f) * eb + 3 * U32 * (np.abs(f * b) + np.abs(beta * S))
    if pre == "none":
        return (total, e), None
    return (total, e), norm(total, pre, v.get("pre_weight"), v.get("pre_bias"), eps, e)


def norm_gradient(g, eg, x, kind, weight, eps):
    """Of a norm's input from g (off by eg): r (gw - mean(gw) - xm c), c = r^2 mean(gw xm), and its error; and the terms of the
    weight's gradient with theirs."""
    xm, d = x, np.zeros_like(x)
    if kind == "layer":
        mean = x.mean(1, keepdims=True)
        xm = x - mean
        d = CHAIN * U32 * np.abs(x).mean(1, keepdims=True) + U32 * (np.abs(x) + np.abs(mean))
    mean_of = lambda t: t.mean(1, keepdims=True)  # noqa: E731
    r = 1 / np.sqrt(mean_of(xm * xm) + eps)
    rel = r * np.sqrt(mean_of(d * d)) + CHAIN * U32 / 2 + 2.0 ** -22          # of r
    w = 1.0 if weight is None else weight
    gw, ew = g * w, np.abs(w) * eg + U32 * np.abs(g * w)
    c, size = r * r * mean_of(gw * xm), r * r * mean_of(np.abs(gw * xm))
    ec = size * (2 * rel + CHAIN * U32) + r * r * mean_of(ew * np.abs(xm) + np.abs(gw) * d)
    shift = mean_of(gw) if kind == "layer" else 0.0
    es = mean_of(ew) + CHAIN * U32 * mean_of(np.abs(gw)) if kind == "layer" else 0.0
    inner, terms = gw - shift - xm * c, np.abs(gw) + np.abs(shift) + np.abs(xm * c)
    e = r * (ew + es + np.abs(xm) * ec + d * np.abs(c) + 4 * U32 * terms) + np.abs(r * inner) * (rel + U32)
    hat, eh = xm * r, d * r + np.abs(xm * r) * (rel + U32)
    return r * inner, e, hat, eh


def backward(S, B, GS, GU, post, pre, v, alpha, beta, eps=1e-6):
    """{name: (value, bound)}; sums over rows carry the rows' errors and one rounding an addition of at most all terms."""
    out = {}

    def column_sum(name, t, e):
        out[name] = t.sum(0), e.sum(0) + (len(t) + 8) * U32 * np.abs(t).sum(0)

    g, e = GS.copy(), np.zeros_like(GS)
    if pre != "none":
        d, ed, hat, eh = norm_gradient(GU, np.zeros_like(GU), S, pre, v.get("pre_weight"), eps)
        g, e = g + d, ed + U32 * (np.abs(g) + np.abs(d)) * 2
        column_sum("pre_weight", GU * hat, np.abs(GU) * (eh + U32 * np.abs(hat)))
        column_sum("pre_bias", GU, np.zeros_like(GU))
    out["dS"] = beta * g, abs(beta) * e + U32 * np.abs(beta * g)
    if B is None:
        return out
    b, eb = norm(B, post, v.get("post_weight"), v.get("post_bias"), eps)
    ag, ea = alpha * g, abs(alpha) * e + U32 * np.abs(alpha * g)
    column_sum("gate", ag * b, ea * np.abs(b) + np.abs(ag) * eb + 2 * U32 * np.abs(ag * b))
    gate = 1.0 if v.get("gate") is None else v["gate"]
    t, et = ag * gate, ea * np.abs(gate) + U32 * np.abs(ag * gate)
    if post == "none":
        out["dB"] = t, et
        return out
    # (the kernel's means take alpha, g, gate and weight multiplied in another order: two roundings more)
    d, ed, hat, eh = norm_gradient(t, et + 2 * U32 * np.abs(t), B, post, v.get("post_weight"), eps)
    column_sum("post_weight", t * hat, et * np.abs(hat) + np.abs(t) * (eh + U32 * np.abs(hat)))
    column_sum("post_bias", t, et)
    out["dB"] = d, ed
    return out
