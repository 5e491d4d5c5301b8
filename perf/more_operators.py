"""The operators of a block-sparse feed-forward block and of its training, as cases that can be timed.

A transformer's feed-forward block normalises the stream of hidden states, multiplies by two block-sparse projections, gates
one by the other, and adds what comes back, normalised and scaled, to the stream.  An `op` is one of

  "gated"          z_g = X Wg^T + bg,  z_u = X Wu^T + bu,  H = act(z_g) z_u
                   Wg and Wu (n, k) in blocks of bs_r x bs_c.  The sums Z (m, 2 n) are kept block-row by block-row: bs_r columns
                   of z_g, the same columns of z_u, and so on; biases are given in that order.
  "gated_back"     dz_g = G z_u act'(z_g),  dz_u = G act(z_g)  (both in Z's order),  db = the sums of their columns
  "norm"           b = post(B),  S' = beta S + alpha gate b,  U = pre(S')
                   post and pre: none, root mean square, or layer norm, with weights and biases; gate a vector
  "norm_back"      from dL/dS' and dL/dU: dS, dB, and the gradients of the vectors
  "muon"           a step over the blocks of many matrices: M = mu M + g, V = g + mu M; each block of V, divided by its norm, is
                   orthogonalised by five steps X = a X + b (X X^T) X + c (X X^T)^2 X; p = p (1 - lr decay) - lr scale X;
                   each matrix's transposed copy is brought up to date

`dtype` is the type of activations and W (parameters), `out` that of the results (gradients), `stream` that of S.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False                                # True: the framework's entry points; False: the operators in their plain form

_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_NORMS = ("none", "rms", "layer")
_NORM_EPS = 1e-6
_LR, _MOMENTUM, _DECAY, _MUON_EPS = 0.02, 0.95, 0.1, 1e-7
_A, _B, _C = 3.4445, -4.7750, 2.0315       # of the orthogonalising steps
_NS_STEPS = 5
_STEP, _SEED = 1000, 20240                 # of the random roundings of 16-bit parameters without a copy in fp32


# ------------------------------------------------------------------------------------------------ cases
def _gated(name, m, k, n, bs_r, bs_c, dtype, density, act, bias=True, keep_z=False, pattern="uniform", out=None):
    c = {"op": "gated", "m": m, "k": k, "n": n, "bs_r": bs_r, "bs_c": bs_c, "dtype": dtype, "out": out or dtype, "density": density,
         "pattern": pattern, "act": act, "bias": bias, "keep_z": keep_z}
    return dict(c, name=name) if name else c


def _gated_back(name, m, n, unit, dtype, act, out=None):
    c = {"op": "gated_back", "m": m, "n": n, "bs_r": unit, "dtype": dtype, "out": out or dtype, "act": act}
    return dict(c, name=name) if name else c


def _norm(op, name, m, n, stream, dtype, post, pre, gate=True, weights=True, biases=False, alpha=1.0, beta=1.0, weight=None):
    c = {"op": op, "m": m, "n": n, "stream": stream, "dtype": dtype, "out": dtype, "post": post, "pre": pre, "gate": gate,
         "weights": weights, "biases": biases, "alpha": alpha, "beta": beta, "weight": weight or dtype}
    return dict(c, name=name) if name else c


def _muon(name, layers, blocks, bs_r, bs_c, dtype, master, transposed=True, out=None):
    c = {"op": "muon", "layers": layers, "blocks": blocks, "bs_r": bs_r, "bs_c": bs_c, "dtype": dtype, "out": out or dtype,
         "master": master, "transposed": transposed}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token through a small layer: latency of a single call
        _gated("one token", 1, 1024, 1024, 16, 16, "bf16", 0.15, "silu"),
        # a training batch; the sums are kept for the backward pass
        _gated("training batch", 4096, 1024, 4096, 16, 16, "bf16", 0.20, "silu", keep_z=True),
        # prompts of several requests one behind the other: an odd number of rows, results handed on in fp32
        _gated("ragged prompt", 1003, 2080, 1504, 32, 32, "f16", 0.15, "gelu", out="f32"),
        # the largest: 64x64 blocks, a long batch without gradients
        _gated("long batch", 8192, 8192, 8192, 64, 64, "f16", 0.05, "gelu_tanh", bias=False),
        # the gradient of a training batch's gate; and of a small odd one in fp32 whose result is rounded to 16 bits
        _gated_back("gate's gradient", 8192, 4096, 16, "bf16", "silu"),
        _gated_back("odd gate's gradient", 1003, 2080, 32, "f32", "gelu", out="f16"),
        # one token's norms between two blocks
        _norm("norm", "one token's norms", 1, 1024, "f16", "f16", "rms", "rms"),
        # a training batch's, the stream held in fp32, and their gradients
        _norm("norm", "batch's norms", 8192, 4096, "f32", "bf16", "rms", "rms", alpha=0.5),
        _norm("norm_back", "norms' gradient", 8192, 4096, "f32", "bf16", "rms", "rms", alpha=0.5),
        # a step of one small fp32 layer: latency
        _muon("one layer's step", 1, 922, 32, 32, "f32", False),
        # a model of bf16 layers with fp32 copies, in small blocks and in large ones
        _muon("model's step", 12, 13108, 16, 16, "bf16", True),
        _muon("model's step, large blocks", 12, 819, 64, 64, "bf16", True, out="f32"),
    ]


def _cost(c):
    """Seconds, roughly, of a case on one GPU: what a drawn case is held to."""
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / (3e13 if c["dtype"] == "f32" else 1e14 if c["op"] == "muon" else 4e14)


def draw(rng):
    """A case of the same ranges: m 1..8192, widths 128..8192, blocks 8x8 to 64x64 and 16x1, densities 0.03..0.3; gradients of
    1..16384 rows; norms of 1..16384 rows by 1..16384 columns; steps of 1..24 layers of 1..16384 blocks."""
    most = max(_cost(c) for c in listed())

    def log_between(lo, hi):
        return math.exp(rng.uniform(math.log(lo), math.log(hi)))

    while True:
        op = rng.choice(["gated", "gated", "gated", "gated_back", "norm", "norm", "norm_back", "muon", "muon"])
        dtype = rng.choice(["f32", "f16", "bf16"])
        act = rng.choice(_ACTS)
        bs_r, bs_c = rng.choice([(8, 8), (16, 16), (16, 16), (32, 32), (32, 32), (64, 64), (64, 64), (16, 1)])
        if op == "gated":
            dtype = "f32" if bs_c == 1 else dtype
            unit = 64 if rng.random() < 0.7 else bs_r

            def width():
                return max(2, round(log_between(128, 8192) / unit)) * unit

            c = _gated(None, round(log_between(1, 8192)), width(), width(), bs_r, bs_c, dtype, round(log_between(0.03, 0.3), 3), act,
                       rng.random() < 0.7, rng.random() < 0.5, "power" if bs_c > 1 and rng.random() < 0.25 else "uniform",
                       "f32" if dtype != "f32" and rng.random() < 0.2 else dtype)
        elif op == "gated_back":
            unit = rng.choice([1, 4, 8, 16, 16, 32, 64])
            # gradients in fp32 may be rounded to the layer's type
            out = rng.choice(["f32", "f16", "bf16"]) if dtype == "f32" else dtype
            c = _gated_back(None, round(log_between(1, 16384)), max(1, round(log_between(1, 8192) / unit)) * unit, unit, dtype, act, out)
        elif op in ("norm", "norm_back"):
            n = round(log_between(1, 16384))
            n = n if rng.random() < 0.4 else max(1, n // 64) * 64
            post, pre = rng.choice(_NORMS), rng.choice(_NORMS + ("rms",))
            c = _norm(op, None, round(log_between(1, 16384)), n, rng.choice(["f32", dtype]), dtype, post, pre, rng.random() < 0.5,
                      rng.random() < 0.8, rng.random() < 0.3, rng.choice([1.0, 0.5]), rng.choice([1.0, 1.0, 0.75]),
                      rng.choice(["f32", dtype]))
        else:
            bs_r, bs_c = rng.choice([(8, 8), (16, 16), (16, 16), (32, 32), (64, 64), (16, 1), (16, 32), (64, 16), (24, 40)])
            c = _muon(None, round(log_between(1, 24)), round(log_between(1, 16384)), bs_r, bs_c, dtype,
                      dtype != "f32" and rng.random() < 0.7, rng.random() < 0.6, "f32" if rng.random() < 0.3 else dtype)
        if _cost(c) <= most:
            return c


# ------------------------------------------------------------------------------------------------ inputs
def _stored(c):
    return max(1, round(c["density"] * (c["n"] // c["bs_r"]) * (c["k"] // c["bs_c"])))


def _pattern(c, rng):
    """index_pointer and block_indices of one projection, sorted within a block-row."""
    R, C, total = c["n"] // c["bs_r"], c["k"] // c["bs_c"], _stored(c)
    if c["pattern"] == "uniform":
        at = np.sort(rng.choice(R * C, size=total, replace=False, shuffle=False))
        counts, idx = np.bincount(at // C, minlength=R), (at % C).astype(np.int32)
    else:                                  # blocks a block-row by a rank power law, at most all of a row
        share = np.arange(1, R + 1, dtype=np.float64) ** -1.2
        lo, hi = 0.0, float(total) * R ** 1.2 + C
        for _ in range(60):                # the factor at which the rows, cut at C, hold `total` blocks
            mid = (lo + hi) / 2
            lo, hi = (mid, hi) if np.minimum(share * mid, C).sum() < total else (lo, mid)
        wanted = np.minimum(share * hi, C)
        counts = np.floor(wanted).astype(np.int64)
        counts[np.argsort(counts - wanted, kind="stable")[: total - counts.sum()]] += 1
        counts = counts[rng.permutation(R)]
        idx = np.concatenate([np.sort(rng.permutation(C)[:v]) for v in counts]).astype(np.int32)
    ptr = np.zeros(R + 1, dtype=np.int32)
    np.cumsum(counts, out=ptr[1:])
    return ptr, idx


def _inputs(c, seed):
    """What a pass takes, made from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, scale=1.0, shift=0.0, dtype=c["dtype"]):
        return (torch.randn(shape, generator=gen, device="cuda") * scale + shift).to(_TORCH[dtype])

    s = {"case": c}
    if c["op"] == "gated":
        rng = np.random.default_rng(seed)
        for half in ("gate", "up"):
            ptr, idx = _pattern(c, rng)
            s[half] = {"ptr": ptr, "idx": idx, "blocks": normal(len(idx), c["bs_r"], c["bs_c"], scale=(c["density"] * c["k"]) ** -0.5),
                       "rows": torch.from_numpy(np.repeat(np.arange(len(ptr) - 1), np.diff(ptr))).cuda(),
                       "cols": torch.from_numpy(idx.astype(np.int64)).cuda()}
        s["X"] = normal(c["m"], c["k"])
        s["bias"] = normal(2 * c["n"], scale=0.3) if c["bias"] else None
    elif c["op"] == "gated_back":
        s["G"] = normal(c["m"], c["n"])
        s["Z"] = normal(c["m"], 2 * c["n"])
    elif c["op"] in ("norm", "norm_back"):
        m, n = c["m"], c["n"]
        # a stream grows with depth and has a few columns that are much larger than the others
        column = 1 + 8 * (torch.rand(n, generator=gen, device="cuda") < 0.01)
        s["S"] = (torch.randn((m, n), generator=gen, device="cuda") * 2 * column + 0.1).to(_TORCH[c["stream"]])
        s["B"] = normal(m, n, scale=0.7, shift=0.05)
        vector = lambda there, shift: normal(n, scale=0.2, shift=shift, dtype=c["weight"]) if there else None  # noqa: E731
        for side in ("post", "pre"):
            s[side + "_weight"] = vector(c["weights"] and c[side] != "none", 1.0)
            s[side + "_bias"] = vector(c["biases"] and c[side] != "none", 0.0)
        s["gate"] = vector(c["gate"], 0.5)
        if c["op"] == "norm_back":         # S is the sum S' here
            s["GS"] = normal(m, n, scale=1e-2, dtype=c["stream"])
            s["GU"] = normal(m, n, scale=1e-2) if c["pre"] != "none" else None
    else:
        L, shape = c["layers"], (c["layers"], c["blocks"], c["bs_r"], c["bs_c"])
        rand = lambda: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
        # gradients differ in size from row to row of a block, and a part of theirs is of rank one
        size = 1e-3 * torch.exp(torch.randn(shape[:3] + (1,), generator=gen, device="cuda"))
        ones = torch.randn(shape[:3] + (1,), generator=gen, device="cuda") * torch.randn(shape[:2] + (1, c["bs_c"]), generator=gen, device="cuda")
        s["grads"] = ((rand() + 2 * ones) * size).to(_TORCH[c["out"]])
        s["momentum"] = (rand() + 4 * ones) * size * 4
        master = rand() * 0.02
        s["params"] = master.to(_TORCH[c["dtype"]])
        s["master"] = master if c["master"] else None
        s["perm"] = s["transposed"] = None
        if c["transposed"]:                # stored block q of a transposed copy is block perm[q] of the matrix
            s["perm"] = torch.argsort(torch.rand(shape[:2], generator=gen, device="cuda"), dim=1)
            s["transposed"] = torch.zeros((L, c["blocks"], c["bs_c"], c["bs_r"]), dtype=_TORCH[c["dtype"]], device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _prepare_own(s)
    return s


# ------------------------------------------------------------------------------------------------ plain form
def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return z * 0.5 * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return z * 0.5 * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "gelu_tanh":
        a = (2 / math.pi) ** 0.5
        t = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        g = 1 / (1 + torch.exp(-z))
        return g * (1 + z * (1 - g))
    return torch.ones_like(z)


def _halves(z, unit):
    """The gate's and the other half's columns of rows in the order of Z."""
    z = z.view(z.shape[0], -1, 2, unit)
    return z[:, :, 0].reshape(z.shape[0], -1), z[:, :, 1].reshape(z.shape[0], -1)


def _joined(g, u, unit):
    return torch.stack((g.view(g.shape[0], -1, unit), u.view(u.shape[0], -1, unit)), 2).reshape(g.shape[0], -1)


def _plain_gated(s):
    c = s["case"]
    dense = torch.zeros((c["n"] // c["bs_r"], 2, c["bs_r"], c["k"] // c["bs_c"], c["bs_c"]), device="cuda")
    for i, half in enumerate((s["gate"], s["up"])):
        dense[:, i].permute(0, 2, 1, 3)[half["rows"], half["cols"]] = half["blocks"].float()
    z = s["X"].float() @ dense.view(2 * c["n"], c["k"]).t()
    if c["bias"]:
        z = z + s["bias"].float()
    zg, zu = _halves(z, c["bs_r"])
    h = (_act(zg, c["act"]) * zu).to(_TORCH[c["out"]])
    return {"H": h, "Z": z.to(_TORCH[c["out"]])} if c["keep_z"] else {"H": h}


def _plain_gated_back(s):
    c = s["case"]
    g = s["G"].float()
    zg, zu = _halves(s["Z"].float(), c["bs_r"])
    dz = _joined(g * zu * _act_grad(zg, c["act"]), g * _act(zg, c["act"]), c["bs_r"])
    return {"dZ": dz.to(_TORCH[c["out"]]), "db": dz.sum(0, dtype=torch.float64).float()}


def _centred(x, kind):
    """What a norm divides, and what it divides by, inverted."""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    return x, torch.rsqrt((x * x).mean(1, keepdim=True) + _NORM_EPS)


def _plain_vector(v):
    return v.float() if v is not None else None


def _normed(x, kind, weight, bias):
    if kind != "none":
        x, r = _centred(x, kind)
        x = x * r
        if weight is not None:
            x = x * weight
        if bias is not None:
            x = x + bias
    return x


def _plain_norm(s):
    c = s["case"]
    b = _normed(s["B"].float(), c["post"], _plain_vector(s["post_weight"]), _plain_vector(s["post_bias"]))
    if s["gate"] is not None:
        b = b * s["gate"].float()
    total = c["beta"] * s["S"].float() + c["alpha"] * b
    r = {"S": total.to(_TORCH[c["stream"]])}
    if c["pre"] != "none":
        r["U"] = _normed(total, c["pre"], _plain_vector(s["pre_weight"]), _plain_vector(s["pre_bias"])).to(_TORCH[c["out"]])
    return r


def _norm_grad(g, x, kind, weight):
    """Gradient of a norm's input; and the sums that its weight's and bias's gradients are."""
    x, r = _centred(x, kind)
    hat = x * r
    sums = (g.double() * hat).sum(0).float(), g.sum(0, dtype=torch.float64).float()
    if weight is not None:
        g = g * weight
    if kind == "layer":
        g = g - g.mean(1, keepdim=True)
    return r * (g - hat * (g * hat).mean(1, keepdim=True)), sums


def _plain_norm_back(s):
    c = s["case"]
    r = {}
    g = s["GS"].float()
    if c["pre"] != "none":
        d, sums = _norm_grad(s["GU"].float(), s["S"].float(), c["pre"], _plain_vector(s["pre_weight"]))
        g = g + d
        r["pre_weight"], r["pre_bias"] = sums
    r["dS"] = (c["beta"] * g).to(_TORCH[c["stream"]])
    b = s["B"].float()
    if s["gate"] is not None:
        branch = _normed(b, c["post"], _plain_vector(s["post_weight"]), _plain_vector(s["post_bias"]))
        r["gate"] = (g.double() * branch).sum(0).float() * c["alpha"]
        g = g * s["gate"].float()
    g = g * c["alpha"]
    if c["post"] != "none":
        g, sums = _norm_grad(g, b, c["post"], _plain_vector(s["post_weight"]))
        r["post_weight"], r["post_bias"] = sums
    r["dB"] = g.to(_TORCH[c["out"]])
    return _of_vectors(s, r)


def _of_vectors(s, r):
    """Without the gradients of vectors that are not there."""
    return {k: v for k, v in r.items() if k in ("dS", "dB") or s[k] is not None}


def _mix(x):
    """Two rounds of xor-shift and multiply, modulo 2^32."""
    x = x ^ (x >> 16)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(shape):
    """A number below 2^32 for each element, a hash of the seed, the step, the layer and the element."""
    key = _mix((_SEED + 0x9E3779B1 * _STEP) & 0xFFFFFFFF)
    layer = _mix((torch.arange(shape[0], device="cuda") + key) & 0xFFFFFFFF)
    element = torch.arange(shape[1] * shape[2] * shape[3], device="cuda")
    return _mix((layer[:, None] + element) & 0xFFFFFFFF).view(shape)


def _round_at_random(x, random, dtype):
    """fp32 to a 16-bit type: up in size as often as keeps the mean."""
    step = torch.exp2((torch.frexp(x).exponent - 1).clamp_min(-126 if dtype == torch.bfloat16 else -14).double() - (7 if dtype == torch.bfloat16 else 10))
    bits = 16 if dtype == torch.bfloat16 else 13
    size = torch.floor(x.abs().double() / step + (random & ((1 << bits) - 1)).double() * 2.0 ** -bits) * step
    return torch.where(x < 0, -size, size).to(dtype)


def _muon_scale(c):
    """Of an update: tall blocks' are larger, so that an update's root mean square does not hang on the block's sides."""
    return math.sqrt(max(1.0, c["bs_r"] / c["bs_c"]))


def _plain_muon(s):
    c = s["case"]
    g = s["grads"].float()
    s["momentum"].mul_(_MOMENTUM).add_(g)
    v = (g + _MOMENTUM * s["momentum"]).view(-1, c["bs_r"], c["bs_c"])
    x = v / ((v * v).sum((1, 2), keepdim=True).sqrt() + _MUON_EPS)
    tall = c["bs_r"] > c["bs_c"]
    x = x.transpose(1, 2).contiguous() if tall else x
    for _ in range(_NS_STEPS):
        a = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = _A * x + torch.bmm(_B * a + _C * torch.bmm(a, a), x)
    x = x.transpose(1, 2) if tall else x
    p = (s["master"] if c["master"] else s["params"]).float()
    p = p * (1 - _LR * _DECAY) - _LR * _muon_scale(c) * x.reshape(p.shape)
    if c["master"]:
        s["master"].copy_(p)
    if c["dtype"] == "f32" or c["master"]:
        s["params"].copy_(p)
    else:
        s["params"].copy_(_round_at_random(p, _random(p.shape), _TORCH[c["dtype"]]))
    if c["transposed"]:
        at = s["perm"][:, :, None, None].expand(-1, -1, c["bs_r"], c["bs_c"])
        s["transposed"].copy_(torch.gather(s["params"], 1, at).transpose(2, 3))
    return _muon_outputs(s)


def _muon_outputs(s):
    """The parameters and the state as they are after the step."""
    return {k: s[k] for k in ("params", "momentum", "master", "transposed") if s[k] is not None}


# ------------------------------------------------------------------------------------------------ the framework's
def _prepare_own(s):
    """What a user's program keeps: the matrix's handle, the optimizer's."""
    import paper_2007_13055_amd as lib
    c = s["case"]
    s["lib"] = lib
    if c["op"] == "gated":
        arrays = lib.bsr_gated_arrays(*((h["blocks"], h["idx"], h["ptr"]) for h in (s["gate"], s["up"])))
        s["W"] = lib.bsr_create(2 * c["n"], c["k"], *arrays)
    elif c["op"] in ("norm", "norm_back"):
        s["how"] = {"post": c["post"], "pre": c["pre"], "gate": s["gate"], "eps": _NORM_EPS, "stream_scale": c["beta"], "branch_scale": c["alpha"],
                    **{f"{side}_{what}": s[f"{side}_{what}"] for side in ("post", "pre") for what in ("weight", "bias")}}
    elif c["op"] == "muon":
        L = range(c["layers"])
        perm = s["perm"].int().cpu().numpy() if c["transposed"] else None
        s["opt"] = lib.bsr_muon_create([s["params"][i] for i in L], [s["grads"][i] for i in L], weight_decay=_DECAY,
                                       momentum=[s["momentum"][i] for i in L], master=[s["master"][i] for i in L] if c["master"] else None,
                                       transposed=[(s["transposed"][i], perm[i]) for i in L] if c["transposed"] else None)


def _own(s):
    lib, c = s["lib"], s["case"]
    if c["op"] == "gated":
        got = lib.bsr_spmm_gated(s["W"], s["X"], h_dtype=c["out"], bias=s["bias"], act=c["act"], keep_z=c["keep_z"])
        return {"H": got[0], "Z": got[1]} if c["keep_z"] else {"H": got}
    if c["op"] == "gated_back":
        dz, db = lib.bsr_gated_backward(s["G"], s["Z"], c["bs_r"], act=c["act"], dz_dtype=c["out"])
        return {"dZ": dz, "db": db}
    if c["op"] == "norm":
        total, u = lib.bsr_residual_norm(s["S"], s["B"], **s["how"])
        return {"S": total, "U": u} if c["pre"] != "none" else {"S": total}
    if c["op"] == "norm_back":
        ds, db, grads = lib.bsr_residual_norm_backward(s["S"], s["B"], s["GS"], s["GU"], **s["how"])
        return {"dS": ds, "dB": db, **grads}
    lib.bsr_muon_step(s["opt"], _STEP, lr=_LR, momentum=_MOMENTUM, nesterov=True, ns_steps=_NS_STEPS, coefficients=(_A, _B, _C), eps=_MUON_EPS,
                      seed=_SEED)
    return _muon_outputs(s)


def run(state):
    if own:
        return _own(state)
    return {"gated": _plain_gated, "gated_back": _plain_gated_back, "norm": _plain_norm, "norm_back": _plain_norm_back,
            "muon": _plain_muon}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ floors and exact values
def work(case):
    """Each input read once and each output written once."""
    c = case
    s_in, s_out = _SIZE[c["dtype"]], _SIZE[c["out"]]
    if c["op"] == "gated":
        nnzb, R, C, block = 2 * _stored(c), 2 * (c["n"] // c["bs_r"]), c["k"] // c["bs_c"], c["bs_r"] * c["bs_c"]
        used_cols = C * (1.0 - (1.0 - nnzb / (R * C)) ** R)      # block-columns that hold a block, expected
        return {"bytes": c["m"] * used_cols * c["bs_c"] * s_in + nnzb * block * s_in + 4 * (nnzb + R + 1)
                + c["bias"] * 2 * c["n"] * s_in + (1 + 2 * c["keep_z"]) * c["m"] * c["n"] * s_out, "flops": 2 * c["m"] * nnzb * block}
    if c["op"] == "gated_back":
        return {"bytes": c["m"] * c["n"] * (3 * s_in + 2 * s_out) + 8 * c["n"], "flops": 16 * c["m"] * c["n"]}
    if c["op"] in ("norm", "norm_back"):
        s_stream, s_weight = _SIZE[c["stream"]], _SIZE[c["weight"]]
        normed = (c["post"] != "none") + (c["pre"] != "none")
        vectors = c["gate"] + normed * (c["weights"] + c["biases"])
        pre = c["pre"] != "none"
        if c["op"] == "norm":
            return {"bytes": c["m"] * c["n"] * (2 * s_stream + s_in + pre * s_out) + vectors * c["n"] * s_weight,
                    "flops": c["m"] * c["n"] * (4 + 5 * normed)}
        # S' is read for the norm of it, B for the norm of it and for the gate's gradient
        reads = s_stream * (1 + pre) + s_in * (pre + (c["post"] != "none" or c["gate"]))
        return {"bytes": c["m"] * c["n"] * (reads + s_stream + s_out) + vectors * c["n"] * (s_weight + 4),
                "flops": c["m"] * c["n"] * (6 + 12 * normed)}
    blocks = c["layers"] * c["blocks"]
    n = blocks * c["bs_r"] * c["bs_c"]
    small, large = min(c["bs_r"], c["bs_c"]), max(c["bs_r"], c["bs_c"])
    each = s_out + 8 + (8 + s_in if c["master"] else 2 * s_in)
    # of the symmetric products one triangle is enough
    flops = _NS_STEPS * ((small + 1) * small * large + (small + 1) * small * small + 2 * small * small * large)
    return {"bytes": n * each + (n * s_in + 4 * blocks if c["transposed"] else 0), "flops": blocks * flops + 12 * n}


def _exact_act(z, act):
    """From the normal distribution's integral, tanh(x) = 2 s(2x) - 1 and the logistic function s."""
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    if act == "gelu_tanh":
        return z * torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _exact_norm(x, kind, weight, bias):
    if kind == "none":
        return x
    square = x.pow(2).mean(1, keepdim=True)
    if kind == "layer":
        mean = x.mean(1, keepdim=True)
        x, square = x - mean, (x - mean).pow(2).mean(1, keepdim=True)
    y = x / (square + _NORM_EPS).sqrt()
    y = y if weight is None else y * weight
    return y if bias is None else y + bias


def _exact_norms(c, v, S):
    """S' and U, the tensors of `v` in 64 bits; S given: S' as it is."""
    total = S
    branch = _exact_norm(v["B"], c["post"], v.get("post_weight"), v.get("post_bias"))
    if v.get("gate") is not None:
        branch = branch * v["gate"]
    total = c["beta"] * S + c["alpha"] * branch
    return total, lambda t: _exact_norm(t, c["pre"], v.get("pre_weight"), v.get("pre_bias"))


def exact(case, seed):
    """What run() returns, in 64 bits; gradients by differentiation."""
    c, s = case, _inputs(case, seed)
    if c["op"] == "gated":
        sums = []
        a, b = torch.arange(c["bs_r"], device="cuda"), torch.arange(c["bs_c"], device="cuda")
        for i, half in enumerate((s["gate"], s["up"])):
            # W's elements one by one: row and column of each
            row = (half["rows"] * c["bs_r"])[:, None, None] + a[None, :, None] + 0 * b
            col = (half["cols"] * c["bs_c"])[:, None, None] + 0 * a[None, :, None] + b
            w = torch.zeros(c["n"] * c["k"], dtype=torch.float64, device="cuda")
            w.index_add_(0, (row * c["k"] + col).reshape(-1), half["blocks"].double().reshape(-1))
            z = torch.mm(s["X"].double(), w.view(c["n"], c["k"]).t().contiguous())
            if s["bias"] is not None:
                z += s["bias"].double().view(-1, 2, c["bs_r"])[:, i].reshape(-1)
            sums.append(z)
        r = {"H": _exact_act(sums[0], c["act"]) * sums[1]}
        if c["keep_z"]:
            r["Z"] = torch.cat([z.view(c["m"], -1, 1, c["bs_r"]) for z in sums], 2).view(c["m"], 2 * c["n"])
        return r
    if c["op"] == "gated_back":
        z = s["Z"].double().requires_grad_()
        pairs = z.view(c["m"], -1, 2, c["bs_r"])
        h = (_exact_act(pairs[:, :, 0], c["act"]) * pairs[:, :, 1]).reshape(c["m"], c["n"])
        if c["act"] == "relu":             # its slope at 0 is 0
            h = (torch.where(pairs[:, :, 0] > 0, pairs[:, :, 0], 0.0) * pairs[:, :, 1]).reshape(c["m"], c["n"])
        dz, = torch.autograd.grad(h, z, s["G"].double())
        return {"dZ": dz, "db": dz.sum(0)}
    if c["op"] in ("norm", "norm_back"):
        names = [k for k in ("B", "post_weight", "post_bias", "gate", "pre_weight", "pre_bias") if s[k] is not None]
        v = {k: s[k].double() for k in names}
        if c["op"] == "norm":
            total, after = _exact_norms(c, v, s["S"].double())
            return {"S": total, "U": after(total)} if c["pre"] != "none" else {"S": total}
        with torch.enable_grad():
            v = {k: t.requires_grad_() for k, t in v.items()}
            given = torch.zeros_like(v["B"]).requires_grad_()
            total, after = _exact_norms(c, v, given)
            # the sum is what was stored: its gradient is taken there
            at = s["S"].double() + (total - total.detach())
            loss = (at * s["GS"].double()).sum()
            if c["pre"] != "none":
                loss = loss + (after(at) * s["GU"].double()).sum()
            grads = torch.autograd.grad(loss, [given, *v.values()])
        r = dict(zip(["dS", *v], grads))
        r["dB"] = r.pop("B")
        return r
    p = (s["master"] if c["master"] else s["params"]).double()
    g = s["grads"].double()
    momentum = _MOMENTUM * s["momentum"].double() + g
    x = (g + _MOMENTUM * momentum).view(-1, c["bs_r"], c["bs_c"])
    x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + _MUON_EPS)
    for _ in range(_NS_STEPS):             # the Gram matrix of the rows or of the columns: the result is the same
        if c["bs_r"] <= c["bs_c"]:
            gram = torch.bmm(x, x.mT.contiguous())
            x = _A * x + _B * torch.bmm(gram, x) + _C * torch.bmm(gram, torch.bmm(gram, x))
        else:
            gram = torch.bmm(x.mT.contiguous(), x)
            x = _A * x + _B * torch.bmm(x, gram) + _C * torch.bmm(torch.bmm(x, gram), gram)
    p = p - _LR * (_DECAY * p + _muon_scale(c) * x.view(p.shape))
    r = {"params": p, "momentum": momentum}
    if c["master"]:
        r["master"] = p
    if c["transposed"]:
        at = (s["perm"] + torch.arange(c["layers"], device="cuda")[:, None] * c["blocks"]).reshape(-1)
        r["transposed"] = p.reshape(-1, c["bs_r"], c["bs_c"])[at].transpose(1, 2).reshape(c["layers"], c["blocks"], c["bs_c"], c["bs_r"])
    return r
