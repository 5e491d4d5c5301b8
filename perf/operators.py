"""The operators around a block-sparse product that a layer is trained and served with, as cases that can be timed.

A layer holds a weight W (n, k), stored in blocks of bs_r x bs_c, a bias b and an activation.  An `op` is one of

  "product"    Z = X W^T + b,  Y = act(Z) + R                        the layer's forward pass
               with `through`: Y = (X W^T + b) * act'(Z0) + R        a gradient on its way back, through the activation Z0 fed
  "backward"   dZ = G * act'(Z),  db = the sums of dZ's columns      the activation's and the bias's gradients
  "adamw"      one AdamW step over the blocks and the biases of many layers, each matrix's transposed copy brought up to date

`dtype` is the type of X and W (parameters), `out` that of the results (gradients).  8-bit moments are held in blocks of 256
elements: the first as an e4m3 number times a scale, the second on a logarithmic scale between the block's smallest and
largest values, rounded up or down at random so that its mean is kept (in 8 bits a step's change of 0.1 % is below half a
step of any code: rounded to nearest it would never move).  The random numbers are a hash of the seed, the step, the tensor
and the element.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False                                # True: the framework's entry points; False: the operators in their plain form

_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_BLOCK = 256                               # elements that share the scales of 8-bit moments
_HYPER = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8}
_DECAY = 0.1                               # of the blocks; biases have none
_STEP, _SEED = 1000, 20240


# ------------------------------------------------------------------------------------------------ cases
def _product(name, m, k, n, bs_r, bs_c, dtype, density, act, bias=True, residual=False, keep_z=False, through=False,
             pattern="uniform", out=None):
    c = {"op": "product", "m": m, "k": k, "n": n, "bs_r": bs_r, "bs_c": bs_c, "dtype": dtype, "out": out or dtype,
         "density": density, "pattern": pattern, "act": act, "bias": bias, "residual": residual, "keep_z": keep_z, "through": through}
    return dict(c, name=name) if name else c


def _backward(name, m, n, dtype, act, out=None):
    c = {"op": "backward", "m": m, "n": n, "dtype": dtype, "out": out or dtype, "act": act}
    return dict(c, name=name) if name else c


def _adamw(name, layers, blocks, bs_r, bs_c, width, dtype, bits, master, transposed=True, out=None):
    c = {"op": "adamw", "layers": layers, "blocks": blocks, "bs_r": bs_r, "bs_c": bs_c, "width": width, "dtype": dtype,
         "out": out or dtype, "bits": bits, "master": master, "transposed": transposed}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token through a small fp32 layer: latency of a single call
        _product("one row", 1, 1024, 1024, 16, 16, "f32", 0.15, "gelu"),
        # a handful of tokens, small blocks, the layer's input added to its output
        _product("eight rows", 8, 1024, 1024, 8, 8, "f16", 0.20, "silu", residual=True),
        # the first layer of a feed-forward part in training: the activation's input is kept for the backward pass
        _product("ffn up", 4096, 1024, 4096, 16, 16, "bf16", 0.20, "gelu", keep_z=True),
        # its second layer on an odd number of rows, results handed on in fp32
        _product("ffn down ragged", 1003, 2080, 1504, 32, 32, "f16", 0.15, "none", residual=True, out="f32"),
        # the gradient of the second layer's input, taken through the activation in front of it
        _product("ffn inner gradient", 4096, 1024, 4096, 32, 32, "bf16", 0.20, "gelu", bias=False, through=True),
        # blocks of one column (fp32)
        _product("thin", 256, 4096, 4096, 16, 1, "f32", 0.05, "relu"),
        # the largest: 64x64 fp16 blocks, a few block-rows hold most of W
        _product("skewed", 8192, 8192, 8192, 64, 64, "f16", 0.05, "gelu_tanh", residual=True, pattern="power"),
        # a training batch's activation gradient and the bias's, and a small odd one whose result is rounded to 16 bits
        _backward("activation gradient", 8192, 8192, "bf16", "gelu"),
        _backward("odd activation gradient", 1003, 2081, "f32", "silu", out="f16"),
        # the optimizer's step of one small fp32 layer: latency
        _adamw("one layer's step", 1, 922, 32, 32, 1024, "f32", 32, False),
        # a model of bf16 layers with fp32 master copies; and one with 8-bit moments and no copies
        _adamw("model's step", 12, 13108, 16, 16, 4096, "bf16", 32, True),
        _adamw("model's step, 8 bits", 12, 13108, 16, 16, 4096, "bf16", 8, False),
    ]


def _cost(c):
    """Seconds, roughly, of a case on one GPU: what a drawn case is held to."""
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / (3e13 if c["dtype"] == "f32" else 4e14)


def draw(rng):
    """A case of the same ranges: m 1..8192, widths 128..8192, blocks 8x8 to 64x64 and 16x1, densities 0.03..0.3; gradients
    of 1..16384 rows by 1..8192 columns; steps of 1..24 layers of 1..16384 blocks."""
    most = max(_cost(c) for c in listed())

    def log_between(lo, hi):
        return math.exp(rng.uniform(math.log(lo), math.log(hi)))

    while True:
        op = rng.choice(["product", "product", "product", "backward", "adamw", "adamw"])
        dtype = rng.choice(["f32", "f16", "bf16"])
        act = rng.choice(_ACTS)
        bs_r, bs_c = rng.choice([(8, 8), (16, 16), (16, 16), (32, 32), (32, 32), (64, 64), (64, 64), (16, 1)])
        if op == "product":
            dtype = "f32" if bs_c == 1 else dtype
            unit = 64 if rng.random() < 0.7 else bs_r

            def width():
                return max(2, round(log_between(128, 8192) / unit)) * unit

            through = act != "none" and rng.random() < 0.25
            c = _product(None, round(log_between(1, 8192)), width(), width(), bs_r, bs_c, dtype, round(log_between(0.03, 0.3), 3),
                         act, rng.random() < 0.8, rng.random() < 0.4, not through and rng.random() < 0.3, through,
                         "power" if bs_c > 1 and rng.random() < 0.25 else "uniform",
                         "f32" if dtype != "f32" and rng.random() < 0.2 else dtype)
        elif op == "backward":
            n = round(log_between(1, 8192))
            n = n if rng.random() < 0.4 else max(1, n // 64) * 64
            # gradients in fp32 may be rounded to the layer's type
            out = rng.choice(["f32", "f16", "bf16"]) if dtype == "f32" else dtype
            c = _backward(None, round(log_between(1, 16384)), n, dtype, act, out)
        else:
            bits = rng.choice([32, 8])
            c = _adamw(None, round(log_between(1, 24)), round(log_between(1, 16384)), bs_r, bs_c, round(log_between(1, 8192)), dtype,
                       bits, dtype != "f32" and rng.random() < 0.6, rng.random() < 0.6, "f32" if rng.random() < 0.3 else dtype)
        if _cost(c) <= most:
            return c


# ------------------------------------------------------------------------------------------------ inputs
def _stored(c):
    return max(1, round(c["density"] * (c["n"] // c["bs_r"]) * (c["k"] // c["bs_c"])))


def _pattern(c, rng):
    """index_pointer and block_indices, sorted within a block-row."""
    R, C, total = c["n"] // c["bs_r"], c["k"] // c["bs_c"], _stored(c)
    if c["pattern"] == "uniform":
        at = np.sort(rng.choice(R * C, size=total, replace=False, shuffle=False))
        counts = np.bincount(at // C, minlength=R)
        idx = (at % C).astype(np.int32)
    else:                                  # blocks per block-row by a rank power law, at most all of a row
        share, rest = np.arange(1, R + 1, dtype=np.float64) ** -1.2, np.ones(R, dtype=bool)
        counts = np.zeros(R)
        while True:
            counts[rest] = (total - C * (~rest).sum()) * share[rest] / share[rest].sum()
            over = rest & (counts > C)
            if not over.any():
                break
            counts[over] = C
            rest &= ~over
        left = counts - np.floor(counts)
        counts = np.floor(counts).astype(np.int64)
        counts[np.argsort(-left, kind="stable")[: total - counts.sum()]] += 1
        counts = counts[rng.permutation(R)]
        idx = np.concatenate([np.sort(rng.permutation(C)[:v]) for v in counts]).astype(np.int32)
    ptr = np.zeros(R + 1, dtype=np.int32)
    np.cumsum(counts, out=ptr[1:])
    return ptr, idx


def _inputs(c, seed):
    """What a pass takes, made from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, scale=1.0, dtype=c["dtype"]):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).to(_TORCH[dtype])

    s = {"case": c}
    if c["op"] == "product":
        ptr, idx = _pattern(c, np.random.default_rng(seed))
        s["ptr"], s["idx"] = ptr, idx
        s["blocks"] = normal(_stored(c), c["bs_r"], c["bs_c"], scale=(c["density"] * c["k"]) ** -0.5)
        s["rows"] = torch.from_numpy(np.repeat(np.arange(len(ptr) - 1), np.diff(ptr))).cuda()
        s["cols"] = torch.from_numpy(idx.astype(np.int64)).cuda()
        s["X"] = normal(c["m"], c["k"])
        s["bias"] = normal(c["n"], scale=0.3) if c["bias"] else None
        s["residual"] = normal(c["m"], c["n"], dtype=c["out"]) if c["residual"] else None
        s["Z0"] = normal(c["m"], c["n"], dtype=c["out"]) if c["through"] else None
    elif c["op"] == "backward":
        s["G"] = normal(c["m"], c["n"])
        s["Z"] = normal(c["m"], c["n"])
    else:
        s.update(_optimizer_state(c, seed, gen))
    return s


def _layout(c):
    """(elements of a matrix, of its place, of a bias, of its place, of everything): places are whole blocks of 256, a
    buffer's matrices first and its biases behind them."""
    count = c["blocks"] * c["bs_r"] * c["bs_c"]
    up = lambda v: -(-v // _BLOCK) * _BLOCK  # noqa: E731
    return count, up(count), c["width"], up(c["width"]), c["layers"] * (up(count) + up(c["width"]))


def _optimizer_state(c, seed, gen):
    """A model somewhere in its training, its tensors one behind the other in flat buffers (zeros between them)."""
    count, place, width, vplace, total = _layout(c)
    L = c["layers"]
    blocks = total // _BLOCK
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    inside[: L * place].view(L, place)[:, :count] = True
    inside[L * place:].view(L, vplace)[:, :width] = True
    # gradients differ in size from row to row of a matrix, and a little from element to element
    size = 1e-3 * torch.exp(torch.randn((total // 16, 1), generator=gen, device="cuda")).expand(-1, 16).reshape(-1)
    rand = lambda: torch.randn(total, generator=gen, device="cuda") * inside  # noqa: E731
    s = {"grads": (rand() * size).to(_TORCH[c["out"]])}
    master = rand() * 0.02
    s["params"] = master.to(_TORCH[c["dtype"]])
    s["master"] = master if c["master"] else None
    m, v = rand() * size * 0.3, (0.3 + torch.rand(total, generator=gen, device="cuda")) * size.square() * inside
    # the tensor that each block of 256 belongs to, and its first element there
    b = torch.arange(blocks, device="cuda")
    mat = b < L * place // _BLOCK
    per = torch.where(mat, place // _BLOCK, vplace // _BLOCK)
    rel = torch.where(mat, b, b - L * place // _BLOCK)
    s["tensor"], s["first"] = torch.where(mat, 0, L) + rel // per, rel % per * _BLOCK
    s["decay"] = torch.where(mat, _DECAY, 0.0)
    s["perm"] = None
    if c["transposed"]:                    # stored block q of a transposed copy is block perm[q] of the matrix
        s["perm"] = torch.argsort(torch.rand((L, c["blocks"]), generator=gen, device="cuda"), dim=1)
        s["transposed"] = torch.zeros((L, c["blocks"], c["bs_c"], c["bs_r"]), dtype=_TORCH[c["dtype"]], device="cuda")
    if c["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], m_scale = _encode_first(m)
        s["v"], v_scale = _encode_second(v, _random(s, _STEP - 1)[0])
        s["scales"] = torch.cat([m_scale, v_scale], 1)
        s["m_value"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
        s["v_value"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
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


def _plain_product(s):
    c = s["case"]
    out = _TORCH[c["out"]]
    dense = torch.zeros((c["n"] // c["bs_r"], c["bs_r"], c["k"] // c["bs_c"], c["bs_c"]), device="cuda")
    dense.permute(0, 2, 1, 3)[s["rows"], s["cols"]] = s["blocks"].float()
    z = s["X"].float() @ dense.view(c["n"], c["k"]).t()
    if c["bias"]:
        z = z + s["bias"].float()
    y = z * _act_grad(s["Z0"].float(), c["act"]) if c["through"] else _act(z, c["act"])
    if c["residual"]:
        y = y + s["residual"].float()
    return {"Y": y.to(out), "Z": z.to(out)} if c["keep_z"] else {"Y": y.to(out)}


def _plain_backward(s):
    c = s["case"]
    dz = s["G"].float() * _act_grad(s["Z"].float(), c["act"])
    return {"dZ": dz.to(_TORCH[c["out"]]), "db": dz.sum(0, dtype=torch.float64).float()}


def _mix(x):
    """Two rounds of xor-shift and multiply, modulo 2^32."""
    x = x ^ (x >> 16)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(s, step):
    """Two numbers below 2^32 for each element: for the second moment, for the parameter."""
    key = _mix((_SEED + 0x9E3779B1 * step) & 0xFFFFFFFF)
    base = (_mix((s["tensor"] + key) & 0xFFFFFFFF) + s["first"])[:, None] + torch.arange(_BLOCK, device="cuda")
    a = _mix(base & 0xFFFFFFFF)
    return a, _mix((a + 0x3C6EF373) & 0xFFFFFFFF)


def _encode_first(m):
    """e4m3 codes (nearest-even) and a scale per block."""
    m = m.view(-1, _BLOCK)
    top = m.abs().amax(1, keepdim=True)
    scale = torch.where(top >= 2.0 ** -100, top / 448, torch.zeros_like(top))
    code = torch.where(scale > 0, m / scale, torch.zeros_like(m)).clamp(-448, 448).to(torch.float8_e4m3fn)
    return code.view(torch.uint8).view(-1), scale


def _decode_first(code, scale):
    return code.view(torch.float8_e4m3fn).float().view(-1, _BLOCK) * scale


def _encode_second(v, random):
    """Codes 1..255 are spaced evenly in log2 v from the block's smallest positive value to its largest, 0 is zero; the scales
    are log2 of the smallest and the spacing.  Between two codes the upper one is taken as often as keeps the mean."""
    v = v.view(-1, _BLOCK)
    there = v >= 2.0 ** -120
    top = v.amax(1, keepdim=True)
    low = torch.maximum(torch.where(there, v, torch.inf).amin(1, keepdim=True), top * 2.0 ** -40)
    some = there.any(1, keepdim=True)
    start = torch.where(some, torch.log2(low), 0)
    spacing = torch.where(some, ((torch.log2(top) - start) / 254).clamp_min(2.0 ** -12), 2.0 ** -12)
    at = torch.floor((torch.log2(v) - start) / spacing).clamp(0, 253)
    below = torch.exp2(start + at * spacing)
    up = (v / below - 1) / (torch.exp2(spacing) - 1)
    code = at + 1 + ((random >> 8).float() * 2.0 ** -24 < up)
    return torch.where(there, code, 0).to(torch.uint8).view(-1), torch.cat([start, spacing], 1)


def _decode_second(code, scales):
    code = code.view(-1, _BLOCK).float()
    return torch.where(code > 0, torch.exp2(scales[:, :1] + (code - 1) * scales[:, 1:]), 0)


def _round_at_random(x, random, dtype):
    """fp32 to a 16-bit type: up in size as often as keeps the mean."""
    step = torch.exp2((torch.frexp(x).exponent - 1).clamp_min(-126 if dtype == torch.bfloat16 else -14).double() - (7 if dtype == torch.bfloat16 else 10))
    bits = 16 if dtype == torch.bfloat16 else 13
    size = torch.floor(x.abs().double() / step + (random & ((1 << bits) - 1)).double() * 2.0 ** -bits) * step
    return torch.where(x < 0, -size, size).to(dtype)


def _plain_adamw(s):
    c, h = s["case"], _HYPER
    p = (s["master"] if c["master"] else s["params"]).float().view(-1, _BLOCK)
    g = s["grads"].float().view(-1, _BLOCK)
    if c["bits"] == 32:
        m, v = s["m"].view(-1, _BLOCK), s["v"].view(-1, _BLOCK)
    else:
        m, v = _decode_first(s["m"], s["scales"][:, :1]), _decode_second(s["v"], s["scales"][:, 1:])
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    p = p * (1 - h["lr"] * s["decay"][:, None])
    p = p - h["lr"] / (1 - h["beta1"] ** _STEP) * m / (v.sqrt() * (1 - h["beta2"] ** _STEP) ** -0.5 + h["eps"])
    random = _random(s, _STEP) if c["bits"] == 8 or not (c["master"] or c["dtype"] == "f32") else None
    if c["master"]:
        s["master"].copy_(p.view(-1))
    if c["dtype"] == "f32" or c["master"]:
        s["params"].copy_(p.view(-1))
    else:
        s["params"].copy_(_round_at_random(p, random[1], _TORCH[c["dtype"]]).view(-1))
    if c["bits"] == 32:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
    else:
        code, scale = _encode_first(m)
        code2, scale2 = _encode_second(v, random[0])
        s["m"].copy_(code)
        s["v"].copy_(code2)
        s["scales"].copy_(torch.cat([scale, scale2], 1))
        s["m_value"].copy_(_decode_first(code, scale).view(-1))
        s["v_value"].copy_(_decode_second(code2, scale2).view(-1))
    if c["transposed"]:
        count, place, _, _, _ = _layout(c)
        blocks = s["params"][: c["layers"] * place].view(c["layers"], place)[:, :count].reshape(c["layers"], c["blocks"], c["bs_r"], c["bs_c"])
        at = s["perm"][:, :, None, None].expand(-1, -1, c["bs_r"], c["bs_c"])
        s["transposed"].copy_(torch.gather(blocks, 1, at).transpose(2, 3))
    return _optimizer_outputs(s)


def _optimizer_outputs(s):
    """The parameters and the state as they are after the step; 8-bit moments as the values they stand for."""
    c = s["case"]
    r = {"params": s["params"]}
    if c["master"]:
        r["master"] = s["master"]
    if c["transposed"]:
        r["transposed"] = s["transposed"]
    r["m"], r["v"] = (s["m"], s["v"]) if c["bits"] == 32 else (s["m_value"], s["v_value"])
    return r


# ------------------------------------------------------------------------------------------------ the framework's
def _prepare_own(s):
    """What a user's program keeps: the matrix's handle, the optimizer's."""
    import paper_2007_13055_amd as lib
    c = s["case"]
    s["lib"] = lib
    if c["op"] == "product":
        s["W"] = lib.bsr_create(c["n"], c["k"], s["blocks"], s["idx"], s["ptr"])
    elif c["op"] == "adamw":
        count, place, width, vplace, _ = _layout(c)
        L = c["layers"]
        at = [(i * place, count) for i in range(L)] + [(L * place + i * vplace, width) for i in range(L)]

        def cut(flat, per=1):
            return [flat[a // per: -(-(a + n) // per)] for a, n in at]

        moments = list(zip(cut(s["m"]), cut(s["v"]))) if c["bits"] == 32 else list(zip(cut(s["m"]), cut(s["v"]), cut(s["scales"], _BLOCK)))
        transposed = None
        if c["transposed"]:
            perm = s["perm"].int().cpu().numpy()
            transposed = [(s["transposed"][i], perm[i]) for i in range(L)] + [None] * L
        params = [v.view(c["blocks"], c["bs_r"], c["bs_c"]) if i < L else v for i, v in enumerate(cut(s["params"]))]
        s["opt"] = lib.bsr_adamw_create(params, cut(s["grads"]), weight_decay=[_DECAY] * L + [0.0] * L, state_bits=c["bits"],
                                        moments=moments, master=cut(s["master"]) if c["master"] else None, transposed=transposed)
        s["values"] = None if c["bits"] == 32 else list(zip(cut(s["m_value"]), cut(s["v_value"])))


def _own(s):
    lib, c = s["lib"], s["case"]
    if c["op"] == "product":
        got = lib.bsr_spmm_epilogue(s["W"], s["X"], y_dtype=c["out"], bias=s["bias"], act=c["act"], residual=s["residual"],
                                    keep_z=c["keep_z"], through=s["Z0"])
        return {"Y": got[0], "Z": got[1]} if c["keep_z"] else {"Y": got}
    if c["op"] == "backward":
        dz, db = lib.bsr_epilogue_backward(s["G"], s["Z"], act=c["act"], dz_dtype=c["out"])
        return {"dZ": dz, "db": db}
    lib.bsr_adamw_step(s["opt"], _STEP, lr=_HYPER["lr"], betas=(_HYPER["beta1"], _HYPER["beta2"]), eps=_HYPER["eps"], seed=_SEED)
    if c["bits"] == 8:
        lib.bsr_adamw_moments(s["opt"], out=s["values"])
    return _optimizer_outputs(s)


def run(state):
    if own:
        return _own(state)
    return {"product": _plain_product, "backward": _plain_backward, "adamw": _plain_adamw}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ floors and exact values
def work(case):
    """Each input read once and each output written once."""
    c = case
    s_in, s_out = _SIZE[c["dtype"]], _SIZE[c["out"]]
    if c["op"] == "product":
        nnzb, R, C, block = _stored(c), c["n"] // c["bs_r"], c["k"] // c["bs_c"], c["bs_r"] * c["bs_c"]
        used_cols = C * (1.0 - (1.0 - nnzb / (R * C)) ** R)      # block-columns that hold a block, expected
        outs = 1 + c["residual"] + c["keep_z"] + c["through"]
        return {"bytes": c["m"] * used_cols * c["bs_c"] * s_in + nnzb * block * s_in + 4 * (nnzb + R + 1)
                + c["bias"] * c["n"] * s_in + outs * c["m"] * c["n"] * s_out, "flops": 2 * c["m"] * nnzb * block}
    if c["op"] == "backward":
        # without an activation dZ is G
        moved = 2 * s_in + s_out if c["act"] != "none" else s_in + (s_out if c["out"] != c["dtype"] else 0)
        return {"bytes": c["m"] * c["n"] * moved + 4 * c["n"], "flops": 8 * c["m"] * c["n"]}
    matrix, vector = c["layers"] * c["blocks"] * c["bs_r"] * c["bs_c"], c["layers"] * c["width"]
    n = matrix + vector
    each = s_out + (8 + s_in if c["master"] else 2 * s_in)
    # 8 bits: codes and three scales a block in and out, and the values that are returned
    each += 16 if c["bits"] == 32 else 4 + 24 / _BLOCK + 4
    return {"bytes": n * each + (matrix * s_in + 4 * c["layers"] * c["blocks"] if c["transposed"] else 0), "flops": 16 * n}


def exact(case, seed):
    """What run() returns, in 64 bits."""
    c, s = case, _inputs(case, seed)
    if c["op"] == "product":
        # W's elements one by one: row and column of each
        a, b = torch.arange(c["bs_r"], device="cuda"), torch.arange(c["bs_c"], device="cuda")
        row = (s["rows"] * c["bs_r"])[:, None, None] + a[None, :, None] + 0 * b
        col = (s["cols"] * c["bs_c"])[:, None, None] + 0 * a[None, :, None] + b
        w = torch.zeros(c["n"] * c["k"], dtype=torch.float64, device="cuda")
        w.index_add_(0, (row * c["k"] + col).reshape(-1), s["blocks"].double().reshape(-1))
        z = torch.mm(s["X"].double(), w.view(c["n"], c["k"]).t().contiguous())
        if s["bias"] is not None:
            z += s["bias"].double()
        value, slope = _exact_act(s["Z0"].double() if c["through"] else z, c["act"])
        y = z * slope if c["through"] else value
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return {"Y": y, "Z": z} if c["keep_z"] else {"Y": y}
    if c["op"] == "backward":
        dz = s["G"].double() * _exact_act(s["Z"].double(), c["act"])[1]
        return {"dZ": dz, "db": dz.sum(0)}
    return _exact_adamw(c, s)


def _exact_act(z, act):
    """Value and slope, from the normal distribution's integral, tanh(x) = 2 s(2x) - 1 and the logistic function s."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp_min(0), (z > 0).double()
    if act == "gelu":
        below = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * below, below + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a, b = math.sqrt(8 / math.pi), 0.044715
        share = torch.sigmoid(a * (z + b * z ** 3))
        return z * share, share + z * share * (1 - share) * a * (1 + 3 * b * z ** 2)
    share = torch.sigmoid(z)
    return z * share, share + z * share * (1 - share)


def _exact_adamw(c, s):
    L, beta1, beta2 = c["layers"], _HYPER["beta1"], _HYPER["beta2"]
    p = (s["master"] if c["master"] else s["params"]).double()
    g = s["grads"].double()
    eight = c["bits"] == 8
    if eight:
        scales = s["scales"].double().repeat_interleave(_BLOCK, 0)
        code = s["v"].double()
        m = s["m"].view(torch.float8_e4m3fn).double() * scales[:, 0]
        v = 2.0 ** (scales[:, 1] + (code - 1) * scales[:, 2]) * (code > 0)
    else:
        m, v = s["m"].double(), s["v"].double()
    m = torch.lerp(g, m, beta1)
    v = torch.lerp(g ** 2, v, beta2)
    decay = s["decay"].repeat_interleave(_BLOCK).double()
    rate = m / (1 - beta1 ** _STEP) / ((v / (1 - beta2 ** _STEP)) ** 0.5 + _HYPER["eps"])
    p = p - _HYPER["lr"] * (decay * p + rate)
    r = {"params": p}
    if c["master"]:
        r["master"] = p
    if c["transposed"]:
        count, place, _, _, _ = _layout(c)
        blocks = p[: L * place].view(L, place)[:, :count].reshape(L * c["blocks"], c["bs_r"], c["bs_c"])
        at = (s["perm"] + torch.arange(L, device="cuda")[:, None] * c["blocks"]).reshape(-1)
        r["transposed"] = blocks[at].transpose(1, 2).reshape(L, c["blocks"], c["bs_c"], c["bs_r"])
    if not eight:
        return r | {"m": m, "v": v}
    # the values that the codes stand for hang on the rounding, not on the moments alone
    return r | {"m": None, "v": None}
