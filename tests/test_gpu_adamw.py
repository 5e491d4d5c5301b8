"""bsr_adamw_*: one step over many tensors, against the formulas in 64 bits; what 8 bits hold; transposed copies; a layer's
whole training step."""
import math

import numpy as np
import pytest

import workloads as wl
from act_reference import ROUNDING, slope, value
from gpu_util import to_device, torch_dtype
from helpers import dense_expand

pytestmark = pytest.mark.gpu

H = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8)


def _f64(t):
    import torch
    return t.to(torch.float64).cpu().numpy().reshape(-1)


def _tensors(counts, dtype, grad, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda c, scale, t: (torch.randn(c, generator=gen, device="cuda") * scale).to(torch_dtype(t))  # noqa: E731
    return [new(c, 0.5, dtype) for c in counts], [new(c, 0.1, grad) for c in counts]


def _reference(p, g, m, v, t, decay, grad_scale=1.0, h=H):
    g = g * grad_scale
    b1, b2 = h["betas"]
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    step = h["lr"] / (1 - b1 ** t) * m / (np.sqrt(v) / math.sqrt(1 - b2 ** t) + h["eps"])
    return p * (1 - h["lr"] * decay) - step, m, v, np.abs(step)


COUNTS = [1, 3, 4, 255, 256, 257, 1023, 4095, 4096, 4097, 0, 20001]
KINDS = [("f32", "f32", False), ("f16", "f16", True), ("bf16", "bf16", True), ("bf16", "f32", True), ("f16", "f32", False), ("bf16", "bf16", False)]


@pytest.mark.parametrize("dtype,grad,master", KINDS)
def test_fp32_moments(dtype, grad, master):
    import torch
    import paper_2007_13055_amd as lib
    params, grads = _tensors(COUNTS, dtype, grad, 1)
    decay = [0.1 * (i % 2) for i in range(len(COUNTS))]
    opt = lib.bsr_adamw_create(params, grads, weight_decay=decay, master=True if master else None)
    # what the step starts from is what is stored: a step's error does not reach the next one's check
    for t in (1, 2, 7):
        before = [(_f64(opt.master[i] if master else params[i]), _f64(g), _f64(opt.exp_avg[i]), _f64(opt.exp_avg_sq[i])) for i, g in enumerate(grads)]
        lib.bsr_adamw_step(opt, t, grad_scale=0.5, seed=t, **H)
        for i in range(len(COUNTS)):
            p, m, v, step = _reference(*before[i], t, decay[i], 0.5)
            # a few fp32 roundings of each term; sqrt, its reciprocal and the corrections within a few 2^-23 of theirs
            assert np.all(np.abs(_f64(opt.exp_avg[i]) - m) <= 2.0 ** -22 * (np.abs(before[i][2]) + np.abs(before[i][1])) + 1e-40), (t, i)
            assert np.all(np.abs(_f64(opt.exp_avg_sq[i]) - v) <= 2.0 ** -21 * v + 1e-40), (t, i)
            close = 2.0 ** -22 * np.abs(before[i][0]) + 2.0 ** -19 * step + 2.0 ** -22 * H["lr"] * 12
            if master:
                assert np.all(np.abs(_f64(opt.master[i]) - p) <= close), (t, i)
                assert torch.equal(params[i], opt.master[i].to(params[i].dtype)), (t, i)
            elif dtype == "f32":
                assert np.all(np.abs(_f64(params[i]) - p) <= close), (t, i)
            else:                                                        # rounded at random: either neighbour
                u, tiny = ROUNDING[dtype]
                assert np.all(np.abs(_f64(params[i]) - p) <= close + 2.02 * u * np.abs(p) + 2 * tiny), (t, i)
        for g in grads:
            g.copy_(torch.randn_like(g, dtype=torch.float32) * 0.1)


def test_many_kinds_and_many_tensors_in_one_list():
    """Each tensor gets what a list of its own gives it (but for the random roundings, which know its place)."""
    import torch
    import paper_2007_13055_amd as lib
    params, grads, master = [], [], []
    for i in range(150):
        dtype, grad, has = KINDS[i % 4]
        p, g = _tensors([37 * i % 5000], dtype, grad, i)
        params += p
        grads += g
        master.append(p[0].float() if has else None)
    alone = [([p.clone()], [g], [None if m is None else m.clone()]) for p, g, m in zip(params, grads, master)]
    opt = lib.bsr_adamw_create(params, grads, master=master, weight_decay=0.01)
    for t in (1, 2):
        lib.bsr_adamw_step(opt, t, **H)
    for i, (p, g, m) in enumerate(alone):
        one = lib.bsr_adamw_create(p, g, master=m, weight_decay=0.01)
        for t in (1, 2):
            lib.bsr_adamw_step(one, t, **H)
        assert torch.equal(params[i], p[0]) and torch.equal(opt.exp_avg[i], one.exp_avg[0]) and torch.equal(opt.exp_avg_sq[i], one.exp_avg_sq[0]), i
    got = lib.bsr_adamw_moments(opt)
    assert all(torch.equal(a[0], m) and torch.equal(a[1], v) for a, m, v in zip(got, opt.exp_avg, opt.exp_avg_sq))
    got = lib.bsr_adamw_moments(opt, "bf16")
    assert all(torch.equal(a[0], m.bfloat16()) and torch.equal(a[1], v.bfloat16()) for a, m, v in zip(got, opt.exp_avg, opt.exp_avg_sq))


@pytest.mark.parametrize("dtype,grad,master", KINDS)
def test_8_bit_moments(dtype, grad, master):
    import torch
    import paper_2007_13055_amd as lib
    params, grads = _tensors(COUNTS, dtype, grad, 2)
    for g in grads:                                                      # sizes that differ by a factor of 10^4 in a group
        g.mul_(torch.exp(2 * torch.randn_like(g, dtype=torch.float32)).to(g.dtype))
    decay = [0.1] * len(COUNTS)
    opt = lib.bsr_adamw_create(params, grads, weight_decay=decay, state_bits=8, master=True if master else None)
    for t in (1, 2, 9):
        values = lib.bsr_adamw_moments(opt)
        before = [(_f64(opt.master[i] if master else params[i]), _f64(g), _f64(values[i][0]), _f64(values[i][1])) for i, g in enumerate(grads)]
        lib.bsr_adamw_step(opt, t, seed=5, **H)
        values = lib.bsr_adamw_moments(opt)
        for i, count in enumerate(COUNTS):
            p, m, v, step = _reference(*before[i], t, decay[i])
            close = 2.0 ** -22 * np.abs(before[i][0]) + 2.0 ** -19 * step + 2.0 ** -22 * H["lr"] * 12
            new = opt.master[i] if master else params[i]
            u, tiny = ROUNDING[dtype] if not master and dtype != "f32" else (0.0, 0.0)
            assert np.all(np.abs(_f64(new) - p) <= close + 2.02 * u * np.abs(p) + 2 * tiny), (t, i)
            scales = np.repeat(_f64(opt.scales[i]).reshape(-1, 3), 256, 0)[:count]
            # e4m3: half a step of 2^-3 relative, 2^-10 below 2^-6; the scale is of the largest
            assert np.all(np.abs(_f64(values[i][0]) - m) <= 1.0001 * (2.0 ** -4 * np.abs(m) + 2.0 ** -10 * scales[:, 0])), (t, i)
            held = _f64(values[i][1])
            assert np.all((held > 0) == (v > 0)), (t, i)
            ratio = held[v > 0] / np.maximum(v[v > 0], 0)
            step_up = 2.0 ** scales[v > 0, 2] * (1 + 1e-4)
            # one spacing up or down; what is below 2^-40 of its group's largest is lifted to that
            low = v[v > 0] < 2.0 ** scales[v > 0, 1] * 0.999
            assert np.all((ratio <= step_up) | low) and np.all(ratio >= 1 / step_up), (t, i)
            assert np.all(held[v > 0][low] <= 2.0 ** (scales[v > 0, 1] + scales[v > 0, 2])[low] * 1.0001), (t, i)
        for g in grads:
            g.copy_(torch.randn_like(g, dtype=torch.float32) * 0.1)


def test_8_bit_rounding_keeps_the_mean_and_repeats():
    """v of one group over many seeds: the mean of what is held is v; one seed gives the same bits again, another others."""
    import torch
    import paper_2007_13055_amd as lib
    n, seeds = 256 * 40, 300
    g = torch.exp(torch.randn(n, device="cuda") * 1.5)
    total = torch.zeros(n, dtype=torch.float64, device="cuda")
    codes = []
    for seed in range(seeds):
        opt = lib.bsr_adamw_create([torch.zeros(n, device="cuda")], [g], state_bits=8)
        lib.bsr_adamw_step(opt, 1, seed=seed, **H)
        total += lib.bsr_adamw_moments(opt)[0][1].double()
        codes.append(opt.exp_avg_sq[0].clone())
    v = 0.05 * g.double() ** 2
    off = ((total / seeds - v) / v).cpu().numpy()
    # spacings are below log2(2^27) / 254 = 0.107, so one draw is off by at most 7.7 %: half of that is a standard
    # deviation's bound, and the mean of 300 x 10240 draws is within 5 of its standard deviations
    assert np.abs(off).max() <= 6 * 0.0385 / math.sqrt(seeds)
    assert abs(off.mean()) <= 5 * 0.0385 / math.sqrt(seeds * n) + 1e-5
    opt = lib.bsr_adamw_create([torch.zeros(n, device="cuda")], [g], state_bits=8)
    lib.bsr_adamw_step(opt, 1, seed=7, **H)
    assert torch.equal(opt.exp_avg_sq[0], codes[7]) and not torch.equal(codes[7], codes[8])


def test_second_moments_do_not_stop():
    """A thousand steps with beta2 = 0.999 of gradients of one size: v comes to its mean, as rounding to nearest would not."""
    import torch
    import paper_2007_13055_amd as lib
    n = 256 * 64
    g = torch.empty(n, device="cuda")
    opt = lib.bsr_adamw_create([torch.zeros(n, device="cuda")], [g], state_bits=8)
    gen = torch.Generator(device="cuda").manual_seed(1)
    exact = torch.zeros(n, dtype=torch.float64, device="cuda")
    for t in range(1, 1001):
        g.normal_(generator=gen)
        exact.mul_(0.999).add_(g.double() ** 2, alpha=0.001)
        lib.bsr_adamw_step(opt, t, lr=0.0)
    v = lib.bsr_adamw_moments(opt)[0][1].double()
    # each step's rounding keeps the mean; a spacing of at most 10 % adds up to less than v itself over 1000 steps, and
    # 16384 elements' mean is within 5 % of the exact one's
    assert abs(float(v.mean() / exact.mean()) - 1) < 0.05


def test_16_bit_parameters_without_a_copy_keep_their_mean():
    import torch
    import paper_2007_13055_amd as lib
    for T in (torch.bfloat16, torch.float16):
        n = 65536
        p = torch.ones(n, dtype=T, device="cuda")
        g = torch.ones(n, dtype=T, device="cuda")
        opt = lib.bsr_adamw_create([p], [g])
        lr = float(torch.finfo(T).eps) / 16                               # an update of 1/8 of the step below 1 (eps / 2)
        lib.bsr_adamw_step(opt, 1, lr=lr, betas=(0.9, 0.999), eps=0.0, seed=3)
        # Bernoulli(1/8) over 65536: standard deviation 0.0013
        assert abs(float((p.double() < 1).double().mean()) - 0.125) < 0.0065, T
        assert bool(((p == 1) | (p == 1 - torch.finfo(T).eps / 2)).all())


SHAPES = [(16, 16), (32, 32), (8, 8), (64, 64), (16, 1), (1, 16), (8, 32), (64, 16), (5, 7), (128, 64), (4, 2), (1, 1)]


@pytest.mark.parametrize("dtype,bits,master", [("f32", 32, False), ("bf16", 32, True), ("f16", 8, False), ("bf16", 8, True)])
def test_transposed_copies(dtype, bits, master):
    """After a step each copy is the transpose of what the step left, bit for bit, whatever the blocks."""
    import torch
    import paper_2007_13055_amd as lib
    rng = np.random.default_rng(4)
    params, transposed = [], []
    for i, (r, c) in enumerate(SHAPES):
        nnzb = [37, 9, 300, 5, 700, 513, 64, 16, 90, 3, 2000, 4097][i]
        params.append(torch.randn((nnzb, r, c), device="cuda").to(torch_dtype(dtype)))
        copy = torch.full((nnzb, c, r), float("nan"), device="cuda").to(torch_dtype(dtype))
        transposed.append((copy, rng.permutation(nnzb).astype(np.int32)))
    params.append(torch.randn(1000, device="cuda").to(torch_dtype(dtype)))
    transposed.append(None)
    grads = [torch.randn_like(p) for p in params]
    opt = lib.bsr_adamw_create(params, grads, state_bits=bits, master=True if master else None, transposed=transposed)
    for t in (1, 2):
        lib.bsr_adamw_step(opt, t, **H)
        for (r, c), p, (copy, perm) in zip(SHAPES, params, transposed):
            assert torch.equal(copy, p[torch.from_numpy(perm).long().cuda()].transpose(1, 2).contiguous()), (r, c, t)


def test_skipped_steps_and_settings_on_the_device():
    """A step of scale 0 writes nothing; settings read on the device give the bits of the same settings from the host, and a
    captured step follows them."""
    import torch
    import paper_2007_13055_amd as lib
    make = lambda: lib.bsr_adamw_create(*_tensors([5000, 77], "bf16", "bf16", 6), state_bits=8, weight_decay=0.1)  # noqa: E731
    a, b, c = make(), make(), make()
    step, lr = torch.ones(1, dtype=torch.int64, device="cuda"), torch.full((1,), 3e-3, device="cuda")
    scale = torch.ones(1, device="cuda")
    state = lambda o: [t.clone() for t in o.params + o.exp_avg + o.exp_avg_sq + o.scales]  # noqa: E731
    same = lambda x, y: all(torch.equal(s, t) for s, t in zip(x, y))  # noqa: E731
    begin = state(a)
    lib.bsr_adamw_step(a, 1, lr=3e-3, grad_scale=0.0)
    scale.zero_()
    lib.bsr_adamw_step(b, step, lr=lr, grad_scale=scale)
    assert same(begin, state(a)) and same(begin, state(b))
    scale.fill_(0.25)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.bsr_adamw_step(c, step, lr=lr, grad_scale=scale, seed=9)
    for t in range(1, 6):
        step.fill_(t)
        lr.fill_(3e-3 / t)
        lib.bsr_adamw_step(a, t, lr=float(np.float32(3e-3 / t)), grad_scale=0.25, seed=9)
        lib.bsr_adamw_step(b, step, lr=lr, grad_scale=scale, seed=9)
        graph.replay()
        torch.cuda.synchronize()
        assert same(state(b), state(c)), t
        for x, y in zip(a.params, b.params):
            # the corrections' powers are fp32 on the device: a rounding may fall the other way, by one place of a parameter
            # or by a code of a moment, a tenth of an update of a few times the rate
            assert bool(((x.float() - y.float()).abs() <= 2.0 ** -7 * x.float().abs() + 2e-3).all()), t
        for o in (a, b, c):
            for g in o.grads:
                g.copy_(torch.randn(g.shape, generator=torch.Generator(device="cuda").manual_seed(t), device="cuda") * 0.1)


def test_on_another_stream():
    import torch
    import paper_2007_13055_amd as lib
    params, grads = _tensors([70000], "f32", "f32", 8)
    want, _ = _tensors([70000], "f32", "f32", 8)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    opt = lib.bsr_adamw_create(params, grads)                              # its upload is on the current stream
    with torch.cuda.stream(side):
        lib.bsr_adamw_step(opt, 1, **H)
    torch.cuda.synchronize()
    one = lib.bsr_adamw_create(want, grads)
    lib.bsr_adamw_step(one, 1, **H)
    assert torch.equal(params[0], want[0])


def test_refusals():
    import torch
    import paper_2007_13055_amd as lib
    f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    p, g = f(100), f(100)
    blocks = f(4, 8, 8)
    turned = lambda perm, copy=None: [(f(4, 8, 8) if copy is None else copy, np.array(perm))]  # noqa: E731
    wide = f(204)
    for args, kw, error in [(([p], []), {}, ValueError), (([p], [g[:99]]), {}, ValueError), (([p], [g.half()]), {}, ValueError),
                            (([p.cpu()], [g]), {}, ValueError), (([p[::2]], [g[:50]]), {}, ValueError), (([p.double()], [g]), {}, ValueError),
                            (([p], [g]), dict(state_bits=16), ValueError), (([p], [g]), dict(master=[f(100)]), lib.BsrError),
                            (([p], [g]), dict(moments=[(f(100),)]), ValueError), (([p], [g]), dict(moments=[(f(100), f(100))], state_bits=8), ValueError),
                            (([p], [g]), dict(weight_decay=[0.1, 0.2]), ValueError), (([p, p], [g, g]), {}, lib.BsrError),
                            (([p], [p]), {}, lib.BsrError), (([wide[:100], wide[96:196]], [g, g]), {}, lib.BsrError),
                            (([wide[1:101]], [g]), {}, lib.BsrError), (([p], [g]), dict(transposed=turned([0])), ValueError),
                            (([blocks], [f(4, 8, 8)]), dict(transposed=turned([0, 1, 2, 2])), lib.BsrError),
                            (([blocks], [f(4, 8, 8)]), dict(transposed=turned([0, 1, 2, 4])), lib.BsrError),
                            (([blocks], [f(4, 8, 8)]), dict(transposed=turned([0, 1, 2, 3], f(4, 8, 4))), ValueError),
                            (([blocks], [f(4, 8, 8)]), dict(transposed=turned([0, 1, 2, 3], blocks)), lib.BsrError),
                            (([f(1, 201, 201)], [f(1, 201, 201)]), dict(transposed=turned([0], f(1, 201, 201))), lib.BsrError)]:
        with pytest.raises(error):
            lib.bsr_adamw_create(*args, **kw)
    opt = lib.bsr_adamw_create([p], [g])
    for kw, error in [(dict(step=0), lib.BsrError), (dict(step=1, betas=(1.0, 0.9)), lib.BsrError), (dict(step=1, betas=(0.9, -0.1)), lib.BsrError),
                      (dict(step=1, eps=-1.0), lib.BsrError), (dict(step=1, lr=float("nan")), lib.BsrError),
                      (dict(step=1, grad_scale=float("nan")), lib.BsrError), (dict(step=torch.ones(1, device="cuda")), ValueError),
                      (dict(step=torch.ones(1, dtype=torch.int64)), ValueError), (dict(step=1, lr=f(2)), ValueError)]:
        with pytest.raises(error):
            lib.bsr_adamw_step(opt, **kw)
    with pytest.raises(ValueError):
        lib.bsr_adamw_moments(opt, out=[(f(100), f(99))])
    assert bool((p == 0).all())
    opt.close()
    with pytest.raises(lib.BsrError):
        lib.bsr_adamw_step(opt, 1)
    empty = lib.bsr_adamw_create([], [])
    lib.bsr_adamw_step(empty, 1)
    assert lib.bsr_adamw_moments(empty) == []


@pytest.mark.parametrize("dtype,bits", [("f32", 32), ("bf16", 32), ("bf16", 8)])
def test_training_steps_of_two_layers(dtype, bits):
    """Y = W2 gelu(W1 X + b1) + b2 + X against a target: product, its gradient, the stored blocks' and the step, three times
    over, as a training loop has them; everything that a step changes against 64 bits."""
    import torch
    import paper_2007_13055_amd as lib
    m, d, hidden, b = 200, 128, 256, 16
    T, master = torch_dtype(dtype), dtype != "f32"
    up = wl.make_problem("up", m, d, hidden, b, b, dtype, dtype, ("bernoulli", 0.4), ("normal", 1.0), ("normal", 0.2), 1)
    down = wl.make_problem("down", m, hidden, d, b, b, dtype, dtype, ("bernoulli", 0.4), ("normal", 1.0), ("normal", 0.2), 2)
    X, target = to_device(up.X, dtype), torch.randn((m, d), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(T)
    layers = []
    for p in (up, down):
        W = lib.bsr_create(p.n, p.k, p.block_data, p.block_indices, p.index_pointer, dtype=dtype)
        WT = lib.bsr_create_transposed(p.n, p.k, p.block_data, p.block_indices, p.index_pointer, dtype=dtype)
        perm = lib.bsr_transpose_pattern(p.n, p.k, b, b, p.index_pointer, p.block_indices)[2]
        layers.append((p, W, WT, perm, torch.zeros(p.n, dtype=T, device="cuda")))
    (p1, W1, WT1, perm1, b1), (p2, W2, WT2, perm2, b2) = layers
    params = [W1.block_data, W2.block_data, b1, b2]
    grads = [torch.empty_like(W1.block_data), torch.empty_like(W2.block_data), torch.empty(hidden, device="cuda"), torch.empty(d, device="cuda")]
    opt = lib.bsr_adamw_create(params, grads, weight_decay=[0.1, 0.1, 0.0, 0.0], state_bits=bits, master=True if master else None,
                               transposed=[(WT1, perm1), (WT2, perm2), None, None])
    u = ROUNDING[dtype][0]
    for t in (1, 2, 3):
        before = [(_f64(opt.master[i] if master else q), _f64(a), _f64(v)) for i, (q, (a, v)) in enumerate(zip(params, lib.bsr_adamw_moments(opt)))]
        dense = [dense_expand(_f64(W.block_data).reshape(p.block_data.shape), p.block_indices, p.index_pointer, p.n, p.k) for p, W, *_ in layers]
        bias = [_f64(v) for v in (b1, b2)]
        hid, z = lib.bsr_spmm_epilogue(W1, X, bias=b1, act="gelu", keep_z=True)
        Y = lib.bsr_spmm_epilogue(W2, hid, bias=b2, residual=X)
        G = ((Y.float() - target.float()) / m).to(T)
        lib.bsr_epilogue_backward(G, need_dz=False, DB=grads[3])
        lib.bsr_sddmm(W2, G, hid, grads[1])
        dz = lib.bsr_spmm_epilogue(WT2, G, act="gelu", through=z)
        lib.bsr_epilogue_backward(dz, need_dz=False, DB=grads[2])
        lib.bsr_sddmm(W1, dz, X, grads[0])
        lib.bsr_adamw_step(opt, t, seed=1, **H)
        # the chain in 64 bits
        x = _f64(X).reshape(m, d)
        z64 = x @ dense[0].T + bias[0]
        h64 = value(z64, "gelu")
        g64 = (h64 @ dense[1].T + bias[1] + x - _f64(target).reshape(m, d)) / m
        dz64 = (g64 @ dense[1]) * slope(z64, "gelu")
        full = [dz64.T @ x, g64.T @ h64]
        for (p, W, *_), got, want, left, right in zip(layers, grads[:2], full, (dz64, g64), (x, h64)):
            rows = np.repeat(np.arange(p.n // b), np.diff(p.index_pointer))
            sizes = np.abs(left).T @ np.abs(right)
            got = _f64(got).reshape(-1, b, b)
            for q in range(len(rows)):
                a, c = slice(rows[q] * b, (rows[q] + 1) * b), slice(p.block_indices[q] * b, (p.block_indices[q] + 1) * b)
                # every factor has been rounded a few times on its way: 16 u of the sum of sizes, widened by the chain's own sums
                assert np.all(np.abs(got[q] - want[a, c]) <= 16 * (u + 1e-5) * (sizes[a, c] + sizes.mean())), (t, q)
        for i, g in enumerate((None, None, dz64.sum(0), g64.sum(0))):
            if g is not None:
                size = np.abs((dz64 if i == 2 else g64)).sum(0)
                assert np.all(np.abs(_f64(grads[i]) - g) <= 16 * (u + 1e-5) * (size + size.mean())), (t, i)
        for i, q in enumerate(params):                                    # the step itself, from the gradients that it was given
            want, _, _, step = _reference(before[i][0], _f64(grads[i]), before[i][1], before[i][2], t, (0.1, 0.1, 0, 0)[i])
            new = _f64(opt.master[i] if master else q)
            assert np.all(np.abs(new - want) <= 2.0 ** -22 * np.abs(before[i][0]) + 2.0 ** -19 * step + 2.0 ** -22 * H["lr"] * 12), (t, i)
        for p, W, WT, perm, _ in layers:
            assert torch.equal(WT.block_data, W.block_data[torch.from_numpy(perm).long().cuda()].transpose(1, 2).contiguous())


def test_captured_right_behind_the_handle():
    """No eager step before: the tables' upload is waited for during the capture."""
    import torch
    import paper_2007_13055_amd as lib
    params, grads = _tensors([300000, 5, 9000], "bf16", "bf16", 12)
    want, _ = _tensors([300000, 5, 9000], "bf16", "bf16", 12)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2000000)                                        # the upload comes behind it
        opt = lib.bsr_adamw_create(params, grads, master=True)
    with torch.cuda.graph(graph):
        lib.bsr_adamw_step(opt, 1, **H)
    graph.replay()
    torch.cuda.synchronize()
    one = lib.bsr_adamw_create(want, grads, master=True)
    lib.bsr_adamw_step(one, 1, **H)
    for a, b in zip(opt.params + opt.exp_avg + opt.master, one.params + one.exp_avg + one.master):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_that_are_not_finite(bits):
    """They reach their own element and, held in 8 bits, the moments of its 256; nothing else."""
    import torch
    import paper_2007_13055_amd as lib
    for bad in (float("nan"), float("inf"), -float("inf")):
        params, grads = _tensors([1000], "f32", "f32", 13)
        clean, _ = _tensors([1000], "f32", "f32", 13)
        spoilt = grads[0].clone()
        spoilt[300] = bad
        opt = lib.bsr_adamw_create(params, [spoilt], state_bits=bits)
        one = lib.bsr_adamw_create(clean, grads, state_bits=bits)
        for o in (opt, one):
            lib.bsr_adamw_step(o, 1, **H)
        assert not bool(params[0][300].isfinite())
        rest = torch.arange(1000, device="cuda") != 300
        assert torch.equal(params[0][rest], clean[0][rest])
        m, v = lib.bsr_adamw_moments(opt)[0]
        m1, v1 = lib.bsr_adamw_moments(one)[0]
        group = (torch.arange(1000, device="cuda") // 256 == 1) if bits == 8 else ~rest
        assert torch.equal(m[~group], m1[~group]) and torch.equal(v[~group], v1[~group])
        assert not bool(v[group].isfinite().any()) and not bool(m[300].isfinite())


def test_all_of_a_groups_gradients_are_zero():
    """Groups without a positive value, and ones with a single one: zeros stay zeros, and the one keeps its value."""
    import torch
    import paper_2007_13055_amd as lib
    g = torch.zeros(1024, device="cuda")
    g[300], g[600], g[601] = 2.0, 1e-12, 3e4
    p = torch.ones(1024, device="cuda")
    opt = lib.bsr_adamw_create([p], [g], state_bits=8, weight_decay=0.0)
    for t in (1, 2, 3):
        lib.bsr_adamw_step(opt, t, **H)
    m, v = lib.bsr_adamw_moments(opt)[0]
    assert bool((v[g == 0] == 0).all()) and bool((m[g == 0] == 0).all()) and bool((p[g == 0] == 1).all())
    want = 1 - 0.95 ** 3
    assert abs(float(v[300]) / (want * 4) - 1) < 3 * 2.0 ** -11           # spacing 2^-12 in log2, up or down a few times
    # 3e4 squared is the largest of its group; 1e-12 squared is below 2^-40 of it and is held as that, so its update shrinks
    assert abs(float(v[601]) / (want * 9e8) - 1) < 0.4 and float(v[600]) > 0 and abs(float(p[600]) - 1) < 1e-3
    assert abs(float(p[601]) - (1 - 3 * H["lr"])) < 1e-4


@pytest.mark.parametrize("dtype,grad,master", [("f32", "f32", False), ("bf16", "bf16", True)])
def test_8_bit_codes_are_those_of_plain_arithmetic(dtype, grad, master):
    """First moments code by code as fp32 arithmetic that rounds each operation gives them; second moments within a code of
    their value."""
    import torch
    import paper_2007_13055_amd as lib
    count = 256 * 4000
    params, grads = _tensors([count], dtype, grad, 21)
    opt = lib.bsr_adamw_create(params, grads, state_bits=8, master=True if master else None)
    f32 = torch.float32
    b1, c1, b2, c2 = (torch.tensor(v, dtype=torch.float64, device="cuda").to(f32) for v in (0.9, 1 - 0.9, 0.95, 1 - 0.95))
    for t in (1, 2, 3):
        codes, scales = opt.exp_avg[0].clone(), opt.scales[0].clone()
        v_codes = opt.exp_avg_sq[0].clone().view(-1, 256).float()
        lib.bsr_adamw_step(opt, t, seed=3, **H)
        g = grads[0].float().view(-1, 256)
        m = codes.view(torch.float8_e4m3fn).float().view(-1, 256) * scales[:, :1]
        m = torch.add(torch.mul(m, b1), torch.mul(g, c1))
        scale = m.abs().amax(1, keepdim=True) * torch.tensor(1 / 448, dtype=torch.float64, device="cuda").to(f32)
        assert torch.equal(opt.scales[0][:, :1], scale), t
        want = (m / scale).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        assert torch.equal(opt.exp_avg[0].view(-1, 256), want), t
        # v before its rounding, in 64 bits: the code lies within one step of it
        v = torch.where(v_codes > 0, torch.exp2(scales[:, 1:2].double() + (v_codes.double() - 1) * scales[:, 2:].double()), 0.0)
        v = 0.95 * v + 0.05 * g.double() ** 2
        now = opt.scales[0].double()
        at = ((torch.log2(v) - now[:, 1:2]) / now[:, 2:] + 1).clamp_min(1)    # (below 2^-40 of the largest: the first code)
        # fp32: an argument of some 30 rounded to 2^-19, a step of the codes is at least 2^-6 of it in log2 v here
        off = (opt.exp_avg_sq[0].view(-1, 256).double() - at)[v > 2.0 ** -100]
        assert float(off.abs().max()) < 1 + 2.0 ** -10, t
