"""bsr_muon_*: steps whose updates are orthogonalised block by block, against the formulas in 64 bits."""
import math

import numpy as np
import pytest

from act_reference import ROUNDING
from gpu_util import torch_dtype

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315
KINDS = [("f32", "f32", False), ("f16", "f16", True), ("bf16", "bf16", True), ("bf16", "f32", True), ("f16", "f32", False), ("bf16", "bf16", False)]
SHAPES = [(16, 16), (32, 32), (64, 64), (8, 8), (1, 1), (16, 1), (1, 16), (5, 7), (16, 32), (64, 16), (24, 40), (48, 16), (64, 48), (33, 64), (3, 61)]


def _f64(t):
    import torch
    return t.to(torch.float64).cpu().numpy()


def _orthogonal(v, T, steps=5, eps=1e-7, abc=(A, B, C)):
    """The update in T's arithmetic (products by T's matmul)."""
    v = v.astype(T)
    a, b, c = (T(x) for x in abc)
    x = v / (np.sqrt((v * v).sum((1, 2), keepdims=True, dtype=T)) + T(eps))
    tall = v.shape[1] > v.shape[2]
    x = x.transpose(0, 2, 1) if tall else x
    for _ in range(steps):
        g = x @ x.transpose(0, 2, 1)
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.transpose(0, 2, 1) if tall else x


def _check_update(got, v, what, **kw):
    """As exact as the same formulas in plain fp32 arithmetic: root mean square error within 3 times theirs, largest within 8
    (sums of the same terms in another order; what small singular values make of roundings is in both)."""
    want = _orthogonal(v, np.float64, **kw)
    plain = _orthogonal(v, np.float32, **kw)
    floor = 2.0 ** -22                                                   # a few roundings of an element, whose size is below 1.3
    err, ref = np.abs(got - want), np.abs(plain - want)
    assert np.sqrt((err ** 2).mean()) <= 3 * np.sqrt((ref ** 2).mean()) + floor, (what, err.max(), ref.max())
    assert err.max() <= 8 * ref.max() + floor, (what, err.max(), ref.max())


def _make(counts, shape, dtype, grad, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    params = [(rand(c, *shape) * 0.5).to(torch_dtype(dtype)) for c in counts]
    grads = [((rand(c, *shape) + 2 * rand(c, shape[0], 1) * rand(c, 1, shape[1])) * 0.1).to(torch_dtype(grad)) for c in counts]
    momentum = [rand(c, *shape) * 0.3 for c in counts]
    return params, grads, momentum


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("nesterov", [True, False])
def test_update(shape, nesterov):
    """p = 0, no decay, lr = scale = 1: the parameter is the update."""
    import torch
    import paper_2007_13055_amd as lib
    params, grads, momentum = _make([1, 2, 9], shape, "f32", "f32", 1)
    for p in params:
        p.zero_()
    before = [_f64(m) for m in momentum]
    opt = lib.bsr_muon_create(params, grads, momentum=momentum, scale=1.0)
    lib.bsr_muon_step(opt, 1, lr=1.0, momentum=0.9, nesterov=nesterov, grad_scale=0.5)
    for p, g, m, m0 in zip(params, grads, opt.momentum, before):
        assert m is not None
        g = 0.5 * _f64(g)
        want = 0.9 * m0 + g
        assert np.all(np.abs(_f64(m) - want) <= 2.0 ** -24 * (3 * np.abs(want) + 2 * np.abs(m0) + 2 * np.abs(g)))   # 0.9 in fp32, two roundings
        held = _f64(m)
        _check_update(-_f64(p), (g + 0.9 * held if nesterov else held), shape)
        if nesterov is False and min(shape) > 1:
            s = np.linalg.svd(_f64(p), compute_uv=False)
            assert s.max() < 1.3


@pytest.mark.parametrize("dtype,grad,master", KINDS)
@pytest.mark.parametrize("shape", [(16, 16), (8, 8), (32, 16), (5, 7), (64, 64)])
def test_kinds(dtype, grad, master, shape):
    import torch
    import paper_2007_13055_amd as lib
    counts = [1, 7, 0, 130]
    params, grads, momentum = _make(counts, shape, dtype, grad, 2)
    decay, scale = [0.1, 0.0, 0.1, 0.3], [1.0, 0.5, 1.0, 2.0]
    opt = lib.bsr_muon_create(params, grads, momentum=momentum, weight_decay=decay, scale=scale, master=True if master else None)
    lr = 0.02
    for t in (1, 2):
        before = [_f64(opt.master[i] if master else p) for i, p in enumerate(params)]
        lib.bsr_muon_step(opt, t, lr=lr, momentum=0.95, seed=t)
        for i, p in enumerate(params):
            if counts[i] == 0:
                continue
            v = _f64(grads[i]) + 0.95 * _f64(opt.momentum[i])
            step = lr * scale[i] * _orthogonal(v, np.float64)
            ref = lr * scale[i] * np.abs(_orthogonal(v, np.float32) - _orthogonal(v, np.float64)).max()
            want = before[i] * (1 - lr * decay[i]) - step
            close = 8 * ref + lr * scale[i] * 2.0 ** -22 + 2.0 ** -22 * (np.abs(before[i]) + np.abs(step))   # as above, and the sum's roundings
            got = _f64(opt.master[i] if master else p)
            u, tiny = ROUNDING["f32" if master else dtype]
            if not master and dtype != "f32":                            # rounded at random: either neighbour
                u, tiny = 2.02 * u, 2 * tiny
            assert np.all(np.abs(got - want) <= close + u * np.abs(want) + tiny), (t, i)
            if master:
                assert torch.equal(p, opt.master[i].to(p.dtype))
        for g in grads:
            g.copy_(torch.randn_like(g, dtype=torch.float32) * 0.1)


def test_random_rounding_keeps_the_mean():
    """4096 equal elements a place: the mean of what they are rounded to is the unrounded value within 5 standard errors."""
    import torch
    import paper_2007_13055_amd as lib
    for T in (torch.bfloat16, torch.float16):
        p = torch.full((4096, 16, 16), 1.0, device="cuda").to(T)
        g = torch.ones((4096, 16, 16), device="cuda").to(T)
        opt = lib.bsr_muon_create([p], [g])
        lib.bsr_muon_step(opt, 1, lr=1e-3, ns_steps=0)
        want = 1 - 1e-3 / 16                                             # g / |g| = 1 / 16
        gap = 2.0 ** -8 if T == torch.bfloat16 else 2.0 ** -11           # steps below 1
        assert abs(float(p.double().mean()) - want) <= 5 * gap / 2 / math.sqrt(p.numel()) + 1e-7
        assert set(p.unique().double().tolist()) <= {1.0, 1.0 - gap}


@pytest.mark.parametrize("shape", [(16, 16), (8, 8), (64, 32), (16, 1), (5, 7), (16, 64)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_transposed(shape, dtype):
    import torch
    import paper_2007_13055_amd as lib
    params, grads, _ = _make([50, 3], shape, dtype, dtype, 3)
    rng = np.random.default_rng(1)
    perms = [rng.permutation(50), rng.permutation(3)]
    turned = [torch.full((c, shape[1], shape[0]), 7.0, device="cuda").to(torch_dtype(dtype)) for c in (50, 3)]
    opt = lib.bsr_muon_create(params, grads, master=True if dtype != "f32" else None, transposed=list(zip(turned, perms)))
    lib.bsr_muon_step(opt, 1)
    for p, t, perm in zip(params, turned, perms):
        assert torch.equal(t, p[torch.from_numpy(perm).cuda()].transpose(1, 2))


def test_many_shapes_in_one_list():
    """Each tensor gets what a list of its own gives it."""
    import torch
    import paper_2007_13055_amd as lib
    params, grads, master = [], [], []
    for i, shape in enumerate(SHAPES * 2):
        dtype, grad, has = KINDS[i % 4]
        p, g, _ = _make([1 + 13 * i % 40], shape, dtype, grad, i)
        params += p
        grads += g
        master.append(p[0].float() if has else None)
    ones = [lib.bsr_muon_create([p.clone()], [g], master=[m.clone()] if m is not None else None, weight_decay=0.1) for p, g, m in zip(params, grads, master)]
    opt = lib.bsr_muon_create(params, grads, master=master, weight_decay=0.1)
    for t in (1, 2):
        lib.bsr_muon_step(opt, t)
        for one in ones:
            lib.bsr_muon_step(one, t)
    assert all(torch.equal(p, one.params[0]) for p, one in zip(params, ones))
    assert all(torch.equal(m, one.momentum[0]) for m, one in zip(opt.momentum, ones))


def test_zero_and_small_and_large():
    """Zeros give no update; sizes far below and above 1 give the update of their direction (eps apart)."""
    import torch
    import paper_2007_13055_amd as lib
    g = torch.randn((3, 32, 32), device="cuda")
    g[0] = 0
    p = torch.zeros_like(g)
    lib.bsr_muon_step(lib.bsr_muon_create([p], [g], scale=1.0), 1, lr=1.0, eps=2.0 ** -60)
    assert bool((p[0] == 0).all())
    for size in (2.0 ** -30, 2.0 ** 60, 2.0 ** 80):
        q = torch.zeros_like(g)
        lib.bsr_muon_step(lib.bsr_muon_create([q], [g * size], scale=1.0), 1, lr=1.0, eps=2.0 ** -60)
        assert float((q - p).abs().max()) <= 1e-4                        # powers of two: the same numbers but for eps / |V| = 2^-35
    tiny = torch.zeros_like(g)
    lib.bsr_muon_step(lib.bsr_muon_create([tiny], [g * 1e-25], scale=1.0), 1, lr=1.0, eps=1e-7)
    assert float(tiny.abs().max()) < 1e-12                               # far below eps


def test_not_finite_stays_in_its_block():
    import torch
    import paper_2007_13055_amd as lib
    for shape in ((16, 16), (64, 64), (8, 8)):
        params, grads, _ = _make([9], shape, "f32", "f32", 5)
        clean, g = params[0].clone(), grads[0].clone()
        lib.bsr_muon_step(lib.bsr_muon_create([clean], [g.clone()]), 1)
        g[4, 1, 2], g[7, 0, 0] = float("nan"), float("inf")
        lib.bsr_muon_step(lib.bsr_muon_create(params, [g]), 1)
        rest = [0, 1, 2, 3, 5, 6, 8]
        assert torch.equal(params[0][rest], clean[rest]) and bool(params[0][4].isnan().all()) and bool(params[0][7].isnan().any())


def test_skipped_steps_and_settings_on_the_device():
    import torch
    import paper_2007_13055_amd as lib
    params, grads, _ = _make([20], (16, 16), "bf16", "bf16", 6)
    p0, twin = params[0].clone(), params[0].clone()
    opt, one = lib.bsr_muon_create(params, grads), lib.bsr_muon_create([twin], grads)
    number, lr, scale = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), 0.01, device="cuda"), torch.ones(1, device="cuda")
    lib.bsr_muon_step(opt, number, lr=lr, grad_scale=scale)              # no step 0
    lib.bsr_muon_step(opt, 1, grad_scale=0.0)
    scale.zero_()
    lib.bsr_muon_step(opt, 1, grad_scale=scale)
    assert torch.equal(params[0], p0) and bool((opt.momentum[0] == 0).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.bsr_muon_step(opt, number, lr=lr, grad_scale=scale, seed=3)
    for t in range(1, 5):
        number.fill_(t)
        lr.fill_(0.01 * t)
        scale.fill_(2.0)
        graph.replay()
        torch.cuda.synchronize()
        lib.bsr_muon_step(one, t, lr=float(np.float32(0.01 * t)), grad_scale=2.0, seed=3)
        assert torch.equal(params[0], twin) and torch.equal(opt.momentum[0], one.momentum[0]), t


@pytest.mark.parametrize("steps", [0, 1, 3, 16])
def test_other_settings(steps):
    import torch
    import paper_2007_13055_amd as lib
    _, grads, _ = _make([11], (32, 48), "f32", "f32", 7)
    p = torch.zeros((11, 32, 48), device="cuda")
    abc = (1.875, -1.25, 0.375)                                          # singular values to 1 exactly, in more steps
    lib.bsr_muon_step(lib.bsr_muon_create([p], grads, scale=1.0), 1, lr=1.0, momentum=0.0, ns_steps=steps, coefficients=abc, eps=1e-6)
    _check_update(-_f64(p), _f64(grads[0]), steps, steps=steps, eps=1e-6, abc=abc)


@pytest.mark.parametrize("shape", [(16, 16), (64, 64), (8, 8), (5, 7), (33, 64), (64, 16)])
@pytest.mark.parametrize("abc,steps", [((1.9, 0.0, 0.0), 2), ((1.0, 2.8, 0.0), 1), ((0.9, 0.0, 2.9), 1), ((0.0, 0.0, 0.0), 2), ((-1.5, 0.5, 1e-30), 5),   # |X| below 3.9
                                       ((6.0, -1.0, 0.0), 2), ((1.0, 0.0, 3.0), 2), ((2.0, 3.0, 0.0), 3), ((1.0, -4e4, 4e4), 1), ((1e9, 0.0, 0.0), 2)])
def test_coefficients(shape, abc, steps):
    """Steps that keep X small and steps that do not (whose products cannot be of fp16 parts); first singular values near 1."""
    import torch
    import paper_2007_13055_amd as lib
    gen = torch.Generator(device="cuda").manual_seed(9)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    g = rand(9, *shape) * 0.05 + 2 * rand(9, shape[0], 1) * rand(9, 1, shape[1])
    p = torch.zeros_like(g)
    lib.bsr_muon_step(lib.bsr_muon_create([p], [g], scale=1.0), 1, lr=1.0, momentum=0.0, ns_steps=steps, coefficients=abc, eps=1e-6)
    want = _orthogonal(_f64(g), np.float64, steps=steps, eps=1e-6, abc=abc)
    size = max(1.0, float(np.abs(want).max()))                           # the floor's sizes are those of updates below 1.3
    got, plain = -_f64(p), _orthogonal(_f64(g), np.float32, steps=steps, eps=1e-6, abc=abc)
    err, ref = np.abs(got - want), np.abs(plain - want)
    assert np.sqrt((err ** 2).mean()) <= 3 * np.sqrt((ref ** 2).mean()) + 2.0 ** -22 * size, (err.max(), ref.max())
    assert err.max() <= 8 * ref.max() + 2.0 ** -22 * size, (err.max(), ref.max())


@pytest.mark.parametrize("shape", [(16, 16), (64, 64), (32, 48)])
def test_steps_that_shrink(shape):
    """X = X X^T X twice: numbers far below 1 keep their relative accuracy (27 roundings' worth and as many of the sums')."""
    import torch
    import paper_2007_13055_amd as lib
    g = torch.randn((5, *shape), generator=torch.Generator(device="cuda").manual_seed(11), device="cuda")
    p = torch.zeros_like(g)
    abc = (0.0, 1.0, 0.0)
    lib.bsr_muon_step(lib.bsr_muon_create([p], [g], scale=1.0), 1, lr=1.0, momentum=0.0, ns_steps=2, coefficients=abc, eps=1e-6)
    want, plain = (_orthogonal(_f64(g), T, steps=2, eps=1e-6, abc=abc) for T in (np.float64, np.float32))
    err, ref = np.abs(-_f64(p) - want), np.abs(plain - want)
    assert np.abs(want).max() < 2.0 ** -8
    assert err.max() <= 8 * ref.max() + 2.0 ** -19 * np.abs(want).max(), (err.max(), ref.max())


@pytest.mark.parametrize("count", [1, 5, 1100])
@pytest.mark.parametrize("shape", [(48, 48), (64, 64), (41, 50), (64, 48), (48, 61)])
def test_large_blocks_few_and_many(shape, count):
    """A workgroup a block up to 1024 of them, a wavefront a block beyond."""
    import torch
    import paper_2007_13055_amd as lib
    params, grads, momentum = _make([count], shape, "f32", "f32", 10)
    params[0].zero_()
    held = _f64(momentum[0])
    perm = np.random.default_rng(2).permutation(count)
    turned = torch.full((count, shape[1], shape[0]), 7.0, device="cuda")
    opt = lib.bsr_muon_create(params, grads, momentum=momentum, scale=1.0, transposed=[(turned, perm)])
    lib.bsr_muon_step(opt, 1, lr=1.0, momentum=0.9)
    now = _f64(opt.momentum[0]).reshape(held.shape)
    g = _f64(grads[0])
    want = g + 0.9 * held
    assert np.all(np.abs(now - want) <= 2.0 ** -24 * (3 * np.abs(want) + 2 * np.abs(held) + 2 * np.abs(g)))
    _check_update(-_f64(params[0]), g + 0.9 * now, shape)
    assert torch.equal(turned, params[0][torch.from_numpy(perm).cuda()].transpose(1, 2))


def test_dropped_while_a_step_on_another_stream_is_still_to_run():
    """Its tables, momentum and master copies are no one else's before that step is done."""
    import torch
    import paper_2007_13055_amd as lib
    params, grads, _ = _make([500, 30], (16, 16), "bf16", "bf16", 8)
    twin = [p.clone() for p in params]
    one, opt = lib.bsr_muon_create(twin, grads, master=True), lib.bsr_muon_create(params, grads, master=True)
    for o in (one, opt):
        lib.bsr_muon_step(o, 1)
    room = [torch.empty(500 * 1024, dtype=torch.uint8, device="cuda") for _ in range(24)]
    del room
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)                                    # a tenth of a second and more
        lib.bsr_muon_step(opt, 2)
    own = [t for t in opt._keep if isinstance(t, torch.Tensor)] + opt.momentum + opt.master
    sizes, held = [(t.numel(), t.dtype) for t in own], [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in own]
    del opt, own, o
    new = [torch.empty(n, dtype=t, device="cuda") for n, t in sizes for _ in range(2)]   # (not written to)
    still_to_run = not side.query()
    taken = [a for a in new for b in held if a.data_ptr() < b[1] and b[0] < a.data_ptr() + a.numel() * a.element_size()]
    torch.cuda.synchronize()
    assert still_to_run and not taken
    lib.bsr_muon_step(one, 2)
    assert all(torch.equal(p, q) for p, q in zip(params, twin))


def test_refusals():
    import torch
    import paper_2007_13055_amd as lib
    p = torch.zeros((4, 16, 16), device="cuda")
    for args, kw in (([[p], []], {}), ([[p.view(-1)], [p.clone()]], {}), ([[p], [p.clone().half()]], {}), ([[p], [p.clone()[:2]]], {}), ([[p.cpu()], [p.clone()]], {}),
                     ([[p], [p.clone()]], dict(momentum=[p.clone().half()])), ([[p], [p.clone()]], dict(weight_decay=[0.1, 0.2])),
                     ([[p], [p.clone()]], dict(transposed=[(p.clone(), [0, 1])])), ([[p], [p.clone()]], dict(scale=[1.0, 2.0]))):
        with pytest.raises(ValueError):
            lib.bsr_muon_create(*args, **kw)
    wide = torch.zeros((2, 65, 16), device="cuda")
    for args, kw in (([[p], [p]], {}), ([[wide], [wide.clone()]], {}), ([[p, p], [p.clone(), p.clone()]], {}), ([[p], [p.clone()]], dict(transposed=[(p.clone(), [0, 1, 1, 2])]))):
        with pytest.raises(lib.BsrError):
            lib.bsr_muon_create(*args, **kw)
    opt = lib.bsr_muon_create([p], [p.clone()])
    for kw in (dict(momentum=1.0), dict(momentum=-0.1), dict(eps=0.0), dict(eps=float("nan")), dict(lr=-1.0), dict(ns_steps=17), dict(ns_steps=-1), dict(grad_scale=1e30),
               dict(coefficients=(float("inf"), 0.0, 0.0))):
        with pytest.raises(lib.BsrError):
            lib.bsr_muon_step(opt, 1, **kw)
    with pytest.raises(lib.BsrError):
        lib.bsr_muon_step(opt, 0)
    empty = lib.bsr_muon_create([], [])
    lib.bsr_muon_step(empty, 1)
    opt.close()
    with pytest.raises(lib.BsrError):
        lib.bsr_muon_step(opt, 1)
