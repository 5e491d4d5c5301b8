"""AdamW steps at the edges of what they take: step numbers, moments and gradients of the smallest sizes, eps of 0."""
import pytest

pytestmark = pytest.mark.gpu


def _state(opt):
    return [t.clone() for t in opt.params + opt.exp_avg + opt.exp_avg_sq + [s for s in opt.scales + opt.master if s is not None]]


def _same(a, b):
    import torch
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype,bits,master", [("float32", 32, False), ("bfloat16", 32, True), ("bfloat16", 8, False)])
def test_step_numbers_below_one_on_the_device(dtype, bits, master):
    """They are skipped, as the host refuses them: a graph whose counter begins at 0 loses nothing in its first replay."""
    import torch
    import paper_2007_13055_amd as lib
    T = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    make = lambda: lib.bsr_adamw_create([torch.ones(c, device="cuda").to(T) for c in (5000, 77)], grads, state_bits=bits,  # noqa: E731
                                        weight_decay=0.1, master=True if master else None)
    grads = [torch.randn(c, generator=gen, device="cuda").to(T) for c in (5000, 77)]
    opt, one = make(), make()
    number = torch.zeros(1, dtype=torch.int64, device="cuda")
    before = _state(opt)
    for t in (0, -1, -2 ** 40):
        number.fill_(t)
        lib.bsr_adamw_step(opt, number)
        assert _same(before, _state(opt)), t
    number.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.bsr_adamw_step(opt, number, seed=3)
        number.add_(1)
    for t in range(4):
        graph.replay()
        torch.cuda.synchronize()
        if t:
            lib.bsr_adamw_step(one, torch.full((1,), t, dtype=torch.int64, device="cuda"), seed=3)
        assert _same(_state(one), _state(opt)), t
    assert all(bool(p.isfinite().all()) for p in opt.params)


def _formula(p, g, m, v, t, lr, b1, b2, eps):
    """One step in 64 bits; 0 / 0 counts as 0."""
    import torch
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    down = v.sqrt() / (1 - b2 ** t) ** 0.5 + eps
    return p - torch.where(m == 0, 0.0, lr / (1 - b1 ** t) * m / torch.where(down == 0, 1.0, down)), m, v


def test_gradients_whose_squares_are_subnormal():
    """eps of 0 and moments in fp32: no gradient, however small, makes an update larger than the formula's, and none makes
    none; from where v is a normal number the update is the formula's."""
    import torch
    import paper_2007_13055_amd as lib
    size = torch.exp2(-torch.arange(40, 149, dtype=torch.float64))
    g = torch.cat([size, -size, torch.zeros(5, dtype=torch.float64)]).float().cuda()
    p = torch.zeros_like(g)
    opt = lib.bsr_adamw_create([p], [g.clone()])
    want, m, v = (torch.zeros_like(g, dtype=torch.float64) for _ in range(3))
    lr, betas = 1e-2, (0.9, 0.95)
    for t in (1, 2, 3):
        before = p.double()
        lib.bsr_adamw_step(opt, t, lr=lr, betas=betas, eps=0.0)
        want, m, v = _formula(before, g.double(), m, v, t, lr, *betas, 0.0)
        update, full = (p.double() - before), (want - before)
        assert bool(p.isfinite().all()), t
        assert bool((update.abs() <= full.abs() * (1 + 2.0 ** -18) + 2.0 ** -24 * p.double().abs()).all()), t
        normal = v >= 2.0 ** -125                                         # of the same gradients all the time, so of every step
        assert int(normal.sum()) > 40
        # a few roundings of the update and the last place of p
        assert bool(((update - full).abs() <= 2.0 ** -19 * full.abs() + 2.0 ** -24 * p.double().abs())[normal].all()), t
        assert bool((p[g == 0] == 0).all()), t


@pytest.mark.parametrize("eps", [0.0, 1e-20, 1e-15])
def test_second_moments_that_8_bits_hold_as_zero(eps):
    """v below 2^-120 with an m that is held: the next step, whose gradient is 0, divides by nothing."""
    import torch
    import paper_2007_13055_amd as lib
    g = torch.zeros(1024, device="cuda")
    g[:256] = 2.0 ** -60                                                  # v = 0.05 2^-120
    g[256:512] = torch.randn(256, device="cuda") * 2.0 ** -59
    g[512:768] = torch.randn(256, device="cuda")                          # ordinary ones, which are not touched by the rule
    p = torch.zeros(1024, device="cuda")
    opt = lib.bsr_adamw_create([p], [g], state_bits=8)
    lr, betas = 1e-2, (0.9, 0.95)
    lib.bsr_adamw_step(opt, 1, lr=lr, betas=betas, eps=eps)
    m, v = lib.bsr_adamw_moments(opt)[0]
    assert bool((m[:256] > 0).all()) and bool((v[:256] == 0).all())
    first = p.clone()
    assert bool((p[:256] == 0).all()) and bool((p[768:] == 0).all())
    rest = g[512:768].double()
    full = lr * rest / (rest.abs() + eps)
    assert bool(((p[512:768].double() + full).abs() <= 2.0 ** -18 * lr).all())
    g[:512] = 0
    for t in (2, 3):
        lib.bsr_adamw_step(opt, t, lr=lr, betas=betas, eps=eps)
    assert bool(p.isfinite().all()) and bool((p[:256] == 0).all()) and bool((p[768:] == 0).all())
    # at most what two steps of the formula give for what is held at least: m hat / root of v hat <= 2 here
    assert bool(((p[256:512] - first[256:512]).abs() <= 2 * 2 * lr).all())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [2.0 ** -40, -1.0, 2.0 ** 40])
def test_the_largest_and_smallest_scales(bits, scale):
    """Gradients times the scale's inverse take the step that they take by themselves: a power of two moves exponents only."""
    import torch
    import paper_2007_13055_amd as lib
    gen = torch.Generator(device="cuda").manual_seed(2)
    g = torch.randn(5000, generator=gen, device="cuda")
    p, q = torch.zeros(5000, device="cuda"), torch.zeros(5000, device="cuda")
    opt, one = lib.bsr_adamw_create([p], [g / scale], state_bits=bits), lib.bsr_adamw_create([q], [g], state_bits=bits)
    for t in (1, 2):
        lib.bsr_adamw_step(opt, t, grad_scale=scale, seed=1)
        lib.bsr_adamw_step(one, t, seed=1)
    assert torch.equal(p, q) and _same(_state(opt), _state(one))
