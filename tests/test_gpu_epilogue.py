"""bsr_spmm_epilogue in every kernel of the product, and bsr_epilogue_backward, against 64 bits."""
import numpy as np
import pytest

import workloads as wl
from act_reference import ACTS, ROUNDING, slope, slope_bound, value, value_bound
from gpu_util import to_device, torch_dtype
from helpers import dense_expand

pytestmark = pytest.mark.gpu

# (m, k, n, bs_r, bs_c, type, BSR_SPMM_TUNE): the kernel named runs (or what it leaves to another one)
KERNELS = [
    (1, 64, 48, 16, 16, "f32", ""), (5, 70, 63, 7, 5, "bf16", ""), (9, 96, 80, 8, 8, "f16", ""),          # wavefronts
    (67, 64, 96, 16, 16, "f32", "variant=1"), (131, 128, 96, 32, 16, "bf16", "variant=1"), (70, 64, 64, 64, 32, "f16", "variant=1,mt=2"),
    (35, 128, 96, 16, 32, "bf16", "variant=2"), (33, 128, 128, 32, 32, "f16", "variant=2,mt=1"), (65, 64, 128, 64, 64, "f32", "variant=2,mt=2"),
    (21, 96, 64, 32, 32, "f32", "variant=2,mt=3"),
    (150, 128, 192, 64, 64, "f16", "variant=3,mt=1"), (300, 96, 128, 32, 32, "f32", "variant=3,mt=2"), (129, 64, 96, 32, 16, "bf16", "variant=3,mt=1,a=4"),
    (77, 192, 208, 16, 16, "f16", "variant=4"), (100, 64, 96, 16, 16, "bf16", "variant=4,mt=4"), (40, 80, 48, 16, 16, "f16", "variant=4,mt=2"),
    (90, 192, 160, 16, 16, "bf16", "variant=6"), (50, 136, 88, 8, 8, "bf16", "variant=6"), (70, 96, 112, 8, 16, "f32", "variant=6"),
    (45, 64, 80, 8, 8, "f32", "variant=7"), (33, 96, 48, 16, 8, "f16", "variant=7"),
    (70, 132, 96, 16, 1, "f32", "variant=1"), (37, 200, 80, 16, 1, "f32", "variant=2"), (40, 96, 130, 1, 16, "f32", ""),
    (3, 32, 32, 16, 1, "f32", ""),
]


def _problem(m, k, n, bs_r, bs_c, dtype, density=0.4, seed=3):
    rng = np.random.default_rng(seed)
    counts = rng.binomial(k // bs_c, density, size=n // bs_r)
    counts[0] = min(2, k // bs_c)
    if len(counts) > 2:
        counts[1] = 0                                                    # a block-row without blocks: z is the bias
    return wl.make_problem("epilogue", m, k, n, bs_r, bs_c, dtype, dtype, ("counts", counts), ("normal", 0.3), ("normal", 1.0), seed)


def _handle(p):
    import paper_2007_13055_amd as lib
    return lib.bsr_create(p.n, p.k, p.block_data, p.block_indices, p.index_pointer, dtype=p.in_dtype)


def _f64(t):
    import torch
    return t.to(torch.float64).cpu().numpy()


def _check_fp32_epilogue(W, X, act, bias_dtype, seed, what):
    """fp32 results: Z is the product's own sum, bit for bit, and the bias; Y follows from Z."""
    import torch
    import paper_2007_13055_amd as lib
    m, n = X.shape[0], W.n
    gen = torch.Generator(device="cuda").manual_seed(seed)
    bias = torch.randn(n, generator=gen, device="cuda").to(torch_dtype(bias_dtype))
    R = torch.randn((m, n), generator=gen, device="cuda")
    Z0 = torch.randn((m, n), generator=gen, device="cuda") * 2
    plain = lib.bsr_spmm(W, X, y_dtype="f32")
    Y, Z = lib.bsr_spmm_epilogue(W, X, y_dtype="f32", bias=bias, act=act, residual=R, keep_z=True)
    assert torch.equal(Z, plain + bias.float()), what
    z = _f64(Z)
    want = value(z, act) + _f64(R)
    assert np.all(np.abs(_f64(Y) - want) <= value_bound(z, act) + 2.0 ** -23 * np.abs(want)), what
    alone = lib.bsr_spmm_epilogue(W, X, y_dtype="f32", act=act)                       # nothing but the activation
    z = _f64(plain)
    assert np.all(np.abs(_f64(alone) - value(z, act)) <= value_bound(z, act) + 2.0 ** -23 * np.abs(z)), what
    Y = lib.bsr_spmm_epilogue(W, X, y_dtype="f32", act=act, through=Z0, residual=R)
    g = slope(_f64(Z0), act)
    want = z * g + _f64(R)
    assert np.all(np.abs(_f64(Y) - want) <= np.abs(z) * (slope_bound(g, act) + 2.0 ** -23) + 2.0 ** -23 * np.abs(want)), what


@pytest.mark.parametrize("shape", KERNELS, ids=lambda s: "x".join(map(str, s)))
def test_every_kernel_finishes_its_sums(shape, monkeypatch):
    m, k, n, bs_r, bs_c, dtype, tune = shape
    if tune:
        monkeypatch.setenv("BSR_SPMM_TUNE", tune)
    p = _problem(m, k, n, bs_r, bs_c, dtype)
    W, X = _handle(p), to_device(p.X, dtype)
    for i, act in enumerate(ACTS):
        _check_fp32_epilogue(W, X, act, dtype if i % 2 else "f32", 10 + i, f"{shape} {act}")


@pytest.mark.parametrize("shape", [s for s in KERNELS if s[5] != "f32"], ids=lambda s: "x".join(map(str, s)))
def test_16_bit_results_are_rounded_once(shape, monkeypatch):
    import torch
    import paper_2007_13055_amd as lib
    m, k, n, bs_r, bs_c, dtype, tune = shape
    if tune:
        monkeypatch.setenv("BSR_SPMM_TUNE", tune)
    p = _problem(m, k, n, bs_r, bs_c, dtype, seed=4)
    W, X = _handle(p), to_device(p.X, dtype)
    T = torch_dtype(dtype)
    gen = torch.Generator(device="cuda").manual_seed(5)
    wide = torch.randn((m, n + 24), generator=gen, device="cuda").to(T)
    bias = torch.randn(n, generator=gen, device="cuda").to(T)
    dense = dense_expand(p.block_data, p.block_indices, p.index_pointer, p.n, p.k)
    z = p.X.astype(np.float64) @ dense.T + _f64(bias)
    # |z| error: fp32 sums of at most k products, in any order; 1.13: the steepest slope of the activations
    sums = np.abs(p.X).astype(np.float64) @ np.abs(dense).T + np.abs(_f64(bias))
    dz = (k + 4) * 2.0 ** -24 * sums
    u, tiny = ROUNDING[dtype]
    rows = wide[:, 8:8 + n] if (n + 24) % 8 == 0 and n % 8 == 0 else wide[:, :n].contiguous()   # rows wider than the result's
    for act in ACTS:
        Y, Z = lib.bsr_spmm_epilogue(W, X, bias=bias, act=act, residual=rows, keep_z=True)
        assert Y.dtype == T and Z.dtype == T
        want = value(z, act) + _f64(rows)
        bound = 1.13 * dz + value_bound(z, act) + 2.0 ** -23 * np.abs(want)
        assert np.all(np.abs(_f64(Z) - z) <= dz + u * (np.abs(z) + dz) + tiny), (shape, act)
        assert np.all(np.abs(_f64(Y) - want) <= bound + u * (np.abs(want) + bound) + tiny), (shape, act)
        Z0 = torch.randn((m, n), generator=gen, device="cuda").to(T)
        Y = lib.bsr_spmm_epilogue(W, X, bias=bias, act=act, through=Z0)
        g = slope(_f64(Z0), act)
        want = z * g
        bound = 1.13 * dz + np.abs(z) * (slope_bound(g, act) + 2.0 ** -22)
        assert np.all(np.abs(_f64(Y) - want) <= bound + u * (np.abs(want) + bound) + tiny), (shape, act)


@pytest.mark.parametrize("shape", KERNELS, ids=lambda s: "x".join(map(str, s)))
def test_parts_do_not_change_each_other(shape, monkeypatch):
    """Y is the same whether or not Z is kept, and a residual of zeros and a bias of zeros change nothing."""
    import torch
    import paper_2007_13055_amd as lib
    m, k, n, bs_r, bs_c, dtype, tune = shape
    if tune:
        monkeypatch.setenv("BSR_SPMM_TUNE", tune)
    p = _problem(m, k, n, bs_r, bs_c, dtype, seed=6)
    W, X = _handle(p), to_device(p.X, dtype)
    T = torch_dtype(dtype)
    bias = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda").to(T)
    none = torch.zeros((m, n), dtype=T, device="cuda")
    for act in ACTS:
        Y = lib.bsr_spmm_epilogue(W, X, bias=bias, act=act)
        assert torch.equal(lib.bsr_spmm_epilogue(W, X, bias=bias, act=act, keep_z=True)[0], Y), act
        assert torch.equal(lib.bsr_spmm_epilogue(W, X, bias=bias, act=act, residual=none), Y), act   # (-0 + 0 equals -0)
        assert torch.equal(lib.bsr_spmm_epilogue(W, X, bias=torch.zeros_like(bias), act=act), lib.bsr_spmm_epilogue(W, X, act=act)), act
    assert torch.equal(lib.bsr_spmm_epilogue(W, X), lib.bsr_spmm(W, X))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_row_groups_and_the_tiles_behind_them(dtype):
    """64x64 blocks, a few block-rows with most of them, from 1024 rows on: two kernels write one result."""
    rng = np.random.default_rng(6)
    counts = np.full(24, 2)
    counts[rng.permutation(24)[:8]] = 20
    p = wl.make_problem("groups", 1030, 24 * 64, 24 * 64, 64, 64, dtype, dtype, ("counts", counts), ("normal", 0.1), ("normal", 1.0), 6)
    W, X = _handle(p), to_device(p.X, dtype)
    for act in ("gelu", "none"):
        _check_fp32_epilogue(W, X, act, dtype, 7, act)


def test_no_stored_block_and_no_rows():
    import torch
    import paper_2007_13055_amd as lib
    W = lib.bsr_create(48, 32, torch.zeros((0, 16, 16), device="cuda"), np.zeros(0, np.int32), np.zeros(4, np.int32), dtype="f32")
    bias, R = torch.arange(48.0, device="cuda"), torch.ones((70, 48), device="cuda")
    X = torch.full((70, 32), float("nan"), device="cuda")
    Y, Z = lib.bsr_spmm_epilogue(W, X, bias=bias, act="relu", residual=R, keep_z=True)
    assert torch.equal(Y, bias + R) and torch.equal(Z, bias.expand(70, 48))
    assert lib.bsr_spmm_epilogue(W, X[:0], bias=bias, act="gelu").shape == (0, 48)


def test_infinities_and_nan():
    """Limits at infinite sums, NaN where the sum is one; a NaN in X stays with the rows and blocks that read it."""
    import torch
    import paper_2007_13055_amd as lib
    data = torch.eye(16, device="cuda").reshape(1, 16, 16)
    W = lib.bsr_create(16, 16, data, np.array([0]), np.array([0, 1]))
    inf, nan = float("inf"), float("nan")
    bias = torch.tensor([inf, -inf, nan, 1e30, -1e30, 30.0, -30.0, 0.0] * 2, device="cuda")
    X = torch.zeros((20, 16), device="cuda")
    for act, far in (("relu", 0.0), ("gelu", 0.0), ("gelu_tanh", 0.0), ("silu", 0.0), ("none", -inf)):
        y = lib.bsr_spmm_epilogue(W, X, bias=bias, act=act)
        assert bool((y[:, 0] == inf).all()) and bool((y[:, 1] == far).all()) and bool(y[:, 2].isnan().all()), act
        assert bool((y[:, 3] == 1e30).all()) and bool((y[:, 5] == 30).all()) and bool((y[:, 7] == 0).all()), act
        Z0 = bias.expand(20, 16).contiguous()
        y = lib.bsr_spmm_epilogue(W, torch.ones_like(X), act=act, through=Z0)
        flat = 1.0 if act == "none" else 0.0
        assert bool((y[:, 0] == 1).all()) and bool((y[:, 1] == flat).all()), act
        assert bool((y[:, 3] == 1).all()) and bool((y[:, 4] == flat).all()), act


def test_infinities_stay_with_their_blocks():
    """Sizes without whole tiles on the sweep kernel: sums that came out as NaN are summed, and finished, again."""
    import torch
    import paper_2007_13055_amd as lib
    p = _problem(4100, 136, 1032, 8, 8, "bf16", density=0.3, seed=8)
    W, X = _handle(p), to_device(p.X, "bf16")
    T = torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(1)
    bias, R = torch.randn(p.n, generator=gen, device="cuda").to(T), torch.randn((p.m, p.n), generator=gen, device="cuda").to(T)
    clean, clean_z = lib.bsr_spmm_epilogue(W, X, bias=bias, act="silu", residual=R, keep_z=True)
    X[7, 3] = float("inf")
    X[200, 100] = float("nan")
    Y, Z = lib.bsr_spmm_epilogue(W, X, bias=bias, act="silu", residual=R, keep_z=True)
    dense = dense_expand(p.block_data, p.block_indices, p.index_pointer, p.n, p.k)
    stored = dense_expand(np.ones_like(p.block_data), p.block_indices, p.index_pointer, p.n, p.k) > 0
    hit = torch.zeros((p.m, p.n), dtype=torch.bool)
    hit[7], hit[200] = torch.from_numpy(stored[:, 3]), torch.from_numpy(stored[:, 100])
    hit = hit.cuda()
    assert bool(Y[200][hit[200]].isnan().all()) and bool(Z[200][hit[200]].isnan().all())
    rest = ~hit
    rest[[7, 200]] = False
    assert torch.equal(Y[rest], clean[rest]) and torch.equal(Z[rest], clean_z[rest])
    for i in (7, 200):                                                    # their other outputs may be summed in another order
        keep = ~hit[i]
        z = clean_z[i][keep].double()
        assert bool(((Z[i][keep].double() - z).abs() <= 2.0 ** -7 * z.abs() + 1e-4).all()), i


def test_refusals():
    import torch
    import paper_2007_13055_amd as lib
    p = _problem(20, 64, 48, 16, 16, "f16")
    W, X = _handle(p), to_device(p.X, "f16")
    T = torch.float16
    new = lambda *s, dtype=T: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    Y, R = new(20, 48), new(20, 48)
    flat = new(20 * 48 + 8)
    for args, error in [(dict(act="tanh"), KeyError), (dict(bias=new(47)), ValueError), (dict(bias=new(48, dtype=torch.bfloat16)), ValueError),
                        (dict(bias=new(96)[::2]), ValueError), (dict(bias=torch.zeros(48, dtype=T)), ValueError),
                        (dict(residual=new(20, 47)), ValueError), (dict(residual=new(48, 20).t()), ValueError),
                        (dict(residual=new(20, 48, dtype=torch.float32)), ValueError), (dict(residual=torch.zeros((20, 48), dtype=T)), ValueError),
                        (dict(residual=new(1, 48).expand(20, 48)), ValueError), (dict(through=new(20, 96)[:, ::2]), ValueError),
                        (dict(Z=new(19, 48)), ValueError), (dict(Y=new(20, 48, dtype=torch.float32)), ValueError),
                        (dict(Y=Y, residual=Y), lib.BsrError), (dict(Y=Y, Z=Y), lib.BsrError), (dict(Z=R, residual=R), lib.BsrError),
                        (dict(Y=Y, through=Y, act="relu"), lib.BsrError), (dict(residual=flat[4:964].view(20, 48)), lib.BsrError),
                        (dict(residual=new(20, 52)[:, :48]), lib.BsrError), (dict(Z=flat[4:964].view(20, 48)), lib.BsrError)]:
        with pytest.raises(error):
            lib.bsr_spmm_epilogue(W, X, **args)
    with pytest.raises(ValueError):
        lib.bsr_spmm_epilogue(W, X.cpu(), act="relu")
    W.close()
    with pytest.raises(lib.BsrError):
        lib.bsr_spmm_epilogue(W, X, act="relu")


def test_on_another_stream_and_in_a_graph():
    """A captured epilogue and its gradient, replayed with new inputs and eager work between, against the eager calls."""
    import torch
    import paper_2007_13055_amd as lib
    p = _problem(600, 256, 512, 16, 16, "bf16", seed=9)
    W, X = _handle(p), to_device(p.X, "bf16")
    T = torch.bfloat16
    bias, R, G = torch.randn(512, device="cuda").to(T), torch.randn((600, 512), device="cuda").to(T), torch.randn((600, 512), device="cuda").to(T)
    Y, Z, DZ, DB = torch.empty_like(R), torch.empty_like(R), torch.empty_like(R), torch.empty(512, device="cuda")

    def run():
        lib.bsr_spmm_epilogue(W, X, Y, bias=bias, act="gelu", residual=R, Z=Z)
        lib.bsr_epilogue_backward(G, Z, "gelu", DZ, DB=DB)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(4):
        X.copy_(torch.randn_like(X, dtype=torch.float32))
        G.copy_(torch.randn_like(G, dtype=torch.float32))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (Y, Z, DZ, DB)]
        for t in (Y, Z, DZ, DB):
            t.fill_(float("nan"))
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (Y, Z, DZ, DB))), seed


# ---------------------------------------------------------------------------------------------- the gradient
@pytest.mark.parametrize("act", ACTS)
def test_slopes_against_differences(act):
    import torch
    import paper_2007_13055_amd as lib
    z = torch.linspace(-9, 9, 4000, device="cuda").reshape(8, 500)
    z = z[z.abs() > 1e-3].reshape(-1, 1)                                  # relu has no slope at 0
    dz, _ = lib.bsr_epilogue_backward(torch.ones_like(z), z, act)
    x, h = _f64(z), 1e-5
    differences = (value(x + h, act) - value(x - h, act)) / (2 * h)
    # differences: h^2 / 6 times a third derivative below 2, and 1e-16 * 9 / h
    assert np.all(np.abs(_f64(dz) - differences) <= 2e-6 + 1e-9)
    assert np.all(np.abs(_f64(dz) - slope(x, act)) <= 2e-6)


@pytest.mark.parametrize("m,n", [(1, 1), (1, 2081), (3, 8), (17, 5), (64, 64), (255, 513), (1000, 1), (5000, 3), (700, 520), (2500, 1024), (33, 8192), (16384, 40)])
@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("f16", "f16"), ("bf16", "bf16")])
def test_backward(m, n, types):
    import torch
    import paper_2007_13055_amd as lib
    g_dtype, dz_dtype = types
    gen = torch.Generator(device="cuda").manual_seed(m * 7 + n)
    G, Z = (torch.randn((m, n), generator=gen, device="cuda").to(torch_dtype(g_dtype)) for _ in range(2))
    u, tiny = ROUNDING[dz_dtype]
    for act in ("gelu", "silu", "none"):
        dz, db = lib.bsr_epilogue_backward(G, Z, act, dz_dtype=dz_dtype)
        assert dz.dtype == torch_dtype(dz_dtype) and db.dtype == torch.float32
        s = slope(_f64(Z), act)
        want = _f64(G) * s
        off = np.abs(_f64(G)) * (slope_bound(s, act) + 2.0 ** -23)
        assert np.all(np.abs(_f64(dz) - want) <= off + u * np.abs(want) * 1.001 + tiny), act
        # sums: at most ceil(m / 2) + 300 additions one behind the other, each off by half a step of at most the sum of sizes
        assert np.all(np.abs(_f64(db) - want.sum(0)) <= off.sum(0) + (m / 2 + 300) * 2.0 ** -24 * np.abs(want).sum(0) + 1e-30), act
        again = lib.bsr_epilogue_backward(G, Z, act, dz_dtype=dz_dtype)[1]
        assert torch.equal(db, again)
    only, none = lib.bsr_epilogue_backward(G, Z, "gelu", dz_dtype=dz_dtype, need_db=False)
    assert none is None and torch.equal(only, lib.bsr_epilogue_backward(G, Z, "gelu", dz_dtype=dz_dtype)[0])
    none, db = lib.bsr_epilogue_backward(G, Z, "relu", need_dz=False)
    assert none is None and torch.equal(db, lib.bsr_epilogue_backward(G, Z, "relu")[1])


def test_backward_in_place_empty_and_refused():
    import torch
    import paper_2007_13055_amd as lib
    G, Z = torch.randn((50, 72), device="cuda"), torch.randn((50, 72), device="cuda")
    want, db = lib.bsr_epilogue_backward(G, Z, "silu")
    g, z = G.clone(), Z.clone()
    assert torch.equal(lib.bsr_epilogue_backward(g, Z, "silu", g)[0], want) and torch.equal(g, want)
    assert torch.equal(lib.bsr_epilogue_backward(G, z, "silu", z)[0], want) and torch.equal(z, want)
    assert lib.bsr_epilogue_backward(G)[0] is G                           # no activation: dZ is G
    copy = torch.empty_like(G)
    assert lib.bsr_epilogue_backward(G, DZ=copy)[0] is copy and torch.equal(copy, G)
    dz, db = lib.bsr_epilogue_backward(G[:0], Z[:0], "gelu")
    assert dz.shape == (0, 72) and torch.equal(db, torch.zeros(72, device="cuda"))
    dz, db = lib.bsr_epilogue_backward(G[:, :0].contiguous(), act="none")
    assert db.shape == (0,)
    wide = torch.zeros(50 * 72 + 4, device="cuda")
    for args, error in [((G, None, "gelu"), ValueError), ((G, Z[:, :70], "gelu"), ValueError), ((G, Z.half(), "gelu"), ValueError),
                        ((G.t(), Z.t(), "gelu"), ValueError), ((G.cpu(), Z, "gelu"), ValueError), ((G, Z.cpu(), "gelu"), ValueError),
                        ((G.double(), Z, "gelu"), KeyError), ((G, Z, "swish"), KeyError), ((G.half(), Z.half(), "gelu", None, "f32"), ValueError),
                        ((G, Z, "gelu", None, None, torch.zeros(71, device="cuda")), ValueError),
                        ((wide[4:].view(50, 72), Z, "gelu", wide[:-4].view(50, 72)), lib.BsrError),          # moved against each other
                        ((G, Z, "gelu", None, None, Z.view(-1)[:72]), lib.BsrError)]:
        with pytest.raises(error):
            lib.bsr_epilogue_backward(*args)


@pytest.mark.parametrize("dtype,blocks", [("f32", (16, 16)), ("f32", (16, 1)), ("bf16", (32, 32)), ("f16", (8, 8))])
def test_a_layers_gradients(dtype, blocks):
    """Forward and backward of one layer: dX, dW, db and the gradient taken on through an activation in front, against the
    formulas in 64 bits and, in one direction, against differences of the loss."""
    import torch
    import paper_2007_13055_amd as lib
    bs_r, bs_c = blocks
    m, k, n = 150, 192, 128
    p = _problem(m, k, n, bs_r, bs_c, dtype, seed=11)
    p.block_data = wl.round_to_storage(p.block_data, dtype)
    W, X = _handle(p), to_device(p.X, dtype)
    WT = lib.bsr_create_transposed(n, k, p.block_data, p.block_indices, p.index_pointer, dtype=dtype)
    T = torch_dtype(dtype)
    gen = torch.Generator(device="cuda").manual_seed(2)
    bias, G = torch.randn(n, generator=gen, device="cuda").to(T), torch.randn((m, n), generator=gen, device="cuda").to(T)
    H = torch.randn((m, k), generator=gen, device="cuda").to(T)            # X = act of it, in the layer before
    Y, Z = lib.bsr_spmm_epilogue(W, X, bias=bias, act="gelu", keep_z=True)
    dZ, db = lib.bsr_epilogue_backward(G, Z, "gelu")
    dX = lib.bsr_spmm(WT, dZ)
    dH = lib.bsr_spmm_epilogue(WT, dZ, act="silu", through=H)
    dW = lib.bsr_sddmm(W, dZ, X, d_dtype="f32")
    dense = dense_expand(p.block_data, p.block_indices, p.index_pointer, n, k)
    u = ROUNDING[dtype][0]
    z = _f64(X) @ dense.T + _f64(bias)
    g = _f64(G) * slope(z, "gelu")
    # dZ: Z's own rounding moves the slope by at most 1.13 u |z|, then two roundings; the sums over it add its error up
    dg = np.abs(_f64(G)) * (1.2 * (u + 2e-5) * (np.abs(z) + 1) + 4e-6) + u * np.abs(g) * 1.01 + 1e-7
    assert np.all(np.abs(_f64(dZ) - g) <= dg)
    assert np.all(np.abs(_f64(db) - g.sum(0)) <= dg.sum(0) + 1e-4)
    fp32 = (m + n + k) * 2.0 ** -24
    ex = dg @ np.abs(dense) + fp32 * (np.abs(g) @ np.abs(dense))
    assert np.all(np.abs(_f64(dX) - g @ dense) <= ex + u * np.abs(g @ dense) * 1.01 + 1e-6)
    s = slope(_f64(H), "silu")
    assert np.all(np.abs(_f64(dH) - (g @ dense) * s) <= ex * 1.2 + (u * 1.01 + 4e-6) * np.abs(g @ dense) * 1.2 + 1e-6)
    full = g.T @ _f64(X)
    ew = dg.T @ np.abs(_f64(X)) + fp32 * (np.abs(g).T @ np.abs(_f64(X)))
    rows = np.repeat(np.arange(n // bs_r), np.diff(p.index_pointer))
    for q in range(len(rows)):
        a, c = slice(rows[q] * bs_r, (rows[q] + 1) * bs_r), slice(p.block_indices[q] * bs_c, (p.block_indices[q] + 1) * bs_c)
        assert np.all(np.abs(_f64(dW[q]) - full[a, c]) <= ew[a, c] + 1e-6), q
    if dtype == "f32":                                                    # the loss sum(G * Y) along a random direction of W
        step = np.random.default_rng(3).normal(size=p.block_data.shape)
        loss = lambda t: (_f64(G) * value(_f64(X) @ dense_expand(p.block_data + t * step, p.block_indices, p.index_pointer, n, k).T + _f64(bias), "gelu")).sum()  # noqa: E731
        along = (loss(1e-5) - loss(-1e-5)) / 2e-5
        assert abs(along - (_f64(dW) * step).sum()) <= 1e-4 * np.abs(_f64(dW) * step).sum()
