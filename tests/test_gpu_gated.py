"""bsr_spmm_gated and bsr_gated_backward against the formulas in 64 bits."""
import numpy as np
import pytest

import workloads as wl
from act_reference import ACTS, ROUNDING, slope, slope_bound, value, value_bound
from gpu_util import to_device, torch_dtype
from helpers import dense_expand

pytestmark = pytest.mark.gpu


def _f64(t):
    import torch
    return t.to(torch.float64).cpu().numpy()


def _halves(z, unit):
    z = z.reshape(z.shape[0], -1, 2, unit)
    return z[:, :, 0].reshape(z.shape[0], -1), z[:, :, 1].reshape(z.shape[0], -1)


def _joined(g, u, unit):
    return np.stack((g.reshape(g.shape[0], -1, unit), u.reshape(u.shape[0], -1, unit)), 2).reshape(g.shape[0], -1)


def _pair(n, k, bs_r, bs_c, dtype, density, seed, pattern=None):
    """Two matrices' problems of one shape (the second with empty block-rows)."""
    R, C = n // bs_r, k // bs_c
    rng = np.random.default_rng(seed)
    out = []
    for i in range(2):
        counts = rng.binomial(C, density, R) if pattern is None else pattern(rng, R, C)
        if i and R > 1:
            counts[rng.integers(R)] = 0
        out.append(wl.make_problem("gated", 4, k, n, bs_r, bs_c, dtype, dtype, ("counts", np.minimum(counts, C)), ("normal", 0.3), ("normal", 1.0), seed + i))
    return out


def _handle(gate, up, dtype):
    import paper_2007_13055_amd as lib
    arrays = lib.bsr_gated_arrays(*((p.block_data, p.block_indices, p.index_pointer) for p in (gate, up)))
    return lib.bsr_create(2 * gate.n, gate.k, *arrays, dtype=dtype), arrays


def _reference(X, gate, up, bias, act):
    """z in W's order, its fp32 error, H and its error (before H's rounding)."""
    u = gate.bs_r
    z, dz = [], []
    for i, p in enumerate((gate, up)):
        dense = dense_expand(p.block_data, p.block_indices, p.index_pointer, p.n, p.k)
        b = np.zeros(p.n) if bias is None else _halves(bias[None], u)[i][0]
        z.append(X @ dense.T + b)
        most = max(1, int(np.diff(p.index_pointer).max(initial=0)) * p.bs_c)
        dz.append((most + 4) * 2.0 ** -24 * (np.abs(X) @ np.abs(dense).T + np.abs(b)))       # fp32 sums of at most `most` products and the bias
    a = value(z[0], act)
    ea = 1.13 * dz[0] + value_bound(z[0], act)                                                # 1.13: the steepest slope
    h = a * z[1]
    return _joined(*z, u), _joined(*dz, u), h, ea * (np.abs(z[1]) + dz[1]) + np.abs(a) * dz[1] + 2.0 ** -24 * np.abs(h)


def _close(got, want, bound, dtype, what):
    u, tiny = ROUNDING[dtype]
    got = _f64(got)
    assert np.all(np.isfinite(got)), what
    over = np.abs(got - want) - (bound + u * (np.abs(want) + bound) + tiny)
    assert np.all(over <= 0), (what, float(over.max()), np.unravel_index(int(np.argmax(over)), over.shape))


def _run(m, gate, up, dtype, out, act, bias, seed=0, W=None):
    import torch
    import paper_2007_13055_amd as lib
    if W is None:
        W, _ = _handle(gate, up, dtype)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn((m, gate.k), generator=gen, device="cuda").to(torch_dtype(dtype))
    b = None if bias is None else (torch.randn(2 * gate.n, generator=gen, device="cuda") * 0.3).to(torch_dtype(bias))
    T = torch_dtype(out)
    flat_h, flat_z = (torch.full((m * n + 64,), 7.0, dtype=T, device="cuda") for n in (gate.n, 2 * gate.n))
    H, Z = lib.bsr_spmm_gated(W, X, flat_h[:m * gate.n].view(m, -1), h_dtype=out, bias=b, act=act, Z=flat_z[:2 * m * gate.n].view(m, -1))
    assert bool((flat_h[m * gate.n:] == 7).all()) and bool((flat_z[2 * m * gate.n:] == 7).all())
    z, dz, h, dh = _reference(_f64(X), gate, up, None if b is None else _f64(b), act)
    _close(Z, z, dz, out, "Z")
    _close(H, h, dh, out, "H")
    alone = lib.bsr_spmm_gated(W, X, h_dtype=out, bias=b, act=act)        # the sums not kept: the same H
    _close(alone, h, dh, out, "H alone")
    return X, b, H, Z


# blocks of every kernel family; widths that leave tiles, strips and quads ragged; rows from one to several tiles
SHAPES = [(16, 16, 96, 160), (32, 32, 160, 96), (64, 64, 192, 128), (64, 32, 128, 96), (16, 64, 80, 192), (32, 16, 96, 80), (8, 8, 72, 104), (8, 16, 80, 96),
          (16, 8, 96, 88), (5, 7, 35, 42), (12, 20, 60, 100), (1, 1, 9, 13)]


@pytest.mark.parametrize("m", [1, 5, 16, 33, 300, 1100])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("bs_r,bs_c,n,k", SHAPES)
def test_shapes(bs_r, bs_c, n, k, dtype, out, m):
    gate, up = _pair(n, k, bs_r, bs_c, dtype, 0.4, m)
    _run(m, gate, up, dtype, out, ACTS[1 + (m + bs_r) % 4], "f32" if m % 2 else dtype, seed=m)


@pytest.mark.parametrize("bs_r,bs_c,n,k", [(16, 1, 96, 200), (1, 16, 40, 96)])
@pytest.mark.parametrize("m", [1, 20, 257])
def test_blocks_of_one_row_or_column(bs_r, bs_c, n, k, m):
    gate, up = _pair(n, k, bs_r, bs_c, "f32", 0.2, m)
    _run(m, gate, up, "f32", "f32", "silu", "f32")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bias", [None, "f32", "bf16"])
def test_activations(act, bias):
    gate, up = _pair(128, 128, 16, 16, "bf16", 0.5, 3)
    _run(70, gate, up, "bf16", "bf16", act, bias)


@pytest.mark.parametrize("bs,dtype", [(16, "bf16"), (32, "f16"), (64, "bf16"), (8, "f16"), (32, "f32"), (64, "f16")])
@pytest.mark.parametrize("m", [64, 700, 2100])
def test_larger(bs, dtype, m):
    """Enough block-rows for every kernel that is chosen by size; a few of them hold most of W."""
    def power(rng, R, C):
        return np.where(rng.random(R) < 0.1, C, 1 + rng.integers(0, 3, R))
    for pattern in (None, power):
        gate, up = _pair(1024, 768, bs, bs, dtype, 0.15, bs + m, pattern)
        _run(m, gate, up, dtype, dtype, "silu", dtype)


def test_no_blocks_and_no_rows():
    import torch
    import paper_2007_13055_amd as lib
    empty = (np.zeros((0, 16, 16), np.float32), np.zeros(0, np.int32), np.zeros(7, np.int32))
    arrays = lib.bsr_gated_arrays(empty, empty)
    W = lib.bsr_create(192, 64, *arrays, dtype="bf16")
    X = torch.randn((5, 64), device="cuda").bfloat16()
    bias = torch.randn(192, device="cuda")
    H, Z = lib.bsr_spmm_gated(W, X, bias=bias, act="silu", keep_z=True)
    zg, zu = _halves(np.broadcast_to(_f64(bias), (5, 192)), 16)
    _close(H, value(zg, "silu") * zu, (value_bound(zg, "silu") + 2.0 ** -24) * np.abs(zu), "bf16", "H")
    assert torch.equal(Z, bias.bfloat16().expand(5, -1))
    assert bool((lib.bsr_spmm_gated(W, X) == 0).all())
    gate, up = _pair(64, 64, 16, 16, "bf16", 0.4, 1)
    W, _ = _handle(gate, up, "bf16")
    H, Z = lib.bsr_spmm_gated(W, X[:0], keep_z=True)
    assert H.shape == (0, 64) and Z.shape == (0, 128)


def test_arrays_are_block_rows_in_turn():
    import torch
    import paper_2007_13055_amd as lib
    gate, up = _pair(96, 80, 16, 16, "f32", 0.3, 2)
    both = [(p.block_data, p.block_indices, p.index_pointer) for p in (gate, up)]
    data, idx, ptr = lib.bsr_gated_arrays(*both)
    dense = dense_expand(np.asarray(data), idx, ptr, 192, 80)
    g, u = _halves(dense.T, 16)
    assert np.array_equal(g.T, dense_expand(*both[0], 96, 80)) and np.array_equal(u.T, dense_expand(*both[1], 96, 80))
    data2, idx2, ptr2 = lib.bsr_gated_arrays(*((torch.from_numpy(d).cuda(), torch.from_numpy(i), torch.from_numpy(p)) for d, i, p in both))
    assert data2.is_cuda and np.array_equal(data2.cpu().numpy(), data) and np.array_equal(idx, idx2) and np.array_equal(ptr, ptr2)


BACK = [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("f32", "bf16"), ("f32", "f16")]


@pytest.mark.parametrize("m,n,unit", [(1, 16, 16), (3, 8, 1), (7, 60, 12), (40, 72, 8), (257, 96, 32), (1003, 520, 4), (1100, 1024, 64), (2, 4096, 16), (5000, 30, 6)])
@pytest.mark.parametrize("dtype,out", BACK)
def test_backward(m, n, unit, dtype, out):
    import torch
    import paper_2007_13055_amd as lib
    gen = torch.Generator(device="cuda").manual_seed(m)
    G = torch.randn((m, n), generator=gen, device="cuda").to(torch_dtype(dtype))
    Z = (torch.randn((m, 2 * n), generator=gen, device="cuda") * 2).to(torch_dtype(dtype))
    for act in ACTS:
        flat = torch.full((2 * m * n + 64,), 7.0, dtype=torch_dtype(out), device="cuda")
        DZ, DB = lib.bsr_gated_backward(G, Z, unit, act, flat[:2 * m * n].view(m, -1), out)
        assert bool((flat[2 * m * n:] == 7).all())
        g, (zg, zu) = _f64(G), _halves(_f64(Z), unit)
        dg, du = g * zu * slope(zg, act), g * value(zg, act)
        eg = np.abs(g * zu) * (slope_bound(zg, act) + 2 * 2.0 ** -24 * np.abs(slope(zg, act)))
        eu = np.abs(g) * value_bound(zg, act) + 2.0 ** -24 * np.abs(du)
        want, bound = _joined(dg, du, unit), _joined(eg, eu, unit)
        _close(DZ, want, bound, out, act)
        _close(DB, want.sum(0), bound.sum(0) + (m + 8) * 2.0 ** -24 * np.abs(want).sum(0), "f32", "db")
        again = lib.bsr_gated_backward(G, Z, unit, act, dz_dtype=out)
        assert torch.equal(again[0], DZ) and torch.equal(again[1], DB)
        only, none = lib.bsr_gated_backward(G, Z, unit, act, dz_dtype=out, need_db=False)
        assert none is None and torch.equal(only, DZ)
        none, only = lib.bsr_gated_backward(G, Z, unit, act, dz_dtype=out, need_dz=False)
        assert none is None and torch.equal(only, DB)
        if out == dtype:                                                  # in Z's place
            place = Z.clone()
            assert lib.bsr_gated_backward(G, place, unit, act, place, need_db=False)[0] is place and torch.equal(place, DZ)


def test_backward_against_differences():
    import torch
    import paper_2007_13055_amd as lib
    rng = np.random.default_rng(2)
    g, z, direction = (rng.normal(size=s).astype(np.float32).astype(np.float64) for s in ((20, 64), (20, 128), (20, 128)))
    for act in ACTS:
        def loss(t):
            zg, zu = _halves(z + t * direction, 16)
            return (g * value(zg, act) * zu).sum()
        DZ, _ = lib.bsr_gated_backward(torch.from_numpy(g).float().cuda(), torch.from_numpy(z).float().cuda(), 16, act)
        got, size = (_f64(DZ) * direction).sum(), np.abs(_f64(DZ) * direction).sum()
        h = 1e-6
        # a difference's own error: 1e-16 / h of the loss's terms, and a kink of relu within h of 0
        assert abs(got - (loss(h) - loss(-h)) / (2 * h)) <= 1e-5 * size, act


def test_backward_without_rows():
    import torch
    import paper_2007_13055_amd as lib
    G, Z = torch.zeros((0, 32), device="cuda"), torch.zeros((0, 64), device="cuda")
    DZ, DB = lib.bsr_gated_backward(G, Z, 16, DB=torch.full((64,), 7.0, device="cuda"))
    assert DZ.shape == (0, 64) and bool((DB == 0).all())


def test_infinite_and_nan():
    """A NaN or an infinity of X reaches its own row only."""
    import torch
    import paper_2007_13055_amd as lib
    gate, up = _pair(128, 128, 16, 16, "bf16", 0.5, 4)
    W, _ = _handle(gate, up, "bf16")
    for m in (20, 400):
        X = torch.randn((m, 128), device="cuda").bfloat16()
        want = lib.bsr_spmm_gated(W, X)
        bad = X.clone()
        bad[3, 5], bad[9, 7] = float("nan"), float("inf")
        got = lib.bsr_spmm_gated(W, bad)
        rest = [i for i in range(m) if i not in (3, 9)]
        assert torch.equal(got[rest], want[rest])


@pytest.mark.parametrize("bs,m", [(16, 4), (16, 600), (32, 600), (8, 300), (64, 40)])
def test_captured_and_replayed(bs, m):
    """Product and gradient in one graph, recorded before and after the handle's first eager product of that size."""
    import torch
    import paper_2007_13055_amd as lib
    gate, up = _pair(1024, 512, bs, bs, "bf16", 0.2, bs)
    X, G = torch.randn((m, 512), device="cuda").bfloat16(), torch.randn((m, 1024), device="cuda").bfloat16()
    for warm in (False, True):
        W, _ = _handle(gate, up, "bf16")
        def run():
            H, Z = lib.bsr_spmm_gated(W, X, keep_z=True)
            return H, Z, *lib.bsr_gated_backward(G, Z, bs)
        if warm:
            run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = run()
        for _ in range(4):
            X.normal_()
            graph.replay()
            torch.cuda.synchronize()
            z, dz, h, dh = _reference(_f64(X), gate, up, None, "silu")
            _close(got[1], z, dz, "bf16", "Z")
            _close(got[0], h, dh, "bf16", "H")
            back = lib.bsr_gated_backward(G, got[1], bs)
            assert torch.equal(back[0], got[2]) and torch.equal(back[1], got[3])
            run()


def test_on_other_streams():
    import torch
    import paper_2007_13055_amd as lib
    gate, up = _pair(1024, 512, 16, 16, "bf16", 0.2, 5)
    W, _ = _handle(gate, up, "bf16")
    X = torch.randn((500, 512), device="cuda").bfloat16()
    want = lib.bsr_spmm_gated(W, X)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(lib.bsr_spmm_gated(W, X))
    got.append(lib.bsr_spmm_gated(W, X))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_refusals():
    import torch
    import paper_2007_13055_amd as lib
    gate, up = _pair(64, 64, 16, 16, "bf16", 0.4, 1)
    W, _ = _handle(gate, up, "bf16")
    X = torch.zeros((4, 64), device="cuda").bfloat16()
    H, Z = torch.zeros((4, 64), device="cuda").bfloat16(), torch.zeros((4, 128), device="cuda").bfloat16()
    odd = lib.bsr_create(48, 64, np.zeros((1, 16, 16), np.float32), [0], [0, 1, 1, 1], dtype="bf16")
    for call in (lambda: lib.bsr_spmm_gated(W, X.float()), lambda: lib.bsr_spmm_gated(W, X[:, :32]), lambda: lib.bsr_spmm_gated(W, X, Z), lambda: lib.bsr_spmm_gated(odd, X),
                 lambda: lib.bsr_spmm_gated(W, X, Z=H), lambda: lib.bsr_spmm_gated(W, X, bias=torch.zeros(64, device="cuda")),
                 lambda: lib.bsr_spmm_gated(W, X, bias=torch.zeros(128, device="cuda").half()), lambda: lib.bsr_spmm_gated(W, X, bias=torch.zeros(128)),
                 lambda: lib.bsr_spmm_gated(W, X.cpu()), lambda: lib.bsr_gated_backward(H, H, 16), lambda: lib.bsr_gated_backward(H, Z, 24),
                 lambda: lib.bsr_gated_backward(H, Z, 0), lambda: lib.bsr_gated_backward(H, Z.float(), 16), lambda: lib.bsr_gated_backward(H, Z, 16, dz_dtype="f32"),
                 lambda: lib.bsr_gated_arrays((np.zeros((1, 16, 16)), [0], [0, 1]), (np.zeros((1, 16, 8)), [0], [0, 1])),
                 lambda: lib.bsr_gated_arrays((np.zeros((1, 16, 16)), [0], [0, 2]), (np.zeros((1, 16, 16)), [0], [0, 1]))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(KeyError):
        lib.bsr_spmm_gated(W, X, act="glu")
    flat = torch.zeros(4 * 64 * 3, device="cuda").bfloat16()
    for call in (lambda: lib.bsr_spmm_gated(W, X, X), lambda: lib.bsr_spmm_gated(W, X, flat[:256].view(4, 64), Z=flat[128:640].view(4, 128)),
                 lambda: lib.bsr_gated_backward(H, Z, 16, DZ=torch.as_strided(Z, (4, 128), (128, 1), 0).view(-1)[:512].view(4, 128).narrow(0, 0, 4), DB=Z.view(-1)[:256].view(torch.float32))):
        with pytest.raises(lib.BsrError):
            call()
