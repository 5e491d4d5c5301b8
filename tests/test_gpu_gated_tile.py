"""The tile kernel's form for gated products, by name and where it is chosen by size, against the formulas in 64 bits."""
import numpy as np
import pytest

import workloads as wl
from gpu_util import torch_dtype
from test_gpu_gated import _handle, _run

pytestmark = pytest.mark.gpu


def _pair(n, k, bs_r, bs_c, dtype, seed, counts):
    return [wl.make_problem("gated tile", 4, k, n, bs_r, bs_c, dtype, dtype, ("counts", np.asarray(c)), ("normal", 0.3), ("normal", 1.0), seed + i)
            for i, c in enumerate(counts)]


def _made(monkeypatch, gate, up, dtype, tune):
    if tune:
        monkeypatch.setenv("BSR_SPMM_TUNE", tune)
    else:
        monkeypatch.delenv("BSR_SPMM_TUNE", raising=False)
    W, _ = _handle(gate, up, dtype)
    monkeypatch.delenv("BSR_SPMM_TUNE", raising=False)
    return W


# stored blocks of the gate's and the other half's block-rows: both, one or none of them empty; more and fewer than are in flight
GATE = [3, 0, 5, 0, 1, 2, 9, 1]
UP = [2, 4, 0, 0, 1, 7, 1, 9]


@pytest.mark.parametrize("bs_r,bs_c", [(32, 16), (32, 32), (32, 64), (64, 16), (64, 32), (64, 64)])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("depth", [1, 2])
def test_by_name(monkeypatch, bs_r, bs_c, dtype, out, depth):
    gate, up = _pair(8 * bs_r, 9 * bs_c, bs_r, bs_c, dtype, bs_r + bs_c, (GATE, UP))
    W = _made(monkeypatch, gate, up, dtype, f"variant=3,a={depth}")
    # rows of one tile, of some, and ones that end inside a tile, a wavefront's part and 16 of its rows
    for m, act, bias in ((1, "silu", None), (128, "gelu_tanh", "f32"), (129, "none", dtype), (300, "relu", None), (1003, "gelu", "f32")):
        _run(m, gate, up, dtype, out, act, bias, seed=m, W=W)


def test_halves_without_blocks(monkeypatch):
    for counts in (([0] * 4, [3, 1, 0, 2]), ([3, 1, 0, 2], [0] * 4), ([0, 0, 0, 1], [0, 0, 0, 0])):
        gate, up = _pair(4 * 64, 3 * 64, 64, 64, "f16", 7, counts)
        W = _made(monkeypatch, gate, up, "f16", "variant=3")
        _run(150, gate, up, "f16", "f16", "silu", "f32", W=W)


def _sums(lib, W, X):
    import torch
    H, Z = lib.bsr_spmm_gated(W, X, h_dtype="f32", keep_z=True)
    torch.cuda.synchronize()
    return H, Z


# 1003 rows are 8 tiles: 64 pairs of 64 rows make 512 of them, 256 pairs of 32 rows 2048
@pytest.mark.parametrize("bs_r,bs_c,n,k,dtype", [(64, 64, 4096, 512, "f16"), (64, 16, 4096, 192, "bf16"), (64, 64, 4096, 512, "f32"), (32, 32, 8192, 320, "bf16"),
                                                 (32, 64, 8192, 512, "f16"), (32, 32, 8192, 320, "f32")])
def test_chosen_by_size(monkeypatch, bs_r, bs_c, n, k, dtype):
    """Which kernel made a result shows in its sums' last bits: they are those of the kernel by name, and not of the k-split kernel."""
    import torch
    import paper_2007_13055_amd as lib
    m, R, C = 1003, n // bs_r, k // bs_c
    rng = np.random.default_rng(bs_r + bs_c)
    counts = [np.where(rng.random(R) < 0.1, C, rng.integers(0, max(2, C // 2), R)) for _ in range(2)]   # long block-rows and empty ones
    gate, up = _pair(n, k, bs_r, bs_c, dtype, 11, counts)
    W = _made(monkeypatch, gate, up, dtype, None)
    _run(m, gate, up, dtype, dtype, "silu", dtype, W=W)
    X = torch.randn((m, k), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(torch_dtype(dtype))
    free, tile, ksplit = (_sums(lib, _made(monkeypatch, gate, up, dtype, tune), X) for tune in (None, "variant=3", "variant=2"))
    assert torch.equal(free[0], tile[0]) and torch.equal(free[1], tile[1])
    assert not torch.equal(free[1], ksplit[1])


def test_rows_that_are_not_finite(monkeypatch):
    import torch
    import paper_2007_13055_amd as lib
    gate, up = _pair(8 * 64, 9 * 64, 64, 64, "bf16", 5, (GATE, UP))
    W = _made(monkeypatch, gate, up, "bf16", "variant=3")
    X = torch.randn((400, 9 * 64), device="cuda").bfloat16()
    want, bad = lib.bsr_spmm_gated(W, X), X.clone()
    bad[3, 5], bad[200, 7] = float("nan"), float("inf")
    rest = [i for i in range(400) if i not in (3, 200)]
    assert torch.equal(lib.bsr_spmm_gated(W, bad)[rest], want[rest])
