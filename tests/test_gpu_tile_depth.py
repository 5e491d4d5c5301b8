"""The tile kernel with as many fp32 64x64 blocks in flight as it has: settings and bsr_tune beyond that take as many."""
import numpy as np
import pytest

import workloads as wl
from gpu_util import check, gpu_product, to_device

pytestmark = pytest.mark.gpu


def _problem(m, bs_r=64, bs_c=64):
    counts = np.random.default_rng(m).integers(0, 12, size=9)
    counts[2], counts[5] = 0, 14
    return wl.make_problem("depth", m, 14 * bs_c, 9 * bs_r, bs_r, bs_c, "f32", "f32", ("counts", counts), ("normal", 1.0), ("normal", 1.0), 40 + m)


@pytest.mark.parametrize("bs_r,bs_c", [(64, 64), (64, 32), (32, 64)])
def test_every_depth_has_the_same_sums(oracle_mod, monkeypatch, bs_r, bs_c):
    import paper_2007_13055_amd as lib
    p = _problem(300, bs_r, bs_c)
    Yo, So = oracle_mod.bsr_spmm(p.X, p.block_data, p.block_indices, p.index_pointer, p.n)
    first = None
    for tiles, depth in ((1, 1), (1, 2), (1, 3), (1, 4), (1, 9), (2, 1), (2, 2)):
        monkeypatch.setenv("BSR_SPMM_TUNE", f"variant=3,mt={tiles},a={depth}")
        Y, _ = gpu_product(p, path=lib.PATH_MFMA)
        check(Y, Yo, So, p.tau, f"{tiles} tiles, depth {depth}")
        first = Y if first is None else first
        assert np.array_equal(Y, first), (tiles, depth)


def test_tuned_product_of_the_largest_blocks(oracle_mod):
    import torch
    import paper_2007_13055_amd as lib
    p = _problem(400)
    Yo, So = oracle_mod.bsr_spmm(p.X, p.block_data, p.block_indices, p.index_pointer, p.n)
    W = lib.bsr_create(p.n, p.k, p.block_data, p.block_indices, p.index_pointer, dtype="f32")
    X, Y = to_device(p.X, "f32"), torch.full((p.m, p.n), float("nan"), device="cuda")
    tried, _ = lib.bsr_tune(W, X, Y, trials=2)
    assert tried > 1
    check(Y.double().cpu().numpy(), Yo, So, p.tau, "after tuning")
    settings = lib.bsr_tune_result(W, p.m, "f32")
    Y.fill_(float("nan"))
    lib.bsr_spmm(W, X, Y)
    torch.cuda.synchronize()
    check(Y.double().cpu().numpy(), Yo, So, p.tau, f"tuned {settings}")
