"""The workspace of gated products of 8-wide blocks: sums in memory stand in for the sweep kernel while its plan, which the first
product builds, may not be there; behind that no call asks for any."""
import ctypes

import numpy as np
import pytest

from test_gpu_gated import _close, _f64, _handle, _pair, _reference

pytestmark = pytest.mark.gpu


def _needs(W, m, code):
    import paper_2007_13055_amd.binding as binding
    size = ctypes.c_size_t(7)
    assert binding.load_library().bsr_spmm_gated_workspace_size(W.handle, m, code, ctypes.byref(size)) == 0
    return size.value


@pytest.mark.parametrize("bs_r,bs_c", [(8, 8), (16, 8), (8, 16)])
def test_none_once_the_plan_is_there(bs_r, bs_c):
    import torch
    import paper_2007_13055_amd as lib
    import paper_2007_13055_amd.binding as binding
    gate, up = _pair(768, 512, bs_r, bs_c, "f32", 0.2, 3)
    W, _ = _handle(gate, up, "f32")
    m = 700
    X = torch.randn((m, 512), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    # a capture in front of the first product has no plan, and takes the sums
    assert _needs(W, m, 0) >= 4 * m * 2 * 768
    early = torch.cuda.CUDAGraph()
    with torch.cuda.graph(early):
        H0 = lib.bsr_spmm_gated(W, X)
    assert _needs(W, m, 0) >= 4 * m * 2 * 768
    H1 = lib.bsr_spmm_gated(W, X)
    torch.cuda.synchronize()
    assert _needs(W, m, 0) == 0 and _needs(W, 64, 0) == 0
    # without any, eagerly and from a graph
    H2 = torch.full_like(H1, 7.0)
    how = binding.Gated(act=4, bias_dtype=0)
    call = lambda: binding.load_library().bsr_spmm_gated(W.handle, m, X.data_ptr(), H2.data_ptr(), 0, ctypes.byref(how), None, 0,  # noqa: E731
                                                         torch.cuda.current_stream().cuda_stream)
    assert call() == 0
    torch.cuda.synchronize()
    assert torch.equal(H2, H1)
    late = torch.cuda.CUDAGraph()
    with torch.cuda.graph(late):
        assert call() == 0
    for _ in range(3):
        X.normal_()
        late.replay()
        early.replay()
        torch.cuda.synchronize()
        z, dz, h, dh = _reference(_f64(X), gate, up, None, "silu")
        _close(H2, h, dh, "f32", "late")
        _close(H0, h, dh, "f32", "early")
        assert torch.equal(lib.bsr_spmm_gated(W, X), H2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sizes_whose_outputs_the_sweep_kernel_sums_again(monkeypatch, dtype):
    """k is no multiple of 16: by name, too, the sums go through memory, whether or not the kernel's plan is there."""
    import torch
    import paper_2007_13055_amd as lib
    from gpu_util import torch_dtype
    gate, up = _pair(72, 104, 8, 8, dtype, 0.4, 6)
    monkeypatch.setenv("BSR_SPMM_TUNE", "variant=6")
    W, _ = _handle(gate, up, dtype)
    monkeypatch.delenv("BSR_SPMM_TUNE")
    code = {"f32": 0, "bf16": 2}[dtype]
    X = torch.randn((90, 104), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(torch_dtype(dtype))
    z, dz, h, dh = _reference(_f64(X), gate, up, None, "silu")
    for _ in range(2):
        assert _needs(W, 90, code) > 0
        _close(lib.bsr_spmm_gated(W, X), h, dh, dtype, "H")
        lib.bsr_spmm_ex(W, X, path=lib.PATH_MFMA)                         # the plan's first use
        torch.cuda.synchronize()
