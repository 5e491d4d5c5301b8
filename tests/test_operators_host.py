"""Refusals of the epilogue, its gradient and the AdamW step that no GPU is needed for: they are decided before any device
call, here on made-up addresses."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def b():
    import os
    from paper_2007_13055_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2007_13055_amd import build
        build.build()
    return binding


OK, NULL, SHAPE, INDEX, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED, OVERLAP = 0, 1, 2, 4, 5, 6, 7, 9, 11
A, B, C, D, E, F = (0x10000000 * i for i in range(1, 7))


def test_structures_follow_the_header(b):
    assert ctypes.sizeof(b.Epilogue) == 48 and b.Epilogue.residual_ld.offset == 24
    assert ctypes.sizeof(b.AdamWTensor) == 96 and b.AdamWTensor.weight_decay.offset == 64 and b.AdamWTensor.t_perm_host.offset == 88
    assert ctypes.sizeof(b.AdamWHyper) == 72 and b.AdamWHyper.grad_scale.offset == 40 and b.AdamWHyper.grad_scale_dev.offset == 64


def test_epilogue_of_no_matrix(b):
    so = b.load_library()
    assert so.bsr_spmm_epilogue(None, 4, A, B, 0, ctypes.byref(b.Epilogue()), None) == NULL
    assert so.bsr_spmm_epilogue(None, 4, A, B, 0, None, None) == NULL


def test_backward_refusals(b):
    so = b.load_library()
    size = ctypes.c_size_t(7)
    assert so.bsr_epilogue_backward_workspace_size(8192, 8192, ctypes.byref(size)) == OK and size.value % 256 == 0 and size.value > 0
    assert so.bsr_epilogue_backward_workspace_size(1, 100, ctypes.byref(size)) == OK and size.value == 0
    assert so.bsr_epilogue_backward_workspace_size(-1, 100, ctypes.byref(size)) == SHAPE
    assert so.bsr_epilogue_backward_workspace_size(1, 1, None) == NULL
    call = lambda m=64, n=64, act=2, g_t=0, g=A, z=B, dz_t=0, dz=C, db=D, ws=E, ws_bytes=1 << 20: so.bsr_epilogue_backward(  # noqa: E731
        m, n, act, g_t, g, z, dz_t, dz, db, ws, ws_bytes, None)
    assert call(m=-1) == SHAPE and call(n=1 << 31) == SHAPE and call(m=1 << 30) == SHAPE and call(m=1 << 20, n=1 << 20) == SHAPE
    assert call(act=5) == DTYPE and call(act=-1) == DTYPE and call(g_t=3) == DTYPE and call(dz_t=7) == DTYPE
    assert call(g_t=1, dz_t=2) == DTYPE and call(g_t=1, dz_t=0) == DTYPE                      # 16 bits to another type
    assert call(g=None) == NULL and call(z=None) == NULL and call(dz=None, db=None) == NULL
    assert call(g=A + 8) == ALIGN and call(z=B + 4) == ALIGN and call(dz=C + 2) == ALIGN and call(db=D + 4) == ALIGN and call(ws=E + 8) == ALIGN
    assert call(m=8192, n=8192, ws=None) == WORKSPACE and call(m=8192, n=8192, ws_bytes=1024) == WORKSPACE
    assert call(dz=A + 64) == OVERLAP and call(dz=B + 64) == OVERLAP and call(dz_t=1, dz=A) == OVERLAP    # fp32 in, 16 bits out: not in place
    assert call(db=A) == OVERLAP and call(db=C + 1024) == OVERLAP and call(m=8192, n=8192, dz=C, ws=C, ws_bytes=1 << 30) == OVERLAP
    assert call(m=0, dz=None, db=None) == NULL and call(n=0) == OK and call(m=0, db=None) == OK


def _tensor(b, **kw):
    t = b.AdamWTensor(count=1024, dtype=0, grad_dtype=0, param_dev=A, grad_dev=B, exp_avg_dev=C, exp_avg_sq_dev=D)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def test_adamw_refusals(b):
    so = b.load_library()
    handle, size = ctypes.c_void_p(5), ctypes.c_size_t(0)
    perm = (ctypes.c_int32 * 4)(0, 1, 2, 2)
    at = ctypes.addressof(perm)

    def create(*tensors, bits=32, ws=F, ws_bytes=1 << 20):
        table = (b.AdamWTensor * max(len(tensors), 1))(*tensors)
        st = so.bsr_adamw_create(ctypes.byref(handle), len(tensors), table, bits, ws, ws_bytes, None)
        assert st != OK and handle.value is None
        return st

    def needs(*tensors, bits=32):
        st = so.bsr_adamw_workspace_size(len(tensors), (b.AdamWTensor * max(len(tensors), 1))(*tensors), bits, ctypes.byref(size))
        return st if st else size.value

    t = lambda **kw: _tensor(b, **kw)  # noqa: E731
    assert needs() == 256 and needs(t()) % 256 == 0 and needs(t(count=1 << 20)) > needs(t())
    assert needs(t(count=-1)) == SHAPE and needs(t(count=1 << 37)) == SHAPE and needs(t(), bits=16) == DTYPE
    assert so.bsr_adamw_workspace_size(1, None, 32, ctypes.byref(size)) == NULL and so.bsr_adamw_workspace_size(1, None, 32, None) == NULL
    assert so.bsr_adamw_create(None, 0, None, 32, F, 256, None) == NULL
    assert create(t(dtype=3)) == DTYPE and create(t(grad_dtype=1)) == DTYPE and create(t(dtype=1, grad_dtype=2)) == DTYPE
    assert create(t(master_dev=E)) == DTYPE                                                   # a copy in fp32 of fp32
    assert create(t(), ws=None) == NULL and create(t(), ws=F + 8) == ALIGN and create(t(), ws_bytes=64) == WORKSPACE
    for k in ("param_dev", "grad_dev", "exp_avg_dev", "exp_avg_sq_dev"):
        assert create(t(**{k: None})) == NULL and create(t(**{k: E + 4})) == ALIGN
    assert create(t(), bits=8) == NULL and create(t(scales_dev=E + 2), bits=8) == ALIGN       # scales
    assert create(t(grad_dev=A)) == OVERLAP and create(t(exp_avg_sq_dev=C + 4080)) == OVERLAP and create(t(), ws=A) == OVERLAP
    assert create(t(), t(param_dev=E, exp_avg_dev=E + 8192, exp_avg_sq_dev=E + 16384, grad_dev=D)) == OVERLAP
    assert create(t(bs_r=16, bs_c=16, t_param_dev=E)) == NULL                                 # no perm
    assert create(t(bs_r=16, bs_c=16, t_param_dev=E, t_perm_host=at)) == INDEX                # 2 twice
    assert create(t(bs_r=16, bs_c=17, t_param_dev=E, t_perm_host=at)) == SHAPE and create(t(bs_r=0, bs_c=16, t_param_dev=E, t_perm_host=at)) == SHAPE
    assert create(t(count=201 * 201, bs_r=201, bs_c=201, t_param_dev=E, t_perm_host=at)) == UNSUPPORTED
    assert create(t(bs_r=16, bs_c=16, t_param_dev=A, t_perm_host=at)) == OVERLAP
    hyper = b.AdamWHyper(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, grad_scale=1.0)
    assert so.bsr_adamw_step(None, ctypes.byref(hyper), None) == NULL
    assert so.bsr_adamw_moments(None, 0, None, None, None) == NULL
    so.bsr_adamw_destroy(None)
    assert b.bsr_status_string(OVERLAP) != b.bsr_status_string(99) and b.bsr_status_string(12) != b.bsr_status_string(99)
