"""Refusals of the gated product's gradient, the norms around a block and the orthogonalised step that no GPU is needed for: they
are decided before any device call, here on made-up addresses.  And those of the gated product, on a made-up handle."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def b():
    from paper_2007_13055_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2007_13055_amd import build
        build.build()
    return binding


OK, NULL, SHAPE, INDEX, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED, OVERLAP = 0, 1, 2, 4, 5, 6, 7, 9, 11
A, B, C, D, E, F, G, H, I, J, K, L = (0x100000000 * i for i in range(1, 13))


def test_structures_follow_the_header(b):
    assert ctypes.sizeof(b.Gated) == 24 and b.Gated.z_dev.offset == 16
    assert ctypes.sizeof(b.Residual) == 72 and b.Residual.post_weight_dev.offset == 16 and b.Residual.branch_scale.offset == 68
    assert ctypes.sizeof(b.ResidualGrads) == 40
    assert ctypes.sizeof(b.MuonTensor) == 80 and b.MuonTensor.param_dev.offset == 24 and b.MuonTensor.scale.offset == 76
    assert ctypes.sizeof(b.MuonHyper) == 88 and b.MuonHyper.step.offset == 48 and b.MuonHyper.grad_scale_dev.offset == 80


def test_gated_product_of_no_matrix(b):
    so, size = b.load_library(), ctypes.c_size_t(7)
    assert so.bsr_spmm_gated(None, 4, A, B, 0, ctypes.byref(b.Gated()), C, 1 << 20, None) == NULL
    assert so.bsr_spmm_gated(None, 4, A, B, 0, None, C, 1 << 20, None) == NULL
    assert so.bsr_spmm_gated_workspace_size(None, 4, 0, ctypes.byref(size)) == NULL and size.value == 0
    assert so.bsr_spmm_gated_workspace_size(None, 4, 0, None) == NULL


def test_gated_product_over_a_handles_arrays(b, tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    exe, folder = str(tmp_path / "host_gated_driver"), os.path.dirname(b.library_path())
    subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2007_13055_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host_gated_driver.cpp"), "-L", folder, "-l:libbsr_spmm.so", "-Wl,-rpath," + folder, "-o", exe],
                   check=True, capture_output=True, timeout=600)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and "all refused" in out.stdout, out.stdout + out.stderr


def test_gated_backward_refusals(b):
    so, size = b.load_library(), ctypes.c_size_t(7)
    need = lambda m, n, u: so.bsr_gated_backward_workspace_size(m, n, u, ctypes.byref(size))  # noqa: E731
    assert need(8192, 4096, 16) == OK and size.value % 256 == 0 and size.value > 0
    assert need(1, 64, 16) == OK and size.value == 0
    assert need(-1, 64, 16) == SHAPE and need(1, 64, 0) == SHAPE and need(1, 64, 24) == SHAPE and need(1, 1 << 27, 16) == SHAPE
    assert so.bsr_gated_backward_workspace_size(1, 1, 1, None) == NULL
    call = lambda m=64, n=64, u=16, act=4, g_t=0, g=A, z=B, dz_t=0, dz=C, db=D, ws=E, ws_bytes=1 << 24: so.bsr_gated_backward(  # noqa: E731
        m, n, u, act, g_t, g, z, dz_t, dz, db, ws, ws_bytes, None)
    assert call(m=-1) == SHAPE and call(u=48) == SHAPE and call(u=-16) == SHAPE and call(m=1 << 30) == SHAPE and call(m=1 << 20, n=1 << 20) == SHAPE
    assert call(act=5) == DTYPE and call(act=-1) == DTYPE and call(g_t=3) == DTYPE and call(dz_t=7) == DTYPE and call(g_t=1, dz_t=2) == DTYPE and call(g_t=1, dz_t=0) == DTYPE
    assert call(g=None) == NULL and call(z=None) == NULL and call(dz=None, db=None) == NULL and call(m=0, dz=None, db=None) == NULL
    assert call(g=A + 8) == ALIGN and call(z=B + 4) == ALIGN and call(dz=C + 2) == ALIGN and call(db=D + 4) == ALIGN and call(ws=E + 8) == ALIGN
    assert call(m=8192, ws=None) == WORKSPACE and call(m=8192, ws_bytes=1024) == WORKSPACE
    assert call(dz=A) == OVERLAP and call(dz=B + 64) == OVERLAP and call(dz=B, dz_t=1) == OVERLAP and call(dz=A + 64 * 64 * 4 - 16) == OVERLAP
    assert call(db=A) == OVERLAP and call(db=C + 1024) == OVERLAP and call(m=8192, n=4096, ws=C, ws_bytes=1 << 30) == OVERLAP
    assert call(n=0) == OK and call(m=0, db=None) == OK


def _how(b, **kw):
    h = b.Residual(post=1, pre=1, w_dtype=0, eps=1e-6, stream_scale=1.0, branch_scale=1.0)
    for k, v in kw.items():
        setattr(h, k, v)
    return ctypes.byref(h)


def test_norm_refusals(b):
    so = b.load_library()
    call = lambda m=64, n=64, s_t=0, s=A, b_t=0, x=B, out=C, u=D, **kw: so.bsr_residual_norm(m, n, s_t, s, b_t, x, out, u, _how(b, **kw), None)  # noqa: E731
    assert so.bsr_residual_norm(4, 4, 0, A, 0, B, C, D, None, None) == NULL
    assert call(m=-1) == SHAPE and call(n=-1) == SHAPE and call(n=16385) == SHAPE and call(m=1 << 30) == SHAPE
    assert call(eps=-1e-9) == SHAPE and call(eps=float("nan")) == SHAPE
    assert call(s_t=3) == DTYPE and call(b_t=-1) == DTYPE and call(s_t=1, b_t=2) == DTYPE and call(s_t=1, b_t=0) == DTYPE and call(post=3) == DTYPE and call(pre=-1) == DTYPE
    assert call(w_dtype=1) == DTYPE and call(s_t=0, b_t=1, w_dtype=2) == DTYPE
    assert call(s=None) == NULL and call(out=None, u=None) == NULL and call(pre=0) == UNSUPPORTED
    assert call(s=A + 4) == ALIGN and call(x=B + 8) == ALIGN and call(out=C + 2) == ALIGN and call(u=D + 8) == ALIGN and call(gate_dev=E + 4) == ALIGN
    assert call(out=A + 16) == OVERLAP and call(u=B + 16) == OVERLAP and call(out=B) == OVERLAP and call(u=A) == OVERLAP and call(u=C) == OVERLAP
    assert call(b_t=1, u=A) == OVERLAP and call(gate_dev=C) == OVERLAP and call(pre_bias_dev=D + 64 * 64 * 4 - 16) == OVERLAP
    assert call(m=0) == OK and call(n=0) == OK


def test_norm_gradient_refusals(b):
    so, size = b.load_library(), ctypes.c_size_t(7)
    need = lambda m, n: so.bsr_residual_norm_backward_workspace_size(m, n, ctypes.byref(size))  # noqa: E731
    assert need(100, 100) == OK and size.value % 256 == 0 and size.value > 0
    small = size.value
    assert need(100, 16384) == OK and size.value > small and need(0, 5) == OK and size.value == 0 and need(4, 16385) == SHAPE and need(-1, 4) == SHAPE
    assert so.bsr_residual_norm_backward_workspace_size(4, 4, None) == NULL

    def call(m=64, n=64, s_t=0, s=A, b_t=0, x=B, gs=C, gu=D, ds=E, db=F, ws=G, ws_bytes=1 << 30, grads=None, **kw):
        g = b.ResidualGrads(**(grads or {}))
        return so.bsr_residual_norm_backward(m, n, s_t, s, b_t, x, gs, gu, ds, db, _how(b, **kw), ctypes.byref(g), ws, ws_bytes, None)

    gate = {"gate_dev": H}
    assert so.bsr_residual_norm_backward(4, 4, 0, A, 0, B, C, D, E, F, None, None, None, 0, None) == NULL
    assert call(m=-1) == SHAPE and call(n=16385) == SHAPE and call(s_t=1, b_t=2) == DTYPE and call(post=7) == DTYPE
    assert call(s=None) == NULL and call(ds=None, db=None) == NULL
    assert call(x=None) == UNSUPPORTED and call(x=None, db=None, grads=gate) == UNSUPPORTED and call(pre=0) == UNSUPPORTED
    assert call(post=0, grads={"post_bias_dev": H}) == UNSUPPORTED and call(pre=0, gu=None, grads={"pre_weight_dev": H}) == UNSUPPORTED
    assert call(gs=C + 4) == ALIGN and call(ds=E + 8) == ALIGN and call(grads={"gate_dev": H + 4}) == ALIGN and call(ws=G + 8, grads=gate) == ALIGN
    assert call(grads=gate, ws=None) == WORKSPACE and call(grads=gate, ws_bytes=64) == WORKSPACE and call(n=16384, ws=None) == WORKSPACE
    assert call(ds=B) == OVERLAP and call(ds=A + 16) == OVERLAP and call(db=C) == OVERLAP and call(db=E) == OVERLAP and call(db=D + 16) == OVERLAP
    assert call(grads=gate, ws=A) == OVERLAP and call(grads={"gate_dev": E}) == OVERLAP and call(grads={"gate_dev": H, "pre_bias_dev": H + 128}) == OVERLAP
    assert call(grads=gate, gate_dev=H) == OVERLAP and call(post_weight_dev=F) == OVERLAP and call(grads={"gate_dev": G}) == OVERLAP
    assert call(n=0) == OK


def _tensor(b, **kw):
    t = b.MuonTensor(blocks=4, bs_r=16, bs_c=16, dtype=0, grad_dtype=0, param_dev=A, grad_dev=B, momentum_dev=C, scale=1.0)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def test_muon_refusals(b):
    so = b.load_library()
    handle, size = ctypes.c_void_p(5), ctypes.c_size_t(0)
    perm = (ctypes.c_int32 * 4)(0, 1, 2, 2)
    at = ctypes.addressof(perm)

    def create(*tensors, ws=F, ws_bytes=1 << 20):
        table = (b.MuonTensor * max(len(tensors), 1))(*tensors)
        st = so.bsr_muon_create(ctypes.byref(handle), len(tensors), table, ws, ws_bytes, None)
        assert st != OK and handle.value is None
        return st

    def needs(*tensors):
        st = so.bsr_muon_workspace_size(len(tensors), (b.MuonTensor * max(len(tensors), 1))(*tensors), ctypes.byref(size))
        return st if st else size.value

    t = lambda **kw: _tensor(b, **kw)  # noqa: E731
    assert needs() == 256 and needs(t()) % 256 == 0 and needs(t(blocks=1 << 16)) > needs(t())
    assert needs(t(blocks=-1)) == SHAPE and needs(t(bs_r=65)) == SHAPE and needs(t(bs_c=0)) == SHAPE and needs(t(blocks=1 << 31)) == SHAPE and needs(t(blocks=1 << 28)) == SHAPE
    assert so.bsr_muon_workspace_size(1, None, ctypes.byref(size)) == NULL and so.bsr_muon_workspace_size(1, None, None) == NULL
    assert so.bsr_muon_create(None, 0, None, F, 256, None) == NULL
    assert create(t(dtype=3)) == DTYPE and create(t(grad_dtype=1)) == DTYPE and create(t(dtype=1, grad_dtype=2)) == DTYPE and create(t(master_dev=E)) == DTYPE
    assert create(t(), ws=None) == NULL and create(t(), ws=F + 8) == ALIGN and create(t(), ws_bytes=64) == WORKSPACE
    for k in ("param_dev", "grad_dev", "momentum_dev"):
        assert create(t(**{k: None})) == NULL and create(t(**{k: E + 4})) == ALIGN
    assert create(t(grad_dev=A)) == OVERLAP and create(t(momentum_dev=A + 4080)) == OVERLAP and create(t(), ws=A) == OVERLAP and create(t(), t(param_dev=E, momentum_dev=D)) != OVERLAP
    assert create(t(t_param_dev=E)) == NULL and create(t(t_param_dev=E, t_perm_host=at)) == INDEX and create(t(t_param_dev=A, t_perm_host=at)) == OVERLAP
    assert so.bsr_muon_step(None, ctypes.byref(b.MuonHyper()), None) == NULL
    so.bsr_muon_destroy(None)


def test_every_buffer_is_recorded_once_a_stream(monkeypatch):
    import torch
    from paper_2007_13055_amd.binding import BsrMuon
    calls = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: calls.append((id(t), s)))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "side")
    new = lambda: torch.zeros(4)  # noqa: E731
    opt = BsrMuon([new(), new()], [new(), new()], [new(), None], [new(), new()])
    copy, workspace = new(), new()
    opt._keep += [copy, np.arange(3), workspace]
    opt._on_stream(77)
    want = {id(t) for held in (opt.params, opt.grads, opt.momentum) for t in held} | {id(opt.master[0]), id(copy), id(workspace)}
    assert {t for t, _ in calls} == want and len(calls) == len(want)
    opt._on_stream(77)
    assert len(calls) == len(want)
    opt._on_stream(78)
    assert len(calls) == 2 * len(want)


def test_gated_arrays(b):
    """Block-rows in turn, gate's first; ragged and empty ones."""
    rng = np.random.default_rng(0)
    g = (rng.normal(size=(3, 2, 3)), np.array([1, 0, 2]), np.array([0, 2, 2, 3]))
    u = (rng.normal(size=(2, 2, 3)), np.array([0, 1]), np.array([0, 0, 1, 2]))
    data, idx, ptr = b.bsr_gated_arrays(g, u)
    assert ptr.tolist() == [0, 2, 2, 2, 3, 4, 5] and idx.tolist() == [1, 0, 0, 2, 1]
    assert np.array_equal(data, np.stack((g[0][0], g[0][1], u[0][0], g[0][2], u[0][1])))
    empty = (np.zeros((0, 2, 3)), np.zeros(0, np.int32), np.zeros(3, np.int32))
    data, idx, ptr = b.bsr_gated_arrays(empty, empty)
    assert data.shape == (0, 2, 3) and idx.size == 0 and ptr.tolist() == [0] * 5
    for bad in ((u[0][:1], u[1], u[2]), (u[0], u[1], u[2][:-1]), (u[0][:, :1], u[1], u[2]), (u[0].astype(np.float32), u[1], u[2]), (u[0], u[1], np.array([0, 2, 1, 2]))):
        with pytest.raises(ValueError):
            b.bsr_gated_arrays(g, bad)
