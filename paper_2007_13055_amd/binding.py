"""Binding for libbsr_spmm.so: same names as the C entry points, marshalling only.

What is called once a product or a step (bsr_spmm, bsr_spmm_ex, bsr_spmm_static, bsr_spmm_epilogue, bsr_epilogue_backward,
bsr_spmm_gated, bsr_gated_backward, bsr_residual_norm, bsr_residual_norm_backward, bsr_sddmm, bsr_adamw_step, bsr_adamw_moments,
bsr_muon_step) goes through the native module _binding, whose calls cost about what the launch
itself does; everything called once per matrix goes through ctypes."""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libbsr_spmm.so")

BSR_F32, BSR_F16, BSR_BF16 = 0, 1, 2
PATH_AUTO, PATH_WAVE, PATH_MFMA = 0, 1, 2
_DTYPE_CODE = {"f32": BSR_F32, "f16": BSR_F16, "bf16": BSR_BF16}



class Epilogue(ctypes.Structure):
    """bsr_epilogue of the C header."""
    _fields_ = [("act", ctypes.c_int), ("bias_dtype", ctypes.c_int), ("bias_dev", ctypes.c_void_p),
                ("residual_dev", ctypes.c_void_p), ("residual_ld", ctypes.c_int64), ("through_dev", ctypes.c_void_p),
                ("z_dev", ctypes.c_void_p)]


class AdamWTensor(ctypes.Structure):
    """bsr_adamw_tensor of the C header."""
    _fields_ = [("count", ctypes.c_int64), ("dtype", ctypes.c_int), ("grad_dtype", ctypes.c_int),
                ("param_dev", ctypes.c_void_p), ("master_dev", ctypes.c_void_p), ("grad_dev", ctypes.c_void_p),
                ("exp_avg_dev", ctypes.c_void_p), ("exp_avg_sq_dev", ctypes.c_void_p), ("scales_dev", ctypes.c_void_p),
                ("weight_decay", ctypes.c_float), ("bs_r", ctypes.c_int32), ("bs_c", ctypes.c_int32),
                ("t_param_dev", ctypes.c_void_p), ("t_perm_host", ctypes.c_void_p)]


class AdamWHyper(ctypes.Structure):
    """bsr_adamw_hyper of the C header."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("step", ctypes.c_int64), ("grad_scale", ctypes.c_float), ("seed", ctypes.c_uint32),
                ("lr_dev", ctypes.c_void_p), ("step_dev", ctypes.c_void_p), ("grad_scale_dev", ctypes.c_void_p)]


class Gated(ctypes.Structure):
    """bsr_gated of the C header."""
    _fields_ = [("act", ctypes.c_int), ("bias_dtype", ctypes.c_int), ("bias_dev", ctypes.c_void_p), ("z_dev", ctypes.c_void_p)]


class Residual(ctypes.Structure):
    """bsr_residual of the C header."""
    _fields_ = [("post", ctypes.c_int), ("pre", ctypes.c_int), ("w_dtype", ctypes.c_int), ("post_weight_dev", ctypes.c_void_p),
                ("post_bias_dev", ctypes.c_void_p), ("gate_dev", ctypes.c_void_p), ("pre_weight_dev", ctypes.c_void_p),
                ("pre_bias_dev", ctypes.c_void_p), ("eps", ctypes.c_double), ("stream_scale", ctypes.c_float), ("branch_scale", ctypes.c_float)]


class ResidualGrads(ctypes.Structure):
    """bsr_residual_grads of the C header."""
    _fields_ = [("post_weight_dev", ctypes.c_void_p), ("post_bias_dev", ctypes.c_void_p), ("gate_dev", ctypes.c_void_p),
                ("pre_weight_dev", ctypes.c_void_p), ("pre_bias_dev", ctypes.c_void_p)]


class MuonTensor(ctypes.Structure):
    """bsr_muon_tensor of the C header."""
    _fields_ = [("blocks", ctypes.c_int64), ("bs_r", ctypes.c_int32), ("bs_c", ctypes.c_int32), ("dtype", ctypes.c_int), ("grad_dtype", ctypes.c_int),
                ("param_dev", ctypes.c_void_p), ("master_dev", ctypes.c_void_p), ("grad_dev", ctypes.c_void_p), ("momentum_dev", ctypes.c_void_p),
                ("t_param_dev", ctypes.c_void_p), ("t_perm_host", ctypes.c_void_p), ("weight_decay", ctypes.c_float), ("scale", ctypes.c_float)]


class MuonHyper(ctypes.Structure):
    """bsr_muon_hyper of the C header."""
    _fields_ = [("lr", ctypes.c_double), ("momentum", ctypes.c_double), ("eps", ctypes.c_double), ("a", ctypes.c_float), ("b", ctypes.c_float),
                ("c", ctypes.c_float), ("ns_steps", ctypes.c_int32), ("nesterov", ctypes.c_int32), ("step", ctypes.c_int64),
                ("grad_scale", ctypes.c_float), ("seed", ctypes.c_uint32), ("lr_dev", ctypes.c_void_p), ("step_dev", ctypes.c_void_p),
                ("grad_scale_dev", ctypes.c_void_p)]


_lib = None
_native = None                             # the module _binding, bound to _lib


class BsrError(RuntimeError):
    """A C entry point returned a status other than BSR_OK."""

    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__(f"{where}: {bsr_status_string(status)} (status {int(status)})")


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load the built library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2007_13055_amd.build` "
                           "(or __graft_entry__.build()); there is no CPU fallback")
    lib = ctypes.CDLL(_LIB_PATH)
    i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
    lib.bsr_validate.argtypes = [i64, i64, i32, i32, i64, vp, vp]
    lib.bsr_workspace_size.argtypes = [i64, i64, i32, i32, i64, ctypes.POINTER(sz)]
    lib.bsr_create.argtypes = [ctypes.POINTER(vp), i64, i64, i32, i32, i64, ctypes.c_int, vp, vp, vp, vp, vp,
                               vp, sz, vp]
    lib.bsr_destroy.argtypes = [vp]
    lib.bsr_destroy.restype = None
    lib.bsr_spmm.argtypes = [vp, i64, vp, vp, ctypes.c_int, vp]
    lib.bsr_spmm_ex.argtypes = [vp, i64, vp, vp, ctypes.c_int, ctypes.c_int, vp]
    lib.bsr_spmm_static.argtypes = [vp, i64, vp, vp, ctypes.c_int, vp]
    lib.bsr_query_path.argtypes = [vp, i64, ctypes.POINTER(ctypes.c_int)]
    lib.bsr_tune.argtypes = [vp, i64, vp, vp, ctypes.c_int, ctypes.c_int, vp, ctypes.POINTER(ctypes.c_int),
                             ctypes.POINTER(ctypes.c_float)]
    lib.bsr_tune_result.argtypes = [vp, i64, ctypes.c_int, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_float)]
    lib.bsr_scratch_size.argtypes = [vp, i64, ctypes.POINTER(sz)]
    lib.bsr_set_scratch.argtypes = [vp, vp, sz]
    lib.bsr_transpose_pattern.argtypes = [i64, i64, i32, i32, i64, vp, vp, vp, vp, vp]
    lib.bsr_transpose_values.argtypes = [ctypes.c_int, i32, i32, i64, vp, vp, vp, vp]
    lib.bsr_sddmm.argtypes = [vp, i64, vp, vp, vp, ctypes.c_int, vp]
    lib.bsr_spmm_epilogue.argtypes = [vp, i64, vp, vp, ctypes.c_int, ctypes.POINTER(Epilogue), vp]
    lib.bsr_epilogue_backward_workspace_size.argtypes = [i64, i64, ctypes.POINTER(sz)]
    lib.bsr_epilogue_backward.argtypes = [i64, i64, ctypes.c_int, ctypes.c_int, vp, vp, ctypes.c_int, vp, vp, vp, sz, vp]
    lib.bsr_adamw_workspace_size.argtypes = [i64, ctypes.POINTER(AdamWTensor), i32, ctypes.POINTER(sz)]
    lib.bsr_adamw_create.argtypes = [ctypes.POINTER(vp), i64, ctypes.POINTER(AdamWTensor), i32, vp, sz, vp]
    lib.bsr_adamw_step.argtypes = [vp, ctypes.POINTER(AdamWHyper), vp]
    lib.bsr_adamw_moments.argtypes = [vp, ctypes.c_int, ctypes.POINTER(vp), ctypes.POINTER(vp), vp]
    lib.bsr_adamw_destroy.argtypes = [vp]
    lib.bsr_adamw_destroy.restype = None
    lib.bsr_spmm_gated_workspace_size.argtypes = [vp, i64, ctypes.c_int, ctypes.POINTER(sz)]
    lib.bsr_spmm_gated.argtypes = [vp, i64, vp, vp, ctypes.c_int, ctypes.POINTER(Gated), vp, sz, vp]
    lib.bsr_gated_backward_workspace_size.argtypes = [i64, i64, i32, ctypes.POINTER(sz)]
    lib.bsr_gated_backward.argtypes = [i64, i64, i32, ctypes.c_int, ctypes.c_int, vp, vp, ctypes.c_int, vp, vp, vp, sz, vp]
    lib.bsr_residual_norm.argtypes = [i64, i64, ctypes.c_int, vp, ctypes.c_int, vp, vp, vp, ctypes.POINTER(Residual), vp]
    lib.bsr_residual_norm_backward_workspace_size.argtypes = [i64, i64, ctypes.POINTER(sz)]
    lib.bsr_residual_norm_backward.argtypes = [i64, i64, ctypes.c_int, vp, ctypes.c_int, vp, vp, vp, vp, vp, ctypes.POINTER(Residual),
                                               ctypes.POINTER(ResidualGrads), vp, sz, vp]
    lib.bsr_muon_workspace_size.argtypes = [i64, ctypes.POINTER(MuonTensor), ctypes.POINTER(sz)]
    lib.bsr_muon_create.argtypes = [ctypes.POINTER(vp), i64, ctypes.POINTER(MuonTensor), vp, sz, vp]
    lib.bsr_muon_step.argtypes = [vp, ctypes.POINTER(MuonHyper), vp]
    lib.bsr_muon_destroy.argtypes = [vp]
    lib.bsr_muon_destroy.restype = None
    lib.bsr_probe_mfma.argtypes = [ctypes.c_int, i32, vp, vp, ctypes.POINTER(ctypes.c_double)]
    lib.bsr_probe_mfma.restype = ctypes.c_int
    lib.bsr_status_string.argtypes = [ctypes.c_int]
    lib.bsr_status_string.restype = ctypes.c_char_p
    for f in ("bsr_validate", "bsr_workspace_size", "bsr_create", "bsr_spmm", "bsr_spmm_ex", "bsr_spmm_static",
              "bsr_query_path", "bsr_scratch_size", "bsr_set_scratch", "bsr_tune", "bsr_tune_result",
              "bsr_transpose_pattern", "bsr_transpose_values", "bsr_sddmm", "bsr_spmm_epilogue",
              "bsr_epilogue_backward_workspace_size", "bsr_epilogue_backward", "bsr_adamw_workspace_size", "bsr_adamw_create",
              "bsr_adamw_step", "bsr_adamw_moments", "bsr_spmm_gated_workspace_size", "bsr_spmm_gated", "bsr_gated_backward_workspace_size",
              "bsr_gated_backward", "bsr_residual_norm", "bsr_residual_norm_backward_workspace_size", "bsr_residual_norm_backward",
              "bsr_muon_workspace_size", "bsr_muon_create", "bsr_muon_step"):
        getattr(lib, f).restype = ctypes.c_int
    _lib = lib
    return lib


def _native_module():
    """The module _binding, bound to the library's entry points.  Only matrices need it (it needs torch); the checks of
    patterns and sizes do not."""
    global _native
    if _native is not None:
        return _native
    lib = load_library()
    import torch                           # noqa: F401  (_binding links to torch's libraries)
    try:
        from . import _binding
    except ImportError as e:
        raise RuntimeError(f"the native module _binding is missing or does not load ({e}): build it with "
                           "`python -m paper_2007_13055_amd.build`") from e
    _binding.bind(*(ctypes.cast(f, ctypes.c_void_p).value
                    for f in (lib.bsr_spmm_ex, lib.bsr_spmm_static, lib.bsr_sddmm_ws, lib.bsr_scratch_size,
                              lib.bsr_sddmm_workspace_size, lib.bsr_spmm_epilogue, lib.bsr_epilogue_backward,
                              lib.bsr_epilogue_backward_workspace_size, lib.bsr_adamw_step, lib.bsr_adamw_moments,
                              lib.bsr_spmm_gated, lib.bsr_spmm_gated_workspace_size, lib.bsr_gated_backward, lib.bsr_gated_backward_workspace_size,
                              lib.bsr_residual_norm, lib.bsr_residual_norm_backward, lib.bsr_residual_norm_backward_workspace_size,
                              lib.bsr_muon_step)), BsrError)
    _native = _binding
    return _native


def bsr_status_string(status: int) -> str:
    return load_library().bsr_status_string(int(status)).decode()


def _i32(a):
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32).reshape(-1))


def bsr_validate(n, k, bs_r, bs_c, index_pointer, block_indices) -> int:
    """Structural check on host arrays; returns the status code (0 = ok)."""
    ptr, idx = _i32(index_pointer), _i32(block_indices)
    return int(load_library().bsr_validate(n, k, bs_r, bs_c, idx.shape[0], ptr.ctypes.data,
                                           idx.ctypes.data if idx.size else None))


def bsr_workspace_size(n, k, bs_r, bs_c, nnzb) -> int:
    out = ctypes.c_size_t(0)
    st = load_library().bsr_workspace_size(n, k, bs_r, bs_c, nnzb, ctypes.byref(out))
    if st != 0:
        raise BsrError(st, "bsr_workspace_size")
    return int(out.value)


def _torch_dtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def _dtype_name(t):
    import torch
    return {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}[t.dtype]


class BsrMatrix:
    """Owns the device tensors of one W (they must outlive the C handle) and the handle itself.

    Products may run on any stream of its device, and it may be dropped while they are still to run.  A graph that one was
    captured into reads its buffers at every replay: it must outlive the graph."""

    def __init__(self, handle, n, k, bs_r, bs_c, dtype, tensors):
        self.handle, self.n, self.k, self.bs_r, self.bs_c, self.dtype = handle, n, k, bs_r, bs_c, dtype
        self._tensors = tensors            # block_data, block_indices, index_pointer, workspace (device)
        self._scratch = None               # device scratch lent to the handle (see ensure_scratch)
        nnzb = int(tensors[0].shape[0]) if tensors[0].dim() == 3 else 0
        import torch
        home = torch.cuda.current_stream()
        self._streams = {home.cuda_stream: home}   # the one its tensors were made on, the others that have been given products
        self._core = _native_module().Core(handle.value, n, k, nnzb, bs_r, bs_c, _DTYPE_CODE[dtype], home.cuda_stream)   # what the calls read

    def _on_stream(self, address):
        """A product on another stream than the last one, torch's current, is about to be queued: the memory of its plan is not
        to be used again before that has run, even if nothing else holds it by then."""
        if address in self._streams:
            return
        import torch
        stream = torch.cuda.current_stream(self._tensors[0].device)
        if stream.cuda_stream != address:
            return                         # another device's stream: not this allocator's business
        for t in (*self._tensors, self._scratch):
            if t is not None:
                t.record_stream(stream)
        self._streams[address] = stream

    @property
    def block_data(self):
        return self._tensors[0]

    def ensure_scratch(self, m: int):
        """Lend the handle enough scratch for a product with m rows (torch allocates it; grows only)."""
        import torch
        need = bsr_scratch_size(self, m)
        have = self._scratch.numel() if self._scratch is not None else 0
        if need > have:
            self._scratch = torch.empty(need, dtype=torch.uint8, device=self._tensors[0].device)
            for stream in self._streams.values():      # products on any of them may use it
                self._scratch.record_stream(stream)
            st = load_library().bsr_set_scratch(self.handle, self._scratch.data_ptr(), self._scratch.numel())
            if st != 0:
                raise BsrError(st, "bsr_set_scratch")
            self._core.lent(self._scratch.numel())

    def close(self):
        if self.handle:
            self._core.closed()
            load_library().bsr_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def bsr_create(n, k, block_data, block_indices, index_pointer, dtype=None, device="cuda") -> BsrMatrix:
    """Upload the three BSR arrays (numpy or torch) and build the handle.

    block_data (nnzb, bs_r, bs_c); dtype "f32" | "f16" | "bf16" selects the storage type the values
    are converted to on upload (they must already be exact in it); torch tensors keep their dtype.
    """
    import torch
    lib = load_library()
    _native_module()
    if isinstance(block_data, torch.Tensor):
        dtype = dtype or _dtype_name(block_data)
        data_dev = block_data.to(device=device, dtype=_torch_dtype(dtype)).contiguous()
    else:
        dtype = dtype or "f32"
        data_dev = torch.from_numpy(np.ascontiguousarray(block_data, dtype=np.float32)).to(
            device=device, dtype=_torch_dtype(dtype)).contiguous()
    if data_dev.dim() != 3:
        raise ValueError("block_data must be (nnzb, bs_r, bs_c)")
    nnzb, bs_r, bs_c = (int(v) for v in data_dev.shape)
    idx_h = _i32(block_indices.cpu().numpy() if isinstance(block_indices, torch.Tensor) else block_indices)
    ptr_h = _i32(index_pointer.cpu().numpy() if isinstance(index_pointer, torch.Tensor) else index_pointer)
    if idx_h.shape[0] != nnzb:
        raise ValueError("block_indices length differs from the number of stored blocks")
    if bs_r <= 0 or n % bs_r or ptr_h.shape[0] != n // bs_r + 1:
        raise BsrError(2 if (bs_r <= 0 or n % bs_r) else 3, "bsr_create")
    idx_dev = torch.from_numpy(idx_h).to(device) if nnzb else torch.zeros(4, dtype=torch.int32, device=device)
    ptr_dev = torch.from_numpy(ptr_h).to(device)
    if nnzb == 0:
        data_dev = torch.zeros(4, dtype=_torch_dtype(dtype), device=device)
    ws = torch.empty(bsr_workspace_size(n, k, bs_r, bs_c, nnzb), dtype=torch.uint8, device=device)
    handle = ctypes.c_void_p()
    stream = torch.cuda.current_stream().cuda_stream
    st = lib.bsr_create(ctypes.byref(handle), n, k, bs_r, bs_c, nnzb, _DTYPE_CODE[dtype],
                        data_dev.data_ptr(), idx_dev.data_ptr(), ptr_dev.data_ptr(),
                        idx_h.ctypes.data if nnzb else None, ptr_h.ctypes.data,
                        ws.data_ptr(), ws.numel(), stream)
    if st != 0:
        raise BsrError(st, "bsr_create")
    return BsrMatrix(handle, n, k, bs_r, bs_c, dtype, (data_dev, idx_dev, ptr_dev, ws))


def bsr_transpose_pattern(n, k, bs_r, bs_c, index_pointer, block_indices):
    """Pattern of W^T: (t_index_pointer, t_block_indices, perm) as int32 numpy arrays."""
    ptr, idx = _i32(index_pointer), _i32(block_indices)
    nnzb = int(idx.shape[0])
    if bs_c <= 0 or k % bs_c:
        raise BsrError(2, "bsr_transpose_pattern")
    t_ptr = np.zeros(k // bs_c + 1, dtype=np.int32)
    t_idx = np.zeros(max(nnzb, 1), dtype=np.int32)
    perm = np.zeros(max(nnzb, 1), dtype=np.int32)
    st = load_library().bsr_transpose_pattern(n, k, bs_r, bs_c, nnzb, ptr.ctypes.data, idx.ctypes.data if nnzb else None,
                                              t_ptr.ctypes.data, t_idx.ctypes.data, perm.ctypes.data)
    if st != 0:
        raise BsrError(st, "bsr_transpose_pattern")
    return t_ptr, t_idx[:nnzb], perm[:nnzb]


def bsr_create_transposed(n, k, block_data, block_indices, index_pointer, dtype=None, device="cuda") -> BsrMatrix:
    """Handle of W^T (k x n, blocks bs_c x bs_r) for the sibling product Z = G * W = bsr_spmm(W^T, G).
    Arguments as bsr_create (they describe W); the transposed values are computed on the device."""
    import torch
    if isinstance(block_data, torch.Tensor):
        dtype = dtype or _dtype_name(block_data)
        data_dev = block_data.to(device=device, dtype=_torch_dtype(dtype)).contiguous()
    else:
        dtype = dtype or "f32"
        data_dev = torch.from_numpy(np.ascontiguousarray(block_data, dtype=np.float32)).to(
            device=device, dtype=_torch_dtype(dtype)).contiguous()
    nnzb, bs_r, bs_c = (int(v) for v in data_dev.shape)
    t_ptr, t_idx, perm = bsr_transpose_pattern(n, k, bs_r, bs_c, index_pointer, block_indices)
    t_data = torch.empty((nnzb, bs_c, bs_r), dtype=data_dev.dtype, device=device)
    if nnzb:
        perm_dev = torch.from_numpy(perm).to(device)
        st = load_library().bsr_transpose_values(_DTYPE_CODE[dtype], bs_r, bs_c, nnzb, perm_dev.data_ptr(),
                                                 data_dev.data_ptr(), t_data.data_ptr(),
                                                 torch.cuda.current_stream().cuda_stream)
        if st != 0:
            raise BsrError(st, "bsr_transpose_values")
        torch.cuda.current_stream().synchronize()     # perm_dev and data_dev may be freed on return
    return bsr_create(k, n, t_data, t_idx, t_ptr, dtype=dtype, device=device)


def bsr_spmm_ex(W: BsrMatrix, X, Y=None, y_dtype=None, path=PATH_AUTO):
    """Y = X * W^T on torch's current stream; X (m, k) device tensor of W's dtype.  Returns Y."""
    return _native.spmm(W, W._core, X, Y, y_dtype, int(path))


def bsr_spmm(W: BsrMatrix, X, Y=None, y_dtype=None):
    return _native.spmm(W, W._core, X, Y, y_dtype, PATH_AUTO)


def bsr_spmm_epilogue(W: BsrMatrix, X, Y=None, y_dtype=None, *, bias=None, act="none", residual=None, through=None, Z=None,
                      keep_z=False):
    """Y = act(X W^T + bias) + residual, or (X W^T + bias) * act'(through) + residual, in the product's own launches.

    act "none" | "relu" | "gelu" | "gelu_tanh" | "silu"; bias (n,) of W's dtype or fp32; residual (m, n) of the result's
    type, its rows contiguous; through (m, n): the sums that the activation in front of the layer was given, whose slope the
    result is multiplied by.  Z: a buffer for the sums (bias added) before the activation; keep_z: a new one.  Returns Y, or
    (Y, Z) where Z or keep_z is given.  Y and Z must not overlap each other or an input."""
    return _native.spmm_epilogue(W, W._core, X, Y, y_dtype, bias, act, residual, through, Z, keep_z)


def bsr_epilogue_backward(G, Z=None, act="none", DZ=None, dz_dtype=None, DB=None, *, need_dz=True, need_db=True):
    """(DZ, DB) = (G * act'(Z), the sums of its columns in fp32): what bsr_spmm_epilogue's activation and bias have as
    gradients, from G = dL/dY and the Z that it kept.  dz_dtype: G's type, or any where G is fp32.  DZ may be G or Z itself.
    Without an activation dZ is G: G is returned unless its type changes or a DZ is given.  need_dz, need_db: leave out the
    one or the other (None in its place)."""
    return _native_module().epilogue_backward(G, Z, act, DZ, dz_dtype, DB, need_dz, need_db)


def bsr_gated_arrays(gate, up):
    """(block_data, block_indices, index_pointer) of the one matrix of 2n rows that holds two of the same block shape and sizes,
    a block-row of gate's and one of up's in turn (for bsr_create, bsr_create_transposed).  gate, up: such triples, numpy or
    torch; the blocks stay where and of the type that they are."""
    import torch
    halves, starts = [], []
    for data, idx, ptr in (gate, up):
        data = data if isinstance(data, torch.Tensor) else np.asarray(data)
        if data.ndim != 3:
            raise ValueError("block_data must be (nnzb, bs_r, bs_c)")
        idx, ptr = (_i32(v.cpu().numpy() if isinstance(v, torch.Tensor) else v) for v in (idx, ptr))
        if len(idx) != len(data) or len(ptr) < 1 or ptr[0] != 0 or ptr[-1] != len(idx) or np.any(np.diff(ptr) < 0):
            raise ValueError("index_pointer must start at 0, never decrease and end at the number of blocks")
        halves.append((data, idx, np.diff(ptr).astype(np.int64)))
        starts.append(ptr[:-1].astype(np.int64))
    (gd, gi, gc), (ud, ui, uc) = halves
    if gd.shape[1:] != ud.shape[1:] or gd.dtype != ud.dtype or isinstance(gd, torch.Tensor) != isinstance(ud, torch.Tensor) or len(gc) != len(uc):
        raise ValueError("gate and up must have the same block-rows, block shape and type")
    counts = np.stack((gc, uc), 1).reshape(-1)
    first = np.stack((starts[0], starts[1] + len(gi)), 1).reshape(-1)     # of each block-row, in gate's blocks and up's behind them
    ptr = np.zeros(len(counts) + 1, dtype=np.int32)
    np.cumsum(counts, out=ptr[1:])
    order = np.repeat(first - ptr[:-1], counts) + np.arange(int(ptr[-1]))
    idx = np.concatenate((gi, ui))[order]
    if isinstance(gd, torch.Tensor):
        return torch.cat((gd, ud))[torch.from_numpy(order).to(gd.device)], idx, ptr
    return np.concatenate((gd, ud))[order], idx, ptr


def bsr_spmm_gated(W: BsrMatrix, X, H=None, h_dtype=None, *, bias=None, act="silu", Z=None, keep_z=False):
    """H = act(X Wg^T + bias_g) * (X Wu^T + bias_u), H (m, n): W (2n, k) from bsr_gated_arrays, a block-row of Wg and one of Wu
    in turn; bias (2n,) in that order, of W's dtype or fp32.

    act "none" | "relu" | "gelu" | "gelu_tanh" | "silu".  Z: a buffer (m, 2n) of H's type for the sums, bias added, in W's order;
    keep_z: a new one.  Returns H, or (H, Z) where Z or keep_z is given.  H and Z must not overlap each other or an input."""
    return _native.spmm_gated(W, W._core, X, H, h_dtype, bias, act, Z, keep_z)


def bsr_gated_backward(G, Z, bs_r, act="silu", DZ=None, dz_dtype=None, DB=None, *, need_dz=True, need_db=True):
    """(DZ, DB), the gradients of bsr_spmm_gated's sums (in Z's order) and of its bias (fp32), from G = dL/dH (m, n) and the
    Z (m, 2n) that it kept; bs_r: W's.  dz_dtype: G's type, or any where G is fp32.  DZ may be Z itself.  need_dz, need_db: leave
    out the one or the other (None in its place)."""
    return _native_module().gated_backward(G, Z, bs_r, act, DZ, dz_dtype, DB, need_dz, need_db)


def bsr_residual_norm(S, B=None, *, post="none", pre="rms", post_weight=None, post_bias=None, gate=None, pre_weight=None, pre_bias=None, eps=1e-6,
                      stream_scale=1.0, branch_scale=1.0, out=None, U=None, u_dtype=None, need_sum=True):
    """(S', U): S' = stream_scale S + branch_scale gate post(B), U = pre(S'), row by row in one pass.

    S (m, n): the stream, fp32 or of B's type; B (m, n): what a block adds to it, or None (S' = stream_scale S).  post, pre:
    "none" | "rms" | "layer"; weights, biases and gate (n,), all of B's type or all fp32, or None.  out, U: buffers; out may be S
    itself, U B.  Without a B U is of u_dtype (S's type).  pre "none": no U (None).  need_sum: leave out S'.  Where S' is S -- no B, a
    stream_scale of 1, no out -- the tensor S itself is returned, not a copy."""
    return _native_module().residual_norm(S, B, post, pre, post_weight, post_bias, gate, pre_weight, pre_bias, eps, stream_scale, branch_scale, out, U,
                                          u_dtype, need_sum)


_VECTORS = ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")


def bsr_residual_norm_backward(S, B, GS, GU, *, post="none", pre="rms", post_weight=None, post_bias=None, gate=None, pre_weight=None, pre_bias=None,
                               eps=1e-6, stream_scale=1.0, branch_scale=1.0, DS=None, DB=None, need_ds=True, need_db=True, grads=None):
    """(DS, DB, grads): the gradients of bsr_residual_norm's S, B and vectors, from S = the S' that it gave, its B and settings,
    GS = dL/dS' (or None: zeros) and GU = dL/dU (or None).

    grads: None (a new fp32 tensor for each vector that is given) or a dict of names and (n,) fp32 tensors to fill; returned as
    a dict.  DS may be GS or S itself, DB GU or B.  need_ds, need_db: leave out the one or the other (None in its place)."""
    given = (post_weight, post_bias, gate, pre_weight, pre_bias)
    if grads is None:
        want = [None if v is None else True for v in given]
        if B is None:
            want[:3] = (None,) * 3
        if post == "none" or post is None:
            want[:2] = (None,) * 2
        if pre == "none" or pre is None:
            want[3:] = (None,) * 2
    else:
        if not set(grads) <= set(_VECTORS):
            raise ValueError(f"grads: names among {', '.join(_VECTORS)}")
        want = [grads.get(k) for k in _VECTORS]
    ds, db, sums = _native_module().residual_norm_backward(S, B, GS, GU, post, pre, *given, eps, stream_scale, branch_scale, DS, DB, need_ds, need_db, want)
    return ds, db, {k: v for k, v in zip(_VECTORS, sums) if v is not None}


STATIC_SCRATCH_BYTES = 8 << 20


def bsr_spmm_static(W: BsrMatrix, X, Y):
    """bsr_spmm for thin-block W on the library's built-in scratch array: nothing is allocated or lent, so Y
    must be given.  X (m, k) fp32, Y (m, n) fp32, both contiguous device tensors.  Returns Y."""
    return _native.spmm_static(W, W._core, X, Y)


def bsr_tune(W: BsrMatrix, X, Y=None, y_dtype=None, trials: int = 20):
    """Times the library's candidate kernels for this W, X.shape[0] and output type on torch's current
    stream and makes later bsr_spmm calls of that size use the fastest.  Returns (candidates tried,
    microseconds per product of the fastest).  Waits for the stream."""
    import torch
    if X.dim() != 2 or X.shape[1] != W.k or _dtype_name(X) != W.dtype or not X.is_contiguous():
        raise ValueError("X must be a contiguous (m, k) tensor of W's dtype")
    y_dtype = y_dtype or W.dtype
    m = int(X.shape[0])
    W.ensure_scratch(m)
    if Y is None:
        Y = torch.empty((m, W.n), dtype=_torch_dtype(y_dtype), device=X.device)
    elif tuple(Y.shape) != (m, W.n) or _dtype_name(Y) != y_dtype or not Y.is_contiguous():
        raise ValueError("Y must be a contiguous (m, n) tensor of y_dtype")
    tried, best = ctypes.c_int(0), ctypes.c_float(0.0)
    st = load_library().bsr_tune(W.handle, m, X.data_ptr(), Y.data_ptr(), _DTYPE_CODE[y_dtype], int(trials),
                                 torch.cuda.current_stream().cuda_stream, ctypes.byref(tried), ctypes.byref(best))
    if st != 0:
        raise BsrError(st, "bsr_tune")
    return int(tried.value), float(best.value)


def bsr_tune_result(W: BsrMatrix, m: int, y_dtype=None):
    """What bsr_tune remembered for (m, y_dtype): dict of settings and microseconds, or None."""
    out, us = (ctypes.c_int32 * 6)(), ctypes.c_float(0.0)
    st = load_library().bsr_tune_result(W.handle, m, _DTYPE_CODE[y_dtype or W.dtype], out, ctypes.byref(us))
    if st == 9:
        return None
    if st != 0:
        raise BsrError(st, "bsr_tune_result")
    keys = ("path", "variant", "nw", "mt", "a", "b")
    return {**{k: int(v) for k, v in zip(keys, out)}, "us": float(us.value)}


def bsr_sddmm(W: BsrMatrix, G, X, D=None, d_dtype=None, lend_scratch=True):
    """D[p] = G[:, block-row of p]^T @ X[:, block-column of p] for every stored block of W (the gradient
    of the block values); G (m, n), X (m, k) device tensors of W's dtype.  Returns D (nnzb, bs_r, bs_c).
    lend_scratch: lend the handle the scratch its thin-block kernel wants (as bsr_spmm does) and the product the memory
    its splits want; without, nothing is allocated but a D that is not given."""
    return _native.sddmm(W, W._core, G, X, D, d_dtype, lend_scratch)


def bsr_scratch_size(W: BsrMatrix, m: int) -> int:
    out = ctypes.c_size_t(0)
    st = load_library().bsr_scratch_size(W.handle, m, ctypes.byref(out))
    if st != 0:
        raise BsrError(st, "bsr_scratch_size")
    return int(out.value)


def bsr_query_path(W: BsrMatrix, m: int) -> int:
    out = ctypes.c_int(0)
    st = load_library().bsr_query_path(W.handle, m, ctypes.byref(out))
    if st != 0:
        raise BsrError(st, "bsr_query_path")
    return int(out.value)


class BsrAdamW:
    """Owns the tensors of one list (parameters, gradients, moments, ...; they must outlive the C handle) and the handle.

    Steps may run on any stream of its device, and it may be dropped while they are still to run.  A graph that a step was
    captured into reads its buffers at every replay: it must outlive the graph.

    params, grads, master, exp_avg, exp_avg_sq, scales: lists in the order given to bsr_adamw_create (None where a tensor has
    none)."""

    def __init__(self, state_bits, params, grads, master, exp_avg, exp_avg_sq, scales):
        self.state_bits, self.params, self.grads, self.master = state_bits, params, grads, master
        self.exp_avg, self.exp_avg_sq, self.scales = exp_avg, exp_avg_sq, scales
        self.handle, self.device, self._keep = None, None, []
        self._address, self._index, self._counts = 0, 0, tuple(int(p.numel()) for p in params)   # what the calls read
        self._known, self._streams = 0, set()   # the stream that was given work last; all, the one its buffers were made on first

    def _on_stream(self, address):
        """Work on another stream than the last one, torch's current, is about to be queued: its buffers' memory is not to be
        used again before that has run, even if nothing else holds them by then."""
        if address not in self._streams:
            import torch
            stream = torch.cuda.current_stream(self.device)
            for held in (self.params, self.grads, self.master, self.exp_avg, self.exp_avg_sq, self.scales, self._keep):
                for t in held:
                    if isinstance(t, torch.Tensor):
                        t.record_stream(stream)
            self._streams.add(address)
        self._known = address

    def close(self):
        if self.handle:
            self._address = 0
            load_library().bsr_adamw_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _adamw_buffer(t, what, dtypes, count, device):
    """t, checked: a contiguous tensor of `count` elements of one of the types on `device`."""
    if t.dtype not in dtypes or t.numel() != count or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{what} must be contiguous, of {count} elements of {' or '.join(map(str, dtypes))}, on {device}")
    return t


def bsr_adamw_create(params, grads, *, weight_decay=0.0, state_bits=32, moments=None, master=None, transposed=None) -> BsrAdamW:
    """The handle of AdamW steps over a list of tensors on the current GPU.

    params, grads: contiguous tensors of any shapes, f32, f16 or bf16; a gradient has its parameter's type or fp32 and is read
    by every step from where it is (let bsr_sddmm and bsr_epilogue_backward write there).  weight_decay: one number or one a
    tensor.  state_bits: 32 or 8 (e4m3 and logarithmic codes with scales for each 256 elements).  master: True (fp32 copies
    of the 16-bit parameters, made here) or a list of fp32 tensors and None; without one a 16-bit parameter is rounded at
    random so that its mean is kept.  moments: None (zeros), or per tensor (m, v) or, for 8 bits, (m codes, v codes, scales):
    fp32, or uint8 and (groups of 256, 3) fp32.  transposed: None, or per tensor None or (t, perm): the tensor is a W's
    block_data (stored blocks, bs_r, bs_c), t the handle or the block_data of its transpose, which every step brings up to
    date, perm from bsr_transpose_pattern."""
    import torch
    lib = load_library()
    _native_module()
    params, grads = list(params), list(grads)
    n = len(params)
    if len(grads) != n or (moments is not None and len(moments) != n) or (transposed is not None and len(transposed) != n) or \
            (isinstance(master, (list, tuple)) and len(master) != n):
        raise ValueError("one gradient (pair of moments, master copy, transpose) a parameter is wanted")
    if state_bits not in (32, 8):
        raise ValueError("state_bits must be 32 or 8")
    decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(v) for v in weight_decay]
    if len(decay) != n:
        raise ValueError("one weight_decay, or one a parameter, is wanted")
    device = torch.device("cuda", torch.cuda.current_device())
    f32 = torch.float32
    code, zeros = (torch.uint8, f32)[state_bits == 32], lambda count, dtype: torch.zeros(count, dtype=dtype, device=device)
    opt = BsrAdamW(state_bits, params, grads, [None] * n, [None] * n, [None] * n, [None] * n)
    opt.device = device
    table = (AdamWTensor * max(n, 1))()
    for i, (p, g) in enumerate(zip(params, grads)):
        count = p.numel()
        _adamw_buffer(p, f"params[{i}]", (f32, torch.float16, torch.bfloat16), count, device)
        _adamw_buffer(g, f"grads[{i}]", (p.dtype, f32), count, device)
        own = master[i] if isinstance(master, (list, tuple)) else (p.detach().to(f32, copy=True) if master and p.dtype != f32 else None)
        opt.master[i] = None if own is None else _adamw_buffer(own, f"master[{i}]", (f32,), count, device)
        groups = -(-count // 256)
        given = moments[i] if moments is not None else None
        if given is None:
            given = (zeros(count, code), zeros(count, code)) + ((zeros((groups, 3), f32),) if state_bits == 8 else ())
        if len(given) != (2 if state_bits == 32 else 3):
            raise ValueError(f"moments[{i}]: (m, v), for 8 bits (m, v, scales)")
        opt.exp_avg[i] = _adamw_buffer(given[0], f"moments[{i}][0]", (code,), count, device)
        opt.exp_avg_sq[i] = _adamw_buffer(given[1], f"moments[{i}][1]", (code,), count, device)
        if state_bits == 8:
            opt.scales[i] = _adamw_buffer(given[2], f"moments[{i}][2]", (f32,), 3 * groups, device)
        t = table[i]
        t.count, t.dtype, t.grad_dtype, t.weight_decay = count, _DTYPE_CODE[_dtype_name(p)], _DTYPE_CODE[_dtype_name(g)], decay[i]
        t.param_dev, t.grad_dev = p.data_ptr(), g.data_ptr()
        t.master_dev = None if own is None else own.data_ptr()
        t.exp_avg_dev, t.exp_avg_sq_dev = opt.exp_avg[i].data_ptr(), opt.exp_avg_sq[i].data_ptr()
        t.scales_dev = opt.scales[i].data_ptr() if state_bits == 8 else None
        turned = transposed[i] if transposed is not None else None
        if turned is not None:
            copy, perm = turned
            copy = copy.block_data if isinstance(copy, BsrMatrix) else copy
            if p.dim() != 3 or tuple(copy.shape) != (p.shape[0], p.shape[2], p.shape[1]):
                raise ValueError(f"transposed[{i}]: (stored blocks, bs_c, bs_r) for a parameter (stored blocks, bs_r, bs_c)")
            _adamw_buffer(copy, f"transposed[{i}]", (p.dtype,), count, device)
            perm = _i32(perm.cpu().numpy() if isinstance(perm, torch.Tensor) else perm)
            if perm.shape[0] != p.shape[0]:
                raise ValueError(f"transposed[{i}]: one entry of perm a stored block")
            if count:
                t.bs_r, t.bs_c, t.t_param_dev, t.t_perm_host = int(p.shape[1]), int(p.shape[2]), copy.data_ptr(), perm.ctypes.data
            opt._keep += [copy, perm]
    size = ctypes.c_size_t(0)
    st = lib.bsr_adamw_workspace_size(n, table, state_bits, ctypes.byref(size))
    if st != 0:
        raise BsrError(st, "bsr_adamw_workspace_size")
    workspace = torch.empty(size.value, dtype=torch.uint8, device=device)
    opt._keep.append(workspace)
    handle = ctypes.c_void_p()
    st = lib.bsr_adamw_create(ctypes.byref(handle), n, table, state_bits, workspace.data_ptr(), workspace.numel(),
                              torch.cuda.current_stream().cuda_stream)
    if st != 0:
        raise BsrError(st, "bsr_adamw_create")
    opt.handle, opt._address, opt._index = handle, handle.value, device.index
    opt._known = torch.cuda.current_stream().cuda_stream
    opt._streams.add(opt._known)
    return opt


def bsr_adamw_step(opt: BsrAdamW, step, *, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, grad_scale=1.0, seed=0):
    """One step on torch's current stream, updating opt's parameters, master copies, moments and transposes in place.

    step counts from 1.  step, lr and grad_scale may be GPU tensors of one int64, fp32 and fp32, which a step captured into a
    graph reads at every replay; a grad_scale of 0 skips the step, and so does a step below 1 on the GPU.  seed: of the random roundings."""
    _native.adamw_step(opt, opt._address, opt._index, opt._known, step, lr, betas[0], betas[1], eps, grad_scale, seed)


def bsr_adamw_moments(opt: BsrAdamW, dtype="f32", out=None):
    """[(m, v), ...]: the moments as values of `dtype` ("f32" | "f16" | "bf16"), whatever they are held in; out: such a list to
    fill (of one type, each entry a pair of tensors of a parameter's number of elements, apart from one another and from opt's own)."""
    if out is None:
        import torch
        new = lambda p: torch.empty(p.numel(), dtype=_torch_dtype(dtype), device=opt.device)  # noqa: E731
        out = [(new(p), new(p)) for p in opt.params]
    _native.adamw_moments(opt, opt._address, opt._index, opt._known, opt._counts, out if isinstance(out, list) else list(out))
    return out


class BsrMuon:
    """Owns the tensors of one list (parameters, gradients, momentum, ...; they must outlive the C handle) and the handle.

    Steps may run on any stream of its device, and it may be dropped while they are still to run.  A graph that a step was
    captured into reads its buffers at every replay: it must outlive the graph.

    params, grads, master, momentum: lists in the order given to bsr_muon_create (None where a tensor has none)."""

    def __init__(self, params, grads, master, momentum):
        self.params, self.grads, self.master, self.momentum = params, grads, master, momentum
        self.handle, self.device, self._keep = None, None, []
        self._address, self._index = 0, 0       # what the calls read
        self._known, self._streams = 0, set()   # the stream that was given work last; all, the one its buffers were made on first

    def _on_stream(self, address):
        """As BsrAdamW's."""
        if address not in self._streams:
            import torch
            stream = torch.cuda.current_stream(self.device)
            for held in (self.params, self.grads, self.master, self.momentum, self._keep):
                for t in held:
                    if isinstance(t, torch.Tensor):
                        t.record_stream(stream)
            self._streams.add(address)
        self._known = address

    def close(self):
        if self.handle:
            self._address = 0
            load_library().bsr_muon_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def bsr_muon_create(params, grads, *, weight_decay=0.0, momentum=None, master=None, transposed=None, scale=None) -> BsrMuon:
    """The handle of steps over a list of block_data tensors whose updates are orthogonalised block by block, on the current GPU.

    params, grads: contiguous (stored blocks, bs_r, bs_c), sides from 1 to 64, f32, f16 or bf16; a gradient has its parameter's
    type or fp32 and is read by every step from where it is (let bsr_sddmm write there).  weight_decay, scale: one number or one
    a tensor; scale is the update's, None: sqrt(max(1, bs_r / bs_c)).  momentum: None (zeros) or fp32 tensors.  master,
    transposed: as bsr_adamw_create's."""
    import torch
    lib = load_library()
    _native_module()
    params, grads = list(params), list(grads)
    n = len(params)
    one_each = lambda v: [float(v)] * n if isinstance(v, (int, float)) else [float(x) for x in v]  # noqa: E731
    for given in (grads, momentum, transposed, master if isinstance(master, (list, tuple)) else None):
        if given is not None and len(given) != n:
            raise ValueError("one gradient (momentum, master copy, transpose) a parameter is wanted")
    device = torch.device("cuda", torch.cuda.current_device())
    f32 = torch.float32
    for i, p in enumerate(params):
        if p.dim() != 3:
            raise ValueError(f"params[{i}] must be (stored blocks, bs_r, bs_c)")
    decay = one_each(weight_decay)
    scales = [max(1.0, p.shape[1] / max(p.shape[2], 1)) ** 0.5 for p in params] if scale is None else one_each(scale)
    if len(decay) != n or len(scales) != n:
        raise ValueError("one weight_decay (scale), or one a parameter, is wanted")
    opt = BsrMuon(params, grads, [None] * n, [None] * n)
    opt.device = device
    table = (MuonTensor * max(n, 1))()
    for i, (p, g) in enumerate(zip(params, grads)):
        count = p.numel()
        _adamw_buffer(p, f"params[{i}]", (f32, torch.float16, torch.bfloat16), count, device)
        _adamw_buffer(g, f"grads[{i}]", (p.dtype, f32), count, device)
        own = master[i] if isinstance(master, (list, tuple)) else (p.detach().to(f32, copy=True) if master and p.dtype != f32 else None)
        opt.master[i] = None if own is None else _adamw_buffer(own, f"master[{i}]", (f32,), count, device)
        held = momentum[i] if momentum is not None else torch.zeros(count, dtype=f32, device=device)
        opt.momentum[i] = _adamw_buffer(held, f"momentum[{i}]", (f32,), count, device)
        t = table[i]
        t.blocks, t.bs_r, t.bs_c = (int(v) for v in p.shape)
        t.dtype, t.grad_dtype, t.weight_decay, t.scale = _DTYPE_CODE[_dtype_name(p)], _DTYPE_CODE[_dtype_name(g)], decay[i], scales[i]
        t.param_dev, t.grad_dev, t.momentum_dev = p.data_ptr(), g.data_ptr(), opt.momentum[i].data_ptr()
        t.master_dev = None if own is None else own.data_ptr()
        turned = transposed[i] if transposed is not None else None
        if turned is not None:
            copy, perm = turned
            copy = copy.block_data if isinstance(copy, BsrMatrix) else copy
            if count and tuple(copy.shape) != (p.shape[0], p.shape[2], p.shape[1]):
                raise ValueError(f"transposed[{i}]: (stored blocks, bs_c, bs_r) for a parameter (stored blocks, bs_r, bs_c)")
            perm = _i32(perm.cpu().numpy() if isinstance(perm, torch.Tensor) else perm)
            if perm.shape[0] != p.shape[0]:
                raise ValueError(f"transposed[{i}]: one entry of perm a stored block")
            if count:
                _adamw_buffer(copy, f"transposed[{i}]", (p.dtype,), count, device)
                t.t_param_dev, t.t_perm_host = copy.data_ptr(), perm.ctypes.data
            opt._keep += [copy, perm]
    size = ctypes.c_size_t(0)
    st = lib.bsr_muon_workspace_size(n, table, ctypes.byref(size))
    if st != 0:
        raise BsrError(st, "bsr_muon_workspace_size")
    workspace = torch.empty(size.value, dtype=torch.uint8, device=device)
    opt._keep.append(workspace)
    handle = ctypes.c_void_p()
    st = lib.bsr_muon_create(ctypes.byref(handle), n, table, workspace.data_ptr(), workspace.numel(), torch.cuda.current_stream().cuda_stream)
    if st != 0:
        raise BsrError(st, "bsr_muon_create")
    opt.handle, opt._address, opt._index = handle, handle.value, device.index
    opt._known = torch.cuda.current_stream().cuda_stream
    opt._streams.add(opt._known)
    return opt


def bsr_muon_step(opt: BsrMuon, step, *, lr=0.02, momentum=0.95, nesterov=True, ns_steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7,
                  grad_scale=1.0, seed=0):
    """One step on torch's current stream, updating opt's parameters, master copies, momentum and transposes in place.

    coefficients: a, b, c of the Newton-Schulz steps X = a X + b (X X^T) X + c (X X^T)^2 X, of which there are ns_steps (0 to 16).
    The default's are those published for this step (K. Jordan and others, 2024), steep at 0: five steps bring singular values of
    0.003 to 1 times the norm to between 0.68 and 1.21, not to 1.
    step counts from 1 (for the random roundings).  step, lr and grad_scale may be GPU tensors of one int64, fp32 and fp32, which a
    step captured into a graph reads at every replay; a grad_scale of 0 skips the step, and so does a step below 1 on the GPU."""
    a, b, c = coefficients
    _native_module().muon_step(opt, opt._address, opt._index, opt._known, step, lr, momentum, nesterov, ns_steps, a, b, c, eps, grad_scale, seed)
