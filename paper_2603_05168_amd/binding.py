"""ctypes binding of libsbn.so: argument marshalling only (see include/sbn.h for semantics).

Every function takes torch tensors (or raw integers) for device buffers, passes their data
pointers and sizes straight to the C ABI on the current torch stream, and raises SbnError on a
non-zero status.  No step of the method runs here.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libsbn.so")

SBN_OK, SBN_EINVAL, SBN_EUNSUPPORTED, SBN_ESIZE, SBN_EALIGN, SBN_EHIP = 0, -1, -2, -3, -4, -5
SBN_F32, SBN_BF16 = 0, 1
SBN_PATH_AUTO, SBN_PATH_GEMV, SBN_PATH_SMFMAC, SBN_PATH_DENSE_MFMA, SBN_PATH_GENERIC = 0, 1, 2, 3, 4
SBN_OP_QUANTIZE_MASK_PACK, SBN_OP_LINEAR, SBN_OP_BACKWARD, SBN_OP_MASK_FLIPS = 0, 1, 2, 3

_STATUS_NAMES = {0: "SBN_OK", -1: "SBN_EINVAL", -2: "SBN_EUNSUPPORTED", -3: "SBN_ESIZE", -4: "SBN_EALIGN", -5: "SBN_EHIP"}


class SbnError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        super().__init__(f"{where}: {_STATUS_NAMES.get(status, status)} {detail}".strip())


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'` "
            "(hipcc, gfx950).  There is no fallback path.")
    lib = ctypes.CDLL(_LIB_PATH)
    i64, cint, vp, sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    pp = ctypes.POINTER(ctypes.c_void_p)
    pi64 = ctypes.POINTER(ctypes.c_int64)
    lib.sbn_last_error.restype = ctypes.c_char_p
    lib.sbn_last_error.argtypes = []
    lib.sbn_packed_bytes.restype = cint
    lib.sbn_packed_bytes.argtypes = [i64, i64, cint, cint, ctypes.POINTER(sz)]
    lib.sbn_workspace_bytes.restype = cint
    lib.sbn_workspace_bytes.argtypes = [cint, i64, i64, i64, cint, cint, ctypes.POINTER(sz)]
    lib.sbn_quantize_mask_pack.restype = cint
    lib.sbn_quantize_mask_pack.argtypes = [vp, cint, i64, i64, i64, cint, cint, vp, vp, vp, sz, vp]
    lib.sbn_quantize_mask_pack_batched.restype = cint
    lib.sbn_quantize_mask_pack_batched.argtypes = [cint, pp, cint, pi64, pi64, cint, cint, pp, pp, vp, sz, vp]
    lib.sbn_quantize_mask_pack_flips_batched.restype = cint
    lib.sbn_quantize_mask_pack_flips_batched.argtypes = [cint, pp, cint, pi64, pi64, cint, cint, pp, pp, vp, vp, sz, vp]
    lib.sbn_act_quant.restype = cint
    lib.sbn_act_quant.argtypes = [vp, i64, i64, vp, vp, vp]
    lib.sbn_sparse_ternary_linear.restype = cint
    lib.sbn_sparse_ternary_linear.argtypes = [vp, i64, i64, i64, cint, cint, vp, vp, vp, vp, vp, vp, vp, cint, vp, sz, vp]
    lib.sbn_sparse_ternary_linear_static.restype = cint
    lib.sbn_sparse_ternary_linear_static.argtypes = [vp, i64, i64, i64, cint, cint, vp, vp, vp, vp, vp, vp, vp, cint, vp]
    lib.sbn_sparse_ternary_linear_grouped.restype = cint
    lib.sbn_sparse_ternary_linear_grouped.argtypes = [cint, pp, pi64, pi64, pi64, cint, cint, pp, pp, pp, cint, vp, sz, vp]
    lib.sbn_sparse_ternary_linear_backward.restype = cint
    lib.sbn_sparse_ternary_linear_backward.argtypes = [vp, i64, i64, i64, cint, cint, vp, vp, vp, vp, vp, vp, cint, vp, sz, vp]
    lib.sbn_sparse_ternary_linear_backward_grouped.restype = cint
    lib.sbn_sparse_ternary_linear_backward_grouped.argtypes = [cint, pp, pi64, pi64, pi64, cint, cint, pp, pp, pp, pp, pp, pp, cint,
                                                               vp, sz, vp]
    lib.sbn_dense_ternary_linear.restype = cint
    lib.sbn_dense_ternary_linear.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp, vp, vp, vp]
    lib.sbn_unpack.restype = cint
    lib.sbn_unpack.argtypes = [vp, i64, i64, cint, cint, vp, vp, vp]
    lib.sbn_convert_packed.restype = cint
    lib.sbn_convert_packed.argtypes = [vp, i64, i64, cint, cint, cint, cint, vp, vp]
    lib.sbn_rmsnorm_act_quant.restype = cint
    lib.sbn_rmsnorm_act_quant.argtypes = [vp, i64, i64, vp, ctypes.c_float, vp, vp, vp, vp]
    lib.sbn_test_set_spin_limits.restype = None
    lib.sbn_test_set_spin_limits.argtypes = [cint, cint]
    lib.sbn_test_set_head_tiles.restype = None
    lib.sbn_test_set_head_tiles.argtypes = [cint, cint, cint]
    lib.sbn_test_chosen_mxfp4_tile.restype = cint
    lib.sbn_test_chosen_mxfp4_tile.argtypes = [i64, i64, i64, ctypes.POINTER(cint), pi64]
    lib.sbn_test_linear_kernel.restype = cint
    lib.sbn_test_linear_kernel.argtypes = [cint, cint, pp, pp, pi64, pi64, pi64, cint, cint, pp, pp, pp, pp, pp, vp]
    lib.sbn_test_self_kernel.restype = cint
    lib.sbn_test_self_kernel.argtypes = [cint, cint, pp, pi64, pi64, pi64, cint, cint, pp, pp, pp, pp, pp, vp]
    lib.sbn_test_takes_blocks.restype = cint
    lib.sbn_test_takes_blocks.argtypes = [cint, pi64, pi64, pi64, cint, cint, ctypes.POINTER(cint)]
    lib.sbn_test_forward_kernels.restype = cint
    lib.sbn_test_forward_kernels.argtypes = [cint, pp, pi64, pi64, pi64, cint, cint, pp, ctypes.POINTER(cint)]
    lib.sbn_test_chosen_kernels.restype = cint
    lib.sbn_test_chosen_kernels.argtypes = [cint, pi64, pi64, pi64, cint, cint, ctypes.POINTER(cint)]
    lib.sbn_head_workspace_bytes.restype = cint
    lib.sbn_head_workspace_bytes.argtypes = [i64, i64, i64, i64, cint, ctypes.POINTER(sz)]
    lib.sbn_head_cross_entropy.restype = cint
    lib.sbn_head_cross_entropy.argtypes = [vp, vp, vp, i64, i64, i64, vp, vp, vp, sz, vp]
    lib.sbn_head_cross_entropy_backward.restype = cint
    lib.sbn_head_cross_entropy_backward.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp, vp, vp, sz, vp]
    lib.sbn_head_distill.restype = cint
    lib.sbn_head_distill.argtypes = [vp, vp, vp, vp, cint, i64, ctypes.c_float, vp, i64, i64, i64, vp, vp, vp, vp, sz, vp]
    lib.sbn_head_distill_backward.restype = cint
    lib.sbn_head_distill_backward.argtypes = [vp, vp, vp, vp, cint, i64, ctypes.c_float, vp, vp, vp, vp, i64, i64, i64, vp, vp, vp, sz, vp]
    lib.sbn_mxfp4_bytes.restype = cint
    lib.sbn_mxfp4_bytes.argtypes = [i64, i64, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    lib.sbn_mxfp4_quantize.restype = cint
    lib.sbn_mxfp4_quantize.argtypes = [vp, cint, i64, i64, vp, vp, vp]
    lib.sbn_mxfp4_dequantize.restype = cint
    lib.sbn_mxfp4_dequantize.argtypes = [vp, vp, i64, i64, vp, cint, vp]
    lib.sbn_mxfp4_workspace_bytes.restype = cint
    lib.sbn_mxfp4_workspace_bytes.argtypes = [i64, i64, ctypes.POINTER(sz)]
    lib.sbn_mxfp4_linear.restype = cint
    lib.sbn_mxfp4_linear.argtypes = [vp, i64, i64, i64, vp, vp, vp, vp, vp, sz, vp]
    f32, f64, pvp = ctypes.c_float, ctypes.c_double, ctypes.POINTER(ctypes.c_float)
    for name, types in (("sbn_norm", [vp, vp, cint, i64, i64, vp, vp, f32, cint, vp, vp, vp]),
                        ("sbn_norm_workspace_bytes", [i64, i64, ctypes.POINTER(sz)]),
                        ("sbn_norm_backward", [vp, vp, vp, cint, i64, i64, vp, f32, cint, vp, vp, vp, vp, sz, vp]),
                        ("sbn_embedding", [vp, cint, i64, i64, vp, i64, f32, vp, cint, vp]),
                        ("sbn_embedding_workspace_bytes", [i64, i64, i64, ctypes.POINTER(sz)]),
                        ("sbn_embedding_backward", [vp, cint, vp, i64, i64, i64, f32, cint, vp, cint, vp, sz, vp]),
                        ("sbn_grad_norm_workspace_bytes", [cint, pi64, ctypes.POINTER(sz)]),
                        ("sbn_grad_norm", [cint, pp, cint, pi64, f32, vp, vp, sz, vp]),
                        ("sbn_adamw_state_bytes", [i64, ctypes.POINTER(sz), ctypes.POINTER(sz)]),
                        ("sbn_adamw_state_values", [vp, vp, i64, cint, vp, cint, vp]),
                        ("sbn_adamw_step", [cint, pp, cint, pp, cint, pp, pp, pp, pp, pi64, pvp, vp, vp, f64, f64, f64, vp, ctypes.POINTER(ctypes.c_uint64), vp])):
        getattr(lib, name).restype, getattr(lib, name).argtypes = cint, types
    lib.sbn_mask_flips.restype = cint
    lib.sbn_mask_flips.argtypes = [vp, vp, i64, i64, cint, cint, vp, vp, sz, vp]
    return lib


_lib = _load()


def _load_fastcall(path=os.path.join(_HERE, "_fastcall.so")):
    """The marshalling of the forward calls, the head's and the training step's in C++ (csrc/sbn_fastcall.cpp), or None where it was not built, or was built for
    another torch: the Python code here does the same."""
    if not os.path.exists(path):
        return None
    try:
        spec = importlib.util.spec_from_file_location("_fastcall", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError:
        return None
    if module.torch_version != torch.__version__:
        return None
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value   # noqa: E731
    module.bind(address(_lib.sbn_sparse_ternary_linear), address(_lib.sbn_sparse_ternary_linear_grouped))
    module.bind_head(*(address(f) for f in (
        _lib.sbn_head_cross_entropy, _lib.sbn_head_cross_entropy_backward, _lib.sbn_head_distill, _lib.sbn_head_distill_backward, _lib.sbn_mxfp4_quantize,
        _lib.sbn_mxfp4_dequantize, _lib.sbn_mxfp4_linear, _lib.sbn_head_workspace_bytes, _lib.sbn_mxfp4_bytes, _lib.sbn_mxfp4_workspace_bytes)))
    module.bind_step(*(address(f) for f in (
        _lib.sbn_norm, _lib.sbn_norm_backward, _lib.sbn_embedding, _lib.sbn_embedding_backward, _lib.sbn_grad_norm, _lib.sbn_adamw_step, _lib.sbn_adamw_state_values,
        _lib.sbn_norm_workspace_bytes, _lib.sbn_embedding_workspace_bytes)))
    return module


_fastcall = _load_fastcall()
_fast_linear = _fastcall.linear if _fastcall else lambda *args: None
_fast_grouped = _fastcall.grouped if _fastcall else lambda *args: None


def _fast(name):
    """A call in C++: its status, or None where the Python code beside it is to do it."""
    return getattr(_fastcall, name) if _fastcall else lambda *args: None


_fast_head_ce, _fast_head_ce_backward = _fast("head_ce"), _fast("head_ce_backward")
_fast_head_distill, _fast_head_distill_backward = _fast("head_distill"), _fast("head_distill_backward")
_fast_mxfp4_quantize, _fast_mxfp4_dequantize, _fast_mxfp4_linear = _fast("mxfp4_quantize"), _fast("mxfp4_dequantize"), _fast("mxfp4_linear")
_fast_norm, _fast_norm_backward, _fast_embedding, _fast_embedding_backward = _fast("norm"), _fast("norm_backward"), _fast("embedding"), _fast("embedding_backward")
_fast_grad_norm, _fast_adamw, _fast_state_values = _fast("grad_norm"), _fast("adamw"), _fast("state_values")
_fast_norm_bytes, _fast_embedding_bytes, _fast_gather = _fast("norm_bytes"), _fast("embedding_bytes"), _fast("gather")
_fast_head_bytes, _fast_mxfp4_bytes, _fast_mxfp4_workspace_bytes = _fast("head_bytes"), _fast("mxfp4_bytes"), _fast("mxfp4_workspace_bytes")


def lib_path() -> str:
    return _LIB_PATH


def _ptr(t):
    """Device (or host) address of a tensor, an int address, or None; the declared argument types turn it into a pointer."""
    return t if t is None or isinstance(t, int) else t.data_ptr()


# The stream of the current device, asked of torch without the Stream object around it: a decode call is 4 us of GPU time, and
# torch.cuda.current_stream() with torch.cuda.is_available() in front took 3.3 us of it on the host, this takes 0.3.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    if not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    if _raw_stream is None or _current_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_current_device())


def _check(status: int, where: str):
    if status != SBN_OK:
        detail = _lib.sbn_last_error().decode() if status == SBN_EHIP else ""
        raise SbnError(status, where, detail)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return SBN_BF16
    if t.dtype == torch.float32:
        return SBN_F32
    raise TypeError("latent weights must be bf16 or fp32")


def sbn_last_error() -> str:
    return _lib.sbn_last_error().decode()


def sbn_packed_bytes(d_out: int, d_in: int, N: int, M: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.sbn_packed_bytes(d_out, d_in, N, M, ctypes.byref(out)), "sbn_packed_bytes")
    return out.value


def sbn_workspace_bytes(op: int, tokens: int, d_out: int, d_in: int, N: int, M: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.sbn_workspace_bytes(op, tokens, d_out, d_in, N, M, ctypes.byref(out)), "sbn_workspace_bytes")
    return out.value


def sbn_quantize_mask_pack(W_latent, N: int, M: int, packed, gamma, workspace, ld_w: int | None = None):
    d_out, d_in = W_latent.shape
    ld = W_latent.stride(0) if ld_w is None else ld_w
    _check(_lib.sbn_quantize_mask_pack(_ptr(W_latent), _dtype_code(W_latent), d_out, d_in, ld, N, M, _ptr(packed),
                                       _ptr(gamma), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                       _stream()), "sbn_quantize_mask_pack")


def _ptr_array(tensors):
    arr = (ctypes.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = None if t is None else (t.data_ptr() if not isinstance(t, int) else t)
    return arr


def _i64_array(values):
    arr = (ctypes.c_int64 * len(values))()
    for i, v in enumerate(values):
        arr[i] = int(v)
    return arr


class PackBatch:
    """Host-side argument arrays of sbn_quantize_mask_pack_batched, marshalled once and reusable."""

    def __init__(self, W_list, N, M, packed_list, gamma_list, workspace, flips_out=None):
        self.flips_out = flips_out   # int64 device tensor of len(W_list): pack in place over the old forms and count flips
        self.count = len(W_list)
        self.dtype = _dtype_code(W_list[0])
        self.W = _ptr_array(W_list)
        self.d_out = _i64_array([w.shape[0] for w in W_list])
        self.d_in = _i64_array([w.shape[1] for w in W_list])
        self.packed = _ptr_array(packed_list)
        self.gamma = _ptr_array(gamma_list)
        self.N, self.M = N, M
        self.workspace = workspace
        self.keep = (W_list, packed_list, gamma_list)

    def run(self):
        ws = self.workspace
        if self.flips_out is not None:
            _check(_lib.sbn_quantize_mask_pack_flips_batched(self.count, self.W, self.dtype, self.d_out, self.d_in, self.N,
                                                             self.M, self.packed, self.gamma, _ptr(self.flips_out), _ptr(ws),
                                                             ws.numel() * ws.element_size(), _stream()),
                   "sbn_quantize_mask_pack_flips_batched")
            return
        _check(_lib.sbn_quantize_mask_pack_batched(self.count, self.W, self.dtype, self.d_out, self.d_in, self.N,
                                                   self.M, self.packed, self.gamma, _ptr(ws),
                                                   ws.numel() * ws.element_size(), _stream()),
               "sbn_quantize_mask_pack_batched")


def sbn_quantize_mask_pack_batched(W_list, N: int, M: int, packed_list, gamma_list, workspace):
    PackBatch(W_list, N, M, packed_list, gamma_list, workspace).run()


def sbn_quantize_mask_pack_flips_batched(W_list, N: int, M: int, packed_list, gamma_list, flips_out, workspace):
    """Packs in place over the previous packed forms; flips_out (int64 device tensor, one per matrix) gets the mask flips."""
    PackBatch(W_list, N, M, packed_list, gamma_list, workspace, flips_out).run()


def sbn_act_quant(X, xq, sx):
    tokens, d_in = X.shape
    if X.dtype != torch.bfloat16:
        raise TypeError("X must be bf16")
    _check(_lib.sbn_act_quant(_ptr(X), tokens, d_in, _ptr(xq), _ptr(sx), _stream()), "sbn_act_quant")


def sbn_sparse_ternary_linear(X, packed, gamma, Y, N: int, M: int, workspace, bias=None, xq_out=None, sx_out=None,
                              acc_out=None, path: int = SBN_PATH_AUTO):
    """X = None runs on activations already quantized into xq_out / sx_out (then inputs)."""
    status = _fast_linear(X, packed, gamma, Y, N, M, workspace, bias, xq_out, sx_out, acc_out, path)
    if status is not None:
        if status:
            _check(status, "sbn_sparse_ternary_linear")
        return
    tokens, d_in = X.shape if X is not None else xq_out.shape
    d_out = Y.shape[1]
    if (X is not None and X.dtype != torch.bfloat16) or Y.dtype != torch.float32:
        raise TypeError("X must be bf16 and Y fp32")
    _check(_lib.sbn_sparse_ternary_linear(_ptr(X), tokens, d_in, d_out, N, M, _ptr(packed), _ptr(gamma), _ptr(bias),
                                          _ptr(Y), _ptr(xq_out), _ptr(sx_out), _ptr(acc_out), path, _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream()),
           "sbn_sparse_ternary_linear")


SBN_STATIC_SCRATCH_MIB = 16


def sbn_sparse_ternary_linear_static(X, packed, gamma, Y, N: int, M: int, bias=None, xq_out=None, sx_out=None, acc_out=None,
                                     path: int = SBN_PATH_AUTO):
    """sbn_sparse_ternary_linear on the library's own scratch: no workspace argument, nothing allocated."""
    tokens, d_in = X.shape if X is not None else xq_out.shape
    d_out = Y.shape[1]
    if (X is not None and X.dtype != torch.bfloat16) or Y.dtype != torch.float32:
        raise TypeError("X must be bf16 and Y fp32")
    status = _lib.sbn_sparse_ternary_linear_static(_ptr(X), tokens, d_in, d_out, N, M, _ptr(packed), _ptr(gamma), _ptr(bias),
                                                   _ptr(Y), _ptr(xq_out), _ptr(sx_out), _ptr(acc_out), path, _stream())
    if status != SBN_OK:
        raise SbnError(status, "sbn_sparse_ternary_linear_static", _lib.sbn_last_error().decode() if status in (SBN_EHIP, SBN_ESIZE) else "")


class LinearGroup:
    """Host-side argument arrays of sbn_sparse_ternary_linear_grouped, marshalled once and reusable."""

    def __init__(self, X_list, packed_list, gamma_list, Y_list, N, M, workspace, path=SBN_PATH_AUTO):
        self.count = len(X_list)
        self.X = _ptr_array(X_list)
        self.tokens = _i64_array([x.shape[0] for x in X_list])
        self.d_in = _i64_array([x.shape[1] for x in X_list])
        self.d_out = _i64_array([y.shape[1] for y in Y_list])
        self.packed = _ptr_array(packed_list)
        self.gamma = _ptr_array(gamma_list)
        self.Y = _ptr_array(Y_list)
        self.N, self.M, self.path, self.workspace = N, M, path, workspace
        self.keep = (X_list, packed_list, gamma_list, Y_list)

    def run(self):
        ws = self.workspace
        status = _fast_grouped(self.count, self.X, self.tokens, self.d_in, self.d_out, self.N, self.M, self.packed, self.gamma, self.Y,
                               self.path, ws)
        if status is not None:
            if status:
                _check(status, "sbn_sparse_ternary_linear_grouped")
            return
        _check(_lib.sbn_sparse_ternary_linear_grouped(self.count, self.X, self.tokens, self.d_in, self.d_out, self.N,
                                                      self.M, self.packed, self.gamma, self.Y, self.path, _ptr(ws),
                                                      ws.numel() * ws.element_size(), _stream()),
               "sbn_sparse_ternary_linear_grouped")


def sbn_sparse_ternary_linear_grouped(X_list, packed_list, gamma_list, Y_list, N, M, workspace, path=SBN_PATH_AUTO):
    LinearGroup(X_list, packed_list, gamma_list, Y_list, N, M, workspace, path).run()


SBN_BWD_ACCUMULATE, SBN_BWD_MASK_DW = 1, 2


def sbn_sparse_ternary_linear_backward(dY, packed, gamma, xq, sx, N: int, M: int, workspace, d_in: int, dX=None, dW=None,
                                       accumulate: bool = False, mask_dw: bool = False):
    tokens, d_out = dY.shape
    if dY.dtype != torch.bfloat16:
        raise TypeError("dY must be bf16")
    _check(_lib.sbn_sparse_ternary_linear_backward(_ptr(dY), tokens, d_in, d_out, N, M, _ptr(packed), _ptr(gamma),
                                                   _ptr(xq), _ptr(sx), _ptr(dX), _ptr(dW),
                                                   (SBN_BWD_ACCUMULATE if accumulate else 0) | (SBN_BWD_MASK_DW if mask_dw else 0),
                                                   _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                   _stream()), "sbn_sparse_ternary_linear_backward")


class BackwardGroup:
    """Host-side argument arrays of sbn_sparse_ternary_linear_backward_grouped, marshalled once and reusable.
    Lists hold one entry per layer; entries of dX_list / dW_list may be None."""

    def __init__(self, dY_list, packed_list, gamma_list, xq_list, sx_list, N, M, workspace, d_in_list, dX_list, dW_list,
                 accumulate=False, mask_dw=False):
        for dY in dY_list:
            if dY.dtype != torch.bfloat16:
                raise TypeError("dY must be bf16")
        self.count = len(dY_list)
        self.dY = _ptr_array(dY_list)
        self.tokens = _i64_array([d.shape[0] for d in dY_list])
        self.d_out = _i64_array([d.shape[1] for d in dY_list])
        self.d_in = _i64_array(list(d_in_list))
        self.packed, self.gamma = _ptr_array(packed_list), _ptr_array(gamma_list)
        self.xq, self.sx = _ptr_array(xq_list), _ptr_array(sx_list)
        self.dX, self.dW = _ptr_array(dX_list), _ptr_array(dW_list)
        self.flags = (SBN_BWD_ACCUMULATE if accumulate else 0) | (SBN_BWD_MASK_DW if mask_dw else 0)
        self.N, self.M, self.workspace = N, M, workspace
        self.keep = (dY_list, packed_list, gamma_list, xq_list, sx_list, dX_list, dW_list)

    def run(self):
        ws = self.workspace
        _check(_lib.sbn_sparse_ternary_linear_backward_grouped(self.count, self.dY, self.tokens, self.d_in, self.d_out, self.N,
                                                               self.M, self.packed, self.gamma, self.xq, self.sx, self.dX,
                                                               self.dW, self.flags, _ptr(ws), ws.numel() * ws.element_size(),
                                                               _stream()),
               "sbn_sparse_ternary_linear_backward_grouped")


def sbn_sparse_ternary_linear_backward_grouped(dY_list, packed_list, gamma_list, xq_list, sx_list, N, M, workspace, d_in_list,
                                               dX_list, dW_list, accumulate=False, mask_dw=False):
    BackwardGroup(dY_list, packed_list, gamma_list, xq_list, sx_list, N, M, workspace, d_in_list, dX_list, dW_list, accumulate,
                  mask_dw).run()


def sbn_unpack(packed, d_out: int, d_in: int, N: int, M: int, W_eff=None, mask=None):
    _check(_lib.sbn_unpack(_ptr(packed), d_out, d_in, N, M, _ptr(W_eff), _ptr(mask), _stream()), "sbn_unpack")


def sbn_rmsnorm_act_quant(X, xq, sx, gain=None, eps: float = 1e-6, xn_out=None):
    """x~, s_x = Q_a(Norm(x)); X bf16 [tokens, d_in]; gain fp32 [d_in] or None; xn_out bf16 or None."""
    tokens, d_in = X.shape
    _check(_lib.sbn_rmsnorm_act_quant(_ptr(X), tokens, d_in, _ptr(gain), eps, _ptr(xq), _ptr(sx), _ptr(xn_out), _stream()),
           "sbn_rmsnorm_act_quant")


def sbn_convert_packed(packed, d_out: int, d_in: int, N: int, M: int, to_N: int, to_M: int, out):
    """Rewrite a packed N:M matrix into the packed form of to_N:to_M (2:4 or M:M) for decode."""
    _check(_lib.sbn_convert_packed(_ptr(packed), d_out, d_in, N, M, to_N, to_M, _ptr(out), _stream()), "sbn_convert_packed")


def sbn_dense_ternary_linear(xq, sx, W_eff, gamma, Y, bias=None, acc_out=None):
    """The dense comparison kernel alone: Y = (xq @ W_eff^T) * gamma / s_x (+ bias) with W_eff int8 [d_out, d_in]."""
    tokens, d_in = xq.shape
    _check(_lib.sbn_dense_ternary_linear(_ptr(xq), _ptr(sx), tokens, d_in, W_eff.shape[0], _ptr(W_eff), _ptr(gamma), _ptr(bias),
                                         _ptr(Y), _ptr(acc_out), _stream()), "sbn_dense_ternary_linear")


SBN_SPIN_DEFAULT = -2 ** 31


def sbn_test_set_spin_limits(gemv_polls: int = SBN_SPIN_DEFAULT, pack_polls: int = SBN_SPIN_DEFAULT):
    """Test hook: polls of the two bounded inter-block waits (negative: never wait; SBN_SPIN_DEFAULT restores)."""
    _lib.sbn_test_set_spin_limits(gemv_polls, pack_polls)


SBN_KERNEL_TILES, SBN_KERNEL_STREAM, SBN_KERNEL_PIECES, SBN_KERNEL_DECODE, SBN_KERNEL_BLOCKS, SBN_KERNEL_SELF = 0, 1, 2, 3, 16, 32


def sbn_test_linear_kernel(kernel: int, xq_list, sx_list, packed_list, gamma_list, Y_list, N: int, M: int, bias_list=None, acc_list=None):
    """Test hook: the products of quantized rows through one kernel of SBN_PATH_SMFMAC by name (SBN_KERNEL_...)."""
    _check(_lib.sbn_test_linear_kernel(kernel, len(xq_list), _ptr_array(xq_list), _ptr_array(sx_list), _i64_array([x.shape[0] for x in xq_list]),
                                       _i64_array([x.shape[1] for x in xq_list]), _i64_array([y.shape[1] for y in Y_list]), N, M,
                                       _ptr_array(packed_list), _ptr_array(gamma_list), None if bias_list is None else _ptr_array(bias_list),
                                       _ptr_array(Y_list), None if acc_list is None else _ptr_array(acc_list), _stream()),
           "sbn_test_linear_kernel")


def sbn_test_self_kernel(form: int, X_list, packed_list, gamma_list, Y_list, N: int, M: int, bias_list=None, acc_list=None):
    """Test hook: the products of bf16 rows in one shape of the kernel that quantizes them itself."""
    _check(_lib.sbn_test_self_kernel(form, len(X_list), _ptr_array(X_list), _i64_array([x.shape[0] for x in X_list]),
                                     _i64_array([x.shape[1] for x in X_list]), _i64_array([y.shape[1] for y in Y_list]), N, M,
                                     _ptr_array(packed_list), _ptr_array(gamma_list), None if bias_list is None else _ptr_array(bias_list),
                                     _ptr_array(Y_list), None if acc_list is None else _ptr_array(acc_list), _stream()),
           "sbn_test_self_kernel")


def sbn_test_takes_blocks(problems, N: int, M: int) -> bool:
    """Test hook: whether SBN_PATH_SMFMAC takes block tiles for a call of these problems (tokens, d_in, d_out)."""
    blocks = ctypes.c_int(0)
    _check(_lib.sbn_test_takes_blocks(len(problems), *(_i64_array(column) for column in zip(*problems)), N, M, ctypes.byref(blocks)),
           "sbn_test_takes_blocks")
    return bool(blocks.value)


def sbn_test_forward_kernels(problems, N: int, M: int, X=None, Y=None, rows: bool = True):
    """Test hook: the kernel (SBN_KERNEL_...) of each problem (tokens, d_in, d_out) of one forward call.  X, Y: addresses, by default
    buffers that lie apart; rows False: quantized rows are handed in or wanted back."""
    kernel = (ctypes.c_int * len(problems))()
    X = X or [(i + 1) << 44 for i in range(len(problems))]
    Y = Y or [(i + 1) << 44 | 1 << 43 for i in range(len(problems))]
    _check(_lib.sbn_test_forward_kernels(len(problems), _ptr_array(X) if rows else None, *(_i64_array(column) for column in zip(*problems)), N, M,
                                         _ptr_array(Y), kernel), "sbn_test_forward_kernels")
    return list(kernel)


def sbn_test_chosen_kernels(problems, N: int, M: int):
    """Test hook: the kernel (SBN_KERNEL_...) of each problem (tokens, d_in, d_out) of one call on SBN_PATH_SMFMAC."""
    kernel = (ctypes.c_int * len(problems))()
    _check(_lib.sbn_test_chosen_kernels(len(problems), *(_i64_array(column) for column in zip(*problems)), N, M, kernel),
           "sbn_test_chosen_kernels")
    return list(kernel)


def sbn_mask_flips(packed_a, packed_b, d_out: int, d_in: int, N: int, M: int, flips_out, workspace):
    """flips_out: int64 device tensor of one element (the count is non-negative and below 2**63)."""
    _check(_lib.sbn_mask_flips(_ptr(packed_a), _ptr(packed_b), d_out, d_in, N, M, _ptr(flips_out), _ptr(workspace),
                               workspace.numel() * workspace.element_size(), _stream()), "sbn_mask_flips")


def _expect(name, t, shape, *dtypes):
    """t, where it is a contiguous tensor of this shape and one of these types (or None)."""
    if t is not None:
        if t.dtype not in dtypes:
            raise TypeError(f"{name} must be {' or '.join(str(d).removeprefix('torch.') for d in dtypes)}")
        if t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous {list(shape)}, not {list(t.shape)} with strides {list(t.stride())}")
    return t


def _on_gpu(*tensors):
    """A host address given to a kernel is a fault of the device."""
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError("tensors must be on the GPU")


def _bytes_of(ws):
    return ws.numel() * ws.element_size()


def sbn_head_workspace_bytes(tokens: int, d_in: int, vocab: int, top_k: int = 0, backward: bool = True) -> int:
    """Workspace of the forward calls of the output head, and of their backward calls where `backward` is set."""
    nbytes = _fast_head_bytes(tokens, d_in, vocab, top_k, int(backward))
    if nbytes is not None:
        return nbytes
    out = ctypes.c_size_t(0)
    _check(_lib.sbn_head_workspace_bytes(tokens, d_in, vocab, top_k, int(backward), ctypes.byref(out)), "sbn_head_workspace_bytes")
    return out.value


def _head_sizes(H, W, targets, ce, dH=None, dW=None):
    bf16, f32 = torch.bfloat16, torch.float32
    (tokens, d_in), vocab = H.shape, W.shape[0]
    _expect("H", H, (tokens, d_in), bf16)
    _expect("W", W, (vocab, d_in), bf16)
    _expect("targets", targets, (tokens,), torch.int64)
    _expect("ce", ce, (tokens,), f32)
    _expect("dH", dH, (tokens, d_in), bf16)
    _expect("dW", dW, (vocab, d_in), bf16)
    return tokens, d_in, vocab


def sbn_head_cross_entropy(H, W, targets, ce, lse, workspace):
    """ce, lse (fp32 [tokens]) of z = H W^T against targets (int64; outside the vocabulary: left out), the logits never stored."""
    status = _fast_head_ce(H, W, targets, ce, lse, workspace)
    if status is not None:
        if status:
            _check(status, "sbn_head_cross_entropy")
        return
    tokens, d_in, vocab = _head_sizes(H, W, targets, ce)
    _expect("lse", lse, (tokens,), torch.float32)
    _on_gpu(H, W, targets, ce, lse, workspace)
    _check(_lib.sbn_head_cross_entropy(_ptr(H), _ptr(W), _ptr(targets), tokens, d_in, vocab, _ptr(ce), _ptr(lse), _ptr(workspace),
                                       _bytes_of(workspace), _stream()), "sbn_head_cross_entropy")


def sbn_head_cross_entropy_backward(H, W, targets, lse, d_ce, workspace, dH=None, dW=None):
    """dH, dW (bf16, overwritten; None: not wanted) for the gradient d_ce (fp32 [tokens]) of ce."""
    status = _fast_head_ce_backward(H, W, targets, lse, d_ce, workspace, dH, dW)
    if status is not None:
        if status:
            _check(status, "sbn_head_cross_entropy_backward")
        return
    tokens, d_in, vocab = _head_sizes(H, W, targets, d_ce, dH, dW)
    _expect("lse", lse, (tokens,), torch.float32)
    _on_gpu(H, W, targets, lse, d_ce, workspace, dH, dW)
    _check(_lib.sbn_head_cross_entropy_backward(_ptr(H), _ptr(W), _ptr(targets), _ptr(lse), _ptr(d_ce), tokens, d_in, vocab, _ptr(dH), _ptr(dW),
                                                _ptr(workspace), _bytes_of(workspace), _stream()), "sbn_head_cross_entropy_backward")


def _teacher(top_idx, top_logits, tokens):
    top_k = top_idx.shape[1]
    _expect("top_idx", top_idx, (tokens, top_k), torch.int64)
    _expect("top_logits", top_logits, (tokens, top_k), torch.float32, torch.bfloat16)
    return SBN_BF16 if top_logits.dtype == torch.bfloat16 else SBN_F32, top_k


def sbn_head_distill(H, W, top_idx, top_logits, tau: float, kd, lse, workspace, targets=None, ce=None):
    """kd (fp32 [tokens]) against the teacher's entries top_idx (int64) and top_logits (fp32 or bf16), both [tokens, k], at temperature
    tau; lse fp32 [2, tokens]; with targets and ce the cross entropy from the same pass."""
    status = _fast_head_distill(H, W, top_idx, top_logits, tau, kd, lse, workspace, targets, ce)
    if status is not None:
        if status:
            _check(status, "sbn_head_distill")
        return
    tokens, d_in, vocab = _head_sizes(H, W, targets, ce)
    dtype, top_k = _teacher(top_idx, top_logits, tokens)
    _expect("kd", kd, (tokens,), torch.float32)
    _expect("lse", lse, (2, tokens), torch.float32)
    _on_gpu(H, W, top_idx, top_logits, kd, lse, workspace, targets, ce)
    _check(_lib.sbn_head_distill(_ptr(H), _ptr(W), _ptr(top_idx), _ptr(top_logits), dtype, top_k, tau, _ptr(targets), tokens, d_in, vocab,
                                 _ptr(kd), _ptr(ce), _ptr(lse), _ptr(workspace), _bytes_of(workspace), _stream()), "sbn_head_distill")


def sbn_head_distill_backward(H, W, top_idx, top_logits, tau: float, lse, d_kd, workspace, targets=None, d_ce=None, dH=None, dW=None):
    """dH, dW (bf16, overwritten; None: not wanted) for the gradients d_kd and, with targets, d_ce of the two losses."""
    status = _fast_head_distill_backward(H, W, top_idx, top_logits, tau, lse, d_kd, workspace, targets, d_ce, dH, dW)
    if status is not None:
        if status:
            _check(status, "sbn_head_distill_backward")
        return
    tokens, d_in, vocab = _head_sizes(H, W, targets, d_ce, dH, dW)
    dtype, top_k = _teacher(top_idx, top_logits, tokens)
    _expect("d_kd", d_kd, (tokens,), torch.float32)
    _expect("lse", lse, (2, tokens), torch.float32)
    _on_gpu(H, W, top_idx, top_logits, lse, d_kd, workspace, targets, d_ce, dH, dW)
    _check(_lib.sbn_head_distill_backward(_ptr(H), _ptr(W), _ptr(top_idx), _ptr(top_logits), dtype, top_k, tau, _ptr(targets), _ptr(lse),
                                          _ptr(d_kd), _ptr(d_ce), tokens, d_in, vocab, _ptr(dH), _ptr(dW), _ptr(workspace),
                                          _bytes_of(workspace), _stream()), "sbn_head_distill_backward")


def sbn_mxfp4_bytes(rows: int, cols: int):
    """Bytes of the codes and of the scales of a [rows, cols] matrix."""
    nbytes = _fast_mxfp4_bytes(rows, cols)
    if nbytes is not None:
        return nbytes
    codes, scales = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(_lib.sbn_mxfp4_bytes(rows, cols, ctypes.byref(codes), ctypes.byref(scales)), "sbn_mxfp4_bytes")
    return codes.value, scales.value


def _mxfp4(codes, scales, rows, cols):
    """Codes and scales as uint8 buffers of any shape that hold a [rows, cols] matrix."""
    wide = -(-cols // 128) * 128
    for name, t, nbytes in (("codes", codes, rows * wide // 2), ("scales", scales, rows * wide // 32)):
        if t.dtype != torch.uint8:
            raise TypeError(f"{name} must be uint8")
        if t.numel() != nbytes or not t.is_contiguous():
            raise ValueError(f"{name} must be {nbytes} contiguous bytes for [{rows}, {cols}], not {t.numel()}")


def sbn_mxfp4_quantize(X, codes, scales):
    """X (fp32 or bf16 [rows, cols]) to microscaled 4-bit codes and block scales (uint8)."""
    status = _fast_mxfp4_quantize(X, codes, scales)
    if status is not None:
        if status:
            _check(status, "sbn_mxfp4_quantize")
        return
    rows, cols = X.shape
    _expect("X", X, (rows, cols), torch.float32, torch.bfloat16)
    _mxfp4(codes, scales, rows, cols)
    _on_gpu(X, codes, scales)
    _check(_lib.sbn_mxfp4_quantize(_ptr(X), _dtype_code(X), rows, cols, _ptr(codes), _ptr(scales), _stream()), "sbn_mxfp4_quantize")


def sbn_mxfp4_dequantize(codes, scales, Y):
    """The values that codes and scales stand for, exactly, into Y (fp32 or bf16 [rows, cols])."""
    status = _fast_mxfp4_dequantize(codes, scales, Y)
    if status is not None:
        if status:
            _check(status, "sbn_mxfp4_dequantize")
        return
    rows, cols = Y.shape
    _expect("Y", Y, (rows, cols), torch.float32, torch.bfloat16)
    _mxfp4(codes, scales, rows, cols)
    _on_gpu(codes, scales, Y)
    _check(_lib.sbn_mxfp4_dequantize(_ptr(codes), _ptr(scales), rows, cols, _ptr(Y), _dtype_code(Y), _stream()), "sbn_mxfp4_dequantize")


def sbn_mxfp4_workspace_bytes(tokens: int, d_in: int) -> int:
    nbytes = _fast_mxfp4_workspace_bytes(tokens, d_in)
    if nbytes is not None:
        return nbytes
    out = ctypes.c_size_t(0)
    _check(_lib.sbn_mxfp4_workspace_bytes(tokens, d_in, ctypes.byref(out)), "sbn_mxfp4_workspace_bytes")
    return out.value


def sbn_mxfp4_linear(X, codes, scales, Y, workspace, bias=None):
    """Y (fp32 [tokens, d_out]) = q(X) W^T (+ bias): X bf16, quantized on the way; W as codes and scales."""
    status = _fast_mxfp4_linear(X, codes, scales, Y, workspace, bias)
    if status is not None:
        if status:
            _check(status, "sbn_mxfp4_linear")
        return
    (tokens, d_in), d_out = X.shape, Y.shape[1]
    _expect("X", X, (tokens, d_in), torch.bfloat16)
    _expect("Y", Y, (tokens, d_out), torch.float32)
    _expect("bias", bias, (d_out,), torch.float32)
    _mxfp4(codes, scales, d_out, d_in)
    _on_gpu(X, codes, scales, Y, workspace, bias)
    _check(_lib.sbn_mxfp4_linear(_ptr(X), tokens, d_in, d_out, _ptr(codes), _ptr(scales), _ptr(bias), _ptr(Y), _ptr(workspace),
                                 _bytes_of(workspace), _stream()), "sbn_mxfp4_linear")


def _here(*tensors):
    """Tensors of a call lie on the current device: its stream is the one that the kernels run on."""
    _on_gpu(*tensors)
    device = (_current_device or torch.cuda.current_device)()
    for t in tensors:
        if t is not None and t.device.index != device:
            raise ValueError(f"tensors must be on the current device (cuda:{device}), not on {t.device}")


def _size_query(fn, where, *args):
    out = ctypes.c_size_t(0)
    _check(fn(*args, ctypes.byref(out)), where)
    return out.value


def _row_type(name, t):
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"{name} must be float32 or bfloat16")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions")
    return _dtype_code(t)


def sbn_norm(X, Y, gain=None, bias=None, eps: float = 1e-6, layer: bool = False, residual=None, sum_out=None):
    """Y = the RMS norm (layer: layer norm) of the rows of X, or of X + residual, which is then given back in sum_out; gain, bias fp32."""
    status = _fast_norm(X, Y, gain, bias, eps, layer, residual, sum_out)
    if status is not None:
        if status:
            _check(status, "sbn_norm")
        return
    dtype, shape = _row_type("X", X), X.shape
    for name, t in (("X", X), ("Y", Y), ("residual", residual), ("sum_out", sum_out)):
        _expect(name, t, shape, X.dtype)
    _expect("gain", gain, shape[1:], torch.float32)
    _expect("bias", bias, shape[1:], torch.float32)
    _here(X, Y, gain, bias, residual, sum_out)
    _check(_lib.sbn_norm(_ptr(X), _ptr(residual), dtype, *shape, _ptr(gain), _ptr(bias), eps, int(layer), _ptr(Y), _ptr(sum_out), _stream()), "sbn_norm")


def sbn_norm_workspace_bytes(tokens: int, d_in: int) -> int:
    nbytes = _fast_norm_bytes(tokens, d_in)
    return nbytes if nbytes is not None else _size_query(_lib.sbn_norm_workspace_bytes, "sbn_norm_workspace_bytes", tokens, d_in)


def sbn_norm_backward(X, dY, workspace, dX=None, dgain=None, dbias=None, gain=None, eps: float = 1e-6, layer: bool = False, d_residual=None):
    """dX (+ d_residual), dgain and dbias (fp32) of sbn_norm for the gradient dY of its Y; X is what was normalised.  None: not wanted."""
    status = _fast_norm_backward(X, dY, workspace, dX, dgain, dbias, gain, eps, layer, d_residual)
    if status is not None:
        if status:
            _check(status, "sbn_norm_backward")
        return
    dtype, shape = _row_type("X", X), X.shape
    for name, t in (("X", X), ("dY", dY), ("dX", dX), ("d_residual", d_residual)):
        _expect(name, t, shape, X.dtype)
    for name, t in (("gain", gain), ("dgain", dgain), ("dbias", dbias)):
        _expect(name, t, shape[1:], torch.float32)
    _here(X, dY, workspace, dX, dgain, dbias, gain, d_residual)
    _check(_lib.sbn_norm_backward(_ptr(X), _ptr(dY), _ptr(d_residual), dtype, *shape, _ptr(gain), eps, int(layer), _ptr(dX), _ptr(dgain), _ptr(dbias),
                                  _ptr(workspace), _bytes_of(workspace), _stream()), "sbn_norm_backward")


def _embedding(table_name, table, rows_name, rows, ids):
    """Types and sizes of a table and of the rows that go with ids."""
    types = _row_type(table_name, table), _row_type(rows_name, rows)
    (vocab, d), tokens = table.shape, ids.numel()
    _expect(table_name, table, (vocab, d), table.dtype)
    _expect(rows_name, rows, (tokens, d), rows.dtype)
    _expect("ids", ids, (tokens,), torch.int64)
    return (*types, vocab, d, tokens)


def sbn_embedding(E, ids, Y, scale: float = 1.0):
    """Y[t,:] = scale E[ids[t],:] (fp32 or bf16 each); zeros where the id (int64) is outside the table."""
    status = _fast_embedding(E, ids, Y, scale)
    if status is not None:
        if status:
            _check(status, "sbn_embedding")
        return
    table, rows, vocab, d, tokens = _embedding("E", E, "Y", Y, ids)
    _here(E, ids, Y)
    _check(_lib.sbn_embedding(_ptr(E), table, vocab, d, _ptr(ids), tokens, scale, _ptr(Y), rows, _stream()), "sbn_embedding")


def sbn_embedding_workspace_bytes(tokens: int, d_in: int, vocab: int) -> int:
    nbytes = _fast_embedding_bytes(tokens, d_in, vocab)
    return nbytes if nbytes is not None else _size_query(_lib.sbn_embedding_workspace_bytes, "sbn_embedding_workspace_bytes", tokens, d_in, vocab)


def sbn_embedding_backward(dY, ids, dE, workspace, scale: float = 1.0, accumulate: bool = False):
    """dE[v,:] = scale sum of dY[t,:] over the tokens of id v: every row written, or (accumulate) the sums added to what dE holds."""
    status = _fast_embedding_backward(dY, ids, dE, workspace, scale, accumulate)
    if status is not None:
        if status:
            _check(status, "sbn_embedding_backward")
        return
    table, rows, vocab, d, tokens = _embedding("dE", dE, "dY", dY, ids)
    _here(dY, ids, dE, workspace)
    _check(_lib.sbn_embedding_backward(_ptr(dY), rows, _ptr(ids), tokens, vocab, d, scale, int(accumulate), _ptr(dE), table, _ptr(workspace), _bytes_of(workspace),
                                       _stream()), "sbn_embedding_backward")


class _Tensors:
    """A non-empty list of contiguous tensors of one of these types, as many values each as `like` says: with their addresses and sizes as ctypes arrays."""

    def __init__(self, name, tensors, *dtypes, like=None):
        self.list = tensors = list(tensors)
        if not tensors or (like is not None and len(tensors) != len(like)):
            raise ValueError(f"{name} must be a list of {len(like) if like is not None else 'one or more'} tensors")
        self.pointers, self.sizes = (ctypes.c_void_p * len(tensors))(), (ctypes.c_int64 * len(tensors))()
        code = _fast_gather(tensors, self.pointers, self.sizes)
        if code is not None and (torch.float32, torch.bfloat16, torch.uint8)[code] in dtypes and (like is None or self.sizes[:] == like):
            return
        dtype = tensors[0].dtype
        for i, t in enumerate(tensors):
            if t.dtype is not dtype or dtype not in dtypes:
                raise TypeError(f"{name} must all be {' or all '.join(str(d).removeprefix('torch.') for d in dtypes)}")
            if not t.is_contiguous() or (like is not None and t.numel() != like[i]):
                raise ValueError(f"{name}[{i}] must be contiguous" + (f" and have {like[i]} values, not {t.numel()}" if like is not None else ""))
        _here(*tensors)
        self.pointers, self.sizes = _ptr_array(tensors), _i64_array([t.numel() for t in tensors])


def sbn_grad_norm_workspace_bytes(sizes) -> int:
    """Workspace of the norm of gradients of so many values each."""
    return _size_query(_lib.sbn_grad_norm_workspace_bytes, "sbn_grad_norm_workspace_bytes", len(sizes), _i64_array(sizes))


class GradNormGroup:
    """Host-side argument arrays of sbn_grad_norm, marshalled once and reusable: with the addresses that the gradients had when it was made, as in AdamWGroup."""

    def __init__(self, grads, workspace):
        grads = _Tensors("grads", grads, torch.float32, torch.bfloat16)
        _here(workspace)
        self.count, self.dtype, self.keep = len(grads.list), _dtype_code(grads.list[0]), grads.list
        self.grads, self.sizes, self.workspace = grads.pointers, grads.sizes, workspace

    def run(self, max_norm: float, out):
        ws = self.workspace
        status = _fast_grad_norm(self.count, self.grads, self.dtype, self.sizes, max_norm, out, ws)
        if status is not None:
            if status:
                _check(status, "sbn_grad_norm")
            return
        _expect("out", out, (2,), torch.float32)
        _here(out, ws)
        _check(_lib.sbn_grad_norm(self.count, self.grads, self.dtype, self.sizes, max_norm, _ptr(out), _ptr(ws), _bytes_of(ws), _stream()), "sbn_grad_norm")


def sbn_grad_norm(grads, max_norm: float, out, workspace):
    """out (fp32 [2]) = the norm of all gradients, and the factor that brings it down to max_norm (at most 1; NaN where the norm is not finite)."""
    GradNormGroup(grads, workspace).run(max_norm, out)


def sbn_adamw_state_bytes(n: int):
    """Bytes of the codes and of the scales of n moments in 8 bits."""
    codes, scales = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(_lib.sbn_adamw_state_bytes(n, ctypes.byref(codes), ctypes.byref(scales)), "sbn_adamw_state_bytes")
    return codes.value, scales.value


def sbn_adamw_state_values(codes, scales, out, second: bool = False):
    """The values that moments in 8 bits stand for, exactly, into out (fp32 or bf16, any shape); second: of v, else of m."""
    status = _fast_state_values(codes, scales, out, second)
    if status is not None:
        if status:
            _check(status, "sbn_adamw_state_values")
        return
    _expect("out", out, out.shape, torch.float32, torch.bfloat16)
    for name, t, nbytes in zip(("codes", "scales"), (codes, scales), sbn_adamw_state_bytes(out.numel())):
        _expect(name, t, (nbytes,), torch.uint8)
    _here(codes, scales, out)
    _check(_lib.sbn_adamw_state_values(_ptr(codes), _ptr(scales), out.numel(), int(second), _ptr(out), _dtype_code(out), _stream()), "sbn_adamw_state_values")


class AdamWGroup:
    """Host-side argument arrays of sbn_adamw_step, marshalled once and reusable.  Lists hold one tensor per weight: params and grads fp32 or bf16, m and v
    fp32, or (with m_scales and v_scales) the bytes of moments in 8 bits; weight_decay is a number, or one per weight.

    The group holds the tensors and the addresses that they had when it was made: gradients are written into the same tensors (zero_grad(set_to_none=False)).
    Where a tensor is another one at each step, or its storage is exchanged (p.data = ...), make a new group, or call sbn_adamw_step, which makes one."""

    def __init__(self, params, grads, m, v, m_scales=None, v_scales=None, weight_decay=0.0, betas=(0.9, 0.95), eps: float = 1e-8):
        params = _Tensors("params", params, torch.float32, torch.bfloat16)
        sizes = params.sizes[:]
        grads = _Tensors("grads", grads, torch.float32, torch.bfloat16, like=sizes)
        if (m_scales is None) != (v_scales is None):
            raise ValueError("m_scales and v_scales are both given or neither")
        bits8 = m_scales is not None
        scales = [(n + 31) // 32 for n in sizes]
        m, v = (_Tensors(name, t, torch.uint8 if bits8 else torch.float32, like=[32 * n for n in scales] if bits8 else sizes) for name, t in (("m", m), ("v", v)))
        if bits8:
            m_scales, v_scales = (_Tensors(name, t, torch.uint8, like=scales) for name, t in (("m_scales", m_scales), ("v_scales", v_scales)))
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * len(sizes)
        if len(decay) != len(sizes):
            raise ValueError(f"weight_decay must be a number or {len(sizes)} of them")
        self.count, self.sizes = len(sizes), params.sizes
        self.types = _dtype_code(params.list[0]), _dtype_code(grads.list[0])
        self.params, self.grads, self.m, self.v = params.pointers, grads.pointers, m.pointers, v.pointers
        self.m_scales, self.v_scales = (t.pointers if bits8 else None for t in (m_scales, v_scales))
        self.decay = (ctypes.c_float * len(decay))(*decay)
        self.betas, self.eps = betas, eps
        self.keep = (params, grads, m, v, m_scales, v_scales)
        self.device = params.list[0].get_device()

    def run(self, lr, step, clip=None, seed: int | None = None):
        """One step: lr (fp32 [1]), step (int64 [1], counted from 1) and clip (fp32 [1], or None) on the device; seed: round stochastically."""
        if self.device != (_current_device or torch.cuda.current_device)():
            raise ValueError(f"the group's tensors lie on cuda:{self.device}, which is not the current device")
        status = _fast_adamw(self.count, self.params, self.types[0], self.grads, self.types[1], self.m, self.v, self.m_scales, self.v_scales, self.sizes, self.decay, lr,
                             step, *self.betas, self.eps, clip, seed)
        if status is not None:
            if status:
                _check(status, "sbn_adamw_step")
            return
        _expect("lr", lr, (1,), torch.float32)
        _expect("step", step, (1,), torch.int64)
        _expect("clip", clip, (1,), torch.float32)
        _here(lr, step, clip)
        _check(_lib.sbn_adamw_step(self.count, self.params, self.types[0], self.grads, self.types[1], self.m, self.v, self.m_scales, self.v_scales, self.sizes,
                                   self.decay, _ptr(lr), _ptr(step), *self.betas, self.eps, _ptr(clip),
                                   None if seed is None else ctypes.byref(ctypes.c_uint64(seed)), _stream()), "sbn_adamw_step")


def sbn_adamw_step(params, grads, m, v, lr, step, m_scales=None, v_scales=None, weight_decay=0.0, betas=(0.9, 0.95), eps: float = 1e-8, clip=None, seed=None):
    """One step over lists of tensors that may be others at the next: an AdamWGroup of them, run once."""
    AdamWGroup(params, grads, m, v, m_scales, v_scales, weight_decay, betas, eps).run(lr, step, clip, seed)


def sbn_test_set_head_tiles(logits: int = -1, gradients: int = -1, mxfp4: int = -1):
    """Test hook: block tiles of the output head (0, 1, 2; gradients 3: the kernel of up to 64 tokens; negative: the library's choice)."""
    _lib.sbn_test_set_head_tiles(logits, gradients, mxfp4)


def sbn_test_chosen_mxfp4_tile(tokens: int, d_in: int, d_out: int):
    """Test hook: the block tiles (0, 1, 2) of a 4-bit product of more than 64 tokens, and the threads of its launch."""
    size, threads = ctypes.c_int(0), ctypes.c_int64(0)
    _check(_lib.sbn_test_chosen_mxfp4_tile(tokens, d_in, d_out, ctypes.byref(size), ctypes.byref(threads)), "sbn_test_chosen_mxfp4_tile")
    return size.value, threads.value


def new_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """Device scratch of at least nbytes (torch's allocator returns 512-byte aligned blocks)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
