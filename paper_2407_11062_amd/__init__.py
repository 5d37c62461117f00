"""Thin Python binding of the eqat C ABI (``include/eqat.h``).

Argument marshalling only: every function here turns torch tensors into raw
device pointers and sizes, allocates outputs / workspace with torch when the
caller did not pass them, and calls the entry point of the same name in
``libeqat.so`` on torch's current stream.  No arithmetic of the method runs in
Python, and there is no fallback: without the built library every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("EQAT_LIB", os.path.join(_HERE, "libeqat.so"))   # EQAT_LIB: a build under test

F32, BF16 = 0, 1
OP_FQ_FWD, OP_FQ_BWD, OP_Q_FWD, OP_Q_BWD, OP_QP_FWD, OP_QP_BWD = 0, 1, 2, 3, 4, 5
STATE_FQ_KEPT, STATE_Q_KEPT, STATE_PREPARED = 0, 1, 2
GATE_SILU, GATE_GELU = 0, 1

STATUS_NAMES = ["EQAT_OK", "EQAT_ERR_NULL", "EQAT_ERR_SHAPE", "EQAT_ERR_BITS", "EQAT_ERR_GROUP", "EQAT_ERR_DTYPE",
                "EQAT_ERR_ALIGN", "EQAT_ERR_WORKSPACE", "EQAT_ERR_DEVICE", "EQAT_ERR_HYPER"]

EXPORTS = ["eqat_status_string", "eqat_validate_desc", "eqat_packed_w_bytes", "eqat_packed_z_bytes",
           "eqat_workspace_bytes", "eqat_init_minmax", "eqat_fq_linear_fwd", "eqat_fq_linear_bwd",
           "eqat_fq_linear_fwd_keep", "eqat_fq_linear_bwd_kept", "eqat_fq_linear_fwd_kept", "eqat_pack",
           "eqat_init_minmax_batched", "eqat_pack_batched", "eqat_fq_quantize_batched",
           "eqat_unpack", "eqat_qlinear_fwd", "eqat_qlinear_bwd", "eqat_qlinear_fwd_keep", "eqat_qlinear_bwd_kept",
           "eqat_qlinear_fwd_z", "eqat_qlinear_bwd_z", "eqat_prepared_bytes", "eqat_qlinear_prepare",
           "eqat_qlinear_fwd_prepared", "eqat_qlinear_bwd_prepared", "eqat_qlinear_fwd_prepared_keep",
           "eqat_qlinear_bwd_prepared_kept", "eqat_unpack_state", "eqat_plan_item", "eqat_shared_item", "eqat_plan_scratch", "eqat_fwd_route", "eqat_dx_route",
           "eqat_recon_loss_workspace_bytes", "eqat_recon_loss", "eqat_recon_loss_static", "eqat_block_ap_update",
           "eqat_kv_pool_bytes", "eqat_kv_write", "eqat_kv_read", "eqat_kv_workspace_bytes", "eqat_kv_attention",
           "eqat_norm_fwd", "eqat_norm_workspace_bytes", "eqat_norm_bwd", "eqat_rotary", "eqat_kv_rotary_write", "eqat_gate_fwd", "eqat_gate_bwd",
           "eqat_gated_workspace_bytes", "eqat_gated_fwd", "eqat_gated_bwd", "eqat_gated_fwd_prepared", "eqat_gated_bwd_prepared",
           "eqat_profile_kernels", "eqat_profile_kernel_name",
           "eqat_profile_start", "eqat_profile_stop"]


class Desc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("in_features", ctypes.c_int64), ("out_features", ctypes.c_int64),
                ("bits", ctypes.c_int32), ("group", ctypes.c_int32), ("act_dtype", ctypes.c_int32),
                ("w_dtype", ctypes.c_int32)]


class AdamW(ctypes.Structure):
    _fields_ = [("lr_w", ctypes.c_float), ("lr_q", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay_w", ctypes.c_float), ("weight_decay_q", ctypes.c_float),
                ("step", ctypes.c_int32)]


class KvDesc(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int64), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("group", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("act_dtype", ctypes.c_int32)]


class KvBatchDesc(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("starts", ctypes.c_void_p), ("tokens", ctypes.c_int64),
                ("sequences", ctypes.c_int32), ("table_stride", ctypes.c_int32), ("max_new", ctypes.c_int32), ("max_len", ctypes.c_int32)]


class KvAttn(ctypes.Structure):
    _fields_ = [("q_heads", ctypes.c_int32), ("causal", ctypes.c_int32), ("window", ctypes.c_int32), ("scale", ctypes.c_float)]


class NormDesc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("width", ctypes.c_int32), ("group", ctypes.c_int32), ("act_dtype", ctypes.c_int32), ("w_dtype", ctypes.c_int32),
                ("eps", ctypes.c_float)]


class RotaryDesc(ctypes.Structure):
    _fields_ = [("frequencies", ctypes.c_void_p), ("head_dim", ctypes.c_int32), ("part", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("act_dtype", ctypes.c_int32),
                ("amplitude", ctypes.c_float)]


class EqatError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"{fn}: {name}: {lib().eqat_status_string(status).decode()}")


_lib = None


def lib():
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2407_11062_amd.build` "
                               "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, dp, sz = ctypes.c_void_p, ctypes.POINTER(Desc), ctypes.c_size_t
        L.eqat_status_string.restype = ctypes.c_char_p
        L.eqat_status_string.argtypes = [ctypes.c_int]
        L.eqat_validate_desc.argtypes = [dp]
        for f in (L.eqat_packed_w_bytes, L.eqat_packed_z_bytes):
            f.restype, f.argtypes = sz, [dp]
        L.eqat_workspace_bytes.restype, L.eqat_workspace_bytes.argtypes = sz, [dp, ctypes.c_int]
        L.eqat_init_minmax.argtypes = [dp, vp, vp, vp, vp]
        L.eqat_fq_linear_fwd.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_fq_linear_bwd.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_fq_linear_fwd_keep.argtypes = L.eqat_fq_linear_fwd.argtypes
        L.eqat_fq_linear_bwd_kept.argtypes = L.eqat_fq_linear_bwd.argtypes
        L.eqat_fq_linear_fwd_kept.argtypes = L.eqat_fq_linear_fwd.argtypes
        L.eqat_init_minmax_batched.argtypes = [ctypes.c_int, dp, vp, vp, vp, vp]
        L.eqat_pack_batched.argtypes = [ctypes.c_int, dp, vp, vp, vp, vp, vp, vp]
        L.eqat_fq_quantize_batched.argtypes = [ctypes.c_int, dp, vp, vp, vp, vp, vp, vp]
        L.eqat_pack.argtypes = [dp, vp, vp, vp, vp, vp, vp]
        L.eqat_unpack.argtypes = [dp, vp, vp, vp, vp, vp]
        L.eqat_qlinear_fwd.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_qlinear_bwd.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_qlinear_fwd_keep.argtypes = L.eqat_qlinear_fwd.argtypes
        L.eqat_qlinear_bwd_kept.argtypes = L.eqat_qlinear_bwd.argtypes
        L.eqat_qlinear_fwd_z.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_qlinear_bwd_z.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_prepared_bytes.restype, L.eqat_prepared_bytes.argtypes = sz, [dp]
        L.eqat_qlinear_prepare.argtypes = [dp, vp, vp, vp, sz, vp]
        L.eqat_qlinear_fwd_prepared.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_qlinear_bwd_prepared.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_qlinear_fwd_prepared_keep.argtypes = L.eqat_qlinear_fwd_prepared.argtypes
        L.eqat_plan_item.argtypes = [dp, ctypes.c_int, ctypes.c_int, ctypes.c_int, vp, vp]
        L.eqat_shared_item.argtypes = [dp, ctypes.c_int, ctypes.c_int, vp, vp]
        L.eqat_plan_scratch.argtypes = [dp, ctypes.c_int, ctypes.c_int, ctypes.c_int, sz, ctypes.POINTER(sz), ctypes.POINTER(sz)]
        L.eqat_fwd_route.argtypes = [dp, ctypes.c_int, vp]
        L.eqat_dx_route.argtypes = [dp, ctypes.c_int, vp]
        L.eqat_qlinear_bwd_prepared_kept.argtypes = L.eqat_qlinear_bwd_prepared.argtypes
        L.eqat_unpack_state.argtypes = [dp, ctypes.c_int, vp, vp, vp, vp, vp]
        L.eqat_recon_loss_workspace_bytes.restype, L.eqat_recon_loss_workspace_bytes.argtypes = sz, []
        L.eqat_recon_loss.argtypes = [ctypes.c_int64, ctypes.c_int32, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_recon_loss_static.argtypes = [ctypes.c_int64, ctypes.c_int32, vp, vp, vp, vp, vp]
        L.eqat_block_ap_update.argtypes = [dp, ctypes.POINTER(AdamW)] + [vp] * 13
        kd, kb = ctypes.POINTER(KvDesc), ctypes.POINTER(KvBatchDesc)
        L.eqat_kv_pool_bytes.restype, L.eqat_kv_pool_bytes.argtypes = sz, [kd]
        L.eqat_kv_write.argtypes = [kd, kb, vp, vp, vp, vp, vp, vp]
        L.eqat_kv_read.argtypes = L.eqat_kv_write.argtypes
        L.eqat_kv_workspace_bytes.restype, L.eqat_kv_workspace_bytes.argtypes = sz, [kd, kb, ctypes.c_int]
        L.eqat_kv_attention.argtypes = [kd, kb, ctypes.POINTER(KvAttn), vp, vp, vp, vp, vp, vp, vp, sz, vp]
        kn, kr, i64, i32 = ctypes.POINTER(NormDesc), ctypes.POINTER(RotaryDesc), ctypes.c_int64, ctypes.c_int
        L.eqat_norm_fwd.argtypes = [kn, vp, vp, vp, vp, vp, vp, vp, vp]
        L.eqat_norm_workspace_bytes.restype, L.eqat_norm_workspace_bytes.argtypes = sz, [kn]
        L.eqat_norm_bwd.argtypes = [kn, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_rotary.argtypes = [kr, i64, vp, vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, i32, vp]
        L.eqat_kv_rotary_write.argtypes = [kd, kb, kr, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.eqat_gate_fwd.argtypes = [i64, i64, ctypes.c_int32, i32, vp, vp, vp]
        L.eqat_gate_bwd.argtypes = [i64, i64, ctypes.c_int32, i32, vp, vp, vp, vp, vp]
        L.eqat_gated_workspace_bytes.restype, L.eqat_gated_workspace_bytes.argtypes = sz, [dp]
        L.eqat_gated_fwd.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_gated_bwd.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_gated_fwd_prepared.argtypes = [dp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_gated_bwd_prepared.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.eqat_profile_kernel_name.restype = ctypes.c_char_p
        L.eqat_profile_kernel_name.argtypes = [ctypes.c_int]
        L.eqat_profile_stop.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64), ctypes.c_int]
        _lib = L
    return _lib


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _tdt(code: int):
    return torch.bfloat16 if code == BF16 else torch.float32


# The short calls (one token, small linears) would be bound by what happens here, not by the kernel: 8.7 us per call with a
# Stream object, a descriptor and a c_void_p per argument made each time, against 4.6 us for a 4096 x 4096 matrix-vector
# product on the GPU; 5.5 us as it is.  Pointers therefore travel as plain integers (the argument types convert them), the raw stream handle
# is asked for directly, and descriptors of equal contents are made once.
def _p(t):
    if t is None:
        return None
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError("eqat tensors must be contiguous device tensors")
    return t.data_ptr()


try:
    _raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
except AttributeError:                               # not public: a torch without them has the Stream object
    def _raw_stream(device):
        return torch.cuda.current_stream(device).cuda_stream
    _device = torch.cuda.current_device


def _stream():
    """Handle of torch's current stream on the current device."""
    return _raw_stream(_device())


def _check(fn, status):
    if status != 0:
        raise EqatError(fn, status)


def make_desc(T, I, O, bits, group, act_dtype, w_dtype) -> Desc:
    return Desc(int(T), int(I), int(O), int(bits), int(group), int(act_dtype), int(w_dtype))


@functools.lru_cache(maxsize=1024)
def _desc_ref(T, I, O, bits, group, act_dtype, w_dtype):
    """A reference to a descriptor that is only ever read; the cache is by value."""
    return ctypes.byref(make_desc(T, I, O, bits, group, act_dtype, w_dtype))


def workspace(desc: Desc, op: int, device) -> torch.Tensor | None:
    n = lib().eqat_workspace_bytes(ctypes.byref(desc), op)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def _groups(I, group):
    return 1 if group == -1 else I // group


def eqat_init_minmax(W, bits, group, s=None, z=None):
    O, I = W.shape
    d = make_desc(0, I, O, bits, group, BF16, _dt(W))
    G = _groups(I, group)
    s = torch.empty((O, G), dtype=torch.float32, device=W.device) if s is None else s
    z = torch.empty((O, G), dtype=torch.float32, device=W.device) if z is None else z
    _check("eqat_init_minmax", lib().eqat_init_minmax(ctypes.byref(d), _p(W), _p(s), _p(z), _stream()))
    return s, z


class Batch:
    """Host arrays of device pointers (and the descriptors) for the *_batched entry points; build once, call often."""

    def __init__(self, descs, **tensor_lists):
        self.n = len(descs)
        self.descs = (Desc * self.n)(*descs)
        self.keep = tensor_lists                     # the tensors must outlive the pointer arrays
        self.ptr = {k: (ctypes.c_void_p * self.n)(*[t.data_ptr() for t in v]) for k, v in tensor_lists.items()}
        if "ws" in tensor_lists:
            self.ws_bytes = (ctypes.c_size_t * self.n)(*[t.numel() for t in tensor_lists["ws"]])


def eqat_init_minmax_batched(b: Batch):
    """b: Batch(descs, W=[...], s=[...], z=[...])"""
    _check("eqat_init_minmax_batched", lib().eqat_init_minmax_batched(b.n, b.descs, b.ptr["W"], b.ptr["s"], b.ptr["z"], _stream()))


def eqat_pack_batched(b: Batch):
    """b: Batch(descs, W=, s=, z=, Wpacked=, zpacked=)"""
    _check("eqat_pack_batched", lib().eqat_pack_batched(b.n, b.descs, b.ptr["W"], b.ptr["s"], b.ptr["z"], b.ptr["Wpacked"],
                                                        b.ptr["zpacked"], _stream()))


def eqat_fq_quantize_batched(b: Batch):
    """b: Batch(descs, W=, s=, z=, ws=): Eq.(1) of every linear in one launch, kept in its workspace (EQAT_OP_FQ_BWD size)."""
    _check("eqat_fq_quantize_batched", lib().eqat_fq_quantize_batched(b.n, b.descs, b.ptr["W"], b.ptr["s"], b.ptr["z"],
                                                                      b.ptr["ws"], b.ws_bytes, _stream()))


def eqat_fq_linear_fwd(X, W, s, z, bits, group, Y=None, ws=None, keep=False, kept=False):
    """keep=True: `ws` (EQAT_OP_FQ_BWD size, must then be given) is left holding what eqat_fq_linear_bwd(kept=True) needs.
    kept=True: `ws` already holds that (from keep=True or eqat_fq_quantize_batched) and Eq.(1) is not run again."""
    T, I = X.shape
    O = W.shape[0]
    d = _desc_ref(T, I, O, int(bits), int(group), _dt(X), _dt(W))
    Y = torch.empty((T, O), dtype=X.dtype, device=X.device) if Y is None else Y
    if (keep or kept) and ws is None:
        raise ValueError("keep / kept need the caller's workspace (it is the thing that is kept)")
    ws = workspace(make_desc(T, I, O, bits, group, _dt(X), _dt(W)), OP_FQ_FWD, X.device) if ws is None else ws
    name = "eqat_fq_linear_fwd_kept" if kept else "eqat_fq_linear_fwd_keep" if keep else "eqat_fq_linear_fwd"
    _check(name, getattr(lib(), name)(d, _p(X), _p(W), _p(s), _p(z), _p(Y), _p(ws), ws.numel(), _stream()))
    return Y


def eqat_fq_linear_bwd(X, W, s, z, dY, bits, group, want=("dX", "dW", "ds", "dz"), out=None, ws=None, kept=False):
    T, O = dY.shape
    I = W.shape[1]
    d = _desc_ref(T, I, O, int(bits), int(group), _dt(dY), _dt(W))
    G = _groups(I, group)
    out = {} if out is None else out
    if "dX" in want and "dX" not in out: out["dX"] = torch.empty((T, I), dtype=dY.dtype, device=dY.device)
    if "dW" in want and "dW" not in out: out["dW"] = torch.empty((O, I), dtype=W.dtype, device=dY.device)
    if "ds" in want and "ds" not in out: out["ds"] = torch.empty((O, G), dtype=torch.float32, device=dY.device)
    if "dz" in want and "dz" not in out: out["dz"] = torch.empty((O, G), dtype=torch.float32, device=dY.device)
    if kept and ws is None:
        raise ValueError("kept=True needs the workspace the forward call left")
    ws = workspace(make_desc(T, I, O, bits, group, _dt(dY), _dt(W)), OP_FQ_BWD, dY.device) if ws is None else ws
    name = "eqat_fq_linear_bwd_kept" if kept else "eqat_fq_linear_bwd"
    _check(name, getattr(lib(), name)(
        d, _p(X), _p(W), _p(s), _p(z), _p(dY), _p(out.get("dX")), _p(out.get("dW")), _p(out.get("ds")),
        _p(out.get("dz")), _p(ws), ws.numel(), _stream()))
    return out


def eqat_pack(W, s, z, bits, group, Wpacked=None, zpacked=None):
    O, I = W.shape
    d = make_desc(0, I, O, bits, group, BF16, _dt(W))
    nw, nz = lib().eqat_packed_w_bytes(ctypes.byref(d)), lib().eqat_packed_z_bytes(ctypes.byref(d))
    if nw == 0:
        _check("eqat_pack", lib().eqat_validate_desc(ctypes.byref(d)) or 2)
    Wpacked = torch.empty((O, nw // O), dtype=torch.uint8, device=W.device) if Wpacked is None else Wpacked
    zpacked = torch.empty((O, nz // O), dtype=torch.uint8, device=W.device) if zpacked is None else zpacked
    _check("eqat_pack", lib().eqat_pack(ctypes.byref(d), _p(W), _p(s), _p(z), _p(Wpacked), _p(zpacked), _stream()))
    return Wpacked, zpacked


def eqat_unpack(Wpacked, zpacked, in_features, bits, group):
    O, I = Wpacked.shape[0], int(in_features)
    d = make_desc(0, I, O, bits, group, BF16, BF16)
    codes = torch.empty((O, I), dtype=torch.int32, device=Wpacked.device)
    zc = torch.empty((O, _groups(I, group)), dtype=torch.int32, device=Wpacked.device)
    _check("eqat_unpack", lib().eqat_unpack(ctypes.byref(d), _p(Wpacked), _p(zpacked), _p(codes), _p(zc), _stream()))
    return codes, zc


def eqat_qlinear_fwd(X, Wpacked, s, zpacked, bits, group, Y=None, ws=None, keep=False):
    """keep=True: `ws` (EQAT_OP_Q_BWD size, must then be given) is left holding what eqat_qlinear_bwd(kept=True) needs."""
    T, I = X.shape
    O = Wpacked.shape[0]
    d = _desc_ref(T, I, O, int(bits), int(group), _dt(X), BF16)
    Y = torch.empty((T, O), dtype=X.dtype, device=X.device) if Y is None else Y
    if keep and ws is None:
        raise ValueError("keep=True needs the caller's workspace (it is the thing that is kept)")
    ws = workspace(make_desc(T, I, O, bits, group, _dt(X), BF16), OP_Q_FWD, X.device) if ws is None else ws
    name = "eqat_qlinear_fwd_keep" if keep else "eqat_qlinear_fwd"
    _check(name, getattr(lib(), name)(d, _p(X), _p(Wpacked), _p(s), _p(zpacked), _p(Y), _p(ws), ws.numel(),
                                      _stream()))
    return Y


def eqat_qlinear_bwd(X, Wpacked, s, zpacked, dY, in_features, bits, group, want=("dX", "ds"), out=None, ws=None,
                     kept=False):
    T, O = dY.shape
    I = int(in_features)
    d = _desc_ref(T, I, O, int(bits), int(group), _dt(dY), BF16)
    out = {} if out is None else out
    if "dX" in want and "dX" not in out: out["dX"] = torch.empty((T, I), dtype=dY.dtype, device=dY.device)
    if "ds" in want and "ds" not in out: out["ds"] = torch.empty((O, _groups(I, group)), dtype=torch.float32, device=dY.device)
    if kept and ws is None:
        raise ValueError("kept=True needs the workspace the forward call left")
    ws = workspace(make_desc(T, I, O, bits, group, _dt(dY), BF16), OP_Q_BWD, dY.device) if ws is None else ws
    name = "eqat_qlinear_bwd_kept" if kept else "eqat_qlinear_bwd"
    _check(name, getattr(lib(), name)(d, _p(X), _p(Wpacked), _p(s), _p(zpacked), _p(dY),
                                      _p(out.get("dX")), _p(out.get("ds")), _p(ws), ws.numel(), _stream()))
    return out


def eqat_qlinear_fwd_z(X, Wpacked, s, z, bits, group, Y=None, ws=None):
    """E2E-QP forward with floating-point (trained) zero points z [O,G]."""
    T, I = X.shape
    O = Wpacked.shape[0]
    d = _desc_ref(T, I, O, int(bits), int(group), _dt(X), BF16)
    Y = torch.empty((T, O), dtype=X.dtype, device=X.device) if Y is None else Y
    ws = workspace(make_desc(T, I, O, bits, group, _dt(X), BF16), OP_Q_FWD, X.device) if ws is None else ws
    _check("eqat_qlinear_fwd_z", lib().eqat_qlinear_fwd_z(d, _p(X), _p(Wpacked), _p(s), _p(z), _p(Y),
                                                          _p(ws), ws.numel(), _stream()))
    return Y


def eqat_qlinear_bwd_z(X, Wpacked, s, z, dY, in_features, bits, group, want=("dX", "ds", "dz"), out=None, ws=None):
    """E2E-QP backward with trained step sizes and zero points: dX, ds, dz."""
    T, O = dY.shape
    I = int(in_features)
    d = _desc_ref(T, I, O, int(bits), int(group), _dt(dY), BF16)
    out = {} if out is None else out
    G = _groups(I, group)
    if "dX" in want and "dX" not in out: out["dX"] = torch.empty((T, I), dtype=dY.dtype, device=dY.device)
    if "ds" in want and "ds" not in out: out["ds"] = torch.empty((O, G), dtype=torch.float32, device=dY.device)
    if "dz" in want and "dz" not in out: out["dz"] = torch.empty((O, G), dtype=torch.float32, device=dY.device)
    ws = workspace(make_desc(T, I, O, bits, group, _dt(dY), BF16), OP_Q_BWD, dY.device) if ws is None else ws
    _check("eqat_qlinear_bwd_z", lib().eqat_qlinear_bwd_z(d, _p(X), _p(Wpacked), _p(s), _p(z), _p(dY),
                                                          _p(out.get("dX")), _p(out.get("ds")), _p(out.get("dz")),
                                                          _p(ws), ws.numel(), _stream()))
    return out


def eqat_qlinear_prepare(Wpacked, zpacked, in_features, bits, group, act_dtype=BF16, prepared=None):
    """One-time preparation of a packed layer for E2E-QP steps (codes frozen): returns the prepared buffer."""
    O, I = Wpacked.shape[0], int(in_features)
    d = make_desc(0, I, O, bits, group, act_dtype, BF16)
    n = lib().eqat_prepared_bytes(ctypes.byref(d))
    if n == 0:
        _check("eqat_qlinear_prepare", lib().eqat_validate_desc(ctypes.byref(d)) or 2)
    prepared = torch.empty(n, dtype=torch.uint8, device=Wpacked.device) if prepared is None else prepared
    _check("eqat_qlinear_prepare", lib().eqat_qlinear_prepare(ctypes.byref(d), _p(Wpacked), _p(zpacked), _p(prepared),
                                                               prepared.numel(), _stream()))
    return prepared


def eqat_qlinear_fwd_prepared(X, prepared, s, out_features, bits, group, z=None, Y=None, ws=None, keep=False):
    """keep=True: eqat_qlinear_fwd_prepared_keep (ws of OP_QP_BWD size, left holding the (s, z) pairs)."""
    T, I = X.shape
    O = int(out_features)
    d = _desc_ref(T, I, O, int(bits), int(group), _dt(X), BF16)
    Y = torch.empty((T, O), dtype=X.dtype, device=X.device) if Y is None else Y
    ws = workspace(make_desc(T, I, O, bits, group, _dt(X), BF16), OP_QP_BWD if keep else OP_QP_FWD, X.device) if ws is None else ws
    name = "eqat_qlinear_fwd_prepared_keep" if keep else "eqat_qlinear_fwd_prepared"
    _check(name, getattr(lib(), name)(
        d, _p(X), _p(prepared), _p(s), _p(z), _p(Y), _p(ws), ws.numel(), _stream()))
    return Y


def eqat_qlinear_bwd_prepared(X, prepared, s, dY, in_features, bits, group, z=None, want=("dX", "ds"), out=None, ws=None,
                              kept=False):
    """kept=True: eqat_qlinear_bwd_prepared_kept (ws as eqat_qlinear_fwd_prepared_keep left it, same s and z)."""
    T, O = dY.shape
    I = int(in_features)
    d = _desc_ref(T, I, O, int(bits), int(group), _dt(dY), BF16)
    out = {} if out is None else out
    G = _groups(I, group)
    if "dX" in want and "dX" not in out: out["dX"] = torch.empty((T, I), dtype=dY.dtype, device=dY.device)
    if "ds" in want and "ds" not in out: out["ds"] = torch.empty((O, G), dtype=torch.float32, device=dY.device)
    if "dz" in want and "dz" not in out: out["dz"] = torch.empty((O, G), dtype=torch.float32, device=dY.device)
    ws = workspace(make_desc(T, I, O, bits, group, _dt(dY), BF16), OP_QP_BWD, dY.device) if ws is None else ws
    name = "eqat_qlinear_bwd_prepared_kept" if kept else "eqat_qlinear_bwd_prepared"
    _check(name, getattr(lib(), name)(
        d, _p(X), _p(prepared), _p(s), _p(z), _p(dY), _p(out.get("dX")), _p(out.get("ds")), _p(out.get("dz")),
        _p(ws), ws.numel(), _stream()))
    return out


def eqat_unpack_state(kind, state, out_features, in_features, bits, group, want_clamped=False):
    """Test aid: (codes int32 [O,I], clamped uint8 [O,I] or None, zbar float32 [O,G]) of a kept workspace / prepared layer."""
    O, I = int(out_features), int(in_features)
    d = make_desc(0, I, O, bits, group, BF16, BF16)
    codes = torch.empty((O, I), dtype=torch.int32, device=state.device)
    clamped = torch.empty((O, I), dtype=torch.uint8, device=state.device) if want_clamped else None
    zbar = torch.empty((O, _groups(I, group)), dtype=torch.float32, device=state.device)
    _check("eqat_unpack_state", lib().eqat_unpack_state(ctypes.byref(d), int(kind), _p(state), _p(codes), _p(clamped),
                                                        _p(zbar), _stream()))
    return codes, clamped, zbar


def eqat_recon_loss(Y, Yref, want_dY=True, loss=None, dY=None, ws=None):
    """(loss, dY): loss is a 1-element fp32 device tensor, dY has Y's dtype (None if not wanted)."""
    n = Y.numel()
    loss = torch.empty(1, dtype=torch.float32, device=Y.device) if loss is None else loss
    if want_dY and dY is None:
        dY = torch.empty_like(Y)
    if ws is None:
        ws = torch.empty(lib().eqat_recon_loss_workspace_bytes(), dtype=torch.uint8, device=Y.device)
    _check("eqat_recon_loss", lib().eqat_recon_loss(n, _dt(Y), _p(Y), _p(Yref), _p(loss), _p(dY if want_dY else None),
                                                    _p(ws), ws.numel(), _stream()))
    return loss, (dY if want_dY else None)


def eqat_recon_loss_static(Y, Yref, loss, dY=None):
    """eqat_recon_loss without a workspace and without any allocation: the caller passes every output."""
    _check("eqat_recon_loss_static", lib().eqat_recon_loss_static(Y.numel(), _dt(Y), _p(Y), _p(Yref), _p(loss), _p(dY),
                                                                  _stream()))
    return loss, dY


def eqat_block_ap_update(hyper: AdamW, bits, group, W=None, dW=None, mW=None, vW=None, s=None, ds=None, ms=None, vs=None,
                         z=None, dz=None, mz=None, vz=None, shape=None):
    """One AdamW step in place on whichever of W, s, z is given (with its gradient and two fp32 moment tensors).
    `shape` = (O, I) is needed only when W is not given."""
    O, I = W.shape if W is not None else shape
    d = make_desc(0, I, O, bits, group, BF16, _dt(W) if W is not None else F32)
    _check("eqat_block_ap_update", lib().eqat_block_ap_update(
        ctypes.byref(d), ctypes.byref(hyper), _p(W), _p(s), _p(z), _p(dW), _p(ds), _p(dz), _p(mW), _p(vW), _p(ms), _p(vs),
        _p(mz), _p(vz), _stream()))


def _i32(name, value):
    """A number that travels in 32 bits: ctypes would cut it without a word."""
    value = int(value)
    if not -2 ** 31 <= value < 2 ** 31:
        raise ValueError(f"{name} does not fit 32 bits: {value}")
    return value


class KvCache:
    """A pool of pages for keys and values in 4 bits, and its descriptor.  `pool`: the caller's own uint8 device tensor, 256-byte aligned."""

    def __init__(self, heads, head_dim, group, page_tokens, pages, dtype=torch.bfloat16, device="cuda", pool=None):
        self.heads, self.head_dim, self.dtype = _i32("heads", heads), _i32("head_dim", head_dim), dtype
        self.desc = KvDesc(_i32("pages", pages), self.heads, self.head_dim, _i32("group", group), _i32("page_tokens", page_tokens), F32 if dtype == torch.float32 else BF16)
        self.ref = ctypes.byref(self.desc)
        if dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"unsupported dtype {dtype}")
        n = lib().eqat_kv_pool_bytes(self.ref)
        if n == 0:
            raise ValueError(f"eqat_kv_pool_bytes: no cache of {heads} heads of {head_dim}, groups of {group}, {pages} pages of {page_tokens} tokens")
        self.pool = torch.empty(n, dtype=torch.uint8, device=device) if pool is None else pool
        if self.pool.dtype != torch.uint8 or not self.pool.is_contiguous() or self.pool.numel() < n:
            raise ValueError(f"the pool is a contiguous uint8 tensor of at least {n} bytes")


class KvBatch:
    """Where the sequences of a call stand (int32 device tensors, kept and read on the device at every call): the pages of each, how many tokens it holds with the
    newest, and where the newest tokens' rows start.  tokens, max_new, max_len: the rows in all, and bounds on both numbers of any sequence.  Build once, call often."""

    def __init__(self, table, lens, starts, tokens, max_new, max_len):
        B = lens.numel()
        for t in (table, lens, starts):
            if t.dtype != torch.int32:
                raise TypeError("table, lens and starts are int32")
        if table.dim() != 2 or table.shape[0] != B or starts.numel() != B + 1:
            raise ValueError("table is [sequences, pages], lens [sequences], starts [sequences + 1]")
        self.keep = (table, lens, starts)            # they must outlive the pointers
        self.tokens = int(tokens)
        self.desc = KvBatchDesc(_p(table), _p(lens), _p(starts), self.tokens, B, _i32("pages of a sequence", table.shape[1]), _i32("max_new", max_new), _i32("max_len", max_len))
        self.ref = ctypes.byref(self.desc)

    @functools.cached_property
    def device(self):
        """The device that all three are on."""
        table, lens, starts = (t.get_device() for t in self.keep)
        if not table == lens == starts:
            raise ValueError(f"table, lens and starts on devices {table}, {lens} and {starts}")
        return table


@functools.lru_cache(maxsize=1024)
def _kv_strides(shape, stride, tokens, heads, head_dim):
    """{token, head} strides of a [tokens, heads, head_dim] tensor whose heads are contiguous, in memory: (address, the array itself).  The cache is by value."""
    if tuple(shape) != (tokens, heads, head_dim):
        raise ValueError(f"expected [{tokens}, {heads}, {head_dim}], got {list(shape)}")
    if stride[2] != 1:
        raise ValueError("the elements of a head must be contiguous")
    both = (ctypes.c_int64 * 2)(stride[0], stride[1])
    return ctypes.addressof(both), both


@functools.lru_cache(maxsize=1024)
def _kv_attn_ref(q_heads, causal, window, scale):
    return ctypes.byref(KvAttn(_i32("q_heads", q_heads), causal, _i32("window", window), scale))


def _kv_rows(cache, batch, t, heads):
    """(pointer, (address of its strides, their array)) of a [tokens, heads, head_dim] tensor"""
    if t is None:
        return None, _NO_STRIDES
    if t.dtype != cache.dtype or not t.is_cuda:
        raise ValueError(f"expected a {cache.dtype} device tensor, got {t.dtype} on {t.device}")
    return t.data_ptr(), _kv_strides(t.shape, t.stride(), batch.tokens, heads, cache.head_dim)


_NO_STRIDES = (None, None)


def eqat_kv_write(cache: KvCache, batch: KvBatch, k, v):
    """The newest tokens' keys and values [tokens, heads, head_dim] (any token and head strides) into the cache."""
    (kp, ks), (vp, vs) = _kv_rows(cache, batch, k, cache.heads), _kv_rows(cache, batch, v, cache.heads)
    _check("eqat_kv_write", lib().eqat_kv_write(cache.ref, batch.ref, kp, ks[0], vp, vs[0], _p(cache.pool), _stream()))


def eqat_kv_read(cache: KvCache, batch: KvBatch, k=None, v=None, want=("k", "v")):
    """(k, v): the newest tokens' keys and values as they stand in the cache.  Given tensors are filled; `want` says which to make where neither is given."""
    if k is None and v is None:
        k, v = (torch.empty((batch.tokens, cache.heads, cache.head_dim), dtype=cache.dtype, device=cache.pool.device) if name in want else None for name in ("k", "v"))
    (kp, ks), (vp, vs) = _kv_rows(cache, batch, k, cache.heads), _kv_rows(cache, batch, v, cache.heads)
    _check("eqat_kv_read", lib().eqat_kv_read(cache.ref, batch.ref, kp, ks[0], vp, vs[0], _p(cache.pool), _stream()))
    return k, v


def kv_workspace(cache: KvCache, batch: KvBatch, q_heads) -> torch.Tensor:
    """The workspace of eqat_kv_attention, zeroed as its first use wants it.  It serves every later call with bounds no larger than this batch's."""
    n = lib().eqat_kv_workspace_bytes(cache.ref, batch.ref, _i32("q_heads", q_heads))
    return torch.zeros(max(n, 256), dtype=torch.uint8, device=cache.pool.device)


def eqat_kv_attention(cache: KvCache, batch: KvBatch, q, scale=0.0, causal=True, window=0, out=None, lse=None, ws=None):
    """Attention of the newest tokens' queries [tokens, q_heads, head_dim] over what their sequences hold; lse: fp32 [tokens, q_heads] to fill, or None."""
    q_heads = q.shape[1]
    out = torch.empty((batch.tokens, q_heads, cache.head_dim), dtype=q.dtype, device=q.device) if out is None else out
    (qp, qs), (op, os_) = _kv_rows(cache, batch, q, q_heads), _kv_rows(cache, batch, out, q_heads)
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (batch.tokens, q_heads)):
        raise ValueError("lse is fp32 [tokens, q_heads]")
    ws = kv_workspace(cache, batch, q_heads) if ws is None else ws
    a = _kv_attn_ref(q_heads, 1 if causal else 0, int(window), float(scale))
    _check("eqat_kv_attention", lib().eqat_kv_attention(cache.ref, batch.ref, a, qp, qs[0], op, os_[0], _p(lse), _p(cache.pool),
                                                        _p(ws), ws.numel(), _stream()))
    return out


# ---- norm, rotary positions, gated feed-forward ---------------------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=1024)
def _norm_ref(tokens, width, group, act_dtype, w_dtype, eps):
    return ctypes.byref(NormDesc(tokens, _i32("width", width), _i32("group", group), act_dtype, w_dtype, eps))


# As above, what happens here is what bounds the smallest calls (a launch is 3 us of their 6): shapes are compared as they are, what a call goes by is looked up once, and the calls of a decoding step
# look at their tensors in place.  All tensors of a call are on one device, which has to be the current one: the call goes to its current stream.
_CODES = {torch.float32: F32, torch.bfloat16: BF16}


def _unlike(name, t, shape, dtype, device):
    raise ValueError(f"{name}: expected a contiguous {dtype} tensor {list(shape)} on device {device}, got {t.dtype} {list(t.shape)} on {t.device}")


def _stream_at(device):
    """The current stream of the device that a call's tensors are on (-1: the host)."""
    if device < 0 or device != _device():
        raise ValueError(f"tensors of device {device} (-1: the host) that is not the current device")
    return _raw_stream(device)


def _like(name, t, shape, dtype, device):
    """The pointer of a tensor whose shape and type the call goes by; None stays None."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        _unlike(name, t, shape, dtype, device)
    return t.data_ptr()


def _like_w(W, n, device):
    """(pointer, type) of a norm's weights; None stays None."""
    if W is None:
        return None, F32
    dtype = W.dtype
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}")
    if W.shape != (n,) or W.get_device() != device or not W.is_contiguous():
        _unlike("W", W, (n,), dtype, device)
    return W.data_ptr(), code


def _ws_like(ws, device):
    """The pointer of a call's workspace: on the device of the call's tensors."""
    if ws.get_device() != device or not ws.is_contiguous():
        raise ValueError(f"ws: expected a contiguous tensor on device {device}, got one on {ws.device}")
    return ws.data_ptr()


def _codes_ptr(codes, shape, device):
    if codes.dtype is not torch.uint8 and codes.dtype is not torch.float8_e4m3fn:
        raise ValueError(f"codes: expected float8_e4m3fn or uint8, got {codes.dtype}")
    return _like("codes", codes, shape, codes.dtype, device)


_Y, _S_AND_Y, _CODED, _S_AND_CODED = ("Y",), ("S", "Y"), ("codes",), ("S", "codes")


def eqat_norm_fwd(X, W, eps, R=None, group=0, want=None, out=None):
    """Root-mean-square norm of S = X + R (R None: of X) over the rows of [tokens, width]; W [width] or None.  `want`: which of "S", "Y", "codes" (float8_e4m3fn, with "scales", one
    for `group` neighbouring elements, -1: a row) to make, by default Y, or the codes where a group is given, and S where R is; tensors in `out` are filled."""
    shape, dtype, device = X.shape, X.dtype, X.get_device()
    T, n = shape
    act = _CODES.get(dtype)
    if act is None:
        raise TypeError(f"unsupported dtype {dtype}")
    if not X.is_contiguous():
        _unlike("X", X, shape, dtype, device)
    if want is None:
        want = (_Y if R is None else _S_AND_Y) if not group else _CODED if R is None else _S_AND_CODED
    if out is None: out = {}
    r = s = y = codes = scales = None
    if R is not None:
        if R.shape != shape or R.dtype is not dtype or R.get_device() != device or not R.is_contiguous():
            _unlike("R", R, shape, dtype, device)
        r = R.data_ptr()
    if "S" in want:
        S = out.get("S")
        if S is None:
            S = out["S"] = torch.empty_like(X)
        elif S.shape != shape or S.dtype is not dtype or S.get_device() != device or not S.is_contiguous():
            _unlike("S", S, shape, dtype, device)
        s = S.data_ptr()
    if "Y" in want:
        Y = out.get("Y")
        if Y is None:
            Y = out["Y"] = torch.empty_like(X)
        elif Y.shape != shape or Y.dtype is not dtype or Y.get_device() != device or not Y.is_contiguous():
            _unlike("Y", Y, shape, dtype, device)
        y = Y.data_ptr()
    if "codes" in want or "scales" in want:
        group = _i32("group", group)
        if group == 0:
            raise ValueError("codes need a group (-1: one scale a row)")
        per = n // group if group > 0 else 1
        if "codes" not in out: out["codes"] = torch.empty((T, n), dtype=torch.float8_e4m3fn, device=X.device)
        if "scales" not in out: out["scales"] = torch.empty((T, per), dtype=torch.float32, device=X.device)
        codes, scales = _codes_ptr(out["codes"], shape, device), _like("scales", out["scales"], (T, per), torch.float32, device)
    else:
        group = -1
    w, w_type = _like_w(W, n, device)
    status = lib().eqat_norm_fwd(_norm_ref(T, n, group, act, w_type, float(eps)), X.data_ptr(), r, w, s, y, codes, scales, _stream_at(device))
    if status:
        _check("eqat_norm_fwd", status)
    return out


def norm_workspace(tokens, width, dtype=torch.bfloat16, device="cuda") -> torch.Tensor:
    """The workspace of eqat_norm_bwd."""
    n = lib().eqat_norm_workspace_bytes(_norm_ref(int(tokens), int(width), -1, BF16 if dtype == torch.bfloat16 else F32, F32, 0.0))
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def eqat_norm_bwd(S, W, eps, dY, dS=None, want=("dX", "dW"), out=None, ws=None):
    """Gradients of eqat_norm_fwd from S (what it left, or its X): dX (also that of R) in S's type, dW fp32 [width].  dS: the gradient that reaches S along the residual."""
    shape, dtype, device = S.shape, S.dtype, S.get_device()
    T, n = shape
    act = _dt(S)
    out = {} if out is None else out
    dX = dW = None
    if "dX" in want:
        dX = out.get("dX")
        if dX is None: dX = out["dX"] = torch.empty_like(S)
        dX = _like("dX", dX, shape, dtype, device)
    if "dW" in want:
        dW = out.get("dW")
        if dW is None: dW = out["dW"] = torch.empty(n, dtype=torch.float32, device=S.device)
        dW = _like("dW", dW, (n,), torch.float32, device)
        if ws is None: ws = norm_workspace(T, n, dtype, S.device)
    w, w_type = _like_w(W, n, device)
    status = lib().eqat_norm_bwd(_norm_ref(T, n, -1, act, w_type, float(eps)), _like("S", S, shape, dtype, device), w, _like("dY", dY, shape, dtype, device), _like("dS", dS, shape, dtype, device), dX, dW,
                                 None if ws is None else _ws_like(ws, device), 0 if ws is None else ws.numel(), _stream_at(device))
    if status:
        _check("eqat_norm_bwd", status)
    return out


def rotary_frequencies(part, base=10000.0, stretch=1.0, short=256.0, long=2048.0):
    """fp32 frequencies base^(-2 i / part) of `part` / 2 pairs (on the host).  stretch > 1, for contexts that many times longer: wave lengths of `long` tokens and more are stretched by it,
    those below `short` tokens are kept, between the two in proportion to their logarithm."""
    if part % 2 or not (base > 0 and stretch >= 1.0 and 0.0 < short < long):
        raise ValueError("part is even, base positive, stretch 1 or more, 0 < short < long")
    i = torch.arange(int(part) // 2, dtype=torch.float64)
    f = float(base) ** (-2.0 * i / int(part))
    if stretch > 1.0:
        slow = ((2.0 * torch.pi / f / short).log() / torch.tensor(long / short, dtype=torch.float64).log()).clamp(0.0, 1.0)
        f = f * (1.0 - slow) + f / stretch * slow
    return f.float()


class Rotary:
    """How positions turn queries and keys: fp32 device frequencies of the pairs of a head's first 2 * len(frequencies) elements, (i, i + that half), or neighbours where
    `interleaved`; `amplitude` times.  Build once, call often."""

    def __init__(self, frequencies, head_dim, interleaved=False, amplitude=1.0):
        if frequencies.dtype != torch.float32 or frequencies.dim() != 1:
            raise TypeError("frequencies are fp32 [pairs]")
        self.frequencies, self.head_dim, self.device = frequencies, _i32("head_dim", head_dim), frequencies.get_device()          # the tensor must outlive the pointer
        at, part = _p(frequencies), 2 * frequencies.numel()
        self.descs = {dt: RotaryDesc(at, self.head_dim, part, 1 if interleaved else 0, code, float(amplitude)) for dt, code in ((torch.float32, F32), (torch.bfloat16, BF16))}
        self.refs = {dt: ctypes.byref(d) for dt, d in self.descs.items()}


@functools.lru_cache(maxsize=1024)
def _both_rows(shape, stride, out_stride, tokens, head_dim):
    """(heads, addresses of the {token, head} strides in memory of a [tokens, heads, head_dim] tensor and of where it goes, their arrays); the cache is by value"""
    if len(shape) != 3:
        raise ValueError("expected [tokens, heads, head_dim]")
    here, there = (_kv_strides(shape, x, tokens, shape[1], head_dim) for x in (stride, out_stride))
    return shape[1], here[0], there[0], here[1], there[1]


_NOTHING = (None, None, 0, None, None)


def _turned(t, out, tokens, dtype, head_dim, device):
    """(pointer, strides, heads, pointer, strides) of what is turned and of where it goes, and what the strides' addresses live in, which has to be held until the call returns"""
    shape = t.shape
    if t.dtype is not dtype or out.dtype is not dtype or t.get_device() != device or out.get_device() != device:
        raise ValueError(f"expected {dtype} tensors on device {device}, got {t.dtype} on {t.device} and {out.dtype} on {out.device}")
    if out.shape != shape:
        raise ValueError(f"expected {list(shape)}, got {list(out.shape)}")
    rows = _both_rows(shape, t.stride(), out.stride(), tokens, head_dim)
    return (t.data_ptr(), rows[1], rows[0], out.data_ptr(), rows[2]), rows


def eqat_rotary(rot: Rotary, positions, q=None, k=None, q_out=None, k_out=None, inverse=False):
    """(q, k) [tokens, heads, head_dim] (any token and head strides) turned by their tokens' positions (int32 [tokens]); into q_out, k_out (which may be q and k themselves)."""
    device = positions.get_device()
    if positions.dtype is not torch.int32 or positions.dim() != 1:
        raise TypeError("positions are int32 [tokens]")
    if not positions.is_contiguous():
        _unlike("positions", positions, positions.shape, torch.int32, device)
    if rot.device != device:
        raise ValueError(f"frequencies on device {rot.device}, tensors on {device}")
    if (q is None and q_out is not None) or (k is None and k_out is not None):
        raise ValueError("an output without its input")
    T, like = positions.numel(), q if q is not None else k
    if like is None:
        return None, None
    dtype, head_dim = like.dtype, rot.head_dim
    ref = rot.refs.get(dtype)
    if ref is None:
        raise TypeError(f"unsupported dtype {dtype}")
    of_q = of_k = _NOTHING
    if q is not None:
        if q_out is None: q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        of_q, q_rows = _turned(q, q_out, T, dtype, head_dim, device)
    if k is not None:
        if k_out is None: k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        of_k, k_rows = _turned(k, k_out, T, dtype, head_dim, device)
    status = lib().eqat_rotary(ref, T, positions.data_ptr(), *of_q, *of_k, 1 if inverse else 0, _stream_at(device))
    if status:
        _check("eqat_rotary", status)
    return q_out, k_out


def eqat_kv_rotary_write(cache: KvCache, batch: KvBatch, rot: Rotary, q, k, v, q_out=None):
    """The newest tokens' queries turned (returned, into q_out if given, which may be q itself), their keys turned and values into the cache: eqat_rotary and eqat_kv_write in one launch."""
    device, dtype, tokens, head_dim = cache.pool.get_device(), cache.dtype, batch.tokens, cache.head_dim
    if rot.device != device:
        raise ValueError(f"frequencies on device {rot.device}, tensors on {device}")
    if batch.device != device:
        raise ValueError(f"table, lens and starts on device {batch.device}, tensors on {device}")
    if rot.head_dim != head_dim:
        raise ValueError(f"heads of {rot.head_dim} in a cache of heads of {head_dim}")
    if q_out is None: q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k.dtype is not dtype or v.dtype is not dtype or k.get_device() != device or v.get_device() != device:
        raise ValueError(f"expected {dtype} tensors on device {device}, got {k.dtype} on {k.device} and {v.dtype} on {v.device}")
    ks, vs = _kv_strides(k.shape, k.stride(), tokens, cache.heads, head_dim), _kv_strides(v.shape, v.stride(), tokens, cache.heads, head_dim)
    of_q, q_rows = _turned(q, q_out, tokens, dtype, head_dim, device)
    status = lib().eqat_kv_rotary_write(cache.ref, batch.ref, rot.refs[dtype], *of_q, k.data_ptr(), ks[0], v.data_ptr(), vs[0], cache.pool.data_ptr(),
                                        _stream_at(device))
    if status:
        _check("eqat_kv_rotary_write", status)
    return q_out


def eqat_gate_fwd(Y, kind=GATE_SILU, H=None):
    """H [tokens, F] = act(G) U of Y = [G | U] [tokens, 2 F]."""
    T, F, device = Y.shape[0], Y.shape[1] // 2, Y.get_device()
    H = torch.empty((T, F), dtype=Y.dtype, device=Y.device) if H is None else H
    _check("eqat_gate_fwd", lib().eqat_gate_fwd(T, F, _dt(Y), int(kind), _like("Y", Y, (T, 2 * F), Y.dtype, device), _like("H", H, (T, F), Y.dtype, device), _stream_at(device)))
    return H


def eqat_gate_bwd(Y, dH, kind=GATE_SILU, want=("dY",), out=None):
    """The gradient dY of Y = [G | U] from that of H, and H itself where it is wanted."""
    T, F, device = Y.shape[0], Y.shape[1] // 2, Y.get_device()
    out = {} if out is None else out
    if "dY" in want and "dY" not in out: out["dY"] = torch.empty_like(Y)
    if "H" in want and "H" not in out: out["H"] = torch.empty((T, F), dtype=Y.dtype, device=Y.device)
    get = lambda name, shape: _like(name, out.get(name) if name in want else None, shape, Y.dtype, device)
    _check("eqat_gate_bwd", lib().eqat_gate_bwd(T, F, _dt(Y), int(kind), _like("Y", Y, (T, 2 * F), Y.dtype, device), _like("dH", dH, (T, F), Y.dtype, device), get("dY", Y.shape), get("H", (T, F)),
                                                _stream_at(device)))
    return out


def gated_workspace(tokens, in_features, F, bits, group, dtype=torch.bfloat16, prepared=False, device="cuda") -> torch.Tensor:
    """The workspace of eqat_gated_fwd and eqat_gated_bwd (or their calls on a prepared layer); that of more tokens serves fewer."""
    d = _desc_ref(int(tokens), int(in_features), 2 * int(F), int(bits), int(group), BF16 if dtype == torch.bfloat16 else F32, BF16)
    n = lib().eqat_gated_workspace_bytes(d)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


@functools.lru_cache(maxsize=1024)
def _packed_ok(w, s, z, I, bits, group):
    """Whether these are the shapes of a packed layer of an even number of rows and I inputs."""
    G = _groups(I, group)
    return len(w) == 2 and w[0] % 2 == 0 and tuple(w) == (w[0], I * bits // 8) and tuple(s) == (w[0], G) and tuple(z) == (w[0], 4 * ((G * bits + 31) // 32))


def _packed_layer(X, Wpacked, s, zpacked, bits, group):
    if (Wpacked.dtype is not torch.uint8 or zpacked.dtype is not torch.uint8 or s.dtype is not torch.float32 or not _packed_ok(Wpacked.shape, s.shape, zpacked.shape, X.shape[1], bits, group)
            or not (Wpacked.is_contiguous() and zpacked.is_contiguous() and s.is_contiguous()) or not Wpacked.get_device() == zpacked.get_device() == s.get_device() == X.get_device()):
        raise ValueError(f"not a contiguous packed layer of {X.shape[1]} inputs at {bits} bits in groups of {group} on {X.device}: codes {list(Wpacked.shape)}, step sizes {list(s.shape)}, "
                         f"zero points {list(zpacked.shape)}")
    return Wpacked.data_ptr(), s.data_ptr(), zpacked.data_ptr()


@functools.lru_cache(maxsize=1024)
def _prepared_bytes(F, I, bits, group, act_dtype):
    return lib().eqat_prepared_bytes(_desc_ref(0, I, 2 * F, bits, group, act_dtype, BF16))


def _prepared_layer(X, prepared, s, F, bits, group):
    I = X.shape[1]
    if (prepared.dtype is not torch.uint8 or prepared.numel() < _prepared_bytes(F, I, bits, group, _dt(X)) or s.dtype is not torch.float32 or s.shape != (2 * F, _groups(I, group))
            or not (prepared.is_contiguous() and s.is_contiguous()) or not prepared.get_device() == s.get_device() == X.get_device()):
        raise ValueError(f"not a contiguous prepared layer of {I} inputs and 2 x {F} outputs at {bits} bits in groups of {group} on {X.device}: {prepared.numel()} bytes, step sizes {list(s.shape)}")
    return prepared.data_ptr(), s.data_ptr()


def _gated(name, X, F, bits, group, layer, kind, dH, want, out, ws, prepared):
    (T, I), dtype, device = X.shape, X.dtype, X.get_device()
    act = _CODES.get(dtype)
    if act is None:
        raise TypeError(f"unsupported dtype {dtype}")
    if not X.is_contiguous():
        _unlike("X", X, X.shape, dtype, device)
    h = None
    back = ()
    if "H" in want:
        H = out.get("H")
        if H is None:
            H = out["H"] = torch.empty((T, F), dtype=dtype, device=X.device)
        elif H.shape != (T, F) or H.dtype is not dtype or H.get_device() != device or not H.is_contiguous():
            _unlike("H", H, (T, F), dtype, device)
        h = H.data_ptr()
    if dH is not None:
        dY = None
        if "dY" in want:
            dY = out.get("dY")
            if dY is None: dY = out["dY"] = torch.empty((T, 2 * F), dtype=dtype, device=X.device)
        back = (_like("dH", dH, (T, F), dtype, device), _like("dY", dY, (T, 2 * F), dtype, device))
    if ws is None: ws = gated_workspace(T, I, F, bits, group, dtype, prepared, X.device)
    status = getattr(lib(), name)(_desc_ref(T, I, 2 * F, bits, group, act, BF16), kind, X.data_ptr(), *layer, *back, h, _ws_like(ws, device), ws.numel(), _stream_at(device))
    if status:
        _check(name, status)
    return out


def eqat_gated_fwd(X, Wpacked, s, zpacked, bits, group, kind=GATE_SILU, H=None, ws=None):
    """H [tokens, F] = act(X Wg^T) * (X Wu^T) from the packed layer of the stacked projections [Wg; Wu] (2 F rows)."""
    return _gated("eqat_gated_fwd", X, Wpacked.shape[0] // 2, bits, group, _packed_layer(X, Wpacked, s, zpacked, bits, group), kind, None, ("H",), {} if H is None else {"H": H}, ws, False)["H"]


def eqat_gated_bwd(X, Wpacked, s, zpacked, dH, bits, group, kind=GATE_SILU, want=("dY", "H"), out=None, ws=None):
    """The gradient dY [tokens, 2 F] of the stacked projections' outputs from that of H, and H again; both projections are made anew from X."""
    return _gated("eqat_gated_bwd", X, Wpacked.shape[0] // 2, bits, group, _packed_layer(X, Wpacked, s, zpacked, bits, group), kind, dH, want, {} if out is None else out, ws, False)


def eqat_gated_fwd_prepared(X, prepared, s, F, bits, group, kind=GATE_SILU, H=None, ws=None):
    """eqat_gated_fwd on a layer prepared by eqat_qlinear_prepare."""
    return _gated("eqat_gated_fwd_prepared", X, int(F), bits, group, _prepared_layer(X, prepared, s, int(F), bits, group), kind, None, ("H",), {} if H is None else {"H": H}, ws, True)["H"]


def eqat_gated_bwd_prepared(X, prepared, s, dH, bits, group, kind=GATE_SILU, want=("dY", "H"), out=None, ws=None):
    """eqat_gated_bwd on a layer prepared by eqat_qlinear_prepare."""
    return _gated("eqat_gated_bwd_prepared", X, dH.shape[1], bits, group, _prepared_layer(X, prepared, s, dH.shape[1], bits, group), kind, dH, want, {} if out is None else out, ws, True)


def eqat_profile_start():
    _check("eqat_profile_start", lib().eqat_profile_start())


def eqat_profile_stop():
    """{kernel class: (total ms, launches)} for every class that ran since eqat_profile_start()."""
    n = lib().eqat_profile_kernels()
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int64 * n)()
    _check("eqat_profile_stop", lib().eqat_profile_stop(ms, cnt, n))
    return {lib().eqat_profile_kernel_name(k).decode(): (ms[k], cnt[k]) for k in range(n) if cnt[k]}
