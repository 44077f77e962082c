"""GB300 (sm_103a) Kalman Delta Network token mixers.

Thin Python binding of ``libkdn.so`` (C ABI in ``include/kdn.h``).  The
functions below carry the C entry points' names and only marshal arguments:
they check that every tensor is what the C ABI reads through its pointer (a
contiguous CUDA tensor of the expected dtype and element count), allocate
outputs and the scratch workspace with PyTorch (device memory is PyTorch's job
here), pass raw pointers and the current CUDA stream, and raise on any non-OK
status.  Every step of the computation runs in the library's
CUDA kernels; there is no CPU or PyTorch fallback, and importing a function
whose library is missing raises.

Layouts follow the C ABI: q, k [B,T,H,dk]; v [B,T,H,dv]; r [B,T,H];
diag g, omega [B,T,H,dk]; iso omega [B,T,H], g [B,T,H,dk] or [B,T,H];
S0 [B,H,dk,dv] float32; p0 diag [B,H,dk], iso [B,H] float32.

Streams: a call runs on the current stream, or on ``stream=``, which the caller orders
behind whatever made the inputs.  With ``stream=`` the workspace and outputs that the call
makes are that stream's memory and may be dropped at any time; the caller's own tensors stay
the caller's to keep until the stream has passed the call.

Device status: the tensor-core kernels wait for one another's copies and products with a
limit.  A wait that runs out leaves the call's outputs invalid and a code in the first word of
the workspace, not in the return value (the call is over before the kernels are).  A caller
who wants to know passes ``workspace=`` and reads it with kdn_get_device_status, which waits
for the stream; the status of a workspace that the call makes itself goes with it.

The hybrid layer's operators (sliding-window attention with sinks, the residual RMS norm,
rotary positions, the gated feed-forward block) are at the end of the module, with their
layouts.
"""
from __future__ import annotations

import ctypes
import math
import os
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkdn.so")

KDN_OK, KDN_ERR_INVALID_ARG, KDN_ERR_UNSUPPORTED, KDN_ERR_WORKSPACE, KDN_ERR_CUDA, \
    KDN_ERR_TIMEOUT, KDN_ERR_RANGE = range(7)
KDN_F32, KDN_BF16, KDN_F8E4M3 = 0, 1, 2
KDN_GATES_POST, KDN_GATES_LOGITS = 0, 1
KDN_ACT_SILU, KDN_ACT_GELU = 0, 1
R_MIN_DEFAULT = 0.01  # the layer's observation-noise floor

_DTYPES = {torch.float32: KDN_F32, torch.bfloat16: KDN_BF16}


class kdn_desc_t(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("T", ctypes.c_int), ("H", ctypes.c_int),
                ("dk", ctypes.c_int), ("dv", ctypes.c_int), ("chunk", ctypes.c_int),
                ("dtype", ctypes.c_int), ("mu", ctypes.c_float), ("scale", ctypes.c_float),
                ("decay_per_channel", ctypes.c_int), ("out_dtype", ctypes.c_int),
                ("gates", ctypes.c_int), ("r_min", ctypes.c_float)]


class kdn_swa_desc_t(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("T", ctypes.c_int), ("H", ctypes.c_int),
                ("Hk", ctypes.c_int), ("d", ctypes.c_int), ("window", ctypes.c_int),
                ("sinks", ctypes.c_int), ("dtype", ctypes.c_int), ("scale", ctypes.c_float)]


class kdn_norm_desc_t(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_longlong), ("D", ctypes.c_int), ("dtype", ctypes.c_int),
                ("out_dtype", ctypes.c_int), ("block", ctypes.c_int), ("eps", ctypes.c_float)]


class kdn_rope_freqs_t(ctypes.Structure):
    _fields_ = [("rot", ctypes.c_int), ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("trained", ctypes.c_double), ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double)]


class kdn_rope_desc_t(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("T", ctypes.c_int), ("H", ctypes.c_int), ("Hk", ctypes.c_int),
                ("d", ctypes.c_int), ("rot", ctypes.c_int), ("interleaved", ctypes.c_int),
                ("pos_per_token", ctypes.c_int), ("dtype", ctypes.c_int), ("mscale", ctypes.c_float),
                ("ldq", ctypes.c_longlong), ("ldk", ctypes.c_longlong), ("ldqo", ctypes.c_longlong),
                ("ldko", ctypes.c_longlong)]


class kdn_ffn_desc_t(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_longlong), ("D", ctypes.c_int), ("F", ctypes.c_int), ("dtype", ctypes.c_int),
                ("act", ctypes.c_int), ("dw_dtype", ctypes.c_int)]


class KdnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


_lib = None
_lock = threading.Lock()

_P = ctypes.c_void_p
_SIG = {
    "kdn_version": ([], ctypes.c_int),
    "kdn_status_string": ([ctypes.c_int], ctypes.c_char_p),
    "kdn_fwd_workspace_bytes": ([ctypes.POINTER(kdn_desc_t), ctypes.c_int], ctypes.c_size_t),
    "kdn_bwd_workspace_bytes": ([ctypes.POINTER(kdn_desc_t), ctypes.c_int], ctypes.c_size_t),
    "kdn_diag_fwd": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 12 + [ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_iso_fwd": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 12 + [ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_diag_bwd": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 21 + [ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_iso_bwd": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 21 + [ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_diag_decode_step": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 10, ctypes.c_int),
    "kdn_iso_decode_step": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 10, ctypes.c_int),
    "kdn_diag_fwd_noalloc": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 12, ctypes.c_int),
    "kdn_saved_bytes": ([ctypes.POINTER(kdn_desc_t), ctypes.c_int], ctypes.c_size_t),
    "kdn_diag_fwd_save": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 12 + [ctypes.c_size_t, _P,
                                                                   ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_diag_bwd_saved": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 7 + [ctypes.c_size_t] + [_P] * 13
                           + [ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_iso_fwd_save": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 12 + [ctypes.c_size_t, _P,
                                                                  ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_iso_bwd_saved": ([ctypes.POINTER(kdn_desc_t)] + [_P] * 7 + [ctypes.c_size_t] + [_P] * 13
                          + [ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_diag_beta_eff": ([ctypes.POINTER(kdn_desc_t), _P, ctypes.c_size_t, _P, _P, _P], ctypes.c_int),
    "kdn_iso_beta_eff": ([ctypes.POINTER(kdn_desc_t), _P, ctypes.c_size_t, _P, _P, _P], ctypes.c_int),
    "kdn_kernel_launches": ([ctypes.POINTER(kdn_desc_t), ctypes.c_int, ctypes.c_int], ctypes.c_int),
    "kdn_get_device_status": ([_P, _P], ctypes.c_int),
    "kdn_noalloc_device_status": ([_P], ctypes.c_int),
    "kdn_selftest_wait_timeout": ([_P, _P], ctypes.c_int),
    "kdn_swa_fwd_workspace_bytes": ([ctypes.POINTER(kdn_swa_desc_t)], ctypes.c_size_t),
    "kdn_swa_bwd_workspace_bytes": ([ctypes.POINTER(kdn_swa_desc_t)], ctypes.c_size_t),
    "kdn_swa_fwd": ([ctypes.POINTER(kdn_swa_desc_t)] + [_P] * 7 + [ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_swa_bwd": ([ctypes.POINTER(kdn_swa_desc_t)] + [_P] * 11 + [ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_swa_cache_fill": ([ctypes.POINTER(kdn_swa_desc_t)] + [_P] * 6, ctypes.c_int),
    "kdn_swa_decode_step": ([ctypes.POINTER(kdn_swa_desc_t)] + [_P] * 8, ctypes.c_int),
    "kdn_add_rmsnorm_fwd": ([ctypes.POINTER(kdn_norm_desc_t)] + [_P] * 8, ctypes.c_int),
    "kdn_add_rmsnorm_bwd_workspace_bytes": ([ctypes.POINTER(kdn_norm_desc_t)], ctypes.c_size_t),
    "kdn_add_rmsnorm_bwd": ([ctypes.POINTER(kdn_norm_desc_t)] + [_P] * 8 + [ctypes.c_size_t, _P],
                            ctypes.c_int),
    "kdn_rope_freqs": ([ctypes.POINTER(kdn_rope_freqs_t), _P, _P], ctypes.c_int),
    "kdn_rope_fwd": ([ctypes.POINTER(kdn_rope_desc_t)] + [_P] * 8, ctypes.c_int),
    "kdn_rope_bwd": ([ctypes.POINTER(kdn_rope_desc_t)] + [_P] * 8, ctypes.c_int),
    "kdn_ffn_fwd_workspace_bytes": ([ctypes.POINTER(kdn_ffn_desc_t)], ctypes.c_size_t),
    "kdn_ffn_bwd_workspace_bytes": ([ctypes.POINTER(kdn_ffn_desc_t)], ctypes.c_size_t),
    "kdn_ffn_fwd": ([ctypes.POINTER(kdn_ffn_desc_t)] + [_P] * 9 + [ctypes.c_size_t, _P], ctypes.c_int),
    "kdn_ffn_bwd": ([ctypes.POINTER(kdn_ffn_desc_t)] + [_P] * 13 + [ctypes.c_size_t, _P], ctypes.c_int),
}
EXPORTED = tuple(_SIG)


def lib():
    """The loaded ``libkdn.so`` (ctypes), built beforehand by ``build.build()``."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(f"{LIB_PATH} is missing: run paper_2609_07816_gb300.build."
                                   "build() first (there is no fallback implementation)")
            L = ctypes.CDLL(LIB_PATH)
            for name, (args, res) in _SIG.items():
                fn = getattr(L, name)
                fn.argtypes = args
                fn.restype = res
            _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().kdn_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != KDN_OK:
        raise KdnError(status, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    # the current stream's handle without building a Stream object (3 us of a small call)
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _on(fn, args):
    """fn(**args) with args["stream"] as the current stream.  What the call makes (workspace,
    outputs) then comes from that stream's memory, which is handed out again in the stream's own
    order and so never while the call's kernels still use it.  The outputs that it makes are
    recorded on the caller's stream too, so that they may be read and dropped there."""
    stream = args.pop("stream")
    if not isinstance(stream, torch.cuda.Stream):
        handle = stream.cuda_stream
        stream = torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()
    home = torch.cuda.current_stream(stream.device)
    with torch.cuda.stream(stream):
        out = fn(**args)
    given = {id(t) for t in args.values()}  # the caller's own buffers
    if id(out) not in given:
        for t in out.values() if isinstance(out, dict) else out if isinstance(out, tuple) else (out,):
            if t is not None and id(t) not in given:
                t.record_stream(home)
    return out


def _code(dtype):
    return _DTYPES[dtype] if isinstance(dtype, torch.dtype) else int(dtype)


_TORCH = {KDN_F32: torch.float32, KDN_BF16: torch.bfloat16}


def _torch_dtype(dtype):
    return dtype if isinstance(dtype, torch.dtype) else _TORCH[int(dtype)]


def _arg(t, name, dtype=None, numel=None, required=True, dev=None, strided=False):
    """A tensor handed to the C ABI as a raw pointer: it must be device memory (a
    CUDA tensor; on device ``dev`` where the call has one), dense in the ABI's row-major
    layout (contiguous; ``strided``: the caller looks at the strides), of the dtype the
    library reads or writes there and of the element count the descriptor implies.  Anything
    else would make the kernels read or write the wrong memory, so it is refused here, before
    any launch."""
    if t is None:
        if required:
            raise ValueError(f"{name} is required")
        return
    if (isinstance(t, torch.Tensor) and (t.is_cuda if dev is None else t.get_device() == dev)
            and (strided or t.is_contiguous()) and (dtype is None or t.dtype == dtype)
            and (numel is None or t.numel() == numel)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a CUDA tensor (the kernels read device memory), "
                         f"got one on {t.device}")
    if dev is not None and t.get_device() != dev:
        raise ValueError(f"{name}: on {t.device}, the call's other tensors are on cuda:{dev}")
    if not strided and not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous (the C ABI's row-major layout)")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name}: {t.numel()} elements, expected {numel}")


def _device(t, name, strided=False):
    """The device that a call's tensors share: that of its first one, and the current one, since
    that is where the kernels are launched."""
    _arg(t, name, strided=strided)
    dev = t.get_device()
    if torch.cuda.is_initialized() and torch._C._cuda_getDevice() != dev:
        raise ValueError(f"{name}: on {t.device}, the current device is cuda:{torch._C._cuda_getDevice()} "
                         f"(make the call under torch.cuda.device({dev}))")
    return dev


def _check_inputs(variant, q, k, v, g, omega, r, dO=None, tokens=True):
    """The per-token inputs (and dO): one device, which is returned, one activation dtype, the
    ABI's layouts.  ``tokens`` = False for the decode step, whose inputs drop the T axis."""
    dev = _device(q, "q")
    if q.dtype not in _DTYPES:
        raise TypeError(f"q: dtype {q.dtype}, expected torch.float32 or torch.bfloat16")
    if q.dim() != (4 if tokens else 3):
        raise ValueError(f"q: {q.dim()} dimensions, expected {4 if tokens else 3}")
    dk = q.shape[-1]
    n = q.numel() // dk if dk else 0
    _arg(v, "v", q.dtype)
    _arg(g, "g", q.dtype)
    dv = v.shape[-1]
    per_channel = variant == 0 or g.dim() == q.dim()
    for t, name, m in ((k, "k", dk), (v, "v", dv), (g, "g", dk if per_channel else 1),
                       (omega, "omega", dk if variant == 0 else 1), (r, "r", 1)):
        _arg(t, name, q.dtype, n * m, dev=dev)
    if dO is not None:
        _arg(dO, "dO", q.dtype, n * dv, dev=dev)
    return dev


def _state_sizes(variant, q, v, tokens=True):
    B, H = q.shape[0], q.shape[2 if tokens else 1]
    dk, dv = q.shape[-1], v.shape[-1]
    return B * H * dk * dv, B * H * (dk if variant == 0 else 1)


def _check_grads(G, q, k, v, g, omega, r, out_dtype, ns, np_, dev):
    """Gradient buffers: one per input, its element count, the output dtype;
    dS0, dp0 and dmu (optional) in float32."""
    od = _torch_dtype(out_dtype)
    for n, x in (("dq", q), ("dk", k), ("dv", v), ("dg", g), ("domega", omega), ("dr", r)):
        _arg(G.get(n), n, od, x.numel(), dev=dev)
    _arg(G.get("dS0"), "dS0", torch.float32, ns, required=False, dev=dev)
    _arg(G.get("dp0"), "dp0", torch.float32, np_, required=False, dev=dev)
    _arg(G.get("dmu"), "dmu", torch.float32, q.shape[0] * q.shape[2], required=False, dev=dev)


def make_desc(B, T, H, dk, dv, dtype, *, chunk=0, mu=None, scale=None,
              decay_per_channel=1, out_dtype=KDN_F32, gates=KDN_GATES_POST,
              r_min=R_MIN_DEFAULT) -> kdn_desc_t:
    """``gates``: KDN_GATES_POST (g = log alpha, omega, r) or KDN_GATES_LOGITS
    (g, omega, r are the logits of sigmoid / softplus / r_min + softplus)."""
    return kdn_desc_t(B, T, H, dk, dv, chunk, _code(dtype), 0.0 if mu is None else float(mu),
                      math.nan if scale is None else float(scale), int(decay_per_channel),
                      _code(out_dtype), int(gates), float(r_min))


def _desc_from(variant, q, v, g, *, chunk, mu, scale, out_dtype, gates=KDN_GATES_POST,
               r_min=R_MIN_DEFAULT):
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    pcd = 1 if variant == 0 else int(g.dim() == 4)
    return make_desc(B, T, H, dk, dv, q.dtype, chunk=chunk, mu=mu, scale=scale,
                     decay_per_channel=pcd, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def workspace_bytes(desc: kdn_desc_t, variant: int, backward: bool = False) -> int:
    fn = lib().kdn_bwd_workspace_bytes if backward else lib().kdn_fwd_workspace_bytes
    return int(fn(ctypes.byref(desc), int(variant)))


def alloc_workspace(desc, variant, backward=False, device=None):
    n = workspace_bytes(desc, variant, backward)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device or "cuda")


def _fwd(name, variant, q, k, v, g, omega, r, S0, p0, *, chunk, mu, scale, o, ST, pT,
         want_state, workspace, out_dtype,
         gates=KDN_GATES_POST, r_min=R_MIN_DEFAULT, stream=None):
    if stream is not None:
        return _on(_fwd, locals())
    on = _check_inputs(variant, q, k, v, g, omega, r)
    desc = _desc_from(variant, q, v, g, chunk=chunk, mu=mu, scale=scale, out_dtype=out_dtype,
                      gates=gates, r_min=r_min)
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    ns, np_ = _state_sizes(variant, q, v)
    _arg(S0, "S0", torch.float32, ns, required=False, dev=on)
    _arg(p0, "p0", torch.float32, np_, required=False, dev=on)
    if o is None:
        o = torch.empty(B, T, H, dv, dtype=out_dtype, device=dev)
    if want_state and ST is None:
        ST = torch.empty(B, H, dk, dv, dtype=torch.float32, device=dev)
    if want_state and pT is None:
        pT = torch.empty((B, H, dk) if variant == 0 else (B, H), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = alloc_workspace(desc, variant, False, dev)
    _arg(o, "o", _torch_dtype(out_dtype), B * T * H * dv, dev=on)
    _arg(ST, "ST", torch.float32, ns, required=False, dev=on)
    _arg(pT, "pT", torch.float32, np_, required=False, dev=on)
    _arg(workspace, "workspace", torch.uint8, dev=on)
    st = getattr(lib(), name)(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                              _ptr(omega), _ptr(r), _ptr(S0), _ptr(p0), _ptr(o), _ptr(ST),
                              _ptr(pT), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, name)
    return o, ST, pT


def kdn_diag_fwd(q, k, v, g, omega, r, S0=None, p0=None, *, chunk=0, mu=None, scale=None,
                 o=None, ST=None, pT=None, want_state=True, workspace=None, stream=None,
                 out_dtype=torch.float32, gates=KDN_GATES_POST,
                 r_min=R_MIN_DEFAULT):
    """Diagonal KDN forward (Prop. 3).  Returns (o, ST, pT)."""
    return _fwd("kdn_diag_fwd", 0, q, k, v, g, omega, r, S0, p0, chunk=chunk, mu=mu,
                scale=scale, o=o, ST=ST, pT=pT, want_state=want_state, workspace=workspace,
                stream=stream, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def kdn_iso_fwd(q, k, v, g, omega, r, S0=None, p0=None, *, chunk=0, mu=None, scale=None,
                o=None, ST=None, pT=None, want_state=True, workspace=None, stream=None,
                 out_dtype=torch.float32, gates=KDN_GATES_POST,
                 r_min=R_MIN_DEFAULT):
    """Isotropic KDN forward (Prop. 5).  g [B,T,H,dk] = per-channel decay, [B,T,H] = scalar."""
    return _fwd("kdn_iso_fwd", 1, q, k, v, g, omega, r, S0, p0, chunk=chunk, mu=mu,
                scale=scale, o=o, ST=ST, pT=pT, want_state=want_state, workspace=workspace,
                stream=stream, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def _bwd(name, variant, q, k, v, g, omega, r, S0, p0, dO, dST, dpT, *, chunk, mu, scale,
         grads, want_state_grads, workspace, out_dtype,
         gates=KDN_GATES_POST, r_min=R_MIN_DEFAULT, stream=None):
    if stream is not None:
        return _on(_bwd, locals())
    on = _check_inputs(variant, q, k, v, g, omega, r, dO)
    desc = _desc_from(variant, q, v, g, chunk=chunk, mu=mu, scale=scale, out_dtype=out_dtype,
                      gates=gates, r_min=r_min)
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    ns, np_ = _state_sizes(variant, q, v)
    for t, n, m in ((S0, "S0", ns), (p0, "p0", np_), (dST, "dST", ns), (dpT, "dpT", np_)):
        _arg(t, n, torch.float32, m, required=False, dev=on)
    if grads is None:
        grads = {n: torch.empty(x.shape, dtype=out_dtype, device=dev) for n, x in
                 (("dq", q), ("dk", k), ("dv", v), ("dg", g), ("domega", omega), ("dr", r))}
        if want_state_grads:
            grads["dS0"] = torch.empty(B, H, dk, dv, dtype=torch.float32, device=dev)
            grads["dp0"] = torch.empty((B, H, dk) if variant == 0 else (B, H),
                                       dtype=torch.float32, device=dev)
            grads["dmu"] = torch.empty(B, H, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = alloc_workspace(desc, variant, True, dev)
    G = grads
    _check_grads(G, q, k, v, g, omega, r, out_dtype, ns, np_, on)
    _arg(workspace, "workspace", torch.uint8, dev=on)
    st = getattr(lib(), name)(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                              _ptr(omega), _ptr(r), _ptr(S0), _ptr(p0), _ptr(dO), _ptr(dST),
                              _ptr(dpT), _ptr(G["dq"]), _ptr(G["dk"]), _ptr(G["dv"]),
                              _ptr(G["dg"]), _ptr(G["domega"]), _ptr(G["dr"]),
                              _ptr(G.get("dS0")), _ptr(G.get("dp0")), _ptr(G.get("dmu")),
                              _ptr(workspace),
                              workspace.numel(), _stream(stream))
    _check(st, name)
    return grads


def kdn_diag_bwd(q, k, v, g, omega, r, S0, p0, dO, dST=None, dpT=None, *, chunk=0, mu=None,
                 scale=None, grads=None, want_state_grads=True, workspace=None, stream=None,
                 out_dtype=torch.float32, gates=KDN_GATES_POST,
                 r_min=R_MIN_DEFAULT):
    """Gradients of the Diagonal KDN forward.  Returns a dict dq, dk, dv, dg, domega, dr,
    and with want_state_grads dS0, dp0 and dmu [B,H] (the gradient with respect to mu)."""
    return _bwd("kdn_diag_bwd", 0, q, k, v, g, omega, r, S0, p0, dO, dST, dpT, chunk=chunk,
                mu=mu, scale=scale, grads=grads, want_state_grads=want_state_grads,
                workspace=workspace, stream=stream, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def kdn_iso_bwd(q, k, v, g, omega, r, S0, p0, dO, dST=None, dpT=None, *, chunk=0, mu=None,
                scale=None, grads=None, want_state_grads=True, workspace=None, stream=None,
                 out_dtype=torch.float32, gates=KDN_GATES_POST,
                 r_min=R_MIN_DEFAULT):
    """Gradients of the Isotropic KDN forward."""
    return _bwd("kdn_iso_bwd", 1, q, k, v, g, omega, r, S0, p0, dO, dST, dpT, chunk=chunk,
                mu=mu, scale=scale, grads=grads, want_state_grads=want_state_grads,
                workspace=workspace, stream=stream, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def saved_bytes(desc: kdn_desc_t, variant: int = 0) -> int:
    """Bytes of the saved backward context (0: the descriptor has no saved-context path)."""
    return int(lib().kdn_saved_bytes(ctypes.byref(desc), int(variant)))


def _fwd_save(name, variant, q, k, v, g, omega, r, S0, p0, *, mu, scale, o, ST, pT, saved,
              want_state, workspace, out_dtype,
              gates=KDN_GATES_POST, r_min=R_MIN_DEFAULT, stream=None):
    if stream is not None:
        return _on(_fwd_save, locals())
    on = _check_inputs(variant, q, k, v, g, omega, r)
    desc = _desc_from(variant, q, v, g, chunk=0, mu=mu, scale=scale, out_dtype=out_dtype,
                      gates=gates, r_min=r_min)
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    ns, np_ = _state_sizes(variant, q, v)
    _arg(S0, "S0", torch.float32, ns, required=False, dev=on)
    _arg(p0, "p0", torch.float32, np_, required=False, dev=on)
    if o is None:
        o = torch.empty(B, T, H, dv, dtype=out_dtype, device=dev)
    if want_state and ST is None:
        ST = torch.empty(B, H, dk, dv, dtype=torch.float32, device=dev)
    if want_state and pT is None:
        pT = torch.empty((B, H, dk) if variant == 0 else (B, H), dtype=torch.float32, device=dev)
    if saved is None:
        saved = torch.empty(max(saved_bytes(desc, variant), 256), dtype=torch.uint8, device=dev)
    if workspace is None:
        workspace = alloc_workspace(desc, variant, False, dev)
    _arg(o, "o", _torch_dtype(out_dtype), B * T * H * dv, dev=on)
    _arg(ST, "ST", torch.float32, ns, required=False, dev=on)
    _arg(pT, "pT", torch.float32, np_, required=False, dev=on)
    _arg(saved, "saved", torch.uint8, dev=on)
    _arg(workspace, "workspace", torch.uint8, dev=on)
    st = getattr(lib(), name)(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                              _ptr(omega), _ptr(r), _ptr(S0), _ptr(p0), _ptr(o), _ptr(ST),
                              _ptr(pT), _ptr(saved), saved.numel(), _ptr(workspace),
                              workspace.numel(), _stream(stream))
    _check(st, name)
    return o, ST, pT, saved


def kdn_diag_fwd_save(q, k, v, g, omega, r, S0=None, p0=None, *, mu=None, scale=None, o=None,
                      ST=None, pT=None, saved=None, want_state=True, workspace=None, stream=None,
                      out_dtype=torch.float32, gates=KDN_GATES_POST,
                 r_min=R_MIN_DEFAULT):
    """Diagonal KDN forward that also keeps the chunked backward's context.
    Returns (o, ST, pT, saved); pass `saved` to kdn_diag_bwd_saved."""
    return _fwd_save("kdn_diag_fwd_save", 0, q, k, v, g, omega, r, S0, p0, mu=mu, scale=scale,
                     o=o, ST=ST, pT=pT, saved=saved, want_state=want_state, workspace=workspace,
                     stream=stream, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def kdn_iso_fwd_save(q, k, v, g, omega, r, S0=None, p0=None, *, mu=None, scale=None, o=None,
                     ST=None, pT=None, saved=None, want_state=True, workspace=None, stream=None,
                     out_dtype=torch.float32, gates=KDN_GATES_POST,
                 r_min=R_MIN_DEFAULT):
    """Isotropic KDN forward that also keeps the chunked backward's context."""
    return _fwd_save("kdn_iso_fwd_save", 1, q, k, v, g, omega, r, S0, p0, mu=mu, scale=scale,
                     o=o, ST=ST, pT=pT, saved=saved, want_state=want_state, workspace=workspace,
                     stream=stream, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def _bwd_saved(name, variant, q, k, v, g, omega, r, saved, dO, dST, dpT, *, mu, scale, grads,
               want_state_grads, workspace, out_dtype,
               gates=KDN_GATES_POST, r_min=R_MIN_DEFAULT, stream=None):
    if stream is not None:
        return _on(_bwd_saved, locals())
    on = _check_inputs(variant, q, k, v, g, omega, r, dO)
    desc = _desc_from(variant, q, v, g, chunk=0, mu=mu, scale=scale, out_dtype=out_dtype,
                      gates=gates, r_min=r_min)
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    ns, np_ = _state_sizes(variant, q, v)
    _arg(saved, "saved", torch.uint8, dev=on)
    _arg(dST, "dST", torch.float32, ns, required=False, dev=on)
    _arg(dpT, "dpT", torch.float32, np_, required=False, dev=on)
    if grads is None:
        grads = {n: torch.empty(x.shape, dtype=out_dtype, device=dev) for n, x in
                 (("dq", q), ("dk", k), ("dv", v), ("dg", g), ("domega", omega), ("dr", r))}
        if want_state_grads:
            grads["dS0"] = torch.empty(B, H, dk, dv, dtype=torch.float32, device=dev)
            grads["dp0"] = torch.empty((B, H, dk) if variant == 0 else (B, H),
                                       dtype=torch.float32, device=dev)
            grads["dmu"] = torch.empty(B, H, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = alloc_workspace(desc, variant, False, dev)
    G = grads
    _check_grads(G, q, k, v, g, omega, r, out_dtype, ns, np_, on)
    _arg(workspace, "workspace", torch.uint8, dev=on)
    st = getattr(lib(), name)(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                              _ptr(omega), _ptr(r), _ptr(saved), saved.numel(), _ptr(dO),
                              _ptr(dST), _ptr(dpT), _ptr(G["dq"]), _ptr(G["dk"]),
                              _ptr(G["dv"]), _ptr(G["dg"]), _ptr(G["domega"]), _ptr(G["dr"]),
                              _ptr(G.get("dS0")), _ptr(G.get("dp0")), _ptr(G.get("dmu")),
                              _ptr(workspace),
                              workspace.numel(), _stream(stream))
    _check(st, name)
    return grads


def kdn_diag_bwd_saved(q, k, v, g, omega, r, saved, dO, dST=None, dpT=None, *, mu=None,
                       scale=None, grads=None, want_state_grads=True, workspace=None, stream=None,
                       out_dtype=torch.float32, gates=KDN_GATES_POST,
                 r_min=R_MIN_DEFAULT):
    """Gradients of the Diagonal KDN forward from the context kept by kdn_diag_fwd_save."""
    return _bwd_saved("kdn_diag_bwd_saved", 0, q, k, v, g, omega, r, saved, dO, dST, dpT, mu=mu,
                      scale=scale, grads=grads, want_state_grads=want_state_grads,
                      workspace=workspace, stream=stream, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def kdn_iso_bwd_saved(q, k, v, g, omega, r, saved, dO, dST=None, dpT=None, *, mu=None,
                      scale=None, grads=None, want_state_grads=True, workspace=None, stream=None,
                      out_dtype=torch.float32, gates=KDN_GATES_POST,
                 r_min=R_MIN_DEFAULT):
    """Gradients of the Isotropic KDN forward from the context kept by kdn_iso_fwd_save."""
    return _bwd_saved("kdn_iso_bwd_saved", 1, q, k, v, g, omega, r, saved, dO, dST, dpT, mu=mu,
                      scale=scale, grads=grads, want_state_grads=want_state_grads,
                      workspace=workspace, stream=stream, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def _beta_eff(name, variant, k, v, g, r, saved, *, out, stream=None, gates, r_min):
    if stream is not None:
        return _on(_beta_eff, locals())
    desc = _desc_from(variant, k, v, g, chunk=0, mu=None, scale=None, out_dtype=torch.float32,
                      gates=gates, r_min=r_min)
    B, T, H, _ = k.shape
    on = _device(k, "k")
    _arg(saved, "saved", torch.uint8, dev=on)
    _arg(r, "r", k.dtype, B * T * H, dev=on)
    if out is None:
        out = torch.empty(B, T, H, dtype=torch.float32, device=k.device)
    _arg(out, "out", torch.float32, B * T * H, dev=on)
    st = getattr(lib(), name)(ctypes.byref(desc), _ptr(saved), ctypes.c_size_t(saved.numel()),
                              _ptr(r), _ptr(out), _stream(stream))
    _check(st, name)
    return out


def kdn_diag_beta_eff(k, v, g, r, saved, *, out=None, stream=None, gates=KDN_GATES_POST,
                      r_min=R_MIN_DEFAULT):
    """beta_eff = k_t^T kappa_t [B,T,H] (float32) from the context kdn_diag_fwd_save kept;
    k, v, g fix the descriptor, r is the forward's r."""
    return _beta_eff("kdn_diag_beta_eff", 0, k, v, g, r, saved, out=out, stream=stream,
                     gates=gates, r_min=r_min)


def kdn_iso_beta_eff(k, v, g, r, saved, *, out=None, stream=None, gates=KDN_GATES_POST,
                     r_min=R_MIN_DEFAULT):
    """beta_eff = beta_t |k_t|^2 [B,T,H] (float32) from the context kdn_iso_fwd_save kept."""
    return _beta_eff("kdn_iso_beta_eff", 1, k, v, g, r, saved, out=out, stream=stream,
                     gates=gates, r_min=r_min)


def _decode(name, variant, q, k, v, g, omega, r, S, p, *, mu, scale, o, out_dtype,
            gates=KDN_GATES_POST, r_min=R_MIN_DEFAULT, stream=None):
    if stream is not None:
        return _on(_decode, locals())
    on = _check_inputs(variant, q, k, v, g, omega, r, tokens=False)
    B, H, dk = q.shape
    dv = v.shape[-1]
    pcd = 1 if variant == 0 else int(g.dim() == 3)
    desc = make_desc(B, 1, H, dk, dv, q.dtype, mu=mu, scale=scale, decay_per_channel=pcd,
                     out_dtype=out_dtype,
        gates=gates, r_min=r_min)
    ns, np_ = _state_sizes(variant, q, v, tokens=False)
    _arg(S, "S", torch.float32, ns, dev=on)
    _arg(p, "p", torch.float32, np_, dev=on)
    if o is None:
        o = torch.empty(B, H, dv, dtype=out_dtype, device=q.device)
    _arg(o, "o", _torch_dtype(out_dtype), B * H * dv, dev=on)
    st = getattr(lib(), name)(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                              _ptr(omega), _ptr(r), _ptr(S), _ptr(p), _ptr(o), _stream(stream))
    _check(st, name)
    return o


def kdn_diag_decode_step(q, k, v, g, omega, r, S, p, *, mu=None, scale=None, o=None,
                         stream=None, out_dtype=torch.float32, gates=KDN_GATES_POST,
                 r_min=R_MIN_DEFAULT):
    """One Diagonal KDN token for every head, S [B,H,dk,dv] and p [B,H,dk] updated in place."""
    return _decode("kdn_diag_decode_step", 0, q, k, v, g, omega, r, S, p, mu=mu, scale=scale,
                   o=o, stream=stream, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def kdn_iso_decode_step(q, k, v, g, omega, r, S, p, *, mu=None, scale=None, o=None,
                        stream=None, out_dtype=torch.float32, gates=KDN_GATES_POST,
                 r_min=R_MIN_DEFAULT):
    """One Isotropic KDN token for every head; g [B,H,dk] or [B,H]; p [B,H] in place."""
    return _decode("kdn_iso_decode_step", 1, q, k, v, g, omega, r, S, p, mu=mu, scale=scale,
                   o=o, stream=stream, out_dtype=out_dtype,
        gates=gates, r_min=r_min)


def kdn_diag_fwd_noalloc(q, k, v, g, omega, r, S0=None, p0=None, *, o, ST=None, pT=None,
                         mu=None, scale=None, stream=None, gates=KDN_GATES_POST,
                         r_min=R_MIN_DEFAULT):
    """Diagonal KDN forward into caller-provided outputs, using the library's own
    fixed scratch array instead of a workspace, for callers that may not
    allocate device memory.  Problems needing more than
    KDN_NOALLOC_SCRATCH_BYTES of scratch are rejected.  Returns o."""
    if stream is not None:
        return _on(kdn_diag_fwd_noalloc, locals())
    on = _check_inputs(0, q, k, v, g, omega, r)
    _arg(o, "o")
    desc = _desc_from(0, q, v, g, chunk=0, mu=mu, scale=scale, out_dtype=o.dtype, gates=gates,
                      r_min=r_min)
    B, T, H, dk = q.shape
    ns, np_ = _state_sizes(0, q, v)
    _arg(o, "o", None, B * T * H * v.shape[-1], dev=on)
    for t, n, m in ((S0, "S0", ns), (p0, "p0", np_), (ST, "ST", ns), (pT, "pT", np_)):
        _arg(t, n, torch.float32, m, required=False, dev=on)
    st = lib().kdn_diag_fwd_noalloc(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                                    _ptr(omega), _ptr(r), _ptr(S0), _ptr(p0), _ptr(o), _ptr(ST),
                                    _ptr(pT), _stream(stream))
    _check(st, "kdn_diag_fwd_noalloc")
    return o


def kdn_kernel_launches(desc: kdn_desc_t, variant: int, op: int) -> int:
    """Kernels one call launches (op 0 fwd, 1 bwd, 2 decode step)."""
    return int(lib().kdn_kernel_launches(ctypes.byref(desc), int(variant), int(op)))


def kdn_selftest_wait_timeout(workspace, stream=None) -> int:
    """Runs the device self-test of the bounded waits on ``workspace`` (asynchronous);
    kdn_get_device_status then reports KDN_ERR_TIMEOUT."""
    _arg(workspace, "workspace")
    return int(lib().kdn_selftest_wait_timeout(_ptr(workspace), _stream(stream)))


def kdn_get_device_status(workspace, stream=None) -> int:
    """Reads and clears the status word of the last call on ``workspace`` (KDN_OK, KDN_ERR_TIMEOUT
    or KDN_ERR_RANGE), once the stream has passed it."""
    _arg(workspace, "workspace")
    return int(lib().kdn_get_device_status(_ptr(workspace), _stream(stream)))


def kdn_noalloc_device_status(stream=None) -> int:
    """Reads and clears the status word of the last kdn_diag_fwd_noalloc call."""
    return int(lib().kdn_noalloc_device_status(_stream(stream)))


# ------------------------------------------------------------ the hybrid layer's operators
#
# Sliding-window attention with sinks: q, o, dO [B,T,H,d]; k, v [B,T,Hk,d], H a multiple of
# Hk; lse [B,H,T] float32; lens [B] int32 (None: every sequence has T tokens); the decode
# cache kc, vc [B,Hk,sinks+window,d], pos [B] int32.  Query i sees keys j <= i with
# j > i - window or j < sinks.  Residual RMS norm: x, res, h [..., D], w [D].  Rotary positions:
# q [B,T,H,d], k [B,T,Hk,d], or [B,H,d] and [B,Hk,d] for one token of every sequence; the rows of
# tokens may lie apart (a slice of a fused projection's heads); pos [B] or [B,T] int32.
# Feed-forward block: x [..., D], wg, wu [F,D], wd [D,F], g, u, h [..., F].


def make_swa_desc(B, T, H, Hk, d, dtype, *, window, sinks=0, scale=None) -> kdn_swa_desc_t:
    return kdn_swa_desc_t(B, T, H, Hk, d, int(window), int(sinks), _code(dtype),
                          math.nan if scale is None else float(scale))


def _check_swa(q, k, v, tokens=True):
    """q, k, v of one dtype and device, which is returned: [B,T,H,d] and twice [B,T,Hk,d], without
    T for the decode step."""
    dev = _device(q, "q")
    dtype, dims = q.dtype, 4 if tokens else 3
    if dtype not in _DTYPES:
        raise TypeError(f"q: dtype {dtype}, expected torch.float32 or torch.bfloat16")
    _arg(k, "k", dtype, dev=dev)
    _arg(v, "v", dtype, dev=dev)
    qs, ks, vs = q.shape, k.shape, v.shape
    for shape, name in ((qs, "q"), (ks, "k"), (vs, "v")):
        if len(shape) != dims:
            raise ValueError(f"{name}: {len(shape)} dimensions, expected {dims}")
    if ks[:-2] != qs[:-2] or ks[-1] != qs[-1]:
        raise ValueError(f"k: shape {tuple(ks)} does not go with q's {tuple(qs)}")
    if vs != ks:
        raise ValueError(f"v: shape {tuple(vs)}, expected {tuple(ks)}")
    return dev


def _check_cache(kc, vc, k, window, sinks, dev):
    shape = (k.shape[0], k.shape[-2], int(window) + int(sinks), k.shape[-1])
    for t, name in ((kc, "kc"), (vc, "vc")):
        _arg(t, name, k.dtype, dev=dev)
        if t.shape != shape:
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")


def _swa_workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def kdn_swa_fwd(q, k, v, *, window, sinks=0, lens=None, scale=None, o=None, lse=None, want_lse=True,
                workspace=None, stream=None):
    """Sliding-window attention with sinks over whole sequences.  Returns (o, lse); lse is
    None with want_lse=False (kdn_swa_bwd needs it).  Rows at and past lens[b] give o = 0.  The
    status of a device-side wait is in ``workspace`` only (kdn_get_device_status)."""
    if stream is not None:
        return _on(kdn_swa_fwd, locals())
    on = _check_swa(q, k, v)
    B, T, H, d = q.shape
    _arg(lens, "lens", torch.int32, B, required=False, dev=on)
    desc = make_swa_desc(B, T, H, k.shape[2], d, q.dtype, window=window, sinks=sinks, scale=scale)
    if o is None:
        o = torch.empty_like(q)
    else:
        _arg(o, "o", q.dtype, q.numel(), dev=on)
    if lse is not None:
        _arg(lse, "lse", torch.float32, B * H * T, dev=on)
    elif want_lse:
        lse = torch.empty(B, H, T, dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = _swa_workspace(256, q.device)
    else:
        _arg(workspace, "workspace", torch.uint8, dev=on)
    st = lib().kdn_swa_fwd(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(lens), _ptr(o),
                           _ptr(lse), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "kdn_swa_fwd")
    return o, lse


def kdn_swa_bwd(q, k, v, o, lse, dO, *, window, sinks=0, lens=None, scale=None, grads=None,
                workspace=None, stream=None):
    """Gradients of kdn_swa_fwd from its o and lse.  Returns a dict dq, dk, dv (dk and dv
    summed over the query heads that share a kv head).  The status of a device-side wait is in
    ``workspace`` only (kdn_get_device_status)."""
    if stream is not None:
        return _on(kdn_swa_bwd, locals())
    on = _check_swa(q, k, v)
    B, T, H, d = q.shape
    _arg(lens, "lens", torch.int32, B, required=False, dev=on)
    _arg(o, "o", q.dtype, q.numel(), dev=on)
    _arg(lse, "lse", torch.float32, B * H * T, dev=on)
    _arg(dO, "dO", q.dtype, q.numel(), dev=on)
    desc = make_swa_desc(B, T, H, k.shape[2], d, q.dtype, window=window, sinks=sinks, scale=scale)
    if grads is None:
        grads = {"dq": torch.empty_like(q), "dk": torch.empty_like(k), "dv": torch.empty_like(v)}
    else:
        for n, x in (("dq", q), ("dk", k), ("dv", v)):
            _arg(grads.get(n), n, q.dtype, x.numel(), dev=on)
    if workspace is None:
        workspace = _swa_workspace(lib().kdn_swa_bwd_workspace_bytes(ctypes.byref(desc)), q.device)
    else:
        _arg(workspace, "workspace", torch.uint8, dev=on)
    st = lib().kdn_swa_bwd(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(lens), _ptr(o),
                           _ptr(lse), _ptr(dO), _ptr(grads["dq"]), _ptr(grads["dk"]),
                           _ptr(grads["dv"]), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "kdn_swa_bwd")
    return grads


def kdn_swa_cache_fill(k, v, kc, vc, *, window, sinks=0, lens=None, stream=None):
    """Copies the tokens of a prompt (k, v [B,T,Hk,d]) that later tokens still see into the
    decode cache; slots that no token of it belongs to keep what they hold."""
    if stream is not None:
        return _on(kdn_swa_cache_fill, locals())
    on = _check_swa(k, k, v)
    B, T, Hk, d = k.shape
    _arg(lens, "lens", torch.int32, B, required=False, dev=on)
    _check_cache(kc, vc, k, window, sinks, on)
    desc = make_swa_desc(B, T, Hk, Hk, d, k.dtype, window=window, sinks=sinks)
    st = lib().kdn_swa_cache_fill(ctypes.byref(desc), _ptr(k), _ptr(v), _ptr(lens), _ptr(kc),
                                  _ptr(vc), _stream(stream))
    _check(st, "kdn_swa_cache_fill")


def kdn_swa_decode_step(q, k, v, kc, vc, pos, *, window, sinks=0, scale=None, o=None, stream=None):
    """One token of every sequence (q [B,H,d], k, v [B,Hk,d] at position pos[b]): writes its k
    and v into the cache in place and returns its attention o [B,H,d].  pos[b] < 0: idle."""
    if stream is not None:
        return _on(kdn_swa_decode_step, locals())
    on = _check_swa(q, k, v, tokens=False)
    B, H, d = q.shape
    _arg(pos, "pos", torch.int32, B, dev=on)
    _check_cache(kc, vc, k, window, sinks, on)
    desc = make_swa_desc(B, 1, H, k.shape[1], d, q.dtype, window=window, sinks=sinks, scale=scale)
    if o is None:
        o = torch.empty_like(q)
    else:
        _arg(o, "o", q.dtype, q.numel(), dev=on)
    st = lib().kdn_swa_decode_step(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(kc), _ptr(vc),
                                   _ptr(pos), _ptr(o), _stream(stream))
    _check(st, "kdn_swa_decode_step")
    return o


def _norm_desc(x, out_dtype, block, eps):
    D = x.shape[-1]
    return kdn_norm_desc_t(x.numel() // D if D else 0, D, _code(x.dtype), out_dtype, int(block), float(eps))


def kdn_add_rmsnorm_fwd(x, w, res=None, *, eps=1e-6, out_dtype=None, block=0, y=None, h=None,
                        rstd=None, scales=None, want_rstd=True, stream=None):
    """h = x + res and its RMS norm y = h rstd w over the last axis.  Returns (y, h, rstd,
    scales): h is x itself without a residual; out_dtype=torch.float8_e4m3fn gives y in 8 bits
    with float32 scales per row (block=0, [..., 1]) or per 128 columns (block=128), y ~ q * scale."""
    if stream is not None:
        return _on(kdn_add_rmsnorm_fwd, locals())
    on = _device(x, "x")
    if x.dtype not in _DTYPES:
        raise TypeError(f"x: dtype {x.dtype}, expected torch.float32 or torch.bfloat16")
    if x.dim() < 1:
        raise ValueError("x: a scalar, expected [..., D]")
    out_dtype = x.dtype if out_dtype is None else out_dtype
    f8 = out_dtype == torch.float8_e4m3fn
    if not f8 and out_dtype != x.dtype:
        raise TypeError(f"out_dtype: {out_dtype}, expected {x.dtype} or torch.float8_e4m3fn")
    shape, n = x.shape, x.numel()
    D = shape[-1]
    _arg(w, "w", x.dtype, D, dev=on)
    _arg(res, "res", x.dtype, n, required=False, dev=on)
    desc = _norm_desc(x, KDN_F8E4M3 if f8 else _code(x.dtype), block, eps)
    nb = -(-D // block) if block else 1
    if y is None:
        y = torch.empty_like(x, dtype=out_dtype)
    else:
        _arg(y, "y", out_dtype, n, dev=on)
    if h is not None:
        _arg(h, "h", x.dtype, n, dev=on)
    elif res is not None:
        h = torch.empty_like(x)
    if rstd is not None:
        _arg(rstd, "rstd", torch.float32, desc.rows, dev=on)
    elif want_rstd:
        rstd = torch.empty(shape[:-1], dtype=torch.float32, device=x.device)
    if scales is not None:
        _arg(scales, "scales", torch.float32, desc.rows * nb, dev=on)
    elif f8:
        scales = torch.empty(tuple(shape[:-1]) + (nb,), dtype=torch.float32, device=x.device)
    st = lib().kdn_add_rmsnorm_fwd(ctypes.byref(desc), _ptr(x), _ptr(res), _ptr(w), _ptr(y), _ptr(h),
                                   _ptr(rstd), _ptr(scales), _stream(stream))
    _check(st, "kdn_add_rmsnorm_fwd")
    return y, x if h is None else h, rstd, scales


def kdn_add_rmsnorm_bwd(h, w, rstd, dy, dh=None, *, dx=None, dw=None, workspace=None, stream=None):
    """Gradients of kdn_add_rmsnorm_fwd from its h and rstd: dy is the gradient of y, dh that
    of h from the residual stream.  Returns (dx, dw): dx for x and res alike, dw [D] float32."""
    if stream is not None:
        return _on(kdn_add_rmsnorm_bwd, locals())
    on = _device(h, "h")
    if h.dtype not in _DTYPES:
        raise TypeError(f"h: dtype {h.dtype}, expected torch.float32 or torch.bfloat16")
    if h.dim() < 1:
        raise ValueError("h: a scalar, expected [..., D]")
    D = h.shape[-1]
    desc = _norm_desc(h, _code(h.dtype), 0, 0.0)
    _arg(w, "w", h.dtype, D, dev=on)
    _arg(rstd, "rstd", torch.float32, desc.rows, dev=on)
    _arg(dy, "dy", h.dtype, h.numel(), dev=on)
    _arg(dh, "dh", h.dtype, h.numel(), required=False, dev=on)
    if dx is None:
        dx = torch.empty_like(h)
    else:
        _arg(dx, "dx", h.dtype, h.numel(), dev=on)
    if dw is None:
        dw = torch.empty(D, dtype=torch.float32, device=h.device)
    else:
        _arg(dw, "dw", torch.float32, D, dev=on)
    if workspace is None:
        workspace = _swa_workspace(lib().kdn_add_rmsnorm_bwd_workspace_bytes(ctypes.byref(desc)), h.device)
    else:
        _arg(workspace, "workspace", torch.uint8, dev=on)
    st = lib().kdn_add_rmsnorm_bwd(ctypes.byref(desc), _ptr(h), _ptr(w), _ptr(rstd), _ptr(dy), _ptr(dh),
                                   _ptr(dx), _ptr(dw), _ptr(workspace), workspace.numel(),
                                   _stream(stream))
    _check(st, "kdn_add_rmsnorm_bwd")
    return dx, dw


class RopeFreqs:
    """What kdn_rope_freqs returns: the turned channels ``rot``, the frequencies ``turns`` (a
    ctypes array of rot/2, in 2^-64 turns a position) and ``mscale``."""
    __slots__ = ("rot", "turns", "mscale", "at")

    def __init__(self, rot, turns, mscale):
        self.rot, self.turns, self.mscale = int(rot), turns, float(mscale)
        if not isinstance(turns, ctypes.Array) or turns._type_ is not ctypes.c_ulonglong:
            raise TypeError("turns: expected a ctypes array of c_ulonglong")
        self.at = ctypes.addressof(turns)
        if len(turns) != self.rot // 2:
            raise ValueError(f"turns: {len(turns)} entries, expected {self.rot // 2}")


def kdn_rope_freqs(rot, *, base=10000.0, factor=1.0, trained=0, beta_fast=32.0, beta_slow=1.0):
    """The frequencies of ``rot`` turned channels, made once: base^(-2i/rot), and with factor > 1
    scaled for contexts that many times the ``trained`` length (trained=0: positions divided by
    factor).  Host memory only; no CUDA call."""
    f = kdn_rope_freqs_t(int(rot), float(base), float(factor), float(trained), float(beta_fast), float(beta_slow))
    turns, mscale = (ctypes.c_ulonglong * max(int(rot) // 2, 1))(), ctypes.c_float()
    _check(lib().kdn_rope_freqs(ctypes.byref(f), turns, ctypes.byref(mscale)), "kdn_rope_freqs")
    return RopeFreqs(rot, turns, mscale.value)


def _rows(t, name, dtype, shape, dev):
    """Elements between the rows of tokens of t [..., heads, d], of this shape: dense heads, rows equally
    far apart.  0: a contiguous tensor."""
    _arg(t, name, dtype, dev=dev, strided=True)
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.is_contiguous():
        return 0
    heads, d = shape[-2:]
    ld, n = heads * d, 1
    strides = t.stride()
    dense = (d <= 1 or strides[-1] == 1) and (heads <= 1 or strides[-2] == d)
    for size, stride in zip(reversed(shape[:-2]), reversed(strides[:-2])):
        if size > 1:
            if n == 1:
                ld = stride
            dense = dense and stride == n * ld
        n *= size
    if not dense or ld < heads * d:
        raise ValueError(f"{name}: strides {strides}: heads must be dense and tokens' rows equally far apart")
    return ld


def _rope(back, q, k, freqs, qo, ko, pos, lens, interleaved, stream=None):
    if stream is not None:
        return _on(_rope, locals())
    names = ("dqo", "dko", "dq", "dk") if back else ("q", "k", "qo", "ko")
    on = _device(q, names[0], strided=True)
    dtype, shape = q.dtype, q.shape
    if dtype not in _DTYPES:
        raise TypeError(f"{names[0]}: dtype {dtype}, expected torch.float32 or torch.bfloat16")
    if len(shape) == 4:
        B, T, H, d = shape
    elif len(shape) == 3:
        (B, H, d), T = shape, 1
    else:
        raise ValueError(f"{names[0]}: {len(shape)} dimensions, expected 3 or 4")
    if type(freqs) is not RopeFreqs:
        raise TypeError(f"freqs: expected what kdn_rope_freqs returns, got {type(freqs).__name__}")
    ldq = 0 if q.is_contiguous() else _rows(q, names[0], dtype, shape, on)
    ldk = Hk = ldqo = ldko = per_token = 0
    pp = pl = pk = pko = None
    if k is not None:
        _arg(k, names[1], dtype, dev=on, strided=True)
        kshape = k.shape
        if len(kshape) != len(shape) or kshape[:-2] != shape[:-2] or kshape[-1] != d:
            raise ValueError(f"{names[1]}: shape {tuple(kshape)} does not go with {names[0]}'s {tuple(shape)}")
        Hk = kshape[-2]
        ldk = 0 if k.is_contiguous() else _rows(k, names[1], dtype, kshape, on)
        if ko is None:
            ko = torch.empty(kshape, dtype=dtype, device=k.device) if ldk else torch.empty_like(k)
        else:
            ldko = _rows(ko, names[3], dtype, kshape, on)
        pk, pko = _ptr(k), _ptr(ko)
    elif ko is not None:
        raise ValueError(f"{names[3]}: without {names[1]}")
    if pos is not None:
        per_token = int(isinstance(pos, torch.Tensor) and pos.dim() > 1)
        _arg(pos, "pos", torch.int32, B * T if per_token else B, dev=on)
        if per_token and pos.shape != (B, T):
            raise ValueError(f"pos: shape {tuple(pos.shape)}, expected {(B,)} or {(B, T)}")
        pp = _ptr(pos)
    if lens is not None:
        _arg(lens, "lens", torch.int32, B, dev=on)
        pl = _ptr(lens)
    if qo is None:
        qo = torch.empty(shape, dtype=dtype, device=q.device) if ldq else torch.empty_like(q)
    else:
        ldqo = _rows(qo, names[2], dtype, shape, on)
    desc = kdn_rope_desc_t(B, T, H, Hk, d, freqs.rot, 1 if interleaved else 0, per_token, _DTYPES[dtype], freqs.mscale,
                           *((ldqo, ldko, ldq, ldk) if back else (ldq, ldk, ldqo, ldko)))
    L = lib()
    st = (L.kdn_rope_bwd if back else L.kdn_rope_fwd)(ctypes.byref(desc), freqs.at, _ptr(q), pk, pp, pl, _ptr(qo), pko,
                                                      _stream(None))
    if st:
        _check(st, "kdn_rope_bwd" if back else "kdn_rope_fwd")
    return qo, ko


def kdn_rope_fwd(q, k, freqs, *, pos=None, lens=None, interleaved=False, qo=None, ko=None, stream=None):
    """Queries and keys (k may be None) turned by their positions: ``pos`` [B] those of the
    sequences' first tokens (None: 0), or [B,T] those of all tokens.  Of each head the first freqs.rot
    channels are turned in pairs (i, i + rot/2), or (2i, 2i + 1) when interleaved.  Returns (qo, ko),
    0 at and past lens[b].  qo may be q and ko may be k; otherwise outputs share no memory with inputs or
    one another."""
    return _rope(False, q, k, freqs, qo, ko, pos, lens, interleaved, stream)


def kdn_rope_bwd(dqo, dko, freqs, *, pos=None, lens=None, interleaved=False, dq=None, dk=None, stream=None):
    """Gradients of kdn_rope_fwd with respect to q and k from those of qo and ko (dko may be None).
    Returns (dq, dk); dq may be dqo and dk may be dko."""
    return _rope(True, dqo, dko, freqs, dq, dk, pos, lens, interleaved, stream)


def _check_ffn(x, wg, wu, wd):
    """x [..., D], wg, wu [F,D], wd [D,F] of one dtype and device; returns (device, dtype, rows, D, F)."""
    on = _device(x, "x")
    dtype, shape = x.dtype, x.shape
    if dtype not in _DTYPES:
        raise TypeError(f"x: dtype {dtype}, expected torch.float32 or torch.bfloat16")
    if not shape:
        raise ValueError("x: a scalar, expected [..., D]")
    D = shape[-1]
    for t, name in ((wg, "wg"), (wu, "wu"), (wd, "wd")):
        _arg(t, name, dtype, dev=on)
    F = wg.shape[0] if wg.dim() else 0
    if wg.shape != (F, D) or wu.shape != wg.shape or wd.shape != (D, F):
        for t, name, want in ((wg, "wg", (F, D)), (wu, "wu", (F, D)), (wd, "wd", (D, F))):
            if t.shape != want:
                raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {want}")
    return on, dtype, x.numel() // D if D else 0, D, F


_status_words = {}


def _status_word(dev):
    """256 bytes a device, kept: the workspace of calls that only have a status to leave, where nobody
    asked for it.  (Calls of any stream may write there at once; nothing reads it.)  Its memory may have
    been another tensor's, which kernels queued on this stream still use, and only this stream's own calls
    come behind them: the first call waits for them once, before any other stream may write there."""
    t = _status_words.get(dev)
    if t is None:
        t = torch.empty(256, dtype=torch.uint8, device=torch.device("cuda", dev))
        if not torch.cuda.is_current_stream_capturing():  # (a graph's memory goes with it)
            if torch.cuda.is_initialized():
                torch.cuda.current_stream(dev).synchronize()
            _status_words[dev] = t
    return t


def kdn_ffn_fwd(x, wg, wu, wd, *, act=KDN_ACT_SILU, g=None, u=None, h=None, y=None, want_saved=True, workspace=None,
                stream=None):
    """Gated feed-forward block: g = x wg^T, u = x wu^T, h = act(g) u, y = h wd^T over the last axis, act
    KDN_ACT_SILU or KDN_ACT_GELU (the tanh form).  Returns (y, g, u, h); with want_saved=False g and u are
    None (kdn_ffn_bwd needs them).  Outputs share no memory with inputs or one another.  The status of a
    device-side wait is in ``workspace`` only (kdn_get_device_status)."""
    if stream is not None:
        return _on(kdn_ffn_fwd, locals())
    on, dtype, rows, D, F = _check_ffn(x, wg, wu, wd)
    if h is None:
        h = torch.empty((*x.shape[:-1], F), dtype=dtype, device=x.device)
    else:
        _arg(h, "h", dtype, rows * F, dev=on)
    if g is not None or u is not None:
        _arg(g, "g", dtype, rows * F, dev=on)
        _arg(u, "u", dtype, rows * F, dev=on)
    elif want_saved:
        g, u = torch.empty_like(h), torch.empty_like(h)
    if y is None:
        y = torch.empty_like(x)
    else:
        _arg(y, "y", dtype, rows * D, dev=on)
    code, L = _DTYPES[dtype], lib()
    desc = ctypes.byref(kdn_ffn_desc_t(rows, D, F, code, int(act), code))
    if workspace is None:
        n = L.kdn_ffn_fwd_workspace_bytes(desc)
        workspace = _swa_workspace(n, x.device) if n > 256 else _status_word(on)
    else:
        _arg(workspace, "workspace", torch.uint8, dev=on)
    st = L.kdn_ffn_fwd(desc, _ptr(x), _ptr(wg), _ptr(wu), _ptr(wd), _ptr(g), _ptr(u), _ptr(h),
                       _ptr(y), _ptr(workspace), workspace.numel(), _stream(None))
    if st:
        _check(st, "kdn_ffn_fwd")
    return y, g, u, h


def kdn_ffn_bwd(x, wg, wu, wd, g, u, h, dy, *, act=KDN_ACT_SILU, dw_dtype=None, grads=None, workspace=None,
                stream=None):
    """Gradients of kdn_ffn_fwd from its g, u and h; dy is the gradient of y.  Returns a dict dx, dwg, dwu,
    dwd; the weights' gradients have dw_dtype (x's, or torch.float32) and, like dx, share no memory with
    inputs or one another.  The status of a device-side wait is in ``workspace`` only (kdn_get_device_status)."""
    if stream is not None:
        return _on(kdn_ffn_bwd, locals())
    on, dtype, rows, D, F = _check_ffn(x, wg, wu, wd)
    if dw_dtype is None:
        dw_dtype = dtype
    elif dw_dtype not in (dtype, torch.float32):
        raise TypeError(f"dw_dtype: {dw_dtype}, expected {dtype} or torch.float32")
    _arg(g, "g", dtype, rows * F, dev=on)
    _arg(u, "u", dtype, rows * F, dev=on)
    _arg(h, "h", dtype, rows * F, dev=on)
    _arg(dy, "dy", dtype, rows * D, dev=on)
    if grads is None:
        grads = {"dx": torch.empty_like(x), "dwg": torch.empty_like(wg, dtype=dw_dtype),
                 "dwu": torch.empty_like(wu, dtype=dw_dtype), "dwd": torch.empty_like(wd, dtype=dw_dtype)}
    else:
        _arg(grads.get("dx"), "dx", dtype, rows * D, dev=on)
        for n in ("dwg", "dwu", "dwd"):
            _arg(grads.get(n), n, dw_dtype, F * D, dev=on)
    L = lib()
    desc = ctypes.byref(kdn_ffn_desc_t(rows, D, F, _DTYPES[dtype], int(act), _DTYPES[dw_dtype]))
    if workspace is None:
        workspace = _swa_workspace(L.kdn_ffn_bwd_workspace_bytes(desc), x.device)
    else:
        _arg(workspace, "workspace", torch.uint8, dev=on)
    G = grads
    st = L.kdn_ffn_bwd(desc, _ptr(x), _ptr(wg), _ptr(wu), _ptr(wd), _ptr(g), _ptr(u), _ptr(h), _ptr(dy),
                       _ptr(G["dx"]), _ptr(G["dwg"]), _ptr(G["dwu"]), _ptr(G["dwd"]), _ptr(workspace),
                       workspace.numel(), _stream(None))
    if st:
        _check(st, "kdn_ffn_bwd")
    return grads
