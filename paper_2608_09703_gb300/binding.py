"""Python binding of the C ABI in include/mls.h (argument marshalling only).

Every function here has the name of the C entry point it wraps and does
nothing but turn torch tensors into device pointers and the current CUDA
stream into a stream handle; all computation happens in libmls.so.  There is
no fallback: if the library is missing or fails to load, the call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

# MLS_CHECKED=1 selects the checked build (invariant checks in the kernels).
_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)),
                         "libmls_checked.so" if os.environ.get("MLS_CHECKED") == "1"
                         else "libmls.so")
_lib = None

MLS_BF16, MLS_FP32 = 0, 1
MLS_OK = 0
MLS_ERR_ARG, MLS_ERR_ALIGN, MLS_ERR_UNSUPPORTED = -1, -2, -3
MLS_ERR_WORKSPACE, MLS_ERR_CUDA, MLS_ERR_DEVICE = -4, -5, -6
MLS_STATUS_BAD_TARGET, MLS_STATUS_TIMEOUT, MLS_STATUS_CHECK, MLS_STATUS_DRAIN = 1, 2, 4, 8
MLS_STATUS_BAD_SEQ = 16
MLS_AGG_TOKEN_MEAN, MLS_AGG_SEQ_MEAN, MLS_AGG_SUM = 0, 1, 2
MLS_CLIP_MAX_TENSORS = 16384
MLS_POLICY_MAX_SEQS = 1 << 30
MLS_MAX_MODELS = 4


class MLSError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {mls_strerror(code)} (code {code})")
        self.code = code


class mls_problem(ctypes.Structure):
    _fields_ = [
        ("M", ctypes.c_int32),
        ("T", ctypes.c_int64),
        ("V", ctypes.c_int64),
        ("d", ctypes.POINTER(ctypes.c_int32)),
        ("teacher", ctypes.c_int32),
        ("tau", ctypes.c_float),
        ("alpha", ctypes.c_float),
        ("w", ctypes.POINTER(ctypes.c_float)),
        ("in_dtype", ctypes.c_int32),
        ("vocab_group", ctypes.c_int64),
    ]


class mls_spec_problem(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32),
        ("gamma", ctypes.c_int32),
        ("V", ctypes.c_int64),
        ("d_draft", ctypes.c_int32),
        ("d_verify", ctypes.c_int32),
        ("temperature", ctypes.c_float),
        ("top_p", ctypes.c_float),
        ("greedy", ctypes.c_int32),
        ("in_dtype", ctypes.c_int32),
    ]


class mls_policy_problem(ctypes.Structure):
    _fields_ = [
        ("M", ctypes.c_int32),
        ("T", ctypes.c_int64),
        ("V", ctypes.c_int64),
        ("B", ctypes.c_int32),
        ("clip_low", ctypes.c_float),
        ("clip_high", ctypes.c_float),
        ("beta", ctypes.c_float),
        ("agg", ctypes.c_int32),
        ("adv_per_seq", ctypes.c_int32),
        ("w", ctypes.POINTER(ctypes.c_float)),
    ]


class mls_kernel_time(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char_p), ("launches", ctypes.c_int), ("total_ms", ctypes.c_double)]


def library_path() -> str:
    return _LIB_PATH


def lib():
    """The loaded libmls.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "`python -m paper_2608_09703_gb300.build`"
                               + (" --checked" if _LIB_PATH.endswith("_checked.so") else ""))
        L = ctypes.CDLL(_LIB_PATH)
        P = ctypes.POINTER(mls_problem)
        vp = ctypes.c_void_p
        vpp = ctypes.POINTER(ctypes.c_void_p)
        L.mls_workspace_size.argtypes = [P]
        L.mls_workspace_size.restype = ctypes.c_size_t
        L.mls_head_loss_fwd.argtypes = [P, vpp, vpp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.mls_head_loss_fwd.restype = ctypes.c_int
        L.mls_head_loss_bwd.argtypes = [P, vpp, vpp, vp, vp, ctypes.c_float, vpp, vpp, vp,
                                        ctypes.c_size_t, vp]
        L.mls_head_loss_bwd.restype = ctypes.c_int
        L.mls_get_status.argtypes = [vp]
        L.mls_get_status.restype = ctypes.c_int
        L.mls_strerror.argtypes = [ctypes.c_int]
        L.mls_strerror.restype = ctypes.c_char_p
        L.mls_head_pairwise.argtypes = [P, vpp, vpp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.mls_head_pairwise.restype = ctypes.c_int
        i64, i32 = ctypes.c_int64, ctypes.c_int32
        L.mls_junction_fwd.argtypes = [i64, i32, i32, i32, i32, vp, vp, vp, vp]
        L.mls_junction_fwd.restype = ctypes.c_int
        L.mls_junction_bwd.argtypes = [i64, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp]
        L.mls_junction_bwd.restype = ctypes.c_int
        L.mls_head_loss_fwd_noalloc.argtypes = [P, vpp, vpp, vp, vp, vp, vp, vp, vp, vp]
        L.mls_head_loss_fwd_noalloc.restype = ctypes.c_int
        SP = ctypes.POINTER(mls_spec_problem)
        L.mls_spec_workspace_size.argtypes = [SP]
        L.mls_spec_workspace_size.restype = ctypes.c_size_t
        L.mls_spec_verify.argtypes = [SP, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.mls_spec_verify.restype = ctypes.c_int
        f32, sz = ctypes.c_float, ctypes.c_size_t
        L.mls_logp_workspace_size.argtypes = [P]
        L.mls_logp_workspace_size.restype = sz
        L.mls_head_logp_fwd.argtypes = [P, vpp, vpp, vp, vp, vp, vp, sz, vp]
        L.mls_head_logp_fwd.restype = ctypes.c_int
        L.mls_head_logp_bwd.argtypes = [P, vpp, vpp, vp, vp, vp, vpp, vpp, vp, sz, vp]
        L.mls_head_logp_bwd.restype = ctypes.c_int
        L.mls_head_logp_fwd_peak.argtypes = [P, vpp, vpp, vp, vp, vp, vp, vp, sz, vp]
        L.mls_head_logp_fwd_peak.restype = ctypes.c_int
        L.mls_head_logp_bwd_peak.argtypes = [P, vpp, vpp, vp, vp, vp, vp, vpp, vpp, vp, sz, vp]
        L.mls_head_logp_bwd_peak.restype = ctypes.c_int
        L.mls_layer_norm_fwd.argtypes = [i64, i32, i32, f32, vp, vp, vp, vp, vp, vp, vp]
        L.mls_layer_norm_fwd.restype = ctypes.c_int
        L.mls_layer_norm_workspace_size.argtypes = [i64, i32]
        L.mls_layer_norm_workspace_size.restype = sz
        L.mls_layer_norm_bwd.argtypes = [i64, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.mls_layer_norm_bwd.restype = ctypes.c_int
        PP = ctypes.POINTER(mls_policy_problem)
        L.mls_policy_workspace_size.argtypes = [PP]
        L.mls_policy_workspace_size.restype = sz
        L.mls_policy_loss.argtypes = [PP, vp, vp, vp, vp, vp, vp, f32, vp, vp, vp, vp, vp, sz, vp]
        L.mls_policy_loss.restype = ctypes.c_int
        L.mls_grad_clip_workspace_size.argtypes = [i32]
        L.mls_grad_clip_workspace_size.restype = sz
        L.mls_grad_clip.argtypes = [i32, vp, vp, vp, f32, vp, vp, sz, vp]
        L.mls_grad_clip.restype = ctypes.c_int
        L.mls_profile_enable.argtypes = [ctypes.c_int]
        L.mls_profile_enable.restype = ctypes.c_int
        L.mls_profile_read.argtypes = [ctypes.POINTER(mls_kernel_time), ctypes.c_int]
        L.mls_profile_read.restype = ctypes.c_int
        _lib = L
    return _lib


class Problem:
    """Owns an mls_problem and the host arrays it points to."""

    def __init__(self, d: Sequence[int], T: int, V: int, teacher: Optional[int] = None,
                 tau: float = 1.0, alpha: float = 0.5, w: Optional[Sequence[float]] = None,
                 in_dtype: int = MLS_BF16, vocab_group: int = 0):
        M = len(d)
        self.d = (ctypes.c_int32 * M)(*[int(x) for x in d])
        self.w = None if w is None else (ctypes.c_float * M)(*[float(x) for x in w])
        self.c = mls_problem(M, int(T), int(V), self.d, M - 1 if teacher is None else int(teacher),
                             float(tau), float(alpha), self.w, int(in_dtype), int(vocab_group))
        self.sizes = (tuple(self.d), int(T), int(V))  # as Python numbers: read at every call

    @property
    def M(self) -> int:
        return self.c.M

    def ref(self):
        return ctypes.byref(self.c)


# Marshalling is on the path of calls of a few microseconds (a junction of one
# decode step): plain integers instead of c_void_p objects, array types made once,
# and the current stream's handle read without building a Stream object took a
# junction call on the host from 9.9 to 5.1 us.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


_PTR_ARRAYS = [ctypes.c_void_p * n for n in range(MLS_MAX_MODELS + 1)]


def _ptrs(ts: Sequence[torch.Tensor]):
    n = len(ts)
    array = _PTR_ARRAYS[n] if n <= MLS_MAX_MODELS else ctypes.c_void_p * n
    return array(*[t.data_ptr() for t in ts])


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _get_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_get_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(rc: int, what: str):
    if rc != MLS_OK:
        raise MLSError(rc, what)


def mls_workspace_size(prob: Problem) -> int:
    return int(lib().mls_workspace_size(prob.ref()))


def mls_head_loss_fwd(prob: Problem, H, W, targets, loss, tok_loss, tok_diag, argmax, stats, ws,
                      stream=None) -> None:
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = lib().mls_head_loss_fwd(prob.ref(), _ptrs(H), _ptrs(W), _ptr(targets), _ptr(loss),
                                 _ptr(tok_loss), _ptr(tok_diag), _ptr(argmax), _ptr(stats), _ptr(ws),
                                 ws_bytes, _stream(stream))
    _check(rc, "mls_head_loss_fwd")


def mls_head_loss_bwd(prob: Problem, H, W, targets, stats, grad_scale: float, dH, dW, ws,
                      stream=None) -> None:
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = lib().mls_head_loss_bwd(prob.ref(), _ptrs(H), _ptrs(W), _ptr(targets), _ptr(stats),
                                 float(grad_scale), _ptrs(dH), _ptrs(dW), _ptr(ws), ws_bytes,
                                 _stream(stream))
    _check(rc, "mls_head_loss_bwd")


def mls_head_pairwise(prob: Problem, H, W, targets, tok_kl, argmax, pair_stats, ws,
                      stream=None) -> None:
    """Per-token KL(p_i || p_j) between sub-models, their means and top-1 agreement."""
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = lib().mls_head_pairwise(prob.ref(), _ptrs(H), _ptrs(W), _ptr(targets), _ptr(tok_kl),
                                 _ptr(argmax), _ptr(pair_stats), _ptr(ws), ws_bytes, _stream(stream))
    _check(rc, "mls_head_pairwise")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return MLS_BF16
    if t.dtype == torch.float32:
        return MLS_FP32
    raise TypeError(t.dtype)


def mls_junction_fwd(o, e, x, embed_first=False, stream=None) -> None:
    """Eq. 1: x = concat(o * ||e|| / ||o||, e) per row (concat(e, ...) if embed_first)."""
    T, dp = o.shape
    rc = lib().mls_junction_fwd(T, dp, dp + e.shape[1], _dtype_code(o), int(bool(embed_first)),
                                _ptr(o), _ptr(e), _ptr(x), _stream(stream))
    _check(rc, "mls_junction_fwd")


def mls_junction_bwd(o, e, g, d_o, d_e, embed_first=False, stream=None) -> None:
    T, dp = o.shape
    rc = lib().mls_junction_bwd(T, dp, dp + e.shape[1], _dtype_code(o), int(bool(embed_first)),
                                _ptr(o), _ptr(e), _ptr(g), _ptr(d_o), _ptr(d_e), _stream(stream))
    _check(rc, "mls_junction_bwd")


def spec_problem(B: int, gamma: int, V: int, d_draft: int, d_verify: int,
                 temperature: float = 0.4, top_p: float = 0.9, greedy: bool = False,
                 in_dtype: int = MLS_BF16) -> mls_spec_problem:
    return mls_spec_problem(int(B), int(gamma), int(V), int(d_draft), int(d_verify),
                            float(temperature), float(top_p), int(bool(greedy)), int(in_dtype))


def mls_spec_workspace_size(p: mls_spec_problem) -> int:
    return int(lib().mls_spec_workspace_size(ctypes.byref(p)))


def mls_spec_verify(p: mls_spec_problem, H_draft, W_draft, H_verify, W_verify, draft_tokens,
                    uniforms, n_accepted, next_token, ws, stream=None) -> None:
    """Speculative-decoding verify step (see include/mls.h)."""
    rc = lib().mls_spec_verify(ctypes.byref(p), _ptr(H_draft), _ptr(W_draft), _ptr(H_verify),
                               _ptr(W_verify), _ptr(draft_tokens), _ptr(uniforms),
                               _ptr(n_accepted), _ptr(next_token), _ptr(ws),
                               0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    _check(rc, "mls_spec_verify")


# The operators below check what a data pointer alone cannot say.
def _expect(name: str, t: Optional[torch.Tensor], dtype, shape, like: int = -2) -> int:
    """Raises unless t is a dense CUDA tensor of this type and shape on the current
    device (and on device `like`, if given); returns its device."""
    if like >= 0 and t is not None and t.dtype is dtype and t.shape == shape and t.is_contiguous() \
            and t.get_device() == like:
        return like
    if t is None:
        raise TypeError(f"{name}: None")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: not contiguous")
    dev = t.get_device()
    if dev != like:
        if like != -2:
            raise ValueError(f"{name}: on device {t.device}, not with the other tensors")
        if dev < 0:
            raise ValueError(f"{name}: on {t.device}, expected a CUDA device")
        if dev != (_get_device() if _get_device is not None else torch.cuda.current_device()):
            raise ValueError(f"{name}: on {t.device}, which is not the current device")
    return dev


class _Home:
    """The device of an object's buffers.  Its calls run there only while that device is
    the current one."""

    __slots__ = ("index",)

    def __init__(self, buffer: torch.Tensor):
        self.index = buffer.get_device()
        if self.index < 0:
            raise ValueError(f"device {buffer.device}: expected a CUDA device")

    def __call__(self) -> int:
        now = _get_device() if _get_device is not None else torch.cuda.current_device()
        if now != self.index:
            raise ValueError(f"made on cuda:{self.index}, but cuda:{now} is the current device")
        return now


def _ws_args(ws: Optional[torch.Tensor], like: int):
    if ws is None:
        return None, 0
    if not ws.is_contiguous() or ws.get_device() != like:
        raise ValueError("ws: not contiguous or on another device")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _expect_heads(prob: "Problem", H, W, targets, dev: int = -2) -> int:
    d, T, V = prob.sizes
    if len(H) != len(d) or len(W) != len(d):
        raise ValueError(f"{len(H)} hidden states and {len(W)} heads for {len(d)} sub-models")
    dev = _expect("targets", targets, torch.int32, (T,), dev)
    dt = torch.bfloat16 if prob.c.in_dtype == MLS_BF16 else torch.float32
    for h, w, dm in zip(H, W, d):
        _expect("H", h, dt, (T, dm), dev)
        _expect("W", w, dt, (V, dm), dev)
    return dev


def mls_logp_workspace_size(prob: "Problem") -> int:
    return int(lib().mls_logp_workspace_size(prob.ref()))


def mls_head_logp_fwd(prob: "Problem", H, W, targets, logp, lse, ws, stream=None, peak=None) -> None:
    """Log-probabilities of the targets through every head (see include/mls.h); with peak
    the backward keeps the digits of tokens with nearly all of the mass."""
    dev = _expect_heads(prob, H, W, targets)
    rows = (prob.c.M, prob.c.T)
    _expect("logp", logp, torch.float32, rows, dev)
    _expect("lse", lse, torch.float32, rows, dev)
    wsp, wsn = _ws_args(ws, dev)
    if peak is None:
        rc = lib().mls_head_logp_fwd(prob.ref(), _ptrs(H), _ptrs(W), _ptr(targets), _ptr(logp), _ptr(lse),
                                     wsp, wsn, _stream(stream))
    else:
        _expect("peak", peak, torch.float32, (2,) + rows, dev)
        rc = lib().mls_head_logp_fwd_peak(prob.ref(), _ptrs(H), _ptrs(W), _ptr(targets), _ptr(logp), _ptr(lse),
                                          _ptr(peak), wsp, wsn, _stream(stream))
    _check(rc, "mls_head_logp_fwd")


def mls_head_logp_bwd(prob: "Problem", H, W, targets, lse, dlogp, dH, dW, ws, stream=None, peak=None) -> None:
    dev = _expect_heads(prob, H, W, targets)
    d, T, V = prob.sizes
    _expect("lse", lse, torch.float32, (len(d), T), dev)
    _expect("dlogp", dlogp, torch.float32, (len(d), T), dev)
    if len(dH) != len(d) or len(dW) != len(d):
        raise ValueError(f"{len(dH)} and {len(dW)} gradients for {len(d)} sub-models")
    for h, w, dm in zip(dH, dW, d):
        _expect("dH", h, H[0].dtype, (T, dm), dev)
        _expect("dW", w, H[0].dtype, (V, dm), dev)
    wsp, wsn = _ws_args(ws, dev)
    if peak is None:
        rc = lib().mls_head_logp_bwd(prob.ref(), _ptrs(H), _ptrs(W), _ptr(targets), _ptr(lse), _ptr(dlogp),
                                     _ptrs(dH), _ptrs(dW), wsp, wsn, _stream(stream))
    else:
        _expect("peak", peak, torch.float32, (2, len(d), T), dev)
        rc = lib().mls_head_logp_bwd_peak(prob.ref(), _ptrs(H), _ptrs(W), _ptr(targets), _ptr(lse), _ptr(peak),
                                          _ptr(dlogp), _ptrs(dH), _ptrs(dW), wsp, wsn, _stream(stream))
    _check(rc, "mls_head_logp_bwd")


def _width(d: int) -> int:
    if d >> 31:  # ctypes would cut it
        raise ValueError(f"d = {d}: past 32 bits")
    return d


def mls_layer_norm_fwd(x, gain, bias, eps: float, y, mean=None, rstd=None, stream=None) -> None:
    """y = (x - mean) rstd gain + bias per row of x [T, d] (see include/mls.h)."""
    T, d = x.shape[0], _width(x.shape[1])
    code = _dtype_code(x)
    dev = _expect("x", x, x.dtype, (T, d))
    _expect("y", y, x.dtype, (T, d), dev)
    for name, t in (("gain", gain), ("bias", bias)):
        if t is not None:
            _expect(name, t, x.dtype, (d,), dev)
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t is not None:
            _expect(name, t, torch.float32, (T,), dev)
    rc = lib().mls_layer_norm_fwd(T, d, code, float(eps), _ptr(x), _ptr(gain), _ptr(bias), _ptr(y),
                                  _ptr(mean), _ptr(rstd), _stream(stream))
    _check(rc, "mls_layer_norm_fwd")


def mls_layer_norm_workspace_size(T: int, d: int) -> int:
    return int(lib().mls_layer_norm_workspace_size(int(T), int(d)))


def mls_layer_norm_bwd(x, gain, dy, mean, rstd, dx, dgain, dbias, ws, stream=None) -> None:
    T, d = x.shape[0], _width(x.shape[1])
    code = _dtype_code(x)
    dev = _expect("x", x, x.dtype, (T, d))
    _expect("dy", dy, x.dtype, (T, d), dev)
    _expect("dx", dx, x.dtype, (T, d), dev)
    _expect("mean", mean, torch.float32, (T,), dev)
    _expect("rstd", rstd, torch.float32, (T,), dev)
    if gain is not None:
        _expect("gain", gain, x.dtype, (d,), dev)
    for name, t in (("dgain", dgain), ("dbias", dbias)):
        if t is not None:
            _expect(name, t, torch.float32, (d,), dev)
    wsp, wsn = _ws_args(ws, dev)
    rc = lib().mls_layer_norm_bwd(T, d, code, _ptr(x), _ptr(gain), _ptr(dy), _ptr(mean), _ptr(rstd),
                                  _ptr(dx), _ptr(dgain), _ptr(dbias), wsp, wsn, _stream(stream))
    _check(rc, "mls_layer_norm_bwd")


_AGG = {"token": MLS_AGG_TOKEN_MEAN, "seq": MLS_AGG_SEQ_MEAN, "sum": MLS_AGG_SUM}


class PolicyProblem:
    """Owns an mls_policy_problem and the host array it points to.  agg: "token",
    "seq" or "sum"."""

    def __init__(self, T: int, V: int, M: int = 1, B: int = 0, clip_low: float = 0.2,
                 clip_high: float = 0.2, beta: float = 0.0, agg: str = "token",
                 adv_per_seq: bool = False, w: Optional[Sequence[float]] = None):
        if w is not None and len(w) != M:
            raise ValueError(f"w: {len(w)} weights for {M} sub-models")
        if max(M, B) >> 31:  # ctypes would cut it
            raise ValueError(f"M = {M}, B = {B}: past 32 bits")
        self.w = None if w is None else (ctypes.c_float * M)(*[float(x) for x in w])
        self.c = mls_policy_problem(int(M), int(T), int(V), int(B), float(clip_low), float(clip_high),
                                    float(beta), _AGG[agg], int(bool(adv_per_seq)), self.w)

    def ref(self):
        return ctypes.byref(self.c)


def mls_policy_workspace_size(prob: PolicyProblem) -> int:
    return int(lib().mls_policy_workspace_size(prob.ref()))


def mls_policy_loss(prob: PolicyProblem, logp, old_logp, ref_logp, adv, targets, seq_start,
                    grad_scale: float, loss, tok_loss, diag, dlogp, ws, stream=None) -> None:
    """Clipped policy loss with a KL term and its gradient (see include/mls.h)."""
    c = prob.c
    f32, i32, rows = torch.float32, torch.int32, (c.M, c.T)
    dev = _expect("logp", logp, f32, rows)
    _expect("old_logp", old_logp, f32, rows, dev)
    _expect("adv", adv, f32, (c.B if c.adv_per_seq else c.T,), dev)
    _expect("targets", targets, i32, (c.T,), dev)
    _expect("loss", loss, f32, (1,), dev)
    if seq_start is not None:
        _expect("seq_start", seq_start, i32, (c.B + 1,), dev)
    for name, t, shape in (("ref_logp", ref_logp, rows), ("tok_loss", tok_loss, rows),
                           ("diag", diag, (3, c.M)), ("dlogp", dlogp, rows)):
        if t is not None:
            _expect(name, t, f32, shape, dev)
    wsp, wsn = _ws_args(ws, dev)
    rc = lib().mls_policy_loss(prob.ref(), _ptr(logp), _ptr(old_logp), _ptr(ref_logp), _ptr(adv),
                               _ptr(targets), _ptr(seq_start), float(grad_scale), _ptr(loss),
                               _ptr(tok_loss), _ptr(diag), _ptr(dlogp), wsp, wsn, _stream(stream))
    _check(rc, "mls_policy_loss")


def _places(grads):
    """What tells whether a list's table still describes it: a tensor given other memory may keep
    its address and count and be of another type, or no longer be dense."""
    return (list(map(torch.Tensor.data_ptr, grads)), list(map(torch.Tensor.numel, grads)),
            [g.dtype for g in grads], all(map(torch.Tensor.is_contiguous, grads)))


class _ClipTable:
    """The host arrays that describe a list of tensors to mls_grad_clip."""

    def __init__(self, grads: Sequence[torch.Tensor]):
        self.n, self.device = len(grads), None
        for i, g in enumerate(grads):
            dev = _expect(f"grads[{i}]", g, g.dtype, g.shape, -2 if self.device is None else self.device)
            self.device = dev
        self.places = _places(grads)
        self.g = (ctypes.c_void_p * self.n)(*self.places[0])
        self.numel = (ctypes.c_int64 * self.n)(*self.places[1])
        self.dtype = (ctypes.c_int32 * self.n)(*[_dtype_code(g) for g in grads])


def mls_grad_clip_workspace_size(n: int) -> int:
    return int(lib().mls_grad_clip_workspace_size(int(n)))


def mls_grad_clip(grads, max_norm: float, stats, ws, stream=None) -> None:
    """Global norm of a list of tensors, and clipping in place (see include/mls.h)."""
    t = grads if isinstance(grads, _ClipTable) else _ClipTable(grads)
    dev = _expect("stats", stats, torch.float32, (2,))
    if t.device is not None and t.device != dev:
        raise ValueError("stats: not with the gradients")
    wsp, wsn = _ws_args(ws, dev)
    rc = lib().mls_grad_clip(t.n, t.g, t.numel, t.dtype, float(max_norm), _ptr(stats), wsp, wsn,
                             _stream(stream))
    _check(rc, "mls_grad_clip")


def mls_head_loss_fwd_noalloc(prob: Problem, H, W, targets, loss, tok_loss, tok_diag, argmax,
                              stats, stream=None) -> None:
    """Forward with the library's built-in scratch instead of a workspace, for
    callers that cannot allocate device memory when they call; allocates nothing."""
    rc = lib().mls_head_loss_fwd_noalloc(prob.ref(), _ptrs(H), _ptrs(W), _ptr(targets), _ptr(loss),
                                         _ptr(tok_loss), _ptr(tok_diag), _ptr(argmax), _ptr(stats),
                                         _stream(stream))
    _check(rc, "mls_head_loss_fwd_noalloc")


MLS_NOALLOC_SCRATCH_BYTES = 64 << 20


def mls_get_status(stream=None) -> int:
    rc = lib().mls_get_status(_stream(stream))
    if rc < 0:
        raise MLSError(rc, "mls_get_status")
    return rc


def mls_strerror(code: int) -> str:
    try:
        return lib().mls_strerror(int(code)).decode()
    except Exception:  # library missing: still describe the code
        return f"code {code}"


def mls_profile_enable(on: bool = True) -> None:
    lib().mls_profile_enable(1 if on else 0)


def mls_profile_read() -> dict:
    """{kernel name: (launches, total device ms)} since the last enable/read."""
    buf = (mls_kernel_time * 32)()
    n = lib().mls_profile_read(buf, 32)
    if n < 0:
        raise MLSError(n, "mls_profile_read")
    return {buf[i].name.decode(): (buf[i].launches, buf[i].total_ms) for i in range(min(n, 32))}


# ----------------------------------------------------------------------------------------
# Convenience layer: allocates outputs and workspace with torch, then calls the entry points.
# An object's results stay in its buffers until its next call, and its calls must not
# overlap on the GPU: for work on several streams at once make an object for each.
class HeadLoss:
    """Fused suite head + CE + distillation loss over device tensors.

    H[m]: [T, d_m], W[m]: [V, d_m] (bf16 or fp32, contiguous, on one CUDA
    device); targets: int32 [T].  Buffers are allocated once per shape.
    """

    def __init__(self, d, T, V, teacher=None, tau=1.0, alpha=0.5, w=None, dtype=torch.bfloat16,
                 device="cuda", vocab_group=0):
        self.prob = Problem(d, T, V, teacher, tau, alpha, w,
                            MLS_BF16 if dtype == torch.bfloat16 else MLS_FP32, vocab_group)
        M = len(d)
        self.M, self.T, self.V, self.d = M, T, V, list(d)
        dev = torch.device(device)
        self.loss = torch.zeros(1, dtype=torch.float32, device=dev)
        self.tok_loss = torch.empty(M, T, dtype=torch.float32, device=dev)
        self.tok_diag = torch.empty(3, M, T, dtype=torch.float32, device=dev)
        self.argmax = torch.empty(M, T, dtype=torch.int32, device=dev)
        self.stats = torch.empty(2, M, T, dtype=torch.float32, device=dev)
        self.dH = [torch.empty(T, dm, dtype=torch.float32, device=dev) for dm in d]
        self.dW = [torch.empty(V, dm, dtype=torch.float32, device=dev) for dm in d]
        nbytes = mls_workspace_size(self.prob)
        self.ws = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)

    def forward(self, H, W, targets, stream=None):
        mls_head_loss_fwd(self.prob, H, W, targets, self.loss, self.tok_loss, self.tok_diag,
                          self.argmax, self.stats, self.ws, stream)
        return self.loss

    def pairwise(self, H, W, targets=None, stream=None):
        """Evaluation metrics between sub-models; returns (tok_kl [M,M,T],
        argmax [M,T], pair_stats [2,M,M])."""
        dev = self.loss.device
        if not hasattr(self, "tok_kl"):
            self.tok_kl = torch.empty(self.M, self.M, self.T, dtype=torch.float32, device=dev)
            self.pair_stats = torch.empty(2, self.M, self.M, dtype=torch.float32, device=dev)
            self.eval_argmax = torch.empty(self.M, self.T, dtype=torch.int32, device=dev)
        mls_head_pairwise(self.prob, H, W, targets, self.tok_kl, self.eval_argmax, self.pair_stats,
                          self.ws, stream)
        return self.tok_kl, self.eval_argmax, self.pair_stats

    def backward(self, H, W, targets, grad_scale=1.0, stream=None):
        mls_head_loss_bwd(self.prob, H, W, targets, self.stats, grad_scale, self.dH, self.dW,
                          self.ws, stream)
        return self.dH, self.dW


class SpecVerify:
    """Speculative-decoding verify step with its outputs and workspace
    allocated once per shape.  H_draft: [B*gamma, d_draft], W_draft:
    [V, d_draft], H_verify: [B*(gamma+1), d_verify], W_verify: [V, d_verify]
    (bf16 or fp32); draft_tokens int32 [B, gamma]; uniforms fp32
    [B, gamma+1, 2]."""

    def __init__(self, B, gamma, V, d_draft, d_verify, temperature=0.4, top_p=0.9, greedy=False,
                 dtype=torch.bfloat16, device="cuda"):
        self.p = spec_problem(B, gamma, V, d_draft, d_verify, temperature, top_p, greedy,
                              MLS_BF16 if dtype == torch.bfloat16 else MLS_FP32)
        dev = torch.device(device)
        self.n_accepted = torch.empty(B, dtype=torch.int32, device=dev)
        self.next_token = torch.empty(B, dtype=torch.int32, device=dev)
        self.ws = torch.empty(max(mls_spec_workspace_size(self.p), 1), dtype=torch.uint8,
                              device=dev)

    def __call__(self, H_draft, W_draft, H_verify, W_verify, draft_tokens, uniforms, stream=None):
        mls_spec_verify(self.p, H_draft, W_draft, H_verify, W_verify, draft_tokens, uniforms,
                        self.n_accepted, self.next_token, self.ws, stream)
        return self.n_accepted, self.next_token


class HeadLogp:
    """Log-probabilities of given tokens through a suite's heads, and the backward
    of a gradient per token, with outputs and workspace allocated once.  H[m]:
    [T, d_m], W[m]: [V, d_m] bf16; targets int32 [T]; dlogp fp32 [M, T]; dH and dW
    bf16.  lse and peak go from the forward to the backward."""

    def __init__(self, d, T, V, tau=1.0, device="cuda", vocab_group=0):
        self.prob = Problem(d, T, V, tau=tau, vocab_group=vocab_group)
        M, dev = len(d), torch.device(device)
        self.rows = (M, T)
        self.logp = torch.empty(M, T, dtype=torch.float32, device=dev)
        self.lse = torch.empty(M, T, dtype=torch.float32, device=dev)
        self.peak = torch.empty(2, M, T, dtype=torch.float32, device=dev)  # handed on to the backward
        self.dH = [torch.empty(T, dm, dtype=torch.bfloat16, device=dev) for dm in d]
        self.dW = [torch.empty(V, dm, dtype=torch.bfloat16, device=dev) for dm in d]
        self.ws = torch.empty(max(mls_logp_workspace_size(self.prob), 1), dtype=torch.uint8, device=dev)
        self.home = _Home(self.ws)

    # The object's own buffers need no check at every call (some 4 us of a forward and
    # backward of two sub-models).
    def forward(self, H, W, targets, stream=None):
        _expect_heads(self.prob, H, W, targets, self.home())
        rc = lib().mls_head_logp_fwd_peak(self.prob.ref(), _ptrs(H), _ptrs(W), targets.data_ptr(),
                                          self.logp.data_ptr(), self.lse.data_ptr(), self.peak.data_ptr(),
                                          self.ws.data_ptr(), self.ws.numel(), _stream(stream))
        _check(rc, "mls_head_logp_fwd")
        return self.logp

    def backward(self, H, W, targets, dlogp, stream=None):
        """Gradients for the tokens of the last forward; returns (dH, dW)."""
        dev = _expect_heads(self.prob, H, W, targets, self.home())
        _expect("dlogp", dlogp, torch.float32, self.rows, dev)
        rc = lib().mls_head_logp_bwd_peak(self.prob.ref(), _ptrs(H), _ptrs(W), targets.data_ptr(),
                                          self.lse.data_ptr(), self.peak.data_ptr(), dlogp.data_ptr(),
                                          _ptrs(self.dH), _ptrs(self.dW), self.ws.data_ptr(), self.ws.numel(),
                                          _stream(stream))
        _check(rc, "mls_head_logp_bwd")
        return self.dH, self.dW


class LayerNorm:
    """Layer norm of x [T, d] (bf16 or fp32) with its outputs and workspace
    allocated once: y, the row statistics mean and rstd, and, with `backward`, dx
    and the fp32 gradients dgain (if gain) and dbias (if bias)."""

    def __init__(self, T, d, eps=1e-5, gain=True, bias=True, dtype=torch.bfloat16, device="cuda",
                 backward=True):
        self.eps, self.gain, self.bias = float(eps), gain, bias
        self.shape, self.dtype = (T, _width(d)), dtype
        self.code = MLS_BF16 if dtype is torch.bfloat16 else MLS_FP32
        if dtype not in (torch.bfloat16, torch.float32):
            raise TypeError(dtype)
        dev = torch.device(device)
        self.y = torch.empty(T, d, dtype=dtype, device=dev)
        self.home = _Home(self.y)
        self.mean = self.rstd = self.dx = self.dgain = self.dbias = self.ws = None
        if backward:
            self.mean = torch.empty(T, dtype=torch.float32, device=dev)
            self.rstd = torch.empty(T, dtype=torch.float32, device=dev)
            self.dx = torch.empty(T, d, dtype=dtype, device=dev)
            self.dgain = torch.empty(d, dtype=torch.float32, device=dev) if gain else None
            self.dbias = torch.empty(d, dtype=torch.float32, device=dev) if bias else None
            if gain or bias:
                self.ws = torch.empty(max(mls_layer_norm_workspace_size(T, d), 1), dtype=torch.uint8,
                                      device=dev)

    def _gain(self, name, t, has):
        if (t is not None) != has:
            raise ValueError(f"{name}: " + ("missing" if has else "given to a norm made without one"))

    def forward(self, x, gain=None, bias=None, stream=None):
        self._gain("gain", gain, self.gain)
        self._gain("bias", bias, self.bias)
        dev = _expect("x", x, self.dtype, self.shape, self.home())
        T, d = self.shape
        if gain is not None:
            _expect("gain", gain, self.dtype, (d,), dev)
        if bias is not None:
            _expect("bias", bias, self.dtype, (d,), dev)
        rc = lib().mls_layer_norm_fwd(T, d, self.code, self.eps, x.data_ptr(), _ptr(gain), _ptr(bias),
                                      self.y.data_ptr(), _ptr(self.mean), _ptr(self.rstd), _stream(stream))
        _check(rc, "mls_layer_norm_fwd")
        return self.y

    def backward(self, x, dy, gain=None, stream=None):
        """Gradients for the rows of the last forward; returns (dx, dgain, dbias)."""
        self._gain("gain", gain, self.gain)
        if self.dx is None:
            raise ValueError("made with backward=False")
        dev = _expect("x", x, self.dtype, self.shape, self.home())
        _expect("dy", dy, self.dtype, self.shape, dev)
        T, d = self.shape
        if gain is not None:
            _expect("gain", gain, self.dtype, (d,), dev)
        ws = self.ws
        rc = lib().mls_layer_norm_bwd(T, d, self.code, x.data_ptr(), _ptr(gain), dy.data_ptr(),
                                      self.mean.data_ptr(), self.rstd.data_ptr(), self.dx.data_ptr(),
                                      _ptr(self.dgain), _ptr(self.dbias), _ptr(ws),
                                      0 if ws is None else ws.numel(), _stream(stream))
        _check(rc, "mls_layer_norm_bwd")
        return self.dx, self.dgain, self.dbias


class PolicyLoss:
    """Clipped policy loss with a KL term over [M, T] log-probabilities, and its
    gradient dlogp, in one call; outputs and workspace allocated once.  adv: [B]
    with adv_per_seq, else [T]; targets int32 [T] (outside [0, V): left out);
    seq_start int32 [B + 1] when B > 0."""

    def __init__(self, T, V, M=1, B=0, clip_low=0.2, clip_high=0.2, beta=0.0, agg="token",
                 adv_per_seq=False, w=None, device="cuda"):
        self.prob = PolicyProblem(T, V, M, B, clip_low, clip_high, beta, agg, adv_per_seq, w)
        dev = torch.device(device)
        self.rows, self.shapes = (M, T), ((B if adv_per_seq else T,), (T,), (B + 1,))
        self.loss = torch.zeros(1, dtype=torch.float32, device=dev)
        self.tok_loss = torch.empty(M, T, dtype=torch.float32, device=dev)
        self.diag = torch.empty(3, M, dtype=torch.float32, device=dev)
        self.dlogp = torch.empty(M, T, dtype=torch.float32, device=dev)
        self.ws = torch.empty(max(mls_policy_workspace_size(self.prob), 1), dtype=torch.uint8, device=dev)
        self.home = _Home(self.ws)

    def __call__(self, logp, old_logp, adv, targets, ref_logp=None, seq_start=None, grad_scale=1.0,
                 stream=None):
        f32, i32, rows, (adv_s, tok_s, seq_s) = torch.float32, torch.int32, self.rows, self.shapes
        dev = _expect("logp", logp, f32, rows, self.home())
        _expect("old_logp", old_logp, f32, rows, dev)
        _expect("adv", adv, f32, adv_s, dev)
        _expect("targets", targets, i32, tok_s, dev)
        if seq_start is not None:
            _expect("seq_start", seq_start, i32, seq_s, dev)
        if ref_logp is not None:
            _expect("ref_logp", ref_logp, f32, rows, dev)
        rc = lib().mls_policy_loss(self.prob.ref(), logp.data_ptr(), old_logp.data_ptr(), _ptr(ref_logp),
                                   adv.data_ptr(), targets.data_ptr(), _ptr(seq_start), grad_scale,
                                   self.loss.data_ptr(), self.tok_loss.data_ptr(), self.diag.data_ptr(),
                                   self.dlogp.data_ptr(), self.ws.data_ptr(), self.ws.numel(), _stream(stream))
        _check(rc, "mls_policy_loss")
        return self.loss


class GradClip:
    """Global norm of a fixed list of gradient tensors (bf16 or fp32, as HeadLoss
    and the others keep them from step to step) and clipping in place.  Returns
    fp32 [2]: the norm and the factor applied.  A tensor given other memory since
    (`t.data = ...`) is followed, of another type or size too; what a new object would
    refuse is refused."""

    def __init__(self, grads: Sequence[torch.Tensor]):
        self.grads = list(grads)  # keeps the buffers alive
        if not self.grads:
            raise ValueError("grads: empty")
        self.table = _ClipTable(self.grads)
        dev = self.grads[0].device
        self.stats = torch.empty(2, dtype=torch.float32, device=dev)
        self.ws = torch.empty(mls_grad_clip_workspace_size(len(self.grads)), dtype=torch.uint8, device=dev)
        self.home = _Home(self.ws)

    def __call__(self, max_norm, stream=None):
        self.home()
        if _places(self.grads) != self.table.places:
            self.table = _ClipTable(self.grads)  # refuses what it cannot describe
        t, ws = self.table, self.ws
        rc = lib().mls_grad_clip(t.n, t.g, t.numel, t.dtype, max_norm, self.stats.data_ptr(), ws.data_ptr(),
                                 ws.numel(), _stream(stream))
        _check(rc, "mls_grad_clip")
        return self.stats
