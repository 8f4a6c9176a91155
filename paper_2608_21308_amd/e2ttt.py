"""ctypes binding of libe2ttt.so (the HIP implementation, C ABI in include/e2ttt.h).

Argument marshalling only: tensors are passed as device pointers together with
the current HIP stream; every step of the computation runs in the library's
kernels.  PyTorch provides device memory and streams.  Importing this module
on a machine without the built library raises immediately.
"""
from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass
from functools import cached_property, lru_cache

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libe2ttt.so")

FW_MLP = 0
FW_SWIGLU = 1
DT_F32 = 0
DT_BF16 = 1
FLAG_NO_RESIDUAL_LN = 1
FLAG_CHUNK_AVERAGED = 2
FLAG_LN_AFFINE = 4
FLAG_POST_NORM = 8       # post-chunk L2 normalisation of the fast-weight rows (App. B.1)
QK_SILU = 1              # steps of the query/key preparation
QK_UNIT = 2
QK_INTERLEAVED = 4

STATUS = {0: "ok", 1: "null argument", 2: "bad shape", 3: "unsupported",
          4: "workspace too small", 5: "HIP error", 6: "device-side wait expired"}

# Every entry point the header declares (checked by the CPU test-suite).
EXPORTS = ("e2ttt_param_count", "e2ttt_workspace_bytes", "e2ttt_backward_scratch_bytes",
           "e2ttt_chunk_forward", "e2ttt_chunk_backward", "e2ttt_chunk_coeffs",
           "e2ttt_apply", "e2ttt_gates_forward", "e2ttt_gates_backward", "e2ttt_wait_status",
           "e2ttt_chunk_forward_static", "e2ttt_chunk_forward_ln", "e2ttt_chunk_backward_ln",
           "e2ttt_apply_ln", "e2ttt_delta_workspace_bytes", "e2ttt_delta_scratch_bytes",
           "e2ttt_delta_forward", "e2ttt_delta_backward", "e2ttt_delta_step",
           "e2ttt_qk_forward", "e2ttt_qk_backward", "e2ttt_attn_workspace_bytes",
           "e2ttt_attn_forward", "e2ttt_attn_scratch_bytes", "e2ttt_attn_backward", "e2ttt_cache_page_bytes",
           "e2ttt_cache_write", "e2ttt_cache_read", "e2ttt_cache_workspace_bytes",
           "e2ttt_cache_attend", "e2ttt_status_str")


class E2TTTError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (where, STATUS.get(status, "?"), status))


class Desc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("T", ctypes.c_int32),
                ("d", ctypes.c_int32), ("dh", ctypes.c_int32), ("chunk", ctypes.c_int32),
                ("fw", ctypes.c_int32), ("io", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("ln_eps", ctypes.c_float)]


class GateParams(ctypes.Structure):
    """e2ttt_gate_params (the paper's defaults, App. B.1)."""
    _fields_ = [("eta_base", ctypes.c_float), ("alpha_base", ctypes.c_float),
                ("tau", ctypes.c_float)]

    def __init__(self, eta_base=0.01, alpha_base=0.1, tau=32.0):
        super().__init__(eta_base, alpha_base, tau)


class Strides(ctypes.Structure):
    _fields_ = [("b", ctypes.c_int64), ("h", ctypes.c_int64), ("t", ctypes.c_int64)]


class DeltaDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "HK", "H", "T", "dk", "dv", "io")]
    _fields_ += [("scale", ctypes.c_float)]


class DeltaStrides(ctypes.Structure):
    _fields_ = [(n, Strides) for n in ("q", "k", "v", "out", "eta", "log_gamma", "d_out", "dq",
                                       "dk", "dv", "d_eta", "d_log_gamma")]


class QKDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "H", "HK", "T", "d", "rot", "io")]
    _fields_ += [("flags", ctypes.c_uint32), ("eps", ctypes.c_float), ("rot_scale", ctypes.c_float)]


class QKStrides(ctypes.Structure):
    _fields_ = [(n, Strides) for n in ("q", "k", "q_out", "k_out", "d_q_out", "d_k_out", "dq", "dk")]


class AttentionDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "HK", "H", "T", "S", "d", "io")]
    _fields_ += [("scale", ctypes.c_float), ("left", ctypes.c_int32), ("right", ctypes.c_int32)]


class AttentionStrides(ctypes.Structure):
    _fields_ = [(n, Strides) for n in ("q", "k", "v", "out", "d_out", "dq", "dk", "dv")]


class CacheDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "HK", "H", "T", "d", "pages", "io")]
    _fields_ += [("scale", ctypes.c_float), ("left", ctypes.c_int32)]


class CacheStrides(ctypes.Structure):
    _fields_ = [(n, Strides) for n in ("q", "k", "v", "out")]


_lib = None


def load():
    """Load the in-tree HIP library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libe2ttt.so is not built (run __graft_entry__.build() or "
                          "python paper_2608_21308_amd/build_lib.py)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz, i = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    dp = ctypes.POINTER(Desc)
    lib.e2ttt_param_count.argtypes = [dp]
    lib.e2ttt_param_count.restype = sz
    lib.e2ttt_workspace_bytes.argtypes = [dp, i]
    lib.e2ttt_workspace_bytes.restype = sz
    lib.e2ttt_backward_scratch_bytes.argtypes = [dp]
    lib.e2ttt_backward_scratch_bytes.restype = sz
    lib.e2ttt_chunk_forward.argtypes = [dp] + [vp] * 12 + [sz, i, vp]
    lib.e2ttt_chunk_forward.restype = i
    lib.e2ttt_chunk_backward.argtypes = [dp] + [vp] * 9 + [sz] + [vp] * 12 + [sz, vp]
    lib.e2ttt_chunk_backward.restype = i
    lib.e2ttt_chunk_coeffs.argtypes = [dp] + [vp] * 7
    lib.e2ttt_chunk_coeffs.restype = i
    lib.e2ttt_apply.argtypes = [dp] + [vp] * 4
    lib.e2ttt_apply.restype = i
    gp = ctypes.POINTER(GateParams)
    lib.e2ttt_gates_forward.argtypes = [gp, ctypes.c_int64] + [vp] * 7
    lib.e2ttt_gates_forward.restype = i
    lib.e2ttt_gates_backward.argtypes = [gp, ctypes.c_int64] + [vp] * 10
    lib.e2ttt_gates_backward.restype = i
    lib.e2ttt_wait_status.argtypes = [dp, vp, vp, vp]
    lib.e2ttt_wait_status.restype = i
    lib.e2ttt_chunk_forward_static.argtypes = [dp] + [vp] * 12
    lib.e2ttt_chunk_forward_static.restype = i
    lib.e2ttt_chunk_forward_ln.argtypes = [dp] + [vp] * 14 + [sz, i, vp]
    lib.e2ttt_chunk_forward_ln.restype = i
    lib.e2ttt_chunk_backward_ln.argtypes = [dp] + [vp] * 11 + [sz] + [vp] * 14 + [sz, vp]
    lib.e2ttt_chunk_backward_ln.restype = i
    lib.e2ttt_apply_ln.argtypes = [dp] + [vp] * 6
    lib.e2ttt_apply_ln.restype = i
    dd, ds = ctypes.POINTER(DeltaDesc), ctypes.POINTER(DeltaStrides)
    lib.e2ttt_delta_workspace_bytes.argtypes = [dd, i]
    lib.e2ttt_delta_workspace_bytes.restype = sz
    lib.e2ttt_delta_scratch_bytes.argtypes = [dd]
    lib.e2ttt_delta_scratch_bytes.restype = sz
    lib.e2ttt_delta_forward.argtypes = [dd, ds] + [vp] * 10 + [sz, i, vp]
    lib.e2ttt_delta_forward.restype = i
    lib.e2ttt_delta_backward.argtypes = [dd, ds] + [vp] * 7 + [sz] + [vp] * 9 + [sz, vp]
    lib.e2ttt_delta_backward.restype = i
    lib.e2ttt_delta_step.argtypes = [dd, ds] + [vp] * 7 + [ctypes.c_int32, vp, vp]
    lib.e2ttt_delta_step.restype = i
    qd, qs = ctypes.POINTER(QKDesc), ctypes.POINTER(QKStrides)
    lib.e2ttt_qk_forward.argtypes = [qd, qs] + [vp] * 7
    lib.e2ttt_qk_forward.restype = i
    lib.e2ttt_qk_backward.argtypes = [qd, qs] + [vp] * 9
    lib.e2ttt_qk_backward.restype = i
    ad, as_ = ctypes.POINTER(AttentionDesc), ctypes.POINTER(AttentionStrides)
    lib.e2ttt_attn_workspace_bytes.argtypes = [ad]
    lib.e2ttt_attn_workspace_bytes.restype = sz
    lib.e2ttt_attn_forward.argtypes = [ad, as_] + [vp] * 7 + [sz, vp]
    lib.e2ttt_attn_forward.restype = i
    lib.e2ttt_attn_scratch_bytes.argtypes = [ad]
    lib.e2ttt_attn_scratch_bytes.restype = sz
    lib.e2ttt_attn_backward.argtypes = [ad, as_] + [vp] * 12 + [sz, vp]
    lib.e2ttt_attn_backward.restype = i
    cd, cs, i32 = ctypes.POINTER(CacheDesc), ctypes.POINTER(CacheStrides), ctypes.c_int32
    lib.e2ttt_cache_page_bytes.argtypes = [i32, i32]
    lib.e2ttt_cache_page_bytes.restype = sz
    lib.e2ttt_cache_write.argtypes = [cd, cs] + [vp] * 6 + [i32, vp]
    lib.e2ttt_cache_write.restype = i
    lib.e2ttt_cache_read.argtypes = [cd, cs] + [vp] * 4 + [i32] + [vp] * 3
    lib.e2ttt_cache_read.restype = i
    lib.e2ttt_cache_workspace_bytes.argtypes = [cd]
    lib.e2ttt_cache_workspace_bytes.restype = sz
    lib.e2ttt_cache_attend.argtypes = [cd, cs] + [vp] * 5 + [i32] + [vp] * 3 + [sz, vp]
    lib.e2ttt_cache_attend.restype = i
    lib.e2ttt_status_str.argtypes = [i]
    lib.e2ttt_status_str.restype = ctypes.c_char_p
    _lib = lib
    return lib


@dataclass(frozen=True)
class Config:
    B: int
    H: int
    T: int
    d: int
    dh: int
    chunk: int
    fw: int = FW_MLP
    io: int = DT_BF16
    flags: int = 0
    ln_eps: float = 1e-5

    def desc(self) -> Desc:
        return Desc(self.B, self.H, self.T, self.d, self.dh, self.chunk, self.fw, self.io,
                    self.flags, self.ln_eps)

    @cached_property
    def _call(self):
        """What every call derives from the (frozen) fields: the descriptor by
        reference, the io type, and the element counts of the token, gate,
        state and head arrays."""
        n_tok = self.B * self.H * self.T
        return (ctypes.byref(self.desc()), self.torch_io, n_tok * self.d, n_tok,
                self.B * self.H * self.P, self.H * self.d)

    def __getstate__(self):
        # (a reference to a descriptor is of this process)
        return {n: v for n, v in self.__dict__.items() if n != "_call"}

    @property
    def P(self) -> int:
        return (2 if self.fw == FW_MLP else 3) * self.d * self.dh

    @property
    def n_chunks(self) -> int:
        return (self.T + self.chunk - 1) // self.chunk

    @property
    def torch_io(self):
        return torch.bfloat16 if self.io == DT_BF16 else torch.float32


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    # the current stream of the current device, as torch.cuda.current_stream() gives it
    return _raw_stream(_current_device())


try:
    _raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
except AttributeError:   # a build without those bindings
    def _raw_stream(device):
        return torch.cuda.current_stream(device).cuda_stream

    _current_device = torch.cuda.current_device


def _ok(t, dtype, n, device):
    """The checks of _check_tensors for one tensor (None passes) at the price
    a call of a few microseconds can afford; a tensor that fails is then looked
    at by _check_tensors, which says what is wrong with it."""
    return t is None or (type(t) in _TENSORS and t.dtype is dtype and t.numel() == n and
                         t.is_cuda and t.get_device() == device and t.is_contiguous())


_TENSORS = (torch.Tensor, torch.nn.Parameter)


def _check(st: int, where: str):
    if st != 0:
        raise E2TTTError(st, where)


_IO = ("q", "k", "v", "out", "d_out", "dq", "dk", "dv")
_GATE = ("eta", "beta", "gamma", "d_eta", "d_beta", "d_gamma", "kw", "km")
_STATE = ("w_in", "m_in", "w_out", "m_out", "d_w_in", "d_m_in", "d_w_out", "d_m_out")
_HEAD = ("ln_weight", "ln_bias", "d_ln_weight", "d_ln_bias")


def _check_tensors(cfg: Config, **ts):
    """Host-side guard before any launch: every tensor the library will read or
    write is a contiguous device tensor on the device of the first one, with
    the element type and element count the header gives for its role.  The
    library itself checks only sizes it is handed (workspace, scratch)."""
    dev = None
    n_tok = cfg.B * cfg.H * cfg.T
    for name, t in ts.items():
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or not t.is_contiguous():
            raise ValueError("%s must be a contiguous tensor" % name)
        if name in _IO:
            want = (cfg.torch_io, n_tok * cfg.d)
        elif name in _GATE:
            want = (torch.float32, n_tok)
        elif name in _STATE:
            want = (torch.float32, cfg.B * cfg.H * cfg.P)
        elif name in _HEAD:
            want = (torch.float32, cfg.H * cfg.d)
        else:                       # workspace, scratch: byte buffers
            want = (torch.uint8, t.numel())
        if t.dtype != want[0] or t.numel() != want[1]:
            raise ValueError("%s: expected %d elements of %s, got %d of %s"
                             % (name, want[1], want[0], t.numel(), t.dtype))
        if t.device.type != "cuda":
            raise ValueError("%s must be a device tensor" % name)
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError("%s is on %s, expected %s" % (name, t.device, dev))


def workspace_bytes(cfg: Config, save_for_backward: bool) -> int:
    return int(load().e2ttt_workspace_bytes(cfg._call[0], int(bool(save_for_backward))))


def backward_scratch_bytes(cfg: Config) -> int:
    return int(load().e2ttt_backward_scratch_bytes(cfg._call[0]))


def alloc_workspace(cfg: Config, save_for_backward: bool, device="cuda"):
    n = workspace_bytes(cfg, save_for_backward)
    if n == 0:
        raise E2TTTError(3, "e2ttt_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def forward(cfg: Config, q, k, v, eta, beta, gamma, w_in, m_in=None, *, out=None, w_out=None,
            m_out=None, workspace=None, save_for_backward=False, ln_weight=None, ln_bias=None):
    """Runs e2ttt_chunk_forward (e2ttt_chunk_forward_ln with the LayerNorm affine
    ln_weight, ln_bias [H, d]) on the current stream; returns (out, w_out, m_out, workspace)."""
    d, io, n_io, n_gate, n_state, n_head = cfg._call
    f32 = torch.float32
    dev = q.get_device() if isinstance(q, torch.Tensor) else -1
    if not (dev >= 0 and q is not None and _ok(q, io, n_io, dev) and _ok(k, io, n_io, dev) and
            _ok(v, io, n_io, dev) and _ok(out, io, n_io, dev) and _ok(eta, f32, n_gate, dev) and
            _ok(beta, f32, n_gate, dev) and _ok(gamma, f32, n_gate, dev) and
            _ok(w_in, f32, n_state, dev) and _ok(m_in, f32, n_state, dev) and
            _ok(w_out, f32, n_state, dev) and _ok(m_out, f32, n_state, dev) and
            (workspace is None or _ok(workspace, torch.uint8, workspace.numel(), dev)) and
            _ok(ln_weight, f32, n_head, dev) and _ok(ln_bias, f32, n_head, dev)):
        _check_tensors(cfg, q=q, k=k, v=v, eta=eta, beta=beta, gamma=gamma, w_in=w_in, m_in=m_in,
                       out=out, w_out=w_out, m_out=m_out, workspace=workspace,
                       ln_weight=ln_weight, ln_bias=ln_bias)
    lib = load()
    dev = q.device
    if out is None:
        out = torch.empty_like(q)
    if w_out is None:
        w_out = torch.empty_like(w_in)
    if m_out is None:
        m_out = torch.empty_like(w_in)
    if workspace is None:
        workspace = alloc_workspace(cfg, save_for_backward, dev)
    st = lib.e2ttt_chunk_forward_ln(d, _ptr(ln_weight), _ptr(ln_bias), _ptr(q),
                                    _ptr(k), _ptr(v), _ptr(eta), _ptr(beta), _ptr(gamma),
                                    _ptr(w_in), _ptr(m_in), _ptr(out), _ptr(w_out), _ptr(m_out),
                                    _ptr(workspace), workspace.numel(),
                                    int(bool(save_for_backward)), _stream())
    _check(st, "e2ttt_chunk_forward")
    return out, w_out, m_out, workspace


# Bytes of the library-owned workspace of e2ttt_chunk_forward_static.
STATIC_WORKSPACE_BYTES = 64 << 20


def forward_static(cfg: Config, q, k, v, eta, beta, gamma, w_in, m_in, out, w_out, m_out):
    """Runs e2ttt_chunk_forward_static (no save for the backward) on the current
    stream into the caller's out, w_out, m_out; allocates nothing."""
    for name, t in (("out", out), ("w_out", w_out), ("m_out", m_out)):
        if t is None:
            raise ValueError("%s must be given: this entry point allocates nothing" % name)
    _check_tensors(cfg, q=q, k=k, v=v, eta=eta, beta=beta, gamma=gamma, w_in=w_in, m_in=m_in,
                   out=out, w_out=w_out, m_out=m_out)
    st = load().e2ttt_chunk_forward_static(cfg._call[0], _ptr(q), _ptr(k), _ptr(v), _ptr(eta),
                                           _ptr(beta), _ptr(gamma), _ptr(w_in), _ptr(m_in),
                                           _ptr(out), _ptr(w_out), _ptr(m_out), _stream())
    _check(st, "e2ttt_chunk_forward_static")
    return out, w_out, m_out


def backward(cfg: Config, q, k, v, eta, beta, gamma, w_in, m_in, workspace, d_out, d_w_out=None,
             d_m_out=None, *, grads=None, scratch=None, ln_weight=None, ln_bias=None):
    """Runs e2ttt_chunk_backward (e2ttt_chunk_backward_ln with the LayerNorm affine);
    returns a dict of gradients (dq, dk, dv, d_eta, d_beta, d_gamma, d_w_in, d_m_in, and
    d_ln_weight, d_ln_bias [H, d] with the affine)."""
    _check_tensors(cfg, q=q, k=k, v=v, eta=eta, beta=beta, gamma=gamma, w_in=w_in, m_in=m_in,
                   workspace=workspace, d_out=d_out, d_w_out=d_w_out, d_m_out=d_m_out,
                   scratch=scratch, ln_weight=ln_weight, ln_bias=ln_bias, **(grads or {}))
    lib = load()
    dev = q.device
    if grads is None:
        grads = dict(dq=torch.empty_like(q), dk=torch.empty_like(k), dv=torch.empty_like(v),
                     d_eta=torch.empty_like(eta), d_beta=torch.empty_like(beta),
                     d_gamma=None if gamma is None else torch.empty_like(gamma),
                     d_w_in=torch.empty_like(w_in), d_m_in=torch.empty_like(w_in))
        if ln_weight is not None:
            grads["d_ln_weight"] = torch.empty_like(ln_weight)
            grads["d_ln_bias"] = torch.empty_like(ln_weight)
    if scratch is None:
        scratch = torch.empty(backward_scratch_bytes(cfg), dtype=torch.uint8, device=dev)
    g = grads
    st = lib.e2ttt_chunk_backward_ln(
        cfg._call[0], _ptr(ln_weight), _ptr(ln_bias), _ptr(q), _ptr(k), _ptr(v), _ptr(eta),
        _ptr(beta), _ptr(gamma), _ptr(w_in), _ptr(m_in), _ptr(workspace), workspace.numel(),
        _ptr(d_out), _ptr(d_w_out), _ptr(d_m_out), _ptr(g["dq"]), _ptr(g["dk"]), _ptr(g["dv"]),
        _ptr(g["d_eta"]), _ptr(g["d_beta"]), _ptr(g["d_gamma"]), _ptr(g["d_w_in"]),
        _ptr(g["d_m_in"]), _ptr(g.get("d_ln_weight")), _ptr(g.get("d_ln_bias")), _ptr(scratch),
        scratch.numel(), _stream())
    _check(st, "e2ttt_chunk_backward")
    return grads


def apply(cfg: Config, q, w, out=None, ln_weight=None, ln_bias=None):
    """Runs e2ttt_apply (e2ttt_apply_ln with the LayerNorm affine): out = f_W(q)
    for the cfg.T tokens of q per unit, all at the state w [B,H,P]."""
    d, io, n_io, _, n_state, n_head = cfg._call
    dev = q.get_device() if isinstance(q, torch.Tensor) else -1
    if not (dev >= 0 and _ok(q, io, n_io, dev) and _ok(w, torch.float32, n_state, dev) and
            _ok(out, io, n_io, dev) and _ok(ln_weight, torch.float32, n_head, dev) and
            _ok(ln_bias, torch.float32, n_head, dev)):
        _check_tensors(cfg, q=q, w_in=w, out=out, ln_weight=ln_weight, ln_bias=ln_bias)
    lib = load()
    if out is None:
        out = torch.empty_like(q)
    st = lib.e2ttt_apply_ln(d, _ptr(ln_weight), _ptr(ln_bias), _ptr(q), _ptr(w),
                            _ptr(out), _stream())
    _check(st, "e2ttt_apply")
    return out


def wait_status(cfg: Config, workspace=None, scratch=None) -> int:
    """e2ttt_wait_status: waits for the current stream, then returns the status
    code of the bounded waits of the last forward that used `workspace` and the
    last backward that used `scratch` (0, or 6 when a wait expired)."""
    if workspace is None and scratch is None:
        raise ValueError("give a workspace, a scratch buffer or both")
    _check_tensors(cfg, workspace=workspace, scratch=scratch)
    return int(load().e2ttt_wait_status(cfg._call[0], _ptr(workspace), _ptr(scratch),
                                        _stream()))


def chunk_coeffs(cfg: Config, eta, beta, gamma):
    """Scalar kernels: (kw [B,H,T], km [B,H,T], carry [B,H,NC,3])."""
    _check_tensors(cfg, eta=eta, beta=beta, gamma=gamma)
    lib = load()
    kw = torch.empty_like(eta)
    km = torch.empty_like(eta)
    carry = torch.empty((cfg.B, cfg.H, cfg.n_chunks, 3), dtype=torch.float32, device=eta.device)
    st = lib.e2ttt_chunk_coeffs(cfg._call[0], _ptr(eta), _ptr(beta), _ptr(gamma), _ptr(kw),
                                _ptr(km), _ptr(carry), _stream())
    _check(st, "e2ttt_chunk_coeffs")
    return kw, km, carry


def _check_gate_tensors(*ts):
    n = ts[0].numel()
    for t in ts:
        if t is None:
            continue
        if t.dtype != torch.float32 or not t.is_contiguous() or t.numel() != n:
            raise ValueError("gate arrays must be contiguous float32 tensors of one size")
        if t.device.type != "cuda" or t.device != ts[0].device:
            raise ValueError("gate arrays must be device tensors on one GPU")


def gates_forward(params: GateParams, l_eta, l_beta, l_alpha=None, out=None):
    """Gate parameterization, eqs. (12)-(14): (eta, beta, gamma) from the logits
    (gamma None when l_alpha is None).  `out`: optional (eta, beta, gamma)
    tensors to write into."""
    _check_gate_tensors(l_eta, l_beta, l_alpha)
    lib = load()
    if out is None:
        eta = torch.empty_like(l_eta)
        beta = torch.empty_like(l_beta)
        gamma = None if l_alpha is None else torch.empty_like(l_alpha)
    else:
        eta, beta, gamma = out
        _check_gate_tensors(eta, beta, gamma)
        if eta.numel() != l_eta.numel() or (gamma is None) != (l_alpha is None):
            raise ValueError("gate outputs must match the logits")
    st = lib.e2ttt_gates_forward(ctypes.byref(params), l_eta.numel(), _ptr(l_eta), _ptr(l_beta),
                                 _ptr(l_alpha), _ptr(eta), _ptr(beta), _ptr(gamma), _stream())
    _check(st, "e2ttt_gates_forward")
    return eta, beta, gamma


def gates_backward(params: GateParams, l_eta, l_beta, l_alpha, d_eta, d_beta, d_gamma,
                   out=None):
    """Gradients of the logits from the gate gradients: (d_l_eta, d_l_beta,
    d_l_alpha).  `out`: optional tensors of those three to write into."""
    _check_gate_tensors(l_eta, l_beta, l_alpha, d_eta, d_beta, d_gamma)
    lib = load()
    if out is None:
        g_eta = torch.empty_like(l_eta)
        g_beta = torch.empty_like(l_beta)
        g_alpha = None if l_alpha is None else torch.empty_like(l_alpha)
    else:
        g_eta, g_beta, g_alpha = out
        _check_gate_tensors(g_eta, g_beta, g_alpha)
        if g_eta.numel() != l_eta.numel() or (g_alpha is None) != (l_alpha is None):
            raise ValueError("gate gradient outputs must match the logits")
    st = lib.e2ttt_gates_backward(ctypes.byref(params), l_eta.numel(), _ptr(l_eta), _ptr(l_beta),
                                  _ptr(l_alpha), _ptr(d_eta), _ptr(d_beta), _ptr(d_gamma),
                                  _ptr(g_eta), _ptr(g_beta), _ptr(g_alpha), _stream())
    _check(st, "e2ttt_gates_backward")
    return g_eta, g_beta, g_alpha


class E2TTTFunction(torch.autograd.Function):
    """Autograd wrapper: forward saves the workspace, backward calls the library."""

    @staticmethod
    def forward(ctx, cfg, q, k, v, eta, beta, gamma, w_in, m_in):
        out, w_out, m_out, ws = forward(cfg, q, k, v, eta, beta, gamma, w_in, m_in,
                                        save_for_backward=True)
        ctx.cfg = cfg
        ctx.save_for_backward(q, k, v, eta, beta, gamma, w_in, m_in, ws)
        # an unused output's gradient arrives as None (the library's NULL) instead
        # of zeros that would be filled and read
        ctx.set_materialize_grads(False)
        return out, w_out, m_out

    @staticmethod
    def backward(ctx, d_out, d_w_out, d_m_out):
        q, k, v, eta, beta, gamma, w_in, m_in, ws = ctx.saved_tensors
        if d_out is None:
            d_out = torch.zeros_like(q)
        g = backward(ctx.cfg, q, k, v, eta, beta, gamma, w_in, m_in, ws, d_out.contiguous(),
                     None if d_w_out is None else d_w_out.contiguous(),
                     None if d_m_out is None else d_m_out.contiguous())
        return (None, g["dq"], g["dk"], g["dv"], g["d_eta"], g["d_beta"], g["d_gamma"],
                g["d_w_in"], None if m_in is None else g["d_m_in"])


class GatesFunction(torch.autograd.Function):
    """Autograd wrapper of the gate parameterization (eqs. (12)-(14)): logits
    in, (eta, beta, gamma) out; the backward calls e2ttt_gates_backward.
    gamma is None when l_alpha is None."""

    @staticmethod
    def forward(ctx, params, l_eta, l_beta, l_alpha):
        eta, beta, gamma = gates_forward(params, l_eta, l_beta, l_alpha)
        ctx.params = params
        ctx.save_for_backward(l_eta, l_beta, l_alpha)
        return eta, beta, gamma

    @staticmethod
    def backward(ctx, d_eta, d_beta, d_gamma):
        l_eta, l_beta, l_alpha = ctx.saved_tensors
        zero = lambda ref: torch.zeros_like(ref)
        d_eta = zero(l_eta) if d_eta is None else d_eta.contiguous()
        d_beta = zero(l_beta) if d_beta is None else d_beta.contiguous()
        if l_alpha is not None:
            d_gamma = zero(l_alpha) if d_gamma is None else d_gamma.contiguous()
        else:
            d_gamma = None
        g_eta, g_beta, g_alpha = gates_backward(ctx.params, l_eta, l_beta, l_alpha, d_eta,
                                                d_beta, d_gamma)
        return None, g_eta, g_beta, g_alpha


# ------------------------------------------------- gated delta rule, queries and keys
def _strided(name, t, shape, dtype, device):
    """Guard of the delta and qk calls before any launch: a device tensor of this
    shape and type on `device`, contiguous in its last dimension.  Its strides
    (None: C order)."""
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s must be a tensor" % name)
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError("%s: expected %s of %s, got %s of %s"
                         % (name, tuple(shape), dtype, tuple(t.shape), t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.get_device() != device:
        raise ValueError("%s is on %s, expected cuda:%d" % (name, t.device, device))
    if t.is_contiguous():
        return None
    st = t.stride()
    if len(st) == 4 and st[3] != 1 and shape[3] != 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)
    return tuple(s if n > 1 else 0 for s, n in zip(st[:3], shape))


def _plain(name, t, shape, dtype, device):
    """The same for a contiguous tensor (None passes)."""
    if t is None or _flat(t, shape, dtype, device):
        return
    if _strided(name, t, shape, dtype, device) is not None:
        raise ValueError("%s must be contiguous" % name)


@lru_cache(maxsize=256)
def _strides_ref(kind, given):
    """The strides argument for (name, shape, strides) triples."""
    s = kind()
    for name, shape, st in given:
        if st is None:
            _, h, t = shape[:3]
            inner = shape[3] if len(shape) == 4 else 1
            st = (h * t * inner, t * inner, inner)
        setattr(s, name, Strides(*st))
    return ctypes.byref(s)


def _flat(t, shape, dtype, device):
    """Whether t passes _strided's checks as a tensor in C order."""
    return (type(t) in _TENSORS and t.dtype is dtype and t.get_device() == device and
            t.shape == shape and t.is_contiguous())


def _layout(kind, device, *given):
    """Checks (name, tensor, shape, dtype) and gives the call's strides argument
    (None: every tensor in C order, found at the price that a call of a few
    microseconds can afford)."""
    for _, t, shape, dtype in given:
        if not _flat(t, shape, dtype, device):
            break
    else:
        return None
    st = tuple((name, shape, _strided(name, t, shape, dtype, device))
               for name, t, shape, dtype in given)
    return _strides_ref(kind, st) if any(x[2] is not None for x in st) else None


def _device_of(t):
    if not isinstance(t, torch.Tensor) or t.get_device() < 0:
        raise ValueError("the first tensor must be a device tensor")
    return t.get_device()


def _on_device(f):
    """The library works on the current device: make it that of the first tensor."""
    def call(cfg, q, *args, **kw):
        if _device_of(q) == _current_device():
            return f(cfg, q, *args, **kw)
        with torch.cuda.device(q.device):
            return f(cfg, q, *args, **kw)
    call.__name__, call.__doc__, call.__wrapped__ = f.__name__, f.__doc__, f
    return call


def _as_rows(g):
    """A gradient as the library takes it: rows contiguous, on 16 bytes and at
    most 2^23 elements apart."""
    if g.data_ptr() % 16:          # (a contiguous view may start anywhere in its storage)
        return g.clone(memory_format=torch.contiguous_format)
    if g.is_contiguous():
        return g
    if g.stride(-1) != 1 or g.stride(2) > 1 << 23 or any(
            s * g.element_size() % 16 for s, n in zip(g.stride()[:3], g.shape) if n > 1):
        return g.contiguous()
    return g


def _as_state(g):
    """The same of a state's gradient: contiguous, on 16 bytes."""
    return g.clone(memory_format=torch.contiguous_format) if g.data_ptr() % 16 else g.contiguous()


@dataclass(frozen=True)
class DeltaConfig:
    """Gated delta rule: H value heads share HK key heads; o_t = scale W_t q_t."""
    B: int
    HK: int
    H: int
    T: int
    dk: int
    dv: int
    io: int = DT_BF16
    scale: float = 1.0

    def desc(self) -> DeltaDesc:
        return DeltaDesc(self.B, self.HK, self.H, self.T, self.dk, self.dv, self.io, self.scale)

    @cached_property
    def _call(self):
        """The descriptor by reference, the io type and the tensors' shapes."""
        return (ctypes.byref(self.desc()), torch.bfloat16 if self.io == DT_BF16 else torch.float32,
                torch.Size((self.B, self.HK, self.T, self.dk)),
                torch.Size((self.B, self.H, self.T, self.dv)), torch.Size((self.B, self.H, self.T)),
                torch.Size((self.B, self.H, self.dv, self.dk)))

    def __getstate__(self):
        return {n: v for n, v in self.__dict__.items() if n != "_call"}


def delta_workspace_bytes(cfg: DeltaConfig, save_for_backward: bool) -> int:
    return int((_lib or load()).e2ttt_delta_workspace_bytes(cfg._call[0], int(bool(save_for_backward))))


def delta_scratch_bytes(cfg: DeltaConfig) -> int:
    return int((_lib or load()).e2ttt_delta_scratch_bytes(cfg._call[0]))


def alloc_delta_workspace(cfg: DeltaConfig, save_for_backward: bool, device="cuda"):
    n = delta_workspace_bytes(cfg, save_for_backward)
    if n == 0:
        raise E2TTTError(3, "e2ttt_delta_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _buffer(name, t, device):
    if t is not None:
        _plain(name, t, t.shape, torch.uint8, device)


@_on_device
def delta_forward(cfg: DeltaConfig, q, k, v, eta, log_gamma=None, w_in=None, *, lengths=None,
                  out=None, w_out=None, workspace=None, save_for_backward=False):
    """Runs e2ttt_delta_forward on the current stream: the gated delta rule over
    q, k [B, HK, T, dk], v [B, H, T, dv] (any strides with a contiguous last
    dimension, such as a transposed [B, T, H, d]), eta and log_gamma [B, H, T]
    (log_gamma None: no decay), from w_in [B, H, dv, dk] (None: zero), over the
    first lengths [B] (int32) tokens of each sequence.  Returns (out, w_out,
    workspace); out has v's order in memory."""
    d, io, s_k, s_v, s_g, s_w = cfg._call
    dev, f32 = q.get_device(), torch.float32
    if out is None:
        out = torch.empty_like(v)
    st = _layout(DeltaStrides, dev, ("q", q, s_k, io), ("k", k, s_k, io), ("v", v, s_v, io),
                 ("out", out, s_v, io), ("eta", eta, s_g, f32),
                 *(() if log_gamma is None else (("log_gamma", log_gamma, s_g, f32),)))
    _plain("w_in", w_in, s_w, f32, dev)
    _plain("w_out", w_out, s_w, f32, dev)
    _plain("lengths", lengths, s_g[:1], torch.int32, dev)
    _buffer("workspace", workspace, dev)
    if w_out is None:
        w_out = torch.empty(s_w, dtype=f32, device=q.device)
    if workspace is None:
        workspace = alloc_delta_workspace(cfg, save_for_backward, q.device)
    st = (_lib or load()).e2ttt_delta_forward(
        d, st, q.data_ptr(), k.data_ptr(), v.data_ptr(), eta.data_ptr(), _ptr(log_gamma),
        _ptr(lengths), _ptr(w_in), out.data_ptr(), w_out.data_ptr(), workspace.data_ptr(),
        workspace.numel(), int(bool(save_for_backward)), _stream())
    _check(st, "e2ttt_delta_forward")
    return out, w_out, workspace


def _new_grads(cfg, q, k, v, eta, log_gamma):
    return dict(dq=torch.empty_like(q), dk=torch.empty_like(k), dv=torch.empty_like(v),
                d_eta=torch.empty_like(eta),
                d_log_gamma=None if log_gamma is None else torch.empty_like(log_gamma),
                d_w_in=torch.empty(cfg._call[5], dtype=torch.float32, device=q.device))


def _run_delta_backward(cfg, st, q, k, v, eta, log_gamma, workspace, d_out, d_w_out, lengths, g,
                        scratch):
    """The library's call on checked tensors (st: their strides argument)."""
    if scratch is None:
        scratch = torch.empty(delta_scratch_bytes(cfg), dtype=torch.uint8, device=q.device)
    st = (_lib or load()).e2ttt_delta_backward(
        cfg._call[0], st, q.data_ptr(), k.data_ptr(), v.data_ptr(), eta.data_ptr(), _ptr(log_gamma),
        _ptr(lengths), workspace.data_ptr(), workspace.numel(), d_out.data_ptr(), _ptr(d_w_out),
        g["dq"].data_ptr(), g["dk"].data_ptr(), g["dv"].data_ptr(), g["d_eta"].data_ptr(),
        _ptr(g.get("d_log_gamma")), _ptr(g.get("d_w_in")), scratch.data_ptr(), scratch.numel(),
        _stream())
    _check(st, "e2ttt_delta_backward")
    return g


@_on_device
def delta_backward(cfg: DeltaConfig, q, k, v, eta, log_gamma, workspace, d_out, d_w_out=None, *,
                   lengths=None, grads=None, scratch=None):
    """Runs e2ttt_delta_backward with the workspace of a saving delta_forward;
    returns a dict of gradients (dq, dk, dv, d_eta, d_log_gamma, d_w_in)."""
    _, io, s_k, s_v, s_g, s_w = cfg._call
    dev, f32 = q.get_device(), torch.float32
    g = grads = _new_grads(cfg, q, k, v, eta, log_gamma) if grads is None else grads
    st = _layout(DeltaStrides, dev, ("q", q, s_k, io), ("k", k, s_k, io), ("v", v, s_v, io),
                 ("d_out", d_out, s_v, io), ("dq", g["dq"], s_k, io), ("dk", g["dk"], s_k, io),
                 ("dv", g["dv"], s_v, io), ("eta", eta, s_g, f32), ("d_eta", g["d_eta"], s_g, f32),
                 *(() if log_gamma is None else (("log_gamma", log_gamma, s_g, f32),
                                                 ("d_log_gamma", g["d_log_gamma"], s_g, f32))))
    _plain("d_w_out", d_w_out, s_w, f32, dev)
    _plain("d_w_in", g.get("d_w_in"), s_w, f32, dev)
    _plain("lengths", lengths, s_g[:1], torch.int32, dev)
    _buffer("workspace", workspace, dev)
    _buffer("scratch", scratch, dev)
    return _run_delta_backward(cfg, st, q, k, v, eta, log_gamma, workspace, d_out, d_w_out, lengths,
                               grads, scratch)


def delta_step(cfg: DeltaConfig, q, k, v, eta, log_gamma, w, *, slots=None, out=None):
    """Runs e2ttt_delta_step on the current stream: the cfg.T arriving tokens of
    every sequence, on states w [N, H, dv, dk] that are updated in place.
    Sequence b is at state slots[b] (int32 device tensor; None: at state b, N >=
    B); slots outside 0..N-1 are skipped (zero outputs), rows with the same slot
    are taken in order."""
    dev = _device_of(q)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return delta_step(cfg, q, k, v, eta, log_gamma, w, slots=slots, out=out)
    d, io, s_k, s_v, s_g, s_w = cfg._call
    f32 = torch.float32
    if not isinstance(w, torch.Tensor) or w.dim() != 4 or w.shape[0] < 1:
        raise ValueError("w must be a tensor [N, H, dv, dk] of states")
    if out is None:
        out = torch.empty_like(v)
    n = w.shape[0]
    if (_flat(q, s_k, io, dev) and _flat(k, s_k, io, dev) and _flat(v, s_v, io, dev) and
            _flat(out, s_v, io, dev) and _flat(eta, s_g, f32, dev) and
            (log_gamma is None or _flat(log_gamma, s_g, f32, dev))):
        st = None        # (_layout's answer, for a call of a few microseconds)
    else:
        st = _layout(DeltaStrides, dev, ("q", q, s_k, io), ("k", k, s_k, io), ("v", v, s_v, io),
                     ("out", out, s_v, io), ("eta", eta, s_g, f32),
                     *(() if log_gamma is None else (("log_gamma", log_gamma, s_g, f32),)))
    _plain("w", w, (n, *s_w[1:]), f32, dev)
    if slots is not None:
        _plain("slots", slots, s_g[:1], torch.int32, dev)
    st = (_lib or load()).e2ttt_delta_step(
        d, st, q.data_ptr(), k.data_ptr(), v.data_ptr(), eta.data_ptr(),
        None if log_gamma is None else log_gamma.data_ptr(), w.data_ptr(),
        None if slots is None else slots.data_ptr(), n, out.data_ptr(), _stream())
    if st:
        _check(st, "e2ttt_delta_step")
    return out


class DeltaFunction(torch.autograd.Function):
    """Autograd wrapper of the gated delta rule: (out, w_out) of (cfg, q, k, v,
    eta, log_gamma, w_in, lengths); the forward saves the workspace where a
    gradient may be asked for.  A step to be captured into a graph calls delta_forward
    and delta_backward: torch's capture of its own backward ends the process where an
    eager step of the same leaves is still alive."""

    @classmethod
    def apply(cls, cfg, q, k, v, eta, log_gamma=None, w_in=None, lengths=None):
        if torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad
                                           for t in (q, k, v, eta, log_gamma, w_in)):
            return super().apply(cfg, q, k, v, eta, log_gamma, w_in, lengths)
        return delta_forward(cfg, q, k, v, eta, log_gamma, w_in, lengths=lengths)[:2]

    @staticmethod
    def forward(ctx, cfg, q, k, v, eta, log_gamma=None, w_in=None, lengths=None):
        out, w_out, ws = delta_forward(cfg, q, k, v, eta, log_gamma, w_in, lengths=lengths,
                                       save_for_backward=True)
        ctx.cfg, ctx.has_w = cfg, w_in is not None
        ctx.flat = (q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and
                    eta.is_contiguous() and (log_gamma is None or log_gamma.is_contiguous()))
        ctx.save_for_backward(q, k, v, eta, log_gamma, lengths, ws)
        ctx.set_materialize_grads(False)
        return out, w_out

    @staticmethod
    def backward(ctx, d_out, d_w_out):
        return _once(_delta_grads, ctx, d_out, d_w_out)


def _once(f, ctx, *grads):
    """f's gradients, which do not have gradients themselves."""
    if torch.is_grad_enabled():      # a graph of the backward is asked for
        f = torch.autograd.function.once_differentiable(f)
    return f(ctx, *grads)


def _delta_grads(ctx, d_out, d_w_out):
    cfg = ctx.cfg
    q, k, v, eta, log_gamma, lengths, ws = ctx.saved_tensors
    d_out = torch.zeros_like(v) if d_out is None else _as_rows(d_out)
    if d_w_out is not None:
        d_w_out = _as_state(d_w_out)
    _, io, _, s_v, _, s_w = cfg._call
    dev = q.get_device()
    if (ctx.flat and dev == _current_device() and _flat(d_out, s_v, io, dev) and
            (d_w_out is None or _flat(d_w_out, s_w, torch.float32, dev))):
        # (the rest was checked by the forward, and new gradients lie as their tensors do)
        g = _run_delta_backward(cfg, None, q, k, v, eta, log_gamma, ws, d_out, d_w_out, lengths,
                                _new_grads(cfg, q, k, v, eta, log_gamma), None)
    else:
        g = delta_backward(cfg, q, k, v, eta, log_gamma, ws, d_out, d_w_out, lengths=lengths)
    return (None, g["dq"], g["dk"], g["dv"], g["d_eta"], g["d_log_gamma"],
            g["d_w_in"] if ctx.has_w else None, None)


@dataclass(frozen=True)
class QKConfig:
    """Query/key preparation: H query heads and HK key heads (0: queries alone)
    of dim d; the first `rot` elements turn; flags QK_*."""
    B: int
    H: int
    HK: int
    T: int
    d: int
    rot: int
    io: int = DT_BF16
    flags: int = QK_SILU | QK_UNIT
    eps: float = 1e-6
    rot_scale: float = 1.0

    def desc(self) -> QKDesc:
        return QKDesc(self.B, self.H, self.HK, self.T, self.d, self.rot, self.io, self.flags, self.eps,
                      self.rot_scale)

    @cached_property
    def _call(self):
        return (ctypes.byref(self.desc()), torch.bfloat16 if self.io == DT_BF16 else torch.float32,
                torch.Size((self.B, self.H, self.T, self.d)),
                torch.Size((self.B, self.HK, self.T, self.d)), torch.Size((self.B, self.T)),
                torch.Size((self.rot // 2,)))

    def __getstate__(self):
        return {n: v for n, v in self.__dict__.items() if n != "_call"}


def rotary_frequencies(rot, base=10000.0, factor=1.0, original=None, fast=32.0, slow=1.0,
                       device="cuda"):
    """(inv_freq [rot / 2] float32, rot_scale) of rotary positions at `base`.

    factor > 1 stretches them to a context that many times the trained one:
    without `original` every frequency is divided by it (position
    interpolation); with `original`, the trained length, by parts (the YaRN
    paper): a pair that makes more than `fast` turns over the trained length
    keeps its frequency, one below `slow` turns is divided by factor, between
    them a linear ramp in the pair's index, and rot_scale = 0.1 ln(factor) + 1."""
    if rot < 0 or rot % 2 or not (base > 1.0 and factor >= 1.0):
        raise ValueError("rot is even and not negative, base > 1, factor >= 1")
    p = torch.arange(0, rot, 2, dtype=torch.float64)
    f = base ** (-p / max(rot, 1))
    scale = 1.0
    if factor > 1.0 and original is None:
        f = f / factor
    elif factor > 1.0:
        if not (original > 0 and fast > slow > 0):
            raise ValueError("original > 0, fast > slow > 0")

        def pair(turns):     # the (fractional) pair that makes so many turns over `original`
            return rot * math.log(original / (2.0 * math.pi * turns)) / (2.0 * math.log(base))

        lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), rot - 1)
        ramp = ((p / 2.0 - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
        f = f / factor * ramp + f * (1.0 - ramp)
        scale = 0.1 * math.log(factor) + 1.0
    return f.float().to(device), scale


def _qk_common(cfg, dev, inv_freq, positions):
    s_p, s_f = cfg._call[4:]
    if cfg.rot and inv_freq is None:
        raise ValueError("inv_freq must be given where rot > 0")
    _plain("inv_freq", inv_freq, s_f, torch.float32, dev)
    _plain("positions", positions, s_p, torch.int64, dev)


def qk_forward(cfg: QKConfig, q, k, inv_freq=None, positions=None, *, out=None):
    """Runs e2ttt_qk_forward on the current stream: q [B, H, T, d] and k [B, HK,
    T, d] (None where HK = 0) prepared for the state rules; positions [B, T]
    int64 (None: 0 .. T - 1).  `out`: optional (q, k) tensors to write into,
    which may be the inputs.  Returns (q', k')."""
    dev = _device_of(q)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return qk_forward(cfg, q, k, inv_freq, positions, out=out)
    d, io, s_q, s_k, _, _ = cfg._call
    if (k is None) != (cfg.HK == 0):
        raise ValueError("k is given where HK > 0, and only there")
    _qk_common(cfg, dev, inv_freq, positions)
    if out is not None:
        qo, ko = out
    else:
        qo, ko = torch.empty_like(q), None if k is None else torch.empty_like(k)
    if (_flat(q, s_q, io, dev) and _flat(qo, s_q, io, dev) and
            (k is None or (_flat(k, s_k, io, dev) and _flat(ko, s_k, io, dev)))):
        st = None        # (_layout's answer, for a call of a few microseconds)
    else:
        st = _layout(QKStrides, dev, ("q", q, s_q, io), ("q_out", qo, s_q, io),
                     *(() if k is None else (("k", k, s_k, io), ("k_out", ko, s_k, io))))
    st = (_lib or load()).e2ttt_qk_forward(
        d, st, q.data_ptr(), None if k is None else k.data_ptr(),
        None if inv_freq is None else inv_freq.data_ptr(),
        None if positions is None else positions.data_ptr(), qo.data_ptr(),
        None if k is None else ko.data_ptr(), _stream())
    if st:
        _check(st, "e2ttt_qk_forward")
    return qo, ko


def _run_qk_backward(cfg, st, d_q_out, d_k_out, q, k, inv_freq, positions, dq, dk):
    st = (_lib or load()).e2ttt_qk_backward(
        cfg._call[0], st, _ptr(q), _ptr(k), _ptr(inv_freq), _ptr(positions), d_q_out.data_ptr(),
        _ptr(d_k_out), dq.data_ptr(), None if d_k_out is None else dk.data_ptr(), _stream())
    _check(st, "e2ttt_qk_backward")
    return dq, dk


@_on_device
def qk_backward(cfg: QKConfig, d_q_out, d_k_out, q=None, k=None, inv_freq=None, positions=None, *,
                out=None):
    """Gradients (dq, dk) of qk_forward's inputs q, k from those of its outputs
    (q and k are not needed without QK_SILU and QK_UNIT)."""
    _, io, s_q, s_k, _, _ = cfg._call
    dev, need = d_q_out.get_device(), bool(cfg.flags & (QK_SILU | QK_UNIT))
    if (d_k_out is None) != (cfg.HK == 0):
        raise ValueError("d_k_out is given where HK > 0, and only there")
    _qk_common(cfg, dev, inv_freq, positions)
    dq, dk = out if out is not None else (
        torch.empty_like(d_q_out), None if d_k_out is None else torch.empty_like(d_k_out))
    st = _layout(QKStrides, dev, ("d_q_out", d_q_out, s_q, io), ("dq", dq, s_q, io),
                 *((("q", q, s_q, io),) if need else ()),
                 *(() if d_k_out is None else (("d_k_out", d_k_out, s_k, io), ("dk", dk, s_k, io))),
                 *((("k", k, s_k, io),) if need and d_k_out is not None else ()))
    return _run_qk_backward(cfg, st, d_q_out, d_k_out, q if need else None, k if need else None,
                            inv_freq, positions, dq, dk)


class QKFunction(torch.autograd.Function):
    """Autograd wrapper of the query/key preparation: (q', k') of (cfg, q, k,
    inv_freq, positions).  A step to be captured into a graph calls qk_forward and
    qk_backward (see DeltaFunction)."""

    @staticmethod
    def forward(ctx, cfg, q, k, inv_freq=None, positions=None):
        qo, ko = qk_forward(cfg, q, k, inv_freq, positions)
        ctx.cfg = cfg
        need = cfg.flags & (QK_SILU | QK_UNIT)
        ctx.save_for_backward(q if need else None, k if need else None, inv_freq, positions)
        return qo, ko

    @staticmethod
    def backward(ctx, d_q, d_k):
        return _once(_qk_grads, ctx, d_q, d_k)


def _qk_grads(ctx, d_q, d_k):
    cfg = ctx.cfg
    q, k, inv_freq, positions = ctx.saved_tensors
    d_q, d_k = _as_rows(d_q), None if d_k is None else _as_rows(d_k)
    _, io, s_q, s_k, _, _ = cfg._call
    dev = d_q.get_device()
    if (dev == _current_device() and _flat(d_q, s_q, io, dev) and
            (d_k is None or _flat(d_k, s_k, io, dev)) and (q is None or q.is_contiguous()) and
            (k is None or k.is_contiguous())):
        # (the rest was checked by the forward)
        dq, dk = _run_qk_backward(cfg, None, d_q, d_k, q, k, inv_freq, positions,
                                  torch.empty_like(d_q), None if d_k is None else torch.empty_like(d_k))
    else:
        dq, dk = qk_backward(cfg, d_q, d_k, q, k, inv_freq, positions)
    return None, dq, dk, None, None


# ------------------------------------------------------------------ attention
@dataclass(frozen=True)
class AttentionConfig:
    """Attention of H query heads that share HK key heads: T queries, the last of
    them at the last of S keys (0: T); a query at position p sees the keys
    p - left .. p + right (negative: no bound)."""
    B: int
    HK: int
    H: int
    T: int
    d: int
    io: int = DT_BF16
    S: int = 0
    scale: float = 1.0
    left: int = -1
    right: int = 0

    def desc(self) -> AttentionDesc:
        return AttentionDesc(self.B, self.HK, self.H, self.T, self.S or self.T, self.d, self.io,
                             self.scale, self.left, self.right)

    @cached_property
    def _call(self):
        """The descriptor by reference, the io type and the tensors' shapes."""
        return (ctypes.byref(self.desc()), torch.bfloat16 if self.io == DT_BF16 else torch.float32,
                torch.Size((self.B, self.H, self.T, self.d)),
                torch.Size((self.B, self.HK, self.S or self.T, self.d)),
                torch.Size((self.B, self.H, self.T)))

    @cached_property
    def _bytes(self):
        """Those of the workspace and of the scratch."""
        lib = _lib or load()
        return (int(lib.e2ttt_attn_workspace_bytes(self._call[0])),
                int(lib.e2ttt_attn_scratch_bytes(self._call[0])))

    def __getstate__(self):
        return {n: v for n, v in self.__dict__.items() if n not in ("_call", "_bytes")}


def attention_workspace_bytes(cfg: AttentionConfig) -> int:
    return cfg._bytes[0]


def attention_scratch_bytes(cfg: AttentionConfig) -> int:
    return cfg._bytes[1]


@_on_device
def attention_forward(cfg: AttentionConfig, q, k, v, *, lengths=None, out=None, lse=None,
                      workspace=None):
    """Runs e2ttt_attn_forward on the current stream: attention of q [B, H, T, d]
    over k, v [B, HK, S, d] (any strides with a contiguous last dimension) over
    the first lengths [B] (int32) tokens of each sequence.  Returns (out, lse);
    out has q's order in memory, lse [B, H, T] is float32."""
    d, io, s_q, s_k, s_l = cfg._call
    dev = q.get_device()
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = q.new_empty(s_l, dtype=torch.float32)
    st = _layout(AttentionStrides, dev, ("q", q, s_q, io), ("k", k, s_k, io), ("v", v, s_k, io),
                 ("out", out, s_q, io))
    _plain("lse", lse, s_l, torch.float32, dev)
    _plain("lengths", lengths, s_l[:1], torch.int32, dev)
    _buffer("workspace", workspace, dev)
    if workspace is None:
        n = cfg._bytes[0]
        workspace = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    st = (_lib or load()).e2ttt_attn_forward(
        d, st, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(lengths), out.data_ptr(),
        lse.data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream())
    if st:
        _check(st, "e2ttt_attn_forward")
    return out, lse


def _run_attention_backward(cfg, st, q, k, v, out, lse, d_out, d_lse, lengths, g, scratch):
    """The library's call on checked tensors (st: their strides argument)."""
    if scratch is None:
        scratch = torch.empty(cfg._bytes[1], dtype=torch.uint8, device=q.device)
    st = (_lib or load()).e2ttt_attn_backward(
        cfg._call[0], st, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(lengths), out.data_ptr(),
        lse.data_ptr(), d_out.data_ptr(), _ptr(d_lse), g["dq"].data_ptr(), g["dk"].data_ptr(),
        g["dv"].data_ptr(), scratch.data_ptr(), scratch.numel(), _stream())
    if st:
        _check(st, "e2ttt_attn_backward")
    return g


@_on_device
def attention_backward(cfg: AttentionConfig, q, k, v, out, lse, d_out, d_lse=None, *, lengths=None,
                       grads=None, scratch=None):
    """Runs e2ttt_attn_backward with the outputs of attention_forward; returns a
    dict of gradients (dq, dk, dv)."""
    d, io, s_q, s_k, s_l = cfg._call
    dev = q.get_device()
    g = grads if grads is not None else dict(dq=_like(q), dk=_like(k), dv=_like(v))
    st = _layout(AttentionStrides, dev, ("q", q, s_q, io), ("k", k, s_k, io), ("v", v, s_k, io),
                 ("out", out, s_q, io), ("d_out", d_out, s_q, io), ("dq", g["dq"], s_q, io),
                 ("dk", g["dk"], s_k, io), ("dv", g["dv"], s_k, io))
    _plain("lse", lse, s_l, torch.float32, dev)
    _plain("d_lse", d_lse, s_l, torch.float32, dev)
    _plain("lengths", lengths, s_l[:1], torch.int32, dev)
    _buffer("scratch", scratch, dev)
    return _run_attention_backward(cfg, st, q, k, v, out, lse, d_out, d_lse, lengths, g, scratch)


def _like(t):
    """A new tensor of t's order in memory, or C order where t repeats elements."""
    x = torch.empty_like(t)
    return x if x.stride(-1) == 1 else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _capturing(t):
    """Whether the current stream of t's device is being captured into a graph."""
    dev = t.get_device() if isinstance(t, torch.Tensor) else -1
    if dev < 0 or dev == _current_device():
        return dev >= 0 and torch.cuda.is_current_stream_capturing()
    with torch.cuda.device(t.device):
        return torch.cuda.is_current_stream_capturing()


def _no_capture(t):
    if _capturing(t):
        raise RuntimeError("AttentionFunction does not take part in a graph capture: "
                           "capture attention_forward and attention_backward instead")


class AttentionFunction(torch.autograd.Function):
    """Autograd wrapper of attention: (out, lse) of (cfg, q, k, v, lengths).  A step to be
    captured into a graph calls attention_forward and attention_backward; here a capture
    that wants gradients raises RuntimeError (torch ties a capture of its own backward to
    the stream of any eager step of the same leaves that is still alive, and ends the
    process; whether there is one cannot be seen from here)."""

    @classmethod
    def apply(cls, cfg, q, k, v, lengths=None):
        if torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad
                                           for t in (q, k, v)):
            _no_capture(q)
        return super().apply(cfg, q, k, v, lengths)

    @staticmethod
    def forward(ctx, cfg, q, k, v, lengths=None):
        out, lse = attention_forward(cfg, q, k, v, lengths=lengths)
        ctx.cfg = cfg
        ctx.flat = q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
        ctx.save_for_backward(q, k, v, lengths, out, lse)
        ctx.set_materialize_grads(False)
        return out, lse

    @staticmethod
    def backward(ctx, d_out, d_lse):
        _no_capture(d_lse if d_out is None else d_out)
        return _once(_attention_grads, ctx, d_out, d_lse)


def _attention_grads(ctx, d_out, d_lse):
    cfg = ctx.cfg
    q, k, v, lengths, out, lse = ctx.saved_tensors
    d_out = torch.zeros_like(out) if d_out is None else _as_rows(d_out)
    if d_lse is not None:
        d_lse = d_lse.contiguous()
    _, io, s_q, _, _ = cfg._call
    dev = q.get_device()
    if ctx.flat and dev == _current_device() and _flat(d_out, s_q, io, dev):
        # (the rest was checked by the forward; d_lse is of lse's type and shape)
        g = _run_attention_backward(cfg, None, q, k, v, out, lse, d_out, d_lse, lengths,
                                    dict(dq=torch.empty_like(q), dk=torch.empty_like(k),
                                         dv=torch.empty_like(v)), None)
    else:
        g = attention_backward(cfg, q, k, v, out, lse, d_out, d_lse, lengths=lengths)
    return None, g["dq"], g["dk"], g["dv"], None


# ------------------------------------------------------------ cache in 4 bits
@dataclass(frozen=True)
class CacheConfig:
    """Calls of T tokens on a cache of 4 bits: pages of 64 tokens, `pages` of them in
    a sequence's row of the table; HK key heads, H query heads (attention alone)
    whose tokens see themselves and `left` tokens before (negative: all)."""
    B: int
    HK: int
    H: int
    T: int
    d: int
    pages: int
    io: int = DT_BF16
    scale: float = 1.0
    left: int = -1

    def desc(self) -> CacheDesc:
        return CacheDesc(self.B, self.HK, self.H, self.T, self.d, self.pages, self.io, self.scale,
                         self.left)

    @cached_property
    def _call(self):
        """The descriptor by reference, the io type and the tensors' shapes."""
        return (ctypes.byref(self.desc()), torch.bfloat16 if self.io == DT_BF16 else torch.float32,
                torch.Size((self.B, self.H, self.T, self.d)),
                torch.Size((self.B, self.HK, self.T, self.d)), torch.Size((self.B, self.pages)),
                torch.Size((self.B,)), torch.Size((self.HK, 68 * self.d)))

    def __getstate__(self):
        return {n: v for n, v in self.__dict__.items() if n != "_call"}


def cache_page_bytes(HK: int, d: int) -> int:
    return int((_lib or load()).e2ttt_cache_page_bytes(HK, d))


def alloc_cache(cfg: CacheConfig, n_pages: int, device="cuda"):
    """A pool of empty pages [n_pages, HK, 68 d] (uint8)."""
    if not cache_page_bytes(cfg.HK, cfg.d):
        raise E2TTTError(3, "e2ttt_cache_page_bytes")
    return torch.zeros((n_pages, cfg.HK, 68 * cfg.d), dtype=torch.uint8, device=device)


def cache_workspace_bytes(cfg: CacheConfig) -> int:
    return int((_lib or load()).e2ttt_cache_workspace_bytes(cfg._call[0]))


def alloc_cache_workspace(cfg: CacheConfig, device="cuda"):
    n = cache_workspace_bytes(cfg)
    if n == 0:
        raise E2TTTError(3, "e2ttt_cache_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _cache_common(cfg, dev, cache, table, starts, lengths):
    """Checks what every cache call has; the number of pages."""
    s_t, s_b, s_page = cfg._call[4:]
    if not isinstance(cache, torch.Tensor) or cache.dim() != 3 or not 1 <= cache.shape[0] < 1 << 31:
        raise ValueError("cache must be a tensor [n_pages, HK, 68 d] of bytes")
    n = cache.shape[0]
    if not _flat(cache, (n, *s_page), torch.uint8, dev):
        _plain("cache", cache, (n, *s_page), torch.uint8, dev)
    if table is None:
        raise ValueError("table must be a tensor")
    if not _flat(table, s_t, torch.int32, dev):
        _plain("table", table, s_t, torch.int32, dev)
    if starts is not None and not _flat(starts, s_b, torch.int32, dev):
        _plain("starts", starts, s_b, torch.int32, dev)
    if lengths is not None:
        _plain("lengths", lengths, s_b, torch.int32, dev)
    return n


def cache_write(cfg: CacheConfig, k, v, cache, table, starts=None, lengths=None):
    """Runs e2ttt_cache_write on the current stream: the first lengths [B] (int32;
    None: all T) tokens of k, v [B, HK, T, d] (any strides with a contiguous last
    dimension) become positions starts [B] (int32; None: 0) + t of their
    sequences, in the pages of cache that table [B, pages] (int32) names."""
    dev = _device_of(k)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return cache_write(cfg, k, v, cache, table, starts, lengths)
    d, io, _, s_k, _, _, _ = cfg._call
    st = None        # (_layout's answer, for a call of a few microseconds)
    if not (_flat(k, s_k, io, dev) and _flat(v, s_k, io, dev)):
        st = _layout(CacheStrides, dev, ("k", k, s_k, io), ("v", v, s_k, io))
    n = _cache_common(cfg, dev, cache, table, starts, lengths)
    st = (_lib or load()).e2ttt_cache_write(d, st, k.data_ptr(), v.data_ptr(), _ptr(starts),
                                            _ptr(lengths), table.data_ptr(), cache.data_ptr(), n,
                                            _stream())
    if st:
        _check(st, "e2ttt_cache_write")


def cache_read(cfg: CacheConfig, cache, table, starts=None, lengths=None, *, out=None):
    """Runs e2ttt_cache_read on the current stream: the values of positions starts +
    t, t < lengths, as (k, v) [B, HK, T, d]; zeros behind them and where the cache
    holds none.  `out`: optional (k, v) tensors to write into, of any strides."""
    dev = _device_of(cache)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return cache_read(cfg, cache, table, starts, lengths, out=out)
    d, io, _, s_k, _, _, _ = cfg._call
    n = _cache_common(cfg, dev, cache, table, starts, lengths)
    if out is None:
        k = torch.empty(s_k, dtype=io, device=cache.device)
        v, st = torch.empty_like(k), None
    else:
        k, v = out
        st = _layout(CacheStrides, dev, ("k", k, s_k, io), ("v", v, s_k, io))
    st = (_lib or load()).e2ttt_cache_read(d, st, _ptr(starts), _ptr(lengths), table.data_ptr(),
                                           cache.data_ptr(), n, k.data_ptr(), v.data_ptr(), _stream())
    if st:
        _check(st, "e2ttt_cache_read")
    return k, v


def cache_attention(cfg: CacheConfig, q, cache, table, starts=None, lengths=None, *, out=None,
                    lse=None, workspace=None):
    """Runs e2ttt_cache_attend on the current stream: attention of the arriving
    tokens' q [B, H, T, d] at positions starts + t over what the cache holds up to
    them, themselves included (cache_write comes first).  Returns (out, lse); lse
    [B, H, T] is written only if given, else None."""
    dev = _device_of(q)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return cache_attention(cfg, q, cache, table, starts, lengths, out=out, lse=lse,
                                   workspace=workspace)
    d, io, s_q, _, _, _, _ = cfg._call
    if out is None:
        out = torch.empty_like(q)
    st = None        # (_layout's answer, for a call of a few microseconds)
    if not (_flat(q, s_q, io, dev) and _flat(out, s_q, io, dev)):
        st = _layout(CacheStrides, dev, ("q", q, s_q, io), ("out", out, s_q, io))
    n = _cache_common(cfg, dev, cache, table, starts, lengths)
    if lse is not None:
        _plain("lse", lse, s_q[:3], torch.float32, dev)
    if workspace is not None:
        _buffer("workspace", workspace, dev)
    else:
        workspace = alloc_cache_workspace(cfg, q.device)
    st = (_lib or load()).e2ttt_cache_attend(
        d, st, q.data_ptr(), _ptr(starts), _ptr(lengths), table.data_ptr(), cache.data_ptr(), n,
        out.data_ptr(), _ptr(lse), workspace.data_ptr(), workspace.numel(), _stream())
    if st:
        _check(st, "e2ttt_cache_attend")
    return out, lse
