"""Thin ctypes binding of the layers around the states (include/stacklstm_layers.h): attention to an encoder's states, log
probabilities of tokens with entropy and best tokens, and dropout, in the same library as the recurrence.

Argument marshalling only, as in ``head.py``, whose conventions hold: every step runs in the HIP library, on the current stream of
the tensors' device, without a host synchronisation. ``AttendRun``, ``LogProbRun`` and ``DropoutRun`` hold a call's output buffers
and work space, which a program keeps from step to step; their inputs may be replaced by others of the same shape, type and
strides. A run's buffers and work space belong to one call at a time: calls on two streams, or two graphs that may run at
once, take a run each.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import Optional

import torch

from . import stacklstm as _sl
from .head import DTYPES, SLSTM_BF16, SLSTM_F32, _arr, _ld, _mat, _type, _ws
from .stacklstm import StackLSTMError, _check, _stream

EXPORTS = ("stacklstm_attend_stats_width", "stacklstm_attend_fwd_workspace_bytes", "stacklstm_attend_bwd_workspace_bytes", "stacklstm_attend_fwd",
           "stacklstm_attend_bwd", "stacklstm_logprob_workspace_bytes", "stacklstm_logprob_fwd", "stacklstm_logprob_bwd",
           "stacklstm_logprob_step", "stacklstm_dropout_fwd", "stacklstm_dropout_bwd")


class slstm_strides(ctypes.Structure):
    _fields_ = [("b", ctypes.c_int64), ("t", ctypes.c_int64), ("h", ctypes.c_int64)]


class slstm_attend_dims(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Tq", ctypes.c_int32), ("Tk", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hk", ctypes.c_int32), ("D", ctypes.c_int32), ("type", ctypes.c_int32), ("scale", ctypes.c_float),
                ("q", slstm_strides), ("k", slstm_strides), ("v", slstm_strides), ("dy", slstm_strides),
                ("y", slstm_strides), ("dq", slstm_strides), ("dk", slstm_strides), ("dv", slstm_strides)]


class slstm_logprob_dims(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("V", ctypes.c_int32), ("G", ctypes.c_int32), ("N", ctypes.c_int32),
                ("type", ctypes.c_int32), ("ld_logits", ctypes.c_int64), ("ld_dlogits", ctypes.c_int64)]


class slstm_dropout_dims(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("width", ctypes.c_int32), ("type", ctypes.c_int32), ("p", ctypes.c_float),
                ("period", ctypes.c_int64), ("ld_x", ctypes.c_int64), ("ld_res", ctypes.c_int64), ("ld_y", ctypes.c_int64)]


_lib = None


def load_library():
    """The library of ``stacklstm.load_library`` with this header's entry points declared."""
    global _lib
    if _lib is None:
        lib = _sl.load_library()
        P, I32, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        dims = {"attend": slstm_attend_dims, "logprob": slstm_logprob_dims, "dropout": slstm_dropout_dims}
        for name in EXPORTS:
            fn, d = getattr(lib, name), ctypes.POINTER(dims[name.split("_")[1]])
            if name.endswith(("_workspace_bytes", "_width")):
                fn.restype, fn.argtypes = SZ if name.endswith("_bytes") else ctypes.c_int32, [d]
                continue
            fn.restype = I32
            fn.argtypes = [d] + {
                "stacklstm_attend_fwd": [P] * 9 + [SZ, P], "stacklstm_attend_bwd": [P] * 13 + [SZ, P],
                "stacklstm_logprob_fwd": [P] * 9 + [SZ, P], "stacklstm_logprob_bwd": [P] * 8,
                "stacklstm_logprob_step": [P] * 11 + [SZ, P], "stacklstm_dropout_fwd": [P] * 5,
                "stacklstm_dropout_bwd": [P] * 4}[name]
        _lib = lib
    return _lib


def _bytes(name, d):
    n = int(getattr(load_library(), name)(ctypes.byref(d)))
    if n == 0:
        raise StackLSTMError(1, name)
    return n


def _space(t):
    """Address and size of a work space."""
    if t is not None and t.dtype is torch.uint8 and t.is_cuda and t.is_contiguous():
        return t.data_ptr(), t.numel()
    return _ws(t)


def _call(name, t, stream, check, *args):
    """The call on t's device (kernels go to the current one), its stream the one given or t's current one."""
    at = t.get_device()
    fn = getattr(_lib or load_library(), name)
    stream = torch._C._cuda_getCurrentRawStream(at) if stream is None else _stream(stream)
    if at == torch.cuda.current_device():
        rc = fn(*args, stream)
    else:
        with torch.cuda.device(at):
            rc = fn(*args, stream)
    if check and rc:
        _check(rc, name)
    return rc


# ----------------------------------------------------------------------------- attention

def strides_of(t):
    """A [B, T, H, D] tensor's strides for the dims; its last axis has to be contiguous. An axis of one element has any stride."""
    if t is None:
        return slstm_strides(0, 0, 0)
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError(f"a matrix of heads is [B, T, H, D] with neighbouring elements of a head, got {tuple(t.shape)} {t.stride()}")
    B, T, H, D = t.shape
    dense = (T * H * D, H * D, D)
    s = [d if n < 2 else v for v, d, n in zip(t.stride(), dense, (B, T, H))]
    if not any(s) and t.numel():
        raise ValueError("a matrix of heads may not be one head for all sequences, places and heads: such strides stand for dense")
    return slstm_strides(*s)


def make_attend_dims(B, Tq, Tk, Hq, Hk, D, type=SLSTM_F32, scale=None, **strides):
    """strides: q, k, v, dy, y, dq, dk, dv, each slstm_strides (dense where left out); scale: 1 / sqrt(D) by default."""
    return slstm_attend_dims(B, Tq, Tk, Hq, Hk, D, type, D ** -0.5 if scale is None and D > 0 else scale or 0.0, **strides)


def stacklstm_attend_stats_width(dims) -> int:
    return int(load_library().stacklstm_attend_stats_width(ctypes.byref(dims)))


def stacklstm_attend_fwd_workspace_bytes(dims) -> int:
    return int(load_library().stacklstm_attend_fwd_workspace_bytes(ctypes.byref(dims)))


def stacklstm_attend_bwd_workspace_bytes(dims) -> int:
    return int(load_library().stacklstm_attend_bwd_workspace_bytes(ctypes.byref(dims)))


def _heads(t, dtype, what, shape, s, optional=False):
    """Address of a [B, T, H, D] device tensor with the strides of the dims."""
    b, n, h = s.b, s.t, s.h
    if t is not None and t.dtype is dtype and t.is_cuda and t.shape == shape and t.stride() == (b, n, h, 1) and (b or n or h):
        return t.data_ptr()                      # (as most are: a small call takes as long as its checks)
    if t is None:
        if optional:
            return None
        raise ValueError(f"{what} is missing")
    if t.dtype is not dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if t.shape != shape:
        raise ValueError(f"{what} must have shape {shape}, got {tuple(t.shape)}")
    B, T, H, D = shape
    want = (b, n, h) if b or n or h else (T * H * D, H * D, D)
    if t.numel() and (any(m > 1 and v != w for v, w, m in zip(t.stride(), want, shape)) or (D > 1 and t.stride(3) != 1)):
        raise ValueError(f"{what} must have strides {want + (1,)}, got {t.stride()}")
    return t.data_ptr()


def _lens(d, q_len, k_len, mask):
    return (None if q_len is None else _arr(q_len, torch.int32, "q_len", (d.B,)),
            None if k_len is None else _arr(k_len, torch.int32, "k_len", (d.B,)),
            None if mask is None else _arr(mask, torch.uint8, "mask", (d.B, d.Tk)))


def _stats(d, stats):
    return _arr(stats, torch.float32, "stats", (d.B, d.Hq, d.Tq, stacklstm_attend_stats_width(d)))


def stacklstm_attend_fwd(dims, q, k, v, q_len, k_len, mask, y, stats, workspace, stream=None, check=True) -> int:
    d, t = dims, DTYPES[dims.type]
    sq, sk = (d.B, d.Tq, d.Hq, d.D), (d.B, d.Tk, d.Hk, d.D)
    ws, n = _space(workspace)
    return _call("stacklstm_attend_fwd", q, stream, check, d, _heads(q, t, "q", sq, d.q), _heads(k, t, "k", sk, d.k),
                 _heads(v, t, "v", sk, d.v), *_lens(d, q_len, k_len, mask), _heads(y, t, "y", sq, d.y),
                 None if stats is None else _stats(d, stats), ws, n)


def stacklstm_attend_bwd(dims, q, k, v, q_len, k_len, mask, y, stats, dy, dq, dk, dv, workspace, stream=None, check=True) -> int:
    d, t = dims, DTYPES[dims.type]
    sq, sk = (d.B, d.Tq, d.Hq, d.D), (d.B, d.Tk, d.Hk, d.D)
    ws, n = _space(workspace)
    return _call("stacklstm_attend_bwd", q, stream, check, d, _heads(q, t, "q", sq, d.q), _heads(k, t, "k", sk, d.k),
                 _heads(v, t, "v", sk, d.v), *_lens(d, q_len, k_len, mask), _heads(y, t, "y", sq, d.y),
                 _stats(d, stats), _heads(dy, t, "dy", sq, d.dy),
                 _heads(dq, t, "dq", sq, d.dq), _heads(dk, t, "dk", sk, d.dk), _heads(dv, t, "dv", sk, d.dv), ws, n)


def _like(t):
    """An output buffer with the order of t's axes (a [T, B, ...] tensor seen as [B, T, ...] gives another such)."""
    order = sorted(range(3), key=lambda i: (-t.stride(i), i)) + [3]
    return torch.empty([t.shape[i] for i in order], dtype=t.dtype, device=t.device).permute([order.index(i) for i in range(4)])


@dataclass
class AttendRun:
    """Queries attend to keys and values of another length, and the backward: inputs, output buffers, work space."""
    dims: slstm_attend_dims
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    q_len: Optional[torch.Tensor]
    k_len: Optional[torch.Tensor]
    mask: Optional[torch.Tensor]
    dy: Optional[torch.Tensor]
    y: torch.Tensor
    stats: Optional[torch.Tensor]
    dq: Optional[torch.Tensor]
    dk: Optional[torch.Tensor]
    dv: Optional[torch.Tensor]
    workspace: torch.Tensor

    @classmethod
    def of(cls, q, k, v, q_len=None, k_len=None, mask=None, scale=None, dy=None, y=None, train=None):
        """q [B, Tq, Hq, D], k and v [B, Tk, Hk, D], any strides with neighbouring elements of a head (not 0 for all three axes); y: where the outputs go (by
        default a buffer of its own in the order of q's axes); scale: 1 / sqrt(D) by default; train: buffers for a backward too
        (by default where dy is given; a dy that is set later has the strides of y)."""
        (B, Tq, Hq, D), (Tk, Hk) = q.shape, k.shape[1:3]
        train = dy is not None if train is None else train
        y = _like(q) if y is None else y
        grads = [_like(t) for t in (q, k, v)] if train else [None] * 3
        s = dict(zip(("dq", "dk", "dv"), map(strides_of, grads)))
        d = make_attend_dims(B, Tq, Tk, Hq, Hk, D, _type(q), scale, q=strides_of(q), k=strides_of(k), v=strides_of(v),
                             y=strides_of(y), dy=strides_of(y if dy is None else dy), **s)
        n = _bytes("stacklstm_attend_fwd_workspace_bytes", d)
        if train:
            n = max(n, _bytes("stacklstm_attend_bwd_workspace_bytes", d))
        e = lambda *s, dtype: torch.empty(*s, dtype=dtype, device=q.device)
        return cls(d, q, k, v, q_len, k_len, mask, dy, y, e(B, Hq, Tq, stacklstm_attend_stats_width(d), dtype=torch.float32) if train else None, *grads,
                   e(n, dtype=torch.uint8))

    def forward(self, stream=None):
        stacklstm_attend_fwd(self.dims, self.q, self.k, self.v, self.q_len, self.k_len, self.mask, self.y, self.stats,
                             self.workspace, stream)
        return self.y

    def backward(self, stream=None):
        stacklstm_attend_bwd(self.dims, self.q, self.k, self.v, self.q_len, self.k_len, self.mask, self.y, self.stats, self.dy,
                             self.dq, self.dk, self.dv, self.workspace, stream)
        return self.dq


# ----------------------------------------------------------------------------- log probabilities

def make_logprob_dims(rows, V, G=1, N=0, type=SLSTM_F32, ld_logits=0, ld_dlogits=0):
    return slstm_logprob_dims(rows, V, G, N, type, ld_logits, ld_dlogits)


def stacklstm_logprob_workspace_bytes(dims) -> int:
    return int(load_library().stacklstm_logprob_workspace_bytes(ctypes.byref(dims)))


def _rows_in(d, logits, legal, token):
    return (_mat(logits, DTYPES[d.type], "logits", d.rows, d.V, d.ld_logits),
            _arr(legal, torch.uint8, "legal", (d.rows, d.V), True), _arr(token, torch.int32, "token", (d.rows, d.G), d.G == 0))


def _rows_out(d, logp, entropy, index, value):
    f = torch.float32
    return (_arr(logp, f, "logp", (d.rows, d.G), d.G == 0), _arr(entropy, f, "entropy", (d.rows,), True),
            _arr(index, torch.int32, "index", (d.rows, d.N), d.N == 0), _arr(value, f, "value", (d.rows, d.N), d.N == 0))


def _rows_grad(d, dlogp, dentropy):
    return (_arr(dlogp, torch.float32, "dlogp", (d.rows, d.G), True), _arr(dentropy, torch.float32, "dentropy", (d.rows,), True))


def stacklstm_logprob_fwd(dims, logits, legal, token, logp, entropy, index, value, stats, workspace, stream=None, check=True) -> int:
    ws, n = _space(workspace)
    return _call("stacklstm_logprob_fwd", logits, stream, check, dims, *_rows_in(dims, logits, legal, token),
                 *_rows_out(dims, logp, entropy, index, value), _arr(stats, torch.float32, "stats", (dims.rows, 3), True), ws, n)


def stacklstm_logprob_bwd(dims, logits, legal, token, stats, dlogp, dentropy, dlogits, stream=None, check=True) -> int:
    return _call("stacklstm_logprob_bwd", logits, stream, check, dims, *_rows_in(dims, logits, legal, token),
                 _arr(stats, torch.float32, "stats", (dims.rows, 3)), *_rows_grad(dims, dlogp, dentropy),
                 _mat(dlogits, DTYPES[dims.type], "dlogits", dims.rows, dims.V, dims.ld_dlogits))


def stacklstm_logprob_step(dims, logits, legal, token, dlogp, dentropy, logp, entropy, index, value, dlogits, workspace,
                           stream=None, check=True) -> int:
    ws, n = _space(workspace)
    return _call("stacklstm_logprob_step", logits, stream, check, dims, *_rows_in(dims, logits, legal, token),
                 *_rows_grad(dims, dlogp, dentropy), *_rows_out(dims, logp, entropy, index, value),
                 _mat(dlogits, DTYPES[dims.type], "dlogits", dims.rows, dims.V, dims.ld_dlogits), ws, n)


@dataclass
class LogProbRun:
    """Log probabilities of given tokens, entropy and best tokens of rows of logits, and the logits' gradient. The best tokens
    (index, value) are what ``head.DistillRun`` takes from a teacher."""
    dims: slstm_logprob_dims
    logits: torch.Tensor
    token: Optional[torch.Tensor]
    legal: Optional[torch.Tensor]
    dlogp: Optional[torch.Tensor]
    dentropy: Optional[torch.Tensor]
    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    index: Optional[torch.Tensor]
    value: Optional[torch.Tensor]
    stats: torch.Tensor
    dlogits: Optional[torch.Tensor]
    workspace: torch.Tensor

    @classmethod
    def of(cls, logits, token=None, legal=None, top=0, dlogp=None, dentropy=None, dlogits=None, train=None):
        """token [rows, G] int32; top: how many best tokens; dlogits: where the gradient goes (by default a buffer of its own where
        dlogp or dentropy is given, or with train; logits itself is allowed)."""
        R, V = logits.shape
        train = (dlogp is not None or dentropy is not None) if train is None else train
        if train and dlogits is None:
            dlogits = torch.empty(R, V, dtype=logits.dtype, device=logits.device)
        G = 0 if token is None else token.shape[1]
        d = make_logprob_dims(R, V, G, top, _type(logits), _ld(logits), _ld(dlogits))
        e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device=logits.device)
        return cls(d, logits, token, legal, dlogp, dentropy, e(R, G) if G else None, e(R), e(R, top, dtype=torch.int32) if top else None,
                   e(R, top) if top else None, e(R, 3), dlogits, e(_bytes("stacklstm_logprob_workspace_bytes", d), dtype=torch.uint8))

    def forward(self, stream=None):
        stacklstm_logprob_fwd(self.dims, self.logits, self.legal, self.token, self.logp, self.entropy, self.index, self.value,
                              self.stats, self.workspace, stream)
        return self.logp

    def backward(self, stream=None):
        stacklstm_logprob_bwd(self.dims, self.logits, self.legal, self.token, self.stats, self.dlogp, self.dentropy, self.dlogits,
                              stream)
        return self.dlogits

    def step(self, stream=None):
        """Outputs and gradient in one pass."""
        stacklstm_logprob_step(self.dims, self.logits, self.legal, self.token, self.dlogp, self.dentropy, self.logp, self.entropy,
                               self.index, self.value, self.dlogits, self.workspace, stream)
        return self.logp


# ----------------------------------------------------------------------------- dropout

def make_dropout_dims(rows, width, type=SLSTM_F32, p=0.1, period=0, ld_x=0, ld_res=0, ld_y=0):
    return slstm_dropout_dims(rows, width, type, p, period, ld_x, ld_res, ld_y)


def stacklstm_dropout_fwd(dims, x, res, seed, y, stream=None, check=True) -> int:
    R, W, t = dims.rows, dims.width, DTYPES[dims.type]
    return _call("stacklstm_dropout_fwd", x, stream, check, dims, _mat(x, t, "x", R, W, dims.ld_x),
                 _mat(res, t, "res", R, W, dims.ld_res, True), _arr(seed, torch.int64, "seed", (2,)), _mat(y, t, "y", R, W, dims.ld_y))


def stacklstm_dropout_bwd(dims, dy, seed, dx, stream=None, check=True) -> int:
    R, W, t = dims.rows, dims.width, DTYPES[dims.type]
    return _call("stacklstm_dropout_bwd", dy, stream, check, dims, _mat(dy, t, "dy", R, W, dims.ld_x),
                 _arr(seed, torch.int64, "seed", (2,)), _mat(dx, t, "dx", R, W, dims.ld_y))


@dataclass
class DropoutRun:
    """y = dropout(x) + res and its backward: inputs and output buffers. seed [2] int64 on the device: a key and a step (add 1 to
    seed[1] for the next mask; a captured graph takes whatever is there when it runs)."""
    dims: slstm_dropout_dims
    x: torch.Tensor
    seed: torch.Tensor
    res: Optional[torch.Tensor]
    dy: Optional[torch.Tensor]
    y: torch.Tensor
    dx: Optional[torch.Tensor]
    bwd_dims: Optional[slstm_dropout_dims]

    @classmethod
    def of(cls, x, p, seed, res=None, period=0, dy=None, y=None, train=None):
        """period: row r has the mask of row r % period (0: its own); y: where the outputs go (by default a buffer of its own; x or
        res itself is allowed); train: as in AttendRun.of (a dy that is set later is dense)."""
        R, W = x.shape
        train = dy is not None if train is None else train
        e = lambda: torch.empty(R, W, dtype=x.dtype, device=x.device)
        y = e() if y is None else y
        d = make_dropout_dims(R, W, _type(x), p, period, _ld(x), _ld(res), _ld(y))
        return cls(d, x, seed, res, dy, y, e() if train else None,
                   make_dropout_dims(R, W, d.type, p, period, _ld(dy)) if train else None)

    def forward(self, stream=None):
        stacklstm_dropout_fwd(self.dims, self.x, self.res, self.seed, self.y, stream)
        return self.y

    def backward(self, stream=None):
        stacklstm_dropout_bwd(self.bwd_dims, self.dy, self.seed, self.dx, stream)
        return self.dx
