"""Thin ctypes binding of the operators between the states and the answers (include/stacklstm_head.h):
layer norm, linear layer, distillation loss and beam search, in the same library as the recurrence.

Argument marshalling only, as in ``stacklstm.py``: every step runs in the HIP library, on the current stream
of the tensors' device, without a host synchronisation. The functions take the C calls' arguments in
their order; matrices with a stride in the dims may be views whose rows are apart, everything else is contiguous.
``NormRun``, ``LinearRun``, ``DistillRun`` and ``BeamRun`` hold a call's output buffers and work space, which a program keeps
from step to step; their inputs may be replaced by others of the same shape, type and strides.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass, field
from typing import Optional

import torch

from . import stacklstm as _sl
from .stacklstm import StackLSTMError, _check, _stream

SLSTM_F32, SLSTM_BF16 = 0, 1
TYPES = {torch.float32: SLSTM_F32, torch.bfloat16: SLSTM_BF16}
DTYPES = {SLSTM_F32: torch.float32, SLSTM_BF16: torch.bfloat16}
ACTS = {"none": 0, "relu": 1, "tanh": 2, "silu": 3, "gelu": 4}
SLSTM_LINEAR_WIDE_DZ = 0x100
SLSTM_BEAM_MAX_STATES = 8
EXPORTS = ("stacklstm_norm_workspace_bytes", "stacklstm_norm_fwd", "stacklstm_norm_bwd",
           "stacklstm_linear_fwd_workspace_bytes", "stacklstm_linear_bwd_workspace_bytes", "stacklstm_linear_fwd",
           "stacklstm_linear_bwd", "stacklstm_distill_workspace_bytes", "stacklstm_distill_fwd", "stacklstm_distill_bwd",
           "stacklstm_distill_step", "stacklstm_beam_workspace_bytes", "stacklstm_beam_select", "stacklstm_beam_reorder")


class slstm_norm_dims(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("width", ctypes.c_int32), ("type", ctypes.c_int32), ("eps", ctypes.c_float),
                ("ld_x", ctypes.c_int64), ("ld_res", ctypes.c_int64), ("ld_dy", ctypes.c_int64)]


class slstm_linear_dims(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("K", ctypes.c_int32), ("N", ctypes.c_int32), ("type", ctypes.c_int32),
                ("act", ctypes.c_int32), ("ld_x", ctypes.c_int64), ("ld_w", ctypes.c_int64), ("ld_res", ctypes.c_int64),
                ("ld_y", ctypes.c_int64), ("ld_dy", ctypes.c_int64)]


class slstm_distill_dims(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("V", ctypes.c_int32), ("K", ctypes.c_int32), ("type", ctypes.c_int32),
                ("tau", ctypes.c_float), ("alpha", ctypes.c_float), ("ld_logits", ctypes.c_int64),
                ("ld_dlogits", ctypes.c_int64)]


class slstm_beam_dims(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("K", ctypes.c_int32), ("V", ctypes.c_int32), ("type", ctypes.c_int32),
                ("eos", ctypes.c_int32), ("ld_logits", ctypes.c_int64)]


class slstm_beam_state(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("slot_bytes", ctypes.c_int64),
                ("slots", ctypes.c_int32), ("reserved", ctypes.c_int32), ("live", ctypes.c_void_p)]


_lib = None


def load_library():
    """The library of ``stacklstm.load_library`` with this header's entry points declared."""
    global _lib
    if _lib is None:
        lib = _sl.load_library()
        P, I32, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        dims = {"norm": slstm_norm_dims, "linear": slstm_linear_dims, "distill": slstm_distill_dims, "beam": slstm_beam_dims}
        for name in EXPORTS:
            fn, d = getattr(lib, name), ctypes.POINTER(dims[name.split("_")[1]])
            if name.endswith("_workspace_bytes"):
                fn.restype, fn.argtypes = SZ, [d]
                continue
            fn.restype = I32
            fn.argtypes = [d] + {
                "stacklstm_norm_fwd": [P] * 8 + [P], "stacklstm_norm_bwd": [P] * 10 + [SZ, P],
                "stacklstm_linear_fwd": [P] * 7 + [SZ, P], "stacklstm_linear_bwd": [P] * 8 + [SZ, P],
                "stacklstm_distill_fwd": [P] * 7 + [SZ, P], "stacklstm_distill_bwd": [P] * 7 + [P],
                "stacklstm_distill_step": [P] * 8 + [SZ, P], "stacklstm_beam_select": [P] * 9 + [SZ, P],
                "stacklstm_beam_reorder": [P, ctypes.POINTER(slstm_beam_state), ctypes.c_int32, P]}[name]
        _lib = lib
    return _lib


# ----------------------------------------------------------------------------- argument checks

def _arr(t, dtype, what, shape, optional=False):
    """Address of a contiguous device tensor of this type and shape."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{what} is missing")
    if t.dtype is dtype and t.is_cuda and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    if t.dtype is not dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if t.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{what} must be contiguous")


def _mat(t, dtype, what, rows, cols, ld, optional=False):
    """Address of a [rows, cols] device tensor whose rows are ld elements apart (0: cols)."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{what} is missing")
    if t.dtype is dtype and t.is_cuda and t.shape == (rows, cols):
        s0, s1 = t.stride()
        if (s1 == 1 or cols == 1) and (s0 == (ld or cols) or rows < 2):
            return t.data_ptr()
        raise ValueError(f"{what} must have strides {(ld or cols, 1)}, got {(s0, s1)}")
    if t.dtype is not dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    raise ValueError(f"{what} must have shape {(rows, cols)}, got {tuple(t.shape)}")


def _ld(t):
    """Row stride of a matrix for the dims (0: dense)."""
    return 0 if t is None or t.dim() != 2 or t.shape[0] < 2 or t.stride(0) == t.shape[1] else t.stride(0)


def _ws(t):
    if t is None:
        return None, 0
    return _arr(t, torch.uint8, "workspace", (t.numel(),)), t.numel()


def _type(t):
    if t.dtype not in TYPES:
        raise ValueError(f"tensors are float32 or bfloat16, got {t.dtype}")
    return TYPES[t.dtype]


def _here(stream, t):
    """The stream given, or the current one of the tensor's device (its raw handle: the stream object of
    torch.cuda.current_stream takes 2 us to make, a third of a small call)."""
    return torch._C._cuda_getCurrentRawStream(t.get_device()) if stream is None else _stream(stream)


def _bytes(name, d):
    n = int(getattr(load_library(), name)(ctypes.byref(d)))
    if n == 0:
        raise StackLSTMError(1, name)
    return n


# ----------------------------------------------------------------------------- layer norm

def make_norm_dims(rows, width, type=SLSTM_F32, eps=1e-5, ld_x=0, ld_res=0, ld_dy=0):
    return slstm_norm_dims(rows, width, type, eps, ld_x, ld_res, ld_dy)


def stacklstm_norm_workspace_bytes(dims) -> int:
    return int(load_library().stacklstm_norm_workspace_bytes(ctypes.byref(dims)))


def stacklstm_norm_fwd(dims, x, res, gamma, beta, sum, y, mean, rstd, stream=None, check=True) -> int:
    R, W, t, f = dims.rows, dims.width, DTYPES[dims.type], torch.float32
    rc = load_library().stacklstm_norm_fwd(
        dims, _mat(x, t, "x", R, W, dims.ld_x), _mat(res, t, "res", R, W, dims.ld_res, True),
        _arr(gamma, f, "gamma", (W,), True), _arr(beta, f, "beta", (W,), True), _arr(sum, t, "sum", (R, W), True),
        _arr(y, t, "y", (R, W)), _arr(mean, f, "mean", (R,), True), _arr(rstd, f, "rstd", (R,), True), _here(stream, x))
    if check:
        _check(rc, "stacklstm_norm_fwd")
    return rc


def stacklstm_norm_bwd(dims, x, gamma, mean, rstd, dy, dsum, dx, dgamma, dbeta, workspace, stream=None, check=True) -> int:
    R, W, t, f = dims.rows, dims.width, DTYPES[dims.type], torch.float32
    ws, n = _ws(workspace)
    rc = load_library().stacklstm_norm_bwd(
        dims, _mat(x, t, "x", R, W, dims.ld_x), _arr(gamma, f, "gamma", (W,), True), _arr(mean, f, "mean", (R,)),
        _arr(rstd, f, "rstd", (R,)), _mat(dy, t, "dy", R, W, dims.ld_dy), _arr(dsum, t, "dsum", (R, W), True),
        _arr(dx, t, "dx", (R, W)), _arr(dgamma, f, "dgamma", (W,), True), _arr(dbeta, f, "dbeta", (W,), True), ws, n,
        _here(stream, x))
    if check:
        _check(rc, "stacklstm_norm_bwd")
    return rc


@dataclass
class NormRun:
    """y = norm(x + res) gamma + beta and its backward: inputs, output buffers, work space."""
    dims: slstm_norm_dims
    x: torch.Tensor
    gamma: Optional[torch.Tensor]
    beta: Optional[torch.Tensor]
    res: Optional[torch.Tensor]
    dy: Optional[torch.Tensor]
    dsum: Optional[torch.Tensor]
    sum: Optional[torch.Tensor]
    y: torch.Tensor
    mean: Optional[torch.Tensor]
    rstd: Optional[torch.Tensor]
    dx: Optional[torch.Tensor]
    dgamma: Optional[torch.Tensor]
    dbeta: Optional[torch.Tensor]
    workspace: Optional[torch.Tensor]
    bwd_dims: Optional[slstm_norm_dims]

    @classmethod
    def of(cls, x, gamma=None, beta=None, res=None, dy=None, dsum=None, eps=1e-5, train=None):
        """train: buffers for a backward too (by default where dy is given; dy may be set later)."""
        R, W = x.shape
        train = dy is not None if train is None else train
        d = make_norm_dims(R, W, _type(x), eps, _ld(x), _ld(res), _ld(dy))
        e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device=x.device)
        n = _bytes("stacklstm_norm_workspace_bytes", d)
        # the backward reads the sum, which is dense
        bd = make_norm_dims(R, W, d.type, eps, 0 if res is not None else d.ld_x, 0, d.ld_dy) if train else None
        return cls(dims=d, x=x, gamma=gamma, beta=beta, res=res, dy=dy, dsum=dsum,
                   sum=e(R, W, dtype=x.dtype) if res is not None else None, y=e(R, W, dtype=x.dtype),
                   mean=e(R) if train else None, rstd=e(R) if train else None, dx=e(R, W, dtype=x.dtype) if train else None,
                   dgamma=e(W) if train and gamma is not None else None, dbeta=e(W) if train and beta is not None else None,
                   workspace=e(n, dtype=torch.uint8) if train else None, bwd_dims=bd)

    def forward(self, stream=None):
        stacklstm_norm_fwd(self.dims, self.x, self.res, self.gamma, self.beta, self.sum, self.y, self.mean, self.rstd, stream)
        return self.y

    def backward(self, stream=None):
        stacklstm_norm_bwd(self.bwd_dims, self.x if self.res is None else self.sum, self.gamma, self.mean, self.rstd, self.dy,
                           self.dsum, self.dx, self.dgamma, self.dbeta, self.workspace, stream)
        return self.dx


# ----------------------------------------------------------------------------- linear layer

def make_linear_dims(M, K, N, type=SLSTM_F32, act=0, ld_x=0, ld_w=0, ld_res=0, ld_y=0, ld_dy=0):
    return slstm_linear_dims(M, K, N, type, act, ld_x, ld_w, ld_res, ld_y, ld_dy)


def stacklstm_linear_fwd_workspace_bytes(dims) -> int:
    return int(load_library().stacklstm_linear_fwd_workspace_bytes(ctypes.byref(dims)))


def stacklstm_linear_bwd_workspace_bytes(dims) -> int:
    return int(load_library().stacklstm_linear_bwd_workspace_bytes(ctypes.byref(dims)))


def stacklstm_linear_fwd(dims, x, W, b, res, y, z, workspace, stream=None, check=True) -> int:
    M, K, N, t = dims.M, dims.K, dims.N, DTYPES[dims.type]
    ws, n = _ws(workspace)
    rc = load_library().stacklstm_linear_fwd(
        dims, _mat(x, t, "x", M, K, dims.ld_x), _mat(W, t, "W", K, N, dims.ld_w), _arr(b, t, "b", (N,), True),
        _mat(res, t, "res", M, N, dims.ld_res, True), _mat(y, t, "y", M, N, dims.ld_y), _arr(z, t, "z", (M, N), True), ws, n,
        _here(stream, x))
    if check:
        _check(rc, "stacklstm_linear_fwd")
    return rc


def stacklstm_linear_bwd(dims, x, W, z, dy, dx, dW, db, workspace, stream=None, check=True) -> int:
    M, K, N, t = dims.M, dims.K, dims.N, DTYPES[dims.type]
    ws, n = _ws(workspace)
    rc = load_library().stacklstm_linear_bwd(
        dims, _mat(x, t, "x", M, K, dims.ld_x, True), _mat(W, t, "W", K, N, dims.ld_w, True), _arr(z, t, "z", (M, N), True),
        _mat(dy, t, "dy", M, N, dims.ld_dy), _arr(dx, t, "dx", (M, K), True), _arr(dW, t, "dW", (K, N), True),
        _arr(db, t, "db", (N,), True), ws, n, _here(stream, dy))
    if check:
        _check(rc, "stacklstm_linear_bwd")
    return rc


@dataclass
class LinearRun:
    """y = act(x W + b) + res and its backward: inputs, output buffers, work space."""
    dims: slstm_linear_dims
    x: torch.Tensor
    W: torch.Tensor
    b: Optional[torch.Tensor]
    res: Optional[torch.Tensor]
    dy: Optional[torch.Tensor]
    y: torch.Tensor
    z: Optional[torch.Tensor]
    dx: Optional[torch.Tensor]
    dW: Optional[torch.Tensor]
    db: Optional[torch.Tensor]
    workspace: torch.Tensor

    @classmethod
    def of(cls, x, W, b=None, res=None, act="none", dy=None, y=None, train=None, wide_dz=False):
        """y: where the outputs go (by default a buffer of its own); train: as in NormRun.of; wide_dz: the backward's 16-bit
        products take dz with 16 significant bits, for twice their time."""
        (M, K), N = x.shape, W.shape[1]
        train = dy is not None if train is None else train
        e = lambda *s, dtype=x.dtype: torch.empty(*s, dtype=dtype, device=x.device)
        y = e(M, N) if y is None else y
        d = make_linear_dims(M, K, N, _type(x), ACTS[act] | (SLSTM_LINEAR_WIDE_DZ if wide_dz else 0), _ld(x), _ld(W), _ld(res),
                             _ld(y), _ld(dy))
        n = _bytes("stacklstm_linear_fwd_workspace_bytes", d)
        if train:
            n = max(n, _bytes("stacklstm_linear_bwd_workspace_bytes", d))
        return cls(dims=d, x=x, W=W, b=b, res=res, dy=dy, y=y, z=e(M, N) if train and act != "none" else None,
                   dx=e(M, K) if train else None, dW=e(K, N) if train else None,
                   db=e(N) if train and b is not None else None, workspace=e(n, dtype=torch.uint8))

    def forward(self, stream=None):
        stacklstm_linear_fwd(self.dims, self.x, self.W, self.b, self.res, self.y, self.z, self.workspace, stream)
        return self.y

    def backward(self, stream=None):
        stacklstm_linear_bwd(self.dims, self.x, self.W, self.z, self.dy, self.dx, self.dW, self.db, self.workspace, stream)
        return self.dx


# ----------------------------------------------------------------------------- distillation loss

def make_distill_dims(rows, V, K, type=SLSTM_F32, tau=1.0, alpha=1.0, ld_logits=0, ld_dlogits=0):
    return slstm_distill_dims(rows, V, K, type, tau, alpha, ld_logits, ld_dlogits)


def stacklstm_distill_workspace_bytes(dims) -> int:
    return int(load_library().stacklstm_distill_workspace_bytes(ctypes.byref(dims)))


def _targets(d, index, value, label):
    R, K = d.rows, d.K
    return (_arr(index, torch.int32, "index", (R, K)), _arr(value, torch.float32, "value", (R, K)),
            _arr(label, torch.int32, "label", (R,), True))


def stacklstm_distill_fwd(dims, logits, index, value, label, loss, stats, workspace, stream=None, check=True) -> int:
    R, t, f = dims.rows, DTYPES[dims.type], torch.float32
    ws, n = _ws(workspace)
    rc = load_library().stacklstm_distill_fwd(
        dims, _mat(logits, t, "logits", R, dims.V, dims.ld_logits), *_targets(dims, index, value, label),
        _arr(loss, f, "loss", (R,)), _arr(stats, f, "stats", (R, 3), True), ws, n, _here(stream, logits))
    if check:
        _check(rc, "stacklstm_distill_fwd")
    return rc


def stacklstm_distill_bwd(dims, logits, index, value, label, stats, grad, dlogits, stream=None, check=True) -> int:
    R, t, f = dims.rows, DTYPES[dims.type], torch.float32
    rc = load_library().stacklstm_distill_bwd(
        dims, _mat(logits, t, "logits", R, dims.V, dims.ld_logits), *_targets(dims, index, value, label),
        _arr(stats, f, "stats", (R, 3)), _arr(grad, f, "grad", (R,), True),
        _mat(dlogits, t, "dlogits", R, dims.V, dims.ld_dlogits), _here(stream, logits))
    if check:
        _check(rc, "stacklstm_distill_bwd")
    return rc


def stacklstm_distill_step(dims, logits, index, value, label, grad, loss, dlogits, workspace, stream=None, check=True) -> int:
    R, t, f = dims.rows, DTYPES[dims.type], torch.float32
    ws, n = _ws(workspace)
    rc = load_library().stacklstm_distill_step(
        dims, _mat(logits, t, "logits", R, dims.V, dims.ld_logits), *_targets(dims, index, value, label),
        _arr(grad, f, "grad", (R,), True), _arr(loss, f, "loss", (R,)),
        _mat(dlogits, t, "dlogits", R, dims.V, dims.ld_dlogits), ws, n, _here(stream, logits))
    if check:
        _check(rc, "stacklstm_distill_step")
    return rc


@dataclass
class DistillRun:
    """Loss of logits against a teacher's top logits and labels, and the logits' gradient."""
    dims: slstm_distill_dims
    logits: torch.Tensor
    index: torch.Tensor
    value: torch.Tensor
    label: Optional[torch.Tensor]
    grad: Optional[torch.Tensor]
    loss: torch.Tensor
    stats: torch.Tensor
    dlogits: torch.Tensor
    workspace: torch.Tensor

    @classmethod
    def of(cls, logits, index, value, label=None, grad=None, tau=1.0, alpha=1.0, dlogits=None):
        """dlogits: where the gradient goes (by default a buffer of its own; logits itself is allowed)."""
        R, V = logits.shape
        dlogits = torch.empty(R, V, dtype=logits.dtype, device=logits.device) if dlogits is None else dlogits
        d = make_distill_dims(R, V, index.shape[1], _type(logits), tau, alpha, _ld(logits), _ld(dlogits))
        e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device=logits.device)
        return cls(dims=d, logits=logits, index=index, value=value, label=label, grad=grad, loss=e(R), stats=e(R, 3),
                   dlogits=dlogits, workspace=e(_bytes("stacklstm_distill_workspace_bytes", d), dtype=torch.uint8))

    def step(self, stream=None):
        """Loss and gradient in one pass."""
        stacklstm_distill_step(self.dims, self.logits, self.index, self.value, self.label, self.grad, self.loss, self.dlogits,
                               self.workspace, stream)
        return self.loss

    def forward(self, stream=None):
        stacklstm_distill_fwd(self.dims, self.logits, self.index, self.value, self.label, self.loss, self.stats,
                              self.workspace, stream)
        return self.loss

    def backward(self, stream=None):
        stacklstm_distill_bwd(self.dims, self.logits, self.index, self.value, self.label, self.stats, self.grad, self.dlogits,
                              stream)
        return self.dlogits


# ----------------------------------------------------------------------------- beam search

def make_beam_dims(B, K, V, type=SLSTM_F32, eos=-1, ld_logits=0):
    return slstm_beam_dims(B, K, V, type, eos, ld_logits)


def stacklstm_beam_workspace_bytes(dims) -> int:
    return int(load_library().stacklstm_beam_workspace_bytes(ctypes.byref(dims)))


def stacklstm_beam_select(dims, logits, legal, score, done, score_next, parent, token, done_next, workspace, stream=None,
                          check=True) -> int:
    B, K, V, f, i32, u8 = dims.B, dims.K, dims.V, torch.float32, torch.int32, torch.uint8
    ws, n = _ws(workspace)
    rc = load_library().stacklstm_beam_select(
        dims, _mat(logits, DTYPES[dims.type], "logits", B * K, V, dims.ld_logits), _arr(legal, u8, "legal", (B * K, V), True),
        _arr(score, f, "score", (B, K)), _arr(done, u8, "done", (B, K), True), _arr(score_next, f, "score_next", (B, K)),
        _arr(parent, i32, "parent", (B, K)), _arr(token, i32, "token", (B, K)), _arr(done_next, u8, "done_next", (B, K)), ws, n,
        _here(stream, logits))
    if check:
        _check(rc, "stacklstm_beam_select")
    return rc


def beam_states(dims, states):
    """The C descriptors of [(src, dst, live)]: src and dst [B K, slots, ...] (or [B K]: one slot), live int32 [B K]
    or None. Kept by a caller that reorders the same buffers at every step."""
    rows = dims.B * dims.K
    out = (slstm_beam_state * max(1, len(states)))()
    for s, (src, dst, live) in zip(out, states):
        if src.dtype != dst.dtype or src.shape != dst.shape or src.dim() < 1 or src.shape[0] != rows:
            raise ValueError(f"a state is two tensors of one type and shape [{rows}, ...]")
        s.src, s.dst = _arr(src, src.dtype, "src", src.shape), _arr(dst, src.dtype, "dst", src.shape)
        s.slots = src.shape[1] if src.dim() > 1 else 1
        s.slot_bytes = src.element_size() * (src[0, 0].numel() if src.dim() > 2 else 1) if rows else 1
        s.live = _arr(live, torch.int32, "live", (rows,), True)
    return out


def stacklstm_beam_reorder(dims, parent, states, count=None, stream=None, check=True) -> int:
    """states: what ``beam_states`` made, or its argument."""
    if not isinstance(states, ctypes.Array):
        count, states = len(states), beam_states(dims, states)
    rc = load_library().stacklstm_beam_reorder(dims, _arr(parent, torch.int32, "parent", (dims.B, dims.K)), states,
                                               len(states) if count is None else count, _here(stream, parent))
    if check:
        _check(rc, "stacklstm_beam_reorder")
    return rc


@dataclass
class BeamRun:
    """One step of a beam search: the K best continuations, then the states of the beams that go on."""
    dims: slstm_beam_dims
    logits: torch.Tensor
    legal: Optional[torch.Tensor]
    score: torch.Tensor
    done: Optional[torch.Tensor]
    states: list                    # set with set_states
    score_next: torch.Tensor
    parent: torch.Tensor
    token: torch.Tensor
    done_next: torch.Tensor
    workspace: torch.Tensor = field(repr=False, default=None)

    @classmethod
    def of(cls, logits, score, done=None, legal=None, eos=-1, states=()):
        """states: [(src, dst, live)] as in ``beam_states``."""
        (B, K), V = score.shape, logits.shape[1]
        d = make_beam_dims(B, K, V, _type(logits), eos, _ld(logits))
        e = lambda dtype: torch.empty(B, K, dtype=dtype, device=logits.device)
        n = _bytes("stacklstm_beam_workspace_bytes", d)
        r = cls(dims=d, logits=logits, legal=legal, score=score, done=done, states=[], score_next=e(torch.float32),
                parent=e(torch.int32), token=e(torch.int32), done_next=e(torch.uint8),
                workspace=torch.empty(n, dtype=torch.uint8, device=logits.device))
        r.set_states(states)
        return r

    def set_states(self, states):
        """The buffers that reorder copies, with their C descriptors (a program that swaps two sets of buffers makes two
        lists, or two BeamRuns)."""
        self.states = list(states)
        self._descriptors = beam_states(self.dims, self.states) if self.states else None

    def select(self, stream=None):
        stacklstm_beam_select(self.dims, self.logits, self.legal, self.score, self.done, self.score_next, self.parent,
                              self.token, self.done_next, self.workspace, stream)
        return self.parent

    def reorder(self, stream=None):
        """Copies every state's src to its dst; swap them for the next step."""
        if self.states:
            stacklstm_beam_reorder(self.dims, self.parent, self._descriptors, stream=stream)
