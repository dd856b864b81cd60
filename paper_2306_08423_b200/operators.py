"""Binding of the layer operators of ``include/distsim.h``: the product with bias, activation and
residual, the gated feed-forward block, and the residual connection with its norms and dropout,
forward and backward.  Argument marshalling only; ``engine`` re-exports every function here.

Matrices are 2-D CUDA tensors whose columns are contiguous (rows any distance apart), vectors
contiguous 1-D tensors.  Outputs are the caller's tensors.  A wrong type, shape or device raises
ValueError before anything is launched; what the library refuses raises DistsimError.
"""
from __future__ import annotations

import ctypes as C

from ._library import OK, _lib

OPERATOR_EXPORTS = ("distsim_operator_status", "distsim_linear_forward", "distsim_linear_backward",
                    "distsim_gated_ffn_forward", "distsim_gated_ffn_backward",
                    "distsim_residual_norm_forward", "distsim_residual_norm_backward")
MAX_COLS = 16384
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
NORMS = {"layer": 0, "rms": 1}


def _fields(ints64, ints32, pointers, lds, between=()):
    return ([(n, C.c_int64) for n in ints64] + [(n, C.c_int32) for n in ints32] + list(between) +
            [(n, C.c_void_p) for n in pointers] + [("ld_" + n, C.c_int64) for n in lds])


class _Linear(C.Structure):
    _fields_ = _fields(("tokens", "d_in", "d_out"), ("dtype", "activation", "grad_dtype", "reserved"),
                       ("x", "weight", "bias", "residual", "y", "preact", "dy", "dx", "dweight", "dweight_in", "dbias"),
                       ("x", "weight", "residual", "y", "preact", "dy", "dx", "dweight", "dweight_in"))


_EARLIER = ("dw_gate_in", "dw_up_in", "dw_down_in")


class _GatedFfn(C.Structure):
    _fields_ = _fields(("tokens", "d_in", "d_hidden"), ("dtype", "activation", "grad_dtype", "reserved"),
                       ("x", "w_gate", "w_up", "w_down", "b_gate", "b_up", "b_down", "residual", "y", "hidden", "gate", "up",
                        "dy", "dx", "dw_gate", "dw_up", "dw_down", "db_gate", "db_up", "db_down"),
                       ("x", "w_gate", "w_up", "w_down", "residual", "y", "hidden", "gate", "up", "dy", "dx", "dw_gate",
                        "dw_up", "dw_down")) + _fields((), (), _EARLIER, _EARLIER)


class _ResidualNorm(C.Structure):
    _fields_ = _fields(("tokens", "cols"), ("dtype", "grad_dtype", "kind", "reserved"),
                       ("x", "residual", "gate", "post_weight", "post_bias", "weight", "bias", "h", "y", "dy", "dh",
                        "dx", "dresidual", "dgate", "dpost_weight", "dpost_bias", "dweight", "dbias"),
                       ("x", "residual", "h", "y", "dy", "dh", "dx", "dresidual"),
                       between=[("alpha", C.c_double), ("eps", C.c_double), ("p", C.c_double),
                                ("seed", C.c_uint64), ("offset", C.c_uint64)])


for _name, _struct in (("linear", _Linear), ("gated_ffn", _GatedFfn), ("residual_norm", _ResidualNorm)):
    for _way in ("forward", "backward"):
        getattr(_lib, f"distsim_{_name}_{_way}").argtypes = [C.c_void_p, C.c_void_p, C.POINTER(_struct)]
_lib.distsim_operator_status.argtypes = [C.c_void_p, C.c_void_p]

_codes = {}


def _code(dtype, what):
    if not _codes:
        import torch
        _codes.update({torch.bfloat16: 0, torch.float16: 1, torch.float32: 2})
    if dtype not in _codes:
        raise ValueError(f"{what}: unsupported type {dtype}")
    return _codes[dtype]


class _Op:
    """Fills a struct from tensors, checking each."""

    __slots__ = ("s", "ctx", "device", "dtype", "grad")

    def __init__(self, struct, ctx, like):
        self.s = struct()
        self.ctx = ctx
        self.device = ctx.device
        self.dtype = like.dtype
        if not like.is_cuda or like.get_device() != ctx.device:
            raise ValueError(f"need tensors on cuda:{ctx.device}, the context's device")
        self.s.dtype = _code(like.dtype, "the operator")

    def _check(self, t, name, dtype):
        if t.get_device() != self.device:
            raise ValueError(f"{name}: need a tensor on cuda:{self.device}")
        if t.dtype != dtype:
            raise ValueError(f"{name}: need {dtype}, got {t.dtype}")

    def matrix(self, name, t, rows, cols, dtype=None):
        if t is None:
            return
        if t.dtype != (dtype or self.dtype) or t.get_device() != self.device:
            self._check(t, name, dtype or self.dtype)
        if t.shape != (rows, cols):
            raise ValueError(f"{name}: need shape ({rows}, {cols}), got {tuple(t.shape)}")
        ld, inner = t.stride()
        if (cols > 1 and inner != 1) or (rows > 1 and ld < cols):
            raise ValueError(f"{name}: columns must be contiguous and rows must not overlap (strides {t.stride()})")
        setattr(self.s, name, t.data_ptr())
        setattr(self.s, "ld_" + name, ld if rows > 1 else cols)

    def vector(self, name, t, n, dtype=None):
        if t is None:
            return
        if t.dtype != (dtype or self.dtype) or t.get_device() != self.device:
            self._check(t, name, dtype or self.dtype)
        if t.shape != (n,) or (n > 1 and t.stride(0) != 1):
            raise ValueError(f"{name}: need a contiguous vector of {n} elements, got {tuple(t.shape)}")
        setattr(self.s, name, t.data_ptr())

    def grad_type(self, *grads):
        """The one type of the parameters' gradients."""
        self.grad = None
        for g in grads:
            if g is not None:
                if self.grad is not None and g.dtype != self.grad:
                    raise ValueError(f"the parameters' gradients need one type, got {self.grad} and {g.dtype}")
                self.grad = g.dtype
        if self.grad is None:
            self.grad = self.dtype
        self.s.grad_dtype = _code(self.grad, "gradients")

    def call(self, fn, stream):
        raw = _raw_stream(self.device) if stream is None else stream.cuda_stream
        rc = fn(self.ctx._h, raw, C.byref(self.s))
        if rc != OK:
            self.ctx._check(rc)


def _raw_stream(device):
    """The handle of PyTorch's current stream of a device."""
    import torch
    return torch._C._cuda_getCurrentRawStream(device)


def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"activation: one of {sorted(ACTIVATIONS)}, got {name!r}")
    return ACTIVATIONS[name]


def _sizes(t, name):
    if t.dim() != 2:
        raise ValueError(f"{name}: need a matrix, got {t.dim()} dimensions")
    return t.shape


def distsim_operator_status(ctx, stream=None) -> None:
    """Waits for ``stream``; raises if a kernel of an earlier operator call gave up waiting."""
    ctx._check(_lib.distsim_operator_status(ctx._h, _raw_stream(ctx.device) if stream is None else stream.cuda_stream))


def distsim_linear_forward(ctx, x, weight, y, bias=None, residual=None, preact=None, activation="none", stream=None) -> None:
    """y = activation(x weight^T + bias) + residual; ``preact`` receives the activation's argument."""
    (t, d), f = _sizes(x, "x"), _sizes(weight, "weight")[0]
    o = _Op(_Linear, ctx, x)
    o.s.tokens, o.s.d_in, o.s.d_out, o.s.activation = t, d, f, _activation(activation)
    o.matrix("x", x, t, d)
    o.matrix("weight", weight, f, d)
    o.vector("bias", bias, f)
    for name, v in (("residual", residual), ("y", y), ("preact", preact)):
        o.matrix(name, v, t, f)
    o.call(_lib.distsim_linear_forward, stream)


def distsim_linear_backward(ctx, dy, x, weight, dx=None, dweight=None, dbias=None, preact=None, activation="none",
                            dweight_in=None, stream=None) -> None:
    """Gradients of ``distsim_linear_forward`` by x, weight and bias (dweight_in + the weight's, if given)."""
    (t, d), f = _sizes(x, "x"), _sizes(weight, "weight")[0]
    o = _Op(_Linear, ctx, x)
    o.s.tokens, o.s.d_in, o.s.d_out, o.s.activation = t, d, f, _activation(activation)
    o.grad_type(dweight, dbias)
    o.matrix("dy", dy, t, f)
    o.matrix("preact", preact, t, f)
    for name, v in (("x", x), ("dx", dx)):
        o.matrix(name, v, t, d)
    o.matrix("weight", weight, f, d)
    for name, v in (("dweight", dweight), ("dweight_in", dweight_in)):
        o.matrix(name, v, f, d, o.grad)
    o.vector("dbias", dbias, f, o.grad)
    o.call(_lib.distsim_linear_backward, stream)


def _ffn(ctx, x, w_gate, w_up, w_down, activation):
    (t, d), f = _sizes(x, "x"), _sizes(w_gate, "w_gate")[0]
    o = _Op(_GatedFfn, ctx, x)
    o.s.tokens, o.s.d_in, o.s.d_hidden, o.s.activation = t, d, f, _activation(activation)
    o.matrix("x", x, t, d)
    for name, v in (("w_gate", w_gate), ("w_up", w_up)):
        o.matrix(name, v, f, d)
    o.matrix("w_down", w_down, d, f)
    return o, t, d, f


def distsim_gated_ffn_forward(ctx, x, w_gate, w_up, w_down, y, b_gate=None, b_up=None, b_down=None, residual=None,
                              hidden=None, gate=None, up=None, activation="silu", stream=None) -> None:
    """y = (activation(x w_gate^T + b_gate) * (x w_up^T + b_up)) w_down^T + b_down + residual; ``gate``,
    ``up`` and ``hidden`` receive the two projections and their product, for the backward pass."""
    o, t, d, f = _ffn(ctx, x, w_gate, w_up, w_down, activation)
    for name, v, n in (("b_gate", b_gate, f), ("b_up", b_up, f), ("b_down", b_down, d)):
        o.vector(name, v, n)
    for name, v in (("residual", residual), ("y", y)):
        o.matrix(name, v, t, d)
    for name, v in (("hidden", hidden), ("gate", gate), ("up", up)):
        o.matrix(name, v, t, f)
    o.call(_lib.distsim_gated_ffn_forward, stream)


def distsim_gated_ffn_backward(ctx, dy, x, w_gate, w_up, w_down, hidden, gate, up, dx=None, dw_gate=None, dw_up=None,
                               dw_down=None, db_gate=None, db_up=None, db_down=None, activation="silu", dw_gate_in=None,
                               dw_up_in=None, dw_down_in=None, stream=None) -> None:
    """Gradients of ``distsim_gated_ffn_forward`` by x, the weights and the biases (any may be None; a weight's is
    added to its ``dw_*_in``, if given)."""
    o, t, d, f = _ffn(ctx, x, w_gate, w_up, w_down, activation)
    o.grad_type(dw_gate, dw_up, dw_down, db_gate, db_up, db_down)
    for name, v in (("dy", dy), ("dx", dx)):
        o.matrix(name, v, t, d)
    for name, v in (("hidden", hidden), ("gate", gate), ("up", up)):
        o.matrix(name, v, t, f)
    for name, v in (("dw_gate", dw_gate), ("dw_up", dw_up), ("dw_gate_in", dw_gate_in), ("dw_up_in", dw_up_in)):
        o.matrix(name, v, f, d, o.grad)
    for name, v in (("dw_down", dw_down), ("dw_down_in", dw_down_in)):
        o.matrix(name, v, d, f, o.grad)
    for name, v, n in (("db_gate", db_gate, f), ("db_up", db_up, f), ("db_down", db_down, d)):
        o.vector(name, v, n, o.grad)
    o.call(_lib.distsim_gated_ffn_backward, stream)


def _norm(ctx, like, kind, alpha, eps, p, seed, offset, **vectors):
    t, n = _sizes(like, "x or h")
    if kind not in NORMS:
        raise ValueError(f"kind: one of {sorted(NORMS)}, got {kind!r}")
    o = _Op(_ResidualNorm, ctx, like)
    s = o.s
    s.tokens, s.cols, s.kind, s.alpha, s.eps, s.p = t, n, NORMS[kind], alpha, eps, p
    s.seed, s.offset = seed & (2 ** 64 - 1), offset & (2 ** 64 - 1)
    for name, v in vectors.items():
        o.vector(name, v, n)
    return o, t, n


def distsim_residual_norm_forward(ctx, x, residual=None, h=None, y=None, gate=None, post_weight=None, post_bias=None,
                                  weight=None, bias=None, kind="layer", alpha=1.0, eps=1e-5, p=0.0, seed=0, offset=0,
                                  stream=None) -> None:
    """h = alpha * residual + gate * dropout(norm(x) post_weight + post_bias); y = norm(h) weight + bias."""
    o, t, n = _norm(ctx, x, kind, alpha, eps, p, seed, offset, gate=gate, post_weight=post_weight, post_bias=post_bias,
                    weight=weight, bias=bias)
    for name, v in (("x", x), ("residual", residual), ("h", h), ("y", y)):
        o.matrix(name, v, t, n)
    o.call(_lib.distsim_residual_norm_forward, stream)


def distsim_residual_norm_backward(ctx, x, h, dy=None, dh=None, dx=None, dresidual=None, dgate=None, dpost_weight=None,
                                   dpost_bias=None, dweight=None, dbias=None, gate=None, post_weight=None, post_bias=None,
                                   weight=None, kind="layer", alpha=1.0, eps=1e-5, p=0.0, seed=0, offset=0,
                                   stream=None) -> None:
    """Gradients of ``distsim_residual_norm_forward`` from ``dy`` (of y) and ``dh`` (of h)."""
    like = next((v for v in (x, h, dh) if v is not None), None)
    if like is None:
        raise ValueError("need x, h or dh")
    o, t, n = _norm(ctx, like, kind, alpha, eps, p, seed, offset, gate=gate, post_weight=post_weight,
                    post_bias=post_bias, weight=weight)
    o.grad_type(dgate, dpost_weight, dpost_bias, dweight, dbias)
    for name, v in (("x", x), ("h", h), ("dy", dy), ("dh", dh), ("dx", dx), ("dresidual", dresidual)):
        o.matrix(name, v, t, n)
    for name, v in (("dgate", dgate), ("dpost_weight", dpost_weight), ("dpost_bias", dpost_bias), ("dweight", dweight),
                    ("dbias", dbias)):
        o.vector(name, v, n, o.grad)
    o.call(_lib.distsim_residual_norm_backward, stream)
