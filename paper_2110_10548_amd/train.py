"""The local ends of a planned reduction, on torch tensors: same names as include/p2_train.h.  Shapes, types and results are seen to
by a small extension module (csrc/p2_train_tensors.cpp), which calls the library.

Tensors live on the current device and are worked on in the current stream; results and workspaces come from torch's
allocator, so calls may be captured into a graph.  Nothing here is recorded for autograd: the gradients are calls of their
own, and where autograd records and an argument requires a gradient a UserWarning says so.  Rows whose last dimension is not contiguous, or whose leading dimensions have no common stride, are copied first.
"""
import ctypes as C

import torch

from . import binding as B
from .binding import P2_EINVAL, P2Error

P2_F32, P2_BF16, P2_F16 = 0, 1, 2
TYPES = {torch.float32: P2_F32, torch.bfloat16: P2_BF16, torch.float16: P2_F16}
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)      # pushes singular values in (0, 1] into about [0.7, 1.2] in five steps

EXPORTS = ("p2_layer_norm_forward", "p2_layer_norm_backward_workspace", "p2_layer_norm_backward", "p2_balance_forward_workspace",
           "p2_balance_forward", "p2_balance_loss", "p2_balance_backward", "p2_orthogonalize_workspace", "p2_orthogonalize")

_lib = _native = None


def lib():
    global _lib
    if _lib is None:
        L = B.lib()
        p, i32, i64, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_double
        sizes = C.POINTER(i64)
        for name, args in (
                ("p2_layer_norm_forward", [p, i32, i64, p, p, i32, i64, i64, f64, p, i64, p, p, p]),
                ("p2_layer_norm_backward_workspace", [i64, i64, sizes]),
                ("p2_layer_norm_backward", [p, i64, p, i64, i32, p, i32, p, p, i64, i64, p, i64, p, p, p, i64, p]),
                ("p2_balance_forward_workspace", [i64, i32, sizes]),
                ("p2_balance_forward", [p, i32, i64, p, i64, i32, i32, p, p, p, p, p, p, p, i64, p]),
                ("p2_balance_loss", [p, p, p, i32, i32, p, p]),
                ("p2_balance_backward", [p, i32, i64, p, i64, i32, i32, p, p, p, p, p, p, i64, p]),
                ("p2_orthogonalize_workspace", [i64, i64, i64, sizes]),
                ("p2_orthogonalize", [p, i32, i64, i64, i64, i64, i64, i32, C.POINTER(f64), f64, f64, p, i32, i64, i64, p, i64, p])):
            getattr(L, name).restype = i32
            getattr(L, name).argtypes = args
        _lib = L
    return _lib


def _native_calls():
    """The extension module, which knows the library's addresses."""
    global _native
    L = lib()
    try:
        from . import _train
    except ImportError as e:
        raise P2Error(P2_EINVAL, "the extension module of the training operators is missing or does not load: build it first (%s)" % e) from e
    _train.bind(*(C.cast(getattr(L, name), C.c_void_p).value for name in EXPORTS), B._check, _refuse)
    _native = _train
    return _native


def _room(name, *sizes):
    """Bytes of the workspace that a call of these sizes takes."""
    out = C.c_int64()
    B._check(getattr(lib(), name)(*sizes, C.byref(out)))
    return out.value


def _refuse(text):
    raise P2Error(P2_EINVAL, text)


def _stream(t):
    """The current stream, after a look at whether the tensor is on its device."""
    here = t.get_device()
    if here < 0 or here != torch._C._cuda_getDevice():
        _refuse("tensors must be on the current device")
    return torch._C._cuda_getCurrentRawStream(here)        # (a Stream object would take 3 us to make)


def _ptr(t):
    return None if t is None else t.data_ptr()


def p2_layer_norm_forward(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd) of the rows of x [..., cols]; mean and rstd are float32 and have x's leading shape."""
    if x.dim() < 1:
        _refuse("x must have at least one dimension")
    return (_native or _native_calls()).layer_norm_forward(x, weight, bias, eps, _stream(x))


def p2_layer_norm_backward(dy, x, weight, mean, rstd, dx=True, dweight=True, dbias=True):
    """(dx, dweight, dbias), None for what is not asked for.  weight may be None: the sums then have x's type."""
    if dy.shape != x.shape or dy.dtype != x.dtype or x.dim() < 1:
        _refuse("dy and x must have the same shape and type")
    return (_native or _native_calls()).layer_norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, _stream(x))


def p2_balance_forward(logits, k, keep=None):
    """A dict: expert int32 and gate float32 [tokens, k]; counts int64 and prob_sum float32 [experts]; tokens int64 (how many
    count) and loss float32, without dimensions."""
    if logits.dim() != 2:
        _refuse("logits must be [tokens, experts]")
    expert, gate, counts, prob_sum, tokens, loss = (_native or _native_calls()).balance_forward(logits, k, keep, _stream(logits))
    return {"expert": expert, "gate": gate, "counts": counts, "prob_sum": prob_sum, "tokens": tokens, "loss": loss}


def p2_balance_loss(counts, prob_sum, tokens, k):
    """The loss, without dimensions, from statistics that may have been summed over devices."""
    return (_native or _native_calls()).balance_loss(counts, prob_sum, tokens, k, _stream(counts))


def p2_balance_backward(logits, expert, counts, tokens, keep=None, dgate=None, dloss=None):
    """dlogits of  dloss * loss + (dgate * gate).sum();  dloss: a float32 of one element, None: 1."""
    if logits.dim() != 2:
        _refuse("logits must be [tokens, experts]")
    return (_native or _native_calls()).balance_backward(logits, expert, counts, tokens, keep, dgate, dloss, _stream(logits))


def p2_orthogonalize(g, steps=5, coefficients=NEWTON_SCHULZ, eps=1e-7, scale=1.0, dtype=None):
    """scale times the Newton-Schulz iterate of each matrix of g [..., rows, cols], in g's type or `dtype`."""
    if g.dim() < 2:
        _refuse("g must have at least two dimensions")
    if len(coefficients) != 3:
        _refuse("three coefficients")
    kind = -1 if dtype is None else TYPES.get(dtype)
    if kind is None:
        _refuse("the result must be float32, bfloat16 or float16")
    a, b, c = coefficients
    return (_native or _native_calls()).orthogonalize(g, steps, a, b, c, eps, scale, kind, _stream(g))
