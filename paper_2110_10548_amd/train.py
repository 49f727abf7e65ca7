"""The local ends of a planned reduction, on torch tensors: same names as include/p2_train.h, argument marshalling only.

Tensors live on the current device and are worked on in the current stream; results and workspaces come from torch's
allocator, so calls may be captured into a graph.  Nothing here is recorded for autograd: the gradients are calls of their
own.  Rows whose last dimension is not contiguous, or whose leading dimensions have no common stride, are copied first.
"""
import ctypes as C
import functools

import torch

from . import binding as B
from .binding import P2_EINVAL, P2Error

P2_F32, P2_BF16, P2_F16 = 0, 1, 2
TYPES = {torch.float32: P2_F32, torch.bfloat16: P2_BF16, torch.float16: P2_F16}
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)      # pushes singular values in (0, 1] into about [0.7, 1.2] in five steps

EXPORTS = ("p2_layer_norm_forward", "p2_layer_norm_backward_workspace", "p2_layer_norm_backward", "p2_balance_forward_workspace",
           "p2_balance_forward", "p2_balance_loss", "p2_balance_backward", "p2_orthogonalize_workspace", "p2_orthogonalize")

_lib = None


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


@functools.lru_cache(maxsize=4096)
def _room(name, *sizes):
    """Bytes of the workspace that a call of these sizes takes."""
    out = C.c_int64()
    B._check(getattr(lib(), name)(*sizes, C.byref(out)))
    return out.value


def _refuse(text):
    raise P2Error(P2_EINVAL, text)


def _on_device(first, *others):
    """The current stream, after a look at whether all tensors are on its device."""
    here = first.get_device()
    if here < 0 or here != torch._C._cuda_getDevice():
        _refuse("tensors must be on the current device")
    for t in others:
        if t is not None and t.get_device() != here:
            _refuse("tensors must be on the current device")
    return torch._C._cuda_getCurrentRawStream(here)        # (a Stream object would take 3 us to make)


def _type(t, what):
    kind = TYPES.get(t.dtype)
    if kind is None:
        _refuse("%s must be float32, bfloat16 or float16" % what)
    return kind


def _rows(t):
    """(matrix whose rows are contiguous, rows, columns, distance between rows) of t [..., columns]."""
    if t.dim() == 2:
        n, cols = t.shape
        stride, one = t.stride()
        if one == 1 and stride >= cols:
            return t, n, cols, stride
    cols = t.shape[-1]
    t = t.reshape(-1, cols) if cols else t.reshape(0, 0)
    n = t.shape[0]
    if (cols > 1 and t.stride(1) != 1) or (n > 1 and t.stride(0) < cols):
        t = t.contiguous()
    return t, n, cols, (t.stride(0) if n > 1 else max(cols, 1))


def _like(t):
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _vector(t, n, what, dtype=None):
    if t is not None and (t.dim() != 1 or t.shape[0] != n or (dtype is not None and t.dtype != dtype)):
        _refuse("%s must have shape [%d]%s" % (what, n, "" if dtype is None else " and type %s" % dtype))
    return t if t is None or t.is_contiguous() else t.contiguous()


def _workspace(name, sizes, like):
    n = _room(name, *sizes)
    return (torch.empty(n, dtype=torch.uint8, device=like.device), n) if n else (None, 0)


def p2_layer_norm_forward(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd) of the rows of x [..., cols]; mean and rstd are float32 and have x's leading shape."""
    if x.dim() < 1:
        _refuse("x must have at least one dimension")
    stream = _on_device(x, weight, bias)
    kind = _type(x, "x")
    rows, n, cols, stride_x = _rows(x)
    weight, bias = _vector(weight, cols, "weight"), _vector(bias, cols, "bias")
    given = weight if weight is not None else bias
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        _refuse("weight and bias must have the same type")
    y = _like(x)
    mean = torch.empty(n if x.dim() == 2 else x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    B._check(lib().p2_layer_norm_forward(rows.data_ptr(), kind, stride_x, _ptr(weight), _ptr(bias), kind if given is None else _type(given, "weight"),
                                         n, cols, eps, y.data_ptr(), cols, mean.data_ptr(), rstd.data_ptr(), stream))
    return y, mean, rstd


def p2_layer_norm_backward(dy, x, weight, mean, rstd, dx=True, dweight=True, dbias=True):
    """(dx, dweight, dbias), None for what is not asked for.  weight may be None: the sums then have x's type."""
    if dy.shape != x.shape or dy.dtype != x.dtype or x.dim() < 1:
        _refuse("dy and x must have the same shape and type")
    stream = _on_device(dy, x, weight, mean, rstd)
    kind = _type(x, "x")
    rows, n, cols, stride_x = _rows(x)
    drows, _, _, stride_dy = _rows(dy)
    weight = _vector(weight, cols, "weight")
    if mean.dim() != 1 or rstd.dim() != 1:
        mean, rstd = mean.reshape(-1), rstd.reshape(-1)
    mean, rstd = _vector(mean, n, "mean", torch.float32), _vector(rstd, n, "rstd", torch.float32)
    like = x if weight is None else weight
    out = _like(x) if dx else None
    dw = torch.empty(cols, dtype=like.dtype, device=x.device) if dweight else None
    db = torch.empty(cols, dtype=like.dtype, device=x.device) if dbias else None
    work, size = _workspace("p2_layer_norm_backward_workspace", (n, cols), x) if dweight or dbias else (None, 0)
    B._check(lib().p2_layer_norm_backward(drows.data_ptr(), stride_dy, rows.data_ptr(), stride_x, kind, _ptr(weight), _type(like, "weight"),
                                          mean.data_ptr(), rstd.data_ptr(), n, cols, _ptr(out), cols, _ptr(dw), _ptr(db), _ptr(work), size, stream))
    return out, dw, db


def _tokens(logits, keep):
    if logits.dim() != 2:
        _refuse("logits must be [tokens, experts]")
    if keep is not None and (keep.dtype not in (torch.bool, torch.uint8) or tuple(keep.shape) != (logits.shape[0],)):
        _refuse("keep must be a truth value for each token")
    return None if keep is None else keep.contiguous()


def p2_balance_forward(logits, k, keep=None):
    """A dict: expert int32 and gate float32 [tokens, k]; counts int64 and prob_sum float32 [experts]; tokens int64 (how many
    count) and loss float32, without dimensions."""
    keep = _tokens(logits, keep)
    stream = _on_device(logits, keep)
    kind = _type(logits, "logits")
    rows, n, e, stride_z = _rows(logits)
    d = logits.device
    expert = torch.empty((n, max(k, 0)), dtype=torch.int32, device=d)
    gate = torch.empty_like(expert, dtype=torch.float32)
    counts = torch.empty(e, dtype=torch.int64, device=d)
    prob_sum = torch.empty_like(counts, dtype=torch.float32)
    kept = torch.empty((), dtype=torch.int64, device=d)
    loss = torch.empty_like(kept, dtype=torch.float32)
    work, size = _workspace("p2_balance_forward_workspace", (n, e), logits)
    B._check(lib().p2_balance_forward(rows.data_ptr(), kind, stride_z, _ptr(keep), n, e, k, expert.data_ptr(), gate.data_ptr(), counts.data_ptr(),
                                      prob_sum.data_ptr(), kept.data_ptr(), loss.data_ptr(), _ptr(work), size, stream))
    return {"expert": expert, "gate": gate, "counts": counts, "prob_sum": prob_sum, "tokens": kept, "loss": loss}


def _statistics(counts, kept, experts):
    if counts.dtype != torch.int64 or tuple(counts.shape) != (experts,) or kept.dtype != torch.int64 or kept.numel() != 1:
        _refuse("counts must be int64 [experts], tokens one int64")
    return counts.contiguous()


def p2_balance_loss(counts, prob_sum, tokens, k):
    """The loss, without dimensions, from statistics that may have been summed over devices."""
    counts = _statistics(counts, tokens, counts.shape[0] if counts.dim() == 1 else -1)
    prob_sum = _vector(prob_sum, counts.shape[0], "prob_sum", torch.float32)
    stream = _on_device(counts, prob_sum, tokens)
    loss = torch.empty((), dtype=torch.float32, device=counts.device)
    B._check(lib().p2_balance_loss(counts.data_ptr(), prob_sum.data_ptr(), tokens.data_ptr(), counts.shape[0], k, loss.data_ptr(), stream))
    return loss


def p2_balance_backward(logits, expert, counts, tokens, keep=None, dgate=None, dloss=None):
    """dlogits of  dloss * loss + (dgate * gate).sum();  dloss: a float32 of one element, None: 1."""
    keep = _tokens(logits, keep)
    stream = _on_device(logits, expert, counts, tokens, keep, dgate, dloss)
    kind = _type(logits, "logits")
    rows, n, e, stride_z = _rows(logits)
    if expert.dtype != torch.int32 or expert.dim() != 2 or expert.shape[0] != n:
        _refuse("expert must be int32 [tokens, k]")
    k = expert.shape[1]
    if dgate is not None and (dgate.dtype != torch.float32 or dgate.shape != expert.shape):
        _refuse("dgate must be float32 [tokens, k]")
    if dloss is not None and (dloss.dtype != torch.float32 or dloss.numel() != 1):
        _refuse("dloss must be one float32")
    counts = _statistics(counts, tokens, e)
    expert, dgate = expert.contiguous(), None if dgate is None else dgate.contiguous()
    out = _like(logits)
    B._check(lib().p2_balance_backward(rows.data_ptr(), kind, stride_z, _ptr(keep), n, e, k, expert.data_ptr(), _ptr(dgate), counts.data_ptr(),
                                       tokens.data_ptr(), _ptr(dloss), out.data_ptr(), max(e, 1), stream))
    return out


def p2_orthogonalize(g, steps=5, coefficients=NEWTON_SCHULZ, eps=1e-7, scale=1.0, dtype=None):
    """scale times the Newton-Schulz iterate of each matrix of g [..., rows, cols], in g's type or `dtype`."""
    if g.dim() < 2:
        _refuse("g must have at least two dimensions")
    if len(coefficients) != 3:
        _refuse("three coefficients")
    stream = _on_device(g)
    kind = _type(g, "g")
    out = torch.empty(g.shape, dtype=dtype or g.dtype, device=g.device)
    out_kind = _type(out, "the result")
    rows, cols = g.shape[-2:]
    m = g if g.dim() == 3 else g.reshape(g.shape[:-2].numel(), rows, cols)
    if (cols > 1 and m.stride(2) != 1) or (rows > 1 and m.stride(1) < cols):
        m = m.contiguous()
    count = m.shape[0]
    work, size = _workspace("p2_orthogonalize_workspace", (count, rows, cols), g)
    B._check(lib().p2_orthogonalize(m.data_ptr(), kind, m.stride(1) if rows > 1 else max(cols, 1), m.stride(0) if count > 1 else 0, count, rows, cols,
                                    steps, (C.c_double * 3)(*coefficients), eps, scale, out.data_ptr(), out_kind, cols, rows * cols,
                                    _ptr(work), size, stream))
    return out
