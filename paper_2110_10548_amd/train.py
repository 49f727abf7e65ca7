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
SCORES = {"softmax": 0, "sigmoid": 1}
ACTIVATIONS = {None: 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
STATE_BLOCK = 256                              # values that share a scale of an 8-bit state
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)      # pushes singular values in (0, 1] into about [0.7, 1.2] in five steps

EXPORTS = ("p2_layer_norm_forward", "p2_layer_norm_backward_workspace", "p2_layer_norm_backward", "p2_balance_forward_workspace",
           "p2_balance_forward", "p2_balance_loss", "p2_balance_backward", "p2_orthogonalize_workspace", "p2_orthogonalize",
           "p2_route_forward_workspace", "p2_route_forward", "p2_route_backward", "p2_route_bias", "p2_square_sum_workspace", "p2_square_sum",
           "p2_adamw_workspace", "p2_adamw", "p2_adamw_values", "p2_linear_forward_workspace", "p2_linear_forward", "p2_linear_backward_workspace",
           "p2_linear_backward_workspace_for", "p2_linear_backward")

_lib = _native = None


class AdamwTensor(C.Structure):
    """p2_adamw_tensor"""
    _fields_ = [(name, C.c_void_p) for name in ("param", "grad", "copy", "mean", "square", "mean_scale", "square_scale")] + [("count", C.c_int64)]


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
                ("p2_orthogonalize", [p, i32, i64, i64, i64, i64, i64, i32, C.POINTER(f64), f64, f64, p, i32, i64, i64, p, i64, p]),
                ("p2_route_forward_workspace", [i64, i32, i32, i32, sizes]),
                ("p2_route_forward", [p, i32, i64, p, p, i64, i32, i32, i32, i32, i32, i32, i32, f64, p, p, p, p, p, i64, p]),
                ("p2_route_backward", [p, i32, i64, i64, i32, i32, i32, i32, f64, p, p, p, i64, p]),
                ("p2_route_bias", [p, p, i32, f64, p, p]),
                ("p2_square_sum_workspace", [i64, sizes]),
                ("p2_square_sum", [C.POINTER(p), sizes, i64, i32, p, p, i64, p]),
                ("p2_adamw_workspace", [sizes]),
                ("p2_adamw", [C.POINTER(AdamwTensor), i64, i32, i32, i32, i32, p, p, f64, f64, f64, f64, f64, f64, p, f64, p, i64, p]),
                ("p2_adamw_values", [C.POINTER(AdamwTensor), i64, C.POINTER(p), C.POINTER(p), p]),
                ("p2_linear_forward_workspace", [p, i64, p, i64, i32, i64, i64, i64, sizes]),
                ("p2_linear_forward", [p, i64, p, i64, p, p, i64, i32, i32, i64, i64, i64, p, i64, p, i64, p, i64, p]),
                ("p2_linear_backward_workspace", [i32, i64, i64, i64, sizes]),
                ("p2_linear_backward_workspace_for", [p, i64, p, i64, p, i64, i32, i32, i64, i64, i64, i32, i32, i32, sizes]),
                ("p2_linear_backward", [p, i64, p, i64, p, i64, p, i64, i32, i32, i64, i64, i64, p, i64, p, i64, p, i32, p, i64, p])):
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


def _kind(names, name, what):
    if name not in names:
        _refuse("%s must be one of %s" % (what, ", ".join(str(n) for n in names)))
    return names[name]


def p2_route_forward(logits, k, score="softmax", bias=None, keep=None, groups=1, group_limit=None, group_best=1, renormalise=False, scale=1.0):
    """A dict: expert int32 and gate float32 [tokens, k]; counts int64 [experts]; tokens int64 (how many count), without dimensions.

    group_limit: in how many of the groups the choice is made, None: all of them.  bias: float32 [experts]."""
    if logits.dim() != 2:
        _refuse("logits must be [tokens, experts]")
    expert, gate, counts, tokens = (_native or _native_calls()).route_forward(
        logits, k, _kind(SCORES, score, "score"), bias, keep, groups, groups if group_limit is None else group_limit, group_best, renormalise, scale, _stream(logits))
    return {"expert": expert, "gate": gate, "counts": counts, "tokens": tokens}


def p2_route_backward(logits, expert, dgate, score="softmax", renormalise=False, scale=1.0):
    """dlogits of  (dgate * gate).sum()."""
    if logits.dim() != 2:
        _refuse("logits must be [tokens, experts]")
    return (_native or _native_calls()).route_backward(logits, expert, dgate, _kind(SCORES, score, "score"), renormalise, scale, _stream(logits))


def p2_route_bias(bias, counts, rate):
    """The biases of the next step, from the counts of the whole batch."""
    return (_native or _native_calls()).route_bias(bias, counts, rate, _stream(bias))


def p2_square_sum(tensors):
    """The sum of the squares of all values of a list of tensors of one type: a float64 without dimensions, which may be summed over devices."""
    if not len(tensors):
        _refuse("no tensors")
    return (_native or _native_calls()).square_sum(tensors, _stream(tensors[0]))


def p2_adamw_state(params, bits=32):
    """What p2_adamw keeps of these tensors, all zeros: a dict of its arguments means, squares, step, mean_scales and square_scales."""
    if bits not in (32, 8):
        _refuse("states have 32 or 8 bits")
    scales = [(p.numel() + STATE_BLOCK - 1) // STATE_BLOCK for p in params]
    zeros = lambda kind: [torch.zeros(p.shape, dtype=kind, device=p.device) for p in params]  # noqa: E731
    scale = lambda: [torch.zeros(n, dtype=torch.float32, device=p.device) for n, p in zip(scales, params)] if bits == 8 else None  # noqa: E731
    return {"means": zeros(torch.float32 if bits == 32 else torch.int8), "squares": zeros(torch.float32 if bits == 32 else torch.uint8),
            "step": torch.zeros((), dtype=torch.int64, device=params[0].device if len(params) else None), "mean_scales": scale(), "square_scales": scale()}


def p2_adamw(params, grads, means, squares, step, mean_scales=None, square_scales=None, copies=None, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0,
             rate=None, grad_factor=1.0, square_sum=None, max_norm=None):
    """One AdamW step in place: lists of tensors, all of a list of one type, contiguous (gradients may be otherwise).  p2_adamw_state makes the
    states.  step: one int64, which the call counts up, so that groups of other types or decays have a state and a step each; rate: one float32 on the
    device that lr is multiplied by.

    square_sum: what p2_square_sum gave, perhaps summed over devices; where it is not finite the step is left out, and with max_norm the
    gradients are scaled down to that norm.  Parameters that require a gradient are updated all the same."""
    if not len(params):
        _refuse("no tensors")
    if max_norm is not None and square_sum is None:
        _refuse("max_norm needs square_sum")
    if len(betas) != 2:
        _refuse("two betas")
    (_native or _native_calls()).adamw(params, grads, means, squares, step, mean_scales, square_scales, copies, rate, lr, betas[0], betas[1], eps, weight_decay, grad_factor,
                                       square_sum, float("inf") if max_norm is None else max_norm, _stream(params[0]))


def p2_adamw_values(means, squares, mean_scales, square_scales):
    """(means, squares): lists of the float32 values that 8-bit states stand for."""
    if not len(means):
        _refuse("no tensors")
    return (_native or _native_calls()).adamw_values(means, squares, mean_scales, square_scales, _stream(means[0]))


def p2_linear_forward(x, weight, bias=None, activation=None, residual=None, keep=False):
    """(y, z): activation(x weight^T + bias) + residual for x [..., inner] and weight [outer, inner]; z, what the activation took, is None unless kept."""
    if x.dim() < 1:
        _refuse("x must have at least one dimension")
    return (_native or _native_calls()).linear_forward(x, weight, bias, _kind(ACTIVATIONS, activation, "activation"), residual, keep, _stream(x))


def p2_linear_backward(dy, x, weight, z=None, activation=None, dx=True, dweight=True, dbias=True, dtype=None):
    """(dx, dweight, dbias), None for what is not asked for.  z: what the forward pass kept; dtype: the weight's gradients', None: the weight's."""
    if x.dim() < 1:
        _refuse("x must have at least one dimension")
    kind = -1 if dtype is None else TYPES.get(dtype)
    if kind is None:
        _refuse("the gradients must be float32, bfloat16 or float16")
    return (_native or _native_calls()).linear_backward(dy, x, weight, z, _kind(ACTIVATIONS, activation, "activation"), dx, dweight, dbias, kind, _stream(x))
