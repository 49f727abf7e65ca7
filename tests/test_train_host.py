"""Refusals of the training operators: they come before anything is queued, so no GPU is needed (pointers are made up)."""
import ctypes as C
import os
import re
import warnings

import pytest
import torch

from conftest import ROOT


@pytest.fixture(scope="module")
def T():
    from paper_2110_10548_amd import binding, train
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    train.lib()
    return train


def test_every_declared_symbol_is_exported(T):
    header = open(os.path.join(ROOT, "include", "p2_train.h")).read()
    declared = set(re.findall(r"\bint32_t (p2_[a-z_]+)\s*\(", header))
    assert declared == set(T.EXPORTS)
    L = C.CDLL(T.B.LIB_PATH)
    assert all(getattr(L, name) is not None for name in declared)


P, ODD, NULL = 4096, 4097, None      # an aligned pointer, one that is aligned to nothing, none


def _norm_forward(T, **kw):
    a = dict(x=P, type=0, x_stride=8, weight=P, bias=P, weight_type=0, rows=4, cols=8, eps=1e-5, y=P, y_stride=8, mean=P, rstd=P) | kw
    return T.lib().p2_layer_norm_forward(*a.values(), None)


def _norm_backward(T, **kw):
    a = dict(dy=P, dy_stride=8, x=P, x_stride=8, type=0, weight=P, weight_type=0, mean=P, rstd=P, rows=4, cols=8, dx=P, dx_stride=8, dweight=P,
             dbias=P, workspace=P, workspace_bytes=1 << 20) | kw
    return T.lib().p2_layer_norm_backward(*a.values(), None)


def _balance_forward(T, **kw):
    a = dict(logits=P, type=0, stride=8, keep=NULL, tokens=4, experts=8, k=2, expert=P, gate=P, counts=P, prob_sum=P, kept=P, loss=P, workspace=P,
             workspace_bytes=1 << 20) | kw
    return T.lib().p2_balance_forward(*a.values(), None)


def _balance_backward(T, **kw):
    a = dict(logits=P, type=0, stride=8, keep=NULL, tokens=4, experts=8, k=2, expert=P, dgate=P, counts=P, kept=P, dloss=P, dlogits=P,
             dlogits_stride=8) | kw
    return T.lib().p2_balance_backward(*a.values(), None)


def _orthogonalize(T, coefficients=(3.4445, -4.7750, 2.0315), **kw):
    a = dict(g=P, type=0, stride=8, matrix_stride=256, count=1, rows=300, cols=8, steps=5, coefficients=coefficients and (C.c_double * 3)(*coefficients),
             eps=1e-7, scale=1.0, out=P, out_type=0, out_stride=8, out_matrix_stride=4096, workspace=P, workspace_bytes=1 << 30) | kw
    return T.lib().p2_orthogonalize(*a.values(), None)


EINVAL, ENOSPC, EUNSUPPORTED = -1, -2, -3


@pytest.mark.parametrize("bad,code", [
    (dict(type=3), EINVAL), (dict(weight_type=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(eps=-1e-9), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(x=NULL), EINVAL), (dict(y=NULL), EINVAL), (dict(x=ODD), EINVAL),
    (dict(type=1, x=ODD), EINVAL), (dict(x_stride=7), EINVAL), (dict(y_stride=7), EINVAL), (dict(y_stride=9), EINVAL), (dict(weight=ODD), EINVAL),
    (dict(mean=4098), EINVAL), (dict(x_stride=1 << 61), EINVAL), (dict(cols=1 << 31, x_stride=1 << 31, y_stride=1 << 31), EUNSUPPORTED),
    (dict(rows=(1 << 40) + 1), EUNSUPPORTED)])
def test_layer_norm_forward_refuses(T, bad, code):
    assert _norm_forward(T, **bad) == code and T.B.lib().p2_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(type=9), EINVAL), (dict(dy=NULL), EINVAL), (dict(mean=NULL), EINVAL), (dict(rstd=NULL), EINVAL), (dict(dy_stride=7), EINVAL),
    (dict(dx_stride=7), EINVAL), (dict(dx=ODD), EINVAL), (dict(dweight=ODD), EINVAL), (dict(workspace=NULL), EINVAL), (dict(workspace=4096 + 128), EINVAL),
    (dict(workspace_bytes=16), ENOSPC), (dict(cols=0), EINVAL), (dict(dx_stride=9), EINVAL)])
def test_layer_norm_backward_refuses(T, bad, code):
    assert _norm_backward(T, **bad) == code and T.B.lib().p2_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(type=4), EINVAL), (dict(tokens=-1), EINVAL), (dict(experts=0), EINVAL), (dict(k=0), EINVAL), (dict(k=9), EINVAL), (dict(stride=7), EINVAL),
    (dict(logits=NULL), EINVAL), (dict(logits=ODD), EINVAL), (dict(expert=NULL), EINVAL), (dict(gate=NULL), EINVAL), (dict(counts=NULL), EINVAL),
    (dict(counts=4100), EINVAL), (dict(loss=NULL), EINVAL), (dict(experts=1025, stride=1025), EUNSUPPORTED),
    (dict(experts=100, stride=100, k=65), EUNSUPPORTED), (dict(tokens=100000, workspace=NULL), EINVAL), (dict(tokens=100000, workspace_bytes=64), ENOSPC)])
def test_balance_forward_refuses(T, bad, code):
    assert _balance_forward(T, **bad) == code and T.B.lib().p2_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(type=4), EINVAL), (dict(k=0), EINVAL), (dict(dlogits=NULL), EINVAL), (dict(counts=NULL), EINVAL), (dict(kept=NULL), EINVAL),
    (dict(expert=NULL), EINVAL), (dict(dlogits_stride=7), EINVAL), (dict(dlogits_stride=9), EINVAL), (dict(dgate=4098), EINVAL)])
def test_balance_backward_refuses(T, bad, code):
    assert _balance_backward(T, **bad) == code and T.B.lib().p2_last_error()


def test_balance_loss_refuses(T):
    f = T.lib().p2_balance_loss
    assert f(NULL, P, P, 8, 2, P, None) == EINVAL and f(P, P, P, 8, 9, P, None) == EINVAL and f(P, P, P, 2000, 2, P, None) == EUNSUPPORTED
    assert f(P, P, 4100, 8, 2, P, None) == EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(type=3), EINVAL), (dict(out_type=3), EINVAL), (dict(count=-1), EINVAL), (dict(rows=0), EINVAL), (dict(cols=0), EINVAL), (dict(steps=0), EINVAL),
    (dict(steps=65), EINVAL), (dict(coefficients=None), EINVAL), (dict(coefficients=(1.0, float("nan"), 0.0)), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(scale=float("inf")), EINVAL), (dict(g=NULL), EINVAL), (dict(out=ODD), EINVAL), (dict(stride=7), EINVAL), (dict(out_stride=7), EINVAL),
    (dict(count=2, out_matrix_stride=100), EINVAL), (dict(count=2, matrix_stride=-1), EINVAL), (dict(workspace=NULL, rows=300, cols=200, stride=200, out_stride=200), EINVAL),
    (dict(workspace_bytes=1000, rows=300, cols=200, stride=200, out_stride=200), ENOSPC), (dict(rows=(1 << 17) + 1), EUNSUPPORTED),
    (dict(count=65536, out_matrix_stride=4096), EUNSUPPORTED), (dict(count=4, rows=1 << 17, cols=1 << 17, stride=1 << 17, out_stride=1 << 17, matrix_stride=1 << 34, out_matrix_stride=1 << 34), EUNSUPPORTED),
    (dict(coefficients=(11.0, 0.0, 0.0)), EUNSUPPORTED), (dict(coefficients=(3.0, -4.0, 2.5), steps=64), EUNSUPPORTED)])
def test_orthogonalize_refuses(T, bad, code):
    assert _orthogonalize(T, **bad) == code and T.B.lib().p2_last_error()


def test_nothing_to_do_is_no_error(T):
    assert _norm_forward(T, rows=0, x=NULL, y=NULL, mean=NULL, rstd=NULL) == 0
    assert _norm_backward(T, rows=0, dweight=NULL, dbias=NULL, workspace=NULL) == 0
    assert _norm_backward(T, dx=NULL, dweight=NULL, dbias=NULL, workspace=NULL) == 0
    assert _balance_backward(T, tokens=0) == 0
    assert _orthogonalize(T, count=0) == 0


def test_workspaces(T):
    n = C.c_int64()
    L = T.lib()
    assert L.p2_layer_norm_backward_workspace(100, 64, C.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0
    assert L.p2_layer_norm_backward_workspace(-1, 64, C.byref(n)) == EINVAL
    assert L.p2_layer_norm_backward_workspace(100, 64, None) == EINVAL
    assert L.p2_balance_forward_workspace(1, 64, C.byref(n)) == 0 and n.value == 0
    assert L.p2_balance_forward_workspace(1 << 20, 64, C.byref(n)) == 0 and n.value > 0
    assert L.p2_balance_forward_workspace(5, 0, C.byref(n)) == EINVAL
    assert L.p2_orthogonalize_workspace(3, 64, 64, C.byref(n)) == 0 and n.value == 0
    assert L.p2_orthogonalize_workspace(1, 4096, 4096, C.byref(n)) == 0 and n.value >= 5 * 4 * 4096 * 4096
    assert L.p2_orthogonalize_workspace(1, 0, 4, C.byref(n)) == EINVAL


def test_tensors_elsewhere_or_of_other_types_are_refused(T):
    x = torch.ones(4, 8)
    refused = [lambda: T.p2_layer_norm_forward(x), lambda: T.p2_layer_norm_backward(x, x, None, x[:, 0], x[:, 0]), lambda: T.p2_balance_forward(x, 2),
               lambda: T.p2_orthogonalize(x), lambda: T.p2_orthogonalize(x[0]), lambda: T.p2_balance_forward(x[0], 1),
               lambda: T.p2_layer_norm_backward(x, x[:2], None, x[:, 0], x[:, 0]), lambda: T.p2_layer_norm_forward(torch.tensor(1.0)),
               lambda: T.p2_orthogonalize(x, coefficients=(1.0, 2.0))]
    for call in refused:
        with pytest.raises(T.P2Error) as e:
            call()
        assert e.value.code == EINVAL


def test_arguments_that_require_a_gradient_bring_a_warning(T):
    """No rows: nothing is queued, so the extension module's calls need no GPU (the entry points look at the device first)."""
    calls = T._native_calls()
    x, w, g = torch.zeros(0, 8), torch.ones(8), torch.zeros(0, 5, 7)
    m, expert, counts, tokens = torch.zeros(0), torch.zeros(0, 2, dtype=torch.int32), torch.zeros(8, dtype=torch.int64), torch.zeros((), dtype=torch.int64)
    one = torch.ones(())

    def all_of(grad):
        p = {n: t.clone().requires_grad_(n == grad) for n, t in dict(x=x, w=w, g=g, one=one).items()}
        calls.layer_norm_forward(p["x"], p["w"], None, 1e-5, 0)
        calls.layer_norm_backward(p["x"], p["x"], p["w"], m, m, True, False, False, 0)
        calls.balance_backward(p["x"], expert, counts, tokens, None, None, p["one"], 0)
        calls.orthogonalize(p["g"], 5, *T.NEWTON_SCHULZ, 1e-7, 1.0, -1, 0)

    for grad, count in (("x", 3), ("w", 2), ("g", 1), ("one", 1), (None, 0)):
        with warnings.catch_warnings(record=True) as caught:
            warnings.simplefilter("always")
            all_of(grad)
        assert [c.category for c in caught] == [UserWarning] * count and all("autograd" in str(c.message) for c in caught)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad():
            all_of("x")
        with pytest.raises(UserWarning):                   # (a warning that is an error is one here, too)
            all_of("x")
