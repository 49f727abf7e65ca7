"""Refusals of routing, AdamW and matrix products: they come before anything is queued, so no GPU is needed (pointers are made up)."""
import ctypes as C
import os

import pytest
import torch

EINVAL, ENOSPC, EUNSUPPORTED = -1, -2, -3
P, ODD, NULL = 4096, 4097, None      # an aligned pointer, one that is aligned to nothing, none
NAN, INF = float("nan"), float("inf")
LONG = dict(inner=8192, x_stride=8192, weight_stride=8192)      # a product whose sum is cut into parts, which need room


@pytest.fixture(scope="module")
def T():
    from paper_2110_10548_amd import binding, train
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    train.lib()
    return train


def _route_forward(T, **kw):
    a = dict(logits=P, type=0, stride=8, keep=NULL, bias=P, tokens=4, experts=8, k=2, score=0, groups=2, group_limit=1, group_best=2, renormalise=1, scale=1.0,
             expert=P, gate=P, counts=P, kept=P, workspace=P, workspace_bytes=1 << 24) | kw
    return T.lib().p2_route_forward(*a.values(), None)


def _route_backward(T, **kw):
    a = dict(logits=P, type=0, stride=8, tokens=4, experts=8, k=2, score=0, renormalise=1, scale=1.0, expert=P, dgate=P, dlogits=2 * P, dlogits_stride=8) | kw
    return T.lib().p2_route_backward(*a.values(), None)


def _square_sum(T, pointers=(P, P), counts=(10, 20), **kw):
    n = len(counts)
    a = dict(tensors=(C.c_void_p * max(n, 1))(*pointers), counts=(C.c_int64 * max(n, 1))(*counts), n=n, type=0, out=P, workspace=P, workspace_bytes=1 << 20) | kw
    return T.lib().p2_square_sum(*a.values(), None)


def _tensor(T, **kw):
    a = dict(param=1 << 12, grad=1 << 20, copy=NULL, mean=1 << 16, square=1 << 17, mean_scale=1 << 18, square_scale=1 << 19, count=100) | kw
    return T.AdamwTensor(*a.values())


def _adamw(T, tensors=None, **kw):
    tensors = [_tensor(T)] if tensors is None else tensors
    a = dict(tensors=(T.AdamwTensor * max(len(tensors), 1))(*tensors), n=len(tensors), type=0, grad_type=0, copy_type=0, state_bits=32, step=P, rate=NULL, lr=1e-3,
             beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, grad_factor=1.0, square_sum=P, max_norm=1.0, workspace=P, workspace_bytes=256) | kw
    return T.lib().p2_adamw(*a.values(), None)


def _values(T, tensors, mean=(P,), square=(P,)):
    return T.lib().p2_adamw_values((T.AdamwTensor * max(len(tensors), 1))(*tensors), len(tensors), (C.c_void_p * max(len(mean), 1))(*mean),
                                   (C.c_void_p * max(len(square), 1))(*square), None)


def _linear_forward(T, **kw):
    a = dict(x=P, x_stride=8, weight=2 * P, weight_stride=8, bias=P, residual=4 * P, residual_stride=16, type=0, activation=4, rows=100, inner=8, outer=16, y=3 * P,
             y_stride=16, z=5 * P, z_stride=16, workspace=P, workspace_bytes=1 << 20) | kw
    return T.lib().p2_linear_forward(*a.values(), None)


def _linear_backward(T, **kw):
    a = dict(dy=P, dy_stride=16, z=2 * P, z_stride=16, x=3 * P, x_stride=8, weight=4 * P, weight_stride=8, type=0, activation=1, rows=100, inner=8, outer=16, dx=5 * P,
             dx_stride=8, dweight=6 * P, dweight_stride=8, dbias=P, weight_type=0, workspace=P, workspace_bytes=1 << 22) | kw
    return T.lib().p2_linear_backward(*a.values(), None)


@pytest.mark.parametrize("bad,code", [
    (dict(type=3), EINVAL), (dict(tokens=-1), EINVAL), (dict(experts=0), EINVAL), (dict(k=0), EINVAL), (dict(k=9), EINVAL), (dict(stride=7), EINVAL),
    (dict(score=2), EINVAL), (dict(score=-1), EINVAL), (dict(groups=3), EINVAL), (dict(groups=0), EINVAL), (dict(group_limit=0), EINVAL), (dict(group_limit=3), EINVAL),
    (dict(group_best=0), EINVAL), (dict(group_best=3), EINVAL), (dict(scale=NAN), EINVAL), (dict(scale=INF), EINVAL), (dict(logits=NULL), EINVAL), (dict(logits=ODD), EINVAL),
    (dict(bias=4098), EINVAL), (dict(expert=NULL), EINVAL), (dict(gate=NULL), EINVAL), (dict(counts=NULL), EINVAL), (dict(kept=NULL), EINVAL), (dict(kept=4100), EINVAL),
    (dict(counts=4100), EINVAL), (dict(experts=1026, stride=1026), EUNSUPPORTED), (dict(experts=130, stride=130, groups=65), EUNSUPPORTED),
    (dict(experts=100, stride=100, k=65), EUNSUPPORTED), (dict(tokens=100000, workspace=NULL), EINVAL), (dict(tokens=100000, workspace=P + 128), EINVAL),
    (dict(tokens=100000, workspace_bytes=64), ENOSPC), (dict(stride=1 << 61), EINVAL)])
def test_route_forward_refuses(T, bad, code):
    assert _route_forward(T, **bad) == code and T.B.lib().p2_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(type=4), EINVAL), (dict(k=0), EINVAL), (dict(score=5), EINVAL), (dict(scale=INF), EINVAL), (dict(dlogits=NULL), EINVAL), (dict(expert=NULL), EINVAL),
    (dict(dgate=NULL), EINVAL), (dict(dgate=4098), EINVAL), (dict(dlogits_stride=7), EINVAL), (dict(dlogits=P, dlogits_stride=9), EINVAL), (dict(logits=ODD), EINVAL)])
def test_route_backward_refuses(T, bad, code):
    assert _route_backward(T, **bad) == code and T.B.lib().p2_last_error()


def test_route_bias_refuses(T):
    f = T.lib().p2_route_bias
    for args, code in (((NULL, P, 8, 0.1, P), EINVAL), ((P, NULL, 8, 0.1, P), EINVAL), ((P, P, 8, 0.1, NULL), EINVAL), ((P, P, 0, 0.1, P), EINVAL), ((P, P, 8, NAN, P), EINVAL),
                       ((P, 4100, 8, 0.1, P), EINVAL), ((4098, P, 8, 0.1, P), EINVAL), ((P, P, 1025, 0.1, P), EUNSUPPORTED)):
        assert f(*args, None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(type=3), EINVAL), (dict(counts=(-1, 5)), EINVAL), (dict(pointers=(NULL, P)), EINVAL), (dict(pointers=(ODD, P)), EINVAL), (dict(out=NULL), EINVAL),
    (dict(out=4100), EINVAL), (dict(workspace=NULL), EINVAL), (dict(workspace=P + 8), EINVAL), (dict(workspace_bytes=100), ENOSPC), (dict(n=-1), EINVAL), (dict(tensors=None), EINVAL),
    (dict(counts=((1 << 40) + 1, 5)), EUNSUPPORTED), (dict(counts=(1 << 40, 5)), EUNSUPPORTED), (dict(n=(1 << 20) + 1), EUNSUPPORTED)])
def test_square_sum_refuses(T, bad, code):
    assert _square_sum(T, **bad) == code and T.B.lib().p2_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(type=3), EINVAL), (dict(grad_type=3), EINVAL), (dict(copy_type=-1), EINVAL), (dict(state_bits=16), EINVAL), (dict(beta1=1.0), EINVAL), (dict(beta2=-0.1), EINVAL),
    (dict(beta1=NAN), EINVAL), (dict(lr=INF), EINVAL), (dict(weight_decay=NAN), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=INF), EINVAL), (dict(eps=NAN), EINVAL),
    (dict(grad_factor=0.0), EINVAL), (dict(grad_factor=INF), EINVAL), (dict(max_norm=0.0), EINVAL), (dict(max_norm=NAN), EINVAL), (dict(step=NULL), EINVAL),
    (dict(step=4100), EINVAL), (dict(rate=4098), EINVAL), (dict(square_sum=4100), EINVAL), (dict(workspace=NULL), EINVAL), (dict(workspace_bytes=8), ENOSPC),
    (dict(state_bits=8, eps=1e-15), EUNSUPPORTED), (dict(tensors=None, n=-1), EINVAL)])
def test_adamw_refuses(T, bad, code):
    assert _adamw(T, **bad) == code and T.B.lib().p2_last_error()


@pytest.mark.parametrize("tensor,more", [
    (dict(param=NULL), {}), (dict(grad=NULL), {}), (dict(mean=NULL), {}), (dict(square=NULL), {}), (dict(count=-1), {}), (dict(param=ODD), {}), (dict(mean=(1 << 16) + 2), {}),
    (dict(mean_scale=NULL), dict(state_bits=8)), (dict(square_scale=NULL), dict(state_bits=8)), (dict(grad=ODD), dict(grad_type=1)), (dict(copy=ODD), dict(copy_type=1)),
    (dict(mean=1 << 12), {}), (dict(square=(1 << 16) + 396), {}), (dict(copy=(1 << 12) + 4), {})])
def test_adamw_refuses_tensors(T, tensor, more):
    assert _adamw(T, [_tensor(T, **tensor)], **more) == EINVAL and T.B.lib().p2_last_error()


def test_adamw_refuses_a_tensor_that_is_listed_twice(T):
    assert _adamw(T, [_tensor(T), _tensor(T)]) == EINVAL and b"overlap" in T.B.lib().p2_last_error()
    assert _adamw(T, [_tensor(T), _tensor(T, param=1 << 13, mean=(1 << 16) + 4 * 99, square=1 << 21)]) == EINVAL
    assert _adamw(T, [_tensor(T, count=(1 << 40) + 1)]) == EUNSUPPORTED


@pytest.mark.parametrize("tensor,more", [
    (dict(mean_scale=1 << 19), dict(state_bits=8)), (dict(square_scale=(1 << 18) + 4, count=300), dict(state_bits=8)), (dict(mean_scale=(1 << 16) + 96), dict(state_bits=8)),
    (dict(grad=1 << 12), {}), (dict(grad=(1 << 16) + 396), {}), (dict(grad=(1 << 16) - 4), {}), (dict(grad=(1 << 17) - 198), dict(grad_type=1)),
    (dict(copy=(1 << 20)), dict(copy_type=1)), (dict(copy=(1 << 20) + 4), {})])
def test_adamw_refuses_gradients_and_scales_in_what_is_written(T, tensor, more):
    assert _adamw(T, [_tensor(T, **tensor)], **more) == EINVAL and b"overlap" in T.B.lib().p2_last_error()


@pytest.mark.parametrize("tensor,mean,square", [(dict(mean=NULL), (P,), (P,)), (dict(square_scale=NULL), (P,), (P,)), (dict(), (ODD,), (P,)), (dict(), (P,), (4098,)),
                                                (dict(count=-1), (P,), (P,))])
def test_adamw_values_refuses(T, tensor, mean, square):
    assert _values(T, [_tensor(T, **tensor)], mean, square) == EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(type=3), EINVAL), (dict(activation=5), EINVAL), (dict(activation=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(inner=0), EINVAL), (dict(outer=0), EINVAL),
    (dict(x=NULL), EINVAL), (dict(weight=NULL), EINVAL), (dict(y=NULL), EINVAL), (dict(x=ODD), EINVAL), (dict(bias=ODD), EINVAL), (dict(x_stride=7), EINVAL),
    (dict(weight_stride=7), EINVAL), (dict(residual_stride=15), EINVAL), (dict(z_stride=15), EINVAL), (dict(y_stride=15), EINVAL), (dict(residual=3 * P, residual_stride=17), EINVAL),
    (dict(y=P), EINVAL), (dict(y=2 * P), EINVAL), (dict(y=5 * P), EINVAL), (dict(z=P), EINVAL), (dict(z=2 * P), EINVAL), (dict(z=4 * P), EINVAL), (dict(rows=(1 << 20) + 1), EUNSUPPORTED),
    (dict(inner=(1 << 20) + 1, x_stride=1 << 21, weight_stride=1 << 21), EUNSUPPORTED), (dict(outer=(1 << 20) + 1, y_stride=1 << 21), EUNSUPPORTED),
    (dict(LONG, workspace=NULL), EINVAL), (dict(LONG, workspace=P + 64), EINVAL), (dict(LONG, workspace_bytes=100), ENOSPC)])
def test_linear_forward_refuses(T, bad, code):
    assert _linear_forward(T, **bad) == code and T.B.lib().p2_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(type=3), EINVAL), (dict(weight_type=3), EINVAL), (dict(activation=7), EINVAL), (dict(rows=-1), EINVAL), (dict(dy=NULL), EINVAL), (dict(z=NULL), EINVAL),
    (dict(x=NULL), EINVAL), (dict(weight=NULL), EINVAL), (dict(dx=ODD), EINVAL), (dict(dweight=ODD), EINVAL), (dict(dbias=ODD), EINVAL), (dict(dy_stride=15), EINVAL),
    (dict(dx_stride=7), EINVAL), (dict(dweight_stride=7), EINVAL), (dict(dx=P), EINVAL), (dict(dx=3 * P), EINVAL), (dict(dx=6 * P), EINVAL), (dict(dweight=P), EINVAL), (dict(dweight=2 * P), EINVAL), (dict(dweight=3 * P), EINVAL), (dict(dweight=4 * P), EINVAL), (dict(workspace=NULL), EINVAL),
    (dict(workspace_bytes=100), ENOSPC), (dict(rows=(1 << 20) + 1), EUNSUPPORTED)])
def test_linear_backward_refuses(T, bad, code):
    assert _linear_backward(T, **bad) == code and T.B.lib().p2_last_error()


def test_nothing_to_do_is_no_error(T):
    assert _route_backward(T, tokens=0) == 0
    assert _linear_forward(T, rows=0, x=NULL, y=NULL, z=NULL, residual=NULL, workspace=NULL, workspace_bytes=0) == 0
    assert _linear_backward(T, rows=0, dweight=NULL, dbias=NULL, workspace=NULL, workspace_bytes=0) == 0
    assert _values(T, []) == 0
    assert _values(T, [_tensor(T, mean=NULL, square=NULL)], (NULL,), (NULL,)) == 0


def test_workspaces(T):
    n, L = C.c_int64(), T.lib()
    assert L.p2_route_forward_workspace(1, 64, 2, 4, C.byref(n)) == 0 and n.value == 0
    assert L.p2_route_forward_workspace(1 << 20, 64, 2, 4, C.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0
    assert L.p2_route_forward_workspace(5, 64, 65, 1, C.byref(n)) == EINVAL and L.p2_route_forward_workspace(5, 64, 2, 4, None) == EINVAL
    assert L.p2_square_sum_workspace(0, C.byref(n)) == 0 and n.value > 0 and L.p2_square_sum_workspace(-1, C.byref(n)) == EINVAL
    assert L.p2_adamw_workspace(C.byref(n)) == 0 and n.value == 256 and L.p2_adamw_workspace(None) == EINVAL
    aligned = (1, 64, 1000, 64, 1000)
    assert L.p2_linear_forward_workspace(P, 64, 2 * P, 64, 1, 4096, 64, 4096, C.byref(n)) == 0 and n.value == 0, aligned
    assert L.p2_linear_forward_workspace(P + 2, 64, 2 * P, 64, 1, 4096, 64, 4096, C.byref(n)) == 0 and n.value >= 4096 * 128
    assert L.p2_linear_forward_workspace(P, 63, 2 * P, 63, 1, 4096, 63, 4096, C.byref(n)) == 0 and n.value >= 2 * 4096 * 126
    assert L.p2_linear_backward_workspace(1, 4096, 64, 4096, C.byref(n)) == 0 and n.value > 0 and L.p2_linear_backward_workspace(1, 0, 64, 64, C.byref(n)) == 0 and n.value == 0
    assert L.p2_linear_backward_workspace(3, 1, 64, 64, C.byref(n)) == EINVAL


@pytest.mark.parametrize("tokens,needed", [(0, False), (1, False), (16, False), (17, True), (32, True), (33, True)])
def test_the_choice_s_workspace_is_enough_with_and_without_a_bias(T, tokens, needed):
    n = C.c_int64()
    assert T.lib().p2_route_forward_workspace(tokens, 256, 8, 8, C.byref(n)) == 0 and (n.value > 0) == needed
    if needed:
        for bias in (NULL, P):
            assert _route_forward(T, tokens=tokens, experts=256, stride=256, k=8, groups=8, bias=bias, workspace=NULL, workspace_bytes=0) == EINVAL


def test_tensors_elsewhere_or_of_other_kinds_are_refused(T):
    x, i = torch.ones(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    s = T.p2_adamw_state([x])
    refused = [lambda: T.p2_route_forward(x, 2), lambda: T.p2_route_forward(x[0], 1), lambda: T.p2_route_forward(x, 2, score="relu"), lambda: T.p2_route_backward(x, i, x[:, :2]),
               lambda: T.p2_route_backward(x[0], i, x[:, :2]), lambda: T.p2_route_bias(x[0], i, 0.1), lambda: T.p2_square_sum([x]), lambda: T.p2_square_sum([]),
               lambda: T.p2_adamw([x], [x], **s), lambda: T.p2_adamw([], [], [], [], s["step"]), lambda: T.p2_adamw([x], [x], **s, max_norm=1.0),
               lambda: T.p2_adamw([x], [x], **s, betas=(0.9,)), lambda: T.p2_adamw_state([x], bits=16), lambda: T.p2_adamw_values([], [], [], []),
               lambda: T.p2_linear_forward(x, x), lambda: T.p2_linear_forward(torch.tensor(1.0), x), lambda: T.p2_linear_forward(x, x, activation="tanh"),
               lambda: T.p2_linear_backward(x, x, x, dtype=torch.int32), lambda: T.p2_linear_backward(x, x, x)]
    for call in refused:
        with pytest.raises(T.P2Error) as e:
            call()
        assert e.value.code == EINVAL


def test_the_extension_module_refuses(T):
    """Shapes, types and lists, seen to before the library is called (the entry points look at the device first)."""
    calls = T._native_calls()
    f, h, i64 = torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.float16), torch.zeros((), dtype=torch.int64)
    e = torch.zeros(4, 2, dtype=torch.int32)
    w = torch.zeros(6, 8)
    many = dict(params=[f], grads=[f], means=[f], squares=[f], step=i64, mean_scales=None, square_scales=None, copies=None, rate=None, lr=1e-3, beta1=0.9, beta2=0.9, eps=1e-8,
                decay=0.0, factor=1.0, square_sum=None, most=1.0)
    small = dict(means=[f.to(torch.int8)], squares=[f.to(torch.uint8)], mean_scales=[f[0, :1]], square_scales=[f[0, :1]])
    for bad in (dict(grads=[]), dict(grads=[w]), dict(grads=[f, f]), dict(means=[h]), dict(squares=[f.t().contiguous().t()]), dict(step=f), dict(rate=f), dict(square_sum=f[0, 0]),
                dict(copies=[w]), dict(copies=[f, f]), dict(params=[f.t()], grads=[f.t()], means=[f.t()], squares=[f.t()]), dict(params=[f, h], grads=[f, f], means=[f, f], squares=[f, f]),
                small | dict(mean_scales=None), small | dict(mean_scales=[f]), small | dict(squares=[f])):
        with pytest.raises(T.P2Error):
            calls.adamw(*(many | bad).values(), 0)
    refused = [lambda: calls.linear_forward(f, w[:, :7], None, 0, None, False, 0), lambda: calls.linear_forward(f, w.half(), None, 0, None, False, 0),
               lambda: calls.linear_forward(f, w, f[0], 0, None, False, 0), lambda: calls.linear_forward(f, w, None, 0, f, False, 0),
               lambda: calls.linear_forward(f, w, torch.zeros(6).half(), 0, None, False, 0), lambda: calls.linear_forward(f.int(), w, None, 0, None, False, 0),
               lambda: calls.linear_backward(f, f, w, None, 0, True, True, True, -1, 0), lambda: calls.linear_backward(f[:, :6], f, w, None, 1, True, True, True, -1, 0),
               lambda: calls.linear_backward(f[:, :6], f, w, f, 1, True, True, True, -1, 0), lambda: calls.linear_backward(h[:, :6], f, w, None, 0, True, True, True, -1, 0),
               lambda: calls.route_backward(f, e.long(), f[:, :2], 0, False, 1.0, 0), lambda: calls.route_backward(f, e, f, 0, False, 1.0, 0),
               lambda: calls.route_forward(f, 2, 0, f[:, 0], None, 1, 1, 1, False, 1.0, 0), lambda: calls.route_forward(f, 2, 0, f[0].double(), None, 1, 1, 1, False, 1.0, 0),
               lambda: calls.route_forward(f, 2, 0, None, torch.ones(3, dtype=torch.bool), 1, 1, 1, False, 1.0, 0), lambda: calls.route_forward(f, 9, 0, None, None, 1, 1, 1, False, 1.0, 0),
               lambda: calls.route_bias(f, i64, 0.1, 0), lambda: calls.route_bias(f[0], torch.zeros(7, dtype=torch.int64), 0.1, 0), lambda: calls.square_sum([f, h], 0),
               lambda: calls.square_sum([e], 0), lambda: calls.adamw_values([f], [f], [f], [f], 0)]
    for call in refused:
        with pytest.raises(T.P2Error):
            call()
    for call in (lambda: calls.square_sum(5, 0), lambda: calls.square_sum([5], 0), lambda: calls.linear_forward(f, 3, None, 0, None, False, 0)):
        with pytest.raises(TypeError):
            call()


def test_states_have_their_tensors_shapes(T):
    p = [torch.zeros(3, 100), torch.zeros(0), torch.zeros(257), torch.zeros(())]
    s = T.p2_adamw_state(p, 8)
    assert [m.shape for m in s["means"]] == [t.shape for t in p] and [v.numel() for v in s["mean_scales"]] == [2, 0, 2, 1]
    assert s["means"][0].dtype == torch.int8 and s["squares"][0].dtype == torch.uint8 and s["step"].dtype == torch.int64
    s = T.p2_adamw_state(p)
    assert s["mean_scales"] is None and s["means"][0].dtype == torch.float32


def test_tensors_that_stand_for_shapes_alone_are_refused(T):
    """Under a mode that follows shapes, and its tensors outside of it: no result without values, and no argument taken for one that is not given."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    calls = T._native_calls()
    with FakeTensorMode():
        q, s, x, w = torch.zeros(300, dtype=torch.int8, device="cuda:0"), torch.zeros(2, device="cuda:0"), torch.zeros(4, 8, device="cuda:0"), torch.zeros(8, device="cuda:0")
        u, n = q.to(torch.uint8), torch.zeros((), dtype=torch.int64, device="cuda:0")
        w2 = torch.zeros(6, 8, device="cuda:0")
    meta = [t.to("meta") for t in (torch.zeros(300, dtype=torch.int8), torch.zeros(300, dtype=torch.uint8), torch.zeros(2), torch.zeros(2))]

    def refused(call):
        with pytest.raises(T.P2Error) as e:
            call()
        assert e.value.code == EINVAL and "no values" in str(e.value)

    with FakeTensorMode(allow_non_fake_inputs=True):
        refused(lambda: calls.adamw_values([q], [u], [s], [s], 0))
        refused(lambda: calls.layer_norm_forward(x, w, None, 1e-5, 0))
        refused(lambda: calls.linear_forward(x, w2, None, 0, None, False, 0))
        refused(lambda: calls.adamw([x], [x], [x], [x], n, None, None, None, None, 1e-3, 0.9, 0.9, 1e-8, 0.0, 1.0, None, 1.0, 0))
    refused(lambda: calls.adamw_values(*([t] for t in meta), 0))
    refused(lambda: calls.square_sum([meta[2]], 0))


Q = 1 << 20                          # far apart
APART = dict(x=1 * Q, weight=2 * Q, bias=3 * Q, residual=4 * Q, y=5 * Q, z=6 * Q, workspace=7 * Q)
APART_BACKWARD = dict(dy=1 * Q, z=2 * Q, x=3 * Q, weight=4 * Q, dx=5 * Q, dweight=6 * Q, dbias=7 * Q, workspace=8 * Q)


@pytest.mark.parametrize("bad", [
    dict(y=Q + 4), dict(y=Q - 64 * 100 + 4), dict(y=2 * Q + 32 * 15), dict(y=3 * Q - 4), dict(y=4 * Q + 4), dict(y=6 * Q + 64 * 99 + 60), dict(z=Q + 32 * 99 + 28), dict(z=2 * Q - 4),
    dict(z=3 * Q), dict(z=4 * Q + 60), dict(z=5 * Q - 60),
    dict(x_stride=40, y_stride=40, y=Q + 28), dict(x_stride=40, y_stride=40, y=Q + 160 * 3 + 28), dict(x_stride=40, y_stride=40, y=Q - 160 * 99 - 60),         # columns of one buffer, one of them both's
    dict(x_stride=24, y_stride=24, y=Q + 36), dict(x_stride=40, y_stride=41, y=Q + 32), dict(y_stride=40, z_stride=40, z=5 * Q + 60), dict(y_stride=40, z_stride=40, z=5 * Q + 100),
    dict(residual_stride=40, y_stride=40, y=4 * Q + 160), dict(rows=1, residual_stride=40, y=4 * Q + 4), dict(LONG, workspace=5 * Q), dict(LONG, workspace=2 * Q)])
def test_linear_forward_refuses_results_in_what_it_reads_or_writes(T, bad):
    assert _linear_forward(T, **(APART | bad)) == EINVAL and b"overlap" in T.B.lib().p2_last_error()


@pytest.mark.parametrize("bad", [
    dict(dx=Q + 4), dict(dx=2 * Q + 64 * 99 + 60), dict(dx=3 * Q - 4), dict(dx=4 * Q + 32 * 15 + 28), dict(dx=6 * Q + 8), dict(dx=7 * Q), dict(dweight=Q - 4), dict(dweight=2 * Q + 4), dict(dweight=3 * Q + 4),
    dict(dweight=4 * Q + 4, dx=NULL, weight=4 * Q, dy=4 * Q + 64), dict(dbias=Q + 4), dict(dbias=2 * Q - 4), dict(dbias=3 * Q + 12), dict(dbias=4 * Q), dict(dbias=5 * Q + 32 * 99 + 28), dict(dbias=6 * Q),
    dict(rows=0, dbias=6 * Q + 4), dict(rows=1, dx=Q + 60), dict(workspace=Q), dict(workspace=5 * Q), dict(workspace=7 * Q), dict(dx_stride=40, x_stride=40, dx=3 * Q + 28),
    dict(dx_stride=40, x_stride=40, dx=3 * Q + 160 * 5 - 4), dict(dx_stride=40, dy_stride=41, dx=Q + 80), dict(weight_type=1, dbias=6 * Q + 16 * 15 + 14)])
def test_linear_backward_refuses_results_in_what_it_reads_or_writes(T, bad):
    assert _linear_backward(T, **(APART_BACKWARD | bad)) == EINVAL and b"overlap" in T.B.lib().p2_last_error()


@pytest.mark.parametrize("bad", [
    dict(step=1 << 12), dict(step=(1 << 16) + 392), dict(step=(1 << 17) - 8, tensor=dict(square=(1 << 17) - 4)), dict(step=1 << 20), dict(square_sum=1 << 12), dict(square_sum=(1 << 16) + 8),
    dict(rate=(1 << 17) + 396), dict(step=1 << 22, square_sum=1 << 22), dict(step=1 << 22, rate=(1 << 22) + 4), dict(workspace=1 << 16), dict(workspace=1 << 20), dict(workspace=1 << 21),
    dict(workspace=1 << 23, step=(1 << 23) + 8), dict(workspace=1 << 23, rate=(1 << 23) + 8)])
def test_adamw_refuses_its_numbers_in_what_it_reads_or_writes(T, bad):
    a = dict(step=1 << 21, square_sum=NULL, workspace=1 << 24) | bad
    tensor = a.pop("tensor", {})
    assert _adamw(T, [_tensor(T, **tensor)], **a) == EINVAL and b"overlap" in T.B.lib().p2_last_error()


def _rooms(T, rows, inner, outer, kind=1, activation=0, wanted=(1, 1, 1), dy=P, x=P, weight=P, pad=0):
    n, most = C.c_int64(), C.c_int64()
    assert T.lib().p2_linear_backward_workspace_for(dy, outer + pad, x, inner + pad, weight, inner + pad, kind, activation, rows, inner, outer, *wanted, C.byref(n)) == 0
    assert T.lib().p2_linear_backward_workspace(kind, rows, inner, outer, C.byref(most)) == 0 and n.value <= most.value and n.value % 256 == 0
    return n.value, most.value


def test_gradients_take_room_for_what_they_use(T):
    mib = 1 << 20
    lines = 128 * 4096 * 4
    assert _rooms(T, 8192, 4096, 4096)[0] == lines                                     # operands that are taken as they lie in memory
    assert _rooms(T, 8192, 4096, 4096, activation=2)[0] == 64 * mib + lines            # dz
    assert _rooms(T, 8192, 4096, 4096, activation=2, wanted=(1, 1, 0))[0] == 64 * mib
    assert _rooms(T, 8192, 4096, 4096, wanted=(0, 0, 1))[0] == lines
    assert _rooms(T, 8192, 4096, 4096, wanted=(0, 0, 0))[0] == 0
    everything, most = _rooms(T, 8192, 4096, 4096, activation=2, x=P + 2, weight=P + 2)
    assert everything == most
    assert _rooms(T, 1, 64, 4096, wanted=(0, 1, 1))[0] == 0 and _rooms(T, 1, 64, 4096, wanted=(1, 0, 0))[0] > 0
    assert _rooms(T, 0, 64, 64) == (0, 0)
    for rows, inner, outer, kind in ((100, 300, 200, 0), (2001, 1023, 515, 2), (16384, 512, 2048, 1), (5, 700, 900, 1), (64, 40, 70, 1)):
        parts = [_rooms(T, rows, inner, outer, kind, activation=1, wanted=w)[0] for w in ((1, 0, 0), (0, 1, 0), (0, 0, 1))]
        assert max(parts) <= _rooms(T, rows, inner, outer, kind, activation=1)[0] <= sum(parts)
    n, f = C.c_int64(), T.lib().p2_linear_backward_workspace_for
    for bad, code in ((dict(kind=3), EINVAL), (dict(rows=-1), EINVAL), (dict(activation=5), EINVAL), (dict(outer=0), EINVAL), (dict(inner=(1 << 20) + 1), EUNSUPPORTED)):
        a = dict(kind=1, activation=0, rows=10, inner=64, outer=64) | bad
        assert f(P, 64, P, 64, P, 64, *a.values(), 1, 1, 1, C.byref(n)) == code
    assert f(P, 64, P, 64, P, 64, 1, 0, 10, 64, 64, 1, 1, 1, None) == EINVAL
    assert _linear_backward(T, workspace_bytes=_rooms(T, 100, 8, 16, 0, activation=1)[0] - 256) == ENOSPC
