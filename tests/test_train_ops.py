"""The training operators on the GPU against their definitions in 64 bits.

Tolerances.  A result rounded to type t is off by at most eps(t)/2 of its value.  What comes before is in 32 bits: a sum of d
terms one after the other is off by at most d 2^-24 of the sum of their absolute values, and no thread, wavefront and block
together add more than 64 terms a row in sequence here (rows of up to 32768), or 64 + rows / 512 a column.
"""
import math
import warnings

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24


@pytest.fixture(scope="module")
def T():
    from paper_2110_10548_amd import train
    train.lib()
    return train


def half(t):
    return torch.finfo(t).eps / 2


def draw(seed, *shape, scale=1.0):
    return torch.from_numpy(np.random.RandomState(seed).standard_normal(shape) * scale).cuda()


def tiny(t):
    """What a value next to zero may be off by: half of the smallest step (fp16: results below its normal numbers)."""
    return float(torch.finfo(t).smallest_normal) * torch.finfo(t).eps


def check(got, want, slack, what):
    """|got - want| <= half a step of want + slack, everywhere; NaN and infinities alike."""
    got = got.double()
    bad = ~((got - want).abs() <= half_of(got, want) + slack) & ~((got == want) | (got.isnan() & want.isnan()))
    assert not bad.any(), (what, int(bad.sum()), float((got - want)[bad].abs().max()), want[bad][:3].tolist(), got[bad][:3].tolist())


def half_of(got, want):
    return want.abs() * half_of.step + half_of.tiny


def compare(got, want, slack, what):
    half_of.step, half_of.tiny = half(got.dtype), tiny(got.dtype)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    check(got, want, slack, what)


# ------------------------------------------------------------------------------------------------ layer norm

def norm_inputs(rows, cols, kind, wkind, pad, seed=0):
    x = draw(seed, rows, cols + pad).mul(torch.exp(draw(seed + 1, rows, 1, scale=0.5))).add(0.5).to(kind)[:, :cols]
    dy = draw(seed + 2, rows, cols + 2 * pad).to(kind)[:, :cols]
    w = None if wkind is None else (1 + 0.3 * draw(seed + 3, cols)).to(wkind)
    b = None if wkind is None else draw(seed + 4, cols, scale=0.2).to(wkind)
    return x, dy, w, b


def norm_reference(x, w, b, eps):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    var = ((x - mean) ** 2).mean(-1, keepdim=True)
    rstd = (var + eps) ** -0.5
    xh = (x - mean) * rstd
    y = xh if w is None else xh * w.double()
    return (y if b is None else y + b.double()), mean[..., 0], rstd[..., 0], xh


SHAPES = [(1, 1), (3, 2), (1, 7), (5, 8), (1, 64), (17, 33), (64, 100), (1, 129), (9, 512), (33, 513), (7, 1023), (6, 1024), (5, 1031), (1, 2048), (3, 2049), (515, 768),
          (2, 4096), (3, 4100), (4, 8192), (2, 9001), (3, 16384), (2, 20003), (1, 40000)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("kind,wkind,pad", [(F32, F32, 0), (BF16, BF16, 0), (F16, F32, 3), (BF16, F16, 1), (F32, None, 5)])
def test_layer_norm(T, rows, cols, kind, wkind, pad):
    x, dy, w, b = norm_inputs(rows, cols, kind, wkind, pad)
    eps = 1e-5
    y, mean, rstd = T.p2_layer_norm_forward(x, w, b, eps)
    ry, rmean, rrstd, xh = norm_reference(x, w, b, eps)
    size = x.double().abs().mean(-1) * rrstd                       # what an error of the mean is worth in units of xh
    compare(mean, rmean, 70 * U * x.double().abs().mean(-1), "mean")
    compare(rstd, rrstd, 80 * U * (1 + size) * rrstd, "rstd")
    one = torch.ones((), dtype=torch.float64, device="cuda")
    wa, ba = (one if w is None else w.double().abs()), (0 * one if b is None else b.double().abs())
    slack = 80 * U * ((1 + size)[:, None] * (1 + xh.abs()) * wa + ba)
    compare(y, ry, slack, "y")
    dx, dw, db = T.p2_layer_norm_backward(dy, x, w, mean, rstd)
    d = dy.double()
    g = d if w is None else d * w.double()
    rdx = rrstd[:, None] * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    parts = g.abs() + g.abs().mean(-1, keepdim=True) + xh.abs() * (g * xh).abs().mean(-1, keepdim=True)
    compare(dx, rdx, 160 * U * rrstd[:, None] * parts * (1 + size)[:, None] * (1 + xh.abs()), "dx")
    terms = 64 + rows / 512 + 2 * 80                              # the sum's, and what xh itself is off by
    compare(dw, (d * xh).sum(0), terms * U * (d.abs() * (1 + xh.abs()) * (1 + size)[:, None]).sum(0), "dweight")
    compare(db, d.sum(0), terms * U * d.abs().sum(0), "dbias")


@pytest.mark.parametrize("rows,cols,kind", [(70001, 48, BF16), (40000, 264, F32), (20000, 1023, F16)])
def test_layer_norm_many_rows(T, rows, cols, kind):
    test_layer_norm(T, rows, cols, kind, F32, 0)


@pytest.mark.parametrize("cols", [1, 2, 3, 4, 5, 6, 7])
@pytest.mark.parametrize("kind,pad", [(F32, 0), (BF16, 1), (F16, 0)])
def test_layer_norm_of_few_columns(T, cols, kind, pad):
    test_layer_norm(T, 150001, cols, kind, F32, pad)
    test_layer_norm(T, 0, cols, kind, kind, pad)


def test_layer_norm_gradient_is_that_of_differences(T):
    """Along a direction: the 64-bit loss at x + h v and x - h v; its own error is h^2 times a third derivative."""
    x, dy, w, b = norm_inputs(6, 40, F32, F32, 0)
    y, mean, rstd = T.p2_layer_norm_forward(x, w, b)
    dx, dw, db = T.p2_layer_norm_backward(dy, x, w, mean, rstd)
    h = 1e-5
    vx, vw, vb = draw(7, 6, 40), draw(8, 40), draw(9, 40)

    def loss(s):
        return float((norm_reference(x.double() + s * vx, w.double() + s * vw, b.double() + s * vb, 1e-5)[0] * dy.double()).sum())

    want = (loss(h) - loss(-h)) / (2 * h)
    got = float((dx.double() * vx).sum() + (dw.double() * vw).sum() + (db.double() * vb).sum())
    size = float((dx.double() * vx).abs().sum() + (dw.double() * vw).abs().sum() + (db.double() * vb).abs().sum())
    assert abs(got - want) <= 400 * U * size + 1e-8 * size


def test_layer_norm_parts_and_forms(T):
    x, dy, w, b = norm_inputs(12, 96, BF16, BF16, 0)
    y, mean, rstd = T.p2_layer_norm_forward(x, w, b)
    all3 = T.p2_layer_norm_backward(dy, x, w, mean, rstd)
    for ask in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1)):
        got = T.p2_layer_norm_backward(dy, x, w, mean, rstd, dx=bool(ask[0]), dweight=bool(ask[1]), dbias=bool(ask[2]))
        for k in range(3):
            assert (got[k] is None) == (not ask[k]) and (got[k] is None or torch.equal(got[k], all3[k]))
    # leading dimensions, rows that lie in another order, rows that are all the same memory
    x3 = x.reshape(3, 4, 96)
    y3, m3, r3 = T.p2_layer_norm_forward(x3, w, b)
    assert torch.equal(y3.reshape(12, 96), y) and m3.shape == (3, 4) and torch.equal(m3.reshape(-1), mean)
    assert all(torch.equal(p, q) for p, q in zip(T.p2_layer_norm_backward(dy.reshape(3, 4, 96), x3, w, m3, r3)[1:], all3[1:]))
    turned = x.t().contiguous().t()
    assert torch.equal(T.p2_layer_norm_forward(turned, w, b)[0], y)
    swapped = x3.transpose(0, 1)
    assert torch.equal(T.p2_layer_norm_forward(swapped, w, b)[0], y3.transpose(0, 1))
    same = x[:1].expand(5, 96)
    assert torch.equal(T.p2_layer_norm_forward(same, w, b)[0], y[:1].expand(5, 96))
    # no rows
    y0, m0, _ = T.p2_layer_norm_forward(x[:0], w, b)
    assert y0.shape == (0, 96) and m0.shape == (0,)
    dx0, dw0, db0 = T.p2_layer_norm_backward(dy[:0], x[:0], w, m0, m0)
    assert dx0.shape == (0, 96) and not dw0.any() and not db0.any()
    # in place, through the C ABI
    z, g = x.clone(), dy.clone()
    L, s = T.lib(), torch.cuda.current_stream().cuda_stream
    T.B._check(L.p2_layer_norm_forward(z.data_ptr(), 1, 96, w.data_ptr(), b.data_ptr(), 1, 12, 96, 1e-5, z.data_ptr(), 96, None, None, s))
    assert torch.equal(z, y)
    work = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    dw, db = torch.empty_like(w), torch.empty_like(w)
    T.B._check(L.p2_layer_norm_backward(g.data_ptr(), 96, x.data_ptr(), 96, 1, w.data_ptr(), 1, mean.data_ptr(), rstd.data_ptr(), 12, 96, g.data_ptr(), 96,
                                        dw.data_ptr(), db.data_ptr(), work.data_ptr(), 1 << 20, s))
    assert torch.equal(g, all3[0]) and torch.equal(dw, all3[1]) and torch.equal(db, all3[2])


def test_layer_norm_long_rows_in_place(T):
    """dx over dy where a row does not fit in registers: the columns' sums come first."""
    x, dy, w, b = norm_inputs(3, 70001, BF16, F32, 0)
    _, mean, rstd = T.p2_layer_norm_forward(x, w, b)
    dx, dw, db = T.p2_layer_norm_backward(dy, x, w, mean, rstd)
    g = dy.contiguous().clone()
    n = T._room("p2_layer_norm_backward_workspace", 3, 70001)
    work, dw2, db2 = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(w), torch.empty_like(w)
    T.B._check(T.lib().p2_layer_norm_backward(g.data_ptr(), 70001, x.data_ptr(), 70001, 1, w.data_ptr(), 0, mean.data_ptr(), rstd.data_ptr(), 3, 70001, g.data_ptr(),
                                              70001, dw2.data_ptr(), db2.data_ptr(), work.data_ptr(), n, torch.cuda.current_stream().cuda_stream))
    assert torch.equal(g, dx) and torch.equal(dw, dw2) and torch.equal(db, db2)


def test_layer_norm_values_at_the_edge(T):
    # a large offset: the variance comes from centred squares (a difference of large sums would lose it)
    x = (4096.0 + draw(1, 4, 256)).float()
    y, mean, rstd = T.p2_layer_norm_forward(x)
    ry, _, rr, _ = norm_reference(x, None, None, 1e-5)
    assert float((y.double() - ry).abs().max()) <= 80 * U * 4096 * 4 and float((rstd.double() / rr - 1).abs().max()) <= 80 * U * 4096
    # constant rows, and rows with NaN or an infinity beside rows without
    x = torch.ones(4, 100, device="cuda")
    x[1, 3], x[2, 99] = math.nan, math.inf
    y, mean, rstd = T.p2_layer_norm_forward(x)
    assert not y[0].any() and not y[3].any() and y[1].isnan().all() and y[2].isnan().all()
    dx, dw, db = T.p2_layer_norm_backward(torch.ones_like(x), x, None, mean, rstd)
    assert dx[1].isnan().all() and torch.isfinite(dx[0]).all() and torch.isfinite(dx[3]).all() and (db == 4).all()


FAR = [(300, 2), (300, 3), (300, 7), (9, 64), (3, 100), (2, 512), (4, 1023), (3, 2048), (2, 4096), (2, 5000), (2, 8192), (2, 9001), (2, 16384), (1, 40000)]


@pytest.mark.parametrize("rows,cols", FAR)
@pytest.mark.parametrize("kind,values", [(F32, (12345.678, 1000.1, -3.3e8, 0.1, 1e30)), (F16, (1000.5, 0.1, -999.0)), (BF16, (1000.0, -3.3e8, 0.1))])
def test_layer_norm_of_equal_values(T, rows, cols, kind, values):
    """Distances from a first mean are whole steps of the value, and what is left of their sum tells how many: nothing remains."""
    for value in values:
        x = torch.full((rows, cols), value, dtype=kind, device="cuda")
        y, mean, rstd = T.p2_layer_norm_forward(x)
        assert not y.any() and torch.equal(mean, x[:, 0].float()), (value, float(y.float().abs().max()), float(mean[0]))
        assert float((rstd.double() * math.sqrt(1e-5) - 1).abs().max()) <= 4 * U


@pytest.mark.parametrize("rows,cols", FAR)
@pytest.mark.parametrize("kind,offset", [(F32, 1e6), (F32, -3e4), (F16, 2000.0)])
def test_layer_norm_of_rows_far_from_zero(T, rows, cols, kind, offset):
    """The first mean is off by up to 70 roundings of the offset, which is taken off again: what remains is off by as many of the distances."""
    x = (offset + draw(cols, rows, cols)).to(kind)
    y, mean, rstd = T.p2_layer_norm_forward(x, eps=1e-12)
    ry, rmean, rr, xh = norm_reference(x, None, None, 1e-12)
    there = torch.isfinite(rr) & (rr < 1e5)               # (two values may be the same)
    low = 70 * U * abs(offset)
    compare(mean[there], rmean[there], (70 * U * (1 / rr + low))[there], "mean")
    compare(rstd[there], rr[there], 200 * U * rr[there], "rstd")
    compare(y[there], ry[there], U * (70 * (1 + low * rr[:, None]) + 300 * (1 + xh.abs()))[there], "y")


@pytest.mark.parametrize("rows,cols", FAR)
def test_layer_norm_of_nearly_equal_values(T, rows, cols):
    """One value a step away from the others: the variance is far below the square of what the first mean is off by."""
    x = torch.full((rows, cols), 12345.678, device="cuda")
    x[:, cols // 2] = torch.nextafter(x[0, 0], x.new_tensor(math.inf))
    y, mean, rstd = T.p2_layer_norm_forward(x, eps=1e-15)
    ry, rmean, rr, xh = norm_reference(x, None, None, 1e-15)
    compare(rstd, rr, 200 * U * rr, "rstd")
    # the taken-off part of the mean is rounded to 24 bits itself, in units of a step over sqrt(cols)
    compare(y, ry, (300 + 35 * math.sqrt(cols)) * U * (1 + xh.abs()), "y")
    compare(mean, rmean, 70 * U / rr, "mean")


def test_layer_norm_statistics_of_what_is_no_number(T):
    for cols in (3, 100, 2048, 5000, 40000):
        x = draw(cols, 4, cols).float()
        x[0, 1], x[1, 2], x[2, 0] = math.inf, -math.inf, math.nan
        y, mean, rstd = T.p2_layer_norm_forward(x)
        assert mean[0] == math.inf and mean[1] == -math.inf and mean[2].isnan() and rstd[:3].isnan().all() and y[:3].isnan().all()
        assert torch.isfinite(y[3]).all()


def test_layer_norm_beyond_32_bits(T):
    """Rows further apart than 2^31 values."""
    stride, cols = (1 << 30) + 8, 264
    wide = torch.empty(3 * stride, dtype=F16, device="cuda")
    x = torch.as_strided(wide, (3, cols), (stride, 1))
    x.copy_(draw(3, 3, cols))
    y, mean, rstd = T.p2_layer_norm_forward(x)
    assert torch.equal(y, T.p2_layer_norm_forward(x.contiguous())[0])
    near = T.p2_layer_norm_backward(x.contiguous(), x.contiguous(), None, mean, rstd)
    far = T.p2_layer_norm_backward(x, x, None, mean, rstd)
    assert all(torch.equal(p, q) for p, q in zip(near, far))


# ------------------------------------------------------------------------------------------------ routing and its balance

def route_reference(logits, keep, k):
    """Choices by exact comparison, one token at a time; the rest in 64 bits."""
    z = logits.float().cpu().numpy().astype(np.float64)
    t, e = z.shape
    expert, gate = np.full((t, k), -1, np.int32), np.zeros((t, k))
    p, on = np.zeros((t, e)), np.zeros(t, bool)
    kept = np.ones(t, bool) if keep is None else keep.cpu().numpy().astype(bool)
    for i in range(t):
        row = z[i]
        if not kept[i] or not (row != -np.inf).any():
            continue
        on[i] = True
        with np.errstate(all="ignore"):
            q = np.exp(row - np.nanmax(row)) if not np.isnan(row).all() else row
            p[i] = q / q.sum()
        order = sorted((j for j in range(e) if row[j] != -np.inf), key=lambda j: (0 if np.isnan(row[j]) else 1, 0.0 if np.isnan(row[j]) else -row[j], j))[:k]
        expert[i, :len(order)] = order
        gate[i, :len(order)] = p[i, order]
    counts = np.bincount(expert[expert >= 0], minlength=e)
    n = int(on.sum())
    loss = e / (k * n * n) * float((counts * p.sum(0)).sum()) if n else 0.0
    return dict(expert=expert, gate=gate, counts=counts, prob_sum=p.sum(0), tokens=n, loss=loss, p=p, on=on)


ROUTES = [(1, 1, 1), (1, 8, 2), (3, 3, 3), (65, 7, 2), (200, 8, 8), (33, 9, 4), (130, 16, 1), (64, 17, 5), (50, 60, 4), (100, 64, 6), (40, 100, 8), (70, 128, 2), (31, 129, 3),
          (20, 160, 6), (90, 256, 8), (12, 257, 20), (9, 500, 8), (10, 512, 64), (7, 777, 10), (5, 1024, 33), (2049, 24, 2)]


@pytest.mark.parametrize("tokens,experts,k", ROUTES)
@pytest.mark.parametrize("kind,masked,pad", [(F32, False, 0), (BF16, True, 3), (F16, True, 0), (F32, True, 1)])
def test_routing(T, tokens, experts, k, kind, masked, pad):
    rng = np.random.RandomState(tokens * 7 + experts)
    # 16-bit logits of this size have many ties
    logits = draw(tokens + experts, tokens, experts + pad, scale=2.0).to(kind)
    keep = None
    if masked:
        logits[torch.from_numpy(rng.rand(tokens, experts + pad) < 0.3).cuda()] = -math.inf
        logits[::5] = -math.inf
        keep = torch.from_numpy(rng.rand(tokens) < 0.8).cuda()
    logits = logits[:, :experts]
    r, want = T.p2_balance_forward(logits, k, keep=keep), route_reference(logits, keep, k)
    assert np.array_equal(r["expert"].cpu().numpy(), want["expert"]) and np.array_equal(r["counts"].cpu().numpy(), want["counts"])
    assert int(r["tokens"]) == want["tokens"]
    # e^(z - m): the product rounds (z - m) log2 e to half a step of up to 30, 2^x to one step; a row's sum, its inverse
    far = 60.0
    gate = torch.from_numpy(want["gate"]).cuda()
    compare(r["gate"], gate, (2 * far + 70) * U * gate, "gate")
    prob = torch.from_numpy(want["prob_sum"]).cuda()
    compare(r["prob_sum"], prob, (2 * far + 70 + 64 + tokens / 512) * U * prob, "prob_sum")
    compare(r["loss"], torch.tensor(want["loss"], dtype=torch.float64, device="cuda"), (2 * far + 140 + tokens / 512) * U * want["loss"], "loss")
    again = T.p2_balance_loss(r["counts"], r["prob_sum"], r["tokens"], k)
    compare(again, r["loss"].double(), 4 * U * r["loss"].double(), "loss again")
    # gradients
    dgate, dloss = draw(5, tokens, k).float(), torch.tensor(3.0, device="cuda")
    p, n = want["p"], want["tokens"]
    c = experts / (k * n * n) if n else 0.0
    for dg, dl in ((dgate, dloss), (None, None)):
        u = np.repeat((c * (3.0 if dl is not None else 1.0) * want["counts"])[None, :], tokens, 0)
        if dg is not None:
            at, values = want["expert"], dg.double().cpu().numpy()
            for i in range(k):
                rows = at[:, i] >= 0
                u[rows, at[rows, i]] += values[rows, i]
        dz = p * (u - (p * u).sum(1, keepdims=True))
        size = p * (np.abs(u) + (p * np.abs(u)).sum(1, keepdims=True))
        got = T.p2_balance_backward(logits, r["expert"], r["counts"], r["tokens"], keep=keep, dgate=dg, dloss=dl)
        compare(got, torch.from_numpy(dz).cuda(), torch.from_numpy((4 * far + 300) * U * size).cuda(), "dlogits")


def test_routing_gradient_is_that_of_differences(T):
    z, v = draw(1, 20, 12).float(), draw(2, 20, 12)
    r = T.p2_balance_forward(z, 3)
    dgate, dloss = draw(3, 20, 3).float(), torch.tensor([0.7], device="cuda")
    got = T.p2_balance_backward(z, r["expert"], r["counts"], r["tokens"], dgate=dgate, dloss=dloss)

    def loss(s):                                          # of the same choice: it has no gradient
        p = torch.softmax(z.double() + s * v, 1)
        balance = 12 / (3 * 20 * 20) * (p.sum(0) * r["counts"]).sum()
        return float(0.7 * balance + (p.gather(1, r["expert"].long()) * dgate.double()).sum())

    h = 1e-5
    size = float((got.double() * v).abs().sum())
    assert abs((loss(h) - loss(-h)) / (2 * h) - float((got.double() * v).sum())) <= 600 * U * size + 1e-8 * size


@pytest.mark.parametrize("tokens,experts,k", [(5, 4, 4), (40, 12, 8), (70, 64, 6), (33, 256, 8), (20, 300, 40), (9, 1024, 64)])
def test_routing_gradient_of_experts_named_twice(T, tokens, experts, k):
    """Not what the forward pass chooses: the gates' gradients of such an expert are added in their order (another order would leave 1 or 2 here)."""
    rng = np.random.RandomState(tokens + k)
    z = draw(tokens, tokens, experts).float()
    expert = rng.randint(-1, 3, (tokens, k)).astype(np.int32)
    values = rng.choice([2.0 ** 24, -2.0 ** 24, 1.0, 1.0, 0.0], (tokens, k)).astype(np.float32)
    expert[0, :], values[0, :4] = 1, (2.0 ** 24, 1.0, 1.0, -2.0 ** 24)
    values[0, 4:] = 0.0
    u = np.zeros((tokens, experts + 1), np.float32)
    for i in range(k):
        u[np.arange(tokens), expert[:, i]] += values[:, i]
    u = torch.from_numpy(u[:, :experts]).double().cuda()
    p = torch.softmax(z.double(), 1)
    counts, kept = torch.zeros(experts, dtype=torch.int64, device="cuda"), torch.tensor(tokens, device="cuda")
    want, size = p * (u - (p * u).sum(1, keepdim=True)), p * (u.abs() + (p * u.abs()).sum(1, keepdim=True))
    args = (z, torch.from_numpy(expert).cuda(), counts, kept, None, torch.from_numpy(values).cuda())
    got = T.p2_balance_backward(*args)
    compare(got, want, 540 * U * size, "dlogits")
    assert not got[0].any() and all(torch.equal(got, T.p2_balance_backward(*args)) for _ in range(5))


@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_routing_of_equal_extreme_and_masked_logits(T, kind):
    lowest, inf, nan = torch.finfo(kind).min, math.inf, math.nan
    rows = torch.tensor([[0.0] * 6, [-0.0, 0.0, -0.0, 0.0, -1.0, -1.0], [lowest] * 6, [-inf, lowest, -inf, -inf, -inf, -inf], [-inf] * 6,
                         [-inf, -inf, 3.0, -inf, -inf, -inf], [1.0, 2.0, nan, 3.0, nan, 0.0], [1.0, inf, 2.0, inf, 0.0, 0.0], [nan] * 6, [1.0, 2.0, 3.0, 4.0, 5.0, 6.0]],
                        device="cuda").to(kind)
    rows[6, 4] = -rows[6, 4]                              # a NaN with the other sign
    keep = torch.ones(10, dtype=torch.bool, device="cuda")
    keep[8] = False                                       # NaN in a row that does not count
    r = T.p2_balance_forward(rows, 3, keep=keep)
    assert r["expert"].tolist() == [[0, 1, 2], [0, 1, 2], [0, 1, 2], [1, -1, -1], [-1, -1, -1], [2, -1, -1], [2, 4, 3], [1, 3, 2], [-1, -1, -1], [5, 4, 3]]
    assert int(r["tokens"]) == 8 and r["counts"].tolist() == [3, 5, 6, 3, 2, 1]
    assert r["gate"][6].isnan().all() and r["gate"][7].isnan().all() and r["loss"].isnan() and r["prob_sum"].isnan().all()
    assert torch.equal(r["gate"][3:6], torch.tensor([[1.0, 0, 0], [0, 0, 0], [1.0, 0, 0]], device="cuda"))
    assert torch.allclose(r["gate"][:3], torch.tensor(1 / 6, device="cuda")[None, None] * torch.tensor([[1.0], [0.0], [1.0]], device="cuda") +
                          torch.tensor([[0.0], [1 / (4 + 2 * math.exp(-1))], [0.0]], device="cuda"), rtol=1e-5, atol=0)
    g = T.p2_balance_backward(rows, r["expert"], r["counts"], r["tokens"], keep=keep)
    assert not g[4].any() and not g[8].any() and torch.isfinite(g[[0, 1, 2, 3, 5, 9]]).all() and g[6].isnan().all()
    assert not g[5].any()                                 # one expert on offer: nothing to shift


def test_routing_without_tokens(T):
    r = T.p2_balance_forward(torch.zeros(0, 16, device="cuda"), 2)
    assert int(r["tokens"]) == 0 and float(r["loss"]) == 0 and not r["counts"].any() and not r["prob_sum"].any() and r["expert"].shape == (0, 2)
    assert T.p2_balance_backward(torch.zeros(0, 16, device="cuda"), r["expert"], r["counts"], r["tokens"]).shape == (0, 16)
    # tokens, but none that counts
    z = draw(1, 50, 16).float()
    r = T.p2_balance_forward(z, 2, keep=torch.zeros(50, dtype=torch.bool, device="cuda"))
    assert int(r["tokens"]) == 0 and float(r["loss"]) == 0 and (r["expert"] == -1).all() and not r["gate"].any()
    assert not T.p2_balance_backward(z, r["expert"], r["counts"], r["tokens"]).any()


@pytest.mark.parametrize("tokens,experts,k,kind", [(131072, 64, 2, BF16), (100003, 8, 1, F32), (50001, 256, 8, F16)])
def test_routing_of_many_tokens(T, tokens, experts, k, kind):
    z = draw(4, tokens, experts).to(kind)
    r = T.p2_balance_forward(z, k)
    best = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(r["expert"].long(), best)
    assert torch.equal(r["counts"], torch.bincount(best.reshape(-1), minlength=experts)) and int(r["tokens"]) == tokens
    p = torch.softmax(z.double(), 1)
    compare(r["prob_sum"], p.sum(0), (254 + tokens / 512) * U * p.sum(0), "prob_sum")
    again = T.p2_balance_forward(z, k)
    assert all(torch.equal(r[n], again[n]) for n in r)


def test_routing_statistics_add_up_over_devices(T):
    """The loss and the gradient of a batch from its halves' summed statistics."""
    z = draw(6, 300, 40).float()
    whole = T.p2_balance_forward(z, 4)
    parts = [T.p2_balance_forward(h, 4) for h in (z[:170], z[170:])]
    counts, prob, kept = (sum(q[n] for q in parts) for n in ("counts", "prob_sum", "tokens"))
    assert torch.equal(counts, whole["counts"]) and int(kept) == 300
    assert abs(float(T.p2_balance_loss(counts, prob, kept, 4)) / float(whole["loss"]) - 1) < 300 * U
    g = torch.cat([T.p2_balance_backward(h, q["expert"], counts, kept) for h, q in zip((z[:170], z[170:]), parts)])
    assert torch.equal(g, T.p2_balance_backward(z, whole["expert"], whole["counts"], whole["tokens"]))


@pytest.mark.parametrize("experts,k", [(6, 6), (16, 8), (60, 9), (64, 64), (130, 20), (256, 8), (500, 33), (1024, 64)])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_routing_of_choices_side_by_side(T, experts, k, kind):
    """The best experts all in one place: a lane has to give far more of them than its share."""
    up = torch.arange(experts, device="cuda", dtype=torch.float64)
    rows = [up / 8, -up / 8, torch.zeros(experts, device="cuda"), (up % 3 == 0) * 2.0, (up // 8 % 2) * 1.0, -(up - experts // 2).abs() / 4, torch.where(up < experts // 2, up / 8, -math.inf),
            torch.where(up % 2 == 0, math.nan, up / 8), torch.where(up < 7, torch.where(up % 2 == 0, -math.nan, math.inf), -up / 8)]
    z = torch.stack([r.double() for r in rows]).to(kind)
    r, want = T.p2_balance_forward(z, k), route_reference(z, None, k)
    assert np.array_equal(r["expert"].cpu().numpy(), want["expert"]) and np.array_equal(r["counts"].cpu().numpy(), want["counts"])
    gate = torch.from_numpy(want["gate"][:7]).cuda()
    compare(r["gate"][:7], gate, (2 * 128 + 70) * U * gate + 2.0 ** -126, "gate")         # (z - m up to 128: what is below fp32's normal numbers may be 0)


@pytest.mark.parametrize("offset", [1e4, -1e4, 3e7, -3e7, 3e38, -3e38])
def test_routing_of_far_logits(T, offset):
    """Softmax of logits a long way from zero; the steps between fp32 numbers there are 2^-10, 2 and 2^105."""
    step = max(0.5, float(np.spacing(np.float32(abs(offset)))))
    whole = torch.randint(-8, 8, (40, 70), generator=torch.Generator().manual_seed(3)).cuda()
    z = (offset + step * whole.double()).float()
    z[5, 7] = -z[5, 7]                                    # the other end, too
    for kind in (F32, BF16):
        r, want = T.p2_balance_forward(z.to(kind), 6), route_reference(z.to(kind), None, 6)
        assert np.array_equal(r["expert"].cpu().numpy(), want["expert"])
        gate = torch.from_numpy(want["gate"]).cuda()
        compare(r["gate"], gate, (2 * 104 + 134) * U * gate + 2.0 ** -126, "gate")
        assert abs(float(r["loss"]) / want["loss"] - 1) <= (2 * 104 + 134 + 140) * U


def test_routing_beyond_32_bits(T):
    stride, experts = (1 << 30) + 64, 24
    wide = torch.empty(3 * stride, dtype=F16, device="cuda")
    z = torch.as_strided(wide, (3, experts), (stride, 1))
    z.copy_(draw(8, 3, experts))
    far, near = T.p2_balance_forward(z, 2), T.p2_balance_forward(z.contiguous(), 2)
    assert all(torch.equal(far[n], near[n]) for n in far)
    assert torch.equal(T.p2_balance_backward(z, far["expert"], far["counts"], far["tokens"]),
                       T.p2_balance_backward(z.contiguous(), far["expert"], far["counts"], far["tokens"]))


# ------------------------------------------------------------------------------------------------ orthogonalised updates

NS = (3.4445, -4.7750, 2.0315)


def newton_schulz(g, steps=5, coefficients=NS, eps=1e-7):
    """The definition in 64 bits, and the norms of the iterates."""
    x = g.double()
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-1, -2).contiguous()
    x = x / (torch.linalg.vector_norm(x, dim=(-2, -1), keepdim=True) + eps)
    a, b, c = coefficients
    sizes = [torch.linalg.vector_norm(x, dim=(-2, -1))]
    for _ in range(steps):
        m = x @ x.transpose(-1, -2).contiguous()
        x = a * x + (b * m + c * (m @ m)) @ x
        sizes.append(torch.linalg.vector_norm(x, dim=(-2, -1)))
    return (x.transpose(-1, -2) if tall else x), sizes


def slope(coefficients, steps):
    """Largest slope of the polynomial applied `steps` times, on [0, 1.25]: what a small change of X may grow by."""
    a, b, c = coefficients
    x, d = np.linspace(0, 1.25, 20001), np.ones(20001)
    for _ in range(steps):
        d = d * np.abs(a + 3 * b * x ** 2 + 5 * c * x ** 4)
        x = a * x + b * x ** 3 + c * x ** 5
    return float(d[np.abs(x) < 10].max())


def update_error(got, g, **kw):
    """(error, bound) of each matrix, as parts of the result's norm.  A step rounds X, A and B and sums their products: four roundings
    to 22 bits of what is at most 1.25^2 times X (B: 2.81 times), worth at most slope() of the steps that follow."""
    want, sizes = newton_schulz(g, **kw)
    steps, coefficients = kw.get("steps", 5), kw.get("coefficients", NS)
    unit = 2.0 ** -22
    bound = sum(4 * 2.81 * unit * sizes[k] * slope(coefficients, steps - k) for k in range(steps)) + 2 * unit * sizes[-1]
    size = sizes[-1]
    bound = bound / size + half(got.dtype)
    if got.dtype == BF16:                                 # upper halves (11 bits) of X in A, of B and X in B X
        bound = bound + 2.0 ** -12 * (2 * 2 * 2.81 + 2 * 2.81) * sizes[-2] / size
    off = torch.linalg.vector_norm(got.double() - want, dim=(-2, -1)) / size
    return off, bound


UPDATES = [(1, 1, 1), (2, 1, 40), (3, 40, 1), (1, 16, 16), (2, 31, 33), (1, 32, 64), (1, 5, 1500), (1, 64, 64), (2, 65, 64), (1, 64, 512), (1, 96, 96), (2, 97, 130), (1, 128, 128),
           (1, 128, 129), (1, 129, 128), (3, 130, 260), (1, 200, 777), (1, 1000, 33), (2, 256, 256), (1, 40, 5000), (1, 333, 3000), (1, 640, 1000), (1, 1100, 1100)]


@pytest.mark.parametrize("count,rows,cols", UPDATES)
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_update(T, count, rows, cols, kind):
    g = draw(rows + cols, count, rows, cols, scale=1e-2).to(kind)
    got = T.p2_orthogonalize(g)
    assert got.shape == g.shape and got.dtype == kind
    off, bound = update_error(got, g)
    assert (off <= bound).all(), (off.tolist(), bound.tolist())


@pytest.mark.parametrize("rows,cols", [(60, 100), (100, 60), (300, 400), (700, 200)])
def test_update_of_low_rank(T, rows, cols):
    """A few large singular values, the others a thousandth: in 11 bits the result would be off by a tenth and more."""
    g = (draw(1, rows, 4) @ draw(2, 4, cols) + 1e-3 * draw(3, rows, cols)).float()
    off, bound = update_error(T.p2_orthogonalize(g), g)
    assert float(off) <= min(float(bound), 2e-3)


@pytest.mark.parametrize("rows,cols", [(2048, 2048), (1600, 3088), (3100, 900), (2400, 2400)])
def test_update_large(T, rows, cols):
    g = draw(9, rows, cols).float()
    off, bound = update_error(T.p2_orthogonalize(g), g)
    assert float(off) <= float(bound)


@pytest.mark.parametrize("rows,cols", [(5, 7), (16, 16), (16, 60), (80, 20), (24, 24), (32, 128), (33, 90), (64, 200), (100, 100), (130, 200), (700, 300)])
def test_update_is_as_exact_as_products_in_32_bits(T, rows, cols):
    """On the average of forty matrices, a tenth for what these differ by."""
    a, b, c = NS
    g = draw(rows * cols, 40, rows, cols).float()
    want, sizes = newton_schulz(g)
    x = g if rows <= cols else g.transpose(1, 2).contiguous()
    x = (x.double() / (torch.linalg.vector_norm(x.double(), dim=(-2, -1), keepdim=True) + 1e-7)).float()
    for _ in range(5):
        m = x @ x.transpose(1, 2).contiguous()
        x = a * x + (b * m + c * (m @ m)) @ x
    plain = x if rows <= cols else x.transpose(1, 2)
    off = [float((torch.linalg.vector_norm(v.double() - want, dim=(-2, -1)) / sizes[-1]).mean()) for v in (T.p2_orthogonalize(g), plain)]
    assert off[0] <= 1.1 * off[1], off


@pytest.mark.parametrize("count,rows,cols", [(64, 16, 16), (64, 60, 100), (64, 100, 100), (64, 128, 90), (32, 200, 200), (8, 300, 500), (2, 1100, 900)])
def test_update_operands_have_22_bits(T, count, rows, cols):
    """Entry by entry: X alone (the coefficients 1, 0, 0), and of diagonal matrices, whose sums have one term each, its powers by way of A and B."""
    g = draw(rows, count, rows, cols).float()
    x = g.double() / torch.linalg.vector_norm(g.double(), dim=(-2, -1), keepdim=True)
    got = T.p2_orthogonalize(g, steps=1, coefficients=(1.0, 0.0, 0.0), eps=0.0).double()
    # a pair is off by half a step of its lower half at most (2^-23; below fp16's normal numbers 2^-25 of 2^-15); the factor, its product, the gain's and the
    # result are rounded to 24 bits
    assert ((got - x).abs() <= 3 * 2.0 ** -23 * x.abs() + 2.0 ** -39).all(), float(((got - x) / x).abs().max())
    n = min(rows, cols)
    g = torch.zeros(count, rows, cols, device="cuda")
    g[:, range(n), range(n)] = 0.5 + torch.rand(count, n, generator=torch.Generator().manual_seed(rows)).cuda()
    x = g.double() / torch.linalg.vector_norm(g.double(), dim=(-2, -1), keepdim=True)
    for power, coefficients in ((3, (0.0, 1.0, 0.0)), (5, (0.0, 0.0, 1.0))):
        got = T.p2_orthogonalize(g, steps=1, coefficients=coefficients, eps=0.0).double()
        # X's pairs and factor in every place, A twice, A A or B, the products' lowest terms (2^-22 each) and the same roundings at the end
        assert ((got - x ** power).abs() <= 20 * 2.0 ** -22 * x.abs() ** power + 2.0 ** -39 * x.abs()).all(), (power, float((got / x ** power - 1).abs().nan_to_num().max()))


def like_a_gradient(form, rows, cols):
    if form == "equal":
        return torch.full((rows, cols), 0.37, dtype=torch.float64, device="cuda")
    if form == "rank one":
        return draw(5, rows, 1) @ draw(6, 1, cols)
    if form == "low rank":
        return draw(1, rows, 4) @ draw(2, 4, cols) + 1e-3 * draw(3, rows, cols)
    return draw(4, rows, cols)


@pytest.mark.parametrize("rows,cols", [(40, 70), (150, 333), (200, 300), (700, 200), (1000, 2777), (2048, 2048)])
@pytest.mark.parametrize("form", ["normal", "low rank", "rank one", "equal"])
def test_update_is_rounded_once(T, rows, cols, form):
    """A 16-bit result is the 32-bit one rounded, also where a X and B X cancel (and would magnify what fewer bits round off)."""
    g = like_a_gradient(form, rows, cols).to(BF16)
    for steps, coefficients in ((5, NS), (1, NS), (1, (100.0, -200.0, 101.0)), (1, (3.0, -4.0, 1.01)), (6, (1.875, -1.25, 0.375))):
        full = T.p2_orthogonalize(g, steps=steps, coefficients=coefficients, dtype=F32)
        for kind in (BF16, F16):
            assert torch.equal(T.p2_orthogonalize(g, steps=steps, coefficients=coefficients, dtype=kind), full.to(kind)), (steps, coefficients, kind)
        if steps == 1:
            # X is in each term once for every power; four roundings to 22 bits each, and a rounding to 24 bits for every 32 terms of three sums
            want, sizes = newton_schulz(g, steps=1, coefficients=coefficients)
            a, b, c = (abs(v) for v in coefficients)
            bound = (4 + 3 * max(rows, cols) / 32 / 4) * 2.0 ** -22 * (a + 3 * b + 5 * c) * sizes[0] / sizes[1]
            assert torch.linalg.vector_norm(full.double() - want) <= bound * sizes[1], (coefficients, float(bound))


@pytest.mark.parametrize("rows,cols", [(48, 80), (300, 200)])
def test_update_forms(T, rows, cols):
    g = draw(4, rows, cols).float()
    plain = T.p2_orthogonalize(g)
    # the transpose's update is the update's transpose (sums of the same products in another order of tiles)
    off = torch.linalg.vector_norm(T.p2_orthogonalize(g.t()) - plain.t()) / torch.linalg.vector_norm(plain)
    assert float(off) <= 2 * float(update_error(plain, g)[1])
    # a power of two in front changes nothing, at whatever size
    for s in (2.0 ** 100, 2.0 ** -90):
        assert torch.equal(T.p2_orthogonalize(g * s, eps=0.0), T.p2_orthogonalize(g, eps=0.0))
    assert torch.equal(T.p2_orthogonalize(g, scale=0.25), plain * 0.25)
    assert torch.equal(T.p2_orthogonalize(g.to(BF16), dtype=F32).to(F16), T.p2_orthogonalize(g.to(BF16), dtype=F16))
    # stacks, of views and of one matrix for all
    stack = torch.stack([g, 2 * g, g.flip(0)])
    got = T.p2_orthogonalize(stack)
    assert torch.equal(got[0], plain) and torch.equal(T.p2_orthogonalize(stack.reshape(3, 1, rows, cols))[:, 0], got)
    wide = torch.zeros(3, rows + 2, cols + 5, device="cuda")
    wide[:, :rows, :cols] = stack
    assert torch.equal(T.p2_orthogonalize(wide[:, :rows, :cols]), got)
    assert torch.equal(T.p2_orthogonalize(g.expand(4, rows, cols))[3], plain)
    assert T.p2_orthogonalize(stack[:0]).shape == (0, rows, cols)
    # other steps and coefficients
    for steps, coefficients in ((1, NS), (2, NS), (12, NS), (8, (1.5, -0.5, 0.0)), (6, (1.875, -1.25, 0.375)), (3, (1.0, 0.0, 0.0)), (2, (0.0, 0.0, 0.0))):
        off, bound = update_error(T.p2_orthogonalize(g, steps=steps, coefficients=coefficients), g, steps=steps, coefficients=coefficients)
        if any(coefficients):
            assert float(off) <= float(bound), (steps, coefficients)
        else:
            assert not T.p2_orthogonalize(g, steps=steps, coefficients=coefficients).any()


@pytest.mark.parametrize("rows,cols", [(40, 70), (200, 150)])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_update_of_zeros_and_of_what_is_no_number(T, rows, cols, kind):
    assert not T.p2_orthogonalize(torch.zeros(rows, cols, dtype=kind, device="cuda")).any()
    assert not T.p2_orthogonalize(torch.zeros(rows, cols, dtype=kind, device="cuda"), eps=0.0).any()
    for value in (math.nan, math.inf, -math.inf):
        g = draw(2, 3, rows, cols).to(kind)
        clean = T.p2_orthogonalize(g)
        g[1, rows - 1, 2] = value
        got = T.p2_orthogonalize(g)
        assert got[1].isnan().all() and torch.equal(got[0], clean[0]) and torch.equal(got[2], clean[2])
    g = torch.full((rows, cols), torch.finfo(kind).max, dtype=kind, device="cuda")      # the squares pass fp32's largest number
    off, bound = update_error(T.p2_orthogonalize(g), g)
    assert float(off) <= float(bound)


def test_update_into_a_part_of_another_tensor(T):
    """Strides of the result, through the C ABI; what lies beside it stays."""
    import ctypes as C
    g = draw(5, 2, 150, 90).float()
    want = T.p2_orthogonalize(g)
    out = torch.full((2, 160, 97), 7.0, device="cuda")
    n = T._room("p2_orthogonalize_workspace", 2, 150, 90)
    work = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    T.B._check(T.lib().p2_orthogonalize(g.data_ptr(), 0, 90, 150 * 90, 2, 150, 90, 5, (C.c_double * 3)(*NS), 1e-7, 1.0, out.data_ptr(), 0, 97, 160 * 97,
                                        T._ptr(work), n, torch.cuda.current_stream().cuda_stream))
    assert torch.equal(out[:, :150, :90], want) and (out[:, 150:] == 7).all() and (out[:, :, 90:] == 7).all()


# ------------------------------------------------------------------------------------------------ streams, graphs, the same bits again

def _step(T, x, dy, w, b, z, g):
    y, mean, rstd = T.p2_layer_norm_forward(x, w, b)
    dx, dw, db = T.p2_layer_norm_backward(dy, x, w, mean, rstd)
    r = T.p2_balance_forward(z, 4)
    dz = T.p2_balance_backward(z, r["expert"], r["counts"], r["tokens"], dgate=r["gate"], dloss=r["loss"])
    return [y, mean, rstd, dx, dw, db, *r.values(), dz, T.p2_orthogonalize(g), T.p2_orthogonalize(g[:, :60])]


def _step_inputs(seed):
    x, dy, w, b = norm_inputs(3000, 520, BF16, F32, 0, seed)
    return [x, dy, w, b, draw(seed + 5, 9000, 72).to(BF16), draw(seed + 6, 300, 330).float()]


def test_the_same_bits_again(T):
    inputs = _step_inputs(1)
    first = _step(T, *inputs)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, _step(T, *inputs)))


def test_another_stream(T):
    inputs = _step_inputs(2)
    want = _step(T, *inputs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _step(T, *inputs)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_two_streams_at_once(T):
    """Calls under way together share nothing: statistics over several blocks, partial sums and updates too large for LDS, alternately, with no wait between."""
    inputs = [_step_inputs(40 + i) for i in range(4)]
    want = [_step(T, *i) for i in inputs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for turn in range(6):
        for i, x in enumerate(inputs):
            with torch.cuda.stream(streams[(turn + i) % 2]):
                got.append((i, _step(T, *x)))
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for i, one in got for p, q in zip(want[i], one))


def test_in_a_graph(T):
    inputs = _step_inputs(3)
    _step(T, *inputs)                                     # first calls load kernels
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(T, *inputs)
    for seed in (10, 20, 30):
        for p, q in zip(inputs, _step_inputs(seed)):
            p.copy_(q)
        graph.replay()
        torch.cuda.synchronize()
        want = _step(T, *inputs)                          # eager work between the replays
        assert all(torch.equal(p, q) for p, q in zip(want, got))


# ------------------------------------------------------------------------------------------------ what is refused, and what is left behind

def test_tensors_that_do_not_fit_are_refused(T):
    x, w, z = draw(1, 6, 40).float(), draw(2, 40).float(), draw(3, 10, 12).float()
    y, mean, rstd = T.p2_layer_norm_forward(x, w, w)
    r = T.p2_balance_forward(z, 3)
    keep, dgate = torch.ones(10, dtype=torch.bool, device="cuda"), torch.ones(10, 3, device="cuda")
    expert, counts, prob, tokens = (r[n] for n in ("expert", "counts", "prob_sum", "tokens"))
    refused = [
        lambda: T.p2_layer_norm_forward(x.double(), w, w), lambda: T.p2_layer_norm_forward(x, w[:39], None), lambda: T.p2_layer_norm_forward(x, w, w.to(BF16)),
        lambda: T.p2_layer_norm_forward(x, None, w.long()), lambda: T.p2_layer_norm_forward(x, w.cpu()), lambda: T.p2_layer_norm_forward(x, w[None]),
        lambda: T.p2_layer_norm_forward(x, w, w, eps=-1.0), lambda: T.p2_layer_norm_forward(x[:, :0]),
        lambda: T.p2_layer_norm_backward(x, x, w, mean[:5], rstd), lambda: T.p2_layer_norm_backward(x, x, w, mean, rstd.double()),
        lambda: T.p2_layer_norm_backward(x.to(F16), x, w, mean, rstd), lambda: T.p2_layer_norm_backward(x, x, w, mean, rstd.cpu()),
        lambda: T.p2_balance_forward(z, 0), lambda: T.p2_balance_forward(z, -1), lambda: T.p2_balance_forward(z, 13), lambda: T.p2_balance_forward(z, 1 << 40),
        lambda: T.p2_balance_forward(z, 3, keep=keep[:9]), lambda: T.p2_balance_forward(z, 3, keep=keep.float()), lambda: T.p2_balance_forward(z, 3, keep=keep.cpu()),
        lambda: T.p2_balance_forward(z[:, :0], 1), lambda: T.p2_balance_forward(z.int(), 1),
        lambda: T.p2_balance_loss(counts.int(), prob, tokens, 3), lambda: T.p2_balance_loss(counts, prob[:11], tokens, 3), lambda: T.p2_balance_loss(counts, prob, counts, 3),
        lambda: T.p2_balance_loss(counts, prob, tokens, 13),
        lambda: T.p2_balance_backward(z, expert.long(), counts, tokens), lambda: T.p2_balance_backward(z, expert[:9], counts, tokens),
        lambda: T.p2_balance_backward(z, expert, counts[:11], tokens), lambda: T.p2_balance_backward(z, expert, counts, tokens, dgate=dgate[:, :2]),
        lambda: T.p2_balance_backward(z, expert, counts, tokens, dgate=dgate.double()), lambda: T.p2_balance_backward(z, expert, counts, tokens, dloss=dgate),
        lambda: T.p2_balance_backward(z, expert, counts, tokens.cpu()),
        lambda: T.p2_orthogonalize(x, steps=0), lambda: T.p2_orthogonalize(x, dtype=torch.float64), lambda: T.p2_orthogonalize(x.long()), lambda: T.p2_orthogonalize(x[:0])]
    torch.cuda.synchronize()
    room = torch.cuda.memory_allocated()
    for i, call in enumerate(refused):
        with pytest.raises(T.P2Error):
            call()
            pytest.fail("call %d was not refused" % i)
    for call in (lambda: T.p2_layer_norm_forward(x, 3), lambda: T.p2_balance_forward(z, 1.5), lambda: T.p2_orthogonalize(x, steps="five"), lambda: T.p2_layer_norm_forward(x, eps=None)):
        with pytest.raises(TypeError):
            call()
    assert torch.cuda.memory_allocated() == room


def test_calls_leave_nothing_behind(T):
    import sys
    inputs = _step_inputs(4)
    _step(T, *inputs)
    torch.cuda.synchronize()
    room, held = torch.cuda.memory_allocated(), [sys.getrefcount(t) for t in inputs]
    for _ in range(20):
        _step(T, *inputs)
    assert torch.cuda.memory_allocated() == room and [sys.getrefcount(t) for t in inputs] == held


def test_forms_of_the_arguments(T):
    """Results have the shapes and types that the arguments call for, whatever these are laid out like."""
    x = draw(1, 3, 5, 24).to(BF16)
    y, mean, rstd = T.p2_layer_norm_forward(x)
    assert y.shape == x.shape and y.dtype == BF16 and mean.shape == rstd.shape == (3, 5) and mean.dtype == F32
    dx, dw, db = T.p2_layer_norm_backward(x, x, None, mean, rstd, dweight=False)
    assert dx.shape == x.shape and dw is None and db.shape == (24,) and db.dtype == BF16
    v, m, s = T.p2_layer_norm_forward(x[1, 2])
    assert v.shape == (24,) and m.shape == s.shape == () and torch.equal(v, y[1, 2]) and torch.equal(m, mean[1, 2])
    turned = x.permute(1, 0, 2)
    assert torch.equal(T.p2_layer_norm_forward(turned)[0], y.permute(1, 0, 2))
    w = torch.nn.Parameter(torch.ones(24, device="cuda"))
    assert torch.equal(T.p2_layer_norm_forward(x, w.to(BF16))[0], y) and not T.p2_layer_norm_forward(x.float(), w)[0].requires_grad
    z = draw(2, 24, 30).float()
    r, t = T.p2_balance_forward(z, 2), T.p2_balance_forward(z.t().contiguous().t(), 2, keep=torch.ones(24, dtype=torch.uint8, device="cuda"))
    assert all(torch.equal(r[n], t[n]) for n in r) and [r[n].shape for n in r] == [(24, 2), (24, 2), (30,), (30,), (), ()]
    assert [r[n].dtype for n in r] == [torch.int32, F32, torch.int64, F32, torch.int64, F32]
    g = T.p2_orthogonalize(x, dtype=F32)
    assert g.shape == x.shape and g.dtype == F32 and T.p2_orthogonalize(x.transpose(1, 2)).shape == (3, 24, 5)


def test_a_parameter_that_would_not_train_is_warned_of(T):
    x, z, g = draw(1, 6, 40).float(), draw(2, 10, 12).float(), draw(3, 20, 30).float()
    w = torch.nn.Parameter(torch.ones(40, device="cuda"))
    y, mean, rstd = T.p2_layer_norm_forward(x, w.detach())
    r = T.p2_balance_forward(z, 3)
    zp, gp, prob = (t.clone().requires_grad_() for t in (z, g, r["prob_sum"]))
    calls = (lambda: T.p2_layer_norm_forward(x, w), lambda: T.p2_layer_norm_backward(x, x, w, mean, rstd), lambda: T.p2_balance_forward(zp, 3),
             lambda: T.p2_balance_loss(r["counts"], prob, r["tokens"], 3), lambda: T.p2_balance_backward(zp, r["expert"], r["counts"], r["tokens"]),
             lambda: T.p2_orthogonalize(gp))
    for call in calls:
        with pytest.warns(UserWarning, match="nothing is recorded for autograd") as caught:
            call()
        assert len(caught) == 1 and caught[0].filename == __file__
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            with torch.no_grad():
                call()
