"""Routing, AdamW and matrix products on the GPU against their definitions in 64 bits.

Tolerances.  A result rounded to type t is off by at most eps(t)/2 of its value.  What comes before is in 32 bits (U = 2^-24 of a value an operation):
 - an exponential's argument z - m is off by U (|z| + |m|) or less and its instruction by two steps, so scores are off by
   (|z| + |m| + 40) 2 U of their value, 40 covering a row's sum of up to 64 terms in sequence a lane and the divisions;
 - a matrix product adds up at most inner/4 + 32 terms in sequence (an MFMA takes four or more at a time, parts of the sum are joined
   after that), and an MFMA may round off twice what an addition does.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16, F16, F64 = torch.float32, torch.bfloat16, torch.float16, torch.float64
U = 2.0 ** -24
INF = math.inf


@pytest.fixture(scope="module")
def T():
    from paper_2110_10548_amd import train
    train.lib()
    return train


def draw(seed, *shape, scale=1.0):
    return torch.from_numpy(np.asarray(np.random.RandomState(seed).standard_normal(shape) * scale)).cuda()


def compare(got, want, slack, what):
    """|got - want| <= half a step of want + slack, everywhere; NaN and infinities alike."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    t = got.dtype
    tiny = float(torch.finfo(t).smallest_normal) * torch.finfo(t).eps
    step = torch.finfo(t).eps / 2
    got = got.double()
    bad = ~((got - want).abs() <= want.abs() * step + tiny + slack) & ~((got == want) | (got.isnan() & want.isnan()))
    assert not bad.any(), (what, int(bad.sum()), float((got - want)[bad].abs().max()), want[bad][:3].tolist(), got[bad][:3].tolist())


# --------------------------------------------------------------------------------------------------- routing

def route_reference(logits, k, score="softmax", bias=None, keep=None, groups=1, group_limit=None, group_best=1, renormalise=False, scale=1.0):
    """In 64 bits, by sorting."""
    z = logits.double()
    t, e = z.shape
    on = (z != -INF).any(1)
    on = on if keep is None else on & keep.bool()
    if score == "softmax":
        w = torch.where(on[:, None], z, 0.0)
        w = (w - w.nan_to_num(nan=-INF, posinf=INF, neginf=-INF).amax(1, keepdim=True)).exp()
        s = w / w.sum(1, keepdim=True)
    else:
        s = 1 / (1 + (-z).exp())
    b = torch.zeros(e, dtype=F64, device=z.device) if bias is None else bias.double()
    v = torch.where(on[:, None] & (z != -INF) & (b != -INF), s + b, -INF)
    limit = groups if group_limit is None else group_limit
    if groups > 1:
        top = v.view(t, groups, -1).sort(2, descending=True).values[..., :group_best]
        value = torch.where(top[..., 0] == -INF, -INF, torch.where(top == -INF, 0.0, top).sum(2))
        first = value.sort(dim=1, descending=True, stable=True).indices[:, :limit]
        open_ = torch.zeros_like(value, dtype=torch.bool).scatter_(1, first, True)
        v = torch.where(open_.repeat_interleave(e // groups, 1), v, -INF)
    best = v.sort(dim=1, descending=True, stable=True).indices[:, :k]
    valid = v.gather(1, best) != -INF
    chosen = torch.where(valid, z.gather(1, best), -INF)
    if score == "softmax":
        log = chosen - torch.where(on[:, None], z, 0.0).logsumexp(1, keepdim=True)
    else:
        log = torch.nn.functional.logsigmoid(chosen)
    gate = log.exp()
    if renormalise:
        gate = (log - torch.where(valid.any(1, keepdim=True), log, 0.0).logsumexp(1, keepdim=True)).exp()
    expert = torch.where(valid, best, -1).int()
    counts = torch.bincount(best[valid], minlength=e)
    return {"expert": expert, "gate": torch.where(valid, gate * scale, 0.0), "counts": counts, "tokens": on.sum(), "score": s, "spread": z.nan_to_num(0, 0, 0).abs().amax(1, keepdim=True)}


def gate_slack(r):
    return (2 * r["spread"] + 40) * 2 * U * r["gate"].abs()


def check_route(T, logits, k, **kw):
    got, want = T.p2_route_forward(logits, k, **kw), route_reference(logits, k, **kw)
    assert torch.equal(got["expert"], want["expert"]), (got["expert"] != want["expert"]).nonzero()[:4].tolist()
    assert torch.equal(got["counts"], want["counts"]) and int(got["tokens"]) == int(want["tokens"])
    assert got["gate"].dtype == F32 and got["expert"].dtype == torch.int32 and got["tokens"].shape == ()
    compare(got["gate"], want["gate"], gate_slack(want), "gate")
    return got, want


# tokens, experts, k, groups, limit, best
CHOICES = [(1, 1, 1, 1, 1, 1), (3, 2, 2, 1, 1, 1), (5, 3, 2, 3, 2, 1), (9, 8, 8, 1, 1, 1), (33, 8, 8, 4, 3, 2), (257, 12, 3, 4, 2, 2), (100, 60, 4, 6, 3, 1), (1, 64, 2, 1, 1, 1),
           (513, 64, 6, 8, 3, 2), (301, 96, 8, 1, 1, 2), (77, 160, 6, 8, 3, 1), (1030, 256, 8, 8, 4, 2), (64, 256, 8, 1, 1, 1), (50, 254, 5, 2, 1, 2), (130, 255, 9, 5, 2, 2),
           (40, 510, 8, 17, 5, 2), (21, 1023, 16, 33, 9, 2), (20, 1024, 64, 64, 64, 1), (19, 1024, 64, 1, 1, 1), (11, 1023, 64, 3, 1, 2), (13, 777, 33, 7, 6, 2), (40, 1000, 33, 40, 7, 1),
           (32, 256, 8, 1, 1, 1), (20, 256, 8, 8, 4, 2), (64, 64, 4, 4, 2, 1)]


@pytest.mark.parametrize("tokens,experts,k,groups,limit,best", CHOICES)
@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("score,biased,renormalise", [("softmax", False, True), ("softmax", True, False), ("sigmoid", True, True), ("sigmoid", False, False)])
def test_route(T, tokens, experts, k, groups, limit, best, kind, score, biased, renormalise):
    pad = (experts + k) % 3
    logits = draw(experts, tokens, experts + pad, scale=1.5).to(kind)[:, :experts]
    bias = draw(1, experts, scale=0.1 if score == "sigmoid" else 1.0 / experts).float() if biased else None
    kw = dict(score=score, groups=groups, group_limit=limit, group_best=best, renormalise=renormalise, scale=2.5 if biased else 1.0)
    check_route(T, logits, k, bias=bias, **kw)
    z = torch.where(draw(2, tokens, experts) < -1.0, -INF, logits.float()).to(kind)          # a sixth is not on offer, a fifth of the tokens does not count
    z[::7] = -INF
    check_route(T, z, k, bias=bias, keep=draw(3, tokens) > -0.84, **kw)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("groups,limit,best", [(1, 1, 1), (8, 4, 2), (8, 3, 1)])
def test_route_ties_go_to_the_lowest_index(T, score, kind, groups, limit, best):
    z = torch.from_numpy(np.random.RandomState(4).randint(-2, 3, (700, 64))).cuda().to(kind)
    z[0], z[1, 1:] = 0, -INF
    for bias in (None, torch.zeros(64, device="cuda"), torch.from_numpy(np.random.RandomState(5).randint(-1, 2, 64) * 0.25).cuda().float()):
        check_route(T, z, 8, score=score, bias=bias, groups=groups, group_limit=limit, group_best=best, renormalise=True)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("size", [2, 4, 8])
@pytest.mark.parametrize("scale", [0.5, 2.0])
def test_route_groups_whose_best_two_add_up_to_nearly_the_same(T, score, kind, size, scale):
    """Many small groups of logits of either sign, without a bias: sums that differ in the fourth digit and less."""
    z = draw(size, 1200, 32 * size, scale=scale).to(kind)
    for limit in (1, 13, 31):
        check_route(T, z, 2, score=score, groups=32, group_limit=limit, group_best=2)


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("tokens", [1, 50])
def test_route_groups_whose_best_two_add_up_to_the_same(T, kind, tokens):
    """sigmoid(x) + sigmoid(-x) is 1 whatever x."""
    for first in (0.5, 1.0, 1.5):
        z = torch.tensor([[-9.0, first, -9.0, -first, 0.0, -9.0, 0.0, -9.0]], device="cuda").to(kind).repeat(tokens, 1)
        assert (T.p2_route_forward(z, 1, score="sigmoid", groups=2, group_limit=1, group_best=2)["expert"] == 1).all()
        assert (T.p2_route_forward(z.roll(4, 1), 1, score="sigmoid", groups=2, group_limit=1, group_best=2)["expert"] == 0).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_tells_scores_apart_that_32_bits_do_not(T, score):
    """Neighbouring 32-bit logits, far out where their scores differ in the ninth digit and less, and biases that all but even them out."""
    r = np.random.RandomState(6)
    base = r.uniform(2.0, 12.0, (400, 1))
    z = torch.from_numpy(base + r.randint(0, 40, (400, 32)) * 2.0 ** -20).cuda().float()
    check_route(T, z, 6, score=score, bias=torch.full((32,), 0.1, device="cuda"), groups=4, group_limit=2, group_best=2)
    check_route(T, z, 6, score=score, groups=4, group_limit=2, group_best=2)
    s = (torch.softmax(z[:1].double(), 1) if score == "softmax" else torch.sigmoid(z[:1].double()))[0]
    check_route(T, z[:1], 6, score=score, bias=(0.5 - s).float())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kind", [F32, F16])
def test_route_far_and_odd_logits(T, score, kind):
    z = draw(8, 64, 40, scale=100.0).to(kind)                  # scores from 1 down to nothing
    if score == "sigmoid":
        z = z.clamp(max=30.0)
    for renormalise in (False, True):
        check_route(T, z, 5, score=score, renormalise=renormalise)
        check_route(T, z, 5, score=score, renormalise=renormalise, bias=draw(9, 40, scale=0.3).float(), groups=5, group_limit=2, group_best=2)
    z = -torch.rand(16, 40, device="cuda").to(kind) - 200      # every sigmoid is 0 in 32 bits
    got, want = check_route(T, z, 4, score=score, renormalise=True)
    assert abs(float(got["gate"].sum(1).double().mean()) - 1) < 1e-6


def check_scores_decide(T, z, k, **kw):
    """Without a bias, and with one of zeros: the choice is that of the scores in 64 bits."""
    for bias in (None, torch.zeros(z.shape[1], device="cuda")):
        got, want = T.p2_route_forward(z, k, bias=bias, **kw), route_reference(z, k, bias=bias, **kw)
        assert torch.equal(got["expert"], want["expert"]), (bias is None, (got["expert"] != want["expert"]).nonzero()[:4].tolist())
        assert torch.equal(got["counts"], want["counts"])


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("score,scale", [("sigmoid", 30.0), ("sigmoid", 1000.0), ("softmax", 1000.0)])
@pytest.mark.parametrize("tokens,experts,k,groups,limit,best", [(1, 8, 8, 1, 1, 1), (300, 8, 1, 1, 1, 1), (300, 8, 2, 4, 2, 1), (20, 64, 6, 1, 1, 1), (700, 64, 6, 8, 3, 1), (700, 64, 6, 8, 3, 2),
                                                                (300, 256, 8, 8, 4, 1), (90, 255, 9, 5, 2, 2), (40, 1024, 64, 1, 1, 1), (40, 1000, 33, 40, 7, 1)])
def test_route_without_a_bias_goes_by_scores(T, kind, score, scale, tokens, experts, k, groups, limit, best):
    """Logits far out have one score: 1 above some 37 as sigmoids, 0 below some -709, or that far below a row's largest as a softmax.  Ties go to the lowest index."""
    check_scores_decide(T, draw(experts, tokens, experts, scale=scale).to(kind), k, score=score, groups=groups, group_limit=limit, group_best=best)


def test_route_without_a_bias_of_a_few_logits_with_one_score(T):
    z = torch.tensor([[38.0, 60.0, 45.0, 1.0]], device="cuda")
    assert T.p2_route_forward(z, 2, score="sigmoid")["expert"].tolist() == [[0, 1]]
    for tokens in (1, 200):
        one = z.repeat(tokens, 1)
        assert (T.p2_route_forward(one, 2, score="sigmoid")["expert"] == torch.tensor([0, 1], device="cuda")).all()
        assert (T.p2_route_forward(one, 1, score="sigmoid", groups=4, group_limit=1)["expert"] == 0).all()
        assert (T.p2_route_forward(one, 1, score="sigmoid")["expert"] == 0).all()
        soft = torch.tensor([[-3e4, -1e4, 2.0, -2e4]], device="cuda").repeat(tokens, 1)                    # masks that are no infinities
        for kind in (F32, BF16, F16):
            assert (T.p2_route_forward(soft.to(kind), 3)["expert"] == torch.tensor([2, 0, 1], device="cuda")).all()
            assert (T.p2_route_forward(soft.to(kind), 2, groups=4, group_limit=2)["expert"] == torch.tensor([2, 0], device="cuda")).all()


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("tokens,experts,groups,limit,best", [(3, 6, 1, 1, 1), (500, 64, 1, 1, 1), (500, 64, 8, 3, 1), (500, 64, 8, 3, 2)])
def test_route_of_logits_next_to_zero(T, kind, score, tokens, experts, groups, limit, best):
    """1e-20 and 2e-20 differ, their scores do not; 0 is not always the smaller one."""
    z = (draw(1, tokens, experts) * 10.0 ** torch.from_numpy(np.random.RandomState(2).randint(-45, -17, (tokens, experts))).cuda()).to(kind)
    z[::3, ::5] = 0.0
    for k in (1, 2, 5):
        check_scores_decide(T, z, k, score=score, groups=groups, group_limit=limit, group_best=best)
        first = z.clone()
        first[:, 1] = 0.5
        check_scores_decide(T, first, k, score=score, groups=groups, group_limit=limit, group_best=best)
        check_scores_decide(T, -z.abs(), k, score=score, groups=groups, group_limit=limit, group_best=best)
        behind = -z.abs()                                      # zeros, and behind them what is next to them, with lower indices
        behind[1::2, experts // 3::2] = 0.0
        check_scores_decide(T, behind, k, score=score, groups=groups, group_limit=limit, group_best=best)
        check_scores_decide(T, 0 * z, k, score=score, groups=groups, group_limit=limit, group_best=best)


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("experts,at", [(48, 7), (48, 3), (8, 0), (64, 41), (256, 100), (1000, 999)])
@pytest.mark.parametrize("tokens", [1, 300])
def test_route_of_one_logit_next_to_zero_among_zeros(T, kind, experts, at, tokens):
    """It comes behind the zeros by its logit, has their score, and one lane alone sees it."""
    z = torch.zeros(tokens, experts, device="cuda")
    z[:, at] = -1e-6
    z = z.mul(1e-14 if kind != F16 else 0.25).to(kind)
    z[:, :at:2] = -INF
    for k in (1, min(at // 2 + 1, 64), min(experts - (at + 1) // 2, 8)):
        check_scores_decide(T, z, k, score="sigmoid")
        check_scores_decide(T, z, k, score="sigmoid", groups=2, group_limit=1)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("offset", [1000.0, -30000.0])
def test_route_of_logits_far_from_zero(T, score, offset):
    """A softmax goes by differences alone: gates are off by what the logits' own steps allow, not by their size."""
    z = (draw(10, 300, 96).float() * 2 + offset).to(F32)
    if score == "sigmoid":
        z = z - offset + 4 * math.copysign(1, offset)
    for bias in (None, draw(11, 96, scale=0.01).float()):
        for kw in (dict(), dict(groups=8, group_limit=3, group_best=2), dict(groups=8, group_limit=3, group_best=1)):
            got, want = T.p2_route_forward(z, 6, score=score, bias=bias, **kw), route_reference(z, 6, score=score, bias=bias, **kw)
            assert torch.equal(got["expert"], want["expert"])
            compare(got["gate"], want["gate"], (2 * 40 + 40) * 2 * U * want["gate"], "gate")


def test_route_with_infinities_and_nan(T):
    nan = math.nan
    z = torch.tensor([[1.0, nan, 3.0, -INF, 2.0, 0.0], [INF, 1.0, 2.0, INF, -INF, 0.0], [-INF] * 6, [nan] * 6, [1.0, 2.0, 3.0, 4.0, 5.0, 6.0]], device="cuda")
    r = T.p2_route_forward(z, 3, score="sigmoid")
    assert r["expert"].tolist() == [[1, 2, 4], [0, 3, 2], [-1] * 3, [0, 1, 2], [5, 4, 3]] and int(r["tokens"]) == 4
    assert r["gate"][0, 0].isnan() and float(r["gate"][1, 0]) == 1.0 and r["gate"][2].tolist() == [0.0] * 3
    r = T.p2_route_forward(z, 3, renormalise=True)               # softmax: all scores are NaN in rows 0, 1 and 3, and all that is on offer ties
    assert r["expert"].tolist() == [[0, 1, 2], [0, 1, 2], [-1] * 3, [0, 1, 2], [5, 4, 3]]
    assert r["gate"][[0, 1, 3]].isnan().all() and not r["gate"][[2, 4]].isnan().any()
    bias = torch.tensor([INF, -INF, 0.0, nan, 0.0, 0.0], device="cuda")
    r = T.p2_route_forward(z[4:], 6, score="sigmoid", bias=bias)
    assert r["expert"].tolist() == [[3, 0, 5, 4, 2, -1]] and not r["gate"].isnan().any() and float(r["gate"][0, 5]) == 0.0
    r = T.p2_route_forward(z[4:], 2, score="sigmoid", bias=bias, groups=3, group_limit=1, group_best=2)      # NaN, then +inf, is the largest sum
    assert r["expert"].tolist() == [[3, 2]]
    r = T.p2_route_forward(z[:1], 3, score="sigmoid", keep=torch.zeros(1, dtype=torch.bool, device="cuda"))
    assert r["expert"].tolist() == [[-1] * 3] and int(r["tokens"]) == 0 and int(r["counts"].sum()) == 0


def test_route_groups_with_less_on_offer_than_are_asked_for(T):
    z = torch.full((1, 12), -INF, device="cuda")
    z[0, 1], z[0, 4], z[0, 5] = 2.0, 1.0, 0.5
    r = T.p2_route_forward(z, 4, score="sigmoid", groups=4, group_limit=1, group_best=2)
    assert r["expert"].tolist() == [[4, 5, -1, -1]]            # 0.73 + 0.62 are more than 0.88 alone
    r = T.p2_route_forward(z, 4, score="sigmoid", groups=4, group_limit=3, group_best=2)
    assert r["expert"].tolist() == [[1, 4, 5, -1]] and int(r["counts"].sum()) == 3


def test_route_of_no_tokens(T):
    r = T.p2_route_forward(torch.zeros(0, 16, device="cuda"), 2)
    assert r["expert"].shape == (0, 2) and int(r["counts"].sum()) == 0 and int(r["tokens"]) == 0
    assert T.p2_route_backward(torch.zeros(0, 16, device="cuda"), r["expert"], r["gate"]).shape == (0, 16)


def gates_of(z, expert, score, renormalise, scale):
    """The gates as a function of the logits, the choice being given."""
    valid = expert >= 0
    s = torch.softmax(z, 1) if score == "softmax" else torch.sigmoid(z)
    g = torch.where(valid, s.gather(1, expert.clamp(min=0).long()), 0.0)
    if renormalise:
        total = g.sum(1, keepdim=True)
        g = g / torch.where(total == 0, 1.0, total)
    return g * scale


def route_gradient(z, expert, dgate, score, renormalise, scale):
    """The formula in 64 bits, and the sum of the sizes of what is added up."""
    valid = expert >= 0
    at = expert.clamp(min=0).long()
    s = torch.softmax(z, 1) if score == "softmax" else torch.sigmoid(z)
    d = torch.where(valid, dgate.double() * scale, 0.0)
    w = torch.where(valid, s.gather(1, at), 0.0)
    zeros = torch.zeros_like(z)
    if renormalise:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
        dot, size = (w * d).sum(1, keepdim=True), (w * d.abs()).sum(1, keepdim=True)
        slope = 1.0 if score == "softmax" else 1 - s.gather(1, at)
        return zeros.scatter_add(1, at, w * slope * (d - dot) * valid), zeros.scatter_add(1, at, w * (d.abs() + size))
    u, ua = zeros.scatter_add(1, at, d), zeros.scatter_add(1, at, d.abs())
    if score == "sigmoid":
        return u * s * (1 - s), ua * s
    on = valid.any(1, keepdim=True)
    return torch.where(on, s * (u - (s * u).sum(1, keepdim=True)), 0.0), s * (ua + (s * ua).sum(1, keepdim=True))


@pytest.mark.parametrize("score,renormalise", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
def test_the_gradient_s_formula_against_differences(score, renormalise):
    z, expert = draw(1, 6, 9), torch.from_numpy(np.stack([np.random.RandomState(i).permutation(9)[:3] for i in range(6)])).cuda().int()
    expert[0, 2], expert[1] = -1, -1
    d = draw(2, 6, 3)
    want, h = torch.zeros_like(z), 1e-5
    for e in range(9):
        step = torch.zeros_like(z)
        step[:, e] = h
        want[:, e] = (((gates_of(z + step, expert, score, renormalise, 2.0) - gates_of(z - step, expert, score, renormalise, 2.0)) * d).sum(1)) / (2 * h)
    got, _ = route_gradient(z, expert, d, score, renormalise, 2.0)
    assert (got - want).abs().max() < 1e-8                     # h^2 and 64 bits' eps / h


@pytest.mark.parametrize("tokens,experts,k", [(1, 1, 1), (7, 3, 2), (33, 8, 8), (100, 60, 4), (65, 256, 8), (9, 1023, 64), (5, 77, 64), (3000, 64, 6), (70000, 16, 2)])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("score,renormalise", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
def test_route_gradient(T, tokens, experts, k, kind, score, renormalise):
    pad = experts % 3
    z = draw(experts, tokens, experts + pad, scale=2.0).to(kind)[:, :experts]
    r = T.p2_route_forward(z, k, score=score, renormalise=renormalise, scale=1.5, keep=draw(1, tokens) > -1.0)
    dgate = draw(2, tokens, k).float()
    got = T.p2_route_backward(z, r["expert"], dgate, score=score, renormalise=renormalise, scale=1.5)
    want, size = route_gradient(z.double(), r["expert"], dgate, score, renormalise, 1.5)
    assert got.dtype == kind
    compare(got, want, size * (4 * z.double().abs().amax(1, keepdim=True) + 100) * 2 * U, "dlogits")
    assert (got[(r["expert"] < 0).all(1)] == 0).all()


def test_route_gradient_of_experts_named_twice_and_out_of_range(T):
    z = draw(3, 4, 12).float()
    expert = torch.tensor([[1, 1, 2], [0, 0, 0], [5, -1, 5], [-1, 12, -7]], dtype=torch.int32, device="cuda")
    dgate = draw(4, 4, 3).float()
    safe = torch.where((expert < 0) | (expert >= 12), -1, expert)
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            got = T.p2_route_backward(z, expert, dgate, score=score, renormalise=renormalise)
            want, size = route_gradient(z.double(), safe, dgate, score, renormalise, 1.0)
            compare(got, want, size * 300 * U, "dlogits")
            assert (got[3] == 0).all()


def test_route_bias(T):
    counts = torch.tensor([3, 5, 4, 4, 0, 8], device="cuda")
    bias = torch.tensor([0.5, 0.5, 0.5, -1.0, 0.0, 0.0], device="cuda")
    assert torch.equal(T.p2_route_bias(bias, counts, 0.25), bias + 0.25 * torch.tensor([1.0, -1.0, 0.0, 0.0, 1.0, -1.0], device="cuda"))
    one = T.p2_route_bias(bias[:1], counts[:1], 0.25)
    assert torch.equal(one, bias[:1])
    big = torch.full((1000,), 2 ** 61 // 1000, device="cuda")
    big[7] += 1
    out = T.p2_route_bias(torch.zeros(1000, device="cuda"), big, 1.0)
    assert float(out[7]) == -1.0 and (out[:7] == 1.0).all() and (out[8:] == 1.0).all()


def test_route_many_tokens(T):
    """More logits than 32 bits count; what lies past them is routed as it is alone."""
    t, e = (1 << 31) // 256 + 1000, 256
    z = torch.zeros(t, e, dtype=BF16, device="cuda")
    z[:, 3] = 1.0
    tail = draw(1, 1500, e).to(BF16)
    z[-1500:] = tail
    kw = dict(score="sigmoid", bias=draw(2, e, scale=0.05).float(), groups=8, group_limit=2, group_best=2, renormalise=True)
    r, alone = T.p2_route_forward(z, 4, **kw), T.p2_route_forward(tail, 4, **kw)
    assert torch.equal(r["expert"][-1500:], alone["expert"]) and torch.equal(r["gate"][-1500:], alone["gate"])
    assert int(r["counts"].sum()) == 4 * t and int(r["tokens"]) == t
    dgate = torch.ones(t, 4, device="cuda")
    d = T.p2_route_backward(z, r["expert"], dgate, score="sigmoid", scale=1.0)
    assert torch.equal(d[-1500:], T.p2_route_backward(tail, alone["expert"], dgate[:1500], score="sigmoid", scale=1.0))


# ----------------------------------------------------------------------------------------------------- AdamW

SIZES = [(1,), (7,), (8,), (9,), (255,), (256,), (257,), (3, 100), (2048,), (2049,), (5, 1031), (0,), (), (64, 64), (100003,)]


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("n", [1, 2, 160, 161, 400])
def test_square_sum(T, kind, n):
    x = [draw(i, *SIZES[i % 14], scale=10.0 ** (i % 3 - 1)).to(kind) for i in range(n)]
    got, want = T.p2_square_sum(x), sum(float(t.double().square().sum()) for t in x)
    assert got.dtype == F64 and got.shape == () and abs(float(got) - want) <= 1e-13 * want
    assert torch.equal(got, T.p2_square_sum(x))


def test_square_sum_of_large_small_and_odd_values(T):
    x = torch.full((1000,), 1e30, device="cuda")
    assert abs(float(T.p2_square_sum([x, x])) / 2e63 - 1) < 1e-6
    assert abs(float(T.p2_square_sum([x * 1e-30 * 1e-30])) / 1e-57 - 1) < 1e-6
    assert float(T.p2_square_sum([x[:0]])) == 0.0
    x[77] = INF
    assert float(T.p2_square_sum([x])) == INF
    x[78] = math.nan
    assert math.isnan(float(T.p2_square_sum([x])))
    y = draw(1, 33, 65).float()
    want = float(y[:, 3:50].double().square().sum())
    assert abs(float(T.p2_square_sum([y[:, 3:50]])) - want) < 1e-12 * want and abs(float(T.p2_square_sum([y.t(), y])) - 2 * float(y.double().square().sum())) < 1e-9


def adam_reference(p, g, m, v, t, lr, betas, eps, decay):
    m, v = betas[0] * m + (1 - betas[0]) * g, betas[1] * v + (1 - betas[1]) * g * g
    step = lr / (1 - betas[0] ** t) * m / ((v / (1 - betas[1] ** t)).sqrt() + eps)
    return p * (1 - lr * decay) - step, m, v, step


def adam_inputs(shapes, kind, grad_kind, bits, seed=0):
    p = [draw(seed + 4 * i, *s, scale=0.02).to(kind) for i, s in enumerate(shapes)]
    g = [(draw(seed + 4 * i + 1, *s) * torch.exp(draw(seed + 4 * i + 2, *s))).mul(1e-2).to(grad_kind) for i, s in enumerate(shapes)]
    return p, g


def decode(q, scale, square):
    n = q.numel()
    s = scale.double().repeat_interleave(256)[:n].view(q.shape)
    q = q.double()
    return s * (q / 255) ** 4 if square else s * (q / 127) * (q / 127).abs()


HYPER = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


@pytest.mark.parametrize("kind,grad_kind,copy", [(F32, F32, None), (F32, BF16, BF16), (BF16, BF16, None), (F16, F32, None), (F32, F16, F16), (BF16, F32, F32)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("clip", [None, 0.5])
def test_adamw(T, kind, grad_kind, copy, bits, clip):
    p, g = adam_inputs(SIZES, kind, grad_kind, bits)
    state = T.p2_adamw_state(p, bits)
    copies = None if copy is None else [torch.zeros(t.shape, dtype=copy, device="cuda") for t in p]
    for t in range(1, 4):
        total = T.p2_square_sum(g) if clip else None
        factor = 1.0 if clip is None else min(1.0, clip / (2.0 * math.sqrt(float(total)))) * 2.0
        before = [(a.double(), *((m.double(), v.double()) if bits == 32 else (decode(m, ms, False), decode(v, vs, True))))
                  for a, m, v, ms, vs in zip(p, state["means"], state["squares"], state["mean_scales"] or p, state["square_scales"] or p)]
        T.p2_adamw(p, g, **state, copies=copies, **HYPER, square_sum=total, max_norm=clip, grad_factor=2.0 if clip else 1.0)
        assert int(state["step"]) == t
        for i, (a, m, v) in enumerate(before):
            d = g[i].double() * factor
            rp, rm, rv, step = adam_reference(a, d, m, v, t, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
            sm, sv = m.abs() + d.abs(), v + d * d              # sizes of what is added up, for the rounding of each term
            compare(p[i], rp, 4 * U * a.abs() + step.abs() * 16 * U + HYPER["lr"] * 16 * U * sm / (rv.sqrt() + 1e-8), "param")
            if copies:
                compare(copies[i], p[i].double() if copy != F32 and kind == F32 else rp, 4 * U * a.abs() + step.abs() * 16 * U + HYPER["lr"] * 16 * U * sm / (rv.sqrt() + 1e-8), "copy")
            if bits == 32:
                compare(state["means"][i], rm, 6 * U * sm, "mean")
                compare(state["squares"][i], rv, 8 * U * sv, "square")
            elif a.numel():
                check_8_bits(state["means"][i], state["mean_scales"][i], rm, 6 * U * sm, False)
                check_8_bits(state["squares"][i], state["square_scales"][i], rv, 8 * U * sv, True)
                mv, sv_ = T.p2_adamw_values([state["means"][i]], [state["squares"][i]], [state["mean_scales"][i]], [state["square_scales"][i]])
                want = decode(state["means"][i], state["mean_scales"][i], False)
                assert mv[0].shape == a.shape and ((mv[0].double() - want).abs() <= 4 * U * want.abs()).all()
                want = decode(state["squares"][i], state["square_scales"][i], True)
                assert ((sv_[0].double() - want).abs() <= 8 * U * want.abs()).all()


def check_8_bits(q, scale, want, slack, square):
    """Each block's scale is its largest value, and each stored number the nearest one to the value within it."""
    n = want.numel()
    q, want, slack = q.reshape(-1).double(), want.reshape(-1), slack.reshape(-1)
    pad = -n % 256
    blocks = torch.nn.functional.pad(want.abs(), (0, pad)).view(-1, 256)
    most = torch.nn.functional.pad(slack, (0, pad)).view(-1, 256)
    top = blocks.amax(1)
    assert ((scale.double() - top).abs() <= most.amax(1) + U * top).all()
    s = scale.double().repeat_interleave(256)[:n]
    low, high = ((want.abs() + sign * slack).clamp(min=0) / s.clamp(min=1e-300) for sign in (-1, 1))
    place = (lambda x: 255 * x ** 0.25) if square else (lambda x: 127 * x ** 0.5)
    off = 0.5 + 127 * 16 * U
    ok = (q.abs() >= place(low) - off) & (q.abs() <= place(high) + off)
    if square:
        ok |= (q == 1) & (want > 0) & (place(low) < 1)
        assert (q[(want > 2 * slack) & (s > 0)] >= 1).all()
    else:
        assert (q * want >= 0)[want.abs() > slack].all()
    assert ok[s > 0].all() and (q[s == 0] == 0).all()


def to_8_bits(v, square):
    """The formula in 32 bits, operation by operation, by numpy, whose roots and divisions are rounded as they are defined (torch's roots on the CPU are off by a step): stored numbers and their places."""
    blocks = v.numpy().reshape(-1, 256)
    scale = np.abs(blocks).max(1, keepdims=True)
    part = np.abs(blocks) * (np.float32(1) / scale)
    place = np.float32(255) * np.sqrt(np.sqrt(part)) if square else np.float32(127) * np.sqrt(part)
    assert place.dtype == np.float32
    q = np.rint(place)
    q = np.where(blocks > 0, np.maximum(q, np.float32(1)), q) if square else np.copysign(q, blocks)
    return (torch.from_numpy(x.reshape(-1)) for x in (q, scale, place))


@pytest.mark.parametrize("shape", [(512 * 256,), (3, 100 * 256)])
def test_adamw_8_bits_next_to_the_middle_of_two_numbers(T, shape):
    """Without what was there before (betas of 0) the mean is g and the square g^2, each at most a few steps off a place where rounding turns: the numbers stored are those of the formula, all of them."""
    n = math.prod(shape)
    r = np.random.RandomState(1)
    sizes = np.repeat(np.exp(3 * r.standard_normal(n // 256)), 256)

    def near(middles, power):                                  # size * middle^power and its neighbours, a block's first value being its size
        x = (sizes * middles ** power).astype(np.float32)
        x = (x.view(np.int32) + r.randint(-4, 5, n).astype(np.int32)).view(np.float32)
        x[::256] = sizes[::256]
        return torch.from_numpy(x * np.where(r.rand(n) < 0.5, -1, 1).astype(np.float32))

    for g, square in ((near((r.randint(0, 126, n) + 0.5) / 127, 2), False), (near((r.randint(1, 254, n) + 0.5) / 255, 2), True)):
        q, scale, place = to_8_bits(g * g if square else g, square)
        turning = ((place - place.floor() - 0.5).abs() < (9.9e-5 if square else 3.8e-5)).double().mean()
        assert turning > 0.5, float(turning)                   # where a root that is off by a step could matter
        p = torch.zeros(shape, device="cuda")
        state = T.p2_adamw_state([p], 8)
        T.p2_adamw([p], [g.view(shape).cuda()], **state, betas=(0.0, 0.0))
        got, got_scale = (state["squares"][0], state["square_scales"][0]) if square else (state["means"][0], state["mean_scales"][0])
        assert torch.equal(got_scale.cpu(), scale)
        assert torch.equal(got.cpu().view(-1).float(), q), int((got.cpu().view(-1).float() != q).sum())


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_steps_that_are_left_out(T, bits):
    shapes = [(300,), (7, 9)]
    for bad in (INF, -INF, math.nan):
        p, g = adam_inputs(shapes, BF16, BF16, bits)
        state = T.p2_adamw_state(p, bits)
        T.p2_adamw(p, g, **state, **HYPER)
        g[1][3, 3] = bad
        flat = [*p, *state["means"], *state["squares"], state["step"], *(state["mean_scales"] or []), *(state["square_scales"] or [])]
        before = [t.clone() for t in flat]
        T.p2_adamw(p, g, **state, **HYPER, square_sum=T.p2_square_sum(g))
        T.p2_adamw(p, g, **state, **HYPER, square_sum=T.p2_square_sum(g), max_norm=1.0)
        assert all(torch.equal(a, b) for a, b in zip(before, flat)) and int(state["step"]) == 1
        g[1][3, 3] = 0.0
        T.p2_adamw(p, g, **state, **HYPER, square_sum=T.p2_square_sum(g))
        assert int(state["step"]) == 2 and not torch.equal(p[0], before[0])


def test_adamw_without_a_check_takes_what_it_is_given(T):
    p, g = adam_inputs([(600,)], F32, F32, 8)
    g[0][300] = math.nan
    state = T.p2_adamw_state(p, 8)
    T.p2_adamw(p, g, **state, **HYPER)
    assert p[0].isnan().sum() == 1 and state["mean_scales"][0].isnan().tolist() == [False, True, False] and state["square_scales"][0].isnan().tolist() == [False, True, False]
    m, v = T.p2_adamw_values(state["means"], state["squares"], state["mean_scales"], state["square_scales"])
    assert m[0].isnan().tolist() == [256 <= i < 512 for i in range(600)] and v[0].isnan().tolist() == m[0].isnan().tolist()


def test_adamw_of_zero_and_tiny_gradients(T):
    """Nothing is divided by 0, blocks below 2^-100 are held as zeros, and a small square beside a large one is not lost."""
    p = [torch.ones(1024, device="cuda")]
    g = [torch.zeros(1024, device="cuda")]
    state = T.p2_adamw_state(p, 8)
    T.p2_adamw(p, g, **state, lr=0.1)
    assert (p[0] == 1).all() and (state["mean_scales"][0] == 0).all()
    g[0][:256], g[0][256], g[0][257:512], g[0][512:] = 1e-25, 1e3, 1e-12, 1e-30
    T.p2_adamw(p, g, **state, lr=0.1)
    assert p[0].isfinite().all() and (state["squares"][0][256:512] > 0).all() and (state["square_scales"][0][[0, 2, 3]] == 0).all()
    assert float(p[0][256]) != 1.0 and (state["squares"][0][:256] == 0).all()
    T.p2_adamw(p, [torch.zeros_like(g[0])], **state, lr=0.1)
    assert p[0].isfinite().all() and ((p[0] - 1).abs() < 0.5).all()


@pytest.mark.parametrize("eps,beta2", [(1e-15, 0.999), (1e-12, 0.999999), (1e-8, 0.9999999), (1e-25, 0.9)])
def test_adamw_of_squares_that_are_no_normal_numbers(T, eps, beta2):
    # A gradient of 2.6e-19 sqrt(1 / (1 - beta2)) leaves (1 - beta2) g^2 = 6.8e-38 / 10 = 6.8e-39 and less, below 2^-126 = 1.2e-38, where a step is 2^-149 = 1.4e-45:
    # rounding to it is 1.4e-45 / 2 of 6e-41 = 1.2e-5 at most, half of that in the root, and at most 20 U for the other operations.
    g = torch.linspace(0.1, 1.0, 500, device="cuda") * (2.6e-19 * math.sqrt(0.1 / (1 - beta2)))
    p = torch.zeros_like(g)
    T.p2_adamw([p], [g], **T.p2_adamw_state([p]), lr=1.0, betas=(0.9, beta2), eps=eps)
    want = -g.double() / (g.double().abs() + eps)
    compare(p, want, (0.6e-5 + 20 * U) * want.abs(), (eps, beta2))


@pytest.mark.parametrize("values", [1, 256 * 8 * 1024, 256 * 8 * 1024 + 1])
def test_adamw_counts_its_steps_whatever_it_launches(T, values):
    p, g = torch.zeros(values, device="cuda"), torch.ones(values, device="cuda")
    state = T.p2_adamw_state([p])
    for t in (0, 1, 2, 2 ** 40 - 10):
        state["step"].fill_(t)
        T.p2_adamw([p], [g], **state, lr=0.0)
        assert int(state["step"]) == t + 1
    T.p2_adamw([p], [g], **state, lr=0.0, square_sum=torch.full((), INF, dtype=F64, device="cuda"))
    assert int(state["step"]) == 2 ** 40 - 9


def test_adamw_copies_into_the_gradients(T):
    p, g = adam_inputs([(1000,), (3, 7)], F32, BF16, 32)
    q, d = [t.clone() for t in p], [t.clone() for t in g]
    T.p2_adamw(p, g, **T.p2_adamw_state(p), **HYPER, copies=g)
    T.p2_adamw(q, d, **T.p2_adamw_state(q), **HYPER)
    assert all(torch.equal(a, b) and torch.equal(c, b.to(BF16)) for a, b, c in zip(p, q, g))


def test_adamw_rate_and_factor_on_the_device(T):
    one, two = (adam_inputs([(1000,)], F32, F32, 32) for _ in range(2))
    s1, s2 = T.p2_adamw_state(one[0]), T.p2_adamw_state(two[0])
    T.p2_adamw(one[0], one[1], **s1, lr=0.5, rate=torch.full((), 0.25, device="cuda"), grad_factor=0.5)
    T.p2_adamw(two[0], [0.5 * g for g in two[1]], **s2, lr=0.125)
    assert torch.equal(one[0][0], two[0][0]) and torch.equal(s1["squares"][0], s2["squares"][0])


def test_adamw_of_many_tensors_is_that_of_each(T):
    shapes = [SIZES[i % len(SIZES)] for i in range(150)]
    for bits in (32, 8):
        p, g = adam_inputs(shapes, BF16, BF16, bits)
        q = [t.clone() for t in p]
        state, alone = T.p2_adamw_state(p, bits), [T.p2_adamw_state([t], bits) for t in q]
        for _ in range(2):
            T.p2_adamw(p, g, **state, **HYPER)
            for t, d, s in zip(q, g, alone):
                T.p2_adamw([t], [d], **s, **HYPER)
        assert all(torch.equal(a, b) for a, b in zip(p, q)) and all(torch.equal(a, s["means"][0]) for a, s in zip(state["means"], alone))


def test_adamw_leaves_what_is_between_tensors(T):
    flat = torch.full((5000,), 7.0, device="cuda")
    m, v = torch.full((5000,), 7.0, device="cuda"), torch.full((5000,), 7.0, device="cuda")
    parts = [(3, 1000), (1004, 257), (2000, 2999)]
    cut = lambda x: [x[a:a + n] for a, n in parts]  # noqa: E731
    T.p2_adamw(cut(flat), [torch.ones(n, device="cuda") for _, n in parts], cut(m), cut(v), torch.zeros((), dtype=torch.int64, device="cuda"))
    inside = torch.zeros(5000, dtype=torch.bool, device="cuda")
    for a, n in parts:
        inside[a:a + n] = True
    for t in (flat, m, v):
        assert (t[~inside] == 7).all() and (t[inside] != 7).all()


def test_what_autograd_saved_of_a_parameter_is_out_of_date_after_a_step(T):
    p = torch.nn.Parameter(torch.ones(8, device="cuda"))
    loss = (p * p).sum()
    T.p2_adamw([p], [torch.ones(8, device="cuda")], **T.p2_adamw_state([p]))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_a_step_that_is_refused_leaves_what_autograd_saved(T):
    p = torch.nn.Parameter(torch.full((8,), 3.0, device="cuda"))
    loss = (p * p).sum()
    with pytest.raises(T.P2Error):
        T.p2_adamw([p], [torch.ones(8, device="cuda")], **T.p2_adamw_state([p]), lr=INF)
    loss.backward()
    assert (p.grad == 6.0).all()


def test_adamw_of_parameters_made_in_inference_mode(T):
    """Autograd keeps no count of their changes, so there is nothing to be out of date; the step is that of ordinary tensors, and no error comes after it."""
    with torch.inference_mode():
        p, copy = torch.ones(300, device="cuda"), torch.zeros(300, dtype=BF16, device="cuda")
    q, g = torch.ones(300, device="cuda"), torch.linspace(-1, 1, 300, device="cuda")
    state, other = T.p2_adamw_state([p]), T.p2_adamw_state([q])
    T.p2_adamw([p], [g], **state, copies=[copy])
    T.p2_adamw([q], [g], **other)
    with torch.inference_mode():
        T.p2_adamw([p], [g], **state, copies=[copy])
        T.p2_adamw([q], [g], **other)
        assert torch.equal(p, q) and torch.equal(copy, q.to(BF16)) and int(state["step"]) == 2


@pytest.mark.parametrize("values", [300, 256 * 8 * 1024 + 1])
@pytest.mark.parametrize("step", [-1, -5, -2 ** 63, 2 ** 40 - 1])
def test_adamw_leaves_out_a_step_whose_number_is_none(T, values, step):
    p, g = torch.ones(values, device="cuda"), torch.ones(values, device="cuda")
    state = T.p2_adamw_state([p])
    state["step"].fill_(step)
    T.p2_adamw([p], [g], **state, lr=0.1)
    assert (p == 1).all() and not state["means"][0].any() and not state["squares"][0].any() and int(state["step"]) == step


def test_adamw_of_more_values_than_32_bits_count(T):
    n = (1 << 31) + 1001
    p, g = torch.zeros(n, dtype=BF16, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    g[-1001:] = draw(1, 1001).to(BF16)
    state = T.p2_adamw_state([p], 8)
    total = T.p2_square_sum([g])
    assert abs(float(total) / float(g[-1001:].double().square().sum()) - 1) < 1e-12
    T.p2_adamw([p], [g], **state, **HYPER)
    small = torch.zeros(1001, dtype=BF16, device="cuda")
    T.p2_adamw([small], [g[-1001:]], **T.p2_adamw_state([small], 32), **HYPER)
    assert torch.equal(p[-1001:], small) and not p[:4096].any() and int(state["squares"][0][-1]) > 0


# -------------------------------------------------------------------------------------------------- products

def activate(z, name):
    f = torch.nn.functional
    return {None: lambda: z, "relu": lambda: f.relu(z), "gelu": lambda: f.gelu(z), "gelu_tanh": lambda: f.gelu(z, approximate="tanh"), "silu": lambda: f.silu(z)}[name]()


def slope(z, name):
    z = z.detach().requires_grad_(True)
    return torch.autograd.grad(activate(z, name).sum(), z)[0] if name else torch.ones_like(z)


def linear_inputs(rows, inner, outer, kind, pad=0, seed=0):
    x = draw(seed, rows, inner + pad).to(kind)[:, pad:]
    w = draw(seed + 1, outer, inner + 2 * pad, scale=inner ** -0.5).to(kind)[:, :inner]
    return x, w, draw(seed + 2, outer, scale=0.3).to(kind), draw(seed + 3, rows, outer + pad).to(kind)[:, :outer]


def check_linear(T, x, w, b, res, activation, keep=True):
    y, z = T.p2_linear_forward(x, w, b, activation=activation, residual=res, keep=keep)
    xd, wd = x.double(), w.double()
    rz = xd @ wd.t() + (0 if b is None else b.double())
    inner = x.shape[-1]
    size = xd.abs() @ wd.abs().t() + (0 if b is None else b.double().abs())
    slack = (inner / 4 + 32) * 2 * U * size
    if keep:
        compare(z, rz, slack, "z")
    # an activation's slope is 1.13 at most, its own exponentials are off by 2 U (|z| + 40) of its value
    ry = activate(rz, activation)
    slack_y = 1.2 * slack + (0 if activation is None else 2 * U * (rz.abs() + 40) * (ry.abs() + 1e-3 * rz.abs()))
    if res is not None:
        ry = ry + res.double()
        slack_y = slack_y + U * ry.abs() + U * res.double().abs()
    compare(y, ry, slack_y, "y")
    return y, z


def check_linear_gradient(T, x, w, z, dy, activation, dtype=None):
    dx, dw, db = T.p2_linear_backward(dy, x, w, z, activation=activation, dtype=dtype)
    xd, wd = x.double(), w.double()
    sl = slope(z.double(), activation) if activation else torch.ones_like(dy, dtype=F64)
    dz = dy.double() * sl
    own = 2 * U * (40 + (0 if z is None else z.double().abs())) * dy.double().abs()        # of the slope
    half = torch.finfo(x.dtype).eps / 2 if activation else 0.0                              # dz is rounded for the products
    if x.dtype == F16 and activation:
        own_product = own + 2.0 ** -25                                                      # (fp16's smallest step)
    else:
        own_product = own
    off = half * dz.abs() + own_product
    rows, outer = dy.shape
    compare(dx, dz @ wd, (outer / 4 + 32) * 2 * U * (dz.abs() @ wd.abs()) + 1.1 * off @ wd.abs(), "dx")
    compare(dw, dz.t() @ xd, (rows / 4 + 32) * 2 * U * (dz.abs().t() @ xd.abs()) + 1.1 * off.t() @ xd.abs(), "dweight")
    compare(db, dz.sum(0), (64 + rows / 64) * U * dz.abs().sum(0) + own.sum(0), "dbias")
    return dx, dw, db


LINEAR = [(1, 1, 1), (1, 7, 3), (1, 8, 4), (1, 64, 17), (1, 1000, 777), (2, 513, 5), (3, 64, 64), (4, 200, 33), (5, 1, 1), (5, 63, 66), (5, 4096, 10), (8, 8, 8), (16, 16, 16),
          (17, 72, 130), (63, 65, 64), (64, 64, 65), (65, 128, 129), (100, 1000, 50), (127, 40, 260), (300, 24, 515), (33, 5000, 40), (70, 20001, 66), (515, 136, 257), (16, 1000, 1000), (32, 520, 8300), (20, 264, 8192), (9, 65, 33),
          (31, 129, 70), (2, 2049, 100), (1, 8192, 40), (12, 2047, 8200)]


@pytest.mark.parametrize("rows,inner,outer", LINEAR)
@pytest.mark.parametrize("kind,pad", [(F32, 0), (BF16, 0), (F16, 3), (BF16, 8), (F32, 1)])
def test_linear(T, rows, inner, outer, kind, pad):
    x, w, b, res = linear_inputs(rows, inner, outer, kind, pad)
    activation = [None, "relu", "gelu", "gelu_tanh", "silu"][(rows + inner + outer) % 5]
    check_linear(T, x, w, b, res, activation)
    y, none = T.p2_linear_forward(x, w)
    assert none is None and y.dtype == kind
    dy = draw(9, rows, outer + pad).to(kind)[:, pad:]
    z = T.p2_linear_forward(x, w, b, activation=activation, keep=True)[1]
    check_linear_gradient(T, x, w, z, dy, activation)
    check_linear_gradient(T, x, w, None, dy, None, dtype=F32)


@pytest.mark.parametrize("activation", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_activations(T, activation, kind):
    """Through a product with ones: from far below 0 to far above, 0 and its neighbours."""
    z = torch.cat([torch.linspace(-30, 30, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e4, -1e4])]).cuda().to(kind)[:, None]
    one = torch.ones(1, 1, dtype=kind, device="cuda")
    for rows in (4, z.numel()):
        check_linear(T, z[:rows], one, None, None, activation)
    dy = torch.ones_like(z)
    dx, _, _ = T.p2_linear_backward(dy, z, one, z, activation=activation)
    want = slope(z.double(), activation)
    compare(dx, want, 2 * U * (40 + z.double().abs()) * (1 + z.double().abs() * (z.double().abs() < 30)), "slope")


@pytest.mark.parametrize("activation", [None, "relu", "gelu", "gelu_tanh", "silu"])
def test_the_slopes_against_differences(activation):
    z = draw(1, 200) * 3
    z = z[z.abs() > 1e-3]
    want = (activate(z + 1e-6, activation) - activate(z - 1e-6, activation)) / 2e-6
    assert (slope(z, activation) - want).abs().max() < 1e-8


@pytest.mark.parametrize("rows,inner,outer,kind", [(3500, 200, 3600, BF16), (3590, 72, 3700, F16), (3500, 33, 3600, F32), (1, 4096, 5000, BF16), (2000, 264, 1500, BF16), (1500, 1500, 1500, F32), (1531, 1000, 777, F32), (1531, 1001, 777, F32), (3500, 8192, 2500, BF16), (4096, 1500, 5120, F16), (4100, 2056, 4104, BF16), (8200, 1032, 4104, F16), (8200, 4096, 1032, BF16)])
def test_linear_large(T, rows, inner, outer, kind):
    x, w, b, res = linear_inputs(rows, inner, outer, kind)
    y, z = check_linear(T, x, w, b, res, "gelu")
    check_linear_gradient(T, x, w, z, res, "gelu")


@pytest.mark.parametrize("kind,rows,inner,outer,activation", [(BF16, 8200, 1032, 4104, None), (F16, 8200, 1032, 4104, "silu"), (BF16, 8192, 2056, 4104, "gelu_tanh"), (BF16, 16391, 1032, 1544, None),
                                                               (BF16, 8, 1003, 777, "silu"), (BF16, 40, 300, 200, "silu"), (F16, 64, 1001, 500, None), (F16, 3, 100, 2000, None), (F32, 5, 515, 300, "gelu"), (BF16, 1, 4100, 9000, "relu")])
def test_gradients_of_matrices_within_others(T, kind, rows, inner, outer, activation):
    # what lies around them is NaN, which any product with it would show
    def within(seed, r, c, scale=1.0):
        around = torch.full((r + 9, c + 24), math.nan, device="cuda", dtype=kind)
        around[4:4 + r, 8:8 + c] = draw(seed, r, c, scale=scale).to(kind)
        return around[4:4 + r, 8:8 + c]

    x, w, dy = within(1, rows, inner), within(2, outer, inner, inner ** -0.5), within(3, rows, outer)
    z = within(4, rows, outer) if activation else None
    dx, dw, db = check_linear_gradient(T, x, w, z, dy, activation)
    one, _, _ = T.p2_linear_backward(dy, x, w, z, activation=activation, dweight=False, dbias=False)
    _, two, _ = T.p2_linear_backward(dy, x, w, z, activation=activation, dx=False, dbias=False)
    _, _, three = T.p2_linear_backward(dy, x, w, z, activation=activation, dx=False, dweight=False)
    assert torch.equal(dx, one) and torch.equal(dw, two) and torch.equal(db, three)
    again = T.p2_linear_backward(dy.contiguous(), x.contiguous(), w.contiguous(), None if z is None else z.contiguous(), activation=activation)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))


@pytest.mark.parametrize("rows,inner,outer", [(1, 64, 40), (2, 515, 300), (5, 1000, 777), (8, 4100, 1000)])
@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("activation", ["gelu", "gelu_tanh", "silu"])
def test_gradients_of_a_few_rows_take_dz_as_it_is(T, rows, inner, outer, kind, activation):
    """Up to eight rows are multiplied in 32 bits: dz = dy activation'(z) is not rounded in between."""
    x, w, _, dy = linear_inputs(rows, inner, outer, kind)
    z = draw(7, rows, outer).to(kind)
    dx, dw, db = T.p2_linear_backward(dy, x, w, z, activation=activation, dtype=F32)
    dz = dy.double() * slope(z.double(), activation)
    own = 2 * U * (40 + z.double().abs()) * dy.double().abs()
    assert dw.dtype == F32
    compare(dw, dz.t() @ x.double(), (rows + 1) * 2 * U * (dz.abs().t() @ x.double().abs()) + 1.1 * own.t() @ x.double().abs(), "dweight")
    compare(dx, dz @ w.double(), (outer / 4 + 32) * 2 * U * (dz.abs() @ w.double().abs()) + 1.1 * own @ w.double().abs(), "dx")


@pytest.mark.parametrize("rows,outer,kinds", [(3, 127, (BF16, F16)), (4, 128, (BF16, F16)), (8, 767, (BF16, F16)), (5, 768, (BF16, F16)), (8, 63, (F32,)), (5, 64, (F32,)), (4, 5, (F32,))])
@pytest.mark.parametrize("inner", [8, 77, 520])
def test_gradients_of_a_few_rows_and_few_of_the_weight_s(T, rows, outer, kinds, inner):
    """On either side of what decides which kernels make them."""
    for kind in kinds:
        x, w, _, dy = linear_inputs(rows, inner, outer, kind, pad=outer % 2)
        z = draw(7, rows, outer).to(kind)
        for activation in (None, "silu"):
            check_linear_gradient(T, x, w, z if activation else None, dy, activation)


def test_linear_of_more_values_than_32_bits_count(T):
    rows, inner = 1 << 20, 2056
    x = torch.zeros(rows, inner, dtype=BF16, device="cuda")
    x[-300:] = draw(1, 300, inner).to(BF16)
    w = draw(2, 16, inner, scale=0.02).to(BF16)
    y, _ = T.p2_linear_forward(x, w)
    assert not y[:-300].any()
    check = (x[-300:].double() @ w.double().t())
    compare(y[-300:], check, (inner / 4 + 32) * 2 * U * (x[-300:].double().abs() @ w.double().abs().t()), "y")
    dy = torch.zeros(rows, 16, dtype=BF16, device="cuda")
    dy[-300:] = draw(3, 300, 16).to(BF16)
    dx, dw, db = T.p2_linear_backward(dy, x, w, dtype=F32)
    assert not dx[:-300].any()
    d = dy[-300:].double()
    compare(dx[-300:], d @ w.double(), 100 * U * (d.abs() @ w.double().abs()), "dx")
    compare(dw, d.t() @ x[-300:].double(), 300 * U * (d.abs().t() @ x[-300:].double().abs()), "dweight")
    compare(db, d.sum(0), 400 * U * d.abs().sum(0), "dbias")


def test_linear_infinities_and_nan_stay_in_their_rows(T):
    for rows in (3, 80):
        x, w, b, _ = linear_inputs(rows, 100, 70, F32)
        x[0, 5], x[1, 6], w[3, 7] = INF, math.nan, INF
        y, _ = T.p2_linear_forward(x, w, b)
        want = x.double() @ w.double().t() + b.double()
        assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.isinf(), want.isinf())
        assert y[2:, :3].isfinite().all()


def test_linear_forms_of_the_arguments(T):
    x, w, b, res = linear_inputs(24, 40, 30, BF16)
    y, z = T.p2_linear_forward(x, w, b, activation="silu", residual=res, keep=True)
    x3 = x.view(2, 3, 4, 40)
    y3, z3 = T.p2_linear_forward(x3, w, b, activation="silu", residual=res.reshape(2, 3, 4, 30), keep=True)
    assert y3.shape == (2, 3, 4, 30) and torch.equal(y3.view(24, 30), y) and torch.equal(z3.view(24, 30), z)
    one = T.p2_linear_forward(x[5], w, b)[0]
    assert one.shape == (30,) and ((one.double() - T.p2_linear_forward(x, w, b)[0][5].double()).abs() <= 0.01 * one.double().abs() + 1e-3).all()
    turned = w.t().contiguous().t()
    assert torch.equal(T.p2_linear_forward(x.t().contiguous().t(), turned, b, activation="silu", residual=res)[0], y)
    wide = torch.zeros(30, 1, dtype=BF16, device="cuda").expand(30, 40)
    assert not T.p2_linear_forward(x, wide)[0].any()
    same = T.p2_linear_forward(x, w, b, activation="silu", residual=res[:1].expand(24, 30))[0]      # a broadcast residual is written out first
    assert torch.equal(same, T.p2_linear_forward(x, w, b, activation="silu", residual=res[:1].repeat(24, 1))[0])
    dx, dw, db = T.p2_linear_backward(res, x, w, z, activation="silu", dx=False, dbias=False)
    assert dx is None and db is None and dw.shape == w.shape and dw.dtype == BF16
    dx, dw, db = T.p2_linear_backward(res, x, w, z, activation="silu", dweight=False, dtype=F32)
    assert dw is None and dx.dtype == BF16 and db.dtype == F32
    dx, dw, db = T.p2_linear_backward(res.view(4, 6, 30), x.view(4, 6, 40), w, z.view(4, 6, 30), activation="silu")
    full = T.p2_linear_backward(res, x, w, z, activation="silu")
    assert dx.shape == (4, 6, 40) and torch.equal(dx.view(24, 40), full[0]) and torch.equal(dw, full[1]) and torch.equal(db, full[2])
    expanded = torch.ones((), dtype=BF16, device="cuda").expand(24, 30)                             # the gradient that a sum sends back
    check_linear_gradient(T, x, w, None, expanded, None)
    none = T.p2_linear_forward(x[:0], w, b, keep=True)
    assert none[0].shape == none[1].shape == (0, 30)
    dx, dw, db = T.p2_linear_backward(res[:0], x[:0], w)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()


@pytest.mark.parametrize("activation,room", [(None, 1 << 22), ("silu", (64 << 20) + (1 << 22))])
def test_gradients_allocate_what_they_use(T, activation, room):
    x, w, _, dy = linear_inputs(8192, 4096, 4096, BF16)
    z = dy.clone()
    for wanted in ((True, True, True), (True, False, False), (False, True, False), (False, False, True)):
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        out = T.p2_linear_backward(dy, x, w, z if activation else None, activation=activation, dx=wanted[0], dweight=wanted[1], dbias=wanted[2])
        results = sum(t.numel() * t.element_size() for t in out if t is not None)
        assert torch.cuda.max_memory_allocated() - before <= results + room
        if not any(wanted[:2]):
            assert torch.cuda.max_memory_allocated() - before <= results + (1 << 22)


def test_results_in_columns_of_the_buffer_they_are_made_from(T):
    """The C ABI's: every matrix has columns of its own in one buffer."""
    import ctypes as C
    rows, inner, outer = 70, 40, 24
    x, w, b, res = linear_inputs(rows, inner, outer, F32)
    want, z = T.p2_linear_forward(x, w, b, activation="silu", residual=res, keep=True)
    wide = torch.full((rows, 2 * inner + 4 * outer), 7.0, device="cuda")
    at, part = 0, {}
    for name, n in (("x", inner), ("y", outer), ("dx", inner), ("z", outer), ("dy", outer), ("res", outer)):
        part[name], at = wide[:, at:at + n], at + n
    part["x"].copy_(x), part["res"].copy_(res), part["dy"].copy_(res)
    p, s = {k: v.data_ptr() for k, v in part.items()}, wide.stride(0)
    L, n, stream = T.lib(), C.c_int64(), torch.cuda.current_stream().cuda_stream
    assert L.p2_linear_forward_workspace(p["x"], s, w.data_ptr(), inner, 0, rows, inner, outer, C.byref(n)) == 0
    work = torch.empty(max(n.value, 256), dtype=torch.uint8, device="cuda")
    assert L.p2_linear_forward(p["x"], s, w.data_ptr(), inner, b.data_ptr(), p["res"], s, 0, 4, rows, inner, outer, p["y"], s, p["z"], s, work.data_ptr(), n.value, stream) == 0
    assert torch.equal(part["y"], want) and torch.equal(part["z"], z)
    assert L.p2_linear_forward(p["x"], s, w.data_ptr(), inner, b.data_ptr(), p["res"], s, 0, 4, rows, inner, outer, p["res"], s, p["z"], s, work.data_ptr(), n.value, stream) == 0
    assert torch.equal(part["res"], want)                      # y may be the residual
    dx, dw, db = T.p2_linear_backward(res, x, w, z, activation="silu")
    assert L.p2_linear_backward_workspace(0, rows, inner, outer, C.byref(n)) == 0
    work = torch.empty(max(n.value, 256), dtype=torch.uint8, device="cuda")
    dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
    assert L.p2_linear_backward(p["dy"], s, p["z"], s, p["x"], s, w.data_ptr(), inner, 0, 4, rows, inner, outer, p["dx"], s, dw2.data_ptr(), inner, db2.data_ptr(), 0, work.data_ptr(), n.value, stream) == 0
    assert torch.equal(part["dx"], dx) and torch.equal(dw2, dw) and torch.equal(db2, db) and torch.equal(part["x"], x)


# ------------------------------------------------------------------------------------------- as they are used

def _step_inputs(seed):
    w = [draw(seed, 96, 64, scale=0.1).float(), draw(seed + 1, 96, scale=0.1).float(), draw(seed + 2, 24, 96, scale=0.1).float()]
    return [draw(seed + 3, 300, 64).float(), draw(seed + 4, 300, 96).float(), draw(seed + 5, 300, 4).float(), draw(seed + 6, 24, scale=0.05).float(), *w]


def _step(T, x, dy, dgate, bias, w, b, router, state, total=None):
    """A layer, a router over experts, their gradients and the weights' step."""
    kw = dict(score="sigmoid", renormalise=True, scale=2.0)
    h, z = T.p2_linear_forward(x, w, b, activation="gelu", keep=True)
    logits, _ = T.p2_linear_forward(h, router)
    r = T.p2_route_forward(logits, 4, bias=bias, groups=4, group_limit=2, group_best=2, **kw)
    dlogits = T.p2_route_backward(logits, r["expert"], dgate, **kw)
    dh, drouter, _ = T.p2_linear_backward(dlogits, h, router, dbias=False)
    dx, dw, db = T.p2_linear_backward(dh + dy, x, w, z, activation="gelu")
    grads = [dw, db, drouter]
    total = T.p2_square_sum(grads)
    T.p2_adamw([w, b, router], grads, **state, **HYPER, square_sum=total, max_norm=1.0)
    return [h, logits, r["expert"], r["gate"], r["counts"], dlogits, dx, *grads, total, T.p2_route_bias(bias, r["counts"], 1e-3)]


def _state(T, inputs, bits=8):
    return T.p2_adamw_state(inputs[4:], bits)


def _all(state):
    return [t for v in state.values() if v is not None for t in (v if isinstance(v, list) else [v])]


def test_a_step_of_them_together(T):
    """Against the same step by torch's own derivatives in 64 bits."""
    inputs = _step_inputs(1)
    x, dy, dgate, bias, w, b, router = (t.double() for t in inputs)
    state = _state(T, inputs, 32)
    out = _step(T, *inputs, state)
    w.requires_grad_(True), b.requires_grad_(True), router.requires_grad_(True), x.requires_grad_(True)
    h = torch.nn.functional.gelu(x @ w.t() + b)
    logits = h @ router.t()
    gate = gates_of(logits, out[2], "sigmoid", True, 2.0)
    dx, dw, db, dr = torch.autograd.grad((gate * dgate).sum() + (h * dy).sum(), (x, w, b, router))
    want = route_reference(out[1], 4, score="sigmoid", bias=inputs[3], groups=4, group_limit=2, group_best=2, renormalise=True, scale=2.0)
    assert torch.equal(out[2], want["expert"]) and torch.equal(out[4], want["counts"])
    # products of some hundred terms each, three of them one after the other
    for got, ref in zip((out[0], out[1], out[6], out[7], out[8], out[9]), (h, logits, dx, dw, db, dr)):
        assert float((got.double() - ref.detach()).norm() / ref.detach().norm()) < 3 * 400 * U
    total = sum(float(g.square().sum()) for g in (dw, db, dr))
    assert abs(float(out[10]) / total - 1) < 1e-4
    for i, (p, g) in enumerate(((w, dw), (b, db), (router, dr))):
        g = g * min(1.0, total ** -0.5)
        rp, _, _, _ = adam_reference(p.detach(), g, 0 * g, 0 * g, 1, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
        assert ((inputs[4 + i].double() - rp).abs() <= 2 * HYPER["lr"] * (g.abs() < 1e-5) + 1e-2 * HYPER["lr"]).all()       # the first step is lr sign(g), where g is not next to 0


def test_the_same_bits_every_time(T):
    for bits in (32, 8):
        seen = []
        for _ in range(3):
            inputs = _step_inputs(2)
            state = _state(T, inputs, bits)
            out = [t for _ in range(2) for t in _step(T, *inputs, state)]
            seen.append([*out, *inputs, *_all(state)])
        assert all(torch.equal(a, b) for s in seen[1:] for a, b in zip(seen[0], s))


def test_a_captured_step(T):
    """Replayed several times, with eager work of the same operators between, each replay is the eager step."""
    inputs, eager = _step_inputs(3), _step_inputs(3)
    state, eager_state = _state(T, inputs), _state(T, eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(T, *inputs, state)                                # warm up, and the first step
    torch.cuda.current_stream().wait_stream(side)
    _step(T, *eager, eager_state)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(T, *inputs, state)
    for _ in range(4):
        graph.replay()
        want = _step(T, *eager, eager_state)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all(torch.equal(a, b) for a, b in zip([*inputs, *_all(state)], [*eager, *_all(eager_state)]))
    assert int(state["step"]) == 5


def test_two_captured_steps_that_share_nothing_but_the_pool(T):
    one, two, ref1, ref2 = (_step_inputs(s) for s in (4, 5, 4, 5))
    states = [_state(T, i) for i in (one, two, ref1, ref2)]
    graphs, outs = [], []
    for inputs, state in ((one, states[0]), (two, states[1])):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            _step(T, *inputs, state)
        torch.cuda.current_stream().wait_stream(side)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], pool=graphs[0].pool() if len(graphs) > 1 else None):
            outs.append(_step(T, *inputs, state))
    for inputs, state in ((ref1, states[2]), (ref2, states[3])):
        _step(T, *inputs, state)
    for _ in range(3):
        for g, inputs, state, n in ((graphs[0], ref1, states[2], 0), (graphs[1], ref2, states[3], 1)):
            g.replay()
            _step(T, *inputs, state)
            torch.cuda.synchronize()
            mine = (one, two)[n]
            assert all(torch.equal(a, b) for a, b in zip([*mine, *_all(states[n])], [*inputs, *_all(state)]))


def test_steps_on_two_streams_at_once(T):
    alone = []
    for s in (6, 7):
        inputs = _step_inputs(s)
        state = _state(T, inputs)
        alone.append([t.clone() for _ in range(3) for t in _step(T, *inputs, state)])
    sets = [(_step_inputs(s), torch.cuda.Stream()) for s in (6, 7)]
    states = [_state(T, i) for i, _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(3):
        for n, (inputs, stream) in enumerate(sets):
            with torch.cuda.stream(stream):
                got[n] += _step(T, *inputs, states[n])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g, a_ in zip(got, alone) for a, b in zip(g, a_))


def test_calls_leave_nothing_behind(T):
    import sys
    inputs = _step_inputs(8)
    state = _state(T, inputs)
    _step(T, *inputs, state)
    torch.cuda.synchronize()
    room, held = torch.cuda.memory_allocated(), [sys.getrefcount(t) for t in inputs]
    for _ in range(20):
        _step(T, *inputs, state)
    with pytest.raises(T.P2Error):
        T.p2_adamw(inputs[4:], inputs[4:], **_state(T, inputs, 32) | {"means": inputs[4:6]})
    assert torch.cuda.memory_allocated() == room and [sys.getrefcount(t) for t in inputs] == held


def test_inputs_are_left_as_they_were(T):
    x, w, b, res = linear_inputs(70, 65, 66, BF16, pad=3)
    z = draw(1, 70, 66).to(BF16)
    logits, bias = draw(2, 300, 64).float(), draw(3, 64).float()
    inputs = [x, w, b, res, z, logits, bias]
    before = [t.clone() for t in inputs]
    T.p2_linear_forward(x, w, b, activation="gelu", residual=res, keep=True)
    T.p2_linear_backward(res, x, w, z, activation="gelu")
    r = T.p2_route_forward(logits, 4, bias=bias, score="sigmoid", groups=8, group_limit=3)
    T.p2_route_backward(logits, r["expert"], r["gate"], score="sigmoid")
    T.p2_route_bias(bias, r["counts"], 0.1)
    T.p2_square_sum([x, w])
    assert all(torch.equal(a, b) for a, b in zip(before, inputs))


def test_results_are_ordinary_tensors(T):
    x, w, _, _ = linear_inputs(6, 40, 24, BF16)
    y, z = T.p2_linear_forward(x, w, keep=True)
    like = torch.empty(6, 24, dtype=BF16, device="cuda")
    for t in (y, z):
        assert (t.shape, t.stride(), t.dtype, t.device, t.is_leaf, t.requires_grad, t.is_inference(), t._version) == (like.shape, like.stride(), BF16, like.device, True, False, False, 0)
    want = 2 * y.double()
    y.requires_grad_()
    (y * y).sum().backward()
    compare(y.grad, want, 0.0, "a result's gradient")
    z.add_(1)
    assert z._version == 1
    with torch.inference_mode():
        assert T.p2_linear_forward(x, w)[0].is_inference()
    before = torch.cuda.memory_allocated()
    big = T.p2_route_forward(torch.zeros(1 << 16, 64, device="cuda"), 8)
    assert torch.cuda.memory_allocated() - before >= (1 << 16) * 64
    del big
    assert torch.cuda.memory_allocated() == before


FIRST_CALL_FOLLOWS_SHAPES = """
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from paper_2110_10548_amd import train as T
x = torch.randn(5, 64, device="cuda")
with FakeTensorMode(allow_non_fake_inputs=True):
    for call in (lambda: T.p2_layer_norm_forward(torch.zeros(5, 64, device="cuda")), lambda: T.p2_layer_norm_forward(x)):
        try:
            call()
            raise SystemExit("not refused")
        except T.P2Error:
            pass
y, mean, rstd = T.p2_layer_norm_forward(x)
r = T.p2_route_forward(x, 3)
for t in (y, mean, rstd, r["gate"], T.p2_square_sum([x])):
    assert t.device == x.device and t.untyped_storage().device == x.device and type(t) is torch.Tensor, t.device
assert abs(float(T.p2_square_sum([x])) / float(x.double().square().sum()) - 1) < 1e-12
assert (y - torch.nn.functional.layer_norm(x, (64,))).abs().max() < 1e-5
print("as ever")
"""


def test_a_first_call_that_follows_shapes_alone_leaves_the_others_as_they_are(T):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", FIRST_CALL_FOLLOWS_SHAPES], cwd=root, capture_output=True, text=True, timeout=100)
    assert run.returncode == 0 and "as ever" in run.stdout, run.stdout + run.stderr


def test_a_parameter_that_would_not_train_is_warned_of(T):
    import warnings
    x, w, b, res = linear_inputs(6, 40, 12, F32)
    p = torch.nn.Parameter(w.clone())
    zp = torch.nn.Parameter(draw(1, 6, 12).float())
    expert = T.p2_route_forward(zp.detach(), 2)["expert"]
    for call in (lambda: T.p2_linear_forward(x, p), lambda: T.p2_linear_backward(res, x, p), lambda: T.p2_route_forward(zp, 2),
                 lambda: T.p2_route_backward(zp, expert, res[:, :2].contiguous()), lambda: T.p2_square_sum([p])):
        with pytest.warns(UserWarning, match="nothing is recorded for autograd") as caught:
            call()
        assert len(caught) == 1 and caught[0].filename == __file__
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        T.p2_adamw([p], [w], **T.p2_adamw_state([p]))            # a step is what parameters are for
        with torch.no_grad():
            T.p2_linear_forward(x, p)
