"""Cases of more training operators: the choice of experts by biased scores in groups, AdamW over many tensors with states in
32 or 8 bits, matrix products with bias, activation and residual.

`run` computes them by elementary torch operations where `own` is false and through `paper_2110_10548_amd.train`
where it is true.  Sizes are those of training steps and of single tokens, odd and ragged ones among them.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
BIAS_RATE = 1e-3                             # how far an expert's bias moves a step
BETAS, ADAM_EPS, DECAY, LR = (0.9, 0.95), 1e-8, 0.1, 1e-3
BLOCK = 256                                  # values that share the scale of an 8-bit state
LEAST = 2.0 ** -100                          # blocks that hold nothing larger are held as zeros


def listed():
    return [
        # one token's choice: latency only
        dict(name="choice one token", op="choice", tokens=1, experts=64, k=2, type="fp32", score="softmax", biased=False, groups=1,
             limit=1, best=1, renormalise=True, scale=1.0, masked=False),
        # a batch over many experts on eight machines, four of which a token may go to: sigmoid scores, a bias that balances
        dict(name="choice batch", op="choice", tokens=65536, experts=256, k=8, type="fp32", score="sigmoid", biased=True, groups=8,
             limit=4, best=2, renormalise=True, scale=2.5, masked=False),
        # ragged sequences: a tenth of the tokens is padding, some experts are not on offer to some tokens; 16-bit logits
        dict(name="choice masked", op="choice", tokens=10007, experts=60, k=4, type="fp16", score="softmax", biased=True, groups=6,
             limit=3, best=1, renormalise=False, scale=1.0, masked=True),
        # the gates' gradient of that batch, and the biases' step
        dict(name="choice gradient", op="choice_grad", tokens=65536, experts=256, k=8, type="fp32", score="sigmoid", biased=True, groups=8,
             limit=4, best=2, renormalise=True, scale=2.5, masked=False),
        # two small layers' tensors: latency only; the gradient's norm is clipped
        dict(name="adam small set", op="adam", width=64, layers=2, type="fp32", grad="fp32", copy="", bits=32, clip=True),
        # a layer of 0.2 billion weights: fp32 masters, bf16 gradients and bf16 copies for the forward pass
        dict(name="adam layer", op="adam", width=4096, layers=1, type="fp32", grad="bf16", copy="bf16", bits=32, clip=False),
        # odd sizes, bf16 weights, states in 8 bits, clipped
        dict(name="adam 8 bits", op="adam", width=2047, layers=2, type="bf16", grad="bf16", copy="", bits=8, clip=True),
        # one token through a wide layer: the weight's bytes
        dict(name="linear one row", op="linear", rows=1, inner=4096, outer=16384, type="bf16", activation="gelu", bias=True, residual=False,
             keep=False),
        # a micro-batch through a wide layer; what the activation took is kept for the backward pass
        dict(name="linear batch", op="linear", rows=8192, inner=4096, outer=16384, type="bf16", activation="gelu_tanh", bias=True,
             residual=False, keep=True),
        # odd sizes in fp32, with a residual
        dict(name="linear odd", op="linear", rows=1531, inner=1000, outer=777, type="fp32", activation="silu", bias=True, residual=True,
             keep=False),
        # the backward pass of a square layer: input, weight and bias
        dict(name="linear gradient", op="linear_grad", rows=8192, inner=4096, outer=4096, type="bf16", activation="gelu_tanh", bias=True,
             residual=False, keep=True),
        # the same of a layer without activation, odd sizes in fp16
        dict(name="linear gradient odd", op="linear_grad", rows=2001, inner=1023, outer=515, type="fp16", activation="", bias=True,
             residual=False, keep=False),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["choice", "choice_grad", "adam", "linear", "linear_grad"])
    kind = rng.choice(["fp32", "bf16", "fp16"])
    if op in ("choice", "choice_grad"):
        groups = rng.choice([1, 1, 2, 4, 6, 8, 16])
        experts = groups * _spread(rng, 4, 512 // groups)
        limit = rng.randint(1, groups)
        tokens = _spread(rng, 1, min(131072, (1 << 24) // experts))
        return dict(op=op, tokens=tokens, experts=experts, k=rng.randint(1, min(8, experts // groups * limit)), type=kind,
                    score=rng.choice(["softmax", "sigmoid"]), biased=rng.choice([False, True]), groups=groups, limit=limit,
                    best=rng.choice([1, 2]), renormalise=rng.choice([False, True]), scale=rng.choice([1.0, 2.5]),
                    masked=rng.choice([False, True]))
    if op == "adam":
        layers = rng.randint(1, 4)
        width = _spread(rng, 16, min(4096, int(math.sqrt((1 << 27) / (12 * layers)))))
        return dict(op=op, width=width, layers=layers, type=kind, grad=rng.choice([kind, "fp32", "bf16"]),
                    copy=rng.choice(["", "bf16", "fp16"]) if kind == "fp32" else "", bits=rng.choice([32, 8]),
                    clip=rng.choice([False, True]))
    rows = _spread(rng, 1, 16384)
    inner = _spread(rng, 16, 8192)
    most = (1 << 39) // (8 if kind == "fp32" else 2 if op == "linear_grad" else 1)
    outer = _spread(rng, 16, max(16, min(16384, most // (rows * inner))))
    return dict(op=op, rows=rows, inner=inner, outer=outer, type=kind, activation=rng.choice(["", "relu", "gelu", "gelu_tanh", "silu"]),
                bias=rng.choice([False, True]), residual=op == "linear" and rng.choice([False, True]),
                keep=op == "linear" and rng.choice([False, True]))


def _shapes(case):
    """The tensors of `layers` layers: four square matrices, two between the width and four times it, four vectors."""
    w = case["width"]
    return ([(w, w)] * 4 + [(4 * w, w), (w, 4 * w)] + [(w,)] * 4) * case["layers"]


def work(case):
    s = BYTES[case["type"]]
    if case["op"] == "choice":               # logits, bias; experts and gates, counts
        t, e, k = case["tokens"], case["experts"], case["k"]
        return {"bytes": t * e * s + 8 * t * k + 12 * e + (t if case["masked"] else 0), "flops": 6 * t * e}
    if case["op"] == "choice_grad":          # what is zero does not go by its logit, but a softmax needs them all
        t, e, k = case["tokens"], case["experts"], case["k"]
        read = t * e if case["score"] == "softmax" and not case["renormalise"] else t * k
        return {"bytes": (read + t * e) * s + 8 * t * k + 16 * e, "flops": 8 * read}
    if case["op"] == "adam":                 # weight, gradient, two states, the weight's copy, the states' values where they are held in 8 bits
        n = sum(math.prod(d) for d in _shapes(case))
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 8
        return {"bytes": n * (2 * s + BYTES[case["grad"]] + state + BYTES.get(case["copy"], 0)), "flops": 16 * n}
    m, k, n = case["rows"], case["inner"], case["outer"]
    if case["op"] == "linear":
        out = 1 + case["keep"] + case["residual"]
        return {"bytes": s * (m * k + n * k + out * m * n + (n if case["bias"] else 0)), "flops": 2 * m * n * k}
    return {"bytes": s * (2 * m * k + 2 * n * k + (2 if case["activation"] else 1) * m * n + (n if case["bias"] else 0)), "flops": 4 * m * n * k}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    kind = TYPES[case["type"]]
    if case["op"] in ("choice", "choice_grad"):
        t, e, k = case["tokens"], case["experts"], case["k"]
        logits = 1.5 * normal(t, e) + 0.7 * normal(e)          # some experts are liked better than others
        keep = None
        if case["masked"]:
            keep = uniform(t) >= 0.1
            logits = torch.where(uniform(t, e) < 0.05, -math.inf, logits)
        # biases of some hundred steps, in the size of the scores
        size = 0.1 if case["score"] == "sigmoid" else 1.0 / e
        s = {"logits": logits.to(kind), "keep": keep, "bias": size * normal(e) if case["biased"] else None}
        if case["op"] == "choice_grad":
            r = _choose(case, s)
            s |= {"expert": r["expert"], "counts": r["counts"], "dgate": 0.1 * normal(t, k)}
            if s["bias"] is None:
                s["bias"] = torch.zeros(e, device="cuda")
        return {"case": case, **s}
    if case["op"] == "adam":
        # tensors lie one after the other in long buffers, each from a whole block on; zeros in between
        at, places = 0, []
        for shape in _shapes(case):
            places.append((at, shape))
            at += -(-math.prod(shape) // BLOCK) * BLOCK
        inside = torch.zeros(at, device="cuda")
        for begin, shape in places:
            inside[begin:begin + math.prod(shape)] = 1.0

        def block_sizes():                   # blocks' gradients differ by orders of magnitude
            return torch.exp(normal(at // BLOCK)).repeat_interleave(BLOCK)

        sizes = 1e-3 * block_sizes()
        s = {"param": (0.02 * normal(at) * inside).to(kind), "grad": (sizes * normal(at) * inside).to(TYPES[case["grad"]])}
        mean = 0.3 * sizes * normal(at) * inside
        square = (sizes * (0.2 + 0.5 * normal(at).abs())).square() * inside
        s["copy"] = s["param"].to(TYPES[case["copy"]]) if case["copy"] else None
        if case["bits"] == 8:
            s["mean"], s["mean_scale"] = _to_8_bits(mean, False)
            s["square"], s["square_scale"] = _to_8_bits(square, True)
        else:
            s |= {"mean": mean, "square": square, "mean_scale": None, "square_scale": None}
        s["step"] = torch.full((), 100, dtype=torch.int64, device="cuda")

        def parts(name):                     # the tensors themselves
            if s[name] is None:
                return None
            if name.endswith("scale"):
                return [s[name][b // BLOCK:b // BLOCK + -(-math.prod(d) // BLOCK)] for b, d in places]
            return [s[name][b:b + math.prod(d)].view(d) for b, d in places]

        names = ("param", "grad", "mean", "square", "mean_scale", "square_scale", "copy")
        return {"case": case, **s, "tensors": {name: parts(name) for name in names}}
    m, k, n = case["rows"], case["inner"], case["outer"]
    # a normed residual stream: a few columns that stand out; weights of a trained size
    x = normal(m, k) * torch.where(uniform(k) < 0.01, 4.0, 1.0)
    s = {"x": x.to(kind), "weight": (normal(n, k) / math.sqrt(k)).to(kind), "bias": (0.1 * normal(n)).to(kind) if case["bias"] else None}
    if case["op"] == "linear":
        s["residual"] = normal(m, n).to(kind) if case["residual"] else None
    else:
        s["dy"] = (0.05 * normal(m, n)).to(kind)
        s["z"] = (s["x"].float() @ s["weight"].float().t()).to(kind) if case["activation"] else None
    return {"case": case, **s}


def _to_8_bits(x, square):
    """Values as whole numbers of 8 bits and a scale, the largest value, for each block: a mean q stands for scale (q / 127) |q / 127|, a
    square for scale (q / 255)^4, of which only zeros are 0."""
    x = x.view(-1, BLOCK)
    scale = x.abs().amax(1, keepdim=True)
    scale = torch.where(scale < LEAST, 0.0, scale)
    part = x.abs() * (1.0 / torch.where(scale == 0.0, math.inf, scale))
    if square:
        q = torch.round(255.0 * torch.sqrt(torch.sqrt(part)))
        q = torch.where((x > 0.0) & (scale > 0.0), q.clamp(min=1.0), q).to(torch.uint8)
    else:
        q = (torch.sign(x) * torch.round(127.0 * torch.sqrt(part))).to(torch.int8)
    return q.view(-1), scale.view(-1)


def _from_8_bits(q, scale, square):
    q, scale = q.view(-1, BLOCK).float(), scale[:, None]
    if square:
        q = q * q
        return ((q * (scale / 65025.0)) * (q * (1.0 / 65025.0))).view(-1)
    return ((q * q.abs()) * (scale / 16129.0)).view(-1)


def _choose(case, s):
    """The k best experts by score + bias among those of the best groups (ties: the lowest index), their gates, and counts."""
    e, groups, k = case["experts"], case["groups"], case["k"]
    z = s["logits"].double()                                   # scores that differ by less than 32 bits tell decide choices
    on = (z != -math.inf).any(1)
    if s["keep"] is not None:
        on = on & s["keep"]
    if case["score"] == "softmax":
        w = torch.where(on[:, None], z, 0.0)
        w = (w - w.amax(1, keepdim=True)).exp()
        score = w / w.sum(1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-z))
    v = score if s["bias"] is None else score + s["bias"].double()
    v = torch.where(on[:, None] & (z != -math.inf), v, -math.inf)
    if groups > 1:
        top = torch.sort(v.view(-1, groups, e // groups), dim=2, descending=True).values[:, :, :case["best"]]
        value = torch.where(top[:, :, 0] == -math.inf, -math.inf, torch.where(top == -math.inf, 0.0, top).sum(2))
        chosen = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :case["limit"]]
        open_ = torch.zeros_like(value, dtype=torch.bool).scatter_(1, chosen, True)
        v = torch.where(open_.repeat_interleave(e // groups, 1), v, -math.inf)
    best = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :k]
    valid = v.gather(1, best) != -math.inf
    gate = torch.where(valid, score.gather(1, best), 0.0)
    if case["renormalise"]:
        total = gate.sum(1, keepdim=True)
        gate = gate / torch.where(total == 0.0, 1.0, total)
    counts = torch.zeros(e + 1, dtype=torch.int64, device=z.device)
    counts = counts.index_add_(0, torch.where(valid, best, e).reshape(-1), valid.reshape(-1).long())[:e]
    return {"expert": torch.where(valid, best, -1).to(torch.int32), "gate": (gate * case["scale"]).float(), "counts": counts,
            "tokens": on.sum()}


def _activate(z, name):
    if name == "relu":
        return torch.where(z < 0.0, 0.0, z)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, name):
    if name == "relu":
        return torch.where(z > 0.0, 1.0, 0.0)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 0.134145 * z * z)
    p = 1.0 / (1.0 + torch.exp(-z))
    return p * (1.0 + z * (1.0 - p))


def run(s):
    return (_run_own if own else _run_plain)(s["case"]["op"], s["case"], s)


def _run_own(op, case, s):
    from paper_2110_10548_amd import train
    if op == "choice":
        return train.p2_route_forward(s["logits"], case["k"], score=case["score"], bias=s["bias"], keep=s["keep"], groups=case["groups"],
                                      group_limit=case["limit"], group_best=case["best"], renormalise=case["renormalise"],
                                      scale=case["scale"])
    if op == "choice_grad":
        dlogits = train.p2_route_backward(s["logits"], s["expert"], s["dgate"], score=case["score"], renormalise=case["renormalise"],
                                          scale=case["scale"])
        return {"dlogits": dlogits, "bias": train.p2_route_bias(s["bias"], s["counts"], BIAS_RATE)}
    if op == "adam":
        t = s["tensors"]
        total = train.p2_square_sum(t["grad"]) if case["clip"] else None
        train.p2_adamw(t["param"], t["grad"], t["mean"], t["square"], s["step"], mean_scales=t["mean_scale"], square_scales=t["square_scale"],
                       copies=t["copy"], lr=LR, betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY, square_sum=total, max_norm=1.0 if case["clip"] else None)
        mean, square = s["mean"], s["square"]
        if case["bits"] == 8:
            (mean,), (square,) = train.p2_adamw_values([mean], [square], [s["mean_scale"]], [s["square_scale"]])
        out = {"param": s["param"], "mean": mean, "square": square}
        return out | ({"copy": s["copy"]} if case["copy"] else {}) | ({"total": total} if case["clip"] else {})
    activation = case["activation"] or None
    if op == "linear":
        y, z = train.p2_linear_forward(s["x"], s["weight"], s["bias"], activation=activation, residual=s["residual"], keep=case["keep"])
        return {"y": y, "z": z} if case["keep"] else {"y": y}
    dx, dweight, dbias = train.p2_linear_backward(s["dy"], s["x"], s["weight"], s["z"], activation=activation, dbias=case["bias"])
    return {"dx": dx, "dweight": dweight} | ({"dbias": dbias} if case["bias"] else {})


def _run_plain(op, case, s):
    if op == "choice":
        return _choose(case, s)
    if op == "choice_grad":
        expert, z, scale = s["expert"].long(), s["logits"].float(), case["scale"]
        valid = expert >= 0
        at = expert.clamp(min=0)
        d = torch.where(valid, s["dgate"], 0.0) * scale
        if case["score"] == "softmax" and not case["renormalise"]:
            on = valid.any(1, keepdim=True)
            z = torch.where(on, z, 0.0)
            p = (z - z.amax(1, keepdim=True)).exp()
            p = p / p.sum(1, keepdim=True)
            u = torch.zeros_like(p).scatter_add_(1, at, d)
            dz = torch.where(on, p * (u - (p * u).sum(1, keepdim=True)), 0.0)
        else:
            chosen = torch.where(valid, z.gather(1, at), -math.inf)
            slope = torch.ones_like(chosen)
            if case["score"] == "sigmoid":
                w = 1.0 / (1.0 + torch.exp(-chosen))
                slope = 1.0 - w
            else:
                w = (chosen - torch.where(valid.any(1, keepdim=True), chosen, 0.0).amax(1, keepdim=True)).exp()
            if case["renormalise"]:
                total = w.sum(1, keepdim=True)
                w = w / torch.where(total == 0.0, 1.0, total)
                d = d - (d * w).sum(1, keepdim=True)
            dz = torch.zeros_like(z).scatter_add_(1, at, torch.where(valid, w * slope * d, 0.0))
        counts = s["counts"]
        bias = s["bias"] + BIAS_RATE * torch.sign(counts.sum() - case["experts"] * counts).float()
        return {"dlogits": dz.to(s["logits"].dtype), "bias": bias}
    if op == "adam":
        return _adam_plain(case, s)
    if op == "linear":
        z = s["x"].float() @ s["weight"].float().t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _activate(z, case["activation"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        kind = s["x"].dtype
        return {"y": y.to(kind), "z": z.to(kind)} if case["keep"] else {"y": y.to(kind)}
    dz = s["dy"].float()
    if case["activation"]:
        dz = dz * _slope(s["z"].float(), case["activation"])
    kind = s["x"].dtype
    out = {"dx": (dz @ s["weight"].float()).to(kind), "dweight": (dz.t() @ s["x"].float()).to(kind)}
    return out | ({"dbias": dz.sum(0).to(kind)} if case["bias"] else {})


def _adam_plain(case, s):
    (b1, b2), out, factor = BETAS, {}, 1.0
    g = s["grad"].float()
    if case["clip"]:
        out["total"] = g.double().square().sum()               # a long sum: in 64 bits
        factor = (1.0 / out["total"].sqrt()).clamp(max=1.0).float()
    g = g * factor
    s["step"].add_(1)
    t = s["step"].double()
    rate, root = (LR / (1.0 - b1 ** t)).float(), (1.0 / (1.0 - b2 ** t).sqrt()).float()
    mean, square = s["mean"], s["square"]
    if case["bits"] == 8:
        mean, square = _from_8_bits(mean, s["mean_scale"], False), _from_8_bits(square, s["square_scale"], True)
    mean = b1 * mean + (1.0 - b1) * g
    square = b2 * square + (1.0 - b2) * (g * g)
    p = s["param"].float() * (1.0 - LR * DECAY) - rate * (mean / (square.sqrt() * root + ADAM_EPS))
    s["param"].copy_(p)
    if case["bits"] == 8:
        for name, values in (("mean", mean), ("square", square)):
            q, scale = _to_8_bits(values, name == "square")
            s[name].copy_(q)
            s[name + "_scale"].copy_(scale)
            out[name] = _from_8_bits(q, scale, name == "square")
    else:
        out |= {"mean": s["mean"].copy_(mean), "square": s["square"].copy_(square)}
    if case["copy"]:
        out["copy"] = s["copy"].copy_(p)
    return out | {"param": s["param"]}


def exact(case, seed):
    """What `run` returns, in 64 bits: choices by ranks, gradients by torch's derivatives, AdamW from its states' values."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "choice":
        z = s["logits"].double()
        r = _choose(case, s)
        valid = r["expert"] >= 0
        chosen = torch.where(valid, z.gather(1, r["expert"].clamp(min=0).long()), -math.inf)
        if case["score"] == "softmax":
            log = chosen - torch.where(valid.any(1, keepdim=True), z, 0.0).logsumexp(1, keepdim=True)
        else:
            log = torch.nn.functional.logsigmoid(chosen)
        if case["renormalise"]:
            log = log - torch.where(valid.any(1, keepdim=True), log, 0.0).logsumexp(1, keepdim=True)
        return {"expert": None, "gate": log.exp() * case["scale"], "counts": None, "tokens": None}
    if op == "choice_grad":
        z = s["logits"].double().requires_grad_(True)
        rows = (s["expert"] >= 0).any(1).nonzero()[:, 0]
        expert = s["expert"][rows].long()
        valid = expert >= 0
        score = torch.softmax(z[rows], 1) if case["score"] == "softmax" else torch.sigmoid(z[rows])
        gate = torch.where(valid, score.gather(1, expert.clamp(min=0)), 0.0)
        if case["renormalise"]:
            gate = gate / gate.sum(1, keepdim=True)
        dlogits = torch.autograd.grad((gate * case["scale"] * s["dgate"][rows].double()).sum(), z)[0]
        counts = s["counts"].double()
        return {"dlogits": dlogits, "bias": s["bias"].double() + BIAS_RATE * torch.sign(counts.mean() - counts)}
    if op == "adam":
        g = s["grad"].double()
        out = {}
        if case["clip"]:
            out["total"] = torch.dot(g, g)
            g = g * min(1.0, 1.0 / math.sqrt(float(out["total"])))
        t = int(s["step"]) + 1
        if case["bits"] == 8:
            shape = (-1, BLOCK)
            q = s["mean"].double().view(shape) / 127.0
            mean = (q * q.abs() * s["mean_scale"].double()[:, None]).view(-1)
            square = ((s["square"].double().view(shape) / 255.0).pow(4) * s["square_scale"].double()[:, None]).view(-1)
        else:
            mean, square = s["mean"].double(), s["square"].double()
        mean = torch.lerp(mean, g, 1.0 - BETAS[0])
        square = torch.lerp(square, g.square(), 1.0 - BETAS[1])
        step = (mean / (1.0 - BETAS[0] ** t)) / ((square / (1.0 - BETAS[1] ** t)).sqrt() + ADAM_EPS)
        p = s["param"].double()
        p = p - LR * DECAY * p - LR * step
        if case["bits"] == 8:                # next to a border 32 bits may give the neighbouring 8-bit value: no states
            mean = square = None
        out |= {"param": p, "mean": mean, "square": square}
        return out | ({"copy": p} if case["copy"] else {})
    weight = s["weight"].double()
    functions = {"relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu, "": lambda z: z,
                 "gelu_tanh": lambda z: torch.nn.functional.gelu(z, approximate="tanh")}
    activate = functions[case["activation"]]
    if op == "linear":
        z = torch.addmm(s["bias"].double(), s["x"].double(), weight.T) if case["bias"] else s["x"].double().mm(weight.T)
        y = activate(z)
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return {"y": y, "z": z} if case["keep"] else {"y": y}
    dz = s["dy"].double()
    if case["activation"]:
        z = s["z"].double().requires_grad_(True)
        dz = torch.autograd.grad(activate(z), z, dz)[0]
    out = {"dx": dz.mm(weight), "dweight": dz.T.mm(s["x"].double())}
    return out | ({"dbias": dz.sum(0)} if case["bias"] else {})
