"""A data-parallel training step whose reductions are planned, on one GPU.

Eight devices (2 nodes of 4) hold a layer norm, a router over experts and a weight, and a share of a batch each.  Per step:

  1. layer norm and routing of the device's own tokens; what they sum up over them are the messages;
  2. the routing statistics are summed over the devices, by the cheapest program for so few bytes;
  3. with the whole batch's statistics the backward pass; its gradients are summed by the cheapest program for their size;
  4. the weight's update: the reduced gradient orthogonalised.

The planner (p2_search_placements) chooses the programs and predicts their times on the system described; here all eight devices'
parts run one after the other on the one GPU, and the programs' instructions are carried out on their messages in its memory.
The result is compared with a single device that sees the whole batch.

    python examples/planned_step.py [--tokens 16384] [--width 1024] [--experts 64] [--chosen 4]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2110_10548_amd import binding as p2, train  # noqa: E402

CARD, BANDWIDTH, LATENCY = [2, 4], [25e9, 300e9], [20e-6, 5e-6]        # 2 nodes of 4 devices, outermost level first
AXES, REDUCE = [8], [0]                                                # data parallelism over all of them


class Program:
    """The cheapest program for a sum of `nbytes` bytes over the data axis, and its instructions' device groups."""

    def __init__(self, nbytes):
        best = p2.p2_search_placements(CARD, AXES, [REDUCE], 4, float(nbytes), bw=BANDWIDTH, alpha=LATENCY)
        placement = best["order"][0]
        row = best["rows"][(placement, 0)]
        self.seconds, self.allreduce_seconds = row["best_cost"], row["allreduce_cost"]
        self.steps = []
        for code in row["best_instr"]:
            d = p2.p2_describe_pattern(CARD, AXES, best["placements"][placement], REDUCE, code // 5)
            groups = {}
            for device, (group, rank) in enumerate(zip(d["group_of"], d["rank"])):
                if group >= 0:
                    groups.setdefault(int(group), {})[int(rank)] = device
            members = [[g[r] for r in range(len(g))] for g in groups.values()]
            self.steps.append((p2.OPS[code % 5], p2.FORMS[d["form"]], members))

    def __str__(self):
        names = " ; ".join("%s in %d groups of %d" % (op, len(groups), len(groups[0])) for op, _, groups in self.steps)
        return "%s  (%.1f us; one AllReduce %.1f us)" % (names, self.seconds * 1e6, self.allreduce_seconds * 1e6)

    def run(self, messages):
        """The sum of the devices' messages, as every device has it in the end."""
        devices, n = len(messages), messages[0].numel()
        size = -(-n // devices)
        state = [list(torch.cat([m, m.new_zeros(size * devices - n)]).view(devices, size)) for m in messages]   # a device's chunks
        for op, _, groups in self.steps:
            for members in groups:
                held = [c for c in range(devices) if state[members[0]][c] is not None]
                if op in ("AllReduce", "ReduceScatter", "Reduce"):
                    total = {c: sum(state[d][c] for d in members[1:]) + state[members[0]][c] for c in held}
                    share = len(held) // len(members)
                    for rank, d in enumerate(members):
                        keep = held if op == "AllReduce" else held[rank * share:(rank + 1) * share] if op == "ReduceScatter" else held if rank == 0 else []
                        state[d] = [total[c] if c in keep else None for c in range(devices)]
                elif op == "AllGather":
                    union = [next((state[d][c] for d in members if state[d][c] is not None), None) for c in range(devices)]
                    for d in members:
                        state[d] = list(union)
                else:
                    for d in members:
                        state[d] = list(state[members[0]])
        out = [torch.cat(s)[:n] for s in state]
        assert all(torch.equal(out[0], o) for o in out[1:]), "the devices disagree"
        return out[0]


class Layer:
    """Layer norm -> router and weight.  The loss is the balance loss, and the sums of the gates and of the weight's results times
    given gradients."""

    def __init__(self, width, experts, chosen):
        self.chosen = chosen
        self.weight, self.bias = torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        self.router = torch.randn(width, experts, device="cuda") / width ** 0.5
        self.matrix = torch.randn(width, width, device="cuda") / width ** 0.5

    def forward(self, x):
        y, mean, rstd = train.p2_layer_norm_forward(x, self.weight, self.bias)
        route = train.p2_balance_forward(y @ self.router, self.chosen)
        return y, mean, rstd, route

    def statistics(self, route):
        return torch.cat([route["counts"].double(), route["prob_sum"].double(), route["tokens"].double()[None]])

    def backward(self, x, dout, dgate, kept, statistics):
        y, mean, rstd, route = kept
        e = self.router.shape[1]
        counts, tokens = statistics[:e].long(), statistics[2 * e].long()
        dlogits = train.p2_balance_backward(y @ self.router, route["expert"], counts, tokens, dgate=dgate)
        dmatrix, drouter = y.t() @ dout, y.t() @ dlogits
        dy = dout @ self.matrix.t() + dlogits @ self.router.t()
        _, dweight, dbias = train.p2_layer_norm_backward(dy, x, self.weight, mean, rstd)
        return torch.cat([g.reshape(-1) for g in (dweight, dbias, drouter, dmatrix)])

    def update(self, gradients, rate=0.02):
        """The weight after an orthogonalised step, of the length that Muon gives it."""
        rows, cols = self.matrix.shape
        dmatrix = gradients[-rows * cols:].view(rows, cols)
        return self.matrix - rate * train.p2_orthogonalize(dmatrix, scale=max(1.0, rows / cols) ** 0.5)


def main(tokens=16384, width=1024, experts=64, chosen=4, say=print):
    torch.manual_seed(0)
    devices = CARD[0] * CARD[1]
    layer = Layer(width, experts, chosen)
    x = torch.randn(tokens, width, device="cuda") * torch.exp(0.5 * torch.randn(tokens, 1, device="cuda"))
    dout, dgate = torch.randn(tokens, width, device="cuda") / tokens, torch.randn(tokens, chosen, device="cuda") / tokens
    shares = torch.arange(tokens, device="cuda").tensor_split(devices)      # (as many for every device, or one more; few tokens: none for some)

    small = Program((2 * experts + 1) * 8)
    large = Program((2 * width + width * experts + width * width) * 4)
    say("statistics:", small)
    say("gradients: ", large)

    kept = [layer.forward(x[s]) for s in shares]
    statistics = small.run([layer.statistics(k[3]) for k in kept])
    loss = train.p2_balance_loss(statistics[:experts].long(), statistics[experts:2 * experts].float(), statistics[2 * experts].long(), chosen)
    gradients = large.run([layer.backward(x[s], dout[s], dgate[s], k, statistics) for s, k in zip(shares, kept)])
    matrix = layer.update(gradients)

    one = layer.forward(x)                                  # a single device with the whole batch
    whole = layer.backward(x, dout, dgate, one, layer.statistics(one[3]))
    off = [float((a - b).norm() / b.norm()) for a, b in ((gradients, whole), (matrix - layer.matrix, layer.update(whole) - layer.matrix))]
    say("balance loss %.6f (whole batch at once: %.6f)" % (float(loss), float(one[3]["loss"])))
    say("off a single device: gradients %.1e, update %.1e" % tuple(off))
    return float(loss), float(one[3]["loss"]), off, small, large


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    for name, value in (("tokens", 16384), ("width", 1024), ("experts", 64), ("chosen", 4)):
        parser.add_argument("--" + name, type=int, default=value)
    main(**vars(parser.parse_args()))
