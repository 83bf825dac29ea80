"""A network that proposes each lane's parameters and trains through the program's replay.

Every lane holds eight noisy readings of its own exponential decay a exp(-b t) + c.  A residual
network reads them and answers with (a, b, c); the program, replayed over all lanes, says how well
that fits, and its gradient goes back through ``loss_op`` into the network: no lane is ever fitted by
itself.  (The readings ride along as parameters of the program that take no gradient.)

    python examples/amortised_fit.py --lanes 4096 --steps 200
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_03574_gb300 as nd  # noqa: E402

TIMES = [0.1, 0.3, 0.6, 1.0, 1.5, 2.2, 3.0, 4.0]
NOISE = 0.02


def program():
    """Mean squared residual of the eight readings, which are the last eight parameters."""
    names = " ".join(f"y{i}" for i in range(len(TIMES)))
    terms = " ".join(f"(let ((r (- (+ (* a (exp (- (* b {t})))) c) y{i}))) (* r r))" for i, t in enumerate(TIMES))
    return f"(model (params a b c {names}) (/ (+ {terms}) {float(len(TIMES))}))"


def readings(lanes, generator):
    """(readings, the parameters behind them)."""
    low, span = torch.tensor([0.5, 0.3, 0.0], device="cuda"), torch.tensor([1.5, 1.5, 0.5], device="cuda")
    truth = low + span * torch.rand(lanes, 3, generator=generator, device="cuda")
    a, b, c = truth[:, :1], truth[:, 1:2], truth[:, 2:]
    y = a * torch.exp(-b * torch.tensor(TIMES, device="cuda")) + c
    return y + NOISE * torch.randn(y.shape, generator=generator, device="cuda"), truth


class Block(torch.nn.Module):
    """x + dropout(down(gated(layer_norm(x)))): binary32 master weights, products in bfloat16."""

    def __init__(self, width, hidden, p):
        super().__init__()
        self.p = p
        self.scale, self.shift = torch.nn.Parameter(torch.ones(width)), torch.nn.Parameter(torch.zeros(width))
        self.gate, self.up = (torch.nn.Parameter(torch.randn(hidden, width) * width ** -0.5) for _ in range(2))
        self.down = torch.nn.Parameter(torch.randn(width, hidden) * hidden ** -0.5 * 0.5)

    def forward(self, x, seed, offset):
        h = nd.layer_norm(x, self.scale, self.shift)
        h = nd.gated(h, self.gate.bfloat16(), self.up.bfloat16(), "silu") @ self.down.bfloat16().t()
        return nd.dropout(h, self.p if self.training else 0.0, seed, offset, residual=x)


class Proposer(torch.nn.Module):
    def __init__(self, width=256, hidden=512, blocks=2, p=0.02):
        super().__init__()
        self.embed = torch.nn.Linear(len(TIMES), width)
        self.blocks = torch.nn.ModuleList(Block(width, hidden, p) for _ in range(blocks))
        self.scale, self.shift = torch.nn.Parameter(torch.ones(width)), torch.nn.Parameter(torch.zeros(width))
        self.head = torch.nn.Linear(width, 3)

    def forward(self, y, step=0):
        x = self.embed(y).bfloat16()
        for i, block in enumerate(self.blocks):  # each block of a step draws from its own range
            x = block(x, seed=step, offset=(i * x.numel() + 3) // 4 * 4)
        return torch.nn.functional.softplus(self.head(nd.layer_norm(x, self.scale, self.shift).float()))


def train(lanes=4096, steps=200, lr=2e-3, seed=0, say=print):
    """(mean loss of unseen lanes before, after, and at their true parameters)."""
    torch.manual_seed(seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    tape = nd.trace_build(program())
    replay = nd.loss_op(tape)
    net = Proposer().cuda()
    opt = torch.optim.Adam(net.parameters(), lr=lr)
    unseen, truth = readings(lanes, g)

    def score(params):
        with torch.no_grad():
            return float(replay(torch.cat((params.double(), unseen.double()), 1), None).mean())

    def evaluate():
        net.eval()
        with torch.no_grad():
            loss = score(net(unseen))
        net.train()
        return loss

    before = evaluate()
    for step in range(steps):
        y, _ = readings(lanes, g)
        loss = replay(torch.cat((net(y, step + 1).double(), y.double()), 1), None).mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        if step % 50 == 0:
            say(f"step {step:4d}: mean loss {float(loss.detach()):.5f}")
    nd.check_device(tape)
    nd.check_operators()
    return before, evaluate(), score(truth)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--lanes", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=200)
    args = ap.parse_args()
    before, after, floor = train(args.lanes, args.steps)
    print(f"mean loss of unseen lanes: {before:.5f} before, {after:.5f} after; {floor:.5f} at their true parameters")
