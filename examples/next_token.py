"""A small language model trained on the next token with the framework's operators, on one GPU:

    python examples/next_token.py [--steps N] [--width D]

Its MLP blocks keep their activations in 8 bits (``train_ops.linear8``, ``train_ops.act8``), the loss at the head never keeps
its logits (``train_ops.linear_cross_entropy``), the blocks' matrices step along their orthogonalised momentum
(``optim.OrthogonalMomentum``), embeddings and head by the sign vote (``optim.SignumVote``), whose flat buffer the head's gradient is added to straight.
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1810_05291_b200 import train_ops as T  # noqa: E402
from paper_1810_05291_b200.optim import OrthogonalMomentum, SignumVote  # noqa: E402


class Model(torch.nn.Module):
    """The next token from this one and the one before it."""

    def __init__(self, vocab, width, hidden, blocks):
        super().__init__()
        new = lambda rows, cols, size: torch.nn.Parameter(torch.randn(rows, cols) * size)  # noqa: E731
        self.now, self.before = new(vocab, width, 0.5), new(vocab, width, 0.5)
        self.gates = torch.nn.ParameterList(new(hidden, width, width ** -0.5) for _ in range(blocks))
        self.ups = torch.nn.ParameterList(new(hidden, width, width ** -0.5) for _ in range(blocks))
        self.downs = torch.nn.ParameterList(new(width, hidden, hidden ** -0.5) for _ in range(blocks))
        self.head = new(vocab, width, width ** -0.5)

    def matrices(self):
        return [*self.gates, *self.ups, *self.downs]

    def forward(self, tokens, previous):
        x = (self.now[tokens] + self.before[previous]).bfloat16()
        for gate, up, down in zip(self.gates, self.ups, self.downs):
            h, kept = T.act8(T.linear8(x, gate), T.linear8(x, up), "silu", keep_output=torch.is_grad_enabled())
            x = x + T.linear8(h, down, kept)
        return x


def batch_of(vocab, rows, gen, device):
    """Sequences that count up or down by a fixed step, as far apart as their first two tokens."""
    start, step = (torch.randint(0, vocab, (rows, 1), generator=gen) for _ in range(2))
    tokens = (start + step * torch.arange(18)) % vocab
    previous, now, targets = tokens[:, :-2], tokens[:, 1:-1], tokens[:, 2:]
    weights = torch.full(targets.shape, 1.0 / targets.numel())
    return [t.reshape(-1).to(device) for t in (now, previous, targets, weights)]


def train(steps=100, width=128, hidden=256, vocab=97, blocks=2, rows=64, seed=0, device="cuda:0", say=print):
    torch.manual_seed(seed)
    gen = torch.Generator().manual_seed(seed)
    model = Model(vocab, width, hidden, blocks).to(device)
    signum = SignumVote([model.now, model.before, model.head], lr=1e-3, momentum=0.9)
    matrices = OrthogonalMomentum(model.matrices(), lr=3e-3)
    history = []
    for _ in range(steps):
        now, previous, targets, weights = batch_of(vocab, rows, gen, device)
        signum.zero_grad()
        matrices.zero_grad()
        loss, _, logp = T.linear_cross_entropy(model(now, previous), model.head, targets, weights, z_coef=1e-4, into_grad=True)
        loss.backward()
        signum.step()
        matrices.step()
        history.append(float(loss.detach()))
    say("loss %.4f -> %.4f, probability of the right token %.3f" % (history[0], history[-1], float(logp.exp().mean())))
    return model, history


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--width", type=int, default=128)
    a = ap.parse_args()
    train(steps=a.steps, width=a.width, hidden=2 * a.width)
