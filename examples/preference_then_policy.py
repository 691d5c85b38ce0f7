"""A small language model trained with the framework's operators from end to end on one GPU:

    python examples/preference_then_policy.py [--steps N] [--width D]

Its MLP blocks keep their activations in 8 bits (``train_ops.linear8``, ``train_ops.act8``), the weight
gradients are added straight into the flat buffer of ``SignumVote``, and every step is one vote and
update of all parameters. First the model learns which of two answers is preferred (sequences of
different lengths, packed, prompts without weight) against the model it starts as, then it is improved
with a clipped policy loss on tokens that it samples, rewarded for a quarter of the vocabulary, with a
KL term towards the model that sampled.
"""

import argparse
import copy
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1810_05291_b200 import train_ops as T  # noqa: E402
from paper_1810_05291_b200.optim import SignumVote  # noqa: E402


class Block(torch.nn.Module):
    def __init__(self, width, hidden):
        super().__init__()
        new = lambda rows, cols: torch.nn.Parameter(torch.randn(rows, cols) * cols ** -0.5)  # noqa: E731
        self.gate, self.up, self.down = new(hidden, width), new(hidden, width), new(width, hidden)

    def forward(self, x):
        kept = None
        if torch.is_grad_enabled():  # one checkpoint for both projections
            kept = T.B.act8_checkpoint(x.shape[0], x.shape[1], x.device)
            T.B.ss_act8_pack(x.detach(), kept)
        gate, up = T.linear8(x, self.gate, kept, into_grad=True), T.linear8(x, self.up, kept, into_grad=True)
        h, kept_h = T.act8(gate, up, "silu", keep_output=torch.is_grad_enabled())
        return x + T.linear8(h, self.down, kept_h, into_grad=True)


class Model(torch.nn.Module):
    """The next token from this one and the one before it."""

    def __init__(self, vocab, width, hidden, blocks):
        super().__init__()
        self.now = torch.nn.Parameter(torch.randn(vocab, width) * 0.5)
        self.before = torch.nn.Parameter(torch.randn(vocab, width) * 0.5)
        self.blocks = torch.nn.ModuleList(Block(width, hidden) for _ in range(blocks))
        self.head = torch.nn.Parameter(torch.randn(vocab, width) * width ** -0.5)

    def forward(self, tokens, previous):
        x = (self.now[tokens] + self.before[previous]).bfloat16()
        for block in self.blocks:
            x = block(x)
        return T.linear8(x, self.head, into_grad=True)


def pairs_of(vocab, n, gen, device):
    """Answers that count upwards are preferred to ones that count downwards; prompts carry no weight."""
    tokens, weights, begin = [], [], [0]
    for _ in range(n):
        start = int(torch.randint(0, vocab, (1,), generator=gen))
        for step in (1, -1):
            length = int(torch.randint(6, 20, (1,), generator=gen))
            tokens.append((start + step * torch.arange(length)) % vocab)
            w = torch.ones(length)
            w[:2] = 0
            weights.append(w)
            begin.append(begin[-1] + length)
    flat = torch.cat(tokens).to(device)
    starts = torch.tensor(begin, device=device)
    previous = flat.roll(1)
    previous[starts[:-1]] = flat[starts[:-1]]
    targets = flat.roll(-1)
    weights = torch.cat(weights).to(device)
    weights[starts[1:] - 1] = 0  # nothing follows the last token of a sequence
    return flat, previous, targets, weights, starts


def train(steps=60, width=128, hidden=256, vocab=211, blocks=2, n_pairs=24, lr=1e-3, seed=0, device="cuda:0", say=print):
    torch.manual_seed(seed)
    gen = torch.Generator().manual_seed(seed)
    model = Model(vocab, width, hidden, blocks).to(device)
    first = copy.deepcopy(model).requires_grad_(False)
    optimizer = SignumVote(model.parameters(), lr=lr, momentum=0.9)
    history = {"preference": [], "reward": []}

    for step in range(steps):
        tokens, previous, targets, weights, starts = pairs_of(vocab, n_pairs, gen, device)
        with torch.no_grad():
            reference = T.preference_loss(first(tokens, previous), targets, weights, starts, torch.zeros(2 * n_pairs, device=device))[2]
        optimizer.zero_grad()
        loss, margins, _, _ = T.preference_loss(model(tokens, previous), targets, weights, starts, reference, beta=0.1)
        loss.backward()
        optimizer.step()
        history["preference"].append(float(loss.detach()))
    say("preference loss %.4f -> %.4f, margin > 0 for %d of %d pairs" % (
        history["preference"][0], history["preference"][-1], int((margins > 0).sum()), n_pairs))

    for step in range(steps):
        now = torch.randint(0, vocab, (512,), generator=gen).to(device)
        with torch.no_grad():
            logits = model(now, now)
            taken = torch.multinomial(torch.softmax(logits.float(), 1), 1)[:, 0]
        reward = (taken % 4 == 0).float()
        advantages = reward - reward.mean()
        old = torch.empty(512, device=device)
        T.B.ss_policy_loss(logits, taken, torch.zeros_like(old), None, advantages, torch.ones_like(old), torch.empty(3, device=device), old)
        weights = torch.full((512,), 1.0 / 512, device=device)
        for _ in range(2):  # two updates on the same answers: the second is held by the clip range
            optimizer.zero_grad()
            loss, _, _ = T.policy_loss(model(now, now), taken, old, advantages, weights, ref_logp=old, kl_coef=0.01)
            loss.backward()
            optimizer.step()
        history["reward"].append(float(reward.mean()))
    say("share of the rewarded tokens %.4f -> %.4f" % (history["reward"][0], history["reward"][-1]))
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--width", type=int, default=128)
    a = ap.parse_args()
    train(steps=a.steps, width=a.width, hidden=2 * a.width)
