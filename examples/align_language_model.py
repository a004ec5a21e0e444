#!/usr/bin/env python3
"""Aligning a small language model with EF21: n workers, each with texts of its own, one Top-k message a round.

    python examples/align_language_model.py [--objective likelihood|preference|policy] [--rounds 60] [--workers 4] ...

The model is one tied table E [vocab][width], the x of EF21: the logits of the token behind token a are E (s E_a), s = sqrt(width).
A round is what a user's training loop does with the library:

    hidden  = s E[tokens]                        ef21_embed
    logits  = hidden E^T                         (a matrix product)
    loss, d loss / d logits                      ef21_token_logps and ef21_token_logps_grad, ef21_preference_loss or ef21_policy_loss
    G_i     = (d logits_i)^T hidden_i            (a matrix product per worker: the table as the output layer)
    G_i    += s sum_t d hidden_it at token_it    ef21_embed_grad, accumulating into the rows of grads [n][d]
    x, g_i, g                                    EF21.step(grads): Top-k of G_i - g_i, d = vocab * width

likelihood: the negative log-likelihood of given texts; preference: pairs of replies with a preferred one, against the model as it
was at the start; policy: tokens drawn from the model, rewarded where they are even, with the clipped ratio and a KL term.
Prints the mean loss and what the objective is after (text log-likelihood, share of pairs in the right order, reward).
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2106_05203_amd import binding as ef21  # noqa: E402


class TiedModel:
    """The gradients of n workers' losses for a tied table; every worker has the same number of rows (tokens)."""

    def __init__(self, n: int, vocab: int, width: int):
        self.n, self.vocab, self.width, self.scale = n, vocab, width, math.sqrt(width)
        self.grads = torch.empty(n, vocab * width, device="cuda")     # the rows that EF21.step takes

    def forward(self, x: torch.Tensor, tokens: torch.Tensor):
        """(hidden [n rows][width], logits [n rows][vocab]) of tokens [n][rows]."""
        table = x.view(self.vocab, self.width)
        hidden = ef21.ef21_embed(table, tokens.reshape(-1), self.scale)
        return hidden, torch.mm(hidden, table.t())

    def backward(self, x: torch.Tensor, tokens: torch.Tensor, hidden: torch.Tensor, dlogits: torch.Tensor) -> torch.Tensor:
        """The rows of gradients, from those of the logits."""
        table, rows = x.view(self.vocab, self.width), tokens.shape[1]
        tables = self.grads.view(self.n, self.vocab, self.width)
        for i in range(self.n):
            part = slice(i * rows, (i + 1) * rows)
            torch.mm(dlogits[part].t(), hidden[part], out=tables[i])
        dhidden = torch.mm(dlogits, table).view(self.n, rows, self.width)
        ef21.ef21_embed_grad(dhidden, tokens, self.vocab, self.scale, out=tables, accumulate=True)
        return self.grads


def likelihood(model: TiedModel, x, tokens, labels):
    """Worker i's loss: the mean of -log p over its rows.  Returns (losses [n], grads)."""
    hidden, logits = model.forward(x, tokens)
    logp, lse = ef21.ef21_token_logps(logits, labels.reshape(-1))
    weight = torch.full_like(logp, -1.0 / tokens.shape[1])
    dlogits = ef21.ef21_token_logps_grad(logits, labels.reshape(-1), lse, weight, out=logits)
    return -logp.view(model.n, -1).mean(1), model.backward(x, tokens, hidden, dlogits)


def preference(model: TiedModel, x, tokens, labels, seq_start, ref_logp, beta: float = 0.5):
    """Worker i's loss: the mean over its pairs.  seq_start [2 pairs + 1]: the replies of all workers' pairs among the rows of all workers, a
    pair's preferred one first; labels outside the vocabulary are prompts.  Returns (losses [n], logp [n rows], grads)."""
    hidden, logits = model.forward(x, tokens)
    pairs = (seq_start.numel() - 1) // 2
    weight = torch.full((pairs,), model.n / pairs, device="cuda")
    loss, logp, dlogits = ef21.ef21_preference_loss(logits, labels.reshape(-1), seq_start, ref_logp, beta, pair_weight=weight, grad=logits)
    return loss.view(model.n, -1).mean(1), logp, model.backward(x, tokens, hidden, dlogits)


def policy(model: TiedModel, x, tokens, labels, old_logp, advantages, ref_logp, clip: float = 0.2, kl: float = 0.04):
    """Worker i's loss: the mean over its rows.  Returns (losses [n], grads)."""
    hidden, logits = model.forward(x, tokens)
    weight = torch.full_like(old_logp, 1.0 / tokens.shape[1])
    _, token_loss, _, dlogits = ef21.ef21_policy_loss(logits, labels.reshape(-1), old_logp, advantages, clip, clip, ref_logp=ref_logp, kl=kl,
                                                      weight=weight, grad=logits)
    return token_loss.view(model.n, -1).mean(1), model.backward(x, tokens, hidden, dlogits)


def texts(g: torch.Generator, shape, vocab: int):
    """Pairs of a token and the one behind it: a + 1, or a + 2 for a third of them."""
    a = torch.randint(0, vocab, shape, generator=g, device="cuda")
    return a, (a + 1 + (torch.rand(shape, generator=g, device="cuda") < 1 / 3)) % vocab


def run(objective: str, rounds: int = 60, workers: int = 4, vocab: int = 512, width: int = 64, rows: int = 256, length: int = 8, share: float = 0.1,
        gamma: float = 2.0, seed: int = 0, report=None):
    """Trains; returns [(mean loss, what the objective is after)] of every round."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    d = vocab * width
    model = TiedModel(workers, vocab, width)
    x = torch.randn(d, generator=g, device="cuda") * 0.3 / math.sqrt(math.sqrt(width))
    start, history = x.clone(), []
    if objective == "preference":
        if rows % (2 * length):
            raise ValueError("a worker's rows must be whole pairs: rows a multiple of 2 length")
        tokens, right = texts(g, (workers, rows), vocab)
        wrong = torch.randint(0, vocab, (workers, rows), generator=g, device="cuda")
        # a pair's replies lie one behind the other: `length` rows with the tokens that follow in the texts, and as many with others
        first = (torch.arange(rows, device="cuda") // length % 2 == 0).expand(workers, rows)
        labels = torch.where(first, right, wrong)
        seq_start = torch.arange(0, workers * rows + 1, length, device="cuda")
        ref_logp, _ = ef21.ef21_token_logps(model.forward(start, tokens)[1], labels.reshape(-1))
    elif objective == "likelihood":
        tokens, labels = texts(g, (workers, rows), vocab)
    with ef21.EF21(workers, d, max(1, int(share * d)), gamma) as h:
        zeros = torch.zeros(workers, d, device="cuda")
        h.set_state(x, zeros, zeros[0])
        for t in range(rounds):
            if objective == "likelihood":
                losses, grads = likelihood(model, x, tokens, labels)
                aim = -losses.mean()
            elif objective == "preference":
                losses, logp, grads = preference(model, x, tokens, labels, seq_start, ref_logp)
                moved = (logp - ref_logp).view(-1, 2, length).sum(2)
                aim = (moved[:, 0] > moved[:, 1]).float().mean()
            else:
                tokens = torch.randint(0, vocab, (workers, rows), generator=g, device="cuda")
                logits = model.forward(x, tokens)[1]
                labels = torch.multinomial(torch.softmax(logits, 1), 1, generator=g).view(workers, rows)
                old_logp, _ = ef21.ef21_token_logps(logits, labels.reshape(-1))
                ref_logp, _ = ef21.ef21_token_logps(model.forward(start, tokens)[1], labels.reshape(-1))
                reward = (labels % 2 == 0).float()
                advantages = (reward - reward.mean(1, keepdim=True)).reshape(-1)
                losses, grads = policy(model, x, tokens, labels, old_logp, advantages, ref_logp)
                aim = reward.mean()
            h.step(grads)
            x = h.get_x()
            history.append((losses.mean(), aim))
            if report and (t % 10 == 0 or t + 1 == rounds):
                report(f"round {t:4d}  loss {float(losses.mean()):.4f}  {dict(likelihood='log-likelihood', preference='right order', policy='reward')[objective]} {float(aim):.4f}")
    return [(float(a), float(b)) for a, b in history]


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--objective", choices=["likelihood", "preference", "policy"], default="preference")
    for name, default in (("rounds", 60), ("workers", 4), ("vocab", 512), ("width", 64), ("rows", 256), ("length", 8), ("seed", 0)):
        p.add_argument(f"--{name}", type=int, default=default)
    p.add_argument("--share", type=float, default=0.1, help="share of the entries that a message carries")
    p.add_argument("--gamma", type=float, default=2.0, help="stepsize")
    run(report=lambda line: print(line, flush=True), **vars(p.parse_args()))


if __name__ == "__main__":
    main()
