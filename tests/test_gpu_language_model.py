"""The example of a language model whose table is EF21's x: its gradients against automatic differentiation in 64 bits and
against differences, and that training reaches what each objective is after."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lm():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import align_language_model
    return align_language_model


N, VOCAB, WIDTH, ROWS, LENGTH, BETA, CLIP, KL = 3, 211, 24, 48, 8, 0.5, 0.2, 0.04


def case(torch, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(VOCAB * WIDTH, generator=g) * 0.15
    tokens = torch.randint(0, VOCAB, (N, ROWS), generator=g)
    tokens[:, ::5] = 7                                                 # a frequent token
    labels = torch.randint(0, VOCAB, (N, ROWS), generator=g)
    return x, tokens, labels, torch.randn(N * ROWS, generator=g)


def losses64(torch, objective, x, tokens, labels, ref, noise):
    """losses [n] of the objectives from their definitions, in 64 bits on the CPU."""
    table = x.view(VOCAB, WIDTH)
    logits = (math.sqrt(WIDTH) * table[tokens.reshape(-1)]) @ table.t()
    logp = torch.log_softmax(logits, 1).gather(1, labels.reshape(-1, 1))[:, 0]
    if objective == "likelihood":
        return -logp.view(N, -1).mean(1)
    if objective == "preference":
        moved = (logp - ref).view(N, -1, 2, LENGTH).sum(3)
        return -torch.nn.functional.logsigmoid(BETA * (moved[..., 0] - moved[..., 1])).mean(1)
    old, advantages = ref, noise
    ratio = torch.exp(logp - old)
    gain = torch.minimum(ratio * advantages, ratio.clamp(1 - CLIP, 1 + CLIP) * advantages)
    k3 = torch.exp(ref - logp) - (ref - logp) - 1
    return (KL * k3 - gain).view(N, -1).mean(1)


@pytest.mark.parametrize("objective", ["likelihood", "preference", "policy"])
def test_gradients_of_the_tied_table(lm, objective):
    import torch
    x, tokens, labels, noise = case(torch, 5)
    x64 = x.double().requires_grad_()
    with torch.no_grad():
        table = x64.view(VOCAB, WIDTH)
        logits = (math.sqrt(WIDTH) * table[tokens.reshape(-1)]) @ table.t()
        ref = torch.log_softmax(logits, 1).gather(1, labels.reshape(-1, 1))[:, 0]
        ref = (ref + 0.05 * noise.flip(0).double()).float()
        noise = noise.float()
    want, grads64 = losses64(torch, objective, x64, tokens, labels, ref.double(), noise.double()), []
    for i in range(N):
        grads64.append(torch.autograd.grad(want[i], x64, retain_graph=True)[0])
    model = lm.TiedModel(N, VOCAB, WIDTH)
    dev = [t.cuda() for t in (x, tokens, labels, ref, noise)]
    if objective == "likelihood":
        got, grads = lm.likelihood(model, *dev[:3])
    elif objective == "preference":
        starts = torch.arange(0, N * ROWS + 1, LENGTH, device="cuda")
        got, _, grads = lm.preference(model, *dev[:3], starts, dev[3], beta=BETA)
    else:
        got, grads = lm.policy(model, *dev[:3], dev[3], dev[4], dev[3], clip=CLIP, kl=KL)
    # A logit is a sum of WIDTH products, so it is off by at most (WIDTH + 2) u sum |h| |E|; log p by two of those and a few u of its
    # size.  That error enters the coefficient of a row's gradient: by beta times the rows of a pair, or once through the ratio;
    # and the probabilities, by two more.  Products over VOCAB and ROWS terms follow, of |d logits| <= its largest possible value.
    table = x.double().view(VOCAB, WIDTH)
    hidden = math.sqrt(WIDTH) * table[tokens.reshape(-1)]
    logit = (WIDTH + 2) * U * float((hidden.abs() @ table.abs().t()).max())
    logp = 2 * logit + 16 * U * 8
    off = 2 * logp + {"likelihood": 0.0, "preference": BETA * 2 * LENGTH, "policy": 2.0}[objective] * logp + (VOCAB + ROWS + WIDTH + 16) * U
    coef = {"likelihood": 1.0 / ROWS, "preference": BETA * 2 * LENGTH / ROWS, "policy": 2.0 * float(noise.abs().max()) / ROWS}[objective]
    most = coef * (ROWS * float(hidden.abs().max()) + math.sqrt(WIDTH) * ROWS * 2 * float(table.abs().max()))
    for i in range(N):
        err = float((grads[i].double().cpu() - grads64[i]).abs().max())
        assert err <= off * most, (err, off * most)
        assert err <= 1e-4 * float(grads64[i].abs().max())             # and small against the gradient itself
    loss_off = 4 * (1 + (BETA * 2 * LENGTH if objective == "preference" else 4.0)) * logp + 64 * U * float(want.abs().max())
    assert float((got.double().cpu() - want.detach()).abs().max()) <= loss_off
    # the formula itself against central differences, in 64 bits
    direction = torch.randn(x.numel(), generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    step = 1e-5
    with torch.no_grad():
        up = losses64(torch, objective, x64 + step * direction, tokens, labels, ref.double(), noise.double())
        down = losses64(torch, objective, x64 - step * direction, tokens, labels, ref.double(), noise.double())
    for i in range(N):
        slope, got_slope = float(up[i] - down[i]) / (2 * step), float(grads[i].double().cpu() @ direction)
        assert abs(slope - got_slope) <= 1e-3 * float(grads64[i].norm() * direction.norm()), (slope, got_slope)


@pytest.mark.parametrize("objective,gamma", [("likelihood", 2.0), ("preference", 2.0), ("policy", 2.0)])
def test_training_reaches_its_aim(lm, objective, gamma):
    history = lm.run(objective, rounds=40, workers=3, vocab=130, width=32, rows=192, length=8, gamma=gamma, seed=3)
    assert all(math.isfinite(a) and math.isfinite(b) for a, b in history)
    first, last = history[:5], history[-5:]
    mean = lambda part, k: sum(p[k] for p in part) / len(part)
    assert mean(last, 1) > mean(first, 1), (first, last)               # more of what the objective is after
    if objective != "policy":                                          # (its loss is of tokens drawn anew)
        assert mean(last, 0) < mean(first, 0)
    again = lm.run(objective, rounds=10, workers=3, vocab=130, width=32, rows=192, length=8, gamma=gamma, seed=3)
    assert again == history[:10], "the same rounds again"


def test_the_command(lm, capsys):
    lm.run("preference", rounds=11, workers=2, vocab=100, width=16, rows=64, length=4, report=print)
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 2 and lines[0].startswith("round    0") and "right order" in lines[-1]
