"""The example's policy objective with an entropy term against automatic differentiation in 64 bits and against differences; its AdamW step on EF21's
estimate against the formula; and a run of everything together, captured and eager."""
import math
import os
import sys

import numpy as np
import pytest

import stats_reference as ref
from test_gpu_language_model import CLIP, KL, N, ROWS, U, VOCAB, WIDTH, case, losses64

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lm():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import align_language_model
    return align_language_model


ENTROPY = 0.3


def entropies64(torch, x, tokens):
    table = x.view(VOCAB, WIDTH)
    logp = torch.log_softmax((math.sqrt(WIDTH) * table[tokens.reshape(-1)]) @ table.t(), 1)
    return -(logp.exp() * logp).sum(1)


def test_policy_with_entropy(lm):
    import torch
    x, tokens, labels, noise = case(torch, 7)
    x64 = x.double().requires_grad_()
    with torch.no_grad():
        table = x64.view(VOCAB, WIDTH)
        logp = torch.log_softmax((math.sqrt(WIDTH) * table[tokens.reshape(-1)]) @ table.t(), 1).gather(1, labels.reshape(-1, 1))[:, 0]
        old = (logp + 0.05 * noise.flip(0).double()).float()

    def loss(y):
        return losses64(torch, "policy", y, tokens, labels, old.double(), noise.double()) - ENTROPY * entropies64(torch, y, tokens).view(N, -1).mean(1)

    want = loss(x64)
    grads64 = [torch.autograd.grad(want[i], x64, retain_graph=True)[0] for i in range(N)]
    model = lm.TiedModel(N, VOCAB, WIDTH)
    dx, dt, dl, do, dn = (t.cuda() for t in (x, tokens, labels, old, noise.float()))
    got, grads = lm.policy(model, dx, dt, dl, do, dn, do, clip=CLIP, kl=KL, entropy=ENTROPY)
    # As in test_gpu_language_model: a logit is off by (WIDTH + 2) u sum |h| |E|, log p by two of those; that error enters the coefficients once through the
    # ratio, and through the entropy's slope p (log p + H), whose derivative in log p is at most 1 + log p's size.
    table = x.double().view(VOCAB, WIDTH)
    hidden = math.sqrt(WIDTH) * table[tokens.reshape(-1)]
    size = float(torch.log_softmax(hidden @ table.t(), 1).abs().max())
    d_logp = 2 * (WIDTH + 2) * U * float((hidden.abs() @ table.abs().t()).max()) + 16 * U * size
    off = (4 + 2 * (1 + size)) * d_logp + (VOCAB + ROWS + WIDTH + 16) * U
    coef = (2.0 * float(noise.abs().max()) + ENTROPY * (1 + size)) / ROWS
    most = coef * (ROWS * float(hidden.abs().max()) + math.sqrt(WIDTH) * ROWS * 2 * float(table.abs().max()))
    for i in range(N):
        err = float((grads[i].double().cpu() - grads64[i]).abs().max())
        assert err <= off * most, (err, off * most)
        assert err <= 1e-4 * float(grads64[i].abs().max())
    assert float((got.double().cpu() - want.detach()).abs().max()) <= (8 + ENTROPY * (1 + size)) * d_logp + 64 * U * float(want.abs().max())
    direction = torch.randn(x.numel(), generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    with torch.no_grad():
        up, down = loss(x64 + 1e-5 * direction), loss(x64 - 1e-5 * direction)
    for i in range(N):
        slope, got_slope = float(up[i] - down[i]) / 2e-5, float(grads[i].double().cpu() @ direction)
        assert abs(slope - got_slope) <= 1e-3 * float(grads64[i].norm() * direction.norm())


@pytest.mark.parametrize("bits", [32, 8])
def test_the_step_on_the_estimate(lm, bits):
    """AdamWStep: x moves by the formula from EF21's g, clipped; EF21's own messages are those of its step."""
    import torch
    from paper_2106_05203_amd import binding as b
    d, n, k = 1000, 3, 100
    g = torch.Generator().manual_seed(3)
    x, grads = torch.randn(d, generator=g), torch.randn(n, d, generator=g)
    zeros = torch.zeros(n, d, device="cuda")
    with b.EF21(n, d, k, 0.5) as h:
        dx = x.cuda()
        h.set_state(dx, zeros, zeros[0])
        adamw = lm.AdamWStep(dx, 0.02, 1.0, bits, seed=4)
        for step in (1, 2):
            before, m = dx.double().cpu().numpy(), adamw.optimizer.m[0].float().double().cpu().numpy()
            v = adamw.optimizer.v[0].float().double().cpu().numpy()
            if bits == 8:
                m, v = (a * ref.spread(s[0].double().cpu().numpy(), d) for a, s in ((m, adamw.optimizer.m_scale), (v, adamw.optimizer.v_scale)))
            h.step(grads.cuda() * step)
            adamw.step(h)
            estimate = h.get_state()[2]
            assert torch.equal(estimate, adamw.g) and torch.equal(h.get_g(), estimate)
            norm = float(np.linalg.norm(estimate.double().cpu().numpy()))
            assert norm > 1.0
            want = ref.Adamw(before, estimate.double().cpu().numpy(), m, v, 0.02, (0.9, 0.999), 1e-8, 0.0, step, float(np.float32(1.0 / norm)), bits == 8)
            # the factor is off by its own rounding, which g' is off by beside what the bound has
            slack = 2 * U * np.abs(want.p - before) * 4
            ref.between(dx.double().cpu().numpy(), want.p - want.d_p - slack, want.p + want.d_p + slack, f"step {step}")


@pytest.mark.parametrize("objective,bits,entropy", [("likelihood", 32, 0.0), ("preference", 8, 0.0), ("policy", 8, 0.05)])
def test_training_with_adamw(lm, objective, bits, entropy):
    settings = dict(rounds=12, workers=3, vocab=130, width=32, rows=192, length=8, seed=3, optimizer="adamw", bits=bits, entropy=entropy)
    history = lm.run(objective, **settings)
    assert len(history) == 12 and all(math.isfinite(a) and math.isfinite(b) for a, b in history)
    assert lm.run(objective, **settings) == history, "the same rounds again"


def test_the_command_with_adamw(lm, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["align_language_model.py", "--objective", "policy", "--optimizer", "adamw", "--bits", "8", "--entropy", "0.02", "--rounds", "3",
                                      "--workers", "2", "--vocab", "100", "--width", "16", "--rows", "64", "--length", "4"])
    lm.main()
    lines = capsys.readouterr().out.splitlines()
    assert lines[0].startswith("round    0") and sum(line.startswith("behind") for line in lines) == 3


def test_a_step_of_everything_captured(lm):
    """Statistics, policy loss, both gradients, the norm and AdamW in one graph, replayed with eager work in between, beside the same eagerly."""
    import torch
    from paper_2106_05203_amd import binding as b
    rows, vocab, width = 200, 3001, 64
    g = torch.Generator(device="cuda").manual_seed(0)
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    tokens, labels = (torch.randint(0, vocab, (1, rows), generator=g, device="cuda") for _ in range(2))
    old, adv = randn(rows) * 0.1 - 8.0, randn(rows)
    weight, bonus = torch.full((rows,), 1.0 / rows, device="cuda"), torch.full((rows,), -0.01 / rows, device="cuda")
    start = (randn(vocab, width) * 0.1).to(torch.bfloat16)

    def make():
        s = {"table": start.clone(), "grad": torch.zeros(1, vocab, width, device="cuda"), "logits": torch.zeros(rows, vocab, device="cuda", dtype=torch.bfloat16)}
        s["dlogits"], s["hidden"] = torch.zeros_like(s["logits"]), torch.zeros(rows, width, device="cuda", dtype=torch.bfloat16)
        s["dhidden"] = torch.zeros(1, rows, width, device="cuda", dtype=torch.bfloat16)
        s["small"] = [torch.zeros(rows, device="cuda") for _ in range(6)]
        s["sums"], s["one"], s["norm"], s["factor"] = torch.zeros(rows, 2, device="cuda"), *(torch.zeros(1, device="cuda") for _ in range(3))
        s["step"] = torch.zeros(1, dtype=torch.int64, device="cuda")
        s["optimizer"] = b.AdamW([s["table"]], [s["grad"][0]], bits=8, stochastic=True, seed=5)
        s["list"] = b.TensorList([s["grad"]])
        s["space"] = {n: torch.zeros(size, dtype=torch.uint8, device="cuda") for n, size in (
            ("stats", max(1, b.ef21_token_stats_workspace(1, rows, vocab, 0))), ("policy", max(1, b.ef21_policy_loss_workspace(rows))),
            ("embed", b.ef21_embed_grad_workspace(1, rows, vocab, width)), ("norm", b.ef21_grad_norm_workspace(1)))}
        return s

    def step(s):
        s["step"].add_(1)
        b.ef21_embed(s["table"], tokens[0], 8.0, out=s["hidden"])
        torch.mm(s["hidden"], s["table"].t(), out=s["logits"])
        logp, lse, entropy, loss_logp, token_loss, _ = s["small"]
        b.ef21_token_stats(s["logits"], labels[0], 0, logp, lse, entropy, sums=s["sums"], workspace=s["space"]["stats"])
        b.ef21_policy_loss(s["logits"], labels[0], old, adv, 0.2, 0.2, weight=weight, out_loss=s["one"], token_loss=token_loss, logp=loss_logp, grad=s["dlogits"],
                           workspace=s["space"]["policy"])
        b.ef21_token_stats_grad(s["logits"], labels[0], s["sums"], entropy, None, bonus, out=s["dlogits"], accumulate=True)
        torch.mm(s["dlogits"], s["table"], out=s["dhidden"][0])
        b.ef21_embed_grad(s["dhidden"], tokens, vocab, 8.0, out=s["grad"], workspace=s["space"]["embed"])
        b.ef21_grad_norm(s["list"], 0.1, norm=s["norm"], factor=s["factor"], workspace=s["space"]["norm"])
        s["optimizer"].step(1e-3, step=s["step"], grad_scale=s["factor"])

    eager, captured, warm, side = make(), make(), make(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(captured)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        for name in ("table", "grad", "dlogits", "sums", "norm", "factor"):
            assert torch.equal(eager[name], captured[name]), name
        for one, other in zip(eager["small"][:5], captured["small"]):
            assert torch.equal(one, other)
        for name in ("m", "v", "m_scale", "v_scale"):
            assert torch.equal(getattr(eager["optimizer"], name)[0].view(torch.uint8), getattr(captured["optimizer"], name)[0].view(torch.uint8)), name
    assert bool((eager["table"] != start).any()) and int(eager["step"]) == 4
