"""The operators on rows of logits at the ends of what they accept, against the 64-bit reference (tests/lm_reference.py)."""
import math

import numpy as np
import pytest

import lm_reference as lm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2106_05203_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load_library()
    return torch, binding


def as64(t):
    return t.detach().double().cpu().numpy()


def test_more_pairs_than_a_launch_has_workgroups(gpu):
    """2^22 + 1 pairs, all but three of them empty: the loss of an empty pair is log 2, within an ulp."""
    torch, b = gpu
    pairs, vocab, rng = 2 ** 22 + 1, 40, np.random.default_rng(0)
    lengths = np.zeros((pairs, 2), dtype=np.int64)
    full = [0, 2 ** 21 + 7, pairs - 1]
    lengths[full] = [[3, 4], [5, 2], [6, 7]]
    start = np.concatenate([[0], np.cumsum(lengths.reshape(-1))])
    rows = int(start[-1])
    x = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32)).cuda()
    labels = rng.integers(0, vocab, rows)
    labels[[1, 9]] = -100
    R = lm.Rows(as64(x), labels)
    ref = (R.logp + 0.2 * rng.standard_normal(rows)).astype(np.float32)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    loss, logp, grad = b.ef21_preference_loss(x, dev(labels), dev(start), dev(ref), 0.5, pair_weight=torch.ones(pairs, device="cuda"),
                                              out_loss=torch.full((pairs,), math.nan, device="cuda"))
    want, d_want, coef, d_coef = lm.preference(R, np.concatenate([[0], np.cumsum(lengths[full].reshape(-1))]), ref, 0.5, 0.0, False, False, np.ones(3))
    lm.inside(as64(loss[full]), want, d_want, "loss")
    lm.inside(as64(logp), R.logp, R.d_logp, "logp")
    g, bound = R.grad(coef, d_coef, "f32")
    lm.inside(as64(grad), g, bound, "gradient")
    loss[full] = math.log(2.0)
    assert float((loss.double() - math.log(2.0)).abs().max()) <= 2.0 ** -24


@pytest.mark.parametrize("top", [2.0, 500.0])
def test_the_longest_row(gpu, top):
    """2^31 - 1 columns, the first and the last one not masked (500: sums that need the row's maximum, gradient entry by entry).  Both have the
    probability 1/2, so everything is exact but for a few roundings; nothing around the row is written."""
    torch, b = gpu
    vocab, around = 2 ** 31 - 1, 4096
    buf = torch.full((vocab + 2 * around,), -math.inf, dtype=torch.bfloat16, device="cuda")
    x = buf[around:around + vocab].view(1, vocab)
    x[0, 0], x[0, -1] = top, top
    buf[:around], buf[around + vocab:] = 7.0, 7.0
    label, one = torch.tensor([vocab - 1], device="cuda"), torch.ones(1, device="cuda")

    def halves(g, coef, what):
        print(f"the longest row, {top}: {what}", flush=True)
        assert float(g[0, -1]) == coef / 2 and float(g[0, 0]) == -coef / 2
        assert not any(int(part.count_nonzero()) for part in g[0, 1:-1].split(1 << 28))

    print(f"the longest row, {top}", flush=True)
    logp, lse = b.ef21_token_logps(x, label)
    assert float(lse) == pytest.approx(top + math.log(2.0), rel=1e-6) and float(logp) == pytest.approx(-math.log(2.0), rel=1e-6)
    # a margin of logp - ref = 0: the slope is -1/2
    start, out = torch.tensor([0, 1, 1], device="cuda"), torch.full_like(x, math.nan)
    loss, logp2, grad = b.ef21_preference_loss(x, label, start, logp, 1.0, grad=out)
    assert torch.equal(logp2, logp) and float(loss) == pytest.approx(math.log(2.0), rel=1e-6)
    halves(grad, -0.5, "preference loss")
    total, _, logp3, grad = b.ef21_policy_loss(x, label, logp, one, 0.2, 0.2, grad=out)
    assert torch.equal(logp3, logp) and float(total) == -1.0
    halves(grad, -1.0, "policy loss")
    del out, grad
    b.ef21_token_logps_grad(x, label, lse, one, out=x)
    halves(x, 1.0, "log-probability")
    assert bool((buf[:around] == 7.0).all()) and bool((buf[around + vocab:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [40, 3000, 40000, 150001])           # the row held by teams of three sizes; two passes
def test_policy_loss_of_an_impossible_token(gpu, vocab, dtype):
    """A label of probability zero: the ratio is zero, and a KL term is infinite, o = ref_logp - logp being so, not a NaN.  The gradient of such a row is not
    finite: where a column has a positive probability it is the infinite slope's sign, for the label the other one.  Other rows keep theirs."""
    torch, b = gpu
    rng = np.random.default_rng(vocab)
    rows = 4
    x = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32)).to(lm.TORCH[dtype]).cuda()
    labels = rng.integers(0, vocab, rows)
    x[1, labels[1]] = -math.inf
    x[3] = -math.inf                                                   # nothing is left of the row: no gradient
    dl = torch.from_numpy(labels).cuda()
    one = torch.ones(rows, device="cuda")
    old, adv = -2.0 * one, torch.tensor([1.0, -1.0, -1.0, 1.0], device="cuda")
    total, tokens, logp, grad = b.ef21_policy_loss(x, dl, old, adv, 0.2, 0.2, ref_logp=old, kl=0.1)
    assert logp.tolist()[1] == logp.tolist()[3] == -math.inf
    assert tokens.tolist()[1] == tokens.tolist()[3] == math.inf and total.item() == math.inf
    assert bool(torch.isfinite(tokens[[0, 2]]).all()) and bool(torch.isfinite(grad[[0, 2]].float()).all())
    assert grad[1, labels[1]].item() == -math.inf
    others = torch.arange(vocab, device="cuda") != labels[1]
    assert bool((grad[1][others].float() == math.inf).all()) and not bool(grad[3].count_nonzero())
    # without the KL term all is finite: q = 0, so min(q A, clip(q) A) is 0 for A > 0 and 0.8 A, which has no slope, for A < 0
    total, tokens, _, grad = b.ef21_policy_loss(x, dl, old, adv, 0.2, 0.2)
    assert tokens.tolist()[1] == pytest.approx(0.8, rel=1e-6) and tokens.tolist()[3] == 0.0 and math.isfinite(total.item())
    assert not bool(grad[[1, 3]].count_nonzero()) and bool(torch.isfinite(grad.float()).all())
    # a reference that is impossible as well leaves o undefined
    ref = torch.where(torch.tensor([False, True, False, False], device="cuda"), -math.inf, old)
    tokens = b.ef21_policy_loss(x, dl, old, adv, 0.2, 0.2, ref_logp=ref, kl=0.1)[1]
    assert math.isnan(tokens.tolist()[1]) and tokens.tolist()[3] == math.inf


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [40, 700, 9000, 40000, 150001])
def test_infinite_slopes_leave_masked_columns_alone(gpu, vocab, dtype):
    """A gradient is slope ([v = label] - p_v), of an infinite slope too: infinite where that factor is not zero, zero and no NaN where it is."""
    torch, b = gpu
    rng = np.random.default_rng(vocab)
    inf, rows = math.inf, 5
    values = rng.standard_normal((rows, vocab)).astype(np.float32)
    values[3] += -6e4 if dtype == "f16" else -5e6                      # a row far from zero
    x = torch.from_numpy(values).to(lm.TORCH[dtype]).cuda()
    masked = torch.from_numpy(rng.random((rows, vocab)) < 0.3).cuda()
    x[masked] = -inf
    labels = np.array([int(rng.choice(np.flatnonzero(~masked[r].cpu().numpy()))) for r in range(rows)])
    labels[0] = int(np.flatnonzero(masked[0].cpu().numpy())[0])       # impossible
    x[4] = -inf
    x[4, labels[4]] = 1.0                                              # certain
    dl, one = torch.from_numpy(labels).cuda(), torch.ones(rows, device="cuda")
    logp, lse = b.ef21_token_logps(x, dl)
    p = torch.softmax(x.double(), 1)
    hot = torch.zeros_like(p)
    hot[torch.arange(rows), dl] = 1.0
    factor = hot - p
    clear = (factor == 0) | (factor.abs() > 1e-30)                     # what fp32 shows without doubt
    clear[4, labels[4]] = False                                        # (1 - p of the certain label is a rounding)

    def expect(grad, slopes, what):
        grad = grad.double()
        for r, slope in enumerate(slopes):
            want = torch.where(factor[r] == 0, 0.0, slope * factor[r]) if math.isinf(slope) else None
            if want is None:
                assert bool(torch.isfinite(grad[r]).all()), f"{what}: row {r}"
            else:
                assert torch.equal(grad[r][clear[r]], want[clear[r]]), f"{what}: row {r}"
                assert not bool(torch.isnan(grad[r]).any()), f"{what}: row {r}"

    expect(b.ef21_token_logps_grad(x, dl, lse, torch.tensor([inf, -inf, 1.0, inf, -inf], device="cuda")), [inf, -inf, 1.0, inf, -inf], "log-probability")
    # least squares: the margin of (0, 1) is -inf, of (2, 3) finite
    start = torch.tensor([0, 1, 2, 3, 4], device="cuda")
    loss, _, grad = b.ef21_preference_loss(x, dl, start, logp.clamp(min=-10.0), 0.5, loss=1, pair_weight=one[:2])
    assert loss.tolist()[0] == inf and math.isfinite(loss.tolist()[1])
    expect(grad, [-inf, inf, 1.0, 1.0, 1.0], "preference loss")
    # the KL term of the impossible label; a ratio beyond fp32 where the advantage is negative
    old = logp.clamp(min=-10.0) + torch.tensor([0.0, -200.0, 0.0, -200.0, -200.0], device="cuda")
    ref = logp.clamp(min=-10.0)
    _, tokens, _, grad = b.ef21_policy_loss(x, dl, old, -one, 0.2, 0.2, ref_logp=ref, kl=0.1, weight=one)
    assert tokens.tolist()[0] == inf
    expect(grad, [-inf, inf, 1.0, inf, inf], "policy loss")
