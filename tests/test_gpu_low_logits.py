"""Rows of logits far below zero, with masks in front of, behind and among what is left: log-probabilities, both losses and their gradients against
the 64-bit reference (tests/lm_reference.py, where the bounds are derived).  A row moved by a constant keeps its log-probabilities.

A gradient's probabilities are formed from one rounded number of the size of lse log2 e where that is far below the type's rounding; the bound of
R.grad counts that up to |lse| = 64, so 2 u (|m| + |lse|) p |c| is added here for every row, with |m| <= |lse| + log V.
"""
import math

import numpy as np
import pytest

import lm_reference as lm

pytestmark = pytest.mark.gpu

TYPES = ["f32", "bf16", "f16"]
LO, HI, BETA, KL = (float(np.float32(v)) for v in (0.2, 0.28, 0.3, 0.1))


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2106_05203_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load_library()
    return torch, binding


def as64(t):
    return t.detach().double().cpu().numpy()


def gradient(R, coef, d_coef, dtype):
    g, bound = R.grad(coef, d_coef, dtype)
    size = np.where(np.isfinite(R.lse), np.abs(R.lse), 0.0)
    return g, bound + 1.01 * np.abs(coef)[:, None] * R.p * (2 * lm.U * (2 * size + math.log(R.V)))[:, None]


def check(torch, b, x, labels, dtype):
    """Every operator on the rows x [rows][V] (an even number of them) against the reference."""
    rows = len(labels)
    R = lm.Rows(as64(x), labels)
    dl = torch.from_numpy(labels).cuda()
    rng = np.random.default_rng(rows + R.V)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    logp, lse = b.ef21_token_logps(x, dl)
    lm.inside(as64(lse), R.lse, R.d_lse, "lse")
    lm.inside(as64(logp), R.logp, R.d_logp, "logp")
    coef = rng.standard_normal(rows).astype(np.float32)
    g, bound = gradient(R, coef.astype(np.float64), np.zeros(rows), dtype)
    lm.inside(as64(b.ef21_token_logps_grad(x, dl, lse, dev(coef))), g, bound, "gradient")
    # pairs of one row each
    ref = (R.logp + 0.2 * rng.standard_normal(rows)).astype(np.float32)
    start = np.arange(rows + 1)
    want, d_want, coef, d_coef = lm.preference(R, start, ref, BETA, 0.0, False, False, None)
    loss, logp2, grad = b.ef21_preference_loss(x, dl, dev(start), dev(ref), BETA)
    lm.inside(as64(logp2), R.logp, R.d_logp, "logp of the preference loss")
    lm.inside(as64(loss), want, d_want, "preference loss")
    g, bound = gradient(R, coef, d_coef, dtype)
    lm.inside(as64(grad), g, bound, "gradient of the preference loss")
    # log ratios away from the clip range's edges, where rounding alone decides
    d = rng.standard_normal(rows) * 0.3
    for edge in (math.log1p(-LO), math.log1p(HI)):
        d = np.where(np.abs(d - edge) < 0.01, edge + 0.02, d)
    old, adv = (R.logp - d).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
    want, d_want, total, d_total, coef, d_coef = lm.policy(R, old, adv, LO, HI, ref, KL, None)
    got, tokens, logp3, grad = b.ef21_policy_loss(x, dl, dev(old), dev(adv), LO, HI, ref_logp=dev(ref), kl=KL)
    lm.inside(as64(logp3), R.logp, R.d_logp, "logp of the policy loss")
    lm.inside(as64(tokens), want, d_want, "token loss")
    lm.inside(as64(got), np.array([total]), np.array([d_total]), "policy loss")
    g, bound = gradient(R, coef, d_coef, dtype)
    lm.inside(as64(grad), g, bound, "gradient of the policy loss")


def masks(rng, vocab):
    """Columns that are masked, never all of them."""
    at = np.arange(vocab)
    front = [at < min(k, vocab - 2) for k in (8, 512, 4096, vocab // 16 + 1, vocab // 8 + 1)]
    some = rng.random(vocab) < 0.95
    some[rng.integers(0, vocab, 2)] = False
    return [at < 0, *front, some, at >= vocab // 2 + 1]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [20, 130, 700, 5003, 20000, 50304, 150001])
def test_masks_and_low_logits(gpu, vocab, dtype):
    """150001 columns: the policy loss in two passes; below, with the row held in registers.  Rows around -5000 lie on both sides of where the library
    takes an entry for a mask."""
    torch, b = gpu
    print(f"low logits vocab={vocab} {dtype}", flush=True)
    rng = np.random.default_rng(vocab)
    kinds, labels = [], []
    for center in (-60.0, -90.0, -100.0, -300.0, -5000.0) if vocab <= 20000 else (-90.0, -120.0, -5000.0):
        for i, masked in enumerate(masks(rng, vocab)):
            low = [-math.inf, -math.inf, -1e4, float(torch.finfo(lm.TORCH[dtype]).min)][i % 4]
            kinds.append(np.where(masked, low, center + 2.0 * rng.standard_normal(vocab)))
            labels.append(rng.choice(np.flatnonzero(~masked)))
    x = torch.from_numpy(np.stack(kinds)).to(lm.TORCH[dtype]).cuda()
    check(torch, b, x, np.array(labels), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("center", [-90.0, -120.0, -5000.0])
def test_short_rows_at_every_alignment(gpu, center, dtype):
    """Rows that are a piece or two and a few entries before and behind them: some threads have nothing but such an entry."""
    torch, b = gpu
    rng = np.random.default_rng(int(-center))
    for vocab in range(1, 41):
        rows, stride = 16, (vocab + 1) | 1                             # odd: the rows start at every alignment
        buf = torch.full((rows * stride + 8,), math.nan, dtype=lm.TORCH[dtype], device="cuda")
        x = buf.as_strided((rows, vocab), (stride, 1))
        x.copy_(torch.from_numpy(center + 3.0 * rng.standard_normal((rows, vocab))))
        check(torch, b, x, rng.integers(0, vocab, rows), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [9, 33, 1201, 9000, 50304, 150001])
def test_a_row_moved_by_a_constant(gpu, vocab, dtype):
    """Multiples of a half: x - 100 is exact in every type, and logp may differ by the two rows' bounds alone."""
    torch, b = gpu
    rng = np.random.default_rng(vocab)
    kinds, labels = [], []
    for masked in masks(rng, vocab):
        kinds.append(np.where(masked, -math.inf, 0.5 * np.clip(np.rint(4 * rng.standard_normal(vocab)), -16, 16)))
        labels.append(rng.choice(np.flatnonzero(~masked)))
    x = torch.from_numpy(np.stack(kinds)).to(lm.TORCH[dtype]).cuda()
    moved = x - 100.0
    assert torch.equal((moved.double() + 100.0), x.double())
    labels = np.array(labels)
    dl, zero = torch.from_numpy(labels).cuda(), torch.zeros(len(labels), device="cuda")
    bound = lm.Rows(as64(x), labels).d_logp + lm.Rows(as64(moved), labels).d_logp
    start = torch.arange(len(labels) + 1, device="cuda")
    for what, logp in [("token_logps", lambda y: b.ef21_token_logps(y, dl)[0]),
                       ("preference_loss", lambda y: b.ef21_preference_loss(y, dl, start, zero, 1.0, grad=False)[1]),
                       ("policy_loss", lambda y: b.ef21_policy_loss(y, dl, zero, zero, 0.2, 0.2, grad=False)[2])]:
        lm.inside(as64(logp(moved)), as64(logp(x)), bound, what)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [24, 130, 700, 5003, 20000, 50304, 150001])
def test_entries_far_from_the_first_ones(gpu, vocab, dtype):
    """A thread adds its part of a row relative to its first entries.  Here others lie 20 to 130 above them (in another thread's reach or not), or below
    where the first ones are masked."""
    torch, b = gpu
    print(f"far entries vocab={vocab} {dtype}", flush=True)
    rng = np.random.default_rng(vocab)
    at, base = np.arange(vocab), rng.standard_normal(vocab)
    kinds = [40 * base, 25 * base - 85, 100 * base + 50]
    for up in (20.0, 30.0, 45.0, 60.0, 75.0, 85.0, 87.0):
        one = base - 50.0
        one[-1 - vocab // 3] += up
        kinds.append(one)
        two = base - 80.0                                              # one more, among the first entries of another thread
        two[3], two[-1 - vocab // 3] = 9.0, -80.0 + up
        kinds.append(two)
    for height in (-80.0, -60.0, -30.0, 30.0, 60.0, 80.0):             # nothing among the first entries
        kinds.append(np.where(at < max(vocab // 2, 4), -math.inf, height + base))
        few = np.where(at % 7 == 5, height + 3 * base, -1e4)
        kinds.append(few)
    for down in (60.0, 86.5, 87.5, 88.0):                              # a few high entries: the first ones of some threads, behind low ones in others
        for share in (0.003, 0.01, 0.03, 0.1):
            high = rng.random(vocab) < share
            high[[0, -2]] = True
            kinds.append(np.where(high, 0.0, -down) + 0.1 * base)
    kinds = kinds[1:] if len(kinds) % 2 else kinds
    if vocab > 20000:
        kinds = kinds[-16:] + kinds[:10]
    x = torch.from_numpy(np.stack(kinds)).to(lm.TORCH[dtype]).cuda()
    labels = np.argmax(as64(x), axis=1)
    likely = np.argsort(-as64(x), axis=1)[:, : min(vocab, 4)]
    labels[::3] = likely[::3, -1]                                      # also one that is not the largest
    far = lm.Rows(as64(x), labels).logp < -60.0
    labels[far] = np.argmax(as64(x), axis=1)[far]
    check(torch, b, x, labels, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_large_sum_beside_a_guess(gpu, dtype):
    """Four wavefronts take 6144 columns, 2048 at first.  One finds masks and then an entry at -44; the others start at -90 and one of them meets an entry at
    -46.25: relative to what they started from 2^-63 and 2^63, and a ninth of the row's sum is the second one's."""
    torch, b = gpu
    vocab, entries = 6144, 4 if dtype == "f32" else 8
    at = np.arange(vocab)
    wave = at // entries % 256 // 64
    row = np.where(wave == 0, -math.inf, -90.0)
    low, high = np.flatnonzero((wave == 1) & (at > 4200))[9], np.flatnonzero((wave == 0) & (at > 4200))[20]
    row[high], row[low] = -44.0, -46.25
    x = torch.from_numpy(np.stack([row, row])).to(lm.TORCH[dtype]).cuda()
    check(torch, b, x, np.array([low, high]), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [24, 700, 5003, 20000, 50304, 150001])
def test_one_entry_beyond_all_scales(gpu, vocab, dtype):
    """A row of ordinary logits with one of 10^9 to 3 10^38: x log2 e of that one is rounded by more than fp32's range of exponents."""
    torch, b = gpu
    print(f"one large entry vocab={vocab} {dtype}", flush=True)
    rng = np.random.default_rng(vocab)
    rows = 24
    values = rng.standard_normal((rows, vocab))
    labels = rng.integers(0, vocab, rows)
    values[np.arange(rows), labels] = np.append(10.0 ** rng.uniform(9, 38, rows - 2), [3.3e38, 2.0 ** 127])
    x = torch.from_numpy(values).to(lm.TORCH[dtype]).cuda()
    check(torch, b, x, labels, dtype)
