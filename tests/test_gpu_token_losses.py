"""Log-probabilities of tokens, the preference loss and the clipped policy loss against a plain implementation in 64 bits
(tests/lm_reference.py, where the bounds are derived)."""
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


def make_logits(torch, rows, vocab, dtype, seed, stride=None, offset=0, spread=2.0):
    """(device view [rows][vocab] at `offset` entries into its memory, rows `stride` apart, its values in 64 bits); what lies between the rows
    is NaN and must not be read."""
    rng = np.random.default_rng(seed)
    stride = stride or vocab
    buf = torch.full((max(rows, 1) * stride + offset + 64,), math.nan, dtype=lm.TORCH[dtype])
    x = torch.from_numpy((rng.standard_normal((rows, vocab)) * spread).astype(np.float32)).to(lm.TORCH[dtype])
    view = buf[offset:].as_strided((rows, vocab), (stride, 1))
    view.copy_(x)
    dev = buf.cuda()[offset:].as_strided((rows, vocab), (stride, 1))
    return dev, x.double().numpy()


def make_labels(torch, rows, vocab, seed, wide=True, ignored=0.2):
    rng = np.random.default_rng(seed + 1000)
    labels = rng.integers(0, vocab, rows)
    labels[rng.random(rows) < ignored] = -100
    return labels, torch.from_numpy(labels.astype(np.int64 if wide else np.int32)).cuda()


def as64(t):
    return t.detach().double().cpu().numpy()


# rows, vocab, stride, offset: around the vector widths, one entry, odd vocabularies, rows that start anywhere
SHAPES = [(1, 1, 1, 0), (3, 2, 2, 1), (5, 7, 9, 3), (4, 63, 63, 0), (4, 64, 64, 0), (9, 65, 67, 5), (2, 255, 255, 0), (7, 1000, 1000, 0),
          (3, 1024, 1024, 8), (2, 2047, 2049, 1), (5, 4096, 4104, 0), (3, 5001, 5001, 2), (2, 16384, 16384, 0), (2, 32001, 32001, 0),
          (1, 65536, 65536, 0), (2, 70003, 70010, 7), (1, 131072, 131072, 0), (1, 150001, 150001, 3), (2, 300000, 300000, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,stride,offset", SHAPES)
def test_logps_and_gradient(gpu, rows, vocab, stride, offset, dtype):
    torch, b = gpu
    print(f"logps rows={rows} vocab={vocab} stride={stride} offset={offset} {dtype}", flush=True)
    x, x64 = make_logits(torch, rows, vocab, dtype, seed=rows * 7 + vocab, stride=stride, offset=offset)
    labels, dl = make_labels(torch, rows, vocab, seed=vocab, wide=vocab % 2 == 0)
    R = lm.Rows(x64, labels)
    logp, lse = b.ef21_token_logps(x, dl)
    lm.inside(as64(lse), R.lse, R.d_lse, "lse")
    lm.inside(as64(logp), R.logp, R.d_logp, "logp")
    coef = np.random.default_rng(5).standard_normal(rows).astype(np.float32)
    grad = b.ef21_token_logps_grad(x, dl, lse, torch.from_numpy(coef).cuda())
    g, bound = R.grad(coef.astype(np.float64), np.zeros(rows), dtype)
    lm.inside(as64(grad), g, bound, "gradient")
    # a gradient with another stride and start than the logits
    other = torch.full((rows * (vocab + 3) + 1,), 7.0, dtype=x.dtype, device="cuda")
    to = other[1:].as_strided((rows, vocab), (vocab + 3, 1))
    b.ef21_token_logps_grad(x, dl, lse, torch.from_numpy(coef).cuda(), out=to)
    assert torch.equal(to, grad)
    gaps = other[1:].as_strided((rows, 3), (vocab + 3, 1), 1 + vocab)[: rows - 1]
    assert bool((gaps == 7.0).all()) and float(other[0]) == 7.0, "entries beside the rows were written"
    # over the logits
    b.ef21_token_logps_grad(x, dl, lse, torch.from_numpy(coef).cuda(), out=x)
    assert torch.equal(x, grad)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [5, 130, 1500, 20000, 90000, 200000])
def test_masked_entries_and_odd_rows(gpu, vocab, dtype):
    torch, b = gpu
    print(f"masks vocab={vocab} {dtype}", flush=True)
    rows = 9
    x, x64 = make_logits(torch, rows, vocab, dtype, seed=vocab)
    labels = np.array([1, vocab - 1, 0, 2, 3, -100, vocab, 4, -1], dtype=np.int64)
    low = torch.finfo(x.dtype).min
    x[0, vocab // 2:] = -math.inf; x64[0, vocab // 2:] = -np.inf                  # masked behind the middle
    x[1, :-1] = -math.inf; x64[1, :-1] = -np.inf                                  # the label alone is left
    x[2] = -math.inf; x64[2] = -np.inf                                            # nothing is left
    x[3] = low; x64[3] = float(low)                                               # the type's lowest value everywhere
    x[4, 1:3] = low; x64[4, 1:3] = float(low)
    x[5] = math.nan; x[6] = math.nan; x[8] = math.inf                             # rows without a label are not read
    x[7, 4] = -math.inf; x64[7, 4] = -np.inf                                      # the label itself has probability zero
    dl = torch.from_numpy(labels).cuda()
    x64[5], x64[6], x64[8] = 0.0, 0.0, 0.0
    R = lm.Rows(x64, labels)
    logp, lse = b.ef21_token_logps(x, dl)
    lm.inside(as64(lse), R.lse, R.d_lse, "lse")
    lm.inside(as64(logp), R.logp, R.d_logp, "logp")
    coef = np.linspace(-1, 1, rows).astype(np.float32)
    grad = b.ef21_token_logps_grad(x, dl, lse, torch.from_numpy(coef).cuda())
    g, bound = R.grad(coef.astype(np.float64), np.zeros(rows), dtype)
    lm.inside(as64(grad), g, bound, "gradient")
    for r in (2, 5, 6, 8):
        assert not bool(grad[r].count_nonzero()), "a row without a distribution has no gradient"
    # the losses read nothing where there is no label, whatever their other inputs hold there
    nan = np.where(R.has, 0.1, np.nan).astype(np.float32)
    dn = torch.from_numpy(nan).cuda()
    start = torch.tensor([0, 1, 2, 5, 9], device="cuda")
    keep = [0, 1, 3, 4]                                                           # rows with a finite log-probability
    dl2 = torch.full_like(dl, -100)
    dl2[keep] = dl[keep]
    dn2 = torch.full_like(dn, math.nan)
    dn2[keep] = dn[keep]
    loss, logp2, grad2 = b.ef21_preference_loss(x, dl2, start, dn2, 0.3)
    assert bool(torch.isfinite(loss).all()) and torch.equal(logp2[keep], logp[keep]) and bool(torch.isfinite(grad2.float()).all())
    total, tokens, logp3, grad3 = b.ef21_policy_loss(x, dl2, dn2, dn2, 0.2, 0.2, ref_logp=dn2, kl=0.1, weight=dn2)
    assert bool(torch.isfinite(total).all()) and bool(torch.isfinite(tokens).all()) and torch.equal(logp3, logp2)
    # (the KL term's slope, 0.01 (exp(0.1 - logp) - 1), passes fp16's largest number at vocab = 200000 and rounds to infinity there)
    assert not bool(torch.isnan(grad3).any()) and not bool(grad3[[2, 5, 6, 7, 8]].count_nonzero())


@pytest.mark.parametrize("vocab", [40, 3000, 40000, 140000])
def test_nan_stays_in_its_row(gpu, vocab):
    torch, b = gpu
    x, x64 = make_logits(torch, 4, vocab, "bf16", seed=3)
    x[1, vocab // 3] = math.nan
    x[2, vocab // 2] = math.inf
    labels, dl = make_labels(torch, 4, vocab, seed=4, ignored=0.0)
    logp, lse = b.ef21_token_logps(x, dl)
    one = torch.ones(4, device="cuda")
    grad = b.ef21_token_logps_grad(x, dl, lse, one)
    assert torch.isnan(lse).tolist() == [False, True, True, False] and torch.isnan(logp).tolist()[1]
    assert bool(torch.isnan(grad[1]).all()) and bool(torch.isfinite(grad[[0, 3]].float()).all())
    total, tokens, _, grad = b.ef21_policy_loss(x, dl, -one, one, 0.2, 0.2)
    assert math.isnan(float(total)) and bool(torch.isfinite(tokens[[0, 3]]).all()) and bool(torch.isfinite(grad[[0, 3]].float()).all())


PAIRS = [  # lengths of the sequences, rows before the first and after the last
    ([1, 1], 0, 0), ([0, 0], 0, 2), ([3, 0, 0, 5], 0, 0), ([4, 9, 1, 2, 30, 17], 2, 3), ([130, 64, 65, 200], 0, 0), ([1] * 40, 0, 0), ([700, 300], 1, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lengths,before,after", PAIRS)
@pytest.mark.parametrize("loss,mean,smoothing", [(0, False, 0.0), (0, True, 0.1), (1, True, 0.0), (1, False, 0.0)])
def test_preference_loss(gpu, lengths, before, after, dtype, loss, mean, smoothing):
    torch, b = gpu
    vocab = 33 if sum(lengths) > 100 else 1201
    start = np.cumsum([before] + lengths)
    rows = int(start[-1]) + after
    print(f"preference rows={rows} pairs={len(lengths) // 2} {dtype} loss={loss} mean={mean}", flush=True)
    x, x64 = make_logits(torch, rows, vocab, dtype, seed=rows, stride=vocab + (rows % 3))
    labels, dl = make_labels(torch, rows, vocab, seed=rows, wide=mean)
    R = lm.Rows(x64, labels)
    rng = np.random.default_rng(9)
    ref = (R.logp + 0.2 * rng.standard_normal(rows)).astype(np.float32)
    ref[~R.has] = np.nan
    weight = None if loss else rng.random(len(lengths) // 2).astype(np.float32)
    ref64 = np.where(R.has, ref, 0.0)
    want, d_want, coef, d_coef = lm.preference(R, start, ref64, float(np.float32(0.3)), float(np.float32(smoothing)), loss == 1, mean, weight)
    dw = None if weight is None else torch.from_numpy(weight).cuda()
    args = (x, dl, torch.from_numpy(start.astype(np.int64)).cuda(), torch.from_numpy(ref).cuda(), 0.3)
    kw = dict(smoothing=smoothing, loss=loss, mean=mean, pair_weight=dw)
    got, logp, grad = b.ef21_preference_loss(*args, **kw)
    lm.inside(as64(got), want, d_want, "loss")
    lm.inside(as64(logp), R.logp, R.d_logp, "logp")
    g, bound = R.grad(coef, d_coef, dtype)
    lm.inside(as64(grad), g, bound, "gradient")
    alone, logp2, none = b.ef21_preference_loss(*args, **kw, grad=False)
    assert none is None and torch.equal(alone, got) and torch.equal(logp2, logp), "the loss alone is the same"
    over = b.ef21_preference_loss(*args, **kw, grad=x)
    assert torch.equal(over[0], got) and torch.equal(x, grad), "over the logits the gradient is the same"


def away_from_edges(logp, rng, rows, lo, hi):
    """Old log-probabilities whose ratio is nowhere near a clip edge, where rounding alone decides."""
    d = rng.standard_normal(rows) * 0.3
    for edge in (math.log1p(-lo) if lo < 1 else -50.0, math.log1p(hi)):
        d = np.where(np.abs(d - edge) < 0.01, edge + 0.02, d)
    return (np.where(np.isfinite(logp), logp, 0.0) - d).astype(np.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,stride,offset", SHAPES + [(300, 50, 50, 0), (1000, 129, 130, 1)])
@pytest.mark.parametrize("kl,weighted", [(0.0, False), (0.1, True)])
def test_policy_loss(gpu, rows, vocab, stride, offset, dtype, kl, weighted):
    torch, b = gpu
    print(f"policy rows={rows} vocab={vocab} {dtype} kl={kl}", flush=True)
    x, x64 = make_logits(torch, rows, vocab, dtype, seed=rows + vocab, stride=stride, offset=offset)
    labels, dl = make_labels(torch, rows, vocab, seed=rows, wide=not weighted)
    R = lm.Rows(x64, labels)
    rng = np.random.default_rng(11)
    lo, hi = float(np.float32(0.2)), float(np.float32(0.28))
    old = away_from_edges(R.logp, rng, rows, lo, hi)
    adv = rng.standard_normal(rows).astype(np.float32)
    ref = (R.logp + 0.2 * rng.standard_normal(rows)).astype(np.float32)
    weight = (rng.random(rows) / rows).astype(np.float32) if weighted else None
    kl32 = float(np.float32(kl))
    want, d_want, total, d_total, coef, d_coef = lm.policy(R, old, adv, lo, hi, ref, kl32, weight)
    nan = np.where(R.has, 0.0, np.nan).astype(np.float32)
    dev = lambda a: None if a is None else torch.from_numpy(a + nan).cuda()  # noqa: E731
    args = (x, dl, dev(old), dev(adv), 0.2, 0.28)
    kw = dict(ref_logp=dev(ref) if kl else None, kl=kl, weight=dev(weight))
    t, tokens, logp, grad = b.ef21_policy_loss(*args, **kw)
    lm.inside(as64(tokens), want, d_want, "token loss")
    lm.inside(as64(t), np.array([total]), np.array([d_total]), "loss")
    lm.inside(as64(logp), R.logp, R.d_logp, "logp")
    g, bound = R.grad(coef, d_coef, dtype)
    lm.inside(as64(grad), g, bound, "gradient")
    t2, tokens2, logp2, none = b.ef21_policy_loss(*args, **kw, grad=False)
    assert none is None and torch.equal(t2, t) and torch.equal(tokens2, tokens) and torch.equal(logp2, logp)
    b.ef21_policy_loss(*args, **kw, grad=x)
    assert torch.equal(x, grad), "over the logits the gradient is the same"


def test_policy_loss_on_the_policy_that_sampled(gpu):
    """old_logp as the library itself gave it: the ratio is exactly one, nothing is clipped, and with clip ranges of zero the tie goes to q A."""
    torch, b = gpu
    x, _ = make_logits(torch, 50, 777, "f32", seed=1)
    labels, dl = make_labels(torch, 50, 777, seed=2, ignored=0.0)
    logp, lse = b.ef21_token_logps(x, dl)
    adv = torch.randn(50, device="cuda")
    t, tokens, logp2, grad = b.ef21_policy_loss(x, dl, logp, adv, 0.0, 0.0)
    assert torch.equal(logp2, logp) and torch.equal(tokens, -adv)
    want = b.ef21_token_logps_grad(x, dl, lse, -adv * (1.0 / 50))
    assert torch.allclose(grad, want, rtol=1e-5, atol=1e-9)


@pytest.mark.parametrize("which", ["logps", "preference", "least_squares", "policy"])
def test_gradients_against_differences(gpu, which):
    """Central differences of the 64-bit loss, step 1e-5: error below 1e-9, far below the allowed 2e-6 of the largest entry."""
    torch, b = gpu
    rows, vocab = 6, 5
    x, x64 = make_logits(torch, rows, vocab, "f32", seed=8, spread=1.0)
    labels = np.array([0, 4, -100, 2, 1, 3])
    dl = torch.from_numpy(labels).cuda()
    start = np.array([0, 3, 6])
    rng = np.random.default_rng(2)
    base = lm.Rows(x64, labels).logp
    ref = (base + 0.3 * rng.standard_normal(rows)).astype(np.float32)
    old = away_from_edges(base, rng, rows, 0.2, 0.2)
    adv = rng.standard_normal(rows).astype(np.float32)
    coef = rng.standard_normal(rows).astype(np.float32)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    f = lambda a: a.astype(np.float64)  # noqa: E731

    def value(y):
        R = lm.Rows(y, labels)
        if which == "logps":
            return float(np.sum(f(coef) * R.logp))
        if which in ("preference", "least_squares"):
            return float(np.mean(lm.preference(R, start, f(ref), 0.5, 0.0 if which == "least_squares" else 0.25, which == "least_squares", True, None)[0]))
        return float(lm.policy(R, old, adv, 0.2, 0.2, ref, 0.5, None)[2])

    if which == "logps":
        grad = b.ef21_token_logps_grad(x, dl, b.ef21_token_logps(x, dl)[1], dev(coef))
    elif which == "policy":
        grad = b.ef21_policy_loss(x, dl, dev(old), dev(adv), 0.2, 0.2, ref_logp=dev(ref), kl=0.5)[3]
    else:
        grad = b.ef21_preference_loss(x, dl, dev(start), dev(ref), 0.5, smoothing=0.0 if which == "least_squares" else 0.25,
                                      loss=1 if which == "least_squares" else 0, mean=True)[2]
    numeric, h = np.zeros((rows, vocab)), 1e-5
    for r in range(rows):
        for v in range(vocab):
            up, down = x64.copy(), x64.copy()
            up[r, v] += h
            down[r, v] -= h
            numeric[r, v] = (value(up) - value(down)) / (2 * h)
    assert np.max(np.abs(as64(grad) - numeric)) <= 2e-6 * max(1.0, np.max(np.abs(numeric)))


def test_rows_beyond_32_bits(gpu):
    """Rows 2^30 entries apart: the last one starts at entry 2^32 and beyond."""
    torch, b = gpu
    rows, vocab, stride = 5, 1111, 1 << 30
    buf = torch.empty(4 * stride + vocab, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, vocab), (stride, 1))
    small, x64 = make_logits(torch, rows, vocab, "bf16", seed=6)
    x.copy_(small)
    labels, dl = make_labels(torch, rows, vocab, seed=7, ignored=0.0)
    R = lm.Rows(x64, labels)
    logp, lse = b.ef21_token_logps(x, dl)
    lm.inside(as64(logp), R.logp, R.d_logp, "logp")
    one = torch.ones(rows, device="cuda")
    want = b.ef21_token_logps_grad(small, dl, lse, one)
    b.ef21_token_logps_grad(x, dl, lse, one, out=x)
    assert torch.equal(x, want)
    x.copy_(small)
    b.ef21_policy_loss(x, dl, logp, one, 0.2, 0.2, weight=one, grad=x)
    assert torch.equal(x, -want)


def test_many_rows_no_rows_and_repeats(gpu):
    torch, b = gpu
    x, x64 = make_logits(torch, 3000, 90, "f16", seed=12)
    labels, dl = make_labels(torch, 3000, 90, seed=12)
    R = lm.Rows(x64, labels)
    logp, lse = b.ef21_token_logps(x, dl)
    lm.inside(as64(logp), R.logp, R.d_logp, "logp")
    again = b.ef21_token_logps(x, dl)
    assert torch.equal(again[0], logp) and torch.equal(again[1], lse)
    none, nl = x[:0], dl[:0]
    e = torch.empty(0, device="cuda")
    assert b.ef21_token_logps(none, nl)[0].numel() == 0
    assert b.ef21_token_logps_grad(none, nl, e, e).shape == (0, 90)
    loss, _, grad = b.ef21_preference_loss(none, nl, torch.zeros(3, dtype=torch.int64, device="cuda"), e, 1.0)
    assert float(loss) == pytest.approx(math.log(2.0), rel=1e-6) and grad.numel() == 0
    assert float(b.ef21_policy_loss(none, nl, e, e, 0.2, 0.2)[0]) == 0.0


def test_offsets_out_of_range_are_not_followed(gpu):
    torch, b = gpu
    x, _ = make_logits(torch, 8, 50, "f32", seed=1)
    labels, dl = make_labels(torch, 8, 50, seed=1, ignored=0.0)
    ref = torch.zeros(8, device="cuda")
    for start in ([0, 4, 1 << 40], [-5, 3, 8], [6, 2, 8]):
        loss, _, _ = b.ef21_preference_loss(x, dl, torch.tensor(start, device="cuda"), ref, 0.1)
        assert bool(torch.isfinite(loss).all())


def test_another_stream_and_a_graph(gpu):
    """The calls go to the current stream, and replays of a captured graph see what their buffers hold then."""
    torch, b = gpu
    rows, vocab = 40, 5003
    x, _ = make_logits(torch, rows, vocab, "bf16", seed=21)
    labels, dl = make_labels(torch, rows, vocab, seed=21)
    ref, adv = torch.full((rows,), -8.0, device="cuda"), torch.randn(rows, device="cuda")
    start = torch.tensor([0, 10, 25, 30, 40], device="cuda")
    bufs = dict(l1=torch.empty(2, device="cuda"), l2=torch.empty(1, device="cuda"), t=torch.empty(rows, device="cuda"),
                p1=torch.empty(rows, device="cuda"), p2=torch.empty(rows, device="cuda"), g1=torch.empty_like(x), g2=torch.empty_like(x),
                ws=torch.empty(b.ef21_preference_loss_workspace(rows, 2), dtype=torch.uint8, device="cuda"),
                ws2=torch.empty(b.ef21_policy_loss_workspace(rows), dtype=torch.uint8, device="cuda"))

    def calls():
        b.ef21_preference_loss(x, dl, start, ref, 0.1, out_loss=bufs["l1"], logp=bufs["p1"], grad=bufs["g1"], workspace=bufs["ws"])
        b.ef21_policy_loss(x, dl, ref, adv, 0.2, 0.2, ref_logp=ref, kl=0.1, out_loss=bufs["l2"], token_loss=bufs["t"], logp=bufs["p2"], grad=bufs["g2"], workspace=bufs["ws2"])

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for seed in (31, 32, 33):
        x.copy_(make_logits(torch, rows, vocab, "bf16", seed=seed)[0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in bufs.items() if not k.startswith("ws")}
        l1, p1, g1 = b.ef21_preference_loss(x, dl, start, ref, 0.1)
        l2, t, p2, g2 = b.ef21_policy_loss(x, dl, ref, adv, 0.2, 0.2, ref_logp=ref, kl=0.1)
        for k, v in dict(l1=l1, l2=l2, t=t, p1=p1, p2=p2, g1=g1, g2=g2).items():
            assert torch.equal(got[k], v), f"replay {seed}: {k} differs"


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [70, 1500, 9001, 40000, 70001, 200000])
def test_rows_of_every_size_and_spread(gpu, vocab, dtype):
    """Rows far from zero, rows whose entries lie hundreds apart, rows that begin with masks: sums that leave fp32's range unless they are
    taken relative to the row's maximum."""
    torch, b = gpu
    print(f"spread vocab={vocab} {dtype}", flush=True)
    rng = np.random.default_rng(vocab)
    base = rng.standard_normal(vocab)
    half = np.arange(vocab) < vocab // 2
    kinds = [40 * base, 300 * base, 1000 + base, -300 + 2 * base, -6000 + base, 20000 + 40 * base, np.where(half, -10000.0, base), np.where(half, -30000.0, 3 * base),
             np.where(half, base, 900 + base), np.where(half[::-1], -60000.0, -100 + base), np.where(np.arange(vocab) == vocab - 2, 500.0, base)]
    if dtype != "f16":
        kinds += [1e6 + 100 * base, -2.8e6 + 1e4 * base, 3.5e6 + 1e5 * base, -5e6 + base, 1e9 * base, 1e20 * base, -1e30 + 0 * base, 1e37 * base, -2.5e38 + 0 * base]
    x = torch.from_numpy(np.stack(kinds)).to(lm.TORCH[dtype]).cuda()
    x64 = as64(x)
    rows = len(kinds)
    labels = rng.integers(0, vocab, rows)
    labels[::3] = np.argmax(x64, axis=1)[::3]
    dl = torch.from_numpy(labels).cuda()
    R = lm.Rows(x64, labels)
    logp, lse = b.ef21_token_logps(x, dl)
    lm.inside(as64(lse), R.lse, R.d_lse, "lse")
    lm.inside(as64(logp), R.logp, R.d_logp, "logp")
    one = torch.ones(rows, device="cuda")
    g, bound = R.grad(np.ones(rows), np.zeros(rows), dtype)
    lm.inside(as64(b.ef21_token_logps_grad(x, dl, lse, one)), g, bound, "gradient")
    # one sequence a row, empty ones beside them: the gradient of row r is -w_r times that of logp
    start = torch.arange(rows + 1, device="cuda").repeat_interleave(2)[1:]
    ref = logp.clone()
    _, logp2, grad2 = b.ef21_preference_loss(x, dl, start, ref, 1.0, pair_weight=one * 2)
    assert torch.equal(logp2, logp)
    ratio = np.where(np.isfinite(as64(logp)), 1.0, np.nan)
    keep = np.isfinite(ratio)
    # beta 1, margin 0: the slope of the loss is -1/2, twice that -1; its own error is the margin's over 4
    lm.inside(as64(grad2)[keep], -g[keep], bound[keep] + (np.abs(R.grad(np.ones(rows), np.ones(rows), "f32")[0]) * 1e-7)[keep], "preference gradient")
    total, tokens, logp3, grad3 = b.ef21_policy_loss(x, dl, logp, one, 0.2, 0.2, weight=one)
    assert torch.equal(logp3, logp)
    lm.inside(as64(grad3)[keep], -g[keep], bound[keep] + (np.abs(g) * 1e-7)[keep], "policy gradient")
    over = x.clone()
    b.ef21_token_logps_grad(over, dl, lse, one, out=over)
    lm.inside(as64(over), g, bound, "gradient over the logits")


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
def test_preference_of_impossible_tokens(gpu, smoothing):
    """A reply with a token of probability zero: the margin is infinite, and the loss and its gradient have their limits; margins at which the sigmoid is within
    an ulp of one keep their slope."""
    torch, b = gpu
    vocab, far = 40, 34.0
    x = torch.zeros(6, vocab, device="cuda")
    labels = torch.tensor([3, 4, 5, 6, 7, 8], device="cuda")
    x[1, 4] = -math.inf                                                # pair 0: the other reply is impossible, pair 1: the preferred one
    x[2, 5] = -math.inf
    ref = torch.full((6,), -math.log(vocab), device="cuda")
    ref[1], ref[2] = -4.0, -4.0
    ref[5] += far                                                      # pair 2: a margin of `far`
    starts = torch.arange(7, device="cuda")
    loss, logp, grad = b.ef21_preference_loss(x, labels, starts, ref, 1.0, smoothing=smoothing, pair_weight=torch.ones(3, device="cuda"))
    want = [math.inf if smoothing else 0.0, math.inf, math.log1p(math.exp(-far)) + smoothing * far]
    assert logp.tolist()[1] == -math.inf and logp.tolist()[2] == -math.inf
    slope = [smoothing, smoothing - 1.0, smoothing - 1.0 / (1.0 + math.exp(far))]
    for p in range(3):
        assert loss[p].item() == pytest.approx(want[p], rel=1e-5)
        for row, sign in ((2 * p, 1.0), (2 * p + 1, -1.0)):
            prob = torch.softmax(x[row].double(), 0)
            hot = torch.zeros(vocab, device="cuda", dtype=torch.float64)
            hot[labels[row]] = 1.0
            expect = sign * slope[p] * (hot - prob)
            assert float((grad[row].double() - expect).abs().max()) <= 1e-5 * abs(slope[p])
