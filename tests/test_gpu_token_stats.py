"""Entropy, most likely tokens and log-probabilities of rows of logits, and their gradient, against a plain implementation in 64 bits
(tests/stats_reference.py, where the bounds are derived)."""
import math

import numpy as np
import pytest

import lm_reference as lm
import stats_reference as ref
from test_gpu_token_losses import as64, make_labels, make_logits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2106_05203_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load_library()
    return torch, binding


def check(torch, st, R, k, wrong=()):
    """All of st against R; rows in `wrong` have NaN."""
    keep = np.array([r for r in range(len(R.x)) if r not in wrong], dtype=np.int64)
    lm.inside(as64(st.lse)[keep], R.lse[keep], R.d_lse[keep], "lse")
    lm.inside(as64(st.entropy)[keep], R.entropy[keep], R.d_entropy[keep], "entropy")
    if R.labelled:
        lm.inside(as64(st.logp)[keep], R.logp[keep], R.d_logp[keep], "logp")
    else:
        assert st.logp is None
    if k:
        tokens, logp, bound = R.top(k)
        assert st.top_tokens.dtype == torch.int32 and np.array_equal(st.top_tokens.cpu().numpy()[keep], tokens[keep]), "top tokens"
        lm.inside(as64(st.top_logp)[keep], logp[keep], bound[keep], "top_logp")
    for r in wrong:
        for t in (st.lse, st.entropy) + ((st.logp,) if R.labelled else ()) + ((st.top_logp,) if k else ()):
            assert bool(torch.isnan(t[r]).all())
        assert not k or bool((st.top_tokens[r] == -1).all())


# rows, vocab, stride, offset: around the vector and slice widths, one entry, odd vocabularies, rows that start anywhere
SHAPES = [(1, 1, 1, 0), (3, 2, 2, 1), (5, 7, 9, 3), (4, 63, 63, 0), (9, 65, 67, 5), (2, 255, 255, 0), (7, 1000, 1000, 0), (3, 2047, 2049, 1), (2, 2048, 2048, 0),
          (2, 4096, 4104, 0), (3, 4097, 4099, 1), (3, 5001, 5001, 2), (2, 8193, 8195, 3), (2, 16384, 16384, 0), (1, 65536, 65536, 0), (2, 70003, 70010, 7),
          (1, 131072, 131072, 0), (1, 300001, 300001, 3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,stride,offset", SHAPES)
def test_stats_and_gradient(gpu, rows, vocab, stride, offset, dtype):
    torch, b = gpu
    print(f"stats rows={rows} vocab={vocab} stride={stride} offset={offset} {dtype}", flush=True)
    x, x64 = make_logits(torch, rows, vocab, dtype, seed=rows * 7 + vocab, stride=stride, offset=offset)
    labels, dl = make_labels(torch, rows, vocab, seed=vocab, wide=vocab % 2 == 0)
    R = ref.Stats(x64, labels)
    rng = np.random.default_rng(5)
    a, c = (rng.standard_normal(rows).astype(np.float32) for _ in range(2))
    da, dc = torch.from_numpy(a).cuda(), torch.from_numpy(c).cuda()
    for k in sorted({0, 1, min(vocab, 20), min(vocab, 64)}):
        st = b.ef21_token_stats(x, dl, k, sums=True)
        check(torch, st, R, k)
    bare = b.ef21_token_stats(x, None, min(vocab, 5))
    check(torch, bare, ref.Stats(x64), min(vocab, 5))
    assert bare.sums is None
    grad = b.ef21_token_stats_grad(x, dl, st.sums, st.entropy, da, dc)
    lm.inside(as64(grad), *R.stats_grad(a, c, dtype), "gradient")
    lm.inside(as64(b.ef21_token_stats_grad(x, dl, st.sums, st.entropy, da)), *R.stats_grad(a, None, dtype), "gradient by logp alone")
    lm.inside(as64(b.ef21_token_stats_grad(x, dl, st.sums, st.entropy, None, dc)), *R.stats_grad(None, c, dtype), "gradient by entropy alone")
    # another stride and start than the logits; added to what is there
    other = torch.full((rows * (vocab + 3) + 1,), 7.0, dtype=x.dtype, device="cuda")
    to = other[1:].as_strided((rows, vocab), (vocab + 3, 1))
    b.ef21_token_stats_grad(x, dl, st.sums, st.entropy, da, dc, out=to)
    assert torch.equal(to, grad)
    base = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32)).to(x.dtype).cuda()
    to.copy_(base)
    b.ef21_token_stats_grad(x, dl, st.sums, st.entropy, da, dc, out=to, accumulate=True)
    lm.inside(as64(to), *R.stats_grad(a, c, dtype, base=as64(base)), "accumulated")
    gaps = other[1:].as_strided((rows, 3), (vocab + 3, 1), 1 + vocab)[: rows - 1]
    assert bool((gaps == 7.0).all()) and float(other[0]) == 7.0, "entries beside the rows were written"
    # without labels, and over the logits
    all_rows = b.ef21_token_stats(x, None, 0, sums=True) if not np.isnan(x64).any() else None
    if all_rows is not None:
        lm.inside(as64(b.ef21_token_stats_grad(x, None, all_rows.sums, all_rows.entropy, None, dc)), *ref.Stats(x64).stats_grad(None, c, dtype), "no labels")
    b.ef21_token_stats_grad(x, dl, st.sums, st.entropy, da, dc, out=x)
    assert torch.equal(x, grad)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [5, 130, 1500, 20000, 90000])
def test_masked_entries_and_odd_rows(gpu, vocab, dtype):
    torch, b = gpu
    print(f"masks vocab={vocab} {dtype}", flush=True)
    rows = 14
    x, x64 = make_logits(torch, rows, vocab, dtype, seed=vocab)
    labels = np.array([1, vocab - 1, 0, 2, 3, -100, vocab, 4, -1, 0, 1, vocab - 1, 3, 4], dtype=np.int64)
    low, most = torch.finfo(x.dtype).min, torch.finfo(x.dtype).max

    def put(r, at, value):
        x[r, at] = value
        x64[r, at] = float(torch.tensor(value, dtype=x.dtype))

    put(0, slice(vocab // 2, None), -math.inf)                         # masked behind the middle
    put(1, slice(None, -1), -math.inf)                                 # the label alone is left
    put(2, slice(None), -math.inf)                                     # nothing is left
    put(3, slice(None), low)                                           # the type's lowest value everywhere
    put(4, slice(1, 3), low)
    x[5] = math.nan; x[6] = math.nan; x[8] = math.inf                  # rows without a label are not read
    put(7, 4, -math.inf)                                               # the label itself has probability zero
    put(9, slice(None), 0.25)                                          # all alike
    put(10, slice(None, None, 2), -0.0); put(10, slice(1, None, 2), 0.0)   # zeros of both signs are alike
    put(11, slice(None), low); put(11, vocab - 1, most)                # as far apart as the type goes
    x[12, vocab // 2] = math.nan; x[13, vocab - 1] = math.inf          # results are NaN
    x64[[5, 6, 8, 12, 13]] = 0.0
    k = min(vocab, 33)
    dl = torch.from_numpy(labels).cuda()
    R = ref.Stats(x64, labels)
    R.x[10] = 0.0
    st = b.ef21_token_stats(x, dl, k, sums=True)
    check(torch, st, R, k, wrong=(12, 13))
    # (of one entry that is left it is zero up to the bound: log2 s and t / s are each rounded)
    assert float(st.entropy[2]) == 0.0 and not bool((st.entropy[:12] < 0).any())
    a, c = np.linspace(-1, 1, rows).astype(np.float32), np.linspace(2, -1, rows).astype(np.float32)
    grad = b.ef21_token_stats_grad(x, dl, st.sums, st.entropy, torch.from_numpy(a).cuda(), torch.from_numpy(c).cuda())
    g, bound = R.stats_grad(a, c, dtype)
    lm.inside(as64(grad)[:12], g[:12], bound[:12], "gradient")
    assert bool(torch.isnan(grad[12:].float()).all())
    for r in (2, 5, 6, 8):
        assert not bool(grad[r].count_nonzero()), "a row without a distribution has no gradient"
    # added to a gradient: rows that are ignored or empty stay as they are
    marked = torch.full_like(x, 3.0)
    b.ef21_token_stats_grad(x, dl, st.sums, st.entropy, torch.from_numpy(a).cuda(), torch.from_numpy(c).cuda(), out=marked, accumulate=True)
    for r in (2, 5, 6, 8):
        assert bool((marked[r] == 3.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [3e6, -3e6, 2.89e6, 1e30, -1e30, 2000.0, -300.0])
def test_large_logits(gpu, offset, dtype):
    """Rows around a large number; in fp32 at 3e6 neighbours are 1/4 apart, at 1e30 they are all one number or infinitely far."""
    torch, b = gpu
    x, _ = make_logits(torch, 4, 9001, "f32", seed=3)
    x = (x.double() * 4 + offset).float().to(lm.TORCH[dtype])
    x64 = as64(x)
    labels = np.array([5, 9000, 0, 77])
    R = ref.Stats(x64, labels)
    st = b.ef21_token_stats(x, torch.from_numpy(labels).cuda(), 10, sums=True)
    check(torch, st, R, 10)
    c = np.ones(4, np.float32)
    grad = b.ef21_token_stats_grad(x, torch.from_numpy(labels).cuda(), st.sums, st.entropy, torch.from_numpy(c).cuda(), torch.from_numpy(c).cuda())
    lm.inside(as64(grad), *R.stats_grad(c, c, dtype), "gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [600, 9000, 70000])
def test_lowest_entries_beside_masked_ones(gpu, vocab, dtype):
    """Tiles of nothing beside tiles of the type's lowest value, or of its largest: M of the one is infinitely far from that of the other."""
    torch, b = gpu
    low, most = torch.finfo(lm.TORCH[dtype]).min, torch.finfo(lm.TORCH[dtype]).max
    x = torch.full((4, vocab), -math.inf, dtype=lm.TORCH[dtype])
    x[0, vocab // 2:] = low
    x[1, : vocab // 3] = low
    x[2, vocab // 2:] = most
    x[3, ::1000] = low
    R = ref.Stats(x.double().numpy(), np.array([vocab - 1, 0, vocab - 1, 0]))
    labels = torch.tensor([vocab - 1, 0, vocab - 1, 0], device="cuda")
    dx, one = x.cuda(), torch.ones(4, device="cuda")
    st = b.ef21_token_stats(dx, labels, 5, sums=True)
    check(torch, st, R, 5)
    lm.inside(as64(b.ef21_token_stats_grad(dx, labels, st.sums, st.entropy, one, one)), *R.stats_grad(np.ones(4), np.ones(4), dtype), "gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("order", ["up", "down", "sawtooth", "ties", "late", "blocks", "masked", "few", "alike"])
@pytest.mark.parametrize("rows,vocab", [(2, 50001), (300, 20003)])
def test_orders_that_are_hard_to_select_from(gpu, rows, vocab, order, dtype):
    torch, b = gpu
    print(f"order {order} rows={rows} vocab={vocab} {dtype}", flush=True)
    v = np.arange(vocab)
    row = {"up": v / vocab * 20, "down": -v / vocab * 20, "sawtooth": (v % 4096) / 4096 * 20, "ties": (v * 7919 % 13).astype(float),
           "late": np.where(v >= vocab - 70, 3.0 + (v % 9), -5.0 + (v % 3)), "blocks": ((v // 8) % 64 == 3) * 4.0 + (v // 512 % 3),
           "masked": np.where(v * 7919 % 997 < 3, (v % 31) / 4, -np.inf), "few": np.where(v % 9973 == 5, v / vocab, -np.inf), "alike": np.full(vocab, -3.25)}[order]
    x = torch.from_numpy(np.tile(row, (rows, 1)).astype(np.float32)).to(lm.TORCH[dtype])
    x = torch.roll(x, 1, 1) if rows > 2 else x
    R = ref.Stats(x.double().numpy()[:2])
    alike = torch.zeros(rows, -(-vocab // 8) * 8, dtype=x.dtype, device="cuda")[:, :vocab]   # rows of one alignment
    alike.copy_(x)
    for k in (1, 20, 64):
        check(torch, b.ef21_token_stats(x[:2].cuda(), None, k), R, k)
        st = b.ef21_token_stats(alike, None, k)
        check(torch, b.TokenStats(None, st.lse[:2], st.entropy[:2], st.top_tokens[:2], st.top_logp[:2], None), R, k)
        assert bool((st.top_tokens == st.top_tokens[0]).all()) and bool((st.entropy == st.entropy[0]).all())


@pytest.mark.parametrize("dtype,vocab", [("bf16", 131072), ("f16", 50001), ("f32", 32064), ("bf16", 1000)])
def test_a_row_does_not_depend_on_the_others(gpu, dtype, vocab):
    """The same bits for a row alone, among a few and among many."""
    torch, b = gpu
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn(1030, -(-vocab // 8) * 8, generator=g, device="cuda").mul_(3).to(lm.TORCH[dtype])[:, :vocab]
    labels = torch.randint(0, vocab, (1030,), generator=g, device="cuda")
    many = b.ef21_token_stats(x, labels, 7, sums=True)
    for some in (slice(0, 1), slice(5, 22), slice(700, 1000)):
        few = b.ef21_token_stats(x[some], labels[some], 7, sums=True)
        for one, other in zip(few, many):
            assert torch.equal(one, other[some])
        coef = torch.randn(1030, generator=g, device="cuda")
        whole = b.ef21_token_stats_grad(x, labels, many.sums, many.entropy, coef, coef)
        assert torch.equal(b.ef21_token_stats_grad(x[some], labels[some], few.sums, few.entropy, coef[some], coef[some]), whole[some])


def test_long_vocabularies(gpu):
    torch, b = gpu
    for rows, vocab, dtype in ((1, 5_000_011, "bf16"), (2, 1_200_003, "f32"), (1, 12_000_001, "f16")):
        print(f"long vocab={vocab} {dtype}", flush=True)
        x, x64 = make_logits(torch, rows, vocab, dtype, seed=vocab % 1000)
        R = ref.Stats(x64)
        check(torch, b.ef21_token_stats(x, None, 64), R, 64)


def test_gradient_against_differences(gpu):
    """The formula itself: central differences in 64 bits of sum a logp + b H."""
    torch, b = gpu
    x, x64 = make_logits(torch, 3, 41, "f32", seed=9)
    labels = np.array([3, 40, 0])
    rng = np.random.default_rng(0)
    a, c = rng.standard_normal(3).astype(np.float32), rng.standard_normal(3).astype(np.float32)
    dl = torch.from_numpy(labels).cuda()
    st = b.ef21_token_stats(x, dl, 0, sums=True)
    grad = as64(b.ef21_token_stats_grad(x, dl, st.sums, st.entropy, torch.from_numpy(a).cuda(), torch.from_numpy(c).cuda()))
    f = lambda y: float((a * ref.Stats(y, labels).logp + c * ref.Stats(y, labels).entropy).sum())  # noqa: E731
    for r, v in [(0, 3), (0, 7), (1, 40), (1, 0), (2, 0), (2, 20)]:
        up, down = x64.copy(), x64.copy()
        up[r, v] += 1e-5
        down[r, v] -= 1e-5
        assert abs((f(up) - f(down)) / 2e-5 - grad[r, v]) < 1e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [3, 700, 9000])
def test_rows_of_nan(gpu, vocab, dtype):
    """NaN everywhere, of both kinds (a signalling one comes out of some instructions where a quiet one does not), and one beside numbers."""
    torch, b = gpu
    whole = {"f32": (torch.int32, 0x7F800001), "bf16": (torch.int16, 0x7F81), "f16": (torch.int16, 0x7C01)}[dtype]
    x = torch.randn(4, vocab, device="cuda").to(lm.TORCH[dtype])
    x[0] = math.nan
    x[1:3].view(whole[0])[0] = whole[1]
    x[2:3].view(whole[0])[0, vocab // 2] = whole[1]
    st = b.ef21_token_stats(x, torch.zeros(4, dtype=torch.int64, device="cuda"), 2, sums=True)
    for r in range(3):
        assert all(bool(torch.isnan(t[r]).all()) for t in (st.logp, st.lse, st.entropy, st.top_logp)) and bool((st.top_tokens[r] == -1).all())
    check(torch, b.TokenStats(st.logp[3:], st.lse[3:], st.entropy[3:], st.top_tokens[3:], st.top_logp[3:], None), ref.Stats(as64(x[3:]), np.array([0])), 2)


def test_nothing_to_do_and_rows_that_are_all_ignored(gpu):
    torch, b = gpu
    x = torch.empty(0, 50, device="cuda")
    st = b.ef21_token_stats(x, torch.empty(0, dtype=torch.int64, device="cuda"), 3, sums=True)
    assert st.top_tokens.shape == (0, 3) and b.ef21_token_stats_grad(x, None, st.sums, st.entropy).shape == (0, 50)
    x = torch.full((5, 6000), math.nan, device="cuda")
    labels = torch.full((5,), -100, device="cuda")
    st = b.ef21_token_stats(x, labels, 2, sums=True)
    assert all(not bool(t.count_nonzero()) for t in (st.logp, st.lse, st.entropy, st.top_logp)) and bool((st.top_tokens == -1).all())
    assert not bool(b.ef21_token_stats_grad(x, labels, st.sums, st.entropy, st.logp, st.logp).count_nonzero())


@pytest.mark.parametrize("rows", [2, 700])
def test_streams_and_graphs(gpu, rows):
    """On a side stream; captured, and replayed on new contents with eager work in between; two graphs that share one workspace."""
    torch, b = gpu
    vocab, k = 30001, 9
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, vocab, generator=g, device="cuda").to(torch.bfloat16)
    labels = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    coef = torch.randn(rows, generator=g, device="cuda")
    space = torch.empty(max(1, b.ef21_token_stats_workspace(1, rows, vocab, k)), dtype=torch.uint8, device="cuda")
    new = lambda: (b.TokenStats(*(torch.zeros(rows, device="cuda") for _ in range(3)), torch.zeros(rows, k, dtype=torch.int32, device="cuda"),  # noqa: E731
                                torch.zeros(rows, k, device="cuda"), torch.zeros(rows, 2, device="cuda")), torch.zeros_like(x))

    def call(to):
        st, grad = to
        b.ef21_token_stats(x, labels, k, *st[:5], sums=st.sums, workspace=space)
        b.ef21_token_stats_grad(x, labels, st.sums, st.entropy, coef, coef, out=grad)

    eager, outs, graphs, side = new(), [new(), new()], [], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(eager)
    side.synchronize()
    for to in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(to)
        graphs.append(graph)
    for turn in range(3):
        x.copy_(torch.randn(rows, vocab, generator=g, device="cuda"))
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        call(eager)
        torch.cuda.synchronize()
        for to in outs:
            for one, other in zip((*to[0], to[1]), (*eager[0], eager[1])):
                assert torch.equal(one, other)


def test_offsets_beyond_32_bits(gpu):
    torch, b = gpu
    rows, vocab = 70, 32000
    stride = 2 ** 31 // 64 + 8                                         # the last rows lie beyond 2^31 entries
    buf = torch.zeros((rows - 1) * stride + vocab, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, vocab), (stride, 1))
    small = torch.randn(rows, vocab, device="cuda").to(torch.bfloat16)
    x.copy_(small)
    labels = torch.arange(rows, device="cuda")
    one, two = b.ef21_token_stats(x, labels, 4, sums=True), b.ef21_token_stats(small, labels, 4, sums=True)
    for p, q in zip(one, two):
        assert torch.equal(p, q)
    coef = torch.ones(rows, device="cuda")
    want = b.ef21_token_stats_grad(small, labels, two.sums, two.entropy, coef, coef)
    assert torch.equal(b.ef21_token_stats_grad(x, labels, one.sums, one.entropy, coef, coef, out=x), want)
