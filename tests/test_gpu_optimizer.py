"""AdamW over many tensors and the norm of their gradients against plain implementations in 64 bits (tests/stats_reference.py, where the bounds are
derived).  8-bit codes and stochastically rounded numbers have to lie between the roundings of the two ends of the bound, by the same random bits."""
import ctypes as C
import math
import threading

import numpy as np
import pytest

import lm_reference as lm
import stats_reference as ref
from lm_reference import U

pytestmark = pytest.mark.gpu
BETAS, EPS = (0.9, 0.999), 1e-8


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2106_05203_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load_library()
    return torch, binding


def as64(t):
    return t.detach().float().double().cpu().numpy() if t.dtype.itemsize == 1 else t.detach().double().cpu().numpy()


class Guarded:
    """A tensor of n entries `offset` entries into memory whose other entries are known, to see that they stay."""

    def __init__(self, torch, values, dtype, offset=0):
        n = len(values)
        self.fill = 3.0
        self.buf = torch.full((n + offset + 64,), self.fill).to(dtype)
        self.buf[offset:offset + n] = torch.from_numpy(np.asarray(values, np.float32)).to(dtype)
        self.buf = self.buf.cuda()
        self.at, self.n = offset, n
        self.t = self.buf[offset:offset + n]

    def untouched(self):
        rest = self.buf.float()
        return bool((rest[:self.at] == self.fill).all()) and bool((rest[self.at + self.n:] == self.fill).all())


def make(torch, n, param, grad, eight, seed, offset=0, size=1e-3, copy=None):
    """Tensors of one parameter with states that an earlier step could have left, and guards around each."""
    rng = np.random.default_rng(seed)
    x = {"p": Guarded(torch, rng.standard_normal(n) * 0.02, lm.TORCH[param], offset), "g": Guarded(torch, rng.standard_normal(n) * size, lm.TORCH[grad], offset)}
    m, root = rng.standard_normal(n) * 0.3 * size, np.sqrt(rng.standard_normal(n) ** 2 + 0.2) * size
    if n > 5:
        m[2:4], root[3:5] = 0.0, 0.0
    if eight:
        for name, v in (("m", m), ("v", root)):
            scale = np.float32(np.maximum(ref.per_block(v, lambda w: np.abs(w).max(axis=1)) / 448.0, 2.0 ** -126)) if n else np.zeros(0, np.float32)
            x[name] = Guarded(torch, ref.rounded(v / ref.spread(scale.astype(np.float64), n), "e4m3").clip(-448, 448), torch.float8_e4m3fn, offset)
            x[name + "_scale"] = Guarded(torch, scale, torch.float32, offset)
    else:
        x["m"], x["v"] = Guarded(torch, m, torch.float32, offset), Guarded(torch, root ** 2, torch.float32, offset)
    if copy:
        x["copy"] = Guarded(torch, np.zeros(n), lm.TORCH[copy], offset)
    return x


def states(x, name):
    """m, or v (32 bits) or sqrt(v) (8 bits), as stored."""
    v = as64(x[name].t)
    return v * ref.spread(as64(x[name + "_scale"].t), len(v)) if name + "_scale" in x else v


def expected(x, decay, step, factor=1.0, lr=1e-3, on_device=False):
    return ref.Adamw(as64(x["p"].t), as64(x["g"].t), states(x, "m"), states(x, "v"), lr, BETAS, EPS, decay, step, factor, "m_scale" in x, on_device)


def compare(x, want, param, copy, bits, what):
    """bits: the random bits of the tensor's entries, or None."""
    for_m, for_v, for_p = bits if bits is not None else (None, None, None)
    ref.between(as64(x["p"].t), *want.params(param, for_p), what + " parameters")
    if copy:
        ref.between(as64(x["copy"].t), ref.rounded(want.p - want.d_p, copy), ref.rounded(want.p + want.d_p, copy), what + " copy")
    if "m_scale" in x:
        for name, (low, high, scale, d_scale) in want.codes(for_m, for_v).items():
            ref.between(as64(x[name + "_scale"].t), scale - d_scale, scale + d_scale, f"{what} {name}_scale")
            ref.between(as64(x[name].t), low, high, f"{what} {name}")
    else:
        ref.between(as64(x["m"].t), want.m - want.d_m, want.m + want.d_m, what + " m")
        ref.between(as64(x["v"].t), want.v - want.d_v, want.v + want.d_v, what + " v")
    for name, part in x.items():
        assert part.untouched(), f"{what}: entries beside {name} were written"


def optimizer(b, xs, eight, decays, stochastic=False, seed=0, copy=None):
    pick = lambda name: [x[name].t for x in xs]  # noqa: E731
    more = dict(m_scale=pick("m_scale"), v_scale=pick("v_scale")) if eight else {}
    return b.AdamW(pick("p"), pick("g"), betas=BETAS, eps=EPS, weight_decay=decays, bits=8 if eight else 32, m=pick("m"), v=pick("v"),
                   copies=pick("copy") if copy else None, stochastic=stochastic, seed=seed, **more)


# around the vector, block and workgroup sizes
SIZES = [0, 1, 3, 4, 17, 255, 256, 257, 1000, 1023, 4096, 4097, 16385, 70001]


@pytest.mark.parametrize("eight,stochastic", [(False, False), (True, False), (True, True), (False, True)])
@pytest.mark.parametrize("param,copy", [("f32", None), ("f32", "bf16"), ("f32", "f16"), ("bf16", None), ("f16", None)])
@pytest.mark.parametrize("grad", ["f32", "bf16", "f16"])
def test_one_step(gpu, grad, param, copy, eight, stochastic):
    torch, b = gpu
    print(f"adamw param={param} copy={copy} grad={grad} eight={eight} stochastic={stochastic}", flush=True)
    for offset in (0, 1, 4):
        xs = [make(torch, n, param, grad, eight, seed=n + offset, offset=offset, copy=copy) for n in SIZES]
        decays = [0.1 if i % 2 else 0.0 for i in range(len(xs))]
        seed = 0x123456789ABCDEF + offset
        opt = optimizer(b, xs, eight, decays, stochastic, seed, copy)
        factor = torch.tensor([0.7], device="cuda")
        for step in (1, 2):
            scale = float(factor[0]) if step == 2 else 1.0
            want = [expected(x, np.float64(np.float32(d)), step, scale) for x, d in zip(xs, decays)]
            opt.step(1e-3, grad_scale=factor if step == 2 else None)
            for i, (x, w) in enumerate(zip(xs, want)):
                bits = ref.random_bits(seed, step, i, SIZES[i]) if stochastic else None
                compare(x, w, param, copy, bits, f"offset {offset} size {SIZES[i]} step {step}")
        assert opt.steps == 2


@pytest.mark.parametrize("eight", [False, True])
def test_many_tensors_of_several_types(gpu, eight):
    """More tensors than a launch takes, types mixed, in one call; and the same call gives the same bits."""
    torch, b = gpu
    rng = np.random.default_rng(1)
    sizes = [int(n) for n in np.exp(rng.uniform(0, 10, 300))]
    kinds = [("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")]
    results = []
    for _ in range(2):
        xs = [make(torch, n, *kinds[i % 4], eight and i % 3 != 0, seed=i) for i, n in enumerate(sizes)]
        pick = lambda name: [x[name].t if name in x else None for x in xs]  # noqa: E731
        opt = b.AdamW(pick("p"), pick("g"), betas=BETAS, eps=EPS, weight_decay=0.05, bits=[8 if "m_scale" in x else 32 for x in xs], m=pick("m"), v=pick("v"),
                      m_scale=pick("m_scale"), v_scale=pick("v_scale"), stochastic=True, seed=7)
        want = [expected(x, np.float64(np.float32(0.05)), 11) for x in xs]
        opt.step(1e-3, step=11)
        for i, (x, w) in enumerate(zip(xs, want)):
            compare(x, w, kinds[i % 4][0], None, ref.random_bits(7, 11, i, sizes[i]), f"tensor {i}")
        results.append([t.clone() for x in xs for t in (x["p"].t, x["m"].t.float(), x["v"].t.float())])
    assert all(torch.equal(p, q) for p, q in zip(*results))


def test_steps_that_are_skipped_and_gradients_that_are_not_finite(gpu):
    torch, b = gpu
    for eight in (False, True):
        x = make(torch, 1000, "f32", "f32", eight, seed=4, copy="bf16")
        opt = optimizer(b, [x], eight, 0.1, copy="bf16")
        before = {name: part.buf.clone() for name, part in x.items()}
        for bad in (math.nan, math.inf, -math.inf):
            opt.step(1e-3, grad_scale=torch.tensor([bad], device="cuda"))
            assert all(torch.equal(part.buf.view(torch.uint8), before[name].view(torch.uint8)) for name, part in x.items()), "a skipped step changed something"
        x["g"].t[300], x["g"].t[700] = math.nan, math.inf
        want = expected(make(torch, 1000, "f32", "f32", eight, seed=4, copy="bf16"), np.float64(np.float32(0.1)), 9)
        opt.step(1e-3, step=9)
        lost = np.zeros(1000, bool)
        lost[[300, 700]] = True
        ref.between(as64(x["p"].t)[~lost], (want.p - want.d_p)[~lost], (want.p + want.d_p)[~lost], "entries beside")
        assert math.isnan(float(x["p"].t[300])) and math.isnan(float(x["p"].t[700]))
        m = states(x, "m")
        if eight:
            assert np.isnan(m[512:768]).all() and np.isnan(m[300]) and np.isfinite(np.delete(m[256:512], 44)).all() and np.isfinite(m[:256]).all()
        else:
            assert np.isnan(m[300]) and np.isinf(m[700]) and np.isfinite(np.delete(m, [300, 700])).all()


@pytest.mark.parametrize("eight", [False, True])
def test_zeros_tiny_and_huge_gradients(gpu, eight):
    """Blocks of zeros stay zero and divide nothing by zero; scales at both ends of fp32."""
    torch, b = gpu
    for size in (0.0, 1e-30, 1e-18, 1e-10, 1e10, 1e18):
        x = make(torch, 600, "f32", "f32", eight, seed=2, size=size)
        want = expected(x, 0.0, 5)
        opt = optimizer(b, [x], eight, 0.0)
        opt.step(1e-3, step=5)
        assert bool(torch.isfinite(x["p"].t).all())
        if size in (0.0, 1e-10, 1e10, 1e18):
            compare(x, want, "f32", None, None, f"size {size}")
        if size == 0.0:
            assert not bool(x["m"].t.float().count_nonzero()) and not bool(x["v"].t.float().count_nonzero())
        if eight:
            stored = x["v"].t.float()
            assert bool((stored[5:] > 0).all()) or size < 1e-18, "a root above zero was stored as zero"


def test_numbers_read_on_the_device_and_graphs(gpu):
    """lr, step and factor in device memory: a captured step, replayed, equals eager steps; on a side stream."""
    torch, b = gpu
    for eight in (False, True):
        xs, ys = ([make(torch, n, "bf16", "f32", eight, seed=n) for n in (1000, 33, 5000)] for _ in range(2))
        one, two = (optimizer(b, part, eight, 0.1, stochastic=True, seed=99) for part in (xs, ys))
        lr, step = torch.tensor([1e-3], device="cuda"), torch.tensor([1], device="cuda")
        norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        grads, space = b.TensorList([x["g"].t for x in xs]), torch.zeros(b.ef21_grad_norm_workspace(3), dtype=torch.uint8, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        first = [expected(x, np.float64(np.float32(0.1)), 1, on_device=True) for x in xs]

        def call(opt):
            b.ef21_grad_norm(grads, 0.01, norm=norm, factor=factor, workspace=space)
            opt.step(lr, step=step, grad_scale=factor)

        with torch.cuda.stream(side):
            call(one)                                                  # eager
        side.synchronize()
        scale = float(factor[0])
        assert scale < 1.0
        first = [expected(y, np.float64(np.float32(0.1)), 1, scale, on_device=True) for y in ys]
        for i, (x, w) in enumerate(zip(xs, first)):
            compare(x, w, "bf16", None, ref.random_bits(99, 1, i, x["p"].n), f"tensor {i}")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(two)
        for t in range(1, 5):
            step.fill_(t)
            lr.fill_(1e-3 / t)
            if t > 1:
                call(one)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for x, y in zip(xs, ys):
                for name in x:
                    assert torch.equal(x[name].buf.view(torch.uint8), y[name].buf.view(torch.uint8)), (t, name)
                x["g"].t.mul_(-0.5).add_(1e-4)
                y["g"].t.copy_(x["g"].t)
        step.fill_(0)                                                  # counts as 1
        call(one)
        assert bool(torch.isfinite(xs[0]["p"].t.float()).all())


def test_random_rounding_is_right_on_average(gpu):
    """N entries with the same constant gradient: m is the exact average up to noise.  A rounding to neighbours of distance d has variance of at most
    d^2 / 4, a step carries b1^2 of the last one's on, and N entries average: six standard deviations of that.  The same for a bf16 parameter that
    moves by a 1/50 of its last bit a step."""
    torch, b = gpu
    N, steps = 65536, 30
    p, g = torch.zeros(N, device="cuda"), torch.full((N,), 1e-3, device="cuda")
    g[::256] = 0.01                                                    # the block's largest: others are off the ends of the grid
    opt = b.AdamW([p], [g], betas=BETAS, eps=EPS, weight_decay=0.0, bits=8, stochastic=True, seed=5)
    for _ in range(steps):
        opt.step(1e-3)
    m = as64(opt.m[0]) * ref.spread(as64(opt.m_scale[0]), N)
    some = np.arange(N) % 256 != 0
    exact = 1e-3 * (1 - BETAS[0] ** steps)
    gap = exact / 8                                                    # e4m3's neighbours are at most an eighth apart
    noise = 6 * gap / 2 / math.sqrt(1 - BETAS[0] ** 2) / math.sqrt(some.sum())
    assert abs(m[some].mean() - exact) <= noise + 8 * steps * U * exact + gap * 2.0 ** -17, (m[some].mean(), exact, noise)
    p = torch.ones(N, dtype=torch.bfloat16, device="cuda") * 1.5
    g = torch.ones(N, device="cuda")
    opt = b.AdamW([p], [g], betas=(0.0, 0.0), eps=1e-8, weight_decay=0.0, stochastic=True, seed=6)
    last_bit, lr = 2.0 ** -7, 2.0 ** -7 / 50
    for _ in range(steps):
        opt.step(lr)
    noise = 6 * last_bit / 2 * math.sqrt(steps) / math.sqrt(N)
    moved = 1.5 - as64(p).mean()
    assert abs(moved - steps * lr) <= noise + steps * last_bit * 2.0 ** -17 + steps * 8 * U, (moved, steps * lr, noise)
    near = torch.ones(N, dtype=torch.bfloat16, device="cuda") * 1.5
    b.AdamW([near], [g], betas=(0.0, 0.0), eps=1e-8, weight_decay=0.0).step(lr)
    assert bool((near == 1.5).all()), "to nearest such a step is lost"


# ---------------------------------------------------------------- the norm
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_norm(gpu, dtype):
    torch, b = gpu
    rng = np.random.default_rng(3)
    for sizes in ([1], [0], [0, 5, 0], [50000], [3, 257, 100003, 8, 64], [int(n) for n in np.exp(rng.uniform(0, 9, 300))], [5_000_001, 3]):
        for offset in (0, 1):
            gs = [Guarded(torch, rng.standard_normal(n), lm.TORCH[dtype], offset).t for n in sizes]
            total = math.sqrt(sum(float((as64(g) ** 2).sum()) for g in gs))
            for scale, limit in ((1.0, math.inf), (0.25, 0.1), (2.0, 1e9)):
                norm, factor = b.ef21_grad_norm(gs, limit, scale)
                want = scale * total
                assert abs(float(norm) - want) <= 2 * U * want
                clipped = scale * min(1.0, limit / want if want else math.inf)
                assert abs(float(factor) - clipped) <= 2 * U * clipped
            again = b.ef21_grad_norm(b.TensorList(gs), limit, scale)
            assert float(again[0]) == float(norm) and float(again[1]) == float(factor)


@pytest.mark.parametrize("sizes", [(5,), (300000,), (1000003, 70000), (1500000,), (3000000,), (1,) * 200 + (50000,) * 10, (20000,) * 500])
def test_norm_of_the_same_list_again_and_again(gpu, sizes):
    """A list's workspace is left as it was found: calls in a row, on two streams at once, and two graphs of the list replayed in turn, all on new contents."""
    torch, b = gpu
    g = torch.Generator(device="cuda").manual_seed(sum(sizes))
    xs = [torch.randn(n, generator=g, device="cuda") for n in sizes]
    lists = b.TensorList(xs)
    outs = [(torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")) for _ in range(4)]
    streams = [torch.cuda.Stream() for _ in range(2)]

    def want():
        return math.sqrt(sum(float((x.double() ** 2).sum()) for x in xs))

    def near(out, norm):
        # fp64 sums, a root and one rounding to fp32; the factor with a product and a quotient in fp64
        assert abs(float(out[0]) - norm) <= 2.0 ** -24 * 1.001 * norm and abs(float(out[1]) - min(1.0, 2.0 / norm)) <= 2.0 ** -24 * 1.001 * min(1.0, 2.0 / norm)

    graphs = []
    for out, stream in zip(outs[2:], streams):
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            b.ef21_grad_norm(lists, 2.0, norm=out[0], factor=out[1])
        stream.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            b.ef21_grad_norm(lists, 2.0, norm=out[0], factor=out[1])
    for turn in range(4):
        for x in xs[:3]:
            x.mul_(1.5)
        torch.cuda.synchronize()
        for out, stream in zip(outs, streams):
            with torch.cuda.stream(stream):
                for _ in range(5):
                    out[0].zero_()
                    b.ef21_grad_norm(lists, 2.0, norm=out[0], factor=out[1])
        torch.cuda.synchronize()
        for out in outs[2:]:
            out[0].zero_()
        for graph, stream in zip(graphs, streams[::-1]):
            with torch.cuda.stream(stream):
                graph.replay()
                graph.replay()
        torch.cuda.synchronize()
        for out in outs:
            near(out, want())
        assert len({(float(a), float(c)) for a, c in outs}) == 1
    space = torch.zeros(b.ef21_grad_norm_workspace(len(xs)), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        near(b.ef21_grad_norm(lists, 2.0, workspace=space), want())
        assert int(space[:4].max()) == 0


def test_norm_of_one_list_by_two_threads(gpu):
    """Calls of several launches each, on the same stream and list, from two threads."""
    torch, b = gpu
    lists = b.TensorList([torch.full((2000,), 0.5, device="cuda") for _ in range(400)] + [torch.full((200000,), 0.5, device="cuda")])
    got, failed = [], []

    def work():
        try:
            outs = [b.ef21_grad_norm(lists, 1.0) for _ in range(50)]
            got.extend(norm for norm, _ in outs)
        except Exception as e:                                          # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed and len(got) == 100
    assert all(float(x) == 500.0 for x in got)                          # the root of a million quarters


def test_norm_of_odd_values(gpu):
    torch, b = gpu
    x = torch.full((1000,), 1e30, device="cuda")                       # squares beyond fp32
    norm, factor = b.ef21_grad_norm([x], 1.0)
    assert abs(float(norm) / (1e30 * math.sqrt(1000)) - 1) < 1e-6 and abs(float(factor) * 1e30 * math.sqrt(1000) - 1) < 1e-6
    norm, _ = b.ef21_grad_norm([torch.full((1000,), 1e-30, device="cuda")], 1.0)
    assert abs(float(norm) / (1e-30 * math.sqrt(1000)) - 1) < 1e-6
    for bad in (math.nan, math.inf, -math.inf):
        y = torch.ones(70001, dtype=torch.bfloat16, device="cuda")
        y[70000] = bad
        norm, factor = b.ef21_grad_norm([x, y], 1.0)
        assert not math.isfinite(float(norm)) and math.isnan(float(factor))
    norm, factor = b.ef21_grad_norm([torch.full((4,), 3e38, device="cuda")], 1.0)    # the norm itself is beyond fp32
    assert math.isinf(float(norm)) and math.isnan(float(factor))
    norm, factor = b.ef21_grad_norm([torch.zeros(5, device="cuda")], 1.0, 0.5)
    assert float(norm) == 0.0 and float(factor) == 0.5


def test_memory_is_held(gpu):
    """A tensor whose .data is exchanged: what it had is kept, read and written, and no memory that others have by now."""
    torch, b = gpu
    n = 1 << 20
    p, g = torch.ones(n, device="cuda"), torch.full((n,), 2.0, device="cuda")
    memory = p.detach()
    opt, grads = b.AdamW([p], [g], weight_decay=0.0), b.TensorList([g])
    p.data, g.data = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    others = [torch.zeros(n, device="cuda") for _ in range(4)]
    opt.step(0.5)
    norm, _ = b.ef21_grad_norm(grads, 1.0)
    assert float(norm) == 2048.0                                   # the root of 2^20 times four
    # m / (1 - beta1) = 2, the root of v / (1 - beta2) = 2: a step of 0.5, but for fp32's roundings, two ulp of which are 2^-22
    assert float((memory - 0.5).abs().max()) <= 2.0 ** -20
    assert all(float(o.abs().max()) == 0.0 for o in others) and float(p) == 0.0


def test_large_tensors(gpu):
    """Beyond 2^31 entries and bytes: the last entries are reached, by their own random bits."""
    torch, b = gpu
    n = 2 ** 31 + 259
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g[-3:] = 2.0
    g[0] = 1.0
    norm, factor = b.ef21_grad_norm([g], 1.0)
    assert abs(float(norm) - math.sqrt(13.0)) < 1e-6 and abs(float(factor) - 1 / math.sqrt(13.0)) < 1e-6
    opt = b.AdamW([p], [g], bits=8, weight_decay=0.0)
    opt.step(1e-3)
    assert abs(float(p[-1]) + 1e-3) < 1e-5 and abs(float(p[0]) + 1e-3) < 1e-5 and int(p.count_nonzero()) == 4
    assert float(opt.m[0][-1].float()) == 448.0 and abs(float(opt.m_scale[0][-1]) * 448 - 0.2) < 1e-6


# ---------------------------------------------------------------- refusals
def test_binding_refuses(gpu):
    torch, b = gpu
    f = lambda n=4, **k: torch.zeros(n, device="cuda", **k)  # noqa: E731
    p, g = f(), f()
    both = f(8)
    for error, call in [
            (ValueError, lambda: b.AdamW([])), (TypeError, lambda: b.AdamW([p.double()])), (TypeError, lambda: b.AdamW([torch.zeros(4)])),
            (TypeError, lambda: b.AdamW([f(8)[::2]])), (ValueError, lambda: b.AdamW([p], [g, g])), (ValueError, lambda: b.AdamW([p], [f(5)])),
            (TypeError, lambda: b.AdamW([p], [g.long()])), (ValueError, lambda: b.AdamW([p], bits=16)), (ValueError, lambda: b.AdamW([p], bits=[8, 32])),
            (ValueError, lambda: b.AdamW([p], m_scale=[f(1)])), (TypeError, lambda: b.AdamW([p], m=[f().half()])), (ValueError, lambda: b.AdamW([p], m=[f(5)])),
            (ValueError, lambda: b.AdamW([p], bits=8, m_scale=[f(2)])), (TypeError, lambda: b.AdamW([p], copies=[f()])), (TypeError, lambda: b.AdamW([p.half()], copies=[p.half()])),
            (ValueError, lambda: b.AdamW([p], copies=[f(3).half()])), (ValueError, lambda: b.AdamW([p, p])), (ValueError, lambda: b.AdamW([both[:5], both[4:]])),
            (ValueError, lambda: b.AdamW([p], [p])), (ValueError, lambda: b.AdamW([p], m=[g], v=[g])), (ValueError, lambda: b.AdamW([p], [g], m=[g])),
            (ValueError, lambda: b.AdamW([p]).step(1e-3)), (b.EF21Error, lambda: b.AdamW([p], [g]).step(math.nan)),
            (b.EF21Error, lambda: b.AdamW([p], [g]).step(1e-3, step=0)), (b.EF21Error, lambda: b.AdamW([p], [g], betas=(1.0, 0.9)).step(1e-3)),
            (b.EF21Error, lambda: b.AdamW([p], [g], betas=(0.9, -0.1)).step(1e-3)), (b.EF21Error, lambda: b.AdamW([p], [g], eps=0.0).step(1e-3)),
            (TypeError, lambda: b.AdamW([p], [g]).step(f(1).double())), (TypeError, lambda: b.AdamW([p], [g]).step(1e-3, step=f(1))),
            (ValueError, lambda: b.AdamW([p], [g]).step(1e-3, grad_scale=f(2))), (b.EF21Error, lambda: b.AdamW([p], [g], weight_decay=math.inf).step(1e-3)),
            (ValueError, lambda: b.ef21_grad_norm([])), (TypeError, lambda: b.ef21_grad_norm([torch.zeros(3)])), (TypeError, lambda: b.ef21_grad_norm([f(8)[::2]])),
            (b.EF21Error, lambda: b.ef21_grad_norm([p], 0.0)), (b.EF21Error, lambda: b.ef21_grad_norm([p], math.nan)), (b.EF21Error, lambda: b.ef21_grad_norm([p], 1.0, 0.0)),
            (b.EF21Error, lambda: b.ef21_grad_norm([p], 1.0, math.inf)), (ValueError, lambda: b.ef21_grad_norm([p], norm=f(2))),
            (b.EF21Error, lambda: b.ef21_grad_norm([p], workspace=torch.empty(8, dtype=torch.uint8, device="cuda")))]:
        with pytest.raises(error):
            call()
    assert not bool(p.count_nonzero())


def test_c_call_without_tensors(gpu):
    torch, b = gpu
    lib = b.load_library()
    o = b.AdamwOptions(1e-3, 0.9, 0.999, 1e-8, 1, None, None, None, 0, 0)
    assert lib.ef21_adamw(None, 0, C.byref(o), None) == b.EF21_OK
    norm = torch.ones(2, device="cuda")
    assert lib.ef21_grad_norm(None, None, None, 0, 0.5, 1.0, norm.data_ptr(), norm.data_ptr() + 4, None, 0, None) == b.EF21_OK
    torch.cuda.synchronize()
    assert norm.tolist() == [0.0, 0.5]
