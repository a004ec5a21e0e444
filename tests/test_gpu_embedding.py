"""Embedding lookup and its gradient by sorted tokens against plain implementations (tests/lm_reference.py)."""
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


@pytest.mark.parametrize("table_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("out_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,width,count,stride,offset", [(1, 1, 1, 1, 0), (10, 3, 7, 5, 1), (100, 64, 33, 64, 0), (50, 127, 20, 129, 3), (1000, 512, 300, 512, 0),
                                                             (77, 1000, 9, 1004, 4), (300, 2056, 65, 2056, 0), (30, 8192, 5, 8192, 8)])
def test_lookup_is_one_product_and_one_rounding(gpu, vocab, width, count, stride, offset, table_type, out_type):
    torch, b = gpu
    print(f"embed vocab={vocab} width={width} count={count} {table_type}->{out_type}", flush=True)
    g = torch.Generator().manual_seed(vocab + width)
    buf = torch.randn(vocab * stride + offset + 8, generator=g).to(lm.TORCH[table_type]).cuda()
    table = buf[offset:].as_strided((vocab, width), (stride, 1))
    tokens = torch.randint(0, vocab, (count,), generator=g)
    tokens[::4] = torch.tensor([-1, vocab, -100, 1 << 40])[torch.arange(len(tokens[::4])) % 4]
    for scale in (1.0, 11.3):
        ok = (tokens >= 0) & (tokens < vocab)
        want = table[tokens.clamp(0, vocab - 1).cuda()].float() * torch.tensor(scale, dtype=torch.float32, device="cuda")
        want = torch.where(ok.cuda()[:, None], want, 0.0).to(lm.TORCH[out_type])
        got = b.ef21_embed(table, tokens.cuda(), scale, dtype=lm.TORCH[out_type])
        assert torch.equal(got, want)
        other = torch.full((count * (width + 5) + 1,), 3.0, dtype=lm.TORCH[out_type], device="cuda")
        to = other[1:].as_strided((count, width), (width + 5, 1))
        narrow = tokens.clone()
        narrow[narrow > vocab] = -7                                    # what does not fit 32 bits
        b.ef21_embed(table, narrow.to(torch.int32).cuda(), scale, out=to)
        assert torch.equal(to, want)
        gaps = other.as_strided((count, 5), (width + 5, 1), 1 + width)[: count - 1]
        assert bool((gaps == 3.0).all()) and float(other[0]) == 3.0, "entries beside the rows were written"


def test_lookup_shapes_infinities_and_no_tokens(gpu):
    torch, b = gpu
    table = torch.randn(20, 24, device="cuda")
    table[3, 5], table[4, 6] = math.inf, math.nan
    tokens = torch.tensor([[3, 4, 5], [0, 19, 3]], device="cuda")
    out = b.ef21_embed(table, tokens, 2.0)
    assert out.shape == (2, 3, 24) and torch.equal(out.nan_to_num(9.0), (table[tokens] * 2.0).nan_to_num(9.0))
    assert b.ef21_embed(table, tokens[:0]).shape == (0, 3, 24)


def test_lookup_beyond_32_bits(gpu):
    torch, b = gpu
    vocab, width = 140000, 32768                                       # 4.6e9 entries
    table = torch.empty(vocab, width, dtype=torch.bfloat16, device="cuda")
    tokens = torch.tensor([139999, 0, 131072, 65536], device="cuda")
    rows = torch.randn(4, width, device="cuda").to(torch.bfloat16)
    table[tokens] = rows
    assert torch.equal(b.ef21_embed(table, tokens), rows)


def token_sets(rng, kind, n, count, vocab):
    if kind == "uniform":
        t = rng.integers(0, vocab, (n, count))
    elif kind == "zipf":
        t = ((vocab + 1.0) ** rng.random((n, count)) - 1.0).astype(np.int64).clip(0, vocab - 1)
    elif kind == "one":
        t = np.full((n, count), vocab - 1)
    elif kind == "none":
        t = np.where(rng.random((n, count)) < 0.5, -1, vocab)
    elif kind == "two":                                                # two tokens in turn, the ends of the table
        t = np.where(rng.random((n, count)) < 0.5, 0, vocab - 1)
    else:                                                              # a third outside the table
        t = rng.integers(-vocab // 4 - 1, vocab + vocab // 4 + 1, (n, count))
    return t


COUNTS = [(1, 1, 1, 1), (2, 0, 5, 8), (3, 2, 4, 3), (2, 63, 17, 16), (1, 64, 1000, 64), (4, 65, 300, 100), (2, 250, 1001, 33), (1, 1023, 50, 72),
          (3, 1500, 257, 24), (2, 2048, 3000, 128), (1, 4097, 700, 520), (2, 9000, 65536, 8), (1, 20000, 300, 12), (1, 70001, 2000, 16), (1, 300, 131073, 40)]


@pytest.mark.parametrize("kind", ["uniform", "zipf", "one", "none", "two", "outside"])
@pytest.mark.parametrize("n,count,vocab,width", COUNTS)
def test_gradient_by_sorted_tokens(gpu, n, count, vocab, width, kind):
    torch, b = gpu
    dtype = ["f32", "bf16", "f16"][(count + width) % 3]
    print(f"embed_grad n={n} count={count} vocab={vocab} width={width} {dtype} {kind}", flush=True)
    rng = np.random.default_rng(count + vocab)
    tokens = token_sets(rng, kind, n, count, vocab)
    g = torch.from_numpy(rng.standard_normal((n, count, width)).astype(np.float32)).to(lm.TORCH[dtype])
    dt = torch.from_numpy(tokens.astype(np.int64 if width % 2 else np.int32)).cuda()
    scale = float(np.float32(0.75))
    got = b.ef21_embed_grad(g.cuda(), dt, vocab, scale, out=torch.full((n, vocab, width), math.nan, device="cuda"))
    want, bound = lm.embed_grad(g.double().numpy(), tokens, vocab, scale)
    lm.inside(as64(got), want, bound, "gradient")
    assert torch.equal(got, b.ef21_embed_grad(g.cuda(), dt, vocab, scale)), "the same bits again"
    base = torch.from_numpy(rng.standard_normal((n, vocab, width)).astype(np.float32))
    got = b.ef21_embed_grad(g.cuda(), dt, vocab, scale, out=base.cuda(), accumulate=True)
    want, bound = lm.embed_grad(g.double().numpy(), tokens, vocab, scale, base.numpy())
    lm.inside(as64(got), want, bound, "accumulated gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width,stride,offset", [(1, 1, 0), (5, 7, 1), (48, 48, 3), (64, 72, 0), (1000, 1000, 0), (1032, 1033, 0), (2500, 2500, 4)])
def test_gradient_strides_and_a_block_of_the_workers_rows(gpu, dtype, width, stride, offset):
    """grad_out with gaps between the rows, written to a block of columns of the rows [n][d] that step() takes; what lies beside it stays."""
    torch, b = gpu
    n, count, vocab, first = 3, 90, 37, 11
    rng = np.random.default_rng(width)
    buf = torch.full((n * count * stride + offset + 8,), math.nan).to(lm.TORCH[dtype])
    g = torch.from_numpy(rng.standard_normal((n, count, width)).astype(np.float32)).to(lm.TORCH[dtype])
    buf[offset:].as_strided((n, count, width), (count * stride, stride, 1)).copy_(g)
    view = buf.cuda()[offset:].as_strided((n, count, width), (count * stride, stride, 1))
    tokens = token_sets(rng, "zipf", n, count, vocab)
    d = first + vocab * width + 5
    grads = torch.full((n, d), 7.0, device="cuda")
    block = grads.as_strided((n, vocab, width), (d, width, 1), first)
    b.ef21_embed_grad(view, torch.from_numpy(tokens).cuda(), vocab, out=block)
    want, bound = lm.embed_grad(g.double().numpy(), tokens, vocab, 1.0)
    lm.inside(as64(block), want, bound, "gradient")
    assert bool((grads[:, :first] == 7.0).all()) and bool((grads[:, first + vocab * width:] == 7.0).all())


def test_gradient_against_differences_of_the_lookup(gpu):
    """<embed(table), R> is linear in the table: its gradient is embed_grad(R), and differences of it are exact but for rounding."""
    torch, b = gpu
    vocab, width, count = 9, 6, 40
    rng = np.random.default_rng(3)
    tokens = torch.from_numpy(rng.integers(-1, vocab, count)).cuda()
    table = torch.from_numpy(rng.integers(-8, 8, (vocab, width)).astype(np.float32)).cuda()
    R = torch.from_numpy(rng.integers(-8, 8, (1, count, width)).astype(np.float32)).cuda()
    grad = b.ef21_embed_grad(R, tokens[None], vocab, 2.0)[0]
    value = lambda: float((b.ef21_embed(table, tokens, 2.0).double() * R[0].double()).sum())  # noqa: E731
    for v in range(vocab):
        for j in range(width):
            table[v, j] += 1.0
            up = value()
            table[v, j] -= 2.0
            down = value()
            table[v, j] += 1.0
            assert (up - down) / 2 == float(grad[v, j])              # small whole numbers: every sum is exact


def test_gradient_in_a_graph_and_on_another_stream(gpu):
    torch, b = gpu
    n, count, vocab, width = 2, 3000, 500, 64
    rng = np.random.default_rng(1)
    grad_out = torch.zeros(n, count, width, dtype=torch.bfloat16, device="cuda")
    tokens = torch.zeros(n, count, dtype=torch.int64, device="cuda")
    out = torch.empty(n, vocab, width, device="cuda")
    ws = torch.empty(b.ef21_embed_grad_workspace(n, count, vocab, width), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        b.ef21_embed_grad(grad_out, tokens, vocab, out=out, workspace=ws)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.ef21_embed_grad(grad_out, tokens, vocab, out=out, workspace=ws)
    for kind in ("zipf", "one", "uniform", "none"):
        grad_out.copy_(torch.from_numpy(rng.standard_normal((n, count, width)).astype(np.float32)))
        tokens.copy_(torch.from_numpy(token_sets(rng, kind, n, count, vocab)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, b.ef21_embed_grad(grad_out, tokens, vocab)), f"replay with {kind} tokens differs"


def test_gradient_beyond_32_bits(gpu):
    """A gradient of 4.3e9 entries: the last worker's and the last token's rows are where they belong."""
    torch, b = gpu
    n, count, vocab, width = 2, 5, 131072, 16500
    tokens = torch.tensor([[0, 131071, 7, 131071, -1], [131071, 131070, 0, 0, 131071]], device="cuda")
    g = torch.randn(n, count, width, device="cuda")
    out = b.ef21_embed_grad(g, tokens, vocab)
    for i in range(n):
        for v in (0, 7, 131070, 131071):
            want = g[i].double()[tokens[i] == v].sum(0)
            assert torch.allclose(out[i, v].double(), want, rtol=1e-6, atol=1e-6)
        assert int(out[i].count_nonzero(dim=1).count_nonzero()) == len({int(t) for t in tokens[i] if t >= 0})


@pytest.mark.parametrize("n,count,vocab,width,dtype,kind", [(5, 60000, 700, 8, "bf16", "zipf"), (3, 50000, 3001, 12, "f16", "zipf"), (3, 50000, 3001, 12, "f32", "uniform"),
                                                            (2, 4000, 37, 16, "f32", "zipf"), (1, 4096, 5, 700, "bf16", "uniform"), (1, 4096, 90000, 9, "f16", "outside"),
                                                            (2, 3000, 2, 5, "f32", "one"), (1, 16384, 131071, 16, "bf16", "zipf"), (1, 16385, 131072, 16, "bf16", "zipf")])
def test_gradient_of_many_tokens(gpu, n, count, vocab, width, dtype, kind):
    torch, b = gpu
    print(f"embed_grad n={n} count={count} vocab={vocab} width={width} {dtype} {kind}", flush=True)
    rng = np.random.default_rng(count + width)
    tokens = token_sets(rng, kind, n, count, vocab)
    g = torch.from_numpy(rng.standard_normal((n, count, width)).astype(np.float32)).to(lm.TORCH[dtype])
    base = torch.from_numpy(rng.standard_normal((n, vocab, width)).astype(np.float32))
    dt = torch.from_numpy(tokens).cuda()
    for before in (None, base):
        out = torch.full((n, vocab, width), math.nan, device="cuda") if before is None else before.cuda()
        got = b.ef21_embed_grad(g.cuda(), dt, vocab, 0.75, out=out, accumulate=before is not None)
        want, bound = lm.embed_grad(g.double().numpy(), tokens, vocab, 0.75, *([] if before is None else [before.numpy()]))
        lm.inside(as64(got), want, bound, "gradient")


@pytest.mark.parametrize("n,count,vocab,width,shift", [(3, 100, 30001, 1003, 1), (1, 4096, 70000, 1024, 0), (2, 9, 70000, 1024, 2), (3, 0, 30001, 1003, 3), (1, 20000, 30000, 2500, 5)])
def test_gradient_of_large_tables(gpu, n, count, vocab, width, shift):
    """Tables of more than 256 MB, at any alignment: each row is written, and nothing between the tables or around them."""
    torch, b = gpu
    print(f"embed_grad n={n} count={count} vocab={vocab} width={width} shift={shift}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(count + shift)
    tokens = torch.randint(0, vocab, (n, count), device="cuda", generator=gen)
    if count > 4:
        tokens[:, 0], tokens[:, 1], tokens[:, 2] = 0, vocab - 1, -1
    grad = torch.randn(n, count, width, device="cuda", generator=gen).mul_(8).round_()   # whole numbers: their sums are exact
    stride = vocab * width + 7
    flat = torch.full((n * stride + shift,), 3.5, device="cuda")
    out = flat[shift:].as_strided((n, vocab, width), (stride, width, 1))
    b.ef21_embed_grad(grad, tokens, vocab, out=out)
    for i in range(n):
        want = torch.zeros(vocab, width, device="cuda")
        ok = tokens[i] >= 0
        want.index_add_(0, tokens[i][ok], grad[i][ok])
        assert torch.equal(out[i], want)
        del want
    assert bool((flat[:shift] == 3.5).all())
    for i in range(n):
        end = shift + i * stride + vocab * width
        assert bool((flat[end:end + 7] == 3.5).all())


def test_gradient_of_very_many_workers(gpu):
    """16 tokens of each of 65535 workers: one chunk of sorted entries a worker, and 4.3e9 entries of grad_out."""
    torch, b = gpu
    n, count, width = 65535, 16, 4100
    grad = torch.empty(n, count, width, dtype=torch.bfloat16, device="cuda")
    grad.random_(-8, 9, generator=torch.Generator(device="cuda").manual_seed(2))
    tokens = torch.zeros(n, count, dtype=torch.int32, device="cuda")
    tokens[::3, 5], tokens[7, :] = -1, 1                               # outside a vocabulary of one
    got = b.ef21_embed_grad(grad, tokens, 1)
    for i in range(0, n, 4096):
        part = grad[i:i + 4096].float() * (tokens[i:i + 4096] == 0)[..., None]
        assert torch.equal(got[i:i + 4096, 0], part.sum(1))
    got.fill_(math.nan)
    b.ef21_embed_grad(grad[:, :0], tokens[:, :0].contiguous(), 1, out=got)
    assert int(got.count_nonzero()) == 0
    del got, part
    # so many columns that workgroups take several tiles' worth of tokens and of sums
    got = b.ef21_embed_grad(grad.view(n, 1, count * width), tokens[:, :1].contiguous(), 1)
    for i in range(0, n, 4096):
        assert torch.equal(got[i:i + 4096, 0], grad[i:i + 4096].view(-1, count * width).float() * (tokens[i:i + 4096, :1] == 0))


@pytest.mark.parametrize("n,count,vocab,width", [(2, 200001, 500, 4), (1, 131073, 262144, 3), (1, 2200000, 3000, 1), (3, 8193, 1 << 20, 2)])
def test_gradient_sorted_in_tiles(gpu, n, count, vocab, width):
    """Tiles of every size, and keys of one, two and three digits."""
    torch, b = gpu
    print(f"embed_grad n={n} count={count} vocab={vocab} width={width}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(count)
    tokens = (torch.rand(n, count, device="cuda", generator=gen).pow_(3) * (vocab + 1)).to(torch.int32) - 1
    grad = torch.randint(-2, 3, (n, count, width), device="cuda", generator=gen).float()   # whole numbers: their sums are exact
    got = b.ef21_embed_grad(grad, tokens, vocab)
    for i in range(n):
        ok = tokens[i] >= 0
        assert torch.equal(got[i], torch.zeros(vocab, width, device="cuda").index_add_(0, tokens[i][ok].long(), grad[i][ok]))
    again = b.ef21_embed_grad(grad, tokens, vocab, out=got.clone(), accumulate=True)
    assert torch.equal(again, 2 * got)
