"""AdamW on tensors as large as models have: the kernel that keeps two blocks in flight, places beyond 2^32, and grids beyond 2^31 threads, each with its
random bits, against the 64-bit formula at blocks all over the tensor."""
import numpy as np
import pytest

import stats_reference as ref
from stats_reference import BLOCK, mixed
from test_gpu_optimizer import BETAS, EPS, as64

pytestmark = pytest.mark.gpu
SEED, STEP, LR, DECAY = 0xFEDCBA987654321, 7, 1e-3, 0.1


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2106_05203_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load_library()
    return torch, binding


def bits_at(places, number):
    """(for m, for v, for the parameter) sixteen random bits of the entries at `places` of tensor `number`, as stats_reference.random_bits has them."""
    key = mixed(SEED & 0xFFFFFFFF)
    for part in (SEED >> 32, STEP, number):
        key = mixed(key + np.uint64(part))
    i = np.asarray(places, dtype=np.uint64)
    h = mixed(i ^ mixed(key + (i >> np.uint64(32))))
    return h & np.uint64(0xFFFF), h >> np.uint64(16), mixed(h + np.uint64(0x3C6EF372)) & np.uint64(0xFFFF)


def test_the_bits_are_the_references():
    places = np.arange(5000)
    for a, b in zip(bits_at(places, 3), ref.random_bits(SEED, STEP, 3, 5000)):
        assert np.array_equal(a, b)


def entries(n, blocks):
    """The places of the entries of these blocks of a tensor of n, the last of which may be shorter."""
    return np.concatenate([np.arange(k * BLOCK, min(n, (k + 1) * BLOCK), dtype=np.int64) for k in blocks])


def read(torch, opt, t, places, blocks):
    """(p, m, v or its root) at places, in 64 bits."""
    at, parts = torch.from_numpy(places).cuda(), [as64(opt.params[t][torch.from_numpy(places).cuda()])]
    for state, scale in ((opt.m, opt.m_scale), (opt.v, opt.v_scale)):
        if scale[t] is None:
            parts.append(as64(state[t][at]))
        else:
            codes = state[t].view(torch.uint8)[at].view(torch.float8_e4m3fn)
            parts.append(as64(codes) * ref.spread(as64(scale[t][torch.tensor(blocks, device="cuda")]), len(places)))
    return parts


def check(torch, opt, t, places, blocks, before, g, kind):
    """The step's results at these blocks."""
    eight = opt.m_scale[t] is not None
    want = ref.Adamw(before[0], g, before[1], before[2], LR, BETAS, EPS, DECAY, STEP, eight=eight)
    for_m, for_v, for_p = bits_at(places, t)
    at = torch.from_numpy(places).cuda()
    ref.between(as64(opt.params[t][at]), *want.params(kind, for_p if kind != "f32" else None), f"tensor {t} parameters")
    if not eight:
        ref.between(as64(opt.m[t][at]), want.m - want.d_m, want.m + want.d_m, f"tensor {t} m")
        ref.between(as64(opt.v[t][at]), want.v - want.d_v, want.v + want.d_v, f"tensor {t} v")
        return
    for name, (low, high, scale, d_scale) in want.codes(for_m, for_v).items():
        state, scales = (opt.m[t], opt.m_scale[t]) if name == "m" else (opt.v[t], opt.v_scale[t])
        ref.between(as64(scales[torch.tensor(blocks, device="cuda")]), scale - d_scale, scale + d_scale, f"tensor {t} {name}_scale")
        ref.between(as64(state.view(torch.uint8)[at].view(torch.float8_e4m3fn)), low, high, f"tensor {t} {name}")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_two_blocks_in_flight(gpu, kind):
    """From 2^25 entries on 8-bit states take another kernel: blocks all over two tensors that together have as many; and the first tensor alone, which the
    other kernel takes, has the same bits in every entry."""
    torch, b = gpu
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[kind]
    sizes = [2 ** 24 + 1031, 2 ** 24 + 777]                            # ends within a workgroup's blocks, and within a block
    gen = torch.Generator(device="cuda").manual_seed(5)
    ps = [(torch.randn(n, generator=gen, device="cuda") * 0.02).to(dtype) for n in sizes]
    gs = [(torch.randn(n, generator=gen, device="cuda") * 1e-3).to(dtype) for n in sizes]

    def make(count):
        opt = b.AdamW([p.clone() for p in ps[:count]], gs[:count], betas=BETAS, eps=EPS, weight_decay=DECAY, bits=8, stochastic=True, seed=SEED)
        opt.step(LR, step=STEP - 1)                                    # states to go on with
        return opt

    both, alone = make(2), make(1)
    rng = np.random.default_rng(1)
    for t, n in enumerate(sizes):
        last = -(-n // BLOCK) - 1
        blocks = sorted({0, 1, 7, 8, 9, last - 8, last - 1, last} | set(int(k) for k in rng.integers(0, last, 60)))
        places = entries(n, blocks)
        before = read(torch, both, t, places, blocks)
        g = as64(gs[t][torch.from_numpy(places).cuda()])
        if t == 0:
            kept = places, blocks, before, g
    both.step(LR, step=STEP)
    alone.step(LR, step=STEP)
    check(torch, both, 0, *kept, kind)
    check(torch, both, 1, places, blocks, before, g, kind)
    for name in ("params", "m", "v", "m_scale", "v_scale"):
        assert torch.equal(getattr(both, name)[0].view(torch.uint8), getattr(alone, name)[0].view(torch.uint8)), name


def sparse(torch, n, blocks, dtype, seed):
    """A tensor of zeros but for these blocks."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.zeros(n, dtype=dtype, device="cuda")
    for k in blocks:
        part = x[k * BLOCK:(k + 1) * BLOCK]
        part.copy_(torch.randn(len(part), generator=gen, device="cuda") * 1e-2)
    return x


@pytest.mark.parametrize("n,bits", [(2 ** 32 + 2 ** 20 + 259, 8), (2 ** 31 + 2 ** 20 + 259, 32)])
def test_places_beyond_32_bits_and_the_largest_grids(gpu, n, bits):
    """8-bit states beyond 2^32 entries: blocks on both sides of 2^31 and 2^32, by random bits of their places.  32-bit states beyond 2^31: the tensor alone
    has more workgroups than a launch of several takes, and one behind it gets a launch of its own.  Blocks without a gradient stay zeros."""
    torch, b = gpu
    print(f"{n} entries, {bits} bits", flush=True)
    last = -(-n // BLOCK) - 1
    marks = {k for k in (0, 1, 12345, 2 ** 23 - 1, 2 ** 23, 2 ** 23 + 1, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, last - 8, last - 1, last) if k <= last}
    blocks = sorted(marks)
    small = 1000
    places = [entries(n, blocks), entries(small, range(4))]
    numbers = [blocks, list(range(4))]
    ps = [sparse(torch, n, blocks, torch.bfloat16, 1), sparse(torch, small, range(4), torch.bfloat16, 2)]
    gs = [sparse(torch, n, blocks, torch.bfloat16, 3), sparse(torch, small, range(4), torch.bfloat16, 4)]
    opt = b.AdamW(ps, gs, betas=BETAS, eps=EPS, weight_decay=DECAY, bits=bits, stochastic=True, seed=SEED)
    before = [read(torch, opt, t, places[t], numbers[t]) for t in range(2)]
    opt.step(LR, step=STEP)
    for t in range(2):
        check(torch, opt, t, places[t], numbers[t], before[t], as64(gs[t][torch.from_numpy(places[t]).cuda()]), "bf16")
    # nothing else: as whole words, block by block of what was set
    for x in (ps[0], opt.m[0], opt.v[0]):
        x = x.view(torch.uint8) if x.itemsize == 1 else x
        for k in blocks:
            x[k * BLOCK:(k + 1) * BLOCK].zero_()
        assert not any(bool(part.any()) for part in x.split(2 ** 30)), "entries without a gradient were written"
    del ps, gs, opt
    torch.cuda.empty_cache()
