"""AdamW at the ends of fp32's range and beyond them, in 64 bits beside the kernel."""
import math

import numpy as np
import pytest

import stats_reference as ref
from lm_reference import U
from test_gpu_optimizer import BETAS, as64, make, states

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2106_05203_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load_library()
    return torch, binding


@pytest.mark.parametrize("size", [1e-17, 1e-18, 1e-19, 1e-20])
def test_roots_below_the_least_normal_number(gpu, size):
    """Gradients whose v lies below 2^-126, with an eps far below their roots.  v is two products and a sum: 7 u of itself and, below 2^-126 where fp32's
    numbers are 2^-149 apart, half of that for its product and its sum; the root is correctly rounded, and counted with 2 u; the rest as in
    stats_reference.  The bounds of v go through the root and the quotient as they are, not to first order."""
    torch, b = gpu
    eps, lr, step = 1e-25, 1e-3, 5
    x = make(torch, 600, "f32", "f32", False, seed=2, size=size)
    p, g, m, v = as64(x["p"].t), as64(x["g"].t), states(x, "m"), states(x, "v")
    b.AdamW([x["p"].t], [x["g"].t], betas=BETAS, eps=eps, weight_decay=0.0, m=[x["m"].t], v=[x["v"].t]).step(lr, step=step)
    b1, b2 = BETAS
    new_m, new_v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    d_m, d_v = 5 * U * (np.abs(b1 * m) + np.abs((1 - b1) * g)), 7 * U * new_v + 2.0 ** -149
    ref.between(as64(x["v"].t), new_v - d_v, new_v + d_v, "v")
    c1, c2 = 1 / (1 - b1 ** step), 1 / math.sqrt(1 - b2 ** step)
    least = np.sqrt(np.maximum(new_v - d_v, 0.0)) * (1 - 2 * U) * c2 + eps
    most = np.sqrt(new_v + d_v) * (1 + 2 * U) * c2 + eps
    q = np.stack([(new_m + s * d_m) * c1 / den for s in (-1, 1) for den in (least, most)])
    q_low, q_high = q.min(0), q.max(0)
    slack = 16 * U * np.maximum(np.abs(q_low), np.abs(q_high))
    end = 4 * U * np.abs(p) + lr * 4 * U * np.abs(q).max(0)
    ref.between(as64(x["p"].t), p - lr * (q_high + slack) - end, p - lr * (q_low - slack) + end, "parameters")
    # and they are updates of the order of lr, but for the two entries that had no v before
    moved = np.abs(as64(x["p"].t) - p)
    assert np.delete(moved, [3, 4]).max() < 10 * lr


@pytest.mark.parametrize("stochastic", [False, True])
def test_a_tiny_root_beside_large_ones_is_not_rounded_to_zero(gpu, stochastic):
    """8-bit blocks with one gradient of 1 and others of 1e-20, whose v of 1e-43 is 71 of fp32's least steps: stored as the least number above zero.
    The first step is lr but for v's two roundings, each half a step of 71, half of which the root has; 2 % is far beyond that."""
    torch, b = gpu
    g = torch.full((1000,), 1e-20, device="cuda")
    g[::256] = 1.0
    p = torch.zeros(1000, device="cuda")
    opt = b.AdamW([p], [g], betas=BETAS, eps=1e-25, weight_decay=0.0, bits=8, stochastic=stochastic, seed=3)
    opt.step(1e-3)
    v = as64(opt.v[0])
    assert np.all(v[::256] == 448.0)
    assert np.all(np.delete(v, np.arange(0, 1000, 256)) == 2.0 ** -9), "a root above zero was stored as something else than the least number"
    assert np.all(np.abs(as64(p) + 1e-3) <= 0.02 * 1e-3)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("stochastic", [False, True])
def test_a_nan_of_any_sign_and_payload_passes_into_8_bits(gpu, stochastic, dtype):
    """A gradient of all ones (memory filled with 0xFF) and the ordinary NaN, of both signs: m, v and p of the entry are NaN, its neighbours are not."""
    torch, b = gpu
    kind, whole = {"f32": (torch.int32, torch.float32), "bf16": (torch.int16, torch.bfloat16), "f16": (torch.int16, torch.float16)}[dtype]
    quiet = {"f32": 0x7fc00000, "bf16": 0x7fc0, "f16": 0x7e00}[dtype]
    g = torch.full((600,), 1e-3, device="cuda").to(whole)
    where = {5: -1, 300: torch.iinfo(kind).max, 301: quiet, 599: quiet + torch.iinfo(kind).min}
    for at, word in where.items():
        g.view(kind)[at] = word
    p = torch.ones(600, device="cuda")
    opt = b.AdamW([p], [g], betas=BETAS, weight_decay=0.0, bits=8, stochastic=stochastic, seed=3)
    for _ in range(3):                                                 # (other random bits)
        opt.step(1e-3)
        for name, t in (("p", p), ("m", opt.m[0]), ("v", opt.v[0])):
            assert np.flatnonzero(np.isnan(as64(t))).tolist() == sorted(where), name


@pytest.mark.parametrize("eight", [False, True])
def test_a_v_that_is_not_a_number_passes_into_the_parameter(gpu, eight):
    """v is NaN where m is not: as a state that is given, and after a finite gradient whose square is beyond fp32, which makes an 8-bit block's v infinite
    and so NaN, or a 32-bit v infinite (which divides m to zero)."""
    torch, b = gpu
    x = make(torch, 600, "f32", "f32", eight, seed=9)
    more = dict(m_scale=[x["m_scale"].t], v_scale=[x["v_scale"].t]) if eight else {}
    x["v"].t[300] = math.nan
    opt = b.AdamW([x["p"].t], [x["g"].t], betas=BETAS, weight_decay=0.0, bits=8 if eight else 32, m=[x["m"].t], v=[x["v"].t], **more)
    opt.step(1e-3)
    assert np.flatnonzero(np.isnan(as64(x["p"].t))).tolist() == [300] and np.isnan(as64(x["v"].t)[300]) and not np.isnan(as64(x["m"].t)[300])
    # (1e20)^2 is beyond fp32, where 8-bit states round it by itself; 1e-3 (1e20)^2 = 1e37 is not, in 32 bits' one product and sum; that of 1e22 is
    for huge in (1e20, 1e22):
        infinite = eight or huge > 1e21
        p, g = torch.ones(600, device="cuda"), torch.full((600,), 1e-3, device="cuda")
        g[7] = huge
        opt = b.AdamW([p], [g], betas=BETAS, weight_decay=0.0, bits=8 if eight else 32)
        opt.step(1e-3)
        assert bool(torch.isfinite(p).all()) and (float(p[7]) == 1.0) == infinite
        after = float(p[7])
        g[7] = 1e-3
        opt.step(1e-3)
        assert np.flatnonzero(np.isnan(as64(p))).tolist() == (list(range(256)) if eight else [])
        assert eight or (float(p[7]) == after) == infinite
