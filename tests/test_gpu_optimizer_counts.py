"""The number of AdamW's steps where some are skipped on the device, or captured: only steps that are taken count."""
import ctypes as C
import math

import pytest

pytestmark = pytest.mark.gpu
BAD = (math.nan, math.inf, -math.inf)


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2106_05203_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load_library()
    return torch, binding


FORMS = [("f32", 32, False), ("bf16", 32, True), ("f32", 8, False), ("bf16", 8, True)]


def make(torch, b, form):
    """An optimizer of three tensors whose gradients are the parameters', and all that it writes."""
    kind, bits, stochastic = form
    g = torch.Generator(device="cuda").manual_seed(1)
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[kind]
    ps = [torch.randn(n, generator=g, device="cuda").to(dtype) for n in (1000, 1, 4099)]
    gs = [torch.randn(n, generator=g, device="cuda") * 1e-2 for n in (1000, 1, 4099)]
    opt = b.AdamW(ps, gs, bits=bits, stochastic=stochastic, seed=11)
    return opt, gs


def same(torch, one, two):
    for name in ("params", "m", "v", "m_scale", "v_scale"):
        for x, y in zip(getattr(one, name), getattr(two, name)):
            if x is not None and not torch.equal(x.view(torch.uint8), y.view(torch.uint8)):
                return False
    return True


def plain(torch, b, form, numbers, factors, grads=None):
    """The steps of these numbers, each given."""
    opt, gs = make(torch, b, form)
    for t, f in zip(numbers, factors):
        opt.step(1e-2, step=t, grad_scale=torch.tensor([f], device="cuda"))
    return opt


@pytest.mark.parametrize("form", FORMS)
def test_skipped_steps_do_not_count(gpu, form):
    """After steps that are skipped the first that is taken is the first: the same bits as without them.  (The factors 1 / (1 - beta^t) are evaluated in
    64 bits on either side and rounded once.)"""
    torch, b = gpu
    opt, _ = make(torch, b, form)
    taken = []
    for factor in (math.nan, math.inf, 0.5, -math.inf, 1.0, 0.25, math.nan, 2.0):
        opt.step(1e-2, grad_scale=torch.tensor([factor], device="cuda"))
        if math.isfinite(factor):
            taken.append(factor)
        assert opt.steps == len(taken)
        assert same(torch, opt, plain(torch, b, form, range(1, len(taken) + 1), taken)), f"after {len(taken)} steps"
    # and on without a factor, by which no step is skipped
    opt.step(1e-2)
    assert opt.steps == 5
    assert same(torch, opt, plain(torch, b, form, range(1, 6), taken + [1.0]))


@pytest.mark.parametrize("form", FORMS)
def test_numbers_given_and_counted_in_turn(gpu, form):
    torch, b = gpu
    one, bad = torch.tensor([1.0], device="cuda"), torch.tensor([math.nan], device="cuda")
    opt, _ = make(torch, b, form)
    for how in ({}, {}, dict(grad_scale=bad), dict(grad_scale=one), dict(step=10), {}, dict(grad_scale=bad), dict(step=20, grad_scale=one), dict(grad_scale=one)):
        opt.step(1e-2, **how)
    assert opt.steps == 21
    numbers = [1, 2, 3, 10, 11, 20, 21]
    assert same(torch, opt, plain(torch, b, form, numbers, [1.0] * 7))
    opt.steps = 99
    opt.step(1e-2)
    opt.step(1e-2, grad_scale=bad)
    assert opt.steps == 100 and same(torch, opt, plain(torch, b, form, numbers + [100], [1.0] * 8))
    fresh, _ = make(torch, b, form)
    fresh.steps = 4
    fresh.step(1e-2)
    assert fresh.steps == 5 and same(torch, fresh, plain(torch, b, form, [5], [1.0]))
    with pytest.raises(ValueError):
        opt.steps = -1


def test_a_tensors_number_is_the_callers(gpu):
    torch, b = gpu
    number, one = torch.tensor([7], device="cuda"), torch.tensor([1.0], device="cuda")
    for counting in (False, True):
        opt, _ = make(torch, b, FORMS[0])
        if counting:
            opt.step(1e-2, grad_scale=one)
        opt.step(1e-2, step=number)
        assert opt.steps is None
        for how in ({}, dict(grad_scale=one)):
            with pytest.raises(ValueError):
                opt.step(1e-2, **how)
        opt.step(1e-2, step=8)
        opt.step(1e-2, grad_scale=one)
        assert opt.steps == 9
        opt.step(1e-2, step=number)
        opt.steps = 3
        opt.step(1e-2)
        assert opt.steps == 4


@pytest.mark.parametrize("form", FORMS)
def test_captured_steps_count_at_each_replay(gpu, form):
    """A graph of a step, replayed with factors of which some skip it, with the object's own eager steps and synchronizations in between."""
    torch, b = gpu
    factor, side = torch.tensor([1.0], device="cuda"), torch.cuda.Stream()
    warm, _ = make(torch, b, form)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.step(1e-2, grad_scale=factor)
    side.synchronize()
    opt, _ = make(torch, b, form)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        opt.step(1e-2, grad_scale=factor)
    assert opt.steps == 0
    taken = []
    for turn, f in enumerate((math.nan, 1.0, 0.5, math.inf, math.nan, 2.0, 1.0)):
        factor.fill_(f)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if math.isfinite(f):
            taken.append(f)
        if turn % 3 == 2:                                              # an eager one
            opt.step(1e-2)
            taken.append(1.0)
        torch.cuda.synchronize()
        assert opt.steps == len(taken)
        assert same(torch, opt, plain(torch, b, form, range(1, len(taken) + 1), taken)), turn


def test_captured_steps_without_a_factor(gpu):
    """They count too; after steps that the host has counted the number has to be on the device first."""
    torch, b = gpu
    side, dummy = torch.cuda.Stream(), torch.zeros(1, device="cuda")
    opt, _ = make(torch, b, FORMS[3])
    opt.step(1e-2)
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        dummy.add_(1)
        with pytest.raises(ValueError):
            opt.step(1e-2)
    opt.steps = opt.steps
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        opt.step(1e-2)
    for t in range(2, 6):
        graph.replay()
        torch.cuda.synchronize()
        assert opt.steps == t and same(torch, opt, plain(torch, b, FORMS[3], range(1, t + 1), [1.0] * t))


def test_the_c_call(gpu):
    """The counter is the caller's to set; a call without tensors counts too."""
    torch, b = gpu
    lib = b.load_library()
    opt, _ = make(torch, b, FORMS[2])
    counter, bad = torch.tensor([41, -1], dtype=torch.int64, device="cuda"), torch.tensor([math.nan], device="cuda")
    options = b.AdamwOptions(1e-2, 0.9, 0.999, 1e-8, -5, None, None, None, 0, 0)
    skipped = b.AdamwOptions(1e-2, 0.9, 0.999, 1e-8, 1, None, None, bad.data_ptr(), 0, 0)
    stream = torch.cuda.current_stream().cuda_stream
    for o in (options, skipped):
        assert lib.ef21_adamw_counted(opt._table, 3, C.byref(o), counter.data_ptr(), stream) == b.EF21_OK
    assert int(counter[0]) == 42 and same(torch, opt, plain(torch, b, FORMS[2], [42], [1.0]))
    counter[0] = -9
    for count in (1, 2):
        assert lib.ef21_adamw_counted(None, 0, C.byref(options), counter.data_ptr(), stream) == b.EF21_OK
        assert int(counter[0]) == count
