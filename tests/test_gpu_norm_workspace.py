"""The norm of gradients with a workspace that holds anything: what other calls left there, or nothing but ones."""
import math

import pytest

pytestmark = pytest.mark.gpu
# workgroups of a launch (a chunk of 64 KB each): one, a few, all that add up by themselves; and beyond, where a second launch does
SIZES = [(1,), (70000,), (82000,), (500000,), (2097152,), (2097153,), (3000000,), (1,) * 200 + (50000,) * 10, (20000,) * 300]
# the workspace as words of 64 bits: nothing, ones, small numbers as tokens or counts are, numbers with the upper half of a counter's and a lower that is none
FILLS = [0, -1, 1, 5, 127, 128, 1 << 32, (1 << 32) + 3, 0x3F8000003F800000, 0x6A09E667 << 32, (0x6A09E667 << 32) + 128, (0x6A09E667 << 32) + 0xFFFFFFFF, 0x6A09E666FFFFFFFF]


def case(torch, sizes):
    g = torch.Generator(device="cuda").manual_seed(len(sizes) + sizes[0])
    xs = [torch.randn(n, generator=g, device="cuda") for n in sizes]
    return xs, math.sqrt(sum(float((x.double() ** 2).sum()) for x in xs))


def near(out, norm):
    # fp64 sums, a root and one rounding to fp32; the factor with a product and a quotient in fp64
    for got, want in zip(out, (norm, min(1.0, 2.0 / norm))):
        assert abs(float(got) - want) <= 2.0 ** -24 * 1.001 * want


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{s[0]}")
def test_any_contents(sizes):
    import torch
    from paper_2106_05203_amd import binding as b
    xs, norm = case(torch, sizes)
    lists, need = b.TensorList(xs), b.ef21_grad_norm_workspace(len(xs))
    words = torch.empty(-(-need // 8), dtype=torch.int64, device="cuda")
    random = torch.randint(-2 ** 62, 2 ** 62, (8, len(words)), device="cuda")
    for fill in FILLS + list(random):
        print("fill", fill if isinstance(fill, int) else "random", flush=True)
        if isinstance(fill, int):
            words.fill_(fill)
        else:
            words.copy_(fill)
        for _ in range(3):                                             # and again with what it left
            out = b.ef21_grad_norm(lists, 2.0, norm=torch.full((1,), -1.0, device="cuda"), factor=torch.full((1,), -1.0, device="cuda"), workspace=words)
            near(out, norm)


def test_a_captured_call_whose_workspace_others_use():
    """Between replays the workspace is other calls' scratch memory, of another list and of another kind."""
    import torch
    from paper_2106_05203_amd import binding as b
    xs, norm = case(torch, (500000, 300))
    ys, other = case(torch, (1500000,))
    space = torch.empty(b.ef21_grad_norm_workspace(2), dtype=torch.uint8, device="cuda")
    lists, more, side = b.TensorList(xs), b.TensorList(ys), torch.cuda.Stream()
    out = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.ef21_grad_norm(lists, 2.0, norm=out[0], factor=out[1], workspace=space)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.ef21_grad_norm(lists, 2.0, norm=out[0], factor=out[1], workspace=space)
    for turn in range(5):
        space.fill_(17 * turn)
        out[0].zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        near(out, norm)
        near(b.ef21_grad_norm(more, 2.0, workspace=space), other)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        near(out, norm)
