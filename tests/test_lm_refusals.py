"""What the operators at the two ends of a language model refuse, by status through the C ABI (before any HIP call, so without a
GPU) and by exception in the binding."""
import ctypes as C
import math
import os

import pytest
import torch

from paper_2106_05203_amd import binding

BAD = binding.EF21_EINVAL


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2106_05203_amd import build
        build.build_library()
    return binding.load_library()


@pytest.fixture(scope="module")
def ptr():
    """A 256-byte aligned address that no refused call follows."""
    raw = (C.c_char * 1024)()
    ptr.keep = raw
    return (C.addressof(raw) + 255) // 256 * 256


def refused(lib, rc):
    assert rc == BAD and lib.ef21_last_error() != b""


def swap(args, at, value):
    return [value if i == at else a for i, a in enumerate(args)]


def test_embed(lib, ptr):
    good = [ptr, 0, 10, 4, 4, ptr, 1, 3, 1.0, ptr, 0, 4, None]
    for at, value in [(0, None), (0, ptr + 2), (1, 3), (1, -1), (2, 0), (2, 2 ** 31), (3, 0), (4, 3), (4, 2 ** 62), (5, None), (5, ptr + 4), (6, 2), (7, -1),
                      (7, 2 ** 31), (8, math.nan), (8, math.inf), (9, None), (10, 5), (11, 3)]:
        refused(lib, lib.ef21_embed(*swap(good, at, value)))


def test_embed_grad(lib, ptr):
    size = C.c_int64()
    assert lib.ef21_embed_grad_workspace(2, 100, 50, 4, C.byref(size)) == binding.EF21_OK
    need = size.value
    good = [ptr, 0, 4, ptr, 1, 2, 100, 50, 4, 1.0, ptr, 200, 0, ptr, need, None]
    for at, value in [(0, None), (0, ptr + 1), (1, 7), (2, 3), (3, None), (4, -1), (5, 0), (5, 65536), (6, -1), (6, 2 ** 31), (7, 0), (7, 2 ** 31), (8, 0),
                      (9, math.inf), (10, None), (10, ptr + 2), (11, 199), (13, None), (13, ptr + 64), (14, need - 1), (14, -1)]:
        refused(lib, lib.ef21_embed_grad(*swap(good, at, value)))
    for args in [(0, 1, 1, 1), (1, -1, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (65535, 2 ** 31 - 1, 1, 1), (65535, 1, 2 ** 31 - 2, 2 ** 31 - 1)]:
        refused(lib, lib.ef21_embed_grad_workspace(*args, C.byref(size)))
    refused(lib, lib.ef21_embed_grad_workspace(1, 1, 1, 1, None))


LOGITS_BAD = [(0, None), (0, "odd"), (1, 3), (2, -1), (2, 2 ** 31), (3, 0), (3, 2 ** 31), (4, 6), (4, 2 ** 61), (5, None), (6, 9)]


def bad_logits(good, ptr):
    for at, value in LOGITS_BAD:
        yield swap(good, at, ptr + 1 if value == "odd" else value)


def test_token_logps(lib, ptr):
    good = [ptr, 1, 5, 7, 7, ptr, 0, ptr, ptr, None]
    for args in [*bad_logits(good, ptr), swap(good, 7, None), swap(good, 8, ptr + 2)]:
        refused(lib, lib.ef21_token_logps(*args))
    good = [ptr, 1, 5, 7, 7, ptr, 0, ptr, ptr, ptr, 7, None]
    for args in [*bad_logits(good, ptr), swap(good, 7, None), swap(good, 8, None), swap(good, 9, None), swap(good, 10, 6), swap(good, 10, 8)]:
        refused(lib, lib.ef21_token_logps_grad(*args))


def test_preference_loss(lib, ptr):
    size = C.c_int64()
    assert lib.ef21_preference_loss_workspace(5, 2, C.byref(size)) == binding.EF21_OK
    need = size.value
    other = ptr + 512
    good = [ptr, 1, 5, 7, 7, ptr, 0, ptr, 2, ptr, 0.1, 0.1, 0, 0, None, ptr, ptr, other, 7, ptr, need, None]
    for args in [*bad_logits(good, ptr)] + [swap(good, at, v) for at, v in [
            (7, None), (7, ptr + 4), (8, 0), (9, None), (10, 0.0), (10, -1.0), (10, math.inf), (10, math.nan), (11, -0.1), (11, 1.0), (11, math.nan), (12, 2),
            (12, -1), (14, ptr + 1), (15, None), (16, None), (17, ptr + 1), (18, 6), (19, None), (19, ptr + 8), (20, need - 1)]]:
        refused(lib, lib.ef21_preference_loss(*args))
    for args in [(-1, 1), (2 ** 31, 1), (5, 0)]:
        refused(lib, lib.ef21_preference_loss_workspace(*args, C.byref(size)))
    refused(lib, lib.ef21_preference_loss_workspace(5, 1, None))


def test_policy_loss(lib, ptr):
    size = C.c_int64()
    assert lib.ef21_policy_loss_workspace(5, C.byref(size)) == binding.EF21_OK
    need = size.value
    other = ptr + 512
    good = [ptr, 1, 5, 7, 7, ptr, 0, ptr, ptr, ptr, ptr, 0.2, 0.2, 0.1, ptr, ptr, ptr, other, 7, ptr, need, None]
    for args in [*bad_logits(good, ptr)] + [swap(good, at, v) for at, v in [
            (7, None), (8, None), (9, None), (9, ptr + 2), (10, ptr + 1), (11, -0.1), (11, 1.1), (11, math.nan), (12, -0.1), (12, math.inf), (13, -1.0),
            (13, math.nan), (14, None), (15, None), (16, None), (17, ptr + 1), (18, 6), (19, None), (19, ptr + 8), (20, need - 1)]]:
        refused(lib, lib.ef21_policy_loss(*args))
    for args in [(-1, C.byref(size)), (2 ** 31, C.byref(size)), (5, None)]:
        refused(lib, lib.ef21_policy_loss_workspace(*args))


def test_binding_refuses_host_tensors():
    x, labels, row = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int64), torch.zeros(3)
    for call in (lambda: binding.ef21_embed(x, labels), lambda: binding.ef21_embed_grad(x[None], labels[None], 8),
                 lambda: binding.ef21_token_logps(x, labels), lambda: binding.ef21_token_logps_grad(x, labels, row, row),
                 lambda: binding.ef21_preference_loss(x, labels, torch.zeros(3, dtype=torch.int64), row, 0.1),
                 lambda: binding.ef21_policy_loss(x, labels, row, row, 0.2, 0.2)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.gpu
def test_binding_refuses_shapes_and_types():
    dev = "cuda"
    x, labels, row = torch.zeros(3, 8, device=dev), torch.zeros(3, dtype=torch.int64, device=dev), torch.zeros(3, device=dev)
    start = torch.tensor([0, 1, 3], device=dev)
    g3, t2 = torch.zeros(2, 4, 8, device=dev), torch.zeros(2, 4, dtype=torch.int64, device=dev)
    b = binding
    for error, call in [
            (TypeError, lambda: b.ef21_embed(x.double(), labels)), (TypeError, lambda: b.ef21_embed(x.t(), labels)), (TypeError, lambda: b.ef21_embed(x, row)),
            (ValueError, lambda: b.ef21_embed(x[0], labels)), (ValueError, lambda: b.ef21_embed(x, labels, out=torch.zeros(2, 8, device=dev))),
            (TypeError, lambda: b.ef21_embed(x, t2.t())), (b.EF21Error, lambda: b.ef21_embed(x, labels, math.inf)),
            (ValueError, lambda: b.ef21_embed_grad(g3, t2[:, :3], 5)), (ValueError, lambda: b.ef21_embed_grad(g3[0], t2, 5)),
            (ValueError, lambda: b.ef21_embed_grad(g3, t2, 5, accumulate=True)), (TypeError, lambda: b.ef21_embed_grad(g3, t2.float(), 5)),
            (TypeError, lambda: b.ef21_embed_grad(g3, t2, 5, out=torch.zeros(2, 5, 7, device=dev))), (b.EF21Error, lambda: b.ef21_embed_grad(g3, t2, 0)),
            (TypeError, lambda: b.ef21_embed_grad(torch.zeros(2, 9, 8, device=dev)[:, :4], t2, 5)),
            (b.EF21Error, lambda: b.ef21_embed_grad(g3, t2, 5, workspace=torch.empty(8, dtype=torch.uint8, device=dev))),
            (ValueError, lambda: b.ef21_token_logps(x, labels[:2])), (ValueError, lambda: b.ef21_token_logps(x, labels, logp=row[:2])),
            (TypeError, lambda: b.ef21_token_logps(x.long(), labels)), (TypeError, lambda: b.ef21_token_logps(x, labels.float())),
            (ValueError, lambda: b.ef21_token_logps_grad(x, labels, row, row, out=x.half())), (ValueError, lambda: b.ef21_token_logps_grad(x, labels, row[:2], row)),
            (TypeError, lambda: b.ef21_preference_loss(x, labels, start.int(), row, 0.1)), (ValueError, lambda: b.ef21_preference_loss(x, labels, start[:2], row, 0.1)),
            (ValueError, lambda: b.ef21_preference_loss(x, labels, start, row[:1], 0.1)), (b.EF21Error, lambda: b.ef21_preference_loss(x, labels, start, row, 0.0)),
            (ValueError, lambda: b.ef21_preference_loss(x, labels, start, row, 0.1, pair_weight=row)),
            (ValueError, lambda: b.ef21_policy_loss(x, labels, row, row[:1], 0.2, 0.2)), (b.EF21Error, lambda: b.ef21_policy_loss(x, labels, row, row, 0.2, 0.2, kl=0.1)),
            (ValueError, lambda: b.ef21_policy_loss(x, labels, row, row, 0.2, 0.2, weight=labels.float().cpu().cuda()[:2]))]:
        with pytest.raises(error):
            call()
