"""What the token statistics and the operators over many tensors refuse, by status through the C ABI (before any HIP call, so without a GPU) and by
exception in the binding; and that the binding's structures are the header's."""
import ctypes as C
import math
import os
import subprocess

import pytest
import torch

from paper_2106_05203_amd import binding
from test_lm_refusals import bad_logits, lib, ptr, refused, swap  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_token_stats(lib, ptr):  # noqa: F811
    size = C.c_int64()
    assert lib.ef21_token_stats_workspace(1, 5, 7, 3, C.byref(size)) == binding.EF21_OK
    good = [ptr, 1, 5, 7, 7, ptr, 0, 3, ptr, ptr, ptr, ptr, ptr, None, ptr, max(size.value, 1), None]
    bad = [args for args in bad_logits(good, ptr) if args[5] is not None]
    for args in bad + [swap(good, at, v) for at, v in [(5, None), (7, -1), (7, 8), (8, None), (8, ptr + 1), (9, None), (9, ptr + 2), (10, None), (11, None), (11, ptr + 2),
                                                       (12, None), (13, ptr + 2)]]:
        refused(lib, lib.ef21_token_stats(*args))
    refused(lib, lib.ef21_token_stats(*swap(swap(good, 3, 100), 4, 100)[:7], 65, *good[8:]))
    for args in [(3, 1, 7, 3), (1, -1, 7, 3), (1, 2 ** 31, 7, 3), (1, 1, 0, 0), (1, 1, 2 ** 31, 3), (1, 1, 7, 8), (1, 1, 7, -1), (1, 1, 100, 65)]:
        refused(lib, lib.ef21_token_stats_workspace(*args, C.byref(size)))
    refused(lib, lib.ef21_token_stats_workspace(1, 5, 7, 3, None))
    # a few long rows need workspace
    assert lib.ef21_token_stats_workspace(1, 1, 131072, 20, C.byref(size)) == binding.EF21_OK
    if size.value:
        good = [ptr, 1, 1, 131072, 131072, ptr, 0, 20, ptr, ptr, ptr, ptr, ptr, None, ptr, size.value, None]
        for at, value in [(14, None), (14, ptr + 8), (15, size.value - 1), (15, -1)]:
            refused(lib, lib.ef21_token_stats(*swap(good, at, value)))


def test_token_stats_grad(lib, ptr):  # noqa: F811
    other = ptr + 512
    good = [ptr, 1, 5, 7, 7, ptr, 0, ptr, ptr, ptr, ptr, other, 7, 0, None]
    bad = [args for args in bad_logits(good, ptr) if args[5] is not None]
    for args in bad + [swap(good, at, v) for at, v in [(5, None), (7, None), (7, ptr + 2), (8, None), (9, ptr + 1), (10, ptr + 2), (11, None), (11, other + 1), (12, 6)]]:
        refused(lib, lib.ef21_token_stats_grad(*args))
    refused(lib, lib.ef21_token_stats_grad(*swap(swap(good, 11, ptr), 12, 8)))
    refused(lib, lib.ef21_token_stats_grad(*swap(swap(good, 11, ptr), 13, 1)))


def tensor(ptr, **change):  # noqa: F811
    fields = dict(param=ptr, grad=ptr + 256, m=ptr + 512, v=ptr + 768, m_scale=None, v_scale=None, copy=None, count=8, param_type=0, grad_type=1, copy_type=0, weight_decay=0.0)
    fields.update(change)
    return (binding.AdamwTensor * 1)(binding.AdamwTensor(**fields))


def options(**change):
    fields = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, lr_device=None, step_device=None, grad_scale=None, seed=0, stochastic=0)
    fields.update(change)
    return C.byref(binding.AdamwOptions(**fields))


def test_adamw(lib, ptr):  # noqa: F811
    for change in [dict(count=-1), dict(count=2 ** 33 + 1), dict(param_type=3), dict(grad_type=-1), dict(weight_decay=math.inf), dict(weight_decay=math.nan), dict(param=None),
                   dict(param=ptr + 2), dict(grad=None), dict(grad=ptr + 1), dict(m=None), dict(v=None), dict(m=ptr + 2), dict(v=ptr + 1), dict(m_scale=ptr),
                   dict(v_scale=ptr), dict(m_scale=ptr + 2, v_scale=ptr), dict(m_scale=ptr, v_scale=ptr + 1), dict(copy=ptr, copy_type=0), dict(copy=ptr, copy_type=3),
                   dict(copy=ptr + 1, copy_type=1), dict(copy=ptr, copy_type=1, param_type=1)]:
        refused(lib, lib.ef21_adamw(tensor(ptr, **change), 1, options(), None))
    for change in [dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=math.nan), dict(beta2=1.0), dict(beta2=-1.0), dict(eps=0.0), dict(eps=-1.0),
                   dict(eps=math.inf), dict(eps=1e-60), dict(eps=1e-38), dict(eps=math.nan), dict(step=0), dict(step=-3), dict(lr_device=ptr + 2), dict(step_device=ptr + 4), dict(grad_scale=ptr + 1)]:
        refused(lib, lib.ef21_adamw(tensor(ptr), 1, options(**change), None))
    refused(lib, lib.ef21_adamw(tensor(ptr), -1, options(), None))
    refused(lib, lib.ef21_adamw(None, 1, options(), None))
    refused(lib, lib.ef21_adamw(tensor(ptr), 1, None, None))


def test_grad_norm(lib, ptr):  # noqa: F811
    size = C.c_int64()
    assert lib.ef21_grad_norm_workspace(1, C.byref(size)) == binding.EF21_OK and size.value > 0
    one = lambda kind, v: (kind * 1)(v)  # noqa: E731
    good = [one(C.c_void_p, ptr), one(C.c_int32, 1), one(C.c_int64, 8), 1, 1.0, 1.0, ptr, ptr + 4, ptr + 256, size.value, None]
    for at, value in [(0, None), (0, one(C.c_void_p, None)), (0, one(C.c_void_p, ptr + 1)), (1, None), (1, one(C.c_int32, 3)), (2, None), (2, one(C.c_int64, -1)),
                      (2, one(C.c_int64, 2 ** 33 + 1)), (3, -1), (4, 0.0), (4, -1.0), (4, math.nan), (4, math.inf), (5, 0.0), (5, math.nan), (5, -1.0), (6, None), (6, ptr + 2),
                      (7, None), (8, None), (8, ptr + 8), (9, size.value - 1), (9, -1)]:
        refused(lib, lib.ef21_grad_norm(*swap(good, at, value)))
    refused(lib, lib.ef21_grad_norm_workspace(-1, C.byref(size)))
    refused(lib, lib.ef21_grad_norm_workspace(1, None))


def test_binding_refuses_host_tensors():
    x, labels, row, sums = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int64), torch.zeros(3), torch.zeros(3, 2)
    for call in (lambda: binding.ef21_token_stats(x, labels), lambda: binding.ef21_token_stats(x), lambda: binding.ef21_token_stats_grad(x, labels, sums, row),
                 lambda: binding.ef21_grad_norm([x]), lambda: binding.TensorList([x]), lambda: binding.AdamW([x])):
        with pytest.raises(TypeError):
            call()


def test_structures_are_the_headers(tmp_path):
    """Sizes and offsets of the two structures, from the C compiler."""
    lines = []
    for c_name, kind in (("ef21_adamw_tensor", binding.AdamwTensor), ("ef21_adamw_options", binding.AdamwOptions)):
        lines.append(f'printf("%zu\\n", sizeof({c_name}));')
        lines += [f'printf("%zu\\n", offsetof({c_name}, {name}));' for name, _ in kind._fields_]
    source = tmp_path / "sizes.c"
    source.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ef21.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "sizes"), str(source)])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "sizes")]).split()]
    want = []
    for kind in (binding.AdamwTensor, binding.AdamwOptions):
        want.append(C.sizeof(kind))
        want += [getattr(kind, name).offset for name, _ in kind._fields_]
    assert got == want


@pytest.mark.gpu
def test_binding_refuses_shapes_and_types():
    dev = "cuda"
    b = binding
    x, labels, row, sums = torch.zeros(3, 8, device=dev), torch.zeros(3, dtype=torch.int64, device=dev), torch.zeros(3, device=dev), torch.zeros(3, 2, device=dev)
    for error, call in [
            (ValueError, lambda: b.ef21_token_stats(x, labels[:2])), (TypeError, lambda: b.ef21_token_stats(x.double(), labels)), (TypeError, lambda: b.ef21_token_stats(x.t(), None)),
            (ValueError, lambda: b.ef21_token_stats(x, None, 0, logp=row)), (b.EF21Error, lambda: b.ef21_token_stats(x, labels, 9)),
            (b.EF21Error, lambda: b.ef21_token_stats(x, labels, -1)), (ValueError, lambda: b.ef21_token_stats(x, labels, 2, top_logp=sums[:2])),
            (TypeError, lambda: b.ef21_token_stats(x, labels, 2, top_tokens=sums)), (ValueError, lambda: b.ef21_token_stats(x, labels, 0, top_logp=sums)),
            (ValueError, lambda: b.ef21_token_stats(x, labels, sums=row)), (ValueError, lambda: b.ef21_token_stats(x, labels, entropy=row[:2])),
            (ValueError, lambda: b.ef21_token_stats_grad(x, labels, row, row)), (ValueError, lambda: b.ef21_token_stats_grad(x, labels, sums, row, row[:2])),
            (b.EF21Error, lambda: b.ef21_token_stats_grad(x, None, sums, row, row)), (ValueError, lambda: b.ef21_token_stats_grad(x, labels, sums, row, accumulate=True)),
            (b.EF21Error, lambda: b.ef21_token_stats_grad(x, labels, sums, row, out=x, accumulate=True)),
            (ValueError, lambda: b.ef21_token_stats_grad(x, labels, sums, row, out=x.half()))]:
        with pytest.raises(error):
            call()
