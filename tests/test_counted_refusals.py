"""What ef21_adamw_counted refuses, by status through the C ABI (before any HIP call, so without a GPU)."""
import math

from test_lm_refusals import lib, ptr, refused  # noqa: F401
from test_train_refusals import options, tensor


def test_adamw_counted(lib, ptr):  # noqa: F811
    for at in (None, ptr + 4):
        refused(lib, lib.ef21_adamw_counted(tensor(ptr), 1, options(), at, None))
    for change in [dict(step_device=ptr), dict(lr=math.nan), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(lr_device=ptr + 2), dict(grad_scale=ptr + 1)]:
        refused(lib, lib.ef21_adamw_counted(tensor(ptr), 1, options(**change), ptr, None))
    for change in [dict(count=-1), dict(param=None), dict(m_scale=ptr)]:
        refused(lib, lib.ef21_adamw_counted(tensor(ptr, **change), 1, options(), ptr, None))
    refused(lib, lib.ef21_adamw_counted(tensor(ptr), -1, options(), ptr, None))
    refused(lib, lib.ef21_adamw_counted(None, 1, options(), ptr, None))
    refused(lib, lib.ef21_adamw_counted(tensor(ptr), 1, None, ptr, None))
