"""The operators on rows of logits at the ends of what they accept, against the 64-bit reference (tests/lm_reference.py)."""
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


def test_more_pairs_than_a_launch_has_workgroups(gpu):
    """2^22 + 1 pairs, all but three of them empty: the loss of an empty pair is log 2, within an ulp."""
    torch, b = gpu
    pairs, vocab, rng = 2 ** 22 + 1, 40, np.random.default_rng(0)
    lengths = np.zeros((pairs, 2), dtype=np.int64)
    full = [0, 2 ** 21 + 7, pairs - 1]
    lengths[full] = [[3, 4], [5, 2], [6, 7]]
    start = np.concatenate([[0], np.cumsum(lengths.reshape(-1))])
    rows = int(start[-1])
    x = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32)).cuda()
    labels = rng.integers(0, vocab, rows)
    labels[[1, 9]] = -100
    R = lm.Rows(as64(x), labels)
    ref = (R.logp + 0.2 * rng.standard_normal(rows)).astype(np.float32)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    loss, logp, grad = b.ef21_preference_loss(x, dev(labels), dev(start), dev(ref), 0.5, pair_weight=torch.ones(pairs, device="cuda"),
                                              out_loss=torch.full((pairs,), math.nan, device="cuda"))
    want, d_want, coef, d_coef = lm.preference(R, np.concatenate([[0], np.cumsum(lengths[full].reshape(-1))]), ref, 0.5, 0.0, False, False, np.ones(3))
    lm.inside(as64(loss[full]), want, d_want, "loss")
    lm.inside(as64(logp), R.logp, R.d_logp, "logp")
    g, bound = R.grad(coef, d_coef, "f32")
    lm.inside(as64(grad), g, bound, "gradient")
    loss[full] = math.log(2.0)
    assert float((loss.double() - math.log(2.0)).abs().max()) <= 2.0 ** -24
