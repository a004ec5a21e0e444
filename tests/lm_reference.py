"""Plain implementations in 64 bits of the operators at the two ends of a language model, and first-order bounds on what fp32
arithmetic may put between them and the kernels.

u = 2^-24.  For a row x with maximum m, s = sum exp(x - m), lse = m + log s:
  - exp(x - m) is taken as 2^((x - m) log2 e): a subtraction, a product with a rounded constant and the hardware's exponential (one ulp), so
    its relative error is at most 3 u |x - m| + 2 u; weighted over the sum that is 3 u E + 2 u with E = sum p |x - m|;
  - s is added up in runs of at most V / 256 entries per thread, then in a tree: (V / 256 + 16) u;
  - the logarithm: 4 u (1 + |log s|) is ample, and d_ls is the sum of these three;
  - lse = m + log s adds 2 u (|m| + |lse|), logp = (x_label - m) - log s adds 2 u (|x_label - m| + |logp|).
grad = c ([v = label] - p), p = 2^((x - m - log s) log2 e): relative error of p 3 u (|x - m| + |x - lse| + |log s|) + 4 u + d_ls, and where p is formed
from lse, which the library does while |lse| <= 64, 2 u (|m| + |lse|) more; the difference and the
product one rounding each, the storing half an ulp of its type.  A coefficient c that is itself computed brings its own error.
"""
import numpy as np
import torch

U = 2.0 ** -24
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {name: torch.finfo(t).eps / 2 for name, t in TORCH.items()}          # relative
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}            # absolute, where the type's numbers end


class Rows:
    """lse, logp, softmax and their error bounds for logits x [rows][V] (float64, exactly the stored values) and labels."""

    def __init__(self, x, labels):
        x = np.asarray(x, dtype=np.float64)
        labels = np.asarray(labels, dtype=np.int64)
        rows, V = x.shape
        self.has = (labels >= 0) & (labels < V)
        self.labels, self.V = labels, V
        at = np.where(self.has, labels, 0)
        safe = np.where(self.has[:, None], x, 0.0)
        with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
            m = safe.max(axis=1) if V else np.zeros(rows)
            self.empty = self.has & (m == -np.inf)
            m0 = np.where(self.empty, 0.0, m)
            e = np.exp(safe - m0[:, None])
            s = e.sum(axis=1)
            lse = np.where(self.empty, -np.inf, m0 + np.log(s))
            label_x = safe[np.arange(rows), at]
            self.logp = np.where(self.has, np.where(self.empty, -np.inf, (label_x - m0) - np.log(s)), 0.0)
            self.lse = np.where(self.has, lse, 0.0)
            self.p = np.where((self.has & ~self.empty)[:, None], e / s[:, None], 0.0)
            dist = np.where(e > 0, m0[:, None] - safe, 0.0)
            E = (self.p * dist).sum(axis=1)
            logs = np.abs(np.where(self.empty, 0.0, np.log(s)))
            fl = np.where(np.isfinite(self.lse), np.abs(self.lse), 0.0)
            fp = np.where(np.isfinite(self.logp), np.abs(self.logp), 0.0)
            d_ls = U * (3 * E + 2 + V / 256 + 16 + 4 * (1 + logs))
            self.d_lse = d_ls + 2 * U * (np.abs(m0) + fl)
            self.d_logp = d_ls + 2 * U * (np.where(np.isfinite(label_x), np.abs(label_x - m0), 0.0) + fp)
            away = np.where(self.p > 0, 3 * dist + 3 * np.abs(safe - np.where(self.empty, 0.0, m0 + np.log(s))[:, None]), 0.0)
            whole = np.where(fl <= 64, 2 * (np.abs(m0) + fl), 0.0)
            self.d_p = self.p * (U * (away + 3 * logs[:, None] + 4 + whole[:, None]) + d_ls[:, None]) + 2.0 ** -126

    def grad(self, coef, d_coef, dtype):
        """(gradient of the logits, its bound) for coefficients [rows] with error d_coef."""
        rows = len(coef)
        c = np.where(self.has & ~self.empty, coef, 0.0)[:, None]
        dc = np.where(self.has & ~self.empty, d_coef, 0.0)[:, None]
        hot = np.zeros((rows, self.V))
        hot[np.arange(rows)[self.has], self.labels[self.has]] = 1.0
        hot[self.empty] = 0.0
        diff = hot - self.p
        g = c * diff
        err = np.abs(c) * (self.d_p + U * np.abs(diff)) + dc * (np.abs(diff) + self.d_p) + U * np.abs(g)
        return g, err + (np.abs(g) + err) * HALF_ULP[dtype] + TINY[dtype]


def preference(R, start, ref, beta, smoothing, least_squares, mean, weight):
    """(loss [pairs], its bound, coef [rows], its bound) from Rows R."""
    rows, pairs = len(R.logp), (len(start) - 1) // 2
    ref = np.asarray(ref, dtype=np.float64)
    loss, d_loss = np.zeros(pairs), np.zeros(pairs)
    coef, d_coef = np.zeros(rows), np.zeros(rows)
    for p in range(pairs):
        S, dS, per = [], [], []
        for s in (2 * p, 2 * p + 1):
            at = np.arange(start[s], start[s + 1])
            at = at[R.has[at]]
            k = 1.0 / len(at) if mean and len(at) else 1.0
            S.append(k * np.sum(R.logp[at] - ref[at]))
            dS.append(k * np.sum(R.d_logp[at]))
            per.append(k)
        D, dD = S[0] - S[1], dS[0] + dS[1]
        if least_squares:
            off = D - 1.0 / (2.0 * beta)
            L, slope, curve = off * off, 2.0 * off, 2.0
        else:
            z = beta * D
            L = (1 - smoothing) * np.logaddexp(0.0, -z) + smoothing * np.logaddexp(0.0, z)
            slope = beta * ((1 - smoothing) * -np.exp(-np.logaddexp(0.0, z)) + smoothing * np.exp(-np.logaddexp(0.0, -z)))
            curve = beta * beta / 4.0
        loss[p] = L
        d_loss[p] = abs(slope) * dD + curve * dD * dD + 2 * U * abs(L) + 1e-15
        w = weight[p] if weight is not None else 1.0 / pairs
        for side, s in enumerate((2 * p, 2 * p + 1)):
            coef[start[s]:start[s + 1]] = w * (slope if side == 0 else -slope) * per[side]
            d_coef[start[s]:start[s + 1]] = abs(w) * per[side] * (curve * dD + 2 * U * abs(slope))
    return loss, d_loss, coef, d_coef


def policy(R, old, adv, lo, hi, ref, kl, weight):
    """(token loss, its bound, total, its bound, coef, its bound)."""
    rows = len(R.logp)
    old, adv = np.asarray(old, np.float64), np.asarray(adv, np.float64)
    w = np.asarray(weight, np.float64) if weight is not None else np.full(rows, 1.0 / rows)
    with np.errstate(over="ignore", invalid="ignore"):
        q = np.exp(R.logp - old)
        one, two = q * adv, np.clip(q, 1 - lo, 1 + hi) * adv
        loss = -np.minimum(one, two)
        slope = np.where(one <= two, -one, 0.0)
        dq = q * (R.d_logp + U * (2 * np.abs(R.logp - old) + 6))
        d_loss = np.abs(adv) * (dq + 3 * U * (q + 1))
        d_slope = np.where(one <= two, np.abs(adv) * (dq + 3 * U * q), 0.0)
        if kl:
            o = np.asarray(ref, np.float64) - R.logp
            e = np.expm1(o)
            loss = loss + kl * (e - o)
            slope = slope - kl * e
            do = R.d_logp + U * np.abs(o)
            d_loss = d_loss + kl * (np.abs(e) * do + U * (6 * np.abs(e) + 3 * np.abs(o))) + 2 * U * np.abs(loss)
            d_slope = d_slope + kl * ((np.abs(e) + 1) * do + 8 * U * np.abs(e)) + 2 * U * np.abs(slope)
    has = R.has
    loss, d_loss = np.where(has, loss, 0.0), np.where(has, d_loss, 0.0)
    total = np.sum(np.where(has, w * loss, 0.0))
    d_total = np.sum(np.where(has, np.abs(w) * d_loss, 0.0)) + 2 * U * abs(total)
    return loss, d_loss, total, d_total, np.where(has, w * slope, 0.0), np.where(has, np.abs(w) * d_slope + 2 * U * np.abs(w * slope), 0.0)


def embed_grad(grad_out, tokens, vocab, scale, base=None):
    """(gradient [n][vocab][width] in 64 bits, bound): an entry with c terms is off by at most (c + 3) u times the sum of the terms' sizes, and with a
    base by one rounding of the result more."""
    g = np.asarray(grad_out, dtype=np.float64)
    n, count, width = g.shape
    out, size, terms = np.zeros((n, vocab, width)), np.zeros((n, vocab, width)), np.zeros((n, vocab, 1))
    for i in range(n):
        t = np.asarray(tokens[i], dtype=np.int64)
        ok = (t >= 0) & (t < vocab)
        np.add.at(out[i], t[ok], g[i][ok])
        np.add.at(size[i], t[ok], np.abs(g[i][ok]))
        np.add.at(terms[i], t[ok], 1.0)
    bound = (terms + 3) * U * size * abs(scale)
    out = out * scale
    if base is not None:
        out = out + np.asarray(base, dtype=np.float64)
        bound = bound + np.where(terms > 0, 2 * U * np.abs(out), 0.0)
    return out, bound


def inside(got, ref, bound, what):
    """Asserts |got - ref| <= bound entry by entry, infinities and NaN in the same places."""
    got = np.asarray(got, dtype=np.float64)
    odd = ~np.isfinite(ref)
    assert np.array_equal(got[odd], np.asarray(ref)[odd], equal_nan=True), f"{what}: infinities or NaN differ"
    err = np.abs(np.where(odd, 0.0, got) - np.where(odd, 0.0, ref))
    bad = ~(err <= np.where(odd, 0.0, bound))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} outside, worst error {np.nanmax(err):.3e} where {np.asarray(bound)[np.unravel_index(np.nanargmax(err - bound), err.shape)]:.3e} is allowed"
