"""Plain implementations in 64 bits of the token statistics and of the operators over many tensors, and first-order bounds on what fp32 arithmetic
may put between them and the kernels.

u = 2^-24.  Entropy (nats, z = x - M with |M - max x| <= 0.35): H = log s - t / s with t = sum exp(z) z.  Beside what lm_reference derives for log s
(d_ls), a term exp(z) z is off by (3 u |z| + 2 u) from the exponential and by 2 u from z and the product, the sum of t by (V / 256 + 16) u of
sum exp(z) |z|, the quotient by d_ls and u more, and the last subtraction, product and a maximum's shift by 4 u (1 + |H| + |t| / s).
grad = a ([v = label] - p) - b p (log p + H): d_p of lm_reference; log p is off by d_ls and 2 u (|x - m| + |log p|), H by d_H, and a product or
sum rounds by u each; the storing half an ulp of its type.

AdamW: m is two products and a sum of numbers that were each rounded once before (g', the constants): 5 u (|b1 m| + |(1 - b1) g'|); v the same with
g'^2: 7 u v, of positive terms, so the root 3.5 u and its own 2 u; the denominator 12 u with its factor and eps; p 4 u of itself for decay and the
final sum, plus lr times what the quotient is off.  Numbers read on the device add 8 u to the factors.
"""
import numpy as np

import lm_reference as lm
from lm_reference import U


class Stats(lm.Rows):
    """Rows with entropy, alternatives and their bounds."""

    def __init__(self, x, labels=None):
        x = np.asarray(x, dtype=np.float64)
        self.labelled = labels is not None
        super().__init__(x, labels if self.labelled else np.zeros(len(x), np.int64))
        rows, V = x.shape
        safe = np.where(self.has[:, None], x, 0.0)
        with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
            m = safe.max(axis=1)
            m0 = np.where(self.empty, 0.0, m)[:, None]
            z = np.where(self.p > 0, safe - m0, 0.0)
            s = np.where(self.empty, 1.0, np.exp(safe - m0).sum(axis=1))[:, None]
            self.log_p = np.where(self.has[:, None], np.where(self.empty[:, None], -np.inf, (safe - m0) - np.log(s)), 0.0)
            weighed = np.where(self.p > 0, self.p * np.where(self.p > 0, self.log_p, 0.0), 0.0)
            self.entropy = np.where(self.has & ~self.empty, -weighed.sum(axis=1), 0.0)
            away = np.abs(z) + 0.35
            t = (self.p * away).sum(axis=1)
            E = (self.p * np.abs(z)).sum(axis=1)
            d_ls = U * (3 * E + 2 + V / 256 + 16 + 4 * (1 + np.abs(np.log(s[:, 0]))))
            self.d_entropy = d_ls + (self.p * away * U * (3 * away + 4)).sum(axis=1) + t * (U * (V / 256 + 17) + d_ls) + 4 * U * (1 + self.entropy + t)
            finite = np.where(np.isfinite(self.log_p), self.log_p, 0.0)
            self.d_log_p = d_ls[:, None] + 2 * U * (np.abs(np.where(np.isfinite(safe), safe, m0) - m0) + np.abs(finite))
        self.x = safe

    def top(self, k):
        """(tokens [rows][k], log-probabilities, bound): by value, ties to the lower token."""
        tokens = np.argsort(-self.x, axis=1, kind="stable")[:, :k]
        at = np.arange(len(self.x))[:, None]
        logp, bound = self.log_p[at, tokens], self.d_log_p[at, tokens]
        logp = np.where(logp < -np.finfo(np.float32).max, -np.inf, logp)          # beyond fp32
        return np.where(self.has[:, None], tokens, -1), np.where(self.has[:, None], logp, 0.0), bound

    def stats_grad(self, a, b, dtype, base=None):
        """(gradient of the logits, its bound) from those of logp (or None) and entropy (or None)."""
        rows = len(self.x)
        live = (self.has & ~self.empty)[:, None]
        a = np.zeros(rows) if a is None else np.asarray(a, np.float64)
        b = np.zeros(rows) if b is None else np.asarray(b, np.float64)
        a, b = np.where(self.has, a, 0.0)[:, None], np.where(self.has, b, 0.0)[:, None]
        hot = np.zeros_like(self.x)
        if self.labelled:
            hot[np.arange(rows)[self.has], self.labels[self.has]] = 1.0
        diff = np.where(live, hot - self.p, 0.0)
        log_p = np.where((self.p > 0) & live, np.where(np.isfinite(self.log_p), self.log_p, 0.0), 0.0)
        h, dh = self.entropy[:, None], self.d_entropy[:, None]
        bend = self.p * (log_p + h)
        g = np.where(live, a * diff - b * bend, 0.0)
        err = np.abs(a) * (self.d_p + 2 * U * np.abs(diff))
        err = err + np.abs(b) * (self.d_p * (np.abs(log_p + h) + 1) + self.p * (self.d_log_p + dh + 3 * U * (np.abs(log_p) + np.abs(h))) + 3 * U * np.abs(bend))
        err = err + U * (np.abs(a * diff) + np.abs(b * bend))
        # where p is below fp32's range log p still counts up to -200 log 2, times a p of 2^-149 at most
        err = err + np.abs(b) * 2.0 ** -126 * 140
        if base is not None:
            touched = np.broadcast_to(live, g.shape)
            g = g + base
            err = np.where(touched, err + U * np.abs(g), 0.0)
            return g, np.where(touched, err + (np.abs(g) + err) * lm.HALF_ULP[dtype] + lm.TINY[dtype], 0.0)
        return g, np.where(live, err + (np.abs(g) + err) * lm.HALF_ULP[dtype] + lm.TINY[dtype], 0.0)


# ---------------------------------------------------------------- AdamW
def mixed(x):
    x = np.asarray(x, dtype=np.uint64) & np.uint64(0xFFFFFFFF)
    low = np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(16))
    x = x * np.uint64(0x6A09E667) & low
    x = x ^ (x >> np.uint64(15))
    x = x * np.uint64(0xBB67AE85) & low
    return x ^ (x >> np.uint64(16))


def random_bits(seed, step, number, count):
    """(for m, for v, for the parameter) sixteen bits of each entry of tensor `number`."""
    key = mixed(int(seed) & 0xFFFFFFFF)
    for part in (int(seed) >> 32, step & 0xFFFFFFFF, number):
        key = mixed(key + np.uint64(part))
    i = np.arange(count, dtype=np.uint64)
    h = mixed(i ^ mixed(key + (i >> np.uint64(32))))
    return h & np.uint64(0xFFFF), h >> np.uint64(16), mixed(h + np.uint64(0x3C6EF372)) & np.uint64(0xFFFF)


GRID = {"e4m3": (3, -6), "bf16": (7, -126), "f16": (10, -14)}


def rounded(x, kind, bits=None):
    """x in 64 bits on the grid of a type: to nearest, ties to even, or by sixteen random bits.  Not decreasing in x for given bits."""
    mantissa, least = GRID[kind]
    x = np.asarray(x, np.float64)
    _, e = np.frexp(np.abs(x))
    e = np.maximum(e - 1, least) - mantissa
    units = np.ldexp(np.abs(x), -e)
    whole = np.rint(units) if bits is None else np.floor(units + (bits.astype(np.float64) + 0.5) / 65536.0)
    return np.copysign(np.ldexp(whole, e), x)


BLOCK = 256


def per_block(x, what):
    n = len(x)
    wide = np.zeros(-(-n // BLOCK) * BLOCK)
    wide[:n] = x
    return what(wide.reshape(-1, BLOCK))


def spread(scale, n):
    return np.repeat(scale, BLOCK)[:n]


class Adamw:
    """One step on one tensor in 64 bits; the arguments are the stored values.  states: m and v themselves (32 bits), or m and sqrt(v) as they are stood for."""

    def __init__(self, p, g, m, v, lr, betas, eps, decay, step, factor=1.0, eight=False, on_device=False):
        b1, b2 = betas
        more = 8 if on_device else 0
        p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
        g = g * factor
        if eight:
            v = v * v
        self.m, self.v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        self.d_m = 5 * U * (np.abs(b1 * m) + np.abs((1 - b1) * g)) + (U * np.abs(b1 * m) if eight else 0)
        self.d_v = (9 if eight else 7) * U * self.v + 2.0 ** -126
        self.root = np.sqrt(self.v)
        self.d_root = 7 * U * self.root + 2.0 ** -63
        c1, c2 = 1 / (1 - b1 ** step), 1 / np.sqrt(1 - b2 ** step)
        den = self.root * c2 + eps
        q = self.m * c1 / den
        d_q = self.d_m * c1 / den + np.abs(q) * (12 + more) * U + np.abs(q) * 2.0 ** -63 * c2 / den
        self.p = p - lr * (decay * p + q)
        self.d_p = U * 4 * (np.abs(p) + np.abs(lr * decay * p)) + abs(lr) * (d_q + 4 * U * np.abs(q)) + 2.0 ** -149

    def codes(self, bits_m, bits_v):
        """{name: (least, largest code value, scale, its bound)} for 8-bit states."""
        out = {}
        for name, x, d, bits in (("m", self.m, self.d_m, bits_m), ("v", self.root, self.d_root, bits_v)):
            scale = np.maximum(per_block(x, lambda w: np.abs(w).max(axis=1)) / 448.0, 2.0 ** -126)
            most = per_block(d, lambda w: w.max(axis=1)) / 448.0
            d_scale = most + 2 * U * scale
            s, ds = spread(scale, len(x)), spread(d_scale, len(x))
            r = x / s
            dr = d / s + np.abs(r) * (ds / s + 3 * U) + 2.0 ** -30      # below 2^-6 random rounding takes r to a multiple of 2^-29 first
            low, high = (np.clip(rounded(y, "e4m3", bits), -448, 448) for y in (r - dr, r + dr))
            if name == "v":
                floor = lambda y: np.where(self.v > 0, np.maximum(y, 2.0 ** -9), y)  # noqa: E731
                low, high = floor(low), floor(high)
                low = np.where(self.v <= self.d_v, np.minimum(low, 0.0), low)
            out[name] = low, high, scale, d_scale
        return out

    def params(self, dtype, bits=None):
        """(least, largest) value of the stored parameter."""
        if dtype == "f32":
            return self.p - self.d_p, self.p + self.d_p
        return rounded(self.p - self.d_p, dtype, bits), rounded(self.p + self.d_p, dtype, bits)


def between(got, low, high, what):
    got = np.asarray(got, np.float64)
    bad = ~((got >= low) & (got <= high))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} outside, first at {int(np.flatnonzero(bad.reshape(-1))[0])}: " \
        f"{got.reshape(-1)[bad.reshape(-1)][:3]} not in [{np.asarray(low).reshape(-1)[bad.reshape(-1)][:3]}, {np.asarray(high).reshape(-1)[bad.reshape(-1)][:3]}]"
