"""The operators at the two ends of a language model whose gradients this library compresses, as a program calls them.

Kinds of case:

  embed       ef21_embed: lookup of table rows, scaled, in the activations' type
  embed_grad  ef21_embed_grad: n workers' gradients of the table from the tokens, written as rows of [n][vocab][width] or
              added to what a tied output layer has left there
  logps       ef21_token_logps, and with backward=True ef21_token_logps_grad: log-probabilities of the label tokens
  preference  ef21_preference_loss: the paired loss on log ratios, logistic or least squares, with the gradient of the logits
  policy      ef21_policy_loss: the clipped policy loss with a KL term, with the gradient of the logits

Rows whose label is -100 (prompt tokens, padding) are ignored; their logits hold NaN here, as memory that nobody filled would.
Inputs are drawn on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
IGNORE = -100


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one decoding step of a small batch: eight tokens, latency alone
        dict(name="embed_decode", kind="embed", vocab=65536, width=4096, tokens=8, table="bf16", out="bf16", scale=1.0, wide=True),
        # the forward lookup of a whole step of 20 workers (the worker count of the headline problem) in an fp32 model
        dict(name="embed_step", kind="embed", vocab=50000, width=1024, tokens=81920, table="f32", out="bf16", scale=32.0, wide=True),
        # a toy model at the smallest test configuration's size: 4 workers, 250 tokens each, width 100, an odd vocabulary
        dict(name="embed_grad_small", kind="embed_grad", n=4, tokens=250, vocab=1001, width=100, dtype="f32", scale=10.0, add=False, wide=False),
        # eight workers' dense gradient rows, as the compressed step takes them: most table rows get no token
        dict(name="embed_grad_workers", kind="embed_grad", n=8, tokens=2048, vocab=32768, width=1024, dtype="bf16", scale=1.0, add=False, wide=True),
        # one long batch added to the gradient that the tied output layer left: few tokens with very many positions
        dict(name="embed_grad_tied", kind="embed_grad", n=1, tokens=65536, vocab=131072, width=2048, dtype="bf16", scale=1.0, add=True, wide=True),
        # scoring the tokens of one decoding step of sixteen sequences
        dict(name="logps_decode", kind="logps", rows=16, vocab=65536, dtype="bf16", ignored=0.0, padded=0, backward=False, wide=True),
        # log-probabilities in training, forward and backward: an odd vocabulary, so no two rows are aligned alike
        dict(name="logps_train", kind="logps", rows=8192, vocab=50001, dtype="f16", ignored=0.125, padded=0, backward=True, wide=True),
        # paired loss of a toy model in fp32, least squares on the mean log ratio
        dict(name="preference_small", kind="preference", pairs=4, length=25, vocab=1000, dtype="f32", loss=1, mean=True, beta=0.5, smoothing=0.0,
             ignored=0.25, padded=0, wide=False),
        # a training step of sixteen pairs of about 512 tokens a sequence, prompts ignored
        dict(name="preference_step", kind="preference", pairs=16, length=512, vocab=32768, dtype="bf16", loss=0, mean=False, beta=0.1, smoothing=0.1,
             ignored=0.25, padded=0, wide=True),
        # a policy step on a few tokens
        dict(name="policy_small", kind="policy", rows=64, vocab=5000, dtype="f16", kl=0.0, ignored=0.0, padded=0, wide=False),
        # fp32 logits with a vocabulary padded to a multiple of 64 by columns of -inf, an odd number of rows
        dict(name="policy_padded", kind="policy", rows=2001, vocab=32064, dtype="f32", kl=0.04, ignored=0.125, padded=63, wide=False),
        # the largest: 8192 tokens of a large vocabulary
        dict(name="policy_step", kind="policy", rows=8192, vocab=131072, dtype="bf16", kl=0.04, ignored=0.125, padded=0, wide=True),
    ]


def _log_int(rng, lo, hi):
    """A whole number in [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "logps", "preference", "policy"])
    wide = rng.random() < 0.5                                            # 64-bit tokens or 32-bit ones
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind == "embed":
        width = _log_int(rng, 32, 8192)
        if rng.random() < 0.6:
            width = -(-width // 16) * 16
        vocab = _log_int(rng, 1000, min(131072, 400000000 // width))
        tokens = _log_int(rng, 1, min(131072, 200000000 // width))
        return dict(kind=kind, vocab=vocab, width=width, tokens=tokens, table=dtype, out=rng.choice([dtype, dtype, "bf16"]),
                    scale=rng.choice([1.0, math.sqrt(width)]), wide=wide)
    if kind == "embed_grad":
        width = _log_int(rng, 32, 4096)
        if rng.random() < 0.6:
            width = -(-width // 16) * 16
        n = _log_int(rng, 1, 20)
        vocab = _log_int(rng, 500, max(500, min(131072, 300000000 // (n * width))))
        tokens = _log_int(rng, 50, max(50, min(65536, 150000000 // (n * width))))
        return dict(kind=kind, n=n, tokens=tokens, vocab=vocab, width=width, dtype=dtype, scale=rng.choice([1.0, math.sqrt(width)]),
                    add=rng.random() < 0.4, wide=wide)
    vocab = _log_int(rng, 500, 131072)
    if rng.random() < 0.5:
        vocab = -(-vocab // 64) * 64
    most = max(2, min(16384, 500000000 // vocab))                        # rows
    padded = rng.choice([0, 0, vocab % 64 and 1, 17])
    ignored = rng.choice([0.0, 0.125, 0.3])
    if kind == "logps":
        return dict(kind=kind, rows=_log_int(rng, 1, most), vocab=vocab, dtype=dtype, ignored=ignored, padded=padded, backward=rng.random() < 0.6, wide=wide)
    if kind == "preference":
        pairs = _log_int(rng, 1, min(32, most // 2))
        length = _log_int(rng, 1, max(1, min(1024, most // (2 * pairs))))
        loss = rng.choice([0, 0, 1])                                     # least squares goes with mean log ratios
        return dict(kind=kind, pairs=pairs, length=length, vocab=vocab, dtype=dtype, loss=loss, mean=loss == 1 or rng.random() < 0.2,
                    beta=rng.choice([0.1, 0.5]), smoothing=rng.choice([0.0, 0.1]), ignored=ignored, padded=padded, wide=wide)
    return dict(kind=kind, rows=_log_int(rng, 1, most), vocab=vocab, dtype=dtype, kl=rng.choice([0.0, 0.04]), ignored=ignored, padded=padded, wide=wide)


def _rows(c):
    return 2 * c["pairs"] * c["length"] if c["kind"] == "preference" else c["rows"]


def _ignored(c):
    """Rows without a label: the same number for every seed, and never all of them."""
    return min(_rows(c) - 1, int(round(c["ignored"] * _rows(c))))


# ---------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _tokens(g, shape, vocab, wide):
    """Tokens by Zipf's law: the logarithm of the rank is uniform."""
    u = torch.rand(shape, generator=g, device=DEV, dtype=torch.float64)
    t = ((float(vocab) + 1.0) ** u - 1.0).to(torch.int64).clamp_(0, vocab - 1)
    return t if wide else t.to(torch.int32)


def _logits(c, g):
    """(logits, labels, the labels' log-probabilities): normal logits with the label's raised; -inf in the padding columns;
    NaN in the rows without a label."""
    rows, vocab, real = _rows(c), c["vocab"], c["vocab"] - c["padded"]
    x = torch.randn(rows, vocab, generator=g, device=DEV, dtype=TYPES[c["dtype"]]).mul_(2.0)
    if c["padded"]:
        x[:, real:] = -math.inf
    labels = _tokens(g, (rows,), real, True)
    at = torch.arange(rows, device=DEV)
    x[at, labels] += torch.rand(rows, generator=g, device=DEV).mul_(6.0).add_(4.0).to(x.dtype)
    logp = torch.empty(rows, device=DEV)
    some = max(1, 100000000 // vocab)
    for r in range(0, rows, some):
        part = x[r:r + some].float()
        logp[r:r + some] = part.gather(1, labels[r:r + some, None])[:, 0] - torch.logsumexp(part, 1)
    k = _ignored(c)
    if k:
        out = torch.randperm(rows, generator=g, device=DEV)[:k]
        labels[out] = IGNORE
        x[out] = math.nan
    return x, labels if c["wide"] else labels.to(torch.int32), logp


def prepare(case, seed):
    c, g = case, _generator(seed)
    s = {"case": c}
    randn = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    if c["kind"] == "embed":
        s["table"] = randn(c["vocab"], c["width"]).mul_(0.02).to(TYPES[c["table"]])
        s["tokens"] = _tokens(g, (c["tokens"],), c["vocab"], c["wide"])
        s["out"] = torch.empty(c["tokens"], c["width"], device=DEV, dtype=TYPES[c["out"]])
    elif c["kind"] == "embed_grad":
        s["grad_out"] = randn(c["n"], c["tokens"], c["width"]).mul_(1e-3).to(TYPES[c["dtype"]])
        s["tokens"] = _tokens(g, (c["n"], c["tokens"]), c["vocab"], c["wide"])
        shape = (c["n"], c["vocab"], c["width"])
        s["out"] = randn(*shape).mul_(1e-3) if c["add"] else torch.empty(shape, device=DEV)
    else:
        s["logits"], s["labels"], logp = _logits(c, g)
        rows = _rows(c)
        s["logp"], s["lse"] = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        if c["kind"] != "logps" or c["backward"]:
            s["grad"] = torch.empty_like(s["logits"])
        if c["kind"] == "logps":
            s["grad_logp"] = randn(rows).mul_((1024.0 if c["dtype"] == "f16" else 1.0) / rows)   # gradients in f16 go with a loss scale
        elif c["kind"] == "preference":
            # ragged lengths with the same sum for every seed, among them now and then none
            cuts = torch.randint(0, rows + 1, (2 * c["pairs"] - 1,), generator=g, device=DEV)
            s["start"] = torch.cat([torch.zeros(1, device=DEV, dtype=torch.int64), cuts.sort().values,
                                    torch.full((1,), rows, device=DEV, dtype=torch.int64)])
            s["ref"] = logp + randn(rows).mul_(0.2)
            s["loss"] = torch.empty(c["pairs"], device=DEV)
        else:
            # The gradient jumps where the ratio meets the clip range's edge on the side that clips it, and there rounding alone
            # decides: no drawn log ratio lies within 0.002 of an edge.
            d = randn(rows).mul_(0.15)
            for edge in (math.log(0.8), math.log(1.28)):
                d = torch.where((d - edge).abs() < 0.002, torch.full_like(d, edge + 0.004), d)
            s["old"] = logp - d
            s["ref"] = logp + randn(rows).mul_(0.1)
            s["advantages"] = randn(-(-rows // 64)).repeat_interleave(64)[:rows].contiguous()
            s["weight"] = (s["labels"] >= 0).float() / max(1, rows - _ignored(c))
            s["loss"], s["token_loss"] = torch.empty(1, device=DEV), torch.empty(rows, device=DEV)
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2106_05203_amd import binding as b
    c = s["case"]
    if c["kind"] == "embed":
        return {"out": b.ef21_embed(s["table"], s["tokens"], c["scale"], out=s["out"])}
    if c["kind"] == "embed_grad":
        return {"grad": b.ef21_embed_grad(s["grad_out"], s["tokens"], c["vocab"], c["scale"], out=s["out"], accumulate=c["add"])}
    if c["kind"] == "logps":
        logp, lse = b.ef21_token_logps(s["logits"], s["labels"], logp=s["logp"], lse=s["lse"])
        if not c["backward"]:
            return {"logp": logp, "lse": lse}
        return {"logp": logp, "lse": lse, "grad": b.ef21_token_logps_grad(s["logits"], s["labels"], lse, s["grad_logp"], out=s["grad"])}
    if c["kind"] == "preference":
        loss, logp, grad = b.ef21_preference_loss(s["logits"], s["labels"], s["start"], s["ref"], c["beta"], smoothing=c["smoothing"], loss=c["loss"],
                                                  mean=c["mean"], out_loss=s["loss"], logp=s["logp"], grad=s["grad"])
        return {"loss": loss, "logp": logp, "grad": grad}
    loss, token_loss, logp, grad = b.ef21_policy_loss(s["logits"], s["labels"], s["old"], s["advantages"], 0.2, 0.28, ref_logp=s["ref"], kl=c["kl"],
                                                      weight=s["weight"], out_loss=s["loss"], token_loss=s["token_loss"], logp=s["logp"], grad=s["grad"])
    return {"loss": loss, "token_loss": token_loss, "logp": logp, "grad": grad}


def _plain_logps(s):
    """(the logits' exponentials, their sums, label or 0, labelled, logp, lse) in fp32; rows without a label give logp = lse = 0."""
    labels = s["labels"].long()
    has = labels >= 0
    x = torch.where(has[:, None], s["logits"], 0.0).float()
    at = labels.clamp(min=0)
    m = x.amax(1, keepdim=True)
    p = torch.exp(x - m)
    total = p.sum(1, keepdim=True)
    lse = (m + torch.log(total))[:, 0]
    logp = torch.where(has, x.gather(1, at[:, None])[:, 0] - lse, 0.0)
    return p, total, at, has, logp, torch.where(has, lse, 0.0)


def _plain_grad(p, total, at, has, coef, dtype):
    """coef (one-hot - softmax) of every row, rounded once."""
    coef = torch.where(has, coef, 0.0)
    grad = p.mul_(-coef[:, None] / total)
    grad[torch.arange(len(at), device=DEV), at] += coef
    return grad.to(dtype)


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "embed":
        return {"out": (s["table"][s["tokens"].long()].float() * c["scale"]).to(TYPES[c["out"]])}
    if c["kind"] == "embed_grad":
        grad = s["out"] if c["add"] else torch.zeros_like(s["out"])
        first = torch.arange(c["n"], device=DEV)[:, None] * c["vocab"]
        grad.view(-1, c["width"]).index_add_(0, (s["tokens"].long() + first).view(-1), s["grad_out"].float().view(-1, c["width"]), alpha=c["scale"])
        return {"grad": grad}
    p, total, at, has, logp, lse = _plain_logps(s)
    dtype = s["logits"].dtype
    if c["kind"] == "logps":
        out = {"logp": logp, "lse": lse}
        if c["backward"]:
            out["grad"] = _plain_grad(p, total, at, has, s["grad_logp"], dtype)
        return out
    if c["kind"] == "preference":
        sequence = torch.searchsorted(s["start"], torch.arange(len(at), device=DEV), right=True) - 1
        ratio = torch.zeros(2 * c["pairs"], device=DEV).index_add_(0, sequence, torch.where(has, logp - s["ref"], 0.0))
        per = torch.ones(2 * c["pairs"], device=DEV)
        if c["mean"]:
            per = torch.zeros(2 * c["pairs"], device=DEV).index_add_(0, sequence, has.float()).clamp(min=1.0)
        ratio = (ratio / per).view(-1, 2)
        margin = ratio[:, 0] - ratio[:, 1]
        if c["loss"] == 0:
            z, e = c["beta"] * margin, c["smoothing"]
            soft = torch.log1p(torch.exp(-z.abs()))
            loss = (1 - e) * (soft + torch.clamp(-z, min=0.0)) + e * (soft + torch.clamp(z, min=0.0))
            slope = c["beta"] * (1.0 / (1.0 + torch.exp(-z)) - (1 - e))
        else:
            off = margin - 0.5 / c["beta"]
            loss, slope = off * off, 2.0 * off
        slope = torch.stack([slope, -slope], 1).view(-1) / per / c["pairs"]
        return {"loss": loss, "logp": logp, "grad": _plain_grad(p, total, at, has, slope[sequence], dtype)}
    ratio, adv = torch.exp(logp - s["old"]), s["advantages"]
    one, two = ratio * adv, ratio.clamp(0.8, 1.28) * adv
    off = s["ref"] - logp
    token_loss = torch.where(has, c["kl"] * (torch.expm1(off) - off) - torch.minimum(one, two), 0.0)
    slope = s["weight"] * (-torch.where(one <= two, one, 0.0) - c["kl"] * torch.expm1(off))
    return {"loss": (s["weight"] * token_loss).sum().view(1), "token_loss": token_loss, "logp": logp, "grad": _plain_grad(p, total, at, has, slope, dtype)}


# ---------------------------------------------------------------- what a pass cannot do without
def _distinct(tokens, vocab):
    """Different tokens expected among so many drawn by _tokens."""
    edge = np.log(np.arange(1, vocab + 2, dtype=np.float64)) / math.log(vocab + 1.0)
    return float(np.sum(-np.expm1(tokens * np.log1p(-np.diff(edge)))))


def work(case):
    c = case
    size = lambda t: 4 if t == "f32" else 2  # noqa: E731
    token = 8 if c["wide"] else 4
    if c["kind"] == "embed":
        n = c["tokens"]
        return {"bytes": n * token + _distinct(n, c["vocab"]) * c["width"] * size(c["table"]) + n * c["width"] * size(c["out"]), "flops": n * c["width"]}
    if c["kind"] == "embed_grad":
        n = c["n"] * c["tokens"]
        rows = 2 * _distinct(c["tokens"], c["vocab"]) if c["add"] else c["vocab"]
        return {"bytes": n * (token + c["width"] * size(c["dtype"])) + c["n"] * rows * c["width"] * 4, "flops": n * c["width"]}
    rows, b = _rows(c), size(c["dtype"])
    read = (rows - _ignored(c)) * c["vocab"]                             # rows without a label need not be read
    small = {"logps": 8 + (8 if c.get("backward") else 0), "preference": 8, "policy": 24}[c["kind"]]
    backward = c["kind"] != "logps" or c["backward"]
    return {"bytes": read * b + (rows * c["vocab"] * b if backward else 0) + rows * (token + small), "flops": read * (7 if backward else 4)}


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "embed":
        return {"out": torch.index_select(s["table"], 0, s["tokens"].reshape(-1).to(torch.int64)).double() * c["scale"]}
    if c["kind"] == "embed_grad":
        out = s["out"].double() if c["add"] else torch.zeros(s["out"].shape, device=DEV, dtype=torch.float64)
        for i in range(c["n"]):
            out[i].index_put_((s["tokens"][i].to(torch.int64),), s["grad_out"][i].double() * c["scale"], accumulate=True)
        return {"grad": out}
    labels, rows = s["labels"].to(torch.int64), _rows(c)
    kept = torch.nonzero(labels >= 0).view(-1)
    lse, logp = (torch.zeros(rows, device=DEV, dtype=torch.float64) for _ in range(2))
    some = max(1, 100000000 // c["vocab"])
    for part in kept.split(some):
        x = s["logits"][part].double()
        lse[part] = torch.logsumexp(x, 1)
        logp[part] = x.gather(1, labels[part, None])[:, 0] - lse[part]
    kept_f = (labels >= 0).double()
    out = {"logp": logp}
    if c["kind"] == "logps":
        out["lse"] = lse
        slope = s["grad_logp"].double()
    elif c["kind"] == "preference":
        start, ratios = s["start"].tolist(), (logp - s["ref"].double()) * kept_f
        slope, losses = torch.zeros(rows, device=DEV, dtype=torch.float64), []
        for p in range(c["pairs"]):
            a, b, e = start[2 * p:2 * p + 3]
            na, nb = (max(1.0, float(v.sum())) if c["mean"] else 1.0 for v in (kept_f[a:b], kept_f[b:e]))
            margin = float(ratios[a:b].sum()) / na - float(ratios[b:e].sum()) / nb
            if c["loss"] == 0:
                z, eps = c["beta"] * margin, c["smoothing"]
                losses.append((1 - eps) * float(np.logaddexp(0.0, -z)) + eps * float(np.logaddexp(0.0, z)))
                d = c["beta"] * ((1 - eps) * (-1.0 / (1.0 + math.exp(z))) + eps / (1.0 + math.exp(-z)))
            else:
                losses.append((margin - 1.0 / (2.0 * c["beta"])) ** 2)
                d = 2.0 * margin - 1.0 / c["beta"]
            slope[a:b], slope[b:e] = d / na / c["pairs"], -d / nb / c["pairs"]
        out["loss"] = torch.tensor(losses, device=DEV, dtype=torch.float64)
    else:
        q, adv, ref = torch.exp(logp - s["old"].double()), s["advantages"].double(), s["ref"].double()
        worse = torch.where(adv >= 0, torch.clamp(q, max=1.28), torch.clamp(q, min=0.8))
        r = torch.exp(ref - logp)
        tokens = (c["kl"] * (r - 1.0 - (ref - logp)) - worse * adv) * kept_f
        w = s["weight"].double()
        out["token_loss"], out["loss"] = tokens, (w * tokens).sum().view(1)
        slope = w * (c["kl"] * (1.0 - r) - torch.where(worse == q, q * adv, 0.0))
    if c["kind"] != "logps" or c["backward"]:
        grad = torch.zeros(rows, c["vocab"], device=DEV, dtype=torch.float64)
        for part in kept.split(some):
            p = torch.exp(s["logits"][part].double() - lse[part, None])
            p.mul_(-slope[part, None]).scatter_add_(1, labels[part, None], slope[part, None])
            grad[part] = p
        out["grad"] = grad
    return out
