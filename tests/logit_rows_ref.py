"""Plain 64-bit reference of the operators on rows of logits, and how far a kernel may be from it.

Tolerances, from the arithmetic.  u = 2^-24 is a float32 rounding (half a step, relative).
  * An exponential 2^((x - m) c): difference, scaling and c itself round once each, which moves the exponent by at most 3 u |d|
    (d = s (x - m), in nats); the instruction adds 2^-22 = 4 u.  Weighted with the probabilities, the mean of |d| is at
    most ln Z + max(-p ln p) summed = at most 2 ln V.  A sum of V terms is V / 256 sequential additions at most (128 threads,
    two halves each) and a tree of at most 20.  So Z is off by at most u (4 + 6 ln V + V / 256 + 20) relative, and ln Z by that
    much absolute: `rel(V)`.  The small-row kernels have shorter sums.
  * A log probability adds its own difference, scaling and subtraction: 3 u |lp| more, and 2 u |d| of the largest difference
    that it is made of; |d| <= |lp| + ln V.
  * An entropy is ln Z plus a mean of |d|, each term off by rel(V) relative: (1 + 2 ln V) rel(V).
  * A gradient is built from p (off by 2 rel(V), and u ln Z for the float32 ln Z kept between the passes), products of it
    (6 roundings), and is rounded once to its type: finfo.eps / 2 relative, at least half of the smallest subnormal step.
"""
import math

import torch

NINF = float("-inf")
U = 2.0 ** -24


def rel(vocab):
    return U * (24 + 6 * math.log(vocab + 1) + vocab / 256)


def log_softmax64(logits, s):
    x = logits.double()
    m = x.amax(1, keepdim=True)
    empty = m == NINF
    d = (x - m.masked_fill(empty, 0.0)) * s
    ln_z = d.exp().sum(1, keepdim=True).log()
    return torch.where(empty, torch.full_like(d, NINF), d - ln_z), m.squeeze(1), ln_z.squeeze(1), empty.squeeze(1)


def logprobs(logits, s, tokens, top):
    """dict of logprob, entropy, top_ids, top_logprobs, max, ln_z."""
    lp, m, ln_z, empty = log_softmax64(logits, s)
    V = logits.shape[1]
    t = tokens.long()
    bad = (t < -1) | (t >= V)
    got = lp.gather(1, t.clamp(0, V - 1).unsqueeze(1)).squeeze(1)
    got = got.masked_fill(t == -1, 0.0).masked_fill(bad, float("nan"))
    p = lp.exp()
    ent = -(p * lp.masked_fill(p == 0, 0.0)).sum(1).masked_fill(empty, 0.0)
    broken = torch.isnan(ln_z) | (m == float("inf"))
    ent = torch.where(broken, torch.full_like(ent, float("nan")), ent)
    got = torch.where(broken & (t >= 0), torch.full_like(got, float("nan")), got)
    out = {"logprob": got, "entropy": ent, "max": m, "ln_z": ln_z, "broken": broken, "empty": empty}
    if top:
        ids = torch.sort(logits.double(), dim=1, descending=True, stable=True).indices[:, :top]
        out["top_ids"] = ids.masked_fill(broken.unsqueeze(1), -1).int()
        out["top_logprobs"] = lp.gather(1, ids).masked_fill(broken.unsqueeze(1), float("nan"))
    return out


def logprobs_grad(logits, s, tokens, g_lp, g_ent):
    """(gradient, size of what it is made of)"""
    lp, _, _, empty = log_softmax64(logits, s)
    p = lp.exp()
    lp0 = lp.masked_fill(p == 0, 0.0)
    ent = -(p * lp0).sum(1, keepdim=True)
    t = tokens.long()
    g = torch.zeros_like(ent) if g_lp is None else g_lp.double().masked_fill(t == -1, 0.0).unsqueeze(1)
    h = torch.zeros_like(ent) if g_ent is None else g_ent.double().unsqueeze(1)
    hit = torch.zeros_like(p).scatter_(1, t.clamp(min=0).unsqueeze(1), 1.0) * (t >= 0).unsqueeze(1)
    dx = s * (g * (hit - p) - h * p * (lp0 + ent))
    size = s * (g.abs() * (hit + p) + h.abs() * p * (lp0.abs() + ent))
    dead = (empty.unsqueeze(1) | ((g == 0) & (h == 0))).expand_as(dx)
    return dx.masked_fill(dead, 0.0), size.masked_fill(dead, 0.0)


def distill(logits, s, ids, y, tail, weight):
    """dict of loss, its size, gradient, its size.  Entry by entry where ids repeat."""
    lp, m, _, empty = log_softmax64(logits, s)
    T, V = logits.shape
    used = ids >= 0
    i = ids.long().clamp(min=0)
    y = torch.where(used, y.double(), torch.full_like(y, NINF, dtype=torch.float64))
    some = (y > NINF).any(1)
    if not tail:
        y = y - torch.where(some, y.logsumexp(1), torch.zeros(T, dtype=torch.float64, device=logits.device)).unsqueeze(1)
    q = y.exp()
    listed = torch.zeros(T, V, dtype=torch.int32, device=logits.device).scatter_add_(1, i, used.int()) > 0
    ln_p = lp.gather(1, i)
    loss = torch.where(q > 0, q * (y - ln_p), torch.zeros_like(q)).sum(1)
    size = torch.where(q > 0, q * (y.abs() + ln_p.abs() + 1), torch.zeros_like(q)).sum(1)
    outside = lp.masked_fill(listed, NINF)
    others = (outside > NINF).any(1)
    p_rest = torch.where(others, outside.masked_fill(~others.unsqueeze(1), 0.0).logsumexp(1).exp(), torch.zeros(T, dtype=torch.float64, device=logits.device))
    q_rest = (1 - q.sum(1)).clamp(min=0) if tail else torch.zeros(T, dtype=torch.float64, device=logits.device)
    q_rest = torch.where(others, q_rest, torch.zeros_like(q_rest))
    both = q_rest > 0
    ln_pr = torch.where(others, outside.masked_fill(~others.unsqueeze(1), 0.0).logsumexp(1), torch.zeros_like(p_rest))
    loss = loss + torch.where(both, q_rest * (q_rest.clamp(min=1e-300).log() - ln_pr), torch.zeros_like(loss))
    size = size + torch.where(both, q_rest * (q_rest.clamp(min=1e-300).log().abs() + ln_pr.abs() + 1), torch.zeros_like(loss))
    p = lp.exp()
    qd = torch.zeros(T, V, dtype=torch.float64, device=logits.device).scatter_add_(1, i, q * used)
    soft_rest = torch.where(others.unsqueeze(1), (outside - ln_pr.unsqueeze(1)).exp(), torch.zeros_like(p)).masked_fill(listed, 0.0)
    # loss = sum q ln q - sum q ln p, and every ln p has the derivative 1[same element] - p: the sum of the q goes with p
    q_all = q.sum(1) + q_rest
    dx = torch.where(listed, q_all.unsqueeze(1) * p - qd, soft_rest * (q_all * p_rest - q_rest).unsqueeze(1))
    dsize = torch.where(listed, q_all.unsqueeze(1) * p + qd, soft_rest * (q_all * p_rest + q_rest).unsqueeze(1))
    w = weight.double()
    inside = some & ~empty & (w != 0)
    zero = ~inside.unsqueeze(1)
    return {"loss": loss.masked_fill(~inside, 0.0), "size": size.masked_fill(~inside, 0.0),
            "grad": (dx * (s * w).unsqueeze(1)).masked_fill(zero, 0.0), "grad_size": (dsize * (s * w.abs()).unsqueeze(1)).masked_fill(zero, 0.0)}


def check_grad(got, want, size, vocab, what="", factor=1.0):
    """A gradient against its 64-bit value: one rounding to its type, and the float32 arithmetic behind it.  An
    exponential below 2^-126 is flushed to zero before it is multiplied by up to `factor` (temperature times weight)."""
    fi = torch.finfo(got.dtype)
    tol = want.abs() * (fi.eps / 2) + size * (2 * rel(vocab) + 40 * U) + fi.smallest_normal * fi.eps / 2 + 2.0 ** -126 * max(1.0, factor)
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (what, float((err - tol).max()), float(err.max()))


def close(got, want, tol, what=""):
    """Equal infinities and NaNs, finite values within tol.  A value past the largest float32 rounds to an infinity
    there (1.5 times the lowest float32, say), so that is what it is compared as."""
    g, w = got.double(), want.double()
    w = torch.where(w.abs() > torch.finfo(torch.float32).max * (1 + 2.0 ** -25), w.sign() * float("inf"), w)
    assert bool((torch.isnan(g) == torch.isnan(w)).all()), (what, "NaN")
    fine = torch.isfinite(w)
    assert bool((g[~fine & ~torch.isnan(w)] == w[~fine & ~torch.isnan(w)]).all()), (what, "inf")
    err = (g - w).abs()[fine]
    t = (tol if torch.is_tensor(tol) else torch.full_like(w, tol))[fine]
    assert bool((err <= t).all()), (what, float((err - t).max()), float(err.max()))
