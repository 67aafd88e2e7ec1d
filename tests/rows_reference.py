"""Plain 64-bit forms of the row operators (sampling, top logits, distillation),
written from their definitions, on CPU tensors."""
import math

import torch

# A weight is taken as 2^((z - m) c) in fp32: the rounding of the difference, of c and of
# the product moves the exponent by at most 3 half-ulps of it, the exponential adds
# one more ulp; over the exponents that can matter (24 below the maximum in log2) that is
# (24 ln 2 * 3 / 2 + 1) 2^-23 = 3.1e-6 of a weight.  Sums are taken in 64 bits or over
# 8 terms before that.
WEIGHT_TOL = 4e-6


def order(z):
    """Tokens by (logit descending, id ascending), masked ones (-inf) left out."""
    z = z.double()
    ids = torch.sort(-z, stable=True).indices
    return ids[: int((z > -math.inf).sum())]


def prefix_size(e, k, p, m):
    """How many of the ordered weights e the filters keep."""
    n = len(e)
    if 0 < k < n:
        n = k
    cum = e.cumsum(0)
    if p < 1:
        mass = cum[n - 1]
        n = min(n, int((cum < p * mass).sum()) + 1)
    if m > 0:
        n = min(n, int((e >= m).sum()))
    return max(n, 1)


def sample_row(z, T, k, p, m):
    """(ordered tokens, their weights, fewest and most tokens that rounding lets the filters keep)."""
    if T == 0:
        T, k, p, m = 1.0, 1, 1.0, 0.0
    ids = order(z)
    x = z.double()[ids]
    e = ((x - x[0]) / T).exp()
    if k >= z.numel():
        k = 0
    tol = WEIGHT_TOL
    lo = prefix_size(e, k, p * (1 - tol) if p < 1 else p, m * (1 + tol))
    hi = prefix_size(e, k, min(p * (1 + tol), 1 - 1e-15) if p < 1 else p, m * (1 - tol))
    return ids, e, min(lo, hi), max(lo, hi)


def check_draw(z, T, k, p, m, u, token, logprob, kept):
    """The token, its log-probability and the kept count of one row against the definition."""
    ids, e, lo, hi = sample_row(z, T, k, p, m)
    assert lo <= kept <= hi, (kept, lo, hi)
    chosen, at = ids[:kept].sort()
    assert token in chosen.tolist(), "a token that the filters do not keep"
    w = e[:kept][at]
    cum = w.cumsum(0)
    i = chosen.tolist().index(token)
    target, tol = u * float(cum[-1]), WEIGHT_TOL * float(cum[-1])
    assert float(cum[i] - w[i]) - tol <= target <= float(cum[i]) + tol, (token, target, float(cum[i] - w[i]), float(cum[i]))
    want = torch.log_softmax(z.double() / (T if T else 1.0), 0)[token]
    assert abs(logprob - float(want)) <= 2e-6 * (1 + abs(float(want)))


def top_row(z, k, T):
    ids = order(z)[:k]
    n = len(ids)
    values = torch.full((k,), -math.inf, dtype=torch.float64)
    out = torch.full((k,), -1, dtype=torch.int64)
    values[:n], out[:n] = z.double()[ids], ids
    return values, out, torch.logsumexp(z.double() / T, 0)


def distill_row(s, ids, t, lse, T):
    """(loss, gradient) of one student row s [V] against entries (ids, t) and, with
    lse (a number or None), the teacher's rest."""
    s = s.double() / T
    V = s.numel()
    use = ids >= 0
    ids, t = ids[use].long(), t[use].double() / T
    logq = torch.log_softmax(s, 0)
    q = logq.exp()
    if lse is None and not (t > -math.inf).any():
        return torch.zeros((), dtype=torch.float64), torch.zeros(V, dtype=torch.float64)
    logp = torch.log_softmax(t, 0) if lse is None else t - float(lse)
    p = logp.exp()
    live = p > 0
    loss = (p[live] * (logp[live] - logq[ids[live]])).sum()
    grad = q.clone()
    outside = torch.ones(V, dtype=torch.bool)
    outside[ids] = False
    outside &= s > -math.inf
    if lse is not None and outside.any():
        r = (1 - p.sum()).clamp(min=0)
        log_rest = torch.logsumexp(logq[outside], 0)
        if r > 0:
            loss = loss + r * (r.log() - log_rest)
        inside = (logq[outside] - log_rest).exp()
        grad[outside] = inside * (log_rest.exp() - r)
    grad[ids] -= p
    return loss, grad / T
