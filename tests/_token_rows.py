"""Plain implementations in 64 bits of the row operators (log-probabilities, distillation, gradients), on the CPU, and the
tolerances that their tests use.

Tolerances.  u = 2^-24 is half a step of fp32 relative to the value.  A sum over a row of V positive weights is taken by 256 threads
(V/256 + 32 additions in a row at most), then over lanes and waves (10) and parts (6): relative error below u (V/256 + 48).  A weight
2^t has the relative error ln 2 |t| u of its exponent's rounding, 2 ln 2 |t| u of the constant log2(e)/T's, and 2 u of the exponential; weights
below 2^-24 of the largest do not matter together (their sum is bounded by V 2^-24, whose errors are below u V 2^-24), so |t| <= 24: 54 u.  DELTA(V)
= u (V/256 + 128) bounds a sum's relative error, and so the absolute one of its logarithm.

A weight below 2^-126, fp32's smallest normal number, comes out as 0: a gradient's entry is then off by q |g + h (log q + H)| / T
< 2^-126 (|g| + 100 |h|) / T (|log q| < 88, H < 12), below TINY = 2^-116 for the |g|, |h| < 5 and T >= 1/2 of the tests.
"""
import math

import torch

U = 2.0 ** -24
TINY = 2.0 ** -116
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def delta(V):
    return U * (V / 256 + 128)


def f64(T):
    """The temperature as the kernels see it."""
    return float(torch.tensor(T, dtype=torch.float32).double())


def log_softmax(x, T):
    """log q [n, V] and (m, l); rows without a finite entry: -inf everywhere."""
    x = x.double()
    m = x.amax(1, keepdim=True)
    d = torch.where(x == m, torch.zeros_like(x), (x - m) / f64(T))     # (m may be -inf)
    d = torch.where(torch.isinf(m), torch.full_like(d, -math.inf), d)
    l = torch.log(torch.exp(d).sum(1, keepdim=True))
    lq = torch.where(torch.isinf(m), torch.full_like(d, -math.inf), d - l)
    return lq, m[:, 0], l[:, 0]


def logprobs(x, tokens, T, k):
    n, V = x.shape
    lq, m, l = log_softmax(x, T)
    q = torch.exp(lq)
    ok = (tokens >= 0) & (tokens < V)
    lp = torch.where(ok, lq.gather(1, torch.where(ok, tokens, 0).long()[:, None])[:, 0], torch.zeros(n, dtype=torch.float64))
    H = -(q * torch.where(q > 0, lq, torch.zeros_like(lq))).sum(1)
    order = torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :k]
    top = lq.gather(1, order)
    ids = torch.where(torch.isinf(x.double().gather(1, order)), -1, order)
    return dict(logprob=lp, entropy=H, stats=torch.stack([m, l], 1), top_logprob=torch.where(ids < 0, -math.inf, top), top_id=ids.int())


def logprobs_grad(x, tokens, T, g_lp, g_H):
    n, V = x.shape
    lq, _, _ = log_softmax(x, T)
    q = torch.exp(lq)
    flat = torch.where(q > 0, lq, torch.zeros_like(lq))
    H = -(q * flat).sum(1, keepdim=True)
    ok = (tokens >= 0) & (tokens < V)
    g = torch.where(ok, g_lp.double(), torch.zeros(n, dtype=torch.float64))[:, None]
    hot = torch.zeros_like(q).scatter_(1, torch.where(ok, tokens, 0).long()[:, None], ok.double()[:, None])
    h = g_H.double()[:, None]
    grad = (g * (hot - q) - h * q * (flat + H)) / f64(T)
    # what its terms amount to, for the tolerance: every one of them may be off by a few delta
    size = (g.abs() * (hot + q) + h.abs() * q * (flat.abs() + H + 1)) / f64(T)
    return grad, size


def distill(x, val, ids, lse, rows, T, flags, w=None):
    """loss, tail, stats, grad and what the gradient's and the loss's terms amount to."""
    n, V = x.shape
    lq, m, l = log_softmax(x, T)
    q = torch.exp(lq)
    out = dict(loss=torch.zeros(n, dtype=torch.float64), tail=torch.zeros(n, dtype=torch.float64), stats=torch.zeros(n, 2, dtype=torch.float64),
               grad=torch.zeros(n, V, dtype=torch.float64), size=torch.zeros(n, V, dtype=torch.float64), terms=torch.zeros(n, dtype=torch.float64))
    w = torch.ones(n, dtype=torch.float64) if w is None else w.double()
    for r in range(n):
        t = r if rows is None else int(rows[r])
        if t < 0 or t >= len(val):
            continue
        entries = [(int(i), float(v) - (0.0 if lse is None else float(lse[t]))) for i, v in zip(ids[t], val[t]) if 0 <= int(i) < V and float(v) > -math.inf]
        P = sum(math.exp(lp) for _, lp in entries)
        if flags & 2 and P > 0:
            entries = [(i, lp - math.log(P)) for i, lp in entries]
            P = 1.0
        rest = max(0.0, 1.0 - P) if flags & 1 else 0.0
        S = sorted({i for i, _ in entries})
        outside = torch.ones(V, dtype=torch.bool)
        outside[S] = False
        q_t = float(q[r][outside].sum())
        tail = math.log(q_t) if q_t > 0 else -math.inf
        loss = terms = 0.0
        add = torch.zeros(V, dtype=torch.float64)
        for i, lp in entries:
            p = math.exp(lp)
            loss += p * (lp - float(lq[r, i])) if p > 0 else 0.0
            terms += p * (abs(lp) + abs(float(lq[r, i])) + 1)
            add[i] += p
        if rest > 0:
            loss += rest * (math.log(rest) - tail)
            terms += rest * (abs(math.log(rest)) + abs(tail) + 1) + U * (1 + abs(math.log(rest)))
        share = torch.where(outside, q[r] / q_t if q_t > 0 else torch.zeros(V, dtype=torch.float64), torch.zeros(V, dtype=torch.float64))
        out["loss"][r], out["tail"][r], out["terms"][r] = loss, tail, terms
        out["stats"][r, 0], out["stats"][r, 1] = m[r], l[r]
        out["grad"][r] = w[r] / f64(T) * ((P + rest) * q[r] - rest * share - add)
        out["size"][r] = w[r].abs() / f64(T) * ((P + rest) * q[r] + rest * share + add)
    return out


def close(got, want, tol, what=""):
    """|got - want| <= tol, infinities in the same places."""
    got, want = got.double().cpu(), want.double()
    tol = tol if isinstance(tol, torch.Tensor) else torch.full_like(want, tol)
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)]), (what, got[~fin], want[~fin])
    err = (got - want).abs()[fin]
    bad = err > tol[fin]
    assert not bad.any(), (what, int(bad.sum()), float(err.max()), float(tol[fin].min()))
