"""Workloads of the row operators that say what a row of logits means for a token, and how far a draft model's rows are
from the target's:

  logprobs       dt_token_logprobs: log-probabilities of given tokens, entropy, the k best alternatives
  logprobs_grad  dt_token_logprobs_grad: the gradient of both in the logits
  distill        dt_distill_rows: the loss of rows against a teacher's top log-probabilities, alone or with its gradient
  distill_grad   dt_distill_rows_grad: the gradient from what the loss has saved

With `own` false run() computes the same in plain torch operations, in 32 bits.  exact() is the definition in 64 bits.

Logits are N(0, 3) in the case's type with one token of every row raised by up to 12, so that rows range from undecided to
certain.  A teacher's row is the student's plus N(0, 1); its entries are its best logits and, for the plain and the
TAIL loss, its log-sum-exp.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"
D_MAX = 8                                   # deepest tree: a step emits up to D_MAX + 1 tokens
TAIL, RENORM = 1, 2                         # flags of the distillation loss


def _logprobs(name, B, rows, per_seq, V, k, dtype="bf16", T=1.0, masked=0.0, path=False, mix=0):
    c = dict(op="logprobs", B=B, rows=rows, per_seq=per_seq, V=V, k=k, dtype=dtype, T=T, masked=masked, path=path, mix=mix)
    return dict(name=name, **c) if name else c


def _logprobs_grad(name, n, V, dtype="bf16", T=1.0):
    c = dict(op="logprobs_grad", n=n, V=V, dtype=dtype, T=T)
    return dict(name=name, **c) if name else c


def _distill(name, n, V, k, dtype="bf16", T=1.0, flags=TAIL, grad=True, teachers=0, mix=0):
    c = dict(op="distill", n=n, V=V, k=k, dtype=dtype, T=T, flags=flags, grad=grad, teachers=teachers, mix=mix)
    return dict(name=name, **c) if name else c


def _distill_grad(name, n, V, k, dtype="bf16", T=1.0, flags=TAIL):
    c = dict(op="distill_grad", n=n, V=V, k=k, dtype=dtype, T=T, flags=flags)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # what one interactive user's step has emitted: up to nine rows out of the tree's, no alternatives asked for
        _logprobs("emitted_b1", 1, 60, D_MAX + 1, 128256, 0, path=True, mix=0),
        # a serving batch whose users ask for twenty alternatives of every emitted token
        _logprobs("emitted_b64_top20", 64, 32, D_MAX + 1, 128256, 20, T=0.8, path=True, mix=2),
        # a short text scored from logits kept in fp32, odd vocabulary, a grammar hiding part of it
        _logprobs("score_f32_odd_masked", 1, 700, 700, 50001, 5, dtype="f32", masked=0.3),
        # a long text scored
        _logprobs("score_long", 1, 4096, 4096, 128256, 5),
        # policy gradient with an entropy bonus on one short answer, small vocabulary
        _logprobs_grad("policy_grad_short", 33, 32000),
        # the same over a batch of answers
        _logprobs_grad("policy_grad_batch", 8192, 32000, T=0.9),
        # the draft rows of one step against the target rows of the nodes they were handed to
        _distill("distill_step", 51, 128256, 10, teachers=60, mix=3),
        # a held-out loss, no gradient, softened and over the teacher's entries only, fp32
        _distill("distill_eval_f32_odd", 300, 50001, 32, dtype="f32", T=2.0, flags=RENORM, grad=False),
        # a training batch of a small vocabulary
        _distill("distill_batch", 4096, 32000, 32),
        # a training batch of a large vocabulary
        _distill("distill_batch_large", 4096, 128256, 20),
        # backward on its own, rows at any 2-byte address
        _distill_grad("distill_grad_odd", 1000, 74365, 16, T=1.5),
        # backward on its own of fp32 logits, many teacher entries, plain loss
        _distill_grad("distill_grad_f32", 2048, 32000, 64, dtype="f32", flags=0),
    ]


# ------------------------------------------------------------------------------------------------- drawn cases

def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "logprobs_grad", "distill", "distill", "distill_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    V = _logint(rng, 1000, 131072)
    if rng.random() < 0.6:
        V = V // 64 * 64                    # a multiple of 64 as most models have
    T = rng.choice([0.6, 0.8, 1.0, 1.0, 1.5, 2.0])
    n = _logint(rng, 1, 4096)
    mix = rng.randrange(1 << 20)
    while n * V * (4 if dtype == "f32" else 2) > 1 << 29:
        n = (n + 1) // 2
    if op == "logprobs":
        k = rng.choice([0, rng.randint(1, 8), rng.randint(1, 32)])
        if rng.random() < 0.4:
            return _logprobs(None, _logint(rng, 1, 64), rng.randint(9, 32), D_MAX + 1, V, k, dtype, T, path=True, mix=mix)
        return _logprobs(None, 1, n, n, V, k, dtype, T, masked=rng.choice([0.0, 0.0, 0.5]), mix=mix)
    if op == "logprobs_grad":
        return _logprobs_grad(None, n, V, dtype, T)
    k = _logint(rng, 1, 128)
    flags = rng.choice([0, TAIL, TAIL, RENORM])
    if op == "distill_grad":
        return _distill_grad(None, n, V, k, dtype, T, flags)
    return _distill(None, n, V, k, dtype, T, flags, rng.random() < 0.7, rng.choice([0, 0, max(1, n // 2), 2 * n]), mix)


# ---------------------------------------------------------------------------------------------------- inputs

def _rows_of_logits(g, n, V, dtype, masked=0.0):
    x = torch.randn((n, V), generator=g, device=DEV).mul_(3.0)
    best = torch.randint(0, V, (n, 1), generator=g, device=DEV)
    lift = torch.rand((n, 1), generator=g, device=DEV) * 12.0
    x.scatter_add_(1, best, lift)
    if masked:
        hidden = torch.rand((1, V), generator=g, device=DEV) < masked
        hidden[0, 0] = False
        x.masked_fill_(hidden, -math.inf)
    return x.to(DTYPES[dtype])


def _path(case):
    """Which row of its sequence every emitted token was read from: ascending, -1 behind the bonus token's."""
    r = random.Random(case["mix"])
    out = []
    for _ in range(case["B"]):
        nodes = [0] + sorted(r.sample(range(1, case["rows"]), r.randint(0, min(D_MAX, case["rows"] - 1))))
        out.append(nodes + [-1] * (case["per_seq"] - len(nodes)))
    return out


def _teacher_rows(case):
    """Which of the teacher's rows every student's row goes by, -1: none."""
    r = random.Random(case["mix"])
    return [r.randrange(case["teachers"]) if r.random() < 0.9 else -1 for _ in range(case["n"])]


def _teacher(g, logits, m, k, T, flags):
    """m rows of a teacher's k best logits: from the student's rows, another opinion added."""
    n, V = logits.shape
    k = min(k, V)
    val = torch.empty((m, k), device=DEV)
    idx = torch.empty((m, k), dtype=torch.int64, device=DEV)
    lse = torch.empty(m, device=DEV)
    step = max(1, (1 << 27) // V)
    for a in range(0, m, step):
        at = torch.arange(a, min(m, a + step), device=DEV)
        x = logits[at % n].float()
        x += torch.randn(x.shape, generator=g, device=DEV)
        x /= T
        val[at], idx[at] = torch.topk(x, k, dim=1)
        lse[at] = torch.logsumexp(x, 1)
    idx = idx.to(torch.int32)
    # a teacher's list may be shorter than its slots
    short = (torch.rand(m, generator=g, device=DEV) < 0.1)[:, None] & (torch.arange(k, device=DEV) >= (k + 1) // 2)[None, :]
    return val.masked_fill_(short, -math.inf), idx.masked_fill_(short, -1), lse


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case=case, T=case["T"])
    if case["op"] == "logprobs":
        B, rows, per, V, k = (case[f] for f in ("B", "rows", "per_seq", "V", "k"))
        s["logits"] = _rows_of_logits(g, B * rows, V, case["dtype"], case["masked"]).view(B, rows, V)
        s["row_of"] = torch.tensor(_path(case), dtype=torch.int32, device=DEV) if case["path"] else None
        tokens = torch.randint(0, V, (B, per), generator=g, device=DEV)
        if case["path"]:                    # emitted: mostly the row's best
            best = s["logits"].argmax(2).gather(1, s["row_of"].long().clamp(min=0))
            tokens = torch.where(torch.rand((B, per), generator=g, device=DEV) < 0.7, best, tokens)
            tokens.masked_fill_(s["row_of"] < 0, -1)
        s["tokens"] = tokens.to(torch.int32)
        s["logprob"], s["entropy"] = torch.empty((B, per), device=DEV), torch.empty((B, per), device=DEV)
        s["stats"] = torch.empty((B, per, 2), device=DEV)
        s["top_logprob"] = torch.empty((B, per, k), device=DEV) if k else None
        s["top_id"] = torch.empty((B, per, k), dtype=torch.int32, device=DEV) if k else None
        n = B * per
    else:
        n, V = case["n"], case["V"]
        s["logits"] = x = _rows_of_logits(g, n, V, case["dtype"])
        s["stats"] = torch.empty((n, 2), device=DEV)
        s["grad"] = torch.empty_like(x) if case.get("grad", True) else None
        if case["op"] == "logprobs_grad":
            s["tokens"] = torch.randint(0, V, (n,), generator=g, device=DEV).to(torch.int32)
            s["g_logprob"] = torch.randn(n, generator=g, device=DEV)
            s["g_entropy"] = torch.randn(n, generator=g, device=DEV) * 0.1
            s["stats"], s["entropy"] = _saved(x, case["T"])
        else:
            m = case.get("teachers") or n
            s["teacher_row"] = torch.tensor(_teacher_rows(case), dtype=torch.int32, device=DEV) if case.get("teachers") else None
            s["val"], s["id"], s["lse"] = _teacher(g, x, m, case["k"], case["T"], case["flags"])
            s["weight"] = torch.rand(n, generator=g, device=DEV) * (2.0 / n)
            s["loss"], s["tail"] = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
            if case["op"] == "distill_grad":
                s["stats"], _ = _saved(x, case["T"])
                s["tail"] = _saved_tail(x, s["id"], case["T"])
    if own:
        import paper_2601_12212_amd as dt
        s["ws"] = torch.empty(dt.dt_logprob_workspace_bytes(n, V), dtype=torch.uint8, device=DEV)
    return s


def _blocks(n, V):
    step = max(1, (1 << 25) // V)
    return [slice(a, min(n, a + step)) for a in range(0, n, step)]


def _saved(x, T):
    """What a forward pass has left for the backward one: (largest logit, log of the sum against it), entropy."""
    stats, entropy = torch.empty((x.shape[0], 2), device=DEV), torch.empty(x.shape[0], device=DEV)
    for b in _blocks(*x.shape):
        y = x[b].double()
        m = y.amax(1)
        z = (y - m[:, None]) / T
        l = torch.logsumexp(z, 1)
        stats[b, 0], stats[b, 1] = m.float(), l.float()
        entropy[b] = (l - (torch.exp(z - l[:, None]) * z.clamp(min=-1e4)).sum(1)).float()
    return stats, entropy


def _saved_tail(x, idx, T):
    """log of the student's probability outside the teacher's entries."""
    tail = torch.empty(x.shape[0], device=DEV)
    for b in _blocks(*x.shape):
        y = x[b].double() / T
        whole = torch.logsumexp(y, 1)
        at = torch.where(idx[b] >= 0, idx[b].long(), idx[b, :1].long())
        tail[b] = (torch.logsumexp(y.scatter(1, at, -math.inf), 1) - whole).float()
    return tail


# --------------------------------------------------------------------------------------- the plain form, 32 bits

def _plain_logprobs(s):
    x, k, T = s["logits"], s["case"]["k"], s["T"]
    B, rows, V = x.shape
    tokens = s["tokens"]
    there = None
    if s["row_of"] is not None:
        there = s["row_of"] >= 0
        at = s["row_of"].clamp(min=0).long() + rows * torch.arange(B, device=DEV)[:, None]
        x = x.reshape(B * rows, V)[at]
    f = x.float()
    m = f.amax(2, keepdim=True)
    z = (f - m) / T
    e = torch.exp(z)
    total = e.sum(2, keepdim=True)
    l = torch.log(total)
    named = tokens.clamp(min=0).long()[..., None]
    logprob = (z.gather(2, named) - l).squeeze(2)
    entropy = (l - (e * z.clamp(min=-1e4)).sum(2, keepdim=True) / total).squeeze(2)
    stats = torch.cat([m, l], 2)
    if there is not None:
        logprob = logprob.masked_fill(~there, 0.0)
        entropy = entropy.masked_fill(~there, 0.0)
        stats = stats.masked_fill(~there[..., None], 0.0)
    out = dict(logprob=logprob, entropy=entropy, stats=stats)
    if k:
        bits = (f + 0.0).view(torch.int32).long()           # larger logit first, then the lower id
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 20) - torch.arange(V, device=DEV)
        top = torch.topk(key, k, dim=2).indices
        lp = z.gather(2, top) - l
        gone = torch.isinf(lp)
        if there is not None:
            gone = gone | ~there[..., None]
        out["top_logprob"] = lp.masked_fill(gone, -math.inf)
        out["top_id"] = top.to(torch.int32).masked_fill(gone, -1)
    return out


def _plain_logprobs_grad(s):
    x, T = s["logits"].float(), s["T"]
    m, l = s["stats"][:, :1], s["stats"][:, 1:]
    lq = (x - m) / T - l
    q = torch.exp(lq)
    d = -q * (s["g_logprob"][:, None] + s["g_entropy"][:, None] * (lq + s["entropy"][:, None]))
    d.scatter_add_(1, s["tokens"].long()[:, None], s["g_logprob"][:, None])
    return dict(grad=(d / T).to(s["logits"].dtype))


def _plain_teacher(s):
    """p [n, k], log p [n, k], the rest's p [n, 1], ids [n, k], and which slots and rows count."""
    flags = s["case"]["flags"]
    val, idx, lse = s["val"], s["id"], s["lse"]
    there = None
    if s["teacher_row"] is not None:
        there = s["teacher_row"] >= 0
        at = s["teacher_row"].clamp(min=0).long()
        val, idx, lse = val[at], idx[at], lse[at]
    lp = val.double() - lse.double()[:, None]
    p = torch.exp(lp)
    if flags & RENORM:
        P = p.sum(1, keepdim=True)
        p, lp = p / P, lp - torch.log(P)
    rest = (1.0 - p.sum(1, keepdim=True)).clamp(min=0.0) if flags & TAIL else torch.zeros_like(p[:, :1])
    return p.float(), lp.float(), rest.float(), idx, there


def _plain_gradient(s, q, q_rest, p, rest, idx, there):
    """d loss / d logits of every row, from its probabilities q and their sum outside the teacher's entries."""
    valid = idx >= 0
    at = torch.where(valid, idx.long(), idx[:, :1].long())
    total = p.sum(1, keepdim=True) + rest
    out = torch.where(q_rest > 0, rest / q_rest, torch.zeros_like(rest))
    own_term = q * (total - out)
    inside = torch.zeros_like(q, dtype=torch.bool).scatter_(1, at, True)
    d = torch.where(inside, q * total, own_term)
    d.scatter_add_(1, at, -p)
    d *= s["weight"][:, None] / s["T"]
    if there is not None:
        d.masked_fill_(~there[:, None], 0.0)
    return d.to(s["logits"].dtype)


def _plain_distill(s):
    x, T = s["logits"].float(), s["T"]
    p, lp, rest, idx, there = _plain_teacher(s)
    m = x.amax(1, keepdim=True)
    z = (x - m) / T
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    l = torch.log(total)
    valid = idx >= 0
    at = torch.where(valid, idx.long(), idx[:, :1].long())
    q_rest = e.scatter(1, at, 0.0).sum(1, keepdim=True) / total
    tail = torch.log(q_rest)
    lq = z.gather(1, at) - l
    loss = torch.where(valid, p * (lp - lq), torch.zeros_like(p)).sum(1, keepdim=True)
    loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - tail), torch.zeros_like(rest))
    loss, tail, stats = loss.squeeze(1), tail.squeeze(1), torch.cat([m, l], 1)
    if there is not None:
        loss, tail, stats = loss.masked_fill(~there, 0.0), tail.masked_fill(~there, 0.0), stats.masked_fill(~there[:, None], 0.0)
    out = dict(loss=loss, tail=tail, stats=stats)
    if s["grad"] is not None:
        out["grad"] = _plain_gradient(s, e / total, q_rest, p, rest, idx, there)
    return out


def _plain_distill_grad(s):
    p, _, rest, idx, there = _plain_teacher(s)
    q = torch.exp((s["logits"].float() - s["stats"][:, :1]) / s["T"] - s["stats"][:, 1:])
    return dict(grad=_plain_gradient(s, q, torch.exp(s["tail"])[:, None], p, rest, idx, there))


_PLAIN = dict(logprobs=_plain_logprobs, logprobs_grad=_plain_logprobs_grad, distill=_plain_distill, distill_grad=_plain_distill_grad)


# ------------------------------------------------------------------------------------------- the framework's calls

def _own(s):
    import paper_2601_12212_amd as dt
    c, op = s["case"], s["case"]["op"]
    if op == "logprobs":
        dt.dt_token_logprobs(s["logits"], s["row_of"], s["tokens"], s["T"], c["k"], s["logprob"], s["entropy"], s["stats"],
                             s["top_logprob"], s["top_id"], s["ws"])
        out = dict(logprob=s["logprob"], entropy=s["entropy"], stats=s["stats"])
        return dict(out, top_logprob=s["top_logprob"], top_id=s["top_id"]) if c["k"] else out
    if op == "logprobs_grad":
        dt.dt_token_logprobs_grad(s["logits"], s["tokens"], s["T"], s["stats"], s["entropy"], s["g_logprob"], s["g_entropy"], s["grad"])
        return dict(grad=s["grad"])
    if op == "distill":
        dt.dt_distill_rows(s["logits"], s["val"], s["id"], s["lse"], s["teacher_row"], s["T"], c["flags"], s["weight"], s["loss"],
                           s["stats"], s["tail"], s["grad"], s["ws"])
        out = dict(loss=s["loss"], tail=s["tail"], stats=s["stats"])
        return dict(out, grad=s["grad"]) if c["grad"] else out
    dt.dt_distill_rows_grad(s["logits"], s["val"], s["id"], s["lse"], s["teacher_row"], s["T"], c["flags"], s["weight"], s["stats"],
                            s["tail"], s["grad"])
    return dict(grad=s["grad"])


def run(s):
    return _own(s) if own else _PLAIN[s["case"]["op"]](s)


# ------------------------------------------------------------------------------------ the definition, in 64 bits

def _exact_rows(x, T):
    y = x.double() / T
    lse = torch.logsumexp(y, 1, keepdim=True)
    return y - lse, x.double().amax(1), (lse[:, 0] - y.amax(1))


def _exact_logprobs(case, s):
    B, rows, per, V, k = (case[f] for f in ("B", "rows", "per_seq", "V", "k"))
    n = B * per
    row_of = s["row_of"] if s["row_of"] is not None else torch.arange(per, device=DEV, dtype=torch.int32).expand(B, per)
    at = (row_of.long() + rows * torch.arange(B, device=DEV)[:, None]).reshape(n)
    live = (row_of >= 0).reshape(n)
    f64 = dict(dtype=torch.float64, device=DEV)
    out = dict(logprob=torch.zeros(n, **f64), entropy=torch.zeros(n, **f64), stats=torch.zeros((n, 2), **f64),
               top_logprob=torch.full((n, k), -math.inf, **f64), top_id=torch.full((n, k), -1, dtype=torch.int32, device=DEV))
    x = s["logits"].reshape(-1, V)
    tokens = s["tokens"].reshape(n).long()
    for b in _blocks(n, V):
        keep = live[b].nonzero()[:, 0] + b.start
        if not len(keep):
            continue
        lq, m, l = _exact_rows(x[at[keep]], s["T"])
        q = torch.exp(lq)
        out["logprob"][keep] = lq.gather(1, tokens[keep][:, None])[:, 0]
        out["entropy"][keep] = -(q * torch.where(q > 0, lq, torch.zeros_like(lq))).sum(1)
        out["stats"][keep] = torch.stack([m, l], 1)
        if k:
            v, i = torch.sort(x[at[keep]].double(), dim=1, descending=True, stable=True)
            v, i = lq.gather(1, i[:, :k]), i[:, :k].to(torch.int32)
            out["top_logprob"][keep] = v
            out["top_id"][keep] = torch.where(torch.isinf(v), torch.full_like(i, -1), i)
    if not k:
        del out["top_logprob"], out["top_id"]
    return {name: v.reshape((B, per) + tuple(v.shape[1:])) for name, v in out.items()}


def _exact_teacher(case, s):
    at = torch.arange(case["n"], device=DEV) if s["teacher_row"] is None else s["teacher_row"].long().clamp(min=0)
    idx = s["id"][at].long()
    p = torch.where(idx >= 0, torch.exp(s["val"][at].double() - s["lse"][at].double()[:, None]), torch.zeros((), dtype=torch.float64, device=DEV))
    if case["flags"] & RENORM:
        p = p / p.sum(1, keepdim=True)
    if s["teacher_row"] is not None:
        p = p * (s["teacher_row"] >= 0)[:, None]
    return p, idx


def _exact_distill(case, s, with_grad):
    n, V, x, T, flags = case["n"], case["V"], s["logits"], s["T"], case["flags"]
    p_all, idx_all = _exact_teacher(case, s)
    none = s["teacher_row"] < 0 if s["teacher_row"] is not None else torch.zeros(n, dtype=torch.bool, device=DEV)
    f64 = dict(dtype=torch.float64, device=DEV)
    out = dict(loss=torch.zeros(n, **f64), tail=torch.zeros(n, **f64), stats=torch.zeros((n, 2), **f64))
    grad = torch.empty((n, V), **f64) if with_grad else None
    for b in _blocks(n, V):
        lq, m, l = _exact_rows(x[b], T)
        q = torch.exp(lq)
        # the teacher's distribution over the vocabulary, and over "none of its entries"
        p, idx = p_all[b], idx_all[b]
        dense = torch.zeros_like(q).scatter_add_(1, idx.clamp(min=0), p)
        listed_ids = torch.zeros_like(q).scatter_add_(1, idx.clamp(min=0), (idx >= 0).double()) > 0
        q_out = torch.where(listed_ids, torch.zeros_like(q), q).sum(1)
        rest = (1.0 - p.sum(1)).clamp(min=0.0) if flags & TAIL else torch.zeros_like(q_out)
        live = ~none[b]
        rest = rest * live
        ratio = torch.where(dense > 0, dense * (torch.log(dense.clamp(min=1e-300)) - lq), torch.zeros_like(q)).sum(1)
        ratio = ratio + torch.where(rest > 0, rest * (torch.log(rest.clamp(min=1e-300)) - torch.log(q_out)), torch.zeros_like(rest))
        out["loss"][b] = ratio
        out["tail"][b] = torch.where(live, torch.log(q_out), torch.zeros_like(q_out))
        out["stats"][b] = torch.stack([m, l], 1) * live[:, None]
        if with_grad:
            mass = (p.sum(1) + rest)[:, None]
            from_rest = torch.where(listed_ids, torch.zeros_like(q), q / q_out[:, None]) * rest[:, None]
            grad[b] = (mass * q - from_rest - dense) * (s["weight"][b].double() * live)[:, None] / T
    return dict(out, grad=grad) if with_grad else out


def _exact_logprobs_grad(case, s):
    grad = torch.empty((case["n"], case["V"]), dtype=torch.float64, device=DEV)
    for b in _blocks(case["n"], case["V"]):
        lq, _, _ = _exact_rows(s["logits"][b], s["T"])
        q = torch.exp(lq)
        entropy = -(q * lq).sum(1, keepdim=True)
        hot = torch.zeros_like(q).scatter_(1, s["tokens"][b].long()[:, None], 1.0)
        grad[b] = (s["g_logprob"][b].double()[:, None] * (hot - q) - s["g_entropy"][b].double()[:, None] * q * (lq + entropy)) / s["T"]
    return dict(grad=grad)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "logprobs":
        return _exact_logprobs(case, s)
    if case["op"] == "logprobs_grad":
        return _exact_logprobs_grad(case, s)
    out = _exact_distill(case, s, case["op"] == "distill_grad" or case["grad"])
    return dict(grad=out["grad"]) if case["op"] == "distill_grad" else out


# ------------------------------------------------------------------------------------------------------------ work

def work(case):
    size, V = 4 if case["dtype"] == "f32" else 2, case["V"]
    if case["op"] == "logprobs":
        B, per = case["B"], case["per_seq"]
        read = sum(r >= 0 for path in _path(case) for r in path) if case["path"] else B * per
        return dict(bytes=read * V * size + B * per * (8 + 16 + 8 * case["k"]), flops=6 * read * V)
    n = case["n"]
    if case["op"] == "logprobs_grad":
        return dict(bytes=2 * n * V * size + 24 * n, flops=7 * n * V)
    teachers = (case.get("teachers") or n) * (8 * min(case["k"], V) + 4)
    if case["op"] == "distill_grad":
        return dict(bytes=2 * n * V * size + teachers + 16 * n, flops=5 * n * V)
    return dict(bytes=(2 if case["grad"] else 1) * n * V * size + teachers + 24 * n, flops=(8 if case["grad"] else 4) * n * V)
