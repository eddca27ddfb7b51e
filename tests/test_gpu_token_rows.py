"""Row operators on the GPU against plain implementations in 64 bits (tests/_token_rows.py, which derives the tolerances)."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2601_12212_amd as dt  # noqa: E402
from tests import _token_rows as ref  # noqa: E402

DEV = "cuda"
NAN = math.nan
F32, BF16 = torch.float32, torch.bfloat16
i32 = dict(dtype=torch.int32)


def rows(n, V, dtype, seed, sigma=3.0, offset=0, pad=0):
    """(host rows as the kernels see them, device view of n rows of V entries, `offset` elements behind an aligned place and
    V + pad apart).  What lies between the rows is NaN."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, V, generator=g) * sigma).to(dtype)
    x[torch.arange(n), torch.randint(0, V, (n,), generator=g)] += torch.tensor(float(seed % 3 * 5), dtype=dtype)
    return x, put(x, offset, pad)


def put(x, offset=0, pad=0):
    n, V = x.shape
    stride = V + pad
    room = torch.full((offset + n * stride + 8,), NAN, dtype=x.dtype, device=DEV)
    view = room[offset:offset + n * stride].view(n, stride)[:, :V]
    view.copy_(x)
    return view


def dirty(*shape, dtype=torch.float32):
    """Memory that nothing has written: NaN, and the lowest integer."""
    return torch.full(shape, NAN if dtype.is_floating_point else -(1 << 31), dtype=dtype, device=DEV)


def workspace(n, V):
    return torch.full((dt.dt_logprob_workspace_bytes(n, V),), 0xFF, dtype=torch.uint8, device=DEV)


def run_logprobs(x3, row_of, tokens, T, k, per, entropy=True):
    B, _, V = x3.shape
    o = dict(logprob=dirty(B, per) if tokens is not None else None, entropy=dirty(B, per) if entropy else None, stats=dirty(B, per, 2),
             top_logprob=dirty(B, per, k) if k else None, top_id=dirty(B, per, k, dtype=torch.int32) if k else None)
    dt.dt_token_logprobs(x3, row_of, tokens, T, k, o["logprob"], o["entropy"], o["stats"], o["top_logprob"], o["top_id"], workspace(B * per, V))
    torch.cuda.synchronize()
    return {name: v for name, v in o.items() if v is not None}


def check_logprobs(got, x, tokens, T, k):
    V = x.shape[1]
    want = ref.logprobs(x, tokens, T, k)
    d = ref.delta(V)
    size = lambda lp: torch.where(torch.isfinite(lp), lp.abs(), 0.0)
    flat = lambda v: v.reshape((len(x),) + tuple(v.shape[2:]))
    if "logprob" in got:
        ref.close(flat(got["logprob"]), want["logprob"], d + 6 * ref.U * size(want["logprob"]), "logprob")
    if "entropy" in got:
        ref.close(flat(got["entropy"]), want["entropy"], 2 * d * (1 + want["entropy"]), "entropy")
    ref.close(flat(got["stats"])[:, 0], want["stats"][:, 0], 0.0, "largest logit")
    ref.close(flat(got["stats"])[:, 1], want["stats"][:, 1], torch.full((len(x),), d, dtype=torch.float64), "log sum")
    if k:
        assert torch.equal(flat(got["top_id"]).cpu(), want["top_id"])
        ref.close(flat(got["top_logprob"]), want["top_logprob"], d + 6 * ref.U * size(want["top_logprob"]), "alternatives")


SHAPES = [(1, 1, 1), (3, 2, 2), (2, 7, 3), (5, 8, 8), (3, 9, 9), (2, 31, 32 - 1), (4, 257, 5), (1, 1000, 32), (6, 2049, 20), (3, 8192, 1), (2, 8193, 20),
          (5, 16391, 7), (4, 50001, 32), (2, 128257, 20), (1, 131072, 32), (300, 515, 4), (2100, 130, 3), (2050, 8200, 5), (2, 300001, 11)]


@pytest.mark.parametrize("n, V, k", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_logprobs(n, V, k, dtype):
    x, xd = rows(n, V, dtype, n + V)
    tokens = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(V), dtype=torch.int32)
    got = run_logprobs(xd[None], None, tokens.to(DEV)[None], 1.0, k, n)
    check_logprobs(got, x, tokens, 1.0, k)


@pytest.mark.parametrize("offset, pad", [(1, 0), (3, 1), (8, 5), (5, 27), (2, 8)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T", [0.3, 2.5])
def test_logprobs_of_rows_anywhere(offset, pad, dtype, T):
    for n, V, k in ((3, 12345, 9), (2, 5, 5), (2, 13, 2)):
        x, xd = rows(n, V, dtype, 7 * offset + pad, offset=offset, pad=pad)
        tokens = torch.arange(n, **i32) * 3 % V
        check_logprobs(run_logprobs(xd[None], None, tokens.to(DEV)[None], T, k, n), x, tokens, T, k)


LOWEST = {BF16: torch.finfo(BF16).min, F32: torch.finfo(F32).min}


def special_rows(V, dtype):
    """Rows that bounds, masks and ties are hard on."""
    g = torch.Generator().manual_seed(V)
    base = torch.randn(V, generator=g) * 3
    out = {}
    out["nothing but masks"] = torch.full((V,), -math.inf)
    out["nothing but the lowest value"] = torch.full((V,), LOWEST[dtype])
    out["the lowest value and masks"] = torch.where(torch.arange(V) % 3 == 0, LOWEST[dtype], -math.inf)
    out["one token"] = torch.full((V,), -math.inf).index_fill(0, torch.tensor([V - 1]), 2.0)
    out["three tokens"] = torch.full((V,), -math.inf).index_copy(0, torch.tensor([0, V // 2, V - 2]), torch.tensor([1.0, 3.0, 1.0]))
    out["half masked"] = torch.where(torch.rand(V, generator=g) < 0.5, base, -math.inf)
    out["masked by the lowest value"] = torch.where(torch.rand(V, generator=g) < 0.5, base, LOWEST[dtype])
    out["all equal"] = torch.full((V,), 1.25)
    out["zeros of both signs"] = torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0)
    out["two values"] = torch.where(torch.rand(V, generator=g) < 0.5, 1.0, 2.0)
    out["ascending"] = torch.linspace(-20, 20, V)
    out["descending"] = torch.linspace(20, -20, V)
    out["neighbours"] = base + 20.0 * ((torch.arange(V) >= V // 3) & (torch.arange(V) < V // 3 + 1500))
    out["ties at the end"] = torch.where(torch.arange(V) >= V - min(V, 2000), 4.0, base.clamp(max=3.0))
    out["certain"] = base.index_fill(0, torch.tensor([V // 5]), 90.0)
    out["large"] = base * 1000.0
    out["very large"] = base * 1e37
    out["far below zero"] = base - 300.0
    return {name: v.to(dtype) for name, v in out.items()}


@pytest.mark.parametrize("V", [40, 5000, 40000])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("many", [False, True], ids=["few", "many"])
def test_logprobs_of_special_rows(V, dtype, many):
    check_special_rows(V, dtype, 2048 if many else 1)    # more rows than are cut into parts


@pytest.mark.parametrize("V", [12000, 20000, 40000])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("at_least", [1, 140, 300, 600])
def test_logprobs_of_special_rows_by_their_number(V, dtype, at_least):
    check_special_rows(V, dtype, at_least)


def check_special_rows(V, dtype, at_least):
    named = special_rows(V, dtype)
    x = torch.stack(list(named.values()))
    n = len(x)
    reps = (at_least - 1) // n + 1
    tokens = torch.full((n,), V // 2, **i32)
    xd = put(x.repeat(reps, 1))
    got = run_logprobs(xd[None], None, tokens.repeat(reps).to(DEV)[None], 1.0, 32, n * reps)
    for name, v in got.items():                          # every copy of a row says the same
        w = v[0].reshape((reps, n) + tuple(v.shape[2:]))
        assert torch.equal(w.cpu().nan_to_num(9e9), w[:1].expand_as(w).cpu().nan_to_num(9e9)), name
    got = {name: v[:, :n] for name, v in got.items()}
    want = ref.logprobs(x, tokens, 1.0, 32)
    assert torch.equal(got["top_id"][0].cpu(), want["top_id"])
    scale = x.double().masked_fill(torch.isinf(x.double()), 0).abs().amax(1).clamp(min=1.0)     # (x - m) is rounded relative to itself
    scale = torch.where(scale > 1e30, torch.ones_like(scale), scale)                             # (and is 0 or below every exponent there)
    for i, name in enumerate(named):
        d = ref.delta(V) * (1 + float(scale[i]) / 32)
        lp, w = got["logprob"][0, i].cpu(), want["logprob"][i]
        rel = 6 * ref.U * abs(float(w)) if math.isfinite(float(w)) else 0.0
        if float(w) < -1e30:
            assert float(lp) < -1e30, (name, lp, w)      # (beyond fp32's range, or next to it)
        else:
            ref.close(lp[None], w[None], d + rel, name)
        ref.close(got["entropy"][0, i][None], want["entropy"][i][None], 2 * d * (1 + float(want["entropy"][i])), name)
        ref.close(got["stats"][0, i, :1], want["stats"][i, :1], 0.0, name)
        ref.close(got["stats"][0, i, 1:], want["stats"][i, 1:], d, name)


def test_chosen_rows():
    """Entries by row_of: rows twice, rows out of range, tokens out of range."""
    B, R, per, V, k = 3, 5, 7, 9001, 6
    x, xd = rows(B * R, V, BF16, 4)
    of = torch.tensor([[0, 3, 3, -1, 4, 5, 2], [4, -7, 1, 0, 0, 1 << 30, 2], [-1, -1, -1, -1, -1, -(1 << 31), 9]], **i32)
    tok = torch.randint(0, V, (B, per), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    tok[0, 1], tok[0, 2], tok[1, 0] = -1, V, 1 << 30
    for T in (1.0, 0.7):
        got = run_logprobs(xd.view(B, R, V), of.to(DEV), tok.to(DEV), T, k, per)
        ok = (of >= 0) & (of < R)
        at = torch.arange(B)[:, None] * R + torch.where(ok, of, 0)
        keep = ok.reshape(-1)
        check_logprobs({name: v.reshape((B * per,) + tuple(v.shape[2:]))[keep.to(DEV)][None] for name, v in got.items()},
                       x[at.reshape(-1)[keep]], tok.reshape(-1)[keep], T, k)
        none = {name: v.reshape((B * per,) + tuple(v.shape[2:])).cpu()[~keep] for name, v in got.items()}
        assert (none["logprob"] == 0).all() and (none["entropy"] == 0).all() and (none["stats"] == 0).all()
        assert (none["top_logprob"] == -math.inf).all() and (none["top_id"] == -1).all()


def test_what_is_not_asked_for():
    n, V = 4, 20001
    x, xd = rows(n, V, BF16, 9)
    tokens = torch.arange(n, **i32)
    check_logprobs(run_logprobs(xd[None], None, None, 1.0, 0, n, entropy=False), x, tokens, 1.0, 0)
    check_logprobs(run_logprobs(xd[None], None, None, 1.0, 3, n, entropy=True), x, tokens, 1.0, 3)
    check_logprobs(run_logprobs(xd[None], None, tokens.to(DEV)[None], 1.0, 0, n, entropy=True), x, tokens, 1.0, 0)
    # sequences of one row each, rows of a padded buffer
    got = run_logprobs(xd[:, None], None, tokens.to(DEV)[:, None], 1.0, 2, 1)
    check_logprobs({name: v.transpose(0, 1) for name, v in got.items()}, x, tokens, 1.0, 2)


def saved(x, T):
    r = ref.logprobs(x, torch.zeros(len(x), **i32), T, 1)
    return r["stats"].float().to(DEV), r["entropy"].float().to(DEV)


def check_grad(got, want, size, dtype, V, what=""):
    ref.close(got, want, ref.HALF[dtype] * want.abs() + 8 * ref.delta(V) * size + ref.TINY, what)


GRADS = [(1, 1), (2, 7), (3, 8), (2, 13), (5, 1000), (3, 8193), (2, 50001), (2, 128257), (2100, 130), (2, 300001)]


@pytest.mark.parametrize("n, V", GRADS)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T", [1.0, 0.6])
def test_logprobs_grad(n, V, dtype, T):
    x, xd = rows(n, V, dtype, n + V, offset=V % 5, pad=3)
    g = torch.Generator().manual_seed(V)
    tokens = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
    tokens[0] = V - 1
    if n > 2:
        tokens[1], tokens[2] = -1, V
    a, b = torch.randn(n, generator=g), torch.randn(n, generator=g)
    stats, entropy = saved(x, T)
    room = dirty(n, V + 9, dtype=dtype)
    for aa, bb in ((a, b), (a, None), (None, b), (None, None)):
        grad = room[:, 2:2 + V]
        room.fill_(NAN)
        dt.dt_token_logprobs_grad(xd, tokens.to(DEV) if aa is not None else None, T, stats, entropy if bb is not None else None,
                                  aa.to(DEV) if aa is not None else None, bb.to(DEV) if bb is not None else None, grad)
        z = torch.zeros(n)
        want, size = ref.logprobs_grad(x, tokens, T, z if aa is None else aa, z if bb is None else bb)
        check_grad(grad, want, size, dtype, V, (aa is None, bb is None))
        assert torch.isnan(room[:, :2]).all() and torch.isnan(room[:, 2 + V:]).all()       # what lies between is left as it was
    same = xd.clone() if n == 1 else put(x, 1, 2)
    dt.dt_token_logprobs_grad(same, tokens.to(DEV), T, stats, entropy, a.to(DEV), b.to(DEV), same)      # in the logits' own place
    dt.dt_token_logprobs_grad(xd, tokens.to(DEV), T, stats, entropy, a.to(DEV), b.to(DEV), grad)
    assert torch.equal(same, grad)


def test_logprobs_grad_of_special_rows():
    for dtype in (BF16, F32):
        V = 5000
        named = special_rows(V, dtype)
        del named["large"], named["very large"]          # (their probabilities are 0 or 1: the next assertion)
        x = torch.stack(list(named.values()))
        n = len(x)
        tokens = torch.full((n,), V // 2, **i32)
        a, b = torch.ones(n), torch.full((n,), 0.5)
        o = run_logprobs(put(x)[None], None, tokens.to(DEV)[None], 1.0, 0, n)
        grad = dirty(n, V, dtype=dtype)
        dt.dt_token_logprobs_grad(put(x), tokens.to(DEV), 1.0, o["stats"][0], o["entropy"][0], a.to(DEV), b.to(DEV), grad)
        want, size = ref.logprobs_grad(x, tokens, 1.0, a, b)
        scale = 1 + 400.0 / 32                           # |x| up to 320: its differences' roundings
        ref.close(grad, want, ref.HALF[dtype] * want.abs() + 8 * ref.delta(V) * scale * size + ref.TINY)


def teacher(n, V, k, seed, short=True):
    g = torch.Generator().manual_seed(seed)
    y = torch.randn(n, V, generator=g) * 2.5
    val, ids = torch.topk(y, min(k, V), dim=1)
    lse = torch.logsumexp(y, 1)
    if k > V:
        val = torch.cat([val, torch.full((n, k - V), -math.inf)], 1)
        ids = torch.cat([ids, torch.full((n, k - V), -1)], 1)
    ids = ids.int()
    if short and k > 2:
        ids[0, k - 1], val[0, k - 2] = -1, -math.inf     # entries that are none: no token, no probability
        if n > 1:
            ids[1, 0] = V                                 # a token out of range
        if n > 2:
            ids[2, 1] = ids[2, 0]                         # a token twice
    return val, ids, lse


def run_distill(xd, val, ids, lse, of, T, flags, w, with_grad, grad=None):
    n, V = xd.shape
    dev = lambda v: None if v is None else v.to(DEV)
    o = dict(loss=dirty(n), stats=dirty(n, 2), tail=dirty(n))
    if with_grad and grad is None:
        grad = dirty(n, V, dtype=xd.dtype)
    t = [dev(val), dev(ids), dev(lse), dev(of)]
    dt.dt_distill_rows(xd, *t, T, flags, dev(w), o["loss"], o["stats"], o["tail"], grad if with_grad else None, workspace(n, V))
    torch.cuda.synchronize()
    if with_grad:
        o["grad"] = grad
        again = dirty(n, V, dtype=xd.dtype)               # and the gradient on its own, if the logits are still there
        if grad.data_ptr() != xd.data_ptr():
            dt.dt_distill_rows_grad(xd, *t, T, flags, dev(w), o["stats"], o["tail"], again)
            o["again"] = again
    return o


def check_distill(o, want, dtype, V):
    d = ref.delta(V)
    n = len(want["loss"])
    ref.close(o["loss"], want["loss"], 2 * d * want["terms"] + ref.U * want["loss"].abs().nan_to_num(posinf=0.0), "loss")
    ref.close(o["stats"][:, 0], want["stats"][:, 0], 0.0, "largest logit")
    ref.close(o["stats"][:, 1], want["stats"][:, 1], torch.full((n,), d, dtype=torch.float64), "log sum")
    # relative to what is small, the probability outside S or inside: log q_t = log(1 - inside)
    ref.close(o["tail"], want["tail"], 2 * d * (1 + want["tail"].abs().nan_to_num(posinf=0.0)), "tail")
    for name in ("grad", "again"):
        if name in o:
            check_grad(o[name], want["grad"], want["size"], dtype, V, name)


DISTILL = [(1, 1, 1), (2, 7, 4), (3, 9, 12), (4, 1000, 10), (3, 8193, 128), (3, 50001, 20), (2, 128257, 32), (2100, 130, 6), (2, 300001, 5)]


@pytest.mark.parametrize("n, V, k", DISTILL)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("flags", [0, dt.DT_DISTILL_TAIL, dt.DT_DISTILL_RENORM], ids=["plain", "tail", "renorm"])
def test_distill(n, V, k, dtype, flags):
    x, xd = rows(n, V, dtype, n + V, offset=V % 3, pad=1)
    val, ids, lse = teacher(n, V, k, V + k)
    w = torch.rand(n, generator=torch.Generator().manual_seed(n))
    T = 1.0 if V % 2 else 1.7
    want = ref.distill(x, val, ids, lse, None, T, flags, w)
    check_distill(run_distill(xd, val, ids, lse, None, T, flags, w, True), want, dtype, V)
    o = run_distill(xd, val, ids, lse, None, T, flags, None, False)
    want["grad"] = None
    check_distill(o, want, dtype, V)
    same = put(x, 1, 2)                                   # in the logits' own place
    o = run_distill(same, val, ids, lse, None, T, flags, w, True, grad=same)
    check_distill(o, ref.distill(x, val, ids, lse, None, T, flags, w), dtype, V)


def test_teachers_for_several_rows_and_for_none():
    n, m, V, k = 9, 4, 3001, 5
    for dtype in (BF16, F32):
        x, xd = rows(n, V, dtype, 3)
        val, ids, lse = teacher(m, V, k, 8)
        of = torch.tensor([0, 0, 3, -1, 2, 1, 4, -(1 << 31), 3], **i32)
        for many in (1, 300):
            X, D = x.repeat(many, 1), put(x.repeat(many, 1))
            w = torch.rand(n, generator=torch.Generator().manual_seed(n)).repeat(many)
            o = run_distill(D, val - lse[:, None], ids, None, of.repeat(many), 1.0, 1, w, True)
            want = ref.distill(x, val - lse[:, None], ids, None, of, 1.0, 1, w)
            # (3,001 entries: the copies of a row lie at other addresses modulo 16 bytes, so that their sums have another order)
            for i in range(0, many, 60):
                part = {v: o[v][i * n:(i + 1) * n] for v in ("loss", "stats", "tail", "grad", "again")}
                check_distill(part, want, dtype, V)
            o = {v: o[v][:n] for v in ("loss", "stats", "tail", "grad", "again")}
            none = ((of < 0) | (of >= m)).to(DEV)
            assert all((o[v][none] == 0).all() for v in ("loss", "stats", "tail", "grad", "again"))


def test_students_that_are_certain_masked_or_listed_whole():
    V, k = 60, 60
    g = torch.Generator().manual_seed(5)
    x = torch.randn(6, V, generator=g) * 2
    x[0, 7] = 60.0                                        # certain: 1e-24 outside S
    x[1, 20:] = -math.inf                                 # nothing outside S
    x[2, 3] = -math.inf                                   # 0 where the teacher has some
    x[3] = -math.inf                                      # nothing
    ids = torch.full((6, k), -1, **i32)
    val = torch.full((6, k), -math.inf)
    y = torch.log_softmax(torch.randn(6, V, generator=g), 1)
    for r in range(6):
        c = V if r == 5 else 20                           # the whole vocabulary listed
        ids[r, :c], val[r, :c] = torch.arange(c, **i32), y[r, :c]
    ids[4] = -1                                           # a teacher without entries
    for dtype in (BF16, F32):
        xr = x.to(dtype)
        for flags in (0, 1, 2):
            want = ref.distill(xr, val, ids, None, None, 1.0, flags)
            o = run_distill(put(xr), val, ids, None, None, 1.0, flags, None, True)
            fin = torch.isfinite(want["loss"])
            want["loss"][~fin] = math.inf
            want["terms"][~fin] = 0.0
            scale = 1 + 60.0 / 24                          # |x| up to 60
            ref.close(o["loss"], want["loss"], 2 * scale * ref.delta(V) * want["terms"] + 1e-6, (flags, "loss"))
            ref.close(o["tail"], want["tail"], 4 * scale * ref.delta(V) * (1 + want["tail"].abs().nan_to_num(posinf=0.0)), (flags, "tail"))
            for name in ("grad", "again"):
                check_grad(o[name], want["grad"], scale * want["size"], dtype, V, (flags, name))


def test_rows_beyond_32_bit_offsets():
    V, n, stride = 1003, 3, (1 << 30) + 5
    room = torch.empty(2 * stride + V + 16, dtype=BF16, device=DEV)
    xd = room.as_strided((n, V), (stride, 1), 3)
    x, _ = rows(n, V, BF16, 11)
    xd.copy_(x)
    tokens = torch.tensor([5, 0, V - 1], **i32)
    check_logprobs(run_logprobs(xd[None], None, tokens.to(DEV)[None], 1.0, 4, n), x, tokens, 1.0, 4)
    val, ids, lse = teacher(n, V, 6, 3)
    want = ref.distill(x, val, ids, lse, None, 1.0, 1)
    check_distill(run_distill(xd, val, ids, lse, None, 1.0, 1, None, True), want, BF16, V)
    o = run_distill(xd, val, ids, lse, None, 1.0, 1, None, True, grad=xd)
    check_distill(o, want, BF16, V)


def _chain(n, V, k, seed):
    """Teacher's rows -> their best -> the student's loss and gradient, and the student's own log-probabilities with theirs."""
    xs, ys = rows(n, V, BF16, seed)[1], rows(n, V, BF16, seed + 1)[1]
    b = dict(xs=xs, ys=ys, tokens=torch.randint(0, V, (1, n), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).to(DEV),
             g=torch.ones(n, device=DEV), lp=dirty(1, n), H=dirty(1, n), st=dirty(1, n, 2), tl=dirty(1, n, k), ti=dirty(1, n, k, dtype=torch.int32),
             st2=dirty(1, n, 2), lp2=dirty(1, n), H2=dirty(1, n), loss=dirty(n), dst=dirty(n, 2), tail=dirty(n), grad=dirty(n, V, dtype=BF16),
             grad2=dirty(n, V, dtype=BF16), ws=workspace(n, V))

    def run():
        dt.dt_token_logprobs(b["ys"][None], None, None, 1.0, k, None, None, b["st"], b["tl"], b["ti"], b["ws"])
        dt.dt_distill_rows(b["xs"], b["tl"][0], b["ti"][0], None, None, 1.0, 1, b["g"], b["loss"], b["dst"], b["tail"], b["grad"], b["ws"])
        dt.dt_token_logprobs(b["xs"][None], None, b["tokens"], 1.0, 0, b["lp2"], b["H2"], b["st2"], None, None, b["ws"])
        dt.dt_token_logprobs_grad(b["xs"], b["tokens"][0], 1.0, b["st2"][0], b["H2"][0], b["g"], b["g"], b["grad2"])
    return b, run


OUT = ("tl", "ti", "loss", "dst", "tail", "grad", "lp2", "H2", "st2", "grad2")


@pytest.mark.parametrize("n, V", [(7, 20003), (2100, 700)])
def test_chain_twice_in_graphs_and_on_other_streams(n, V):
    b, run = _chain(n, V, 5, n)
    run()
    torch.cuda.synchronize()
    first = {name: b[name].clone() for name in OUT}
    x, y = b["xs"].cpu(), b["ys"].cpu()
    want_t = ref.logprobs(y, torch.zeros(n, **i32), 1.0, 5)
    assert torch.equal(b["ti"][0].cpu(), want_t["top_id"])
    if n < 100:
        want = ref.distill(x, b["tl"][0].cpu(), b["ti"][0].cpu(), None, None, 1.0, 1)
        check_distill(dict(loss=b["loss"], stats=b["dst"], tail=b["tail"], grad=b["grad"]), want, BF16, V)

    def same(what):
        for name in OUT:
            assert torch.equal(b[name].view(torch.uint8), first[name].view(torch.uint8)), (what, name)
            b[name].fill_(3)
    run()
    torch.cuda.synchronize()
    same("again")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    same("another stream")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    other, run_other = _chain(3, V, 5, n + 50)
    for i in range(4):                                    # replays with eager work between them, the workspace used by it too
        other["ws"] = b["ws"]
        run_other()
        b["ws"].fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        same("replay %d" % i)


def test_a_step_says_what_it_emitted_and_what_the_draft_can_learn():
    """Tree, acceptance, then the log-probabilities of the emitted tokens and the draft rows' loss against the target's rows."""
    import dt_synth
    from paper_2601_12212_amd.step import Step
    from tests._cases import make_step, oracle_case
    for ci in (1, 2):
        case = oracle_case(ci)
        c, st = case.cfg, make_step(case)
        assert isinstance(st, Step)
        st.build_tree()
        st.accept()
        k = 6
        em = st.token_logprobs(k)
        grad = dirty(st.total_rows, st.V, dtype=st.dtype)
        w = torch.rand(st.total_rows, generator=torch.Generator().manual_seed(1)).to(DEV)
        loss = st.draft_loss(k, grad_loss=w, grad=grad)
        torch.cuda.synchronize()
        T = 1.0 if c.mode == dt_synth.GREEDY else c.temperature
        for b in range(c.B):
            acc = st.accepted(b)
            target = st.target_logits[b].cpu()
            m = acc["accept_len"] + 1
            nodes, toks = torch.from_numpy(acc["path_nodes"][:m].copy()).long(), torch.from_numpy(acc["out_tokens"][:m].copy()).int()
            check_logprobs({name: em[name][b:b + 1, :m] for name in ("logprob", "entropy", "stats", "top_logprob", "top_id")}, target[nodes], toks, T, k)
            assert (em["logprob"][b, m:] == 0).all() and (em["top_id"][b, m:] == -1).all()
            tree = st.tree(b)
            r0, r1 = int(st.host_row_off[b]), int(st.host_row_off[b + 1])
            of = torch.full((r1 - r0,), -1, **i32)
            for i, r in enumerate(tree["src_row"]):
                if r >= 0:
                    of[r] = i
            assert (of >= 0).sum() > 1
            best = ref.logprobs(target[:tree["n_nodes"]], torch.zeros(tree["n_nodes"], **i32), 1.0, k)
            x = st.draft_logits[r0:r1].cpu()
            want = ref.distill(x, best["top_logprob"], best["top_id"], None, of, 1.0, 1, w[r0:r1].cpu())
            d = 3 * ref.delta(st.V)                        # the teacher's values have been rounded and summed once more
            ref.close(loss[r0:r1], want["loss"], d * want["terms"], "loss")
            ref.close(grad[r0:r1], want["grad"], ref.HALF[st.dtype] * want["grad"].abs() + 8 * d * want["size"] + ref.TINY, "grad")


# How rows are cut among workgroups goes by their number, length and type: one of each kind, and the edges between them.
CUTS = [(127, 33001, 3), (128, 33001, 3), (200, 50003, 0), (256, 40001, 20), (257, 40001, 1), (300, 33001, 20), (512, 32769, 0), (513, 33003, 4),
        (600, 50001, 20), (3000, 31, 3), (100, 16384, 7), (100, 16385, 7), (90, 32768, 31),
        (256, 20001, 5), (257, 20001, 5), (600, 30001, 0), (512, 12001, 9), (513, 12001, 9),
        (79, 40001, 6), (80, 40001, 6), (160, 40001, 6), (161, 40001, 6), (256, 90001, 6), (90, 270001, 2), (40, 50001, 32)]


@pytest.mark.parametrize("n, V, k", CUTS)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_logprobs_by_number_of_rows(n, V, k, dtype):
    x, xd = rows(n, V, dtype, n + V, offset=1, pad=2)
    tokens = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(V), dtype=torch.int32)
    got = run_logprobs(xd[None], None, tokens.to(DEV)[None], 1.0, k, n)
    some = torch.unique(torch.cat([torch.arange(0, n, max(1, n // 40)), torch.tensor([n - 1])]))
    check_logprobs({name: v[:, some.to(DEV)] for name, v in got.items()}, x[some], tokens[some], 1.0, k)


@pytest.mark.parametrize("V", [41001, 90001])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B, per", [(5, 8), (7, 40), (9, 80)])
def test_chosen_rows_by_their_number(B, per, V, dtype):
    """Long rows that are named one by one, half of them none: entries in parts, wide, whole."""
    R, k = 4, 5
    x, xd = rows(B * R, V, dtype, V + B)
    g = torch.Generator().manual_seed(per)
    of = torch.randint(-R, R, (B, per), generator=g, dtype=torch.int32)
    tok = torch.randint(0, V, (B, per), generator=g, dtype=torch.int32)
    got = run_logprobs(xd.view(B, R, V), of.to(DEV), tok.to(DEV), 0.8, k, per)
    none = (of < 0).to(DEV)
    assert (got["logprob"][none] == 0).all() and (got["stats"][none] == 0).all() and (got["top_id"][none] == -1).all()
    for b in (0, B - 1):
        keep = of[b] >= 0
        at = keep.nonzero()[:, 0].to(DEV)
        check_logprobs({name: v[b:b + 1, at] for name, v in got.items()}, x[b * R + of[b][keep].long()], tok[b][keep], 0.8, k)


def test_more_entries_than_a_launch_of_large_workgroups_has():
    """2^23 entries of 16,385: by 512 threads each they would be 2^32."""
    n, V = 1 << 23, 16385
    x, xd = rows(2, V, BF16, 1)
    of = torch.arange(n, dtype=torch.int32, device=DEV) % 3 - 1
    stats = dirty(1, n, 2)
    dt.dt_token_logprobs(xd[None], of[None], None, 1.0, 0, None, None, stats, None, None, workspace(n, V))
    torch.cuda.synchronize()
    got = stats[0]
    ref.close(got[1:3, 1], ref.logprobs(x, torch.zeros(2, **i32), 1.0, 1)["stats"][:, 1], ref.delta(V))
    assert (got[0::3] == 0).all() and (got[1::3] == got[1]).all() and (got[2::3] == got[2]).all()


DISTILL_CUTS = [(127, 33001), (130, 33001), (130, 65536), (130, 70001), (256, 40001), (257, 40001), (300, 33001), (383, 32769), (384, 33003), (400, 41001),
                (400, 82001), (90, 32768), (90, 16385), (256, 20001), (257, 20001), (383, 16400), (400, 30001), (161, 40001), (512, 12001), (513, 12001), (352, 82001)]


@pytest.mark.parametrize("n, V", DISTILL_CUTS)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_distill_by_number_of_rows(n, V, dtype):
    k, T = 9, 1.3
    x, xd = rows(n, V, dtype, n + V, offset=3, pad=1)
    val, ids, lse = teacher(n, V, k, V + n)
    w = torch.rand(n, generator=torch.Generator().manual_seed(n))
    some = torch.unique(torch.cat([torch.arange(0, n, max(1, n // 12)), torch.tensor([1, 2, n - 1])]))
    want = ref.distill(x[some], val[some], ids[some], lse[some], None, T, 1, w[some])
    pick = lambda o: {name: v[some.to(DEV)] for name, v in o.items()}
    check_distill(pick(run_distill(xd, val, ids, lse, None, T, 1, w, True)), want, dtype, V)
    check_distill(pick(run_distill(xd, val, ids, lse, None, T, 1, None, False)), want, dtype, V)
    same = put(x, 3, 1)                                   # in the logits' own place
    check_distill(pick(run_distill(same, val, ids, lse, None, T, 1, w, True, grad=same)), want, dtype, V)


@pytest.mark.parametrize("n, m, V", [(20, 3, 50003), (100, 127, 33001), (300, 40, 33001), (200, 300, 40001), (5, 6, 300001)])
def test_graphs_that_share_a_workspace(n, m, V):
    """Two captured calls with one workspace, replayed in turn on one stream with a third call of other sizes between them."""
    one, run_one = _chain(n, V, 5, n)
    two, run_two = _chain(m, V, 2, m + 7)
    third, run_third = _chain(4, V // 2, 3, 1)
    ws = workspace(max(n, m), V)
    one["ws"] = two["ws"] = third["ws"] = ws
    first, graphs = [], []
    for b, run in ((one, run_one), (two, run_two)):
        run()
        torch.cuda.synchronize()
        first.append({name: b[name].clone() for name in OUT})
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        graphs.append(graph)
    want = ref.logprobs(one["ys"][:3].cpu(), torch.zeros(3, **i32), 1.0, 5)
    assert torch.equal(first[0]["ti"][0, :3].cpu(), want["top_id"])
    for i in (0, 1, 1, 0, 0, 1):
        for b in (one, two):
            for name in OUT:
                b[name].fill_(3)
        graphs[i].replay()
        run_third()
        graphs[1 - i].replay()
        torch.cuda.synchronize()
        for b, f in zip((one, two), first):
            for name in OUT:
                assert torch.equal(b[name].view(torch.uint8), f[name].view(torch.uint8)), (i, name)


@pytest.mark.parametrize("n, V, k", [(4, 4480, 1), (4, 4480, 9), (3, 1500, 3), (130, 40001, 5), (6, 50001, 2)])
@pytest.mark.parametrize("noise", [0.0, 1e-3])
def test_gradient_of_students_that_are_near_their_teacher(n, V, k, noise):
    """Outside S the gradient is q_j / q_t (P q_t - p_t q_in), which is known to the digits of its two terms, however near to each other P and p_t + P q_in
    may be: 8 delta times their sum, as for other gradients of size times delta."""
    x, xd = rows(n, V, F32, n + V, offset=1, pad=1)
    g = torch.Generator().manual_seed(k)
    y = torch.log_softmax((x.double() / 2.0) + noise * torch.randn(n, V, generator=g, dtype=torch.float64), 1)
    pick = torch.argsort(torch.rand(n, V, generator=g), 1)[:, :k]               # any entries, not the best: little in S
    val, ids = y.gather(1, pick).float(), pick.int()
    want = ref.distill(x, val, ids, None, None, 2.0, 1)
    o = run_distill(xd, val, ids, None, None, 2.0, 1, None, True)
    check_distill(o, want, F32, V)
    lq = torch.log_softmax(x.double() / 2.0, 1)
    P = torch.exp(val.double()).sum(1, keepdim=True)
    q_in = torch.exp(lq.gather(1, pick)).sum(1, keepdim=True)
    q = torch.exp(lq)
    outside = torch.ones(n, V, dtype=torch.bool).scatter(1, pick, False)
    tol = 8 * ref.delta(V) * q / (1 - q_in) * (P * (1 - q_in) + (1 - P) * q_in) + ref.HALF[F32] * want["grad"].abs() + ref.TINY
    # (p_t is 1 - P, of fp32's digits: its own half step is one of delta's)
    for name in ("grad", "again"):
        ref.close(o[name].cpu()[outside], want["grad"][outside], tol[outside], name)
    ref.close(o["tail"], want["tail"], 2 * ref.delta(V) * want["tail"].abs() * 1.5, "tail")    # relative: q_in is a sum of its own, and log(1 - q_in) is its size


@pytest.mark.parametrize("n, V", [(3, 300), (3, 5000), (130, 40001), (6, 50001), (300, 33001)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("flags", [0, 1, 2])
def test_students_that_are_as_good_as_certain(n, V, dtype, flags):
    """What lies outside S is e^-500: nothing beside the largest logit in fp32, and yet its logarithm and its shares are there."""
    k, T = 4, 0.4
    x, _ = rows(n, V, dtype, V)
    val, ids, lse = teacher(n, V, k, 5, short=False)
    x = x.scatter(1, ids[:, :1].long(), 200.0)
    some = torch.tensor([0, 1, n - 1])
    want = ref.distill(x[some], val[some], ids[some], lse[some], None, T, flags)
    assert torch.isfinite(want["loss"]).all() and (want["tail"] < -400).all()
    o = run_distill(put(x), val, ids, lse, None, T, flags, None, True)
    scale = 1 + 200.0 / T / 24                            # |x| / T up to 500
    d = scale * ref.delta(V)
    o = {name: v[some.to(DEV)] for name, v in o.items()}
    ref.close(o["loss"], want["loss"], 2 * d * want["terms"], "loss")
    ref.close(o["tail"], want["tail"], 2 * d * (1 + want["tail"].abs()), "tail")
    for name in ("grad", "again"):
        check_grad(o[name], want["grad"], scale * want["size"], dtype, V, (flags, name))


@pytest.mark.parametrize("n", [1, 33, 130])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_largest_vocabulary(n, dtype):
    """DT_VOCAB_MAX entries, the most alternatives, the most teacher's entries."""
    V, k = dt.DT_VOCAB_MAX, 32
    g = torch.Generator().manual_seed(n)
    some = torch.unique(torch.tensor([0, n // 2, n - 1]))
    x = (torch.randn(len(some), V, generator=g) * 3).to(dtype)
    xd = (torch.randn(n, V, device=DEV) * 2).to(dtype)
    xd[some.to(DEV)] = x.to(DEV)
    tokens = torch.full((n,), V - 1, **i32)
    got = run_logprobs(xd[None], None, tokens.to(DEV)[None], 1.0, k, n)
    check_logprobs({name: v[:, some.to(DEV)] for name, v in got.items()}, x, tokens[some], 1.0, k)
    val, ids, lse = teacher(len(some), V, 128, n, short=False)
    m = torch.full((n,), -1, **i32)
    m[some] = torch.arange(len(some), **i32)
    o = run_distill(xd, val, ids, lse, m, 1.0, 1, None, True)
    want = ref.distill(x, val, ids, lse, None, 1.0, 1)
    check_distill({name: v[some.to(DEV)] for name, v in o.items()}, want, dtype, V)
    o = run_distill(xd, val, ids, lse, m, 1.0, 1, None, False)
    check_distill({name: v[some.to(DEV)] for name, v in o.items()}, want, dtype, V)


@pytest.mark.parametrize("n, V", [(1, 524288), (5, 50001), (79, 40001), (127, 33001), (300, 33001), (383, 40001), (40, 300001)])
def test_workspaces_hold_what_is_left_in_them(n, V):
    """What lies behind the bytes that were asked for stays as it was."""
    x = torch.randn(n, V, device=DEV).to(BF16)
    size = dt.dt_logprob_workspace_bytes(n, V)
    room = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    ws = room[:size]
    o = dict(st=dirty(1, n, 2), tl=dirty(1, n, 32), ti=dirty(1, n, 32, dtype=torch.int32))
    dt.dt_token_logprobs(x[None], None, None, 1.0, 32, None, None, o["st"], o["tl"], o["ti"], ws)
    val, ids = torch.full((n, 128), -6.0, device=DEV), torch.arange(128, dtype=torch.int32, device=DEV).repeat(n, 1)
    for grad in (None, torch.empty_like(x)):
        dt.dt_distill_rows(x, val, ids, None, None, 1.0, 1, None, dirty(n), dirty(n, 2), dirty(n), grad, ws)
    torch.cuda.synchronize()
    assert (room[size:] == 0x5A).all()


@pytest.mark.parametrize("n, V", [(1, 12000), (140, 20000), (7, 40000), (140, 40000), (300, 40000), (600, 20000)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_best_of_rows_whose_best_are_neighbours_or_far_apart(n, V, dtype):
    """The k best all in one thread's elements, in one go, in the first and last places, one to a go; ties at the k-th."""
    k = 20
    g = torch.Generator().manual_seed(V + n)
    base = (torch.randn(V, generator=g)).to(dtype)
    places = [torch.arange(k) + V // 2, torch.arange(k) * (V // k), torch.cat([torch.arange(k // 2), torch.arange(V - k // 2, V)]), torch.arange(k) * 8 + 3,
              torch.arange(k + 40) * 100, torch.randperm(V, generator=g)[:k]]
    x = torch.stack([base] * len(places))
    for r, at in enumerate(places):
        x[r, at] = (10.0 + torch.arange(len(at)) // 2 * 0.25).to(dtype) if r != 4 else torch.tensor(9.0, dtype=dtype)
    reps = (n - 1) // len(x) + 1
    got = run_logprobs(put(x.repeat(reps, 1), 1, 3)[None], None, None, 1.0, k, reps * len(x))
    want = ref.logprobs(x, torch.zeros(len(x), **i32), 1.0, k)
    ids = got["top_id"][0].cpu().view(reps, len(x), k)
    assert torch.equal(ids, want["top_id"][None].expand_as(ids))
