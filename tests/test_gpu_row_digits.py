"""Digits and ranges of the row operators: results that are known to a few roundings, wherever in a row the tokens lie, at every temperature, and for every
way that rows are cut among workgroups."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2601_12212_amd as dt  # noqa: E402
from tests import _token_rows as ref  # noqa: E402
from tests.test_gpu_token_rows import (BF16, DEV, F32, LOWEST, check_distill, i32, put, rows, run_distill, run_logprobs, special_rows, teacher)  # noqa: E402

U = ref.U
IDS = dict(ids=["bf16", "f32"])
# one of each way that rows are cut: (rows, entries) held by 64, 256, 512 and 1,024 threads; in parts; wide; by 256 threads; too short to be cut
CUTS = [(3, 1501), (3, 8003), (3, 13001), (5, 20011), (3, 50021), (140, 50021), (600, 20011), (3, 19), (2, 5)]


# ---- DT_DISTILL_RENORM: p_i / P does not depend on what all entries share

def _spread(n, k, seed):
    """Teacher's values on a grid of 2^-6, so that they stay what they are when a shift of up to 2^10 is added."""
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, k, generator=g) * 3 * 64).round() / 64


@pytest.mark.parametrize("n, V", CUTS + [(400, 70001)])
@pytest.mark.parametrize("dtype", [BF16, F32], **IDS)
def test_renorm_is_the_same_at_any_shift(n, V, dtype):
    """Values that are logits as they come (30 / 0.25), or log-probabilities of tokens that a sharp teacher gives nothing."""
    k = min(V - 1, 7)
    x, xd = rows(n, V, dtype, n + V, offset=1, pad=1)
    val = _spread(n, k, V)
    ids = torch.stack([torch.randperm(V, generator=torch.Generator().manual_seed(r))[:k] for r in range(n)]).int()
    if k > 3:
        ids[0, 2], val[n - 1, 1] = -1, -math.inf              # entries that are none
        ids[1, 1] = ids[1, 0]
    w = torch.rand(n, generator=torch.Generator().manual_seed(n))
    some = torch.unique(torch.tensor([0, 1, n // 2, n - 1]))
    want = ref.distill(x[some], val[some], ids[some], None, None, 1.3, dt.DT_DISTILL_RENORM, w[some])
    first = run_distill(xd, val, ids, None, None, 1.3, dt.DT_DISTILL_RENORM, w, True)
    check_distill({name: v[some.to(DEV)] for name, v in first.items()}, want, dtype, V)
    alone = run_distill(xd, val, ids, None, None, 1.3, dt.DT_DISTILL_RENORM, w, False)
    for shift, lse in ((-300.0, None), (-104.0, None), (90.0, None), (200.0, None), (1000.0, None), (0.0, 150.0), (0.0, -500.0)):
        at = None if lse is None else torch.full((n,), lse)
        o = run_distill(xd, val + shift, ids, at, None, 1.3, dt.DT_DISTILL_RENORM, w, True)
        for name, v in o.items():
            assert torch.equal(v, first[name]), (shift, lse, name)
        o = run_distill(xd, val + shift, ids, at, None, 1.3, dt.DT_DISTILL_RENORM, w, False)
        assert torch.equal(o["loss"], alone["loss"]), (shift, lse)


def test_renorm_of_entries_next_to_nothing():
    """Three entries at -103, -104 and -105.5 are 0.690, 0.254 and 0.057 of their sum; entries 400 below the largest are nothing of it; no entries are none."""
    V = 300
    x, xd = rows(3, V, F32, 4)
    val = torch.tensor([[-103.0, -104.0, -105.5], [-500.0, -100.0, -501.0], [-math.inf, -math.inf, -math.inf]])
    ids = torch.tensor([[7, 3, 250], [9, 100, 2], [1, 2, 3]], **i32)
    want = ref.distill(x, val + 100, ids, None, None, 1.0, dt.DT_DISTILL_RENORM)      # (the reference is in 64 bits: nothing is lost there)
    o = run_distill(xd, val, ids, None, None, 1.0, dt.DT_DISTILL_RENORM, None, True)
    check_distill(o, want, F32, V)
    assert float(o["loss"][2]) == 0.0 and (o["grad"][2] == 0).all()


# ---- rows with one token that has all of the weight: its log-probability and the log of the sum are 0

def _places(V, dtype):
    """Ends of the row, and of its units, goes and parts wherever its address puts them."""
    unit = 8 if dtype == BF16 else 4
    at = {0, 1, 2, 3, 7, unit, unit + 1, V // 2, V - 1, V - 2, V - 3, V - unit, V - unit - 1}
    for edge in (2048, 8192, 16384, 32768):
        at |= {edge - 1, edge, edge + unit - 1, edge + 7}
    return sorted(a for a in at if 0 <= a < V)


@pytest.mark.parametrize("n, V", CUTS)
@pytest.mark.parametrize("dtype", [BF16, F32], **IDS)
@pytest.mark.parametrize("T", [1.0, 0.01, 1e-4])
@pytest.mark.parametrize("hidden", [True, False], ids=["masked", "far below"])
def test_a_certain_token_anywhere_in_its_row(n, V, dtype, T, hidden):
    """A row's other tokens are -inf, or too far below to count.  The weight is 2^r with |r| <= 2^-4, a rounding's; its exponential is off by one step (2 u) and so is
    the logarithm of that (2 u / ln 2 of a power, times ln 2): 4 u in all."""
    places = _places(V, dtype)
    n = max(n, len(places))
    g = torch.Generator().manual_seed(V)
    at = torch.tensor(places).repeat((n - 1) // len(places) + 1)[:n]
    value = (10.0 + 30.0 * torch.rand(n, generator=g)).to(dtype)
    x = (torch.full((n, V), -math.inf) if hidden else torch.randn(n, V, generator=g) - 200.0).to(dtype)
    x[torch.arange(n), at] = value
    for offset, pad in ((0, 0), (3, 1)):
        got = run_logprobs(put(x, offset, pad)[None], None, at.int().to(DEV)[None], T, 1, n)
        assert (got["logprob"].abs() <= 4 * U).all(), float(got["logprob"].abs().max())
        assert (got["stats"][0, :, 1].abs() <= 4 * U).all(), float(got["stats"][0, :, 1].abs().max())
        assert torch.equal(got["stats"][0, :, 0].cpu(), value.float())
        assert torch.equal(got["top_id"][0, :, 0].cpu(), at.int()) and (got["top_logprob"].abs() <= 4 * U).all()
        assert (got["entropy"].abs() <= 8 * U).all()       # log s - w / s: two terms of up to 2^-4, each off by a few of its steps


@pytest.mark.parametrize("n, V", CUTS + [(400, 70001)])
@pytest.mark.parametrize("dtype", [BF16, F32], **IDS)
@pytest.mark.parametrize("T", [1.0, 0.01, 1e-4])
def test_a_certain_token_among_the_teachers_entries_or_outside(n, V, dtype, T):
    """The certain token in S: the loss is log p of it (p = 1 here: 0), and outside S nothing.  Outside S: log q_t is 0, and so is the loss of a teacher that
    gives all to that outside."""
    g = torch.Generator().manual_seed(V)
    at = torch.tensor(_places(V, dtype)).repeat(n)[:n]
    x = torch.full((n, V), -math.inf).to(dtype)
    value = (10.0 + 30.0 * torch.rand(n, generator=g)).to(dtype)
    x[torch.arange(n), at] = value
    xd = put(x, 1, 1)
    o = run_distill(xd, torch.zeros(n, 1), at.int()[:, None], None, None, T, 0, None, True)
    assert (o["loss"].abs() <= 4 * U).all(), float(o["loss"].abs().max())
    assert (o["stats"][:, 1].abs() <= 4 * U).all() and (o["tail"] == -math.inf).all()
    # d = (q_j - 1) / T at the token, of which q_j is a sum's quotient (4 u) or from the saved logarithm
    for name in ("grad", "again"):
        assert (o[name].double().abs().amax(1) <= 8 * U / T).all(), name
    o = run_distill(xd, torch.full((n, 1), -1e5), ((at + 1) % V).int()[:, None], None, None, T, dt.DT_DISTILL_TAIL, None, False)
    assert (o["loss"].abs() <= 8 * U).all() and (o["tail"].abs() <= 4 * U).all(), float(o["tail"].abs().max())


# ---- the teacher's probabilities

@pytest.mark.parametrize("n, V", CUTS[:-2])
@pytest.mark.parametrize("left", [1e-4, 1e-6])
def test_what_a_teacher_that_is_nearly_certain_gives_to_other_tokens(n, V, left):
    """p_t = 1 - P where it is small: it is known to 2^-40 / p_t, so that the gradient outside S, which is p_t q_j / q_t for a student that is surer still, has
    the digits of others of its size."""
    k = 3
    g = torch.Generator().manual_seed(V)
    p = torch.rand(n, k, generator=g, dtype=torch.float64) * 0.2 + 0.2
    p[:, 0] += 0.3
    p = p / p.sum(1, keepdim=True) * (1 - left * (1 + torch.rand(n, 1, generator=g, dtype=torch.float64)))
    lse = torch.randn(n, generator=g) * 10
    val = (torch.log(p) + lse.double()[:, None]).float()
    P = torch.exp(val.double() - lse.double()[:, None]).sum(1)
    # (rounding val moves P by up to 2^-20: where that is more than what is to be left, the largest entry is lowered until it is not)
    while (1 - P < left).any():
        val[:, 0] = torch.where(1 - P < left, torch.nextafter(val[:, 0], torch.tensor(-math.inf)), val[:, 0])
        P = torch.exp(val.double() - lse.double()[:, None]).sum(1)
    ids = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(n)]).int()
    x = (torch.randn(n, V, generator=g) - 40.0).scatter(1, ids.long(), torch.rand(n, k, generator=g))
    some = torch.unique(torch.tensor([0, 1, n // 2, n - 1]))
    want = ref.distill(x[some], val[some], ids[some], lse[some], None, 1.0, 1)
    o = run_distill(put(x, 1, 1), val, ids, lse, None, 1.0, 1, None, True)
    assert (want["tail"] < -25).all()
    check_distill({name: v[some.to(DEV)] for name, v in o.items()}, want, F32, V)


# ---- the gradient in fp32

@pytest.mark.parametrize("n, V", [(2, 1000), (2, 2047), (3, 8003), (3, 13001), (5, 20011), (3, 50021), (3, 131071), (140, 33001), (140, 50021), (400, 66001), (600, 20011), (3, 19)])
@pytest.mark.parametrize("half", [False, True], ids=["all", "half of them masked"])
def test_gradients_of_equal_logits_have_fp32s_digits(n, V, half):
    """Logits 0 or -inf: every weight is 1 and every sum exact, so q = 1 / count to half a step, and the gradient outside S, P q, has P's rounding and those of q_t,
    P q_t, the sums' quotient (two) and the weight's product: 8 u at most; in S, (P q - p), three more, relative to both terms."""
    k = 2
    x = torch.zeros(n, V)
    if half:
        x[:, 1::2] = -math.inf
    ids = torch.stack([torch.arange(n) % 3 * 2, torch.full((n,), V - 1 - (V - 1) % 2)], 1).int()
    val = torch.log(torch.tensor([[0.3, 0.4]])).expand(n, k).contiguous()
    p = torch.exp(val.double())
    q = torch.where(x == 0, 1.0 / (x == 0).sum(1, keepdim=True).double(), 0.0).double()
    want = p.sum(1, keepdim=True) * q
    size = want.clone()
    want = want.scatter_add(1, ids.long(), -p)
    size = size.scatter_add(1, ids.long(), p)
    o = run_distill(put(x, 1, 1), val, ids, None, None, 1.0, 0, None, True)
    ref.close(o["grad"], want, 8 * U * size)


# ---- tokens that are masked by their type's lowest value

@pytest.mark.parametrize("n, V", CUTS)
@pytest.mark.parametrize("dtype", [BF16, F32], **IDS)
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_tokens_masked_by_the_lowest_value(n, V, dtype, T):
    """Their logits are finite, and so are their log-probabilities, (lowest - m) / T: four roundings, those of log2(e) / T, ln 2, their product and the last."""
    g = torch.Generator().manual_seed(V)
    x = torch.full((n, V), LOWEST[dtype])
    open_ = torch.stack([torch.randperm(V, generator=g)[:3] for _ in range(n)])
    x = x.scatter(1, open_, torch.randn(n, 3, generator=g)).to(dtype)
    masked = (open_[:, 0] + 1) % V
    while True:
        inside = (open_ == masked[:, None]).any(1)
        if not inside.any():
            break
        masked = torch.where(inside, (masked + 1) % V, masked)
    k = min(V, 5)
    some = torch.unique(torch.tensor([0, n // 2, n - 1]))
    want = ref.logprobs(x[some], masked[some].int(), T, k)
    assert torch.isfinite(want["logprob"]).all() and (want["logprob"] < -1e38).all()
    got = run_logprobs(put(x, 1, 1)[None], None, masked.int().to(DEV)[None], T, k, n)
    assert torch.equal(got["top_id"][0, some.to(DEV)].cpu(), want["top_id"])
    size = lambda v: ref.delta(V) + 6 * U * v.abs()
    ref.close(got["logprob"][0, some.to(DEV)], want["logprob"], size(want["logprob"]))
    ref.close(got["top_logprob"][0, some.to(DEV)], want["top_logprob"], size(want["top_logprob"]))
    # a teacher that gives such a token half of its weight: a loss of half of that
    val, ids = torch.full((n, 1), math.log(0.5)), masked.int()[:, None]
    for with_grad in (True, False):
        o = run_distill(put(x, 1, 1), val, ids, None, None, T, 0, None, with_grad)
        ref.close(o["loss"][some.to(DEV)], -0.5 * want["logprob"], 8 * U * want["logprob"].abs())


# ---- sums that nothing may be missing from

@pytest.mark.parametrize("n, V", CUTS + [(40, 300007), (300, 30001), (300, 33001), (400, 70001), (130, dt.DT_VOCAB_MAX)])
@pytest.mark.parametrize("dtype", [BF16, F32], **IDS)
@pytest.mark.parametrize("half", [False, True], ids=["all", "half of them masked"])
def test_sums_of_equal_logits_count_every_token(n, V, dtype, half):
    """Logits 0 or -inf: the sum is their number exactly (below 2^24), so that its logarithm is off by a step of its own, by log2's (one of 1.44 times that), and by the
    constant's and the product's: 6 u of it; the entropy is the same.  A unit of four tokens too few of 524,288 is 128 u, of 80 that are allowed there."""
    for offset, pad in ((0, 0), (3, 1)):
        room = torch.zeros(offset + n * (V + pad) + 8, dtype=dtype, device=DEV)
        xd = room[offset:offset + n * (V + pad)].view(n, V + pad)[:, :V]
        if half:
            xd[:, 1::2] = -math.inf
        count = (V + 1) // 2 if half else V
        tokens = torch.full((n,), (V - 1) // 2 * 2, **i32)
        got = run_logprobs(xd[None], None, tokens.to(DEV)[None], 1.0, 2, n)
        log = math.log(count)
        for name, want in (("logprob", -log), ("entropy", log), ("top_logprob", -log)):
            assert ((got[name].double() - want).abs() <= 6 * U * log).all(), (name, float((got[name].double() - want).abs().max()) / U)
        assert ((got["stats"][0, :, 1].double() - log).abs() <= 6 * U * log).all()
        # the teacher's k tokens taken out: log(1 - k / count), which log1p takes of k / count (a half step, and two of its own), or two logarithms
        k = min(3, (count - 1) // 2)
        ids = (torch.arange(k) * 2)[None].expand(n, k).int().contiguous()
        o = run_distill(xd, torch.full((n, k), math.log(0.25)), ids, None, None, 1.0, 0, None, False)
        rest = math.log1p(-k / count)
        assert ((o["tail"].double() - rest).abs() <= 6 * U * abs(rest)).all(), float((o["tail"].double() - rest).abs().max() / U)
        assert ((o["stats"][:, 1].double() - log).abs() <= 6 * U * log).all()


@pytest.mark.parametrize("dtype", [BF16, F32], **IDS)
def test_distill_of_128_rows(dtype):
    """The first number of long rows that are not in parts."""
    n, V, k, T = 128, 33001, 9, 1.3
    x, xd = rows(n, V, dtype, 5, offset=3, pad=1)
    val, ids, lse = teacher(n, V, k, 6)
    w = torch.rand(n, generator=torch.Generator().manual_seed(n))
    some = torch.tensor([0, 1, 2, 64, 127])
    want = ref.distill(x[some], val[some], ids[some], lse[some], None, T, 1, w[some])
    pick = lambda o: {name: v[some.to(DEV)] for name, v in o.items()}
    check_distill(pick(run_distill(xd, val, ids, lse, None, T, 1, w, True)), want, dtype, V)
    check_distill(pick(run_distill(xd, val, ids, lse, None, T, 1, None, False)), want, dtype, V)
    same = put(x, 3, 1)
    check_distill(pick(run_distill(same, val, ids, lse, None, T, 1, w, True, grad=same)), want, dtype, V)


@pytest.mark.parametrize("V", [41, 5003, 40009])
@pytest.mark.parametrize("dtype", [BF16, F32], **IDS)
@pytest.mark.parametrize("offset, pad, reps", [(1, 0, 1), (3, 2, 1), (5, 1, 1), (6, 3, 9), (7, 0, 17)])
def test_special_rows_at_any_address(V, dtype, offset, pad, reps):
    """Masks, ties and extremes where rows do not start with a unit, and at every part of a row's ends."""
    named = {name: v for name, v in special_rows(V, dtype).items() if not name.startswith(("large", "very"))}
    x = torch.stack(list(named.values())).roll(offset, 1)
    n = len(x)
    tokens = torch.full((n,), V - 2, **i32)
    want = ref.logprobs(x, tokens, 1.0, 20)
    got = run_logprobs(put(x.repeat(reps, 1), offset, pad)[None], None, tokens.repeat(reps).to(DEV)[None], 1.0, 20, n * reps)
    ids = got["top_id"][0].cpu().view(reps, n, 20)
    assert torch.equal(ids, want["top_id"].expand_as(ids))
    d = ref.delta(V) * (1 + 330.0 / 32)                   # |x| up to 330, or masked: (x - m) is rounded relative to itself
    size = lambda v: d + 6 * U * torch.where(torch.isfinite(v), v.abs(), 0.0)
    for name, tol in (("logprob", size(want["logprob"])), ("entropy", 2 * d * (1 + want["entropy"])), ("top_logprob", size(want["top_logprob"])), ("stats", d)):
        for part in got[name][0].reshape((reps, n) + tuple(want[name].shape[1:]))[::4]:
            ref.close(part, want[name], tol, name)


@pytest.mark.parametrize("n, V", [(700, 1001), (140, 50021)])
def test_gradients_in_bf16_are_the_fp32_ones_to_the_nearest(n, V):
    """Logits 0: all sums are exact, in both types the same, and so are the gradients but for bf16's one rounding."""
    g = torch.Generator().manual_seed(n)
    w, val = torch.randn(n, generator=g), torch.log(torch.rand(n, 2, generator=g) * 0.4 + 0.05)
    ids = torch.stack([torch.arange(n) % V, (torch.arange(n) + V // 2) % V], 1).int()
    out = {}
    for dtype in (F32, BF16):
        o = run_distill(torch.zeros(n, V, dtype=dtype, device=DEV), val, ids, None, None, 1.0, 1, w, True)
        tokens, stats = ids[:, 0].contiguous().to(DEV), o["stats"]
        lp = torch.empty(n, V, dtype=dtype, device=DEV)
        dt.dt_token_logprobs_grad(torch.zeros(n, V, dtype=dtype, device=DEV), tokens, 1.0, stats, stats[:, 1].contiguous(), w.to(DEV), val[:, 0].contiguous().to(DEV), lp)
        out[dtype] = (o["grad"], o["again"], lp)
    for a, b in zip(out[F32], out[BF16]):
        assert torch.equal(a.to(BF16), b)
