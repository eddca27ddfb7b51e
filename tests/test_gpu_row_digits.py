"""Digits and ranges of the row operators: results that are known to a few roundings, wherever in a row the tokens lie, at every temperature, and for every
way that rows are cut among workgroups."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2601_12212_amd as dt  # noqa: E402
from tests import _token_rows as ref  # noqa: E402
from tests.test_gpu_token_rows import (BF16, DEV, F32, LOWEST, check_distill, i32, put, rows, run_distill, run_logprobs,  # noqa: E402
                                       teacher)

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
