"""What the row operators refuse, on the host, before anything is launched; the plain implementations that the GPU tests
compare with against differences of their own losses."""
import ctypes as C
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2601_12212_amd as dt  # noqa: E402
from paper_2601_12212_amd import _dtcall, binding  # noqa: E402
from tests import _token_rows as ref  # noqa: E402

one, odd, ws = C.c_void_p(256), C.c_void_p(258), C.c_void_p(4096)
BIG = 1 << 30


def _logprobs(**kw):
    a = dict(stream=None, batch=2, per_seq=3, logits=one, t=1, V=1000, stride=1000, rows=8, row_of=one, tokens=one, T=1.0, k=4, logprob=one,
             entropy=one, stats=one, top=one, ids=one, ws=ws, wsb=BIG)
    a.update(kw)
    return dt.load_library().dt_token_logprobs(*a.values())


def _logprobs_grad(**kw):
    a = dict(stream=None, n=3, logits=one, t=1, V=1000, stride=1000, tokens=one, T=1.0, stats=one, entropy=one, g=one, h=one, grad=ws,
             gstride=1000)
    a.update(kw)
    return dt.load_library().dt_token_logprobs_grad(*a.values())


def _distill(**kw):
    a = dict(stream=None, n=3, logits=one, t=1, V=1000, stride=1000, k=4, m=3, val=one, ids=one, lse=None, rows=None, T=1.0, flags=1, w=None,
             loss=one, stats=one, tail=one, grad=ws, gstride=1000, ws=ws, wsb=BIG)
    a.update(kw)
    return dt.load_library().dt_distill_rows(*a.values())


def _distill_grad(**kw):
    a = dict(stream=None, n=3, logits=one, t=1, V=1000, stride=1000, k=4, m=3, val=one, ids=one, lse=None, rows=None, T=1.0, flags=1, w=None,
             stats=one, tail=one, grad=ws, gstride=1000)
    a.update(kw)
    return dt.load_library().dt_distill_rows_grad(*a.values())


@pytest.mark.parametrize("call, kw, status", [
    (_logprobs, dict(batch=-1), -1), (_logprobs, dict(per_seq=-1), -1), (_logprobs, dict(t=7), -1), (_logprobs, dict(logits=None), -1),
    (_logprobs, dict(stats=None), -1), (_logprobs, dict(tokens=None), -1), (_logprobs, dict(top=None), -1), (_logprobs, dict(ids=None), -1),
    (_logprobs, dict(stride=999), -1), (_logprobs, dict(rows=0), -1), (_logprobs, dict(row_of=None, rows=2), -1), (_logprobs, dict(k=-1), -1),
    (_logprobs, dict(T=0.0), -1), (_logprobs, dict(T=-1.0), -1), (_logprobs, dict(T=1e-5), -1), (_logprobs, dict(T=2e4), -1),
    (_logprobs, dict(T=math.nan), -1), (_logprobs, dict(T=math.inf), -1), (_logprobs, dict(logits=C.c_void_p(257)), -1),
    (_logprobs, dict(t=0, logits=odd), -1), (_logprobs, dict(stats=odd), -1), (_logprobs, dict(logprob=odd), -1), (_logprobs, dict(row_of=odd), -1),
    (_logprobs, dict(V=0), -2), (_logprobs, dict(V=524289, stride=600000), -2), (_logprobs, dict(k=33), -2), (_logprobs, dict(V=3, k=4), -2),
    (_logprobs, dict(batch=1 << 20, per_seq=16), -2), (_logprobs, dict(ws=None), -3), (_logprobs, dict(ws=C.c_void_p(4100)), -3),
    (_logprobs, dict(wsb=16), -3), (_logprobs, dict(batch=0), 0), (_logprobs, dict(per_seq=0), 0),
    (_logprobs_grad, dict(n=-1), -1), (_logprobs_grad, dict(t=2), -1), (_logprobs_grad, dict(logits=None), -1), (_logprobs_grad, dict(stats=None), -1),
    (_logprobs_grad, dict(tokens=None), -1), (_logprobs_grad, dict(entropy=None), -1), (_logprobs_grad, dict(grad=None), -1),
    (_logprobs_grad, dict(gstride=999), -1), (_logprobs_grad, dict(grad=one, gstride=1008), -1), (_logprobs_grad, dict(T=0.0), -1),
    (_logprobs_grad, dict(stride=10), -1), (_logprobs_grad, dict(grad=C.c_void_p(4097)), -1), (_logprobs_grad, dict(V=0), -2),
    (_logprobs_grad, dict(n=1 << 24), -2), (_logprobs_grad, dict(V=524289, stride=600000, gstride=600000), -2), (_logprobs_grad, dict(n=0), 0),
    (_distill, dict(n=-1), -1), (_distill, dict(t=2), -1), (_distill, dict(logits=None), -1), (_distill, dict(k=0), -1), (_distill, dict(m=2), -1),
    (_distill, dict(m=-1, rows=one), -1), (_distill, dict(val=None), -1), (_distill, dict(ids=None), -1), (_distill, dict(flags=3), -1),
    (_distill, dict(flags=4), -1), (_distill, dict(T=0.0), -1), (_distill, dict(loss=None), -1), (_distill, dict(stats=None), -1),
    (_distill, dict(tail=None), -1), (_distill, dict(grad=one, gstride=2000), -1), (_distill, dict(gstride=500), -1), (_distill, dict(stride=500), -1),
    (_distill, dict(k=129), -2), (_distill, dict(V=0), -2), (_distill, dict(n=1 << 24, m=1 << 24), -2), (_distill, dict(ws=None), -3),
    (_distill, dict(wsb=64), -3), (_distill, dict(ws=C.c_void_p(4100)), -3), (_distill, dict(n=0), 0),
    (_distill_grad, dict(grad=None), -1), (_distill_grad, dict(stats=None), -1), (_distill_grad, dict(tail=None), -1),
    (_distill_grad, dict(m=1), -1), (_distill_grad, dict(flags=3), -1), (_distill_grad, dict(k=129), -2), (_distill_grad, dict(n=0), 0),
])
def test_bad_calls_are_refused(call, kw, status):
    assert call(**kw) == status


def test_workspace():
    assert 0 < dt.dt_logprob_workspace_bytes(1, 1000) <= dt.dt_logprob_workspace_bytes(9, 128256) < 1 << 20
    assert dt.dt_logprob_workspace_bytes(0, 1000) > 0
    for bad in ((-1, 1000), (1, 0), (1, 524289), (1 << 24, 1000)):
        with pytest.raises(dt.DtError):
            dt.dt_logprob_workspace_bytes(*bad)


# ---- the binding: what it refuses before a pointer is taken.  The tensors say that they are on device 0, and are not.

class OnGpu:
    def __init__(self, t, index=0):
        self._t = t
        self.device = torch.device("cuda", index)

    def __getattr__(self, name):
        return getattr(self._t, name)


@pytest.fixture
def call():
    binding._native()
    _dtcall.setup(torch.float32, torch.bfloat16, lambda: 0, lambda device: 0)
    yield
    _dtcall.setup(torch.float32, torch.bfloat16, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)


i32 = dict(dtype=torch.int32)


def _args(**kw):
    a = dict(logits=torch.zeros(2, 8, 100), row_of=torch.zeros(2, 3, **i32), tokens=torch.zeros(2, 3, **i32), T=1.0, k=4,
             logprob=torch.zeros(2, 3), entropy=torch.zeros(2, 3), stats=torch.zeros(2, 3, 2), top=torch.zeros(2, 3, 4),
             ids=torch.zeros(2, 3, 4, **i32), ws=torch.zeros(8, dtype=torch.uint8))
    a.update(kw)
    return [OnGpu(v) if isinstance(v, torch.Tensor) else v for v in a.values()]


@pytest.mark.parametrize("kw, error", [
    (dict(logits=torch.zeros(2, 100)), ValueError), (dict(logits=torch.zeros(2, 8, 100, dtype=torch.float16)), TypeError),
    (dict(logits=torch.zeros(2, 100, 8).transpose(1, 2)), ValueError), (dict(logits=torch.zeros(2, 16, 100)[:, :8]), ValueError),
    (dict(row_of=torch.zeros(2, 3, dtype=torch.int64)), TypeError), (dict(row_of=torch.zeros(2, 4, **i32)), ValueError),
    (dict(tokens=torch.zeros(3, 2, **i32).t()), ValueError), (dict(tokens=torch.zeros(2, 3)), TypeError),
    (dict(stats=torch.zeros(2, 3)), ValueError), (dict(stats=torch.zeros(3, 3, 2)), ValueError), (dict(stats=torch.zeros(2, 3, 3)), ValueError),
    (dict(logprob=torch.zeros(2, 3, dtype=torch.float64)), TypeError), (dict(entropy=torch.zeros(2, 2)), ValueError),
    (dict(top=torch.zeros(2, 3, 3)), ValueError), (dict(ids=torch.zeros(2, 3, 4)), TypeError), (dict(ws=torch.zeros(64)), TypeError),
    (dict(T="1"), TypeError), (dict(k=1 << 40), OverflowError),
])
def test_the_binding_refuses_tensors_that_are_not_as_said(call, kw, error):
    with pytest.raises(error):
        dt.dt_token_logprobs(*_args(**kw))


def test_the_binding_refuses_vocabularies_beyond_an_int(call):
    """Rows of 2^32 + 50 entries are not rows of 50.  (Nothing is read of them.)"""
    g = lambda *s, **kw: OnGpu(torch.zeros(*s, **kw))
    long = OnGpu(torch.empty(1).as_strided((1, (1 << 32) + 50), (0, 0)))
    long.stride = lambda dim=None: ((1 << 32) + 50, 1) if dim is None else ((1 << 32) + 50, 1)[dim]
    with pytest.raises(OverflowError):
        dt.dt_token_logprobs_grad(long, g(1, **i32), 1.0, g(1, 2), g(1), g(1), g(1), long)
    with pytest.raises(OverflowError):
        dt.dt_distill_rows(long, g(1, 5), g(1, 5, **i32), None, None, 1.0, 1, None, g(1), g(1, 2), g(1), None, None)


def test_the_binding_refuses_tensors_of_another_device(call):
    with pytest.raises(dt.DtError) as e:                       # as said: refused for the workspace alone
        dt.dt_token_logprobs(*_args(ws=None))
    assert e.value.status == -3
    for at, a in enumerate(_args()):
        if isinstance(a, OnGpu):
            for other in (a._t, OnGpu(a._t, 1)):                # the host's, as a plain tensor; another GPU's
                args = _args()
                args[at] = other
                with pytest.raises(ValueError, match="current device"):
                    dt.dt_token_logprobs(*args)
    g = lambda *s, **kw: OnGpu(torch.zeros(*s, **kw))
    grad = [g(4, 50), g(4, **i32), 1.0, g(4, 2), g(4), g(4), g(4), g(4, 50)]
    for at, bad in ((0, torch.zeros(4, 50)), (7, torch.zeros(4, 50)), (7, g(4, 51)), (7, g(3, 50)), (3, g(4, 3))):
        args = list(grad)
        args[at] = bad
        with pytest.raises(ValueError):
            dt.dt_token_logprobs_grad(*args)
    args = list(grad)
    args[7] = g(4, 50, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        dt.dt_token_logprobs_grad(*args)
    loss = [g(4, 50), g(6, 5), g(6, 5, **i32), g(6), g(4, **i32), 1.0, 1, g(4), g(4), g(4, 2), g(4), g(4, 50), None]
    with pytest.raises(dt.DtError) as e:
        dt.dt_distill_rows(*loss)
    assert e.value.status == -3
    for at, bad in ((0, torch.zeros(4, 50)), (1, g(6, 4)), (2, g(5, 5, **i32)), (3, g(4)), (4, g(6, **i32)), (7, g(5)), (8, g(1)), (9, g(4)), (10, g(3)),
                    (11, g(4, 49)), (12, torch.zeros(64, dtype=torch.uint8))):
        args = list(loss)
        args[at] = bad
        with pytest.raises(ValueError):
            dt.dt_distill_rows(*args)
        if at not in (8, 12):
            with pytest.raises(ValueError):
                dt.dt_distill_rows_grad(*(args[:8] + args[9:12]))
    with pytest.raises(dt.DtError):
        dt.dt_distill_rows_grad(*(loss[:8] + loss[9:11] + [None]))


# ---- the plain gradients against differences of the plain losses, in 64 bits

def test_plain_gradients_are_those_of_the_plain_losses():
    g = torch.Generator().manual_seed(1)
    n, V, T, k = 4, 23, 1.5, 6                          # (a power of two and a half: exact in fp32)
    x = (torch.randn(n, V, generator=g) * 2).double()
    tokens = torch.randint(0, V, (n,), generator=g)
    a, b = torch.randn(n, generator=g), torch.randn(n, generator=g)
    val, ids = torch.topk(torch.randn(n, V, generator=g), k, dim=1)
    ids[0, 3] = ids[0, 1]                                # a token twice
    ids[1, 2] = -1
    lse = torch.full((n,), 3.0)
    h = 1e-5

    def differences(f):
        out = torch.zeros(n, V, dtype=torch.float64)
        for j in range(V):
            d = torch.zeros(n, V, dtype=torch.float64)
            d[:, j] = h
            out[:, j] = (f(x + d) - f(x - d)) / (2 * h)
        return out

    def objective(y):
        r = ref.logprobs(y, tokens, T, 1)
        return a * r["logprob"] + b * r["entropy"]
    got, _ = ref.logprobs_grad(x, tokens, T, a, b)
    assert (got - differences(objective)).abs().max() < 1e-8
    for flags in (0, 1, 2):
        r = ref.distill(x, val, ids, lse, None, T, flags, a)
        want = differences(lambda y: a.double() * ref.distill(y, val, ids, lse, None, T, flags)["loss"])
        assert (r["grad"] - want).abs().max() < 1e-8, flags
