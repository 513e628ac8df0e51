"""What the operators that adapt a model refuse, through the C ABI: no launch is reached, so no GPU is needed.  Where there is one
the calls are not made: one that should be refused and is not would follow the made-up addresses."""
import ctypes as C
import os

import pytest

from paper_1502_00512_amd import binding

pytestmark = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="made-up addresses")

BIG = 1 << 44  # made-up device addresses, never followed
LOGITS, OUT, Y, A, B, MORE, WS = (BIG + (i << 40) for i in range(7))
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_1502_00512_amd.build import build
        build()
    return binding.load()


F = lambda v: C.c_float(v) if isinstance(v, float) else v  # noqa: E731


def refused(f, good, change):
    assert set(change) <= set(good)
    return f(*map(F, {**good, **change}.values())) == -1


POLICY = dict(logits=LOGITS, dtype=1, rows=4, V=100, ld=104, y=Y, old=A, ref=B, advantage=MORE, weight=None, tau=1.0, lo=0.2, hi=0.2, beta=0.1,
              scale=1.0, loss=WS, logp=None, sum=None, dlogits=OUT, ldd=100, flag=None, stream=None)


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(logits=LOGITS + 1), dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 40), dict(V=0),
    dict(V=(1 << 20) + 1, ld=1 << 21, ldd=1 << 21), dict(ld=99), dict(ld=1 << 62), dict(y=None), dict(y=Y + 2), dict(old=A + 1), dict(ref=None),
    dict(ref=B + 2), dict(advantage=None), dict(advantage=MORE + 1), dict(weight=A + 2), dict(tau=0.0), dict(tau=NAN), dict(tau=2e3), dict(lo=-0.1), dict(lo=1.5),
    dict(lo=NAN), dict(hi=-0.1), dict(hi=INF), dict(hi=NAN), dict(beta=-1.0), dict(beta=INF), dict(beta=NAN), dict(scale=NAN), dict(scale=INF), dict(loss=None),
    dict(loss=WS + 1), dict(logp=WS + 2), dict(sum=WS + 4), dict(dlogits=OUT + 1), dict(ldd=99), dict(dlogits=LOGITS), dict(dlogits=LOGITS + 208),
    dict(flag=WS + 2)], ids=str)
def test_policy_refuses(lib, change):
    assert refused(lib.rnnlm_policy_loss, POLICY, change)


PREFER = dict(logits=LOGITS, dtype=0, T=3, pairs=2, V=100, ld=100, y=Y, ref=A, weight=B, kind=0, beta=0.1, smoothing=0.1, mean=0, scale=1.0,
              loss=MORE, logp=None, sum=None, dlogits=OUT, ldd=100, flag=None, ws=WS, bytes=1 << 20, stream=None)


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(logits=LOGITS + 2), dict(dtype=2), dict(T=-1), dict(T=1 << 22), dict(pairs=0), dict(pairs=-1), dict(pairs=1 << 21), dict(V=0),
    dict(V=(1 << 20) + 1, ld=1 << 21, ldd=1 << 21), dict(ld=99), dict(y=None), dict(y=Y + 1), dict(ref=A + 2), dict(weight=B + 2), dict(kind=-1), dict(kind=3),
    dict(kind=1), dict(kind=2), dict(beta=0.0), dict(beta=-1.0), dict(beta=NAN), dict(beta=INF), dict(smoothing=-0.1), dict(smoothing=0.6), dict(smoothing=NAN),
    dict(mean=2), dict(mean=-1), dict(scale=NAN), dict(loss=None), dict(loss=MORE + 2), dict(logp=MORE + 2), dict(sum=MORE + 4), dict(dlogits=OUT + 2), dict(ldd=99),
    dict(dlogits=LOGITS, ldd=101), dict(dlogits=LOGITS + 400), dict(flag=MORE + 1), dict(ws=None), dict(ws=WS + 16), dict(bytes=255), dict(T=0, loss=None)], ids=str)
def test_preference_refuses(lib, change):
    assert refused(lib.rnnlm_preference_loss, PREFER, change)


def test_preference_workspaces(lib):
    ws = binding.rnnlm_preference_workspace_bytes
    assert ws(0, 1) > 0 and ws(20, 64) > ws(10, 64) > ws(0, 64) > 0 and ws(20, 64) % 256 == 0
    assert ws(-1, 1) == ws(1, 0) == ws(1, -1) == ws(1 << 22, 1) == ws(1, 1 << 21) == 0
