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


def test_preference_waits(lib):
    for polls in (-1, (1 << 20) + 1, (1 << 31) - 1):
        with pytest.raises(binding.RnnlmError):
            binding.rnnlm_set_preference_wait(polls)
    for polls in (1 << 20, 0, 256):  # (the default last)
        binding.rnnlm_set_preference_wait(polls)


FORWARD = dict(x=LOGITS, ldx=40, dtype=1, rows=4, K=40, N=100, a=None, ids=Y, base=A, ldb=100, out=OUT, ldo=100, inner=MORE, flag=None, ws=WS,
               bytes=1 << 20, stream=None)
BACKWARD = dict(dout=A, ldd=100, x=LOGITS, ldx=40, inner=MORE, dtype=0, rows=4, K=40, N=100, a=None, ids=Y, ddown=B, dup=B + (1 << 30), dx=OUT,
                ldx2=40, flag=None, ws=WS, bytes=1 << 20, stream=None)
ADAPTERS = dict(down=BIG + (1 << 36), up=BIG + (1 << 37), scale=None, n=3, R=8)


def with_adapters(good, change):
    """The call's arguments; keys of the description are set in it."""
    a = binding.rnnlm_adapters(*{**ADAPTERS, **{k: v for k, v in change.items() if k in ADAPTERS}}.values())
    return {**good, "a": C.byref(a), **{k: v for k, v in change.items() if k not in ADAPTERS}}


COMMON = [dict(a=None), dict(down=None), dict(up=None), dict(down=ADAPTERS["down"] + 1), dict(up=ADAPTERS["up"] + 1), dict(scale=2), dict(n=0), dict(n=65537), dict(R=0),
          dict(R=65), dict(x=None), dict(x=LOGITS + 1), dict(ldx=39), dict(dtype=2), dict(rows=-1), dict(rows=(1 << 17) + 1), dict(K=0), dict(K=65537, ldx=1 << 17), dict(N=0),
          dict(ids=None), dict(ids=Y + 2), dict(inner=MORE + 2), dict(flag=MORE + 1), dict(ws=None), dict(ws=WS + 64), dict(bytes=100)]


@pytest.mark.parametrize("change", COMMON + [
    dict(N=(1 << 20) + 1, ldb=1 << 21, ldo=1 << 21), dict(out=None), dict(out=OUT + 1), dict(ldo=99), dict(base=A + 1), dict(ldb=99), dict(base=OUT, ldb=101, ldo=100),
    dict(base=OUT + 2), dict(out=LOGITS), dict(out=LOGITS + 8)], ids=str)
def test_adapter_forward_refuses(lib, change):
    assert lib.rnnlm_adapter_forward(*with_adapters(FORWARD, change).values()) == -1


@pytest.mark.parametrize("change", COMMON + [
    dict(N=(1 << 20) + 1, ldd=1 << 21), dict(dout=None), dict(dout=A + 2), dict(ldd=99), dict(inner=None), dict(ddown=None), dict(ddown=B + 2), dict(dup=None), dict(dup=B + 1),
    dict(dx=OUT + 2), dict(ldx2=39), dict(dx=LOGITS), dict(dx=A + 400)], ids=str)
def test_adapter_backward_refuses(lib, change):
    assert lib.rnnlm_adapter_backward(*with_adapters(BACKWARD, change).values()) == -1


def test_adapter_workspaces(lib):
    ws = binding.rnnlm_adapter_workspace_bytes
    assert ws(0, 1, 1, 1, 1, 0) > 0 and ws(1 << 17, 1, 1, 1, 64, 1) > 1 << 25
    for good in ((2560, 1024, 64000, 16, 32, 1), (8192, 4096, 131072, 256, 64, 1), (1, 64, 131072, 1, 64, 0)):
        assert 0 < ws(*good, False) < ws(*good, True) <= 1 << 30
    assert [ws(-1, 1, 1, 1, 1, 0), ws((1 << 17) + 1, 1, 1, 1, 1, 0), ws(1, 0, 1, 1, 1, 0), ws(1, 65537, 1, 1, 1, 0), ws(1, 1, 0, 1, 1, 0), ws(1, 1, (1 << 20) + 1, 1, 1, 0),
            ws(1, 1, 1, 0, 1, 0), ws(1, 1, 1, 65537, 1, 0), ws(1, 1, 1, 1, 0, 0), ws(1, 1, 1, 1, 65, 0), ws(1, 1, 1, 1, 1, 2)] == [0] * 11
    assert lib.rnnlm_adapter_workspace_bytes(1, 1, 1, 1, 1, 0, 2) == 0


def test_no_rows_of_a_forward_pass_are_fine(lib):
    assert lib.rnnlm_adapter_forward(*with_adapters(FORWARD, dict(rows=0)).values()) == 0


def test_binding_refuses_what_it_cannot_pass_on():
    import torch
    z = torch.zeros(2, 4, 10)
    i = torch.zeros(2, 4, dtype=torch.int32)
    for call in (lambda: binding.rnnlm_policy_loss(z, i, z[..., 0]), lambda: binding.rnnlm_preference_loss(z, i),
                 lambda: binding.rnnlm_adapter_forward(z, z, z, i), lambda: binding.rnnlm_adapter_backward(z, z, z, z, z, i)):
        with pytest.raises(binding.RnnlmError, match="on a GPU"):
            call()
