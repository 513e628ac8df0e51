"""What the operators on logits refuse, through the C ABI: no launch is reached, so no GPU is needed.  Where there is one the
calls are not made: one that should be refused and is not would follow the made-up addresses."""
import ctypes as C
import os

import pytest

from paper_1502_00512_amd import binding

pytestmark = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="made-up addresses")

BIG = 1 << 44  # made-up device addresses, never followed
LOGITS, OUT, IDS, VALS, MORE, WS = (BIG + (i << 40) for i in range(6))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_1502_00512_amd.build import build
        build()
    return binding.load()


TOP = dict(logits=LOGITS, dtype=0, rows=4, V=100, ld=100, K=5, tau=1.0, ids=IDS, vals=VALS, lse=MORE, ws=WS, bytes=1 << 30, stream=None)
DISTILL = dict(logits=LOGITS, dtype=1, rows=4, V=100, ld=104, ids=IDS, vals=VALS, K=5, lse=None, y=MORE, weight=None, tau=1.0, alpha=0.5,
               scale=1.0, loss=WS, sum=None, dlogits=OUT, ldd=100, flag=None, stream=None)
VERIFY = dict(target=LOGITS, ld=100, draft=OUT, ldd=100, dtype=0, K=3, B=2, V=100, drafts=IDS, lengths=None, u=VALS, tau=1.0, tau_d=1.0,
              accepted=MORE, tokens=MORE + 4096, flag=None, ws=WS, bytes=1 << 30, stream=None)
WIDE = dict(V=1 << 20, ld=1 << 20)  # a row in chunks: the workspace is wanted
F = lambda v: C.c_float(v) if isinstance(v, float) else v  # noqa: E731


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(logits=LOGITS + 2), dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 40), dict(V=0), dict(V=(1 << 20) + 1, ld=1 << 21),
    dict(ld=99), dict(ld=1 << 62), dict(K=0), dict(K=101), dict(V=1000, ld=1000, K=257), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")),
    dict(tau=float("inf")), dict(tau=1e-4), dict(ids=None), dict(vals=None), dict(ids=IDS + 1), dict(lse=MORE + 2),
    dict(rows=(1 << 22) - 63), dict(rows=1 << 20, **WIDE), dict(ws=None, **WIDE), dict(ws=WS + 16, **WIDE), dict(bytes=100, **WIDE)], ids=str)
def test_top_logits(lib, change):
    assert lib.rnnlm_top_logits(*map(F, {**TOP, **change}.values())) == -1


def test_top_logits_without_rows_is_fine(lib):
    assert lib.rnnlm_top_logits(*map(F, {**TOP, "rows": 0}.values())) == 0


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(logits=LOGITS + 1), dict(dtype=3), dict(rows=-2), dict(rows=(1 << 22) - 63), dict(V=0), dict(V=1 << 21, ld=1 << 21, ldd=1 << 21), dict(ld=99), dict(ldd=99),
    dict(ids=None), dict(vals=None), dict(K=0), dict(K=1025), dict(y=None), dict(tau=0.0), dict(alpha=-0.1), dict(alpha=1.5),
    dict(alpha=float("nan")), dict(scale=float("inf")), dict(loss=None), dict(loss=WS + 1), dict(sum=OUT + 4), dict(y=MORE + 2), dict(flag=2),
    dict(weight=VALS + 2), dict(dlogits=LOGITS), dict(dlogits=LOGITS + 2), dict(dlogits=LOGITS - 400), dict(dlogits=OUT + 1)], ids=str)
def test_distill_loss(lib, change):
    assert lib.rnnlm_distill_loss(*map(F, {**DISTILL, **change}.values())) == -1


@pytest.mark.parametrize("change", [
    dict(target=None), dict(target=LOGITS + 2), dict(draft=OUT + 2), dict(ld=99), dict(ldd=99), dict(dtype=5), dict(K=-1), dict(K=1025), dict(B=0),
    dict(B=(1 << 20) + 1), dict(B=1 << 20), dict(V=0), dict(V=1 << 21, ld=1 << 21, ldd=1 << 21), dict(drafts=None), dict(u=None), dict(u=VALS + 2), dict(tau=0.0),
    dict(tau_d=float("nan")), dict(accepted=None), dict(tokens=None), dict(tokens=MORE + 2), dict(lengths=IDS + 2), dict(ws=None),
    dict(ws=WS + 128), dict(bytes=64), dict(flag=1)], ids=str)
def test_verify_drafts(lib, change):
    assert lib.rnnlm_verify_drafts(*map(F, {**VERIFY, **change}.values())) == -1


def test_workspace_sizes(lib):
    top, verify = binding.rnnlm_top_logits_workspace_bytes, binding.rnnlm_verify_workspace_bytes
    assert top(2560, 64000, 64, 1) > 0 and top(0, 10, 1, 0) > 0
    assert top((1 << 22) - 64, 10, 1, 0) > 0 == top((1 << 22) - 63, 10, 1, 0) == top(1 << 20, 1 << 20, 1, 0)
    assert verify(1, 1 << 20, 10) > 0 == verify(2, 1 << 20, 10)
    assert [top(-1, 10, 1, 0), top(1, 10, 11, 0), top(1, 1000, 257, 0), top(1, 10, 1, 2), top(1, 1 << 21, 1, 0)] == [0] * 5
    assert 0 < verify(0, 1, 10) <= verify(4, 1, 10) < verify(4, 64, 100000) < 1 << 26
    assert [verify(-1, 1, 10), verify(1, 0, 10), verify(1, 1, 0), verify(1025, 1, 10), verify(1024, 1 << 20, 10)] == [0] * 5


def test_binding_refuses_what_it_cannot_pass_on():
    import torch
    z = torch.zeros(2, 10)
    for call in (lambda: binding.rnnlm_top_logits(z, 3), lambda: binding.rnnlm_distill_loss(z, z[:, :2].int(), z[:, :2]),
                 lambda: binding.rnnlm_verify_drafts(z[None], None, z[:1, 0])):
        with pytest.raises(binding.RnnlmError, match="on a GPU"):
            call()
