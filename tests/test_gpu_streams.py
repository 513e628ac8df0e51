"""Calls that are given a stream which is not the current one: everything they allocate themselves is this stream's.
(Memory of the current stream's pool could still be in use there when the call's kernels start, and scratch that is dropped with
the call would be given away there while they run.)"""
import numpy as np
import pytest
import torch

from paper_1502_00512_amd import binding, synth

pytestmark = pytest.mark.gpu

FP32, BF16 = binding.RNNLM_FP32, binding.RNNLM_BF16_FP32MASTER


@pytest.fixture
def allocations(monkeypatch):
    """The streams that tensors were allocated under, one entry each."""
    seen = []
    for name in ("empty", "zeros"):
        def make(*a, _real=getattr(torch, name), **k):
            seen.append(torch.cuda.current_stream())
            return _real(*a, **k)
        monkeypatch.setattr(torch, name, make)
    return seen


def given_a_stream(call, allocations):
    """call(stream) without one, and on a busy stream of its own with the current one at work: the same results."""
    want = call(None)
    torch.cuda.synchronize()
    side, a = torch.cuda.Stream(), torch.ones(2048, 2048, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(10):
                a = a @ a * 0.0
        del allocations[:]
        got = call(side)
        assert allocations and all(s == side for s in allocations), allocations
        junk = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (1 << 12, 1 << 16, 1 << 20, 1 << 22, 1 << 24)]
        torch.cuda.synchronize()
        assert len(got) == len(want) and all(torch.equal(x, y) for x, y in zip(got, want))
        del junk


def test_operators_on_rows(allocations):
    M, V, K, B, D = 60, 170007, 40, 5, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(M, V, device="cuda", generator=gen).bfloat16()
    u, drafts = torch.rand(D + 1, B, device="cuda", generator=gen), torch.randint(0, V, (D, B), device="cuda", generator=gen, dtype=torch.int32)
    given_a_stream(lambda s: binding.rnnlm_top_logits(z, K, stream=s), allocations)  # (in chunks: with a workspace)
    ids, vals, lse = binding.rnnlm_top_logits(z, K)
    given_a_stream(lambda s: [binding.rnnlm_distill_loss(z, ids, vals, lse, stream=s)], allocations)
    given_a_stream(lambda s: binding.rnnlm_verify_drafts(z[: (D + 1) * B].view(D + 1, B, V), drafts, u, z[-D * B:].view(D, B, V), stream=s),
                   allocations)


@pytest.mark.parametrize("precision", [FP32, BF16])
@pytest.mark.parametrize("P", [0, 32])
def test_windows_with_rows_of_logits(P, precision, allocations):
    V, H, B, T, K = 5003, 64, 6, 4, 7
    if P:
        E, A, U, C_, b = synth.make_compressed_weights(V, H, P, "uniform", 0.3, 1)
        g = binding.Rnnlm(E, U, None, b, B, T, precision, A=A, C_=C_)
    else:
        E, U, Wo, b = synth.make_weights(V, H, "uniform", 0.3, 1)
        g = binding.Rnnlm(E, U, Wo, b, B, T, precision)
    rng = np.random.default_rng(2)
    cuda = lambda a, t: torch.as_tensor(a.astype(t)).cuda()  # noqa: E731
    x, y = (cuda(rng.integers(0, V, (T, B)), np.int32) for _ in range(2))
    ids, vals, u = cuda(rng.integers(0, V, (T, B, K)), np.int32), cuda(rng.normal(size=(T, B, K)), np.float32), cuda(rng.random((T, B)), np.float32)
    weights = [w for w in (g.E, g.U, g.Wo, g.A, g.C, g.b) if w is not None]
    first = [w.clone() for w in weights]

    def fresh(call):
        def run(s):
            for w, f in zip(weights, first):
                w.copy_(f)
            g.rnnlm_reset_state()
            g.rnnlm_sync_compute_copies()
            if s is not None:
                s.wait_stream(torch.cuda.current_stream())
            return list(call(s))
        return run

    def train(s):
        g.rnnlm_distill_train_chunk(x, y, ids, vals, 0.5, alpha=0.5, stream=s)
        torch.cuda.synchronize()
        return [w.clone() for w in weights]

    given_a_stream(fresh(lambda s: [g.rnnlm_forward_logits(x, stream=s)]), allocations)
    given_a_stream(fresh(lambda s: g.rnnlm_verify_chunk(x, u, stream=s)), allocations)
    given_a_stream(fresh(lambda s: g.rnnlm_distill_grad_chunk(x, y, ids, vals, alpha=0.5, stream=s).values()), allocations)
    given_a_stream(fresh(train), allocations)
    g.rnnlm_check()


@pytest.mark.parametrize("precision", [FP32, BF16])
def test_windows_whose_outputs_the_binding_allocates(precision, allocations):
    V, H, B, T, K, P = 5003, 64, 6, 4, 32, 32
    E, U, Wo, b = synth.make_weights(V, H, "uniform", 0.3, 1)
    g = binding.Rnnlm(E, U, Wo, b, B, T, precision, K_max=K)
    E, A, U, C_, b = synth.make_compressed_weights(V, H, P, "uniform", 0.3, 1)
    c = binding.Rnnlm(E, U, None, b, B, T, precision, A=A, C_=C_)
    rng = np.random.default_rng(2)
    cuda = lambda a, t: torch.as_tensor(a.astype(t)).cuda()  # noqa: E731
    x, y = (cuda(rng.integers(0, V, (T, B)), np.int32) for _ in range(2))
    noise, lnq = cuda(rng.integers(0, V, K), np.int32), torch.full((V,), -float(np.log(V)), device="cuda")
    cand, tok = cuda(rng.integers(0, V, (T, B, 5)), np.int32), cuda(rng.integers(0, V, 2 * T * B + B), np.int32)

    def from_the_start(call):
        def run(s):
            g.rnnlm_reset_state()
            c.rnnlm_reset_state()
            if s is not None:
                s.wait_stream(torch.cuda.current_stream())
            out = call(s)
            out = out.values() if isinstance(out, dict) else out if isinstance(out, tuple) else [out]
            return [t for o in out for t in (o if isinstance(o, tuple) else [o])]
        return run

    for call in (lambda s: g.rnnlm_stream_chunk(tok, 0, T, stream=s), lambda s: g.rnnlm_forward_logprob(x, y, stream=s),
                 lambda s: g.rnnlm_grad_chunk(x, y, stream=s), lambda s: c.rnnlm_grad_chunk_compressed(x, y, stream=s),
                 lambda s: g.rnnlm_forward_score(x, y, stream=s), lambda s: g.rnnlm_forward_score_shortlist(x, cand, stream=s),
                 lambda s: g.rnnlm_nce_grad_chunk(x, y, noise, lnq, 0.0, stream=s), lambda s: g.rnnlm_sort_segments(x, stream=s),
                 lambda s: c.rnnlm_quantize_weights(stream=s)):
        given_a_stream(from_the_start(call), allocations)
    g.rnnlm_check()
    c.rnnlm_check()
