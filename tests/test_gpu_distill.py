"""Windows of a handle whose logits are the caller's: rnnlm_forward_logits, the distilled training window and a step of
drafting and verifying, against the fp64 oracles and autograd in 64 bits.  Tolerances as for the other windows: fp32
log-probabilities 1e-4 relative + 1e-6, gradients 1e-3 of each tensor's scale (max and l2); bf16 gradients 2e-2 (compressed
architecture 3e-2)."""
import numpy as np
import pytest
import torch

from oracle import logits as L
from paper_1502_00512_amd import binding, synth

pytestmark = pytest.mark.gpu

FP32, BF16 = binding.RNNLM_FP32, binding.RNNLM_BF16_FP32MASTER


def cuda(a, dtype=None):
    return None if a is None else torch.as_tensor(np.ascontiguousarray(a, dtype)).cuda()


def handle(V, H, P, B, T, precision, seed, scale=0.3):
    """(handle, the same weights in 64 bits by name)"""
    if P:
        E, A, U, C_, b = synth.make_compressed_weights(V, H, P, "uniform", scale, seed)
        b = synth.uniform_weights((V,), -0.5, 0.5, seed + 99)
        g = binding.Rnnlm(E, U, None, b, B, T, precision, A=A, C_=C_)
        w = dict(E=E, A=A, U=U, C=C_, b=b)
    else:
        E, U, Wo, b = synth.make_weights(V, H, "uniform", scale, seed)
        b = synth.uniform_weights((V,), -0.5, 0.5, seed + 99)
        g = binding.Rnnlm(E, U, Wo, b, B, T, precision)
        w = dict(E=E, U=U, Wo=Wo, b=b)
    return g, {k: torch.as_tensor(np.asarray(v, np.float64)).requires_grad_() for k, v in w.items()}


def logits64(w, x, h):
    """Logits [T][B][V] and the state behind the window, in 64 bits."""
    out = []
    for row in torch.as_tensor(x).long():
        a = w["E"][row] @ w["A"].T if "A" in w else w["E"][row]
        h = torch.sigmoid(a + h @ w["U"].T)
        out.append((h @ w["C"].T) @ w["E"].T + w["b"] if "A" in w else h @ w["Wo"].T + w["b"])
    return torch.stack(out), h


def teacher(T, B, V, K, tau, seed):
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.permutation(V)[:K] for _ in range(T * B)]).reshape(T, B, K).astype(np.int32)
    vals = (rng.normal(size=(T, B, K)) * 2).astype(np.float32)
    lse = (np.log(np.exp(vals / tau).sum(2)) + 0.3).astype(np.float32)
    weight = rng.choice([0.0, 1.0, 2.0], (T, B)).astype(np.float32)
    y = rng.integers(0, V, (T, B)).astype(np.int32)
    y[rng.random((T, B)) < 0.2] = -1
    ids[rng.random((T, B, K)) < 0.1] = -1
    return ids, vals, lse, weight, y


def loss64(z, ids, vals, lse, weight, y, tau, alpha):
    """Losses [T][B] of rnnlm_distill_loss in 64 bits, for autograd."""
    there = torch.as_tensor(ids >= 0)
    t = torch.where(there, torch.as_tensor(vals.astype(np.float64)) / tau, -torch.inf)
    n = torch.logsumexp(t, 2, keepdim=True) if lse is None else torch.as_tensor(lse.astype(np.float64))[..., None]
    p = torch.where(there, torch.exp(t - n), 0.0)
    ln_q = torch.log_softmax(z / tau, 2).gather(2, torch.as_tensor(ids).long().clamp(min=0))
    kd = torch.where(there, p * (torch.where(there, t - n, 0.0) - ln_q), 0.0).sum(2)
    yl = torch.as_tensor(y).long()
    hard = torch.where(yl >= 0, -torch.log_softmax(z, 2).gather(2, yl.clamp(min=0)[..., None])[..., 0], 0.0)
    return torch.as_tensor(weight.astype(np.float64)) * (alpha * tau * tau * kd + (1 - alpha) * hard)


def close(name, got, ref, rel):
    got = got.detach().double().cpu().numpy()
    ref = ref.detach().numpy()
    assert np.isfinite(got).all(), name
    assert np.abs(got - ref).max() <= rel * np.abs(ref).max(), (name, np.abs(got - ref).max(), np.abs(ref).max())
    assert np.linalg.norm(got - ref) <= rel * np.linalg.norm(ref), name


SHAPES = [(1000, 64, 0, 4, 8), (777, 50, 0, 5, 7), (3001, 200, 0, 33, 3), (520, 96, 0, 70, 2), (300, 130, 0, 3, 1), (700, 64, 32, 4, 6),
          (1001, 96, 50, 5, 7), (2500, 256, 128, 32, 10)]


@pytest.mark.parametrize("V,H,P,B,T", SHAPES)
def test_forward_logits_fp32(V, H, P, B, T):
    g, w = handle(V, H, P, B, T, FP32, V)
    h = torch.zeros(B, H, dtype=torch.float64)
    for k in range(2):
        x = synth.zipf_tokens(T * B, V, 1.0, V + k).reshape(T, B).astype(np.int32)
        rows = torch.full((T, B, V + 5), 9.0, device="cuda")
        got = g.rnnlm_forward_logits(cuda(x), rows[:, :, :V])
        assert bool((rows[:, :, V:] == 9.0).all())
        with torch.no_grad():
            z, h = logits64(w, x, h)
        ref = torch.log_softmax(z, 2).numpy()
        lp = torch.log_softmax(got.double(), 2).cpu().numpy()
        assert (np.abs(lp - ref) <= 1e-4 * np.abs(ref) + 1e-6).all(), np.abs(lp - ref).max()
        assert np.abs(g.h_state.cpu().numpy() - h.numpy()).max() < 1e-5
    g.rnnlm_check()


def test_forward_logits_bf16_are_what_the_log_probabilities_come_from():
    V, H, B, T = 3001, 256, 8, 5
    g, _ = handle(V, H, 0, B, T, BF16, 1)
    g2, _ = handle(V, H, 0, B, T, BF16, 1)
    x = synth.zipf_tokens(T * B, V, 1.0, 3).reshape(T, B).astype(np.int32)
    y = synth.zipf_tokens(T * B, V, 1.0, 4).reshape(T, B).astype(np.int32)
    z = g.rnnlm_forward_logits(cuda(x))
    logp = g2.rnnlm_forward_logprob(cuda(x), cuda(y))
    assert z.dtype == torch.bfloat16 and torch.equal(g.h_state, g2.h_state)
    want = torch.log_softmax(z.double(), 2).gather(2, cuda(y).long()[..., None])[..., 0]
    # a logit is off by half a bf16 step; their sum's logarithm by as much at most
    assert float((logp.double() - want).abs().max()) <= 2 * 2.0 ** -8 * float(z.float().abs().max())


@pytest.mark.parametrize("precision", [FP32, BF16])
@pytest.mark.parametrize("V,H,P,B,T", SHAPES)
def test_distill_gradients(V, H, P, B, T, precision):
    K, tau, alpha = 9, 2.0, 0.6
    g, w = handle(V, H, P, B, T, precision, V)
    x = synth.zipf_tokens(T * B, V, 1.0, V + 7).reshape(T, B).astype(np.int32)
    ids, vals, lse, weight, y = teacher(T, B, V, K, tau, V)
    for n in (None, lse):
        for v in w.values():
            v.grad = None
        z, _ = logits64(w, x, torch.zeros(B, H, dtype=torch.float64))
        losses = loss64(z, ids, vals, n, weight, y, tau, alpha)
        losses.mean().backward()
        kept = g.h_state.clone(), g.E.clone()
        got = g.rnnlm_distill_grad_chunk(cuda(x), cuda(y), cuda(ids), cuda(vals), cuda(n), cuda(weight), tau, alpha)
        g.rnnlm_check()
        assert torch.equal(kept[0], g.h_state) and torch.equal(kept[1], g.E)
        if precision == FP32:
            assert np.abs(got["loss"].cpu().numpy() - losses.detach().numpy()).max() <= 1e-4 * float(losses.detach().abs().max())
        for name, v in w.items():
            close(name, got["g" + name], v.grad, 1e-3 if precision == FP32 else 3e-2 if P else 2e-2)


@pytest.mark.parametrize("precision", [FP32, BF16])
def test_labels_alone_are_the_normalised_criterion(precision):
    V, H, B, T = 1500, 96, 6, 5
    g, _ = handle(V, H, 0, B, T, precision, 5)
    x, y = (synth.zipf_tokens(T * B, V, 1.0, s).reshape(T, B).astype(np.int32) for s in (1, 2))
    ids, vals = np.zeros((T, B, 1), np.int32), np.zeros((T, B, 1), np.float32)
    ref = g.rnnlm_grad_chunk(cuda(x), cuda(y))
    got = g.rnnlm_distill_grad_chunk(cuda(x), cuda(y), cuda(ids), cuda(vals), alpha=0.0)
    for name in ("gE", "gU", "gWo", "gb"):
        close(name, got[name], ref[name].double().cpu(), 1e-4 if precision == FP32 else 1e-2)
    assert float((got["loss"] + ref["logp"]).abs().max()) <= (1e-5 if precision == FP32 else 0.1)


@pytest.mark.parametrize("V,H,P,B,T", [(1000, 64, 0, 4, 8), (777, 50, 0, 5, 7), (700, 64, 32, 4, 6), (40000, 64, 0, 64, 20)])
def test_distill_training_windows_fp32(V, H, P, B, T):
    """Several windows of a student's training, against plain gradient descent in 64 bits on autograd's gradients."""
    K, tau, alpha, lr = 6, 1.5, 0.5, 0.3
    g, w = handle(V, H, P, B, T, FP32, V + 1)
    h = torch.zeros(B, H, dtype=torch.float64)
    total = torch.zeros(1, dtype=torch.float64, device="cuda")
    for k in range(3):
        x = synth.zipf_tokens(T * B, V, 1.0, V + k).reshape(T, B).astype(np.int32)
        ids, vals, lse, weight, y = teacher(T, B, V, K, tau, V + k)
        z, h2 = logits64(w, x, h)
        losses = loss64(z, ids, vals, lse, weight, y, tau, alpha)
        losses.mean().backward()
        h = h2.detach()
        with torch.no_grad():
            for v in w.values():
                v -= lr * v.grad
                v.grad = None
        loss = torch.empty(T, B, device="cuda")
        g.rnnlm_distill_train_chunk(cuda(x), cuda(y), cuda(ids), cuda(vals), lr, cuda(lse), cuda(weight), tau, alpha, loss=loss, sum_loss=total)
        assert np.abs(loss.cpu().numpy() - losses.detach().numpy()).max() <= 1e-4 * float(losses.detach().abs().max()) + 1e-6
        assert float(total) == pytest.approx(float(loss.double().sum()), rel=1e-12)
        assert np.abs(g.h_state.cpu().numpy() - h.numpy()).max() < 1e-5
    g.rnnlm_check()
    for name, v in w.items():
        assert np.abs(getattr(g, name).cpu().numpy() - v.detach().numpy()).max() <= 1e-4 * max(1.0, float(v.detach().abs().max())), name
    # the window that follows runs on the updated weights
    x = synth.zipf_tokens(T * B, V, 1.0, 99).reshape(T, B).astype(np.int32)
    with torch.no_grad():
        ref = torch.log_softmax(logits64(w, x, h)[0], 2).numpy()
    lp = torch.log_softmax(g.rnnlm_forward_logits(cuda(x)).double(), 2).cpu().numpy()
    assert (np.abs(lp - ref) <= 2e-4 * np.abs(ref) + 1e-5).all()


@pytest.mark.parametrize("precision", [FP32, BF16])
@pytest.mark.parametrize("V,H,P", [(777, 50, 0), (700, 64, 32)])
def test_windows_of_all_kinds_and_lengths_on_one_handle(V, H, P, precision):
    """What longer windows and other criteria leave in the workspace does not reach a shorter distilled one."""
    B, T_max, K = 5, 20, 7
    g, w = handle(V, H, P, B, T_max, precision, 5)
    fresh, _ = handle(V, H, P, B, T_max, precision, 5)

    def window(T, seed):
        x = synth.zipf_tokens(T * B, V, 1.0, seed).reshape(T, B).astype(np.int32)
        return x, teacher(T, B, V, K, 2.0, seed)

    for T, T2 in ((20, 2), (3, 7), (1, 20)):
        x, (ids, vals, lse, weight, y) = window(T, T)
        g.rnnlm_distill_train_chunk(cuda(x), cuda(y), cuda(ids), cuda(vals), 0.0, cuda(lse), cuda(weight), 2.0, 0.6)
        g.rnnlm_train_chunk(cuda(x), cuda(np.maximum(y, 0)), 0.0)
        g.rnnlm_verify_chunk(cuda(x), torch.full((T, B), 0.5, device="cuda"))
        g.rnnlm_check()
        g.rnnlm_reset_state()
        x, (ids, vals, lse, weight, y) = window(T2, 50 + T2)
        call = lambda h: h.rnnlm_distill_grad_chunk(cuda(x), cuda(y), cuda(ids), cuda(vals), cuda(lse), cuda(weight), 2.0, 0.6)  # noqa: E731
        got, ref = call(g), call(fresh)
        g.rnnlm_check()
        for v in w.values():
            v.grad = None
        loss64(logits64(w, x, torch.zeros(B, H, dtype=torch.float64))[0], ids, vals, lse, weight, y, 2.0, 0.6).mean().backward()
        for name, v in w.items():
            assert torch.equal(got["g" + name], ref["g" + name]), name
            close(name, got["g" + name], v.grad, 1e-3 if precision == FP32 else 3e-2 if P else 2e-2)
        z, z2 = g.rnnlm_forward_logits(cuda(x)), fresh.rnnlm_forward_logits(cuda(x))
        assert torch.equal(z, z2)
        g.rnnlm_reset_state()
        fresh.rnnlm_reset_state()


def test_what_a_distilled_window_reports():
    V, H, B, T = 300, 32, 3, 4
    g, _ = handle(V, H, 0, B, T, FP32, 1)
    x = cuda(np.zeros((T, B), np.int32))
    ids, vals, lse, weight, y = teacher(T, B, V, 4, 1.0, 1)
    run = lambda ids, vals, y: g.rnnlm_distill_train_chunk(x, cuda(y), cuda(ids), cuda(vals), 0.0, alpha=0.5)  # noqa: E731
    run(ids, vals, y)  # absent entries and labels are no errors
    g.rnnlm_check()
    for change in ("ids", "y"):
        i, l = ids.copy(), y.copy()
        (i if change == "ids" else l).flat[3] = V
        run(i, vals, l)
        with pytest.raises(binding.RnnlmError) as e:
            g.rnnlm_check()
        assert e.value.status == -2
    v = vals.copy()
    ids[1, 1, 0], v[1, 1, 0] = 5, np.nan
    run(ids, v, y)
    with pytest.raises(binding.RnnlmError) as e:
        g.rnnlm_check()
    assert e.value.status == -3
    bad = [dict(tau=0.0), dict(alpha=2.0), dict(K=0)]
    for b in bad:
        with pytest.raises(binding.RnnlmError):
            g.rnnlm_distill_train_chunk(x, cuda(y), cuda(ids[..., : b.get("K", 4)]), cuda(vals[..., : b.get("K", 4)]), 0.1, tau=b.get("tau", 1.0),
                                        alpha=b.get("alpha", 0.5))
    with pytest.raises(binding.RnnlmError):  # labels are wanted
        g.rnnlm_distill_train_chunk(x, None, cuda(ids), cuda(vals), 0.1, alpha=0.5)
    with pytest.raises(binding.RnnlmError):
        g.rnnlm_verify_chunk(cuda(np.zeros((T + 1, B), np.int32)), torch.zeros(T + 1, B, device="cuda"))  # longer than T_max


# ---- drafting and verifying ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("precision", [FP32, BF16])
@pytest.mark.parametrize("V,H,P,B", [(1000, 64, 0, 6), (777, 96, 50, 5), (500, 2100, 0, 3)])
def test_a_student_drafts_and_its_teacher_verifies(V, H, P, B, precision):
    """Rounds of K drafted words: accepted and drawn words against the oracle on the teacher's own logits, and the state each
    text is left in against a second handle that reads exactly the words the text keeps."""
    K = 3
    big, _ = handle(V, H, P, B, K + 1, precision, 1, 0.2)
    check, _ = handle(V, H, P, B, K + 1, precision, 1, 0.2)
    small, _ = handle(V, 32, 0, B, 1, precision, 2, 0.2)
    rng = np.random.default_rng(4)
    word = cuda(rng.integers(0, V, B), np.int32)
    for turn in range(4):
        state = small.h_state.clone()
        x = torch.empty(K + 1, B, dtype=torch.int32, device="cuda")
        x[0] = word
        draft = torch.empty(K, B, V, dtype=torch.float32 if precision == FP32 else torch.bfloat16, device="cuda")
        for i in range(K):  # the student's own words, one at a time
            small.rnnlm_forward_logits(x[i: i + 1], draft[i: i + 1])
            x[i + 1] = binding.rnnlm_verify_drafts(draft[i: i + 1], None, cuda(rng.random((1, B)), np.float32))[1][0]
        u = rng.random((K + 1, B)).astype(np.float32)
        lengths = rng.integers(0, K + 1, B).astype(np.int32) if turn % 2 else None
        logits = torch.empty_like(draft[:1].expand(K + 1, B, V)).contiguous()
        before = big.h_state.clone()
        n, tokens = big.rnnlm_verify_chunk(x, cuda(u), draft if turn < 3 else None, cuda(lengths), logits=logits)
        big.rnnlm_check()
        ref, q, drafts = logits.float().cpu().numpy().astype(np.float64), draft.float().cpu().numpy().astype(np.float64), x[1:].cpu().numpy()
        for b in range(B):
            want = L.verify(ref[:, b], drafts[:, b], u[:, b], q[:, b] if turn < 3 else None, None if lengths is None else lengths[b])
            assert int(n[b]) == want[0] and tokens[:, b].tolist() == want[1].tolist()
        for kept in range(K + 1):
            check.h_state.copy_(before)
            check.rnnlm_forward_logits(x[: kept + 1].contiguous())
            mine = (n == kept)
            d = (check.h_state - big.h_state)[mine].abs()
            assert d.numel() == 0 or float(d.max()) <= (1e-6 if precision == FP32 else 2.0 ** -8)
        # the student goes on from where its texts are
        small.h_state.copy_(state)
        for i in range(K):
            small.rnnlm_forward_logits(x[i: i + 1])
        word = tokens.gather(0, n.long()[None])[0].contiguous()


def test_a_verification_step_can_be_captured():
    V, H, B, K = 3000, 128, 4, 2
    g, _ = handle(V, H, 0, B, K + 1, BF16, 1)
    e, _ = handle(V, H, 0, B, K + 1, BF16, 1)
    rng = np.random.default_rng(1)
    x, u = torch.zeros(K + 1, B, dtype=torch.int32, device="cuda"), torch.zeros(K + 1, B, device="cuda")
    mk = lambda: (torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(K + 1, B, dtype=torch.int32, device="cuda"),  # noqa: E731
                  torch.empty(K + 1, B, V, dtype=torch.bfloat16, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    n, tokens, logits, ws = mk()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g.rnnlm_verify_chunk(x, u, None, None, logits=logits, accepted=n, tokens=tokens, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.rnnlm_verify_chunk(x, u, None, None, logits=logits, accepted=n, tokens=tokens, workspace=ws)
    g.rnnlm_reset_state()
    n2, tokens2, logits2, ws2 = mk()
    for _ in range(4):
        x.copy_(cuda(rng.integers(0, V, (K + 1, B)), np.int32))
        u.copy_(cuda(rng.random((K + 1, B)), np.float32))
        graph.replay()
        e.rnnlm_verify_chunk(x, u, None, None, logits=logits2, accepted=n2, tokens=tokens2, workspace=ws2)
        torch.cuda.synchronize()
        assert torch.equal(n, n2) and torch.equal(tokens, tokens2) and torch.equal(logits, logits2) and torch.equal(g.h_state, e.h_state)


@pytest.mark.parametrize("precision", [FP32, BF16])
def test_a_distilled_training_window_can_be_captured(precision):
    V, H, B, T, K = 3001, 128, 8, 4, 10
    g, _ = handle(V, H, 0, B, T, precision, 1)
    e, _ = handle(V, H, 0, B, T, precision, 1)
    x = torch.zeros(T, B, dtype=torch.int32, device="cuda")
    mk = lambda: [cuda(a) for a in teacher(T, B, V, K, 1.0, 0)]  # noqa: E731
    ids, vals, lse, weight, y = mk()
    out = lambda: (torch.empty(T, B, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda"),  # noqa: E731
                   torch.empty(T, B, V, device="cuda", dtype=torch.float32 if precision == FP32 else torch.bfloat16))
    (loss, total, z), (loss2, total2, z2) = out(), out()
    call = lambda h, l, s, r, lr: h.rnnlm_distill_train_chunk(x, y, ids, vals, lr, lse, weight, 1.0, 0.5, logits=r, loss=l, sum_loss=s)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for h in (g, e):
            call(h, loss, total, z, 0.5)  # (the first call outside of a capture)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(g, loss, total, z, 0.5)
    for k in range(4):
        x.copy_(cuda(synth.zipf_tokens(T * B, V, 1.0, k).reshape(T, B).astype(np.int32)))
        for kept, new in zip((ids, vals, lse, weight, y), teacher(T, B, V, K, 1.0, k)):
            kept.copy_(torch.as_tensor(new))
        graph.replay()
        call(e, loss2, total2, z2, 0.5)
        torch.cuda.synchronize()
        assert torch.equal(loss, loss2) and torch.equal(total, total2) and torch.equal(z, z2) and torch.equal(g.h_state, e.h_state), k
        for name in ("E", "U", "Wo", "b"):
            assert torch.equal(getattr(g, name), getattr(e, name)), (k, name)
    g.rnnlm_check()


def test_teacher_to_student_by_way_of_lists():
    """The three calls as they are used together: a teacher's window, its lists, the student's window; the student's gradients
    against autograd on the teacher's own lists."""
    V, B, T, K, tau = 2000, 6, 5, 40, 2.0
    big, _ = handle(V, 128, 0, B, T, BF16, 1, 0.4)
    small, w = handle(V, 64, 32, B, T, FP32, 2)
    x = synth.zipf_tokens(T * B, V, 1.0, 7).reshape(T, B).astype(np.int32)
    z = big.rnnlm_forward_logits(cuda(x))
    ids, vals, lse = binding.rnnlm_top_logits(z, K, tau)
    for b in range(B):
        i, v, n = L.top(z[2, b].float().cpu().numpy(), K, tau)
        assert ids[2, b].tolist() == i.tolist() and np.array_equal(vals[2, b].cpu().numpy(), v) and float(lse[2, b]) == pytest.approx(n, abs=1e-4)
    got = small.rnnlm_distill_grad_chunk(cuda(x), None, ids, vals, lse, tau=tau)
    small.rnnlm_check()
    zs, _ = logits64(w, x, torch.zeros(B, 64, dtype=torch.float64))
    loss64(zs, ids.cpu().numpy(), vals.cpu().numpy(), lse.cpu().numpy(), np.ones((T, B), np.float32), np.full((T, B), -1), tau, 1.0).mean().backward()
    for name, v in w.items():
        close(name, got["g" + name], v.grad, 1e-3)
