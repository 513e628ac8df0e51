"""Windows of a handle that adapt its model: the policy and preference criteria, and adapters beside the output layer, against
autograd in 64 bits and the fp64 oracle.  Tolerances as for the other windows: fp32 log-probabilities 1e-4 relative + 1e-6,
gradients 1e-3 of each tensor's scale (max and l2); bf16 gradients 2e-2 (compressed architecture 3e-2), with criteria whose
slope hangs little on the logits' own rounding."""
import numpy as np
import pytest
import torch

from oracle import adapt as A
from paper_1502_00512_amd import binding, synth
from test_gpu_distill import BF16, FP32, close, cuda, handle, logits64

pytestmark = pytest.mark.gpu

SHAPES = [(1000, 64, 0, 4, 8), (777, 50, 0, 6, 7), (3001, 200, 0, 34, 3), (520, 96, 0, 70, 2), (300, 130, 0, 2, 1), (700, 64, 32, 4, 6),
          (1001, 96, 50, 6, 7), (2500, 256, 128, 32, 10)]


def window(T, B, V, seed):
    x = synth.zipf_tokens(T * B, V, 1.0, seed).reshape(T, B).astype(np.int32)
    y = synth.zipf_tokens(T * B, V, 1.0, seed + 1000).reshape(T, B).astype(np.int32)
    rng = np.random.default_rng(seed)
    y[rng.random((T, B)) < 0.15] = -1
    y[0, 0] = max(y[0, 0], 0)
    return x, y, rng


def word_logp64(z, y):
    y = torch.as_tensor(y).long()
    return torch.where(y >= 0, torch.log_softmax(z, 2).gather(2, y.clamp(min=0)[..., None])[..., 0], 0.0)


def policy64(z, y, adv, old, ref, weight, tau, lo, hi, beta):
    t = lambda a: torch.as_tensor(a.astype(np.float64))  # noqa: E731
    l = word_logp64(z / tau, y)
    rho = torch.exp(l - (l.detach() if old is None else t(old)))
    loss = -torch.minimum(rho * t(adv), rho.clamp(1 - lo, 1 + hi) * t(adv))
    if beta:
        d = t(ref) - l
        loss = loss + beta * (torch.exp(d) - d - 1)
    return torch.where(torch.as_tensor(y) >= 0, t(weight) * loss, 0.0), l


def preference64(z, y, ref, weight, kind, beta, smoothing, mean):
    t = lambda a: torch.as_tensor(np.asarray(a, np.float64))  # noqa: E731
    has, P = torch.as_tensor(y) >= 0, y.shape[1] // 2
    S = word_logp64(z, y).sum(0) / (has.sum(0).clamp(min=1) if mean else 1)
    r = S - t(ref)
    r = r[:P] - r[P:]
    f = torch.nn.functional
    if kind == binding.RNNLM_PREFERENCE_LOGISTIC:
        loss = -(1 - smoothing) * f.logsigmoid(beta * r) - smoothing * f.logsigmoid(-beta * r)
    elif kind == binding.RNNLM_PREFERENCE_SQUARED:
        loss = (r - 0.5 / beta) ** 2
    else:
        loss = torch.relu(1 - beta * r)
    return t(weight) * loss, S


@pytest.mark.parametrize("precision", [FP32, BF16])
@pytest.mark.parametrize("V,H,P,B,T", SHAPES)
def test_policy_gradients(V, H, P, B, T, precision):
    g, w = handle(V, H, P, B, T, precision, V)
    x, y, rng = window(T, B, V, V)
    z, _ = logits64(w, x, torch.zeros(B, H, dtype=torch.float64))
    l = word_logp64(z, y).detach().numpy()
    adv, weight = rng.normal(size=(T, B)).astype(np.float32), rng.choice([0.0, 1.0, 2.0], (T, B)).astype(np.float32)
    weight[0, 0], adv[0, 0] = 1.0, 1.0
    cases = [(None, 0.0, 0.8)]
    if precision == FP32:
        cases += [((l + 0.3 * rng.normal(size=(T, B))).astype(np.float32), 0.2, 1.0)]
    ref = (l + 0.5 * rng.normal(size=(T, B))).astype(np.float32)
    for old, beta, tau in cases:
        for v in w.values():
            v.grad = None
        losses, lp = policy64(logits64(w, x, torch.zeros(B, H, dtype=torch.float64))[0], y, adv, old, ref, weight, tau, 0.2, 0.3, beta)
        losses.mean().backward()
        kept = g.h_state.clone(), g.E.clone()
        got = g.rnnlm_policy_grad_chunk(cuda(x), cuda(y), cuda(adv), cuda(old), cuda(ref) if beta else None, cuda(weight), tau, 0.2, 0.3, beta)
        g.rnnlm_check()
        assert torch.equal(kept[0], g.h_state) and torch.equal(kept[1], g.E)
        if precision == FP32:
            assert np.abs(got["loss"].cpu().numpy() - losses.detach().numpy()).max() <= 1e-3 * float(losses.detach().abs().max())
            has = (y >= 0) & (weight != 0)
            assert (np.abs(got["logp"].cpu().numpy() - lp.detach().numpy())[has] <= 1e-4 * np.abs(lp.detach().numpy())[has] + 1e-6).all()
            assert not got["logp"].cpu().numpy()[~has].any()
        for name, v in w.items():
            close(name, got["g" + name], v.grad, 1e-3 if precision == FP32 else 3e-2 if P else 2e-2)


@pytest.mark.parametrize("precision", [FP32, BF16])
@pytest.mark.parametrize("V,H,P,B,T", SHAPES)
def test_preference_gradients(V, H, P, B, T, precision):
    g, w = handle(V, H, P, B, T, precision, V)
    x, y, rng = window(T, B, V, V + 3)
    S = word_logp64(logits64(w, x, torch.zeros(B, H, dtype=torch.float64))[0], y).sum(0).detach().numpy()
    ref, weight = (S + rng.normal(size=B)).astype(np.float32), rng.uniform(0.5, 1.5, B // 2).astype(np.float32)
    for kind, beta, smoothing, mean in ((binding.RNNLM_PREFERENCE_LOGISTIC, 0.05, 0.1, False), (binding.RNNLM_PREFERENCE_HINGE, 0.01, 0.0, True),
                                        (binding.RNNLM_PREFERENCE_SQUARED, 0.05, 0.0, False)):
        for v in w.values():
            v.grad = None
        losses, S64 = preference64(logits64(w, x, torch.zeros(B, H, dtype=torch.float64))[0], y, ref, weight, kind, beta, smoothing, mean)
        losses.mean().backward()
        kept = g.h_state.clone(), g.E.clone()
        got = g.rnnlm_preference_grad_chunk(cuda(x), cuda(y), cuda(ref), cuda(weight), kind, beta, smoothing, mean)
        g.rnnlm_check()
        assert torch.equal(kept[0], g.h_state) and torch.equal(kept[1], g.E)
        if precision == FP32:
            assert np.abs(got["loss"].cpu().numpy() - losses.detach().numpy()).max() <= 1e-3 * float(losses.detach().abs().max())
            assert (np.abs(got["logp"].cpu().numpy() - S64.detach().numpy()) <= 1e-4 * np.abs(S64.detach().numpy()) + 1e-6).all()
        for name, v in w.items():
            close(name, got["g" + name], v.grad, 1e-3 if precision == FP32 else 3e-2 if P else 2e-2)


@pytest.mark.parametrize("V,H,P,B,T", [(1000, 64, 0, 4, 8), (777, 50, 0, 6, 7), (700, 64, 32, 4, 6)])
def test_training_windows_fp32(V, H, P, B, T):
    """Windows of both criteria in turn, against plain gradient descent in 64 bits on autograd's gradients."""
    lr = 0.3
    g, w = handle(V, H, P, B, T, FP32, V + 1)
    h = torch.zeros(B, H, dtype=torch.float64)
    total = torch.zeros(1, dtype=torch.float64, device="cuda")
    for k in range(4):
        x, y, rng = window(T, B, V, V + k)
        z, h2 = logits64(w, x, h)
        if k % 2:
            ref, weight = rng.normal(size=B).astype(np.float32), np.ones(B // 2, np.float32)
            losses, logp = preference64(z, y, ref, weight, 0, 0.1, 0.0, False)
        else:
            adv, weight = rng.normal(size=(T, B)).astype(np.float32), rng.random((T, B)).astype(np.float32)
            old = (word_logp64(z, y).detach().numpy() + 0.2 * rng.normal(size=(T, B))).astype(np.float32)
            losses, logp = policy64(z, y, adv, old, None, weight, 1.0, 0.2, 0.2, 0.0)
        losses.mean().backward()
        h = h2.detach()
        with torch.no_grad():
            for v in w.values():
                v -= lr * v.grad
                v.grad = None
        loss, lp = torch.empty(losses.shape, device="cuda"), torch.empty(logp.shape, device="cuda")
        if k % 2:
            g.rnnlm_preference_train_chunk(cuda(x), cuda(y), lr, cuda(ref), loss=loss, logp=lp, sum_loss=total)
        else:
            g.rnnlm_policy_train_chunk(cuda(x), cuda(y), cuda(adv), lr, cuda(old), weight=cuda(weight), loss=loss, logp=lp, sum_loss=total)
        assert np.abs(loss.cpu().numpy() - losses.detach().numpy()).max() <= 1e-4 * float(losses.detach().abs().max()) + 1e-6
        assert np.abs(lp.cpu().numpy() - logp.detach().numpy()).max() <= 1e-4 * float(logp.detach().abs().max()) + 1e-6
        assert float(total) == pytest.approx(float(loss.double().sum()), rel=1e-12, abs=1e-12)
        assert np.abs(g.h_state.cpu().numpy() - h.numpy()).max() < 1e-5
    g.rnnlm_check()
    for name, v in w.items():
        assert np.abs(getattr(g, name).cpu().numpy() - v.detach().numpy()).max() <= 1e-4 * max(1.0, float(v.detach().abs().max())), name
    g.rnnlm_policy_train_chunk(cuda(x), cuda(y), cuda(np.ones((T, B), np.float32)), 0.0)  # (without outputs)
    g.rnnlm_preference_train_chunk(cuda(x), cuda(y), 0.0)
    g.rnnlm_check()


def test_what_these_windows_report_and_refuse():
    V, H, B, T = 300, 32, 4, 3
    g, _ = handle(V, H, 0, B, T, FP32, 1)
    x, y, _ = window(T, B, V, 1)
    adv = np.ones((T, B), np.float32)
    for call in (lambda y: g.rnnlm_policy_train_chunk(cuda(x), cuda(y), cuda(adv), 0.0), lambda y: g.rnnlm_preference_train_chunk(cuda(x), cuda(y), 0.0)):
        call(np.where(y < 0, -(1 << 31), y).astype(np.int32))
        g.rnnlm_check()
        call(np.where(y < 0, V, y).astype(np.int32))
        with pytest.raises(binding.RnnlmError) as e:
            g.rnnlm_check()
        assert e.value.status == -2
    g.rnnlm_policy_train_chunk(cuda(x), cuda(y), cuda(adv * np.nan), 0.0)
    with pytest.raises(binding.RnnlmError) as e:
        g.rnnlm_check()
    assert e.value.status == -3
    g.rnnlm_preference_train_chunk(cuda(x), cuda(y), 0.0, cuda(np.full(B, np.inf, np.float32)))
    with pytest.raises(binding.RnnlmError) as e:
        g.rnnlm_check()
    assert e.value.status == -3
    bad = [lambda: g.rnnlm_policy_train_chunk(cuda(x), cuda(y), cuda(adv), 0.1, tau=0.0), lambda: g.rnnlm_policy_train_chunk(cuda(x), cuda(y), None, 0.1),
           lambda: g.rnnlm_policy_train_chunk(cuda(x), cuda(y), cuda(adv), 0.1, beta=0.1), lambda: g.rnnlm_policy_train_chunk(cuda(x), None, cuda(adv), 0.1),
           lambda: g.rnnlm_policy_train_chunk(cuda(x), cuda(y), cuda(adv), 0.1, clip_low=2.0), lambda: g.rnnlm_policy_grad_chunk(cuda(x), cuda(y), cuda(adv), clip_high=-1.0),
           lambda: g.rnnlm_preference_train_chunk(cuda(x), cuda(y), 0.1, kind=3), lambda: g.rnnlm_preference_train_chunk(cuda(x), cuda(y), 0.1, beta=0.0),
           lambda: g.rnnlm_preference_train_chunk(cuda(x), cuda(y), 0.1, kind=1, smoothing=0.1), lambda: g.rnnlm_preference_grad_chunk(cuda(x), None),
           lambda: g.rnnlm_preference_train_chunk(cuda(x), cuda(y), float("nan"))]
    for call in bad:
        with pytest.raises(binding.RnnlmError) as e:
            call()
        assert e.value.status == -1
    odd, _ = handle(V, H, 0, 3, T, FP32, 1)
    with pytest.raises(binding.RnnlmError):  # an odd number of streams has no pairs
        odd.rnnlm_preference_train_chunk(cuda(x[:, :3]), cuda(y[:, :3]), 0.1)
    # nothing ran: the state is where it was
    assert torch.equal(odd.h_state, torch.zeros_like(odd.h_state))


def adapters(n, R, K, V, precision, seed):
    rng = np.random.default_rng(seed)
    dt = torch.float32 if precision == FP32 else torch.bfloat16
    down, up = (cuda(rng.normal(size=s) * f, np.float32).to(dt) for s, f in (((n, R, K), 0.3), ((n, V, R), 0.5)))
    return down, up, cuda(rng.uniform(0.5, 1.5, n), np.float32)


@pytest.mark.parametrize("precision", [FP32, BF16])
@pytest.mark.parametrize("V,H,P,B,T", SHAPES)
def test_forward_adapted(V, H, P, B, T, precision):
    g, w = handle(V, H, P, B, T, precision, V)
    plain, _ = handle(V, H, P, B, T, precision, V)
    n, R, K = 3, 5, P or H
    down, up, scale = adapters(n, R, K, V, precision, V)
    h = torch.zeros(B, H, dtype=torch.float64)
    rng = np.random.default_rng(V)
    for k in range(2):
        x = synth.zipf_tokens(T * B, V, 1.0, V + k).reshape(T, B).astype(np.int32)
        ids = rng.integers(-1, n, (T, B)).astype(np.int32)
        rows = torch.full((T, B, V + 5), 9.0, device="cuda", dtype=down.dtype)
        z, states, inner = g.rnnlm_forward_adapted(cuda(x), down, up, cuda(ids), scale, rows[:, :, :V])
        assert bool((rows[:, :, V:] == 9.0).all())
        base = plain.rnnlm_forward_logits(cuda(x))
        assert torch.equal(g.h_state, plain.h_state)
        # the same as the three steps one by one
        want, inner2 = binding.rnnlm_adapter_forward(states, down, up, cuda(ids), scale, base=base)
        assert torch.equal(z, want) and torch.equal(inner, inner2)
        free = cuda(ids) < 0
        assert torch.equal(z[free], base[free])
        if precision == FP32:  # what the output layer read
            with torch.no_grad():
                out, hh = [], h
                for row in torch.as_tensor(x).long():
                    hh = torch.sigmoid((w["E"][row] @ w["A"].T if P else w["E"][row]) + hh @ w["U"].T)
                    out.append(hh @ w["C"].T if P else hh)
                h = hh
            assert float((states.cpu().double() - torch.stack(out)).abs().max()) < 1e-4
        elif not P:
            assert torch.equal(states[-1], g.h_state.bfloat16())
    g.rnnlm_check()
    g.rnnlm_forward_adapted(cuda(x), down, up, cuda(np.full((T, B), n, np.int32)), scale)
    with pytest.raises(binding.RnnlmError) as e:
        g.rnnlm_check()
    assert e.value.status == -2
    for bad in (dict(down=down[:, :, :-1]), dict(up=up[:, :-1]), dict(ids=None)):
        with pytest.raises(binding.RnnlmError):
            g.rnnlm_forward_adapted(cuda(x), **{**dict(down=down, up=up, ids=cuda(ids)), **bad})


@pytest.mark.parametrize("precision", [FP32, BF16])
@pytest.mark.parametrize("criterion", ["policy", "preference"])
def test_adapters_learn_what_the_criteria_ask(criterion, precision):
    """The calls as they are used together: texts are read with their adapters, a criterion on the logits, gradients of the
    adapters; against autograd in 64 bits on the same states, over two steps of descent; and the step that serves them."""
    V, H, B, T, n, R = 1200, 80, 8, 6, 3, 6
    g, w = handle(V, H, 0, B, T, precision, 9)
    down, up, scale = adapters(n, R, H, V, precision, 3)
    ids = np.tile(np.array([0, 1, 2, -1, 0, 1, 2, 2], np.int32), (T, 1))
    for step in range(2):
        x, y, rng = window(T, B, V, 20 + step)
        g.rnnlm_reset_state()
        z, states, inner = g.rnnlm_forward_adapted(cuda(x), down, up, cuda(ids), scale)
        base = z.clone()
        adv = rng.normal(size=(T, B)).astype(np.float32)
        if criterion == "policy":
            binding.rnnlm_policy_loss(z, cuda(y), cuda(adv), scale=1.0 / (T * B), dlogits=z)
        else:
            binding.rnnlm_preference_loss(z, cuda(y), beta=0.05, scale=2.0 / B, dlogits=z)
        ddown, dup = binding.rnnlm_adapter_backward(z, states, inner, down, up, cuda(ids), scale)
        g.rnnlm_check()
        # the same in 64 bits: from the states and the frozen logits (the adapted ones less the adapters')
        D, U = down.cpu().double().requires_grad_(), up.cpu().double().requires_grad_()
        s, i = states.cpu().double(), torch.as_tensor(ids).long()
        f = torch.where(i >= 0, scale.cpu().double()[i.clamp(min=0)], 0.0)[..., None]
        delta = f * torch.einsum("tbr,tbvr->tbv", torch.einsum("tbk,tbrk->tbr", s, D[i.clamp(min=0)]), U[i.clamp(min=0)])
        adapted = base.cpu().double() - delta.detach() + delta
        if criterion == "policy":
            policy64(adapted, y, adv, None, None, np.ones((T, B)), 1.0, 0.2, 0.2, 0.0)[0].mean().backward()
        else:
            preference64(adapted, y, np.zeros(B), np.ones(B // 2), 0, 0.05, 0.0, False)[0].mean().backward()
        # (bf16: the criterion's gradient is rounded, half a step of 2^-8 each)
        close("ddown", ddown, D.grad, 1e-3 if precision == FP32 else 1e-2)
        close("dup", dup, U.grad, 1e-3 if precision == FP32 else 1e-2)
        down, up = (down.float() - 0.5 * ddown).to(down.dtype), (up.float() - 0.5 * dup).to(up.dtype)
    # a step of serving: one word of every text
    one = g.rnnlm_forward_adapted(cuda(x[:1]), down, up, cuda(ids[:1]), scale)[0]
    words, vals, lse = binding.rnnlm_top_logits(one, 5)
    assert words.shape == (1, B, 5) and bool((lse >= vals[..., 0]).all())
    for b in range(B):
        assert sorted(words[0, b].tolist()) == sorted(np.argsort(-one[0, b].float().cpu().numpy(), kind="stable")[:5].tolist())


@pytest.mark.parametrize("precision", [FP32, BF16])
def test_windows_can_be_captured(precision):
    V, H, B, T, n, R = 3001, 128, 8, 4, 4, 8
    g, _ = handle(V, H, 0, B, T, precision, 1)
    e, _ = handle(V, H, 0, B, T, precision, 1)
    x = torch.zeros(T, B, dtype=torch.int32, device="cuda")
    y, ids = torch.zeros_like(x), torch.zeros_like(x)
    adv = torch.zeros(T, B, device="cuda")
    down, up, scale = adapters(n, R, H, V, precision, 5)
    dt = down.dtype

    def buffers():
        return dict(z=torch.empty(T, B, V, dtype=dt, device="cuda"), s=torch.empty(T, B, H, dtype=dt, device="cuda"), i=torch.empty(T, B, R, device="cuda"),
                    ws=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"), a=torch.empty(T, B, device="cuda"), b=torch.empty(B // 2, device="cuda"),
                    z2=torch.empty(T, B, V, dtype=dt, device="cuda"), z3=torch.empty(T, B, V, dtype=dt, device="cuda"))

    def calls(h, o):
        h.rnnlm_policy_train_chunk(x, y, adv, 0.3, logits=o["z"], loss=o["a"])
        h.rnnlm_preference_train_chunk(x, y, 0.3, logits=o["z2"], loss=o["b"], workspace=o["ws"])
        h.rnnlm_forward_adapted(x, down, up, ids, scale, o["z3"], o["s"], o["i"], o["ws"])
    o, o2 = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(g, o)
        calls(e, o2)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(g, o)
    rng = np.random.default_rng(2)
    for k in range(4):
        x.copy_(cuda(synth.zipf_tokens(T * B, V, 1.0, k).reshape(T, B).astype(np.int32)))
        y.copy_(cuda(rng.integers(-1, V, (T, B)), np.int32))
        ids.copy_(cuda(rng.integers(-1, n, (T, B)), np.int32))
        adv.copy_(cuda(rng.normal(size=(T, B)), np.float32))
        graph.replay()
        calls(e, o2)
        torch.cuda.synchronize()
        assert all(torch.equal(o[key], o2[key]) for key in o if key != "ws") and torch.equal(g.h_state, e.h_state), k
        for name in ("E", "U", "Wo", "b"):
            assert torch.equal(getattr(g, name), getattr(e, name)), (k, name)
    g.rnnlm_check()
