"""The policy and preference losses on rows of logits, through the binding, against the fp64 oracle (oracle/adapt.py).

Tolerances.  An exponential e^{(z - m) / tau} is 2^t with t = z c + b in fp32: c, b and the sum are each rounded, |z| and |m| over
tau at most Z, so |dt| <= 2^-24 * 4 Z log2 e and the exponential is off by at most 2^-24 * 4 Z relative, plus one unit (2^-23) of
the hardware's exponential.  A thread adds at most 26 * 8 + 1 terms one after the other (2^-24 each; rows that do not fit the
registers: 2^20 / 512 of them), trees of at most 6 + 16 sums follow, and rescaling a running sum costs another rounding each 32
terms.  A sum's relative error E is that of its logarithm, the rest of l is in 64 bits: |dl| <= E.  A softmax value is off by E
and by its own exponential, factor and product.  What follows from l in 64 bits moves by its derivative times E, and outputs are
rounded once: eps / 2 of their type."""
import numpy as np
import pytest
import torch

from oracle import adapt as A
from paper_1502_00512_amd import binding

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step
F32 = 2.0 ** -24


def largest(z, tau):
    """Z over the elements that matter: one 110 tau below the row's maximum adds less than 2^-158 of it."""
    z = z[np.isfinite(z)]
    return np.abs(z[z > z.max() - 110.0 * tau]).max() / tau if len(z) else 0.0


def row_err(z, tau):
    V, Z = len(z), largest(z, tau)
    terms = 26 * 8 + 1 if V <= 100000 else V // 512 + 1
    return (terms * 1.1 + 22 + 2) * F32 + F32 * (4 * Z + 2)


def place(z, dtype, pad=0):
    """The rows on the GPU, pad elements of NaN between them; and their values as the type holds them."""
    buf = torch.full((*z.shape[:-1], z.shape[-1] + pad), float("nan"), dtype=DTYPES[dtype], device="cuda")
    buf[..., : z.shape[-1]] = torch.as_tensor(z)
    d = buf[..., : z.shape[-1]]
    return d, d.float().cpu().numpy().astype(np.float64)


def gpu(a, dtype=torch.float32):
    return None if a is None else torch.as_tensor(np.asarray(a)).to(dtype).cuda()


def same(got, want, tol, what):
    got, want, tol = np.broadcast_arrays(np.asarray(got, np.float64), want, tol)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), what
    off = np.abs(got[fine] - want[fine])
    assert np.all(off <= tol[fine]), (what, np.max(off - tol[fine]), np.nanmax(off / np.maximum(tol[fine], 1e-300)))


def gradient_tol(z, y, g, dg, tau, dtype, want):
    """g: factor of the gradient (over tau and all), dg: what it is off by."""
    e = row_err(z, tau)
    q = A.softmax(z, tau)
    hit = np.zeros(len(z))
    hit[y] = 1.0
    soft = e + F32 * (4 * largest(z, tau) + 8)  # a softmax value, relative
    # (denormal results of the exponential and of the type count as zero)
    return abs(g) * (q * soft + hit * 2 * F32) + dg * np.abs(hit - q) + HALF[dtype] * np.abs(want) * (1 + 2 * soft) + abs(g) * 2.0 ** -100 + 2.0 ** -126


# ---- policy -----------------------------------------------------------------------------------------------------------
def draw_policy(rows, V, dtype, tau, seed, kind="normal", spread=0.3):
    rng = np.random.default_rng(seed)
    z = rng.normal(0.0, 3.0, (rows, V))
    if kind == "masked":
        z[rng.random((rows, V)) < 0.9] = -np.inf
    elif kind == "lowest":
        z[rng.random((rows, V)) < 0.9] = -3e38
    elif kind == "front":  # the first words masked: waves whose first slots hold nothing
        z[:, : V // 2] = -np.inf
    elif kind == "steep":
        z = np.linspace(-200.0, 250.0, V)[None] + z
    elif kind == "offset":
        z += 3e4
    elif kind == "equal":
        z[:] = -7.25
    y = rng.integers(0, V, rows)
    y = np.where(np.isfinite(z[np.arange(rows), y]) & (z[np.arange(rows), y] > -1e30), y, z.argmax(1))
    d, ref = place(z, dtype, 3)
    l = np.array([A.word_logp(ref[m], y[m], tau) for m in range(rows)])
    old, prior = (l + spread * rng.normal(size=rows)).astype(np.float32), (l + spread * rng.normal(size=rows)).astype(np.float32)
    return d, ref, y.astype(np.int32), rng.normal(size=rows).astype(np.float32), old, prior, rng


def check_policy(d, z, y, adv, old, ref, weight, dtype, tau=1.0, lo=0.2, hi=0.25, beta=0.1, scale=0.5, in_place=False):
    dz = d if in_place else torch.full(z.shape, 7.0, dtype=DTYPES[dtype], device="cuda")
    total = torch.zeros(1, dtype=torch.float64, device="cuda")
    loss, logp = binding.rnnlm_policy_loss(d, gpu(y, torch.int32), gpu(adv), gpu(old), gpu(ref), gpu(weight), tau, lo, hi, beta, scale,
                                           dlogits=dz, sum_loss=total)
    lo, hi, beta, scale, tau = (float(np.float32(v)) for v in (lo, hi, beta, scale, tau))
    L, l, D, g = A.policy(z, y, adv, old, ref, weight, tau, lo, hi, beta, scale)
    w = np.ones(len(z)) if weight is None else weight.astype(np.float64)
    counts = (y >= 0) & (y < z.shape[1]) & (w != 0)
    E = np.array([row_err(r, tau) if c else 0.0 for r, c in zip(z, counts)])
    with np.errstate(invalid="ignore", over="ignore"):
        rho = np.ones(len(z)) if old is None else np.where(counts, np.exp(l - old.astype(np.float64)), 1.0)
        d_kl = np.zeros(len(z)) if ref is None else np.where(counts, np.exp(ref.astype(np.float64) - l), 0.0)
    near = np.zeros(len(z), bool)  # of its border than l is known: one of the two sides' derivatives (the loss has no step there)
    for border in (1 - lo, 1 + hi):
        if old is not None and border > 0:
            near |= counts & (np.abs(np.log(np.maximum(rho, 1e-300) / border)) < 2 * E)
    assert near.sum() <= len(z) // 100
    same(logp.cpu(), l, E + F32 * np.abs(l), "logp")
    moved = 0.0 if old is None else rho * np.abs(adv)
    same(loss.cpu(), L, np.where(counts, w * (moved + beta * (d_kl + 1.0)) * E * 1.01 + F32 * np.abs(L) + 1e-14 * w, 0.0), "loss")
    fine = np.isfinite(L)
    if fine.all():
        same(total.cpu(), [loss.double().sum().item()], 1e-12 * np.abs(L).sum() + 1e-300, "sum")
    dg = w * scale / tau * ((0.0 if old is None else np.abs(g) + beta) + beta * d_kl) * E * 1.01
    got = dz.float().cpu().numpy()
    for m in range(len(z)):
        if not counts[m] or l[m] == -np.inf:
            assert not got[m].any(), m
            continue
        f = g[m] * w[m] * scale / tau
        if near[m]:  # the side that the word itself shows
            free, kl = -rho[m] * adv[m], (-beta * (d_kl[m] - 1.0) if beta else 0.0)
            f = min((kl, kl + free), key=lambda x: abs(x * w[m] * scale / tau * (1 - A.softmax(z[m], tau)[y[m]]) - got[m][y[m]])) * w[m] * scale / tau
            D[m] = -A.softmax(z[m], tau) * f
            D[m][y[m]] += f
            dg[m] = w[m] * scale / tau * (abs(free) + 2 * beta * d_kl[m] + beta) * E[m] * 1.01
        same(got[m], D[m], gradient_tol(z[m], y[m], f, dg[m] + F32 * abs(f), tau, dtype, D[m]), ("dlogits", m))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 63, 500, 1000, 2047, 2048, 2049, 5000, 10007, 33278])
def test_policy_widths(V, dtype):
    d, z, y, adv, old, ref, _ = draw_policy(6, V, dtype, 1.0, V)
    check_policy(d, z, y, adv, old, ref, None, dtype)


@pytest.mark.parametrize("dtype,V", [("bf16", 64000), ("bf16", 81921), ("bf16", 131072), ("bf16", 204805), ("bf16", 1 << 20), ("fp32", 40960), ("fp32", 64001),
                                     ("fp32", 102400), ("fp32", 150000)])
def test_policy_wide_rows(V, dtype):
    d, z, y, adv, old, ref, _ = draw_policy(3, V, dtype, 0.9, V)
    check_policy(d, z, y, adv, old, ref, None, dtype, tau=0.9)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V", [(1024, 500), (1500, 1025), (1100, 3001), (1, 20000), (1024, 20)])
def test_policy_many_rows(rows, V, dtype):
    d, z, y, adv, old, ref, _ = draw_policy(rows, V, dtype, 1.0, rows)
    check_policy(d, z, y, adv, old, ref, None, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["masked", "lowest", "front", "steep", "offset", "equal"])
@pytest.mark.parametrize("V", [37, 4000, 41000])
def test_policy_rows_of_all_kinds(kind, V, dtype):
    d, z, y, adv, old, ref, _ = draw_policy(5, V, dtype, 1.3, 5, kind)
    check_policy(d, z, y, adv, old, ref, None, dtype, tau=1.3)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("beta,use_old", [(0.0, True), (0.0, False), (0.3, False), (0.3, True)])
@pytest.mark.parametrize("in_place", [False, True])
def test_policy_terms_and_positions_that_do_not_count(beta, use_old, in_place, dtype):
    rows, V = 40, 777
    d, z, y, adv, old, ref, rng = draw_policy(rows, V, dtype, 1.0, 11, spread=0.5)
    w = rng.random(rows).astype(np.float32)
    w[::5] = 0.0
    y[1::7] = -1
    y[2::9] = -(1 << 31)
    adv[3] = 0.0
    d[0] = float("nan")   # rows that do not count hold anything
    d[1] = float("inf")
    z[:2] = d[:2].float().cpu().numpy()
    check_policy(d, z, y, adv, old if use_old else None, ref if beta else None, w, dtype, beta=beta, hi=0.3, in_place=in_place)


def test_policy_words_without_probability():
    V = 300
    d, z, y, adv, old, ref, _ = draw_policy(4, V, "fp32", 1.0, 3)
    d[0, y[0]] = -float("inf")  # the word is masked
    d[1] = -float("inf")  # no word left
    d[2, 5] = float("nan")
    d[3, 6] = float("inf")
    y[3] = 7
    adv[:] = [1.0, -1.0, 1.0, 1.0]
    for beta in (0.0, 0.1):
        dz = torch.empty_like(d)
        loss, logp = binding.rnnlm_policy_loss(d, gpu(y, torch.int32), gpu(adv), gpu(old), gpu(ref), beta=beta, dlogits=dz)
        loss, logp, dz = loss.tolist(), logp.tolist(), dz.cpu()
        assert logp[:2] == [-np.inf, -np.inf] and np.isnan(logp[2]) and np.isnan(logp[3])
        assert loss[:2] == ([np.inf, np.inf] if beta else [0.0, float(np.float32(1.0 - float(np.float32(0.2))))])
        assert np.isnan(loss[2]) and np.isnan(loss[3]) and not dz[:2].any()


def test_policy_flags_words_out_of_range():
    d, z, y, adv, old, _, _ = draw_policy(6, 50, "fp32", 1.0, 4)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    y[0] = -5
    check_policy(d, z, y, adv, old, None, None, "fp32", beta=0.0)
    binding.rnnlm_policy_loss(d, gpu(y, torch.int32), gpu(adv), gpu(old), range_flag=flag)
    assert flag.item() == 0
    y[2], y[3] = 50, (1 << 31) - 1
    check_policy(d, z, y, adv, old, None, None, "fp32", beta=0.0)
    binding.rnnlm_policy_loss(d, gpu(y, torch.int32), gpu(adv), gpu(old), range_flag=flag)
    assert flag.item() == 1


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [90, 5000, 70000])
def test_policy_loss_alone_agrees(V, dtype):
    d, z, y, adv, old, ref, _ = draw_policy(9, V, dtype, 1.0, 6)
    loss, logp = binding.rnnlm_policy_loss(d, gpu(y, torch.int32), gpu(adv), gpu(old), gpu(ref), beta=0.2)
    E = np.array([row_err(r, 1.0) for r in z])
    L, l, _, _ = A.policy(z, y, adv, old, ref, None, beta=float(np.float32(0.2)), lo=float(np.float32(0.2)), hi=float(np.float32(0.2)))
    same(logp.cpu(), l, E + F32 * np.abs(l), "logp")
    scale = np.exp(l - old) * np.abs(adv) + 0.2 * (np.exp(ref - l) + 1)
    same(loss.cpu(), L, scale * E * 1.01 + F32 * np.abs(L), "loss")


def test_policy_strides_and_nothing():
    d, z, y, adv, old, _, _ = draw_policy(8, 100, "bf16", 1.0, 7)
    wide = torch.zeros(4, 3, 2, 128, dtype=torch.bfloat16, device="cuda")
    view = wide[:, 1, :, 5:105]  # rows 384 apart in the outer, 128 in the inner dimension: not evenly spaced
    with pytest.raises(binding.RnnlmError):
        binding.rnnlm_policy_loss(view, gpu(y, torch.int32).view(4, 2), gpu(adv).view(4, 2))
    out = torch.full((8, 2, 77 + 100), 3.0, dtype=torch.bfloat16, device="cuda")
    check = out[:, 1, 20:120]
    ref = torch.empty_like(d)
    a = binding.rnnlm_policy_loss(d, gpu(y, torch.int32), gpu(adv), gpu(old), dlogits=check)
    b = binding.rnnlm_policy_loss(d, gpu(y, torch.int32), gpu(adv), gpu(old), dlogits=ref)
    assert torch.equal(check, ref) and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    rest = out.clone()
    rest[:, 1, 20:120] = 3.0
    assert bool((rest == 3.0).all())
    total = torch.ones(1, dtype=torch.float64, device="cuda")
    e = lambda t: torch.empty(0, dtype=t, device="cuda")  # noqa: E731
    loss, logp = binding.rnnlm_policy_loss(d[:0], e(torch.int32), e(torch.float32), sum_loss=total)
    assert loss.numel() == 0 and logp.numel() == 0 and total.item() == 0.0


# ---- preference -------------------------------------------------------------------------------------------------------
def draw_preference(T, P, V, dtype, seed, ragged=True, kind="normal"):
    rng = np.random.default_rng(seed)
    z = rng.normal(0.0, 3.0, (T, 2 * P, V))
    if kind == "front":
        z[..., : V // 2] = -np.inf
    elif kind == "offset":
        z += 3e4
    elif kind == "lowest":
        z[rng.random(z.shape) < 0.9] = -3e38
    y = rng.integers(0, V, (T, 2 * P))
    at = np.take_along_axis(z, y[..., None], 2)[..., 0]
    y = np.where(at > -1e30, y, z.argmax(2))
    if ragged:
        t = np.arange(T)[:, None]
        y = np.where((t >= rng.integers(0, T // 3 + 1, 2 * P)) & (t < rng.integers(T // 2, T + 1, 2 * P)), y, -1)
    d, z = place(z, dtype, 5)
    return d, z, y.astype(np.int32), rng


def check_preference(d, z, y, ref, weight, dtype, kind="logistic", beta=0.1, smoothing=0.0, mean=False, scale=0.5, in_place=False):
    T, B, V = z.shape
    P = B // 2
    dz = d if in_place else torch.full(z.shape, 7.0, dtype=DTYPES[dtype], device="cuda")
    total = torch.zeros(1, dtype=torch.float64, device="cuda")
    which = dict(logistic=binding.RNNLM_PREFERENCE_LOGISTIC, squared=binding.RNNLM_PREFERENCE_SQUARED, hinge=binding.RNNLM_PREFERENCE_HINGE)[kind]
    loss, logp = binding.rnnlm_preference_loss(d, gpu(y, torch.int32), gpu(ref), gpu(weight), which, beta, smoothing, mean, scale, dlogits=dz,
                                               sum_loss=total)
    beta, smoothing, scale = (float(np.float32(v)) for v in (beta, smoothing, scale))
    L, S, D, r, g = A.preference(z, y, ref, weight, kind, beta, smoothing, mean, scale)
    w = np.ones(P) if weight is None else weight.astype(np.float64)
    counts = (y >= 0) & (y < V) & (np.concatenate([w, w]) != 0)
    n = np.maximum(counts.sum(0), 1) if mean else np.ones(B)
    E = np.array([[row_err(z[t, s], 1.0) if counts[t, s] else 0.0 for s in range(B)] for t in range(T)]).reshape(T, B)
    dS = E.sum(0) / n + 1e-15 * np.abs(S)
    same(logp.cpu(), S, dS + F32 * np.abs(S), "logp")
    dr = dS[:P] + dS[P:]
    slope = np.abs(g) + (2 * dr if kind == "squared" else 0)  # |L'| near r
    curve = {"logistic": beta * beta / 4, "squared": 2.0, "hinge": 0.0}[kind]  # at most |L''|
    if kind == "hinge":
        assert not np.any(np.abs(1 - beta * r) < 2 * beta * dr)
        slope = slope + 0.0
    elif kind == "logistic":
        slope = slope + curve * dr
    same(loss.cpu(), L, w * slope * dr + F32 * np.abs(L) + 1e-14 * w * (1 + beta * np.abs(np.where(np.isfinite(r), r, 0))), "loss")
    same(total.cpu(), [loss.double().sum().item()], 1e-12 * np.abs(L).sum() + 1e-300, "sum")
    got = dz.float().cpu().numpy()
    for t in range(T):
        for s in range(B):
            if not counts[t, s]:
                assert not got[t, s].any()
                continue
            f = w[s % P] * scale / n[s]
            tol = gradient_tol(z[t, s], y[t, s], f * g[s % P], f * curve * dr[s % P] + F32 * abs(f * g[s % P]), 1.0, dtype, D[t, s])
            same(got[t, s], D[t, s], tol, ("dlogits", t, s))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind,smoothing", [("logistic", 0.0), ("logistic", 0.1), ("logistic", 0.5), ("squared", 0.0), ("hinge", 0.0)])
@pytest.mark.parametrize("mean", [False, True])
def test_preference_kinds(kind, smoothing, mean, dtype):
    d, z, y, rng = draw_preference(7, 3, 501, dtype, 21)
    ref = rng.normal(size=6).astype(np.float32) * 3
    check_preference(d, z, y, ref, None, dtype, kind, 0.2, smoothing, mean)
    check_preference(d, z, y, None, rng.random(3).astype(np.float32), dtype, kind, 0.02, smoothing, mean, in_place=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,P,V", [(1, 1, 1), (1, 1, 2), (1, 1, 9), (2, 1, 40000), (3, 2, 64007), (64, 1, 33), (65, 2, 100), (200, 1, 50), (5, 37, 130), (3, 1, 204811),
                                   (20, 8, 2048), (129, 1, 3001), (2, 300, 17)])
def test_preference_sizes(T, P, V, dtype):
    d, z, y, rng = draw_preference(T, P, V, dtype, T + V)
    ref = (A.preference(z, y)[1] + rng.normal(size=2 * P)).astype(np.float32)
    check_preference(d, z, y, ref, None, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["front", "offset", "lowest"])
@pytest.mark.parametrize("V", [50, 30000])
def test_preference_rows_of_all_kinds(kind, V, dtype):
    d, z, y, rng = draw_preference(4, 2, V, dtype, 9, kind=kind)
    ref = (A.preference(z, y)[1] + rng.normal(size=4)).astype(np.float32)
    check_preference(d, z, y, ref, None, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,P,mean", [(1025, 2, False), (2500, 1, True)])
def test_preference_long_texts(T, P, mean, dtype):
    d, z, y, rng = draw_preference(T, P, 9, dtype, T)
    ref = (A.preference(z, y, mean=mean)[1] + rng.normal(size=2 * P)).astype(np.float32)
    check_preference(d, z, y, ref, None, dtype, mean=mean)
    alone = binding.rnnlm_preference_loss(d, gpu(y, torch.int32), gpu(ref), mean=mean)
    both = binding.rnnlm_preference_loss(d, gpu(y, torch.int32), gpu(ref), mean=mean, dlogits=torch.empty_like(d))
    assert all(torch.equal(a, b) for a, b in zip(alone, both))


def test_preference_texts_that_do_not_count():
    d, z, y, rng = draw_preference(6, 4, 90, "fp32", 31)
    w = np.array([1.0, 0.0, 0.5, 2.0], np.float32)
    y[:, 0] = -1  # an empty text
    y[:, [3, 7]] = -1  # a pair of empty texts
    y[2, 2] = 90  # out of range
    d[:, [1, 5]] = float("nan")  # pair 1 has no weight
    d[:, 0] = float("inf")
    z = d.cpu().numpy().astype(np.float64)
    check_preference(d, z, y, rng.normal(size=8).astype(np.float32), w, "fp32")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.rnnlm_preference_loss(d, gpu(y, torch.int32), weight=gpu(w), range_flag=flag)
    assert flag.item() == 1


def test_preference_words_without_probability():
    d, z, y, _ = draw_preference(3, 2, 40, "fp32", 33, ragged=False)
    d[1, 0, y[1, 0]] = -float("inf")  # a masked word of the preferred text
    dz = torch.empty(3, 4, 40, device="cuda")
    loss, logp = binding.rnnlm_preference_loss(d, gpu(y, torch.int32), dlogits=dz)
    assert loss[0].item() == np.inf and logp[0].item() == -np.inf and np.isfinite(loss[1].item())
    assert not dz[1, 0].any() and bool(dz[0, 0].isfinite().all()) and dz[0, 0].any()
    # the slope is at its end: -beta
    assert abs(dz[0, 0, y[0, 0]].item() + 0.1 * (1 - A.softmax(z[0, 0])[y[0, 0]])) < 1e-6


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["logistic", "squared", "hinge"])
@pytest.mark.parametrize("T", [3, 140])
def test_preference_of_two_texts_without_probability(T, kind, dtype):
    """r is no number where both texts of a pair hold a masked word, or their references are infinite: so are the pair's loss and
    its gradient, but for the masked words' rows."""
    d, z, y, _ = draw_preference(T, 3, 40, dtype, 34, ragged=False)
    for t, s in ((1, 0), (2, 3)):  # pair 0
        d[t, s, y[t, s]] = -float("inf")
        z[t, s, y[t, s]] = -np.inf
    ref = np.array([0.0, np.inf, 1.0, 0.5, np.inf, 0.0], np.float32)  # pair 1
    which = dict(logistic=binding.RNNLM_PREFERENCE_LOGISTIC, squared=binding.RNNLM_PREFERENCE_SQUARED, hinge=binding.RNNLM_PREFERENCE_HINGE)[kind]
    dz = torch.full_like(d, 7.0)
    loss, logp = binding.rnnlm_preference_loss(d, gpu(y, torch.int32), gpu(ref), kind=which, dlogits=dz)
    L, S, D, _, _ = A.preference(z, y, ref, kind=kind, beta=float(np.float32(0.1)))
    assert np.isnan(L[:2]).all() and np.isfinite(L[2]) and np.isnan(D[:, [1, 4]]).all()
    assert loss[:2].isnan().all() and loss[2].isfinite() and torch.equal(logp.isinf().cpu(), torch.as_tensor(np.isinf(S)))
    got = dz.float().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(D)) and not got[1, 0].any() and not got[2, 3].any()
    assert np.isfinite(got[:, [2, 5]]).all()


@pytest.mark.parametrize("V", [64, 4097])
def test_preference_loss_alone_agrees(V):
    d, z, y, rng = draw_preference(9, 5, V, "bf16", 8)
    both = binding.rnnlm_preference_loss(d, gpu(y, torch.int32), dlogits=torch.empty(9, 10, V, dtype=torch.bfloat16, device="cuda"))
    alone = binding.rnnlm_preference_loss(d, gpu(y, torch.int32))
    L, S, _, _, _ = A.preference(z, y, beta=float(np.float32(0.1)))
    for loss, logp in (both, alone):
        same(logp.cpu(), S, 9 * row_err(z.reshape(-1), 1.0) + F32 * np.abs(S), "logp")
        same(loss.cpu(), L, 0.1 * 18 * row_err(z.reshape(-1), 1.0) + F32 * np.abs(L), "loss")


@pytest.mark.parametrize("dtype,T,P,V,in_place", [("fp32", 3, 4, 700001, False), ("bf16", 20, 9, 100003, False), ("bf16", 64, 1, 300001, True), ("fp32", 1, 150, 60000, False),
                                                  ("bf16", 5, 700, 5001, False), ("fp32", 40, 30, 7001, True), ("bf16", 2, 60, 160001, False)])
@pytest.mark.parametrize("polls", [256, 0])
def test_preference_rows_that_meet(dtype, T, P, V, in_place, polls):
    """Many large rows: workgroups wait for their pair's, or (no polls) leave their gradients to a second pass; the same bits as
    text by text, where rows are few."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    z = torch.empty(T, 2 * P, V, dtype=DTYPES[dtype], device="cuda").normal_(0.0, 2.0, generator=gen)
    y = torch.randint(0, V, (T, 2 * P), generator=gen, device="cuda", dtype=torch.int32)
    if T > 1:
        y[torch.rand(T, 2 * P, generator=gen, device="cuda") < 0.2] = -1
    y[0, 0] = -1
    z[0, 0] = float("nan")
    z[-1, 1, int(y[-1, 1])] = -float("inf")  # a masked word (where it counts)
    ref, w = torch.randn(2 * P, generator=gen, device="cuda"), torch.rand(P, generator=gen, device="cuda")
    w[P - 1] = 0.0 if P > 2 else 1.0
    parts = []
    for p in range(P):  # a pair at a time: too few rows to meet (or, of one pair, read in halves of its words' order)
        two = z[:, [p, P + p]].contiguous()
        d = torch.empty_like(two)
        loss, logp = binding.rnnlm_preference_loss(two, y[:, [p, P + p]].contiguous(), ref[[p, P + p]].contiguous(), w[p: p + 1].contiguous(), beta=0.3, smoothing=0.1,
                                                   mean=True, scale=0.7, dlogits=d)
        parts.append((loss, logp, d))
    try:
        binding.rnnlm_set_preference_wait(polls)
        dz = z if in_place else torch.full_like(z, 5.0)
        total = torch.zeros(1, dtype=torch.float64, device="cuda")
        loss, logp = binding.rnnlm_preference_loss(z, y, ref, w, beta=0.3, smoothing=0.1, mean=True, scale=0.7, dlogits=dz, sum_loss=total)
        torch.cuda.synchronize()
    finally:
        binding.rnnlm_set_preference_wait(256)
    # sums of a row's exponentials may be formed in another order: E of the logarithms, as above
    E = 2 * row_err(np.full(V, 12.0), 1.0)
    for p, (l, s, d) in enumerate(parts):
        for got, want, scale in ((loss[p], l[0], 1.0), (logp[p], s[0], 1.0), (logp[P + p], s[1], 1.0)):
            assert got.item() == want.item() or abs(got.item() - want.item()) <= E * scale + 2 * F32 * abs(want.item()), p
        got, want = dz[:, [p, P + p]].float(), d.float()
        top = want.abs().amax(2, keepdim=True)
        assert bool(((got - want).abs() <= 2 * HALF[dtype] * want.abs() + 4 * E * want.abs() + E * top + 2.0 ** -126).all()), p
        zero = (y[:, [p, P + p]] < 0) | (w[p] == 0)
        assert not got[zero].any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_preference_waits_leave_no_mark(dtype):
    """Rows that met and rows that did not wait have the same bits, and so do calls that share the GPU: on two streams at once."""
    T, P, V = 20, 40, 40000
    gen = torch.Generator(device="cuda").manual_seed(3)
    z = [torch.empty(T, 2 * P, V, dtype=DTYPES[dtype], device="cuda").normal_(0.0, 2.0, generator=gen) for _ in range(2)]
    z[1][3, 5, : V // 2] = -float("inf")  # (a row whose sum is formed by way of memory)
    y = torch.randint(V // 2, V, (T, 2 * P), generator=gen, device="cuda", dtype=torch.int32)
    y[torch.rand(T, 2 * P, generator=gen, device="cuda") < 0.2] = -1
    want = []
    for a in z:
        d = torch.empty_like(a)
        want.append((*binding.rnnlm_preference_loss(a, y, dlogits=d), d))
    try:
        binding.rnnlm_set_preference_wait(0)
        for a, w in zip(z, want):
            d = torch.empty_like(a)
            got = (*binding.rnnlm_preference_loss(a, y, dlogits=d), d)
            assert all(torch.equal(p, q) for p, q in zip(got, w))
        torch.cuda.synchronize()
    finally:
        binding.rnnlm_set_preference_wait(256)
    streams = [torch.cuda.Stream() for _ in z]
    nbytes = binding.rnnlm_preference_workspace_bytes(T, P)
    outs = [(torch.empty(P, device="cuda"), torch.empty(2 * P, device="cuda"), torch.empty_like(a), torch.empty(nbytes, dtype=torch.uint8, device="cuda")) for a in z]
    torch.cuda.synchronize()
    for _ in range(5):
        for a, stream, (loss, logp, d, ws) in zip(z, streams, outs):
            binding.rnnlm_preference_loss(a, y, loss=loss, logp=logp, dlogits=d, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    for got, w in zip(outs, want):
        assert all(torch.equal(p, q) for p, q in zip(got, w))


def test_more_than_two_to_the_31_logits():
    """The last rows of calls of 2^22 - 64 rows: the bits of the same rows by themselves, and the words' logarithms."""
    V, T, P = 600, 32, 65535
    z = torch.empty(T, 2 * P, V, dtype=torch.bfloat16, device="cuda").normal_(0.0, 2.0, generator=torch.Generator(device="cuda").manual_seed(1))
    assert z.numel() > 1 << 31 and T * 2 * P == (1 << 22) - 64
    gen = torch.Generator(device="cuda").manual_seed(2)
    y = torch.randint(0, V, (T, 2 * P), generator=gen, device="cuda", dtype=torch.int32)
    adv = torch.randn(T, 2 * P, generator=gen, device="cuda")
    d = torch.empty_like(z)
    loss, logp = binding.rnnlm_policy_loss(z, y, adv, dlogits=d)
    few = [t.view(T * 2 * P, *t.shape[2:])[-2000:] for t in (z, y, adv, d, loss, logp)]
    d2 = torch.empty_like(few[0])
    loss2, logp2 = binding.rnnlm_policy_loss(few[0], few[1], few[2], dlogits=d2)
    assert torch.equal(d2, few[3]) and torch.equal(loss2, few[4]) and torch.equal(logp2, few[5])
    want = torch.log_softmax(few[0].double(), 1).gather(1, few[1].long()[:, None])[:, 0]
    E = row_err(np.full(V, few[0].abs().max().item()), 1.0)
    same(logp2.cpu(), want.cpu().numpy(), E + F32 * want.abs().cpu().numpy(), "logp")
    pairs, S = binding.rnnlm_preference_loss(z, y, dlogits=d)
    last = [torch.cat([t[:, P - 100: P], t[:, 2 * P - 100:]], 1).contiguous() for t in (z, y, d)]
    d2 = torch.empty_like(last[0])
    pairs2, S2 = binding.rnnlm_preference_loss(last[0], last[1], dlogits=d2)
    assert torch.equal(d2, last[2]) and torch.equal(pairs2, pairs[-100:]) and torch.equal(S2, torch.cat([S[P - 100: P], S[-100:]]))


def test_preference_of_no_positions():
    d = torch.empty(0, 6, 30, device="cuda")
    y = torch.empty(0, 6, dtype=torch.int32, device="cuda")
    ref = torch.tensor([1.0, 2.0, 3.0, 0.0, 0.0, 0.0], device="cuda")
    loss, logp = binding.rnnlm_preference_loss(d, y, ref, kind=binding.RNNLM_PREFERENCE_HINGE, beta=0.5)
    assert logp.tolist() == [0.0] * 6 and loss.tolist() == [1.5, 2.0, 2.5]


# ---- both: streams, graphs, workspaces ----------------------------------------------------------------------------------
def test_a_captured_call_of_each_replays():
    d, z, y, rng = draw_preference(5, 6, 3000, "bf16", 40, ragged=False)
    yd, adv = gpu(y, torch.int32), gpu(rng.normal(size=y.shape).astype(np.float32))
    ws = torch.empty(binding.rnnlm_preference_workspace_bytes(5, 6), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(d) for _ in range(2)]
    a, l, b, s = (torch.empty(n, device="cuda") for n in (60, 60, 6, 12))
    a, l = a.view(5, 12), l.view(5, 12)

    def calls():
        binding.rnnlm_policy_loss(d, yd, adv, loss=a, logp=l, dlogits=outs[0])
        binding.rnnlm_preference_loss(d, yd, loss=b, logp=s, dlogits=outs[1], workspace=ws)
    calls()
    want = [t.clone() for t in (*outs, a, l, b, s)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        for t in (*outs, a, l, b, s):
            t.fill_(5.0)
        ws.fill_(i * 77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip((*outs, a, l, b, s), want))
        d.copy_(d.clone())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = binding.rnnlm_preference_loss(d, yd, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got[0], want[4]) and torch.equal(got[1], want[5])
