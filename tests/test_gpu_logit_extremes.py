"""The operators on arrays of logits where numbers are at their ends: rows far from zero, rows of fewer words than a load
holds, NaNs of either kind, sums near the end of the type's range.  Against the fp64 oracle (oracle/logits.py) or values known
by hand.

Tolerances.  A row's results do not change when all of its logits move, and neither do these bounds: D is how far a word lies
below the row's greatest, over tau.  An exponential's argument is rounded a few times at the size of D, the hardware's exponential
is off by a unit (2^-23), so it is off by 2^-24 (4 D + 16) relative; a thread adds at most 26 * 8 + 1 terms one after the other, a
tree of at most 6 + 16 sums follows, and ten more roundings: SUM.  A logarithm of such a sum has that as an absolute error.
Outputs are rounded once: eps / 2 of their type."""
import numpy as np
import pytest
import torch

from oracle import logits as L
from paper_1502_00512_amd import binding

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
SUM = (26 * 8 + 1 + 22 + 10) * U


def cuda(a, dtype=None):
    return None if a is None else torch.as_tensor(np.ascontiguousarray(a, dtype)).cuda()


def rows_of(z, dtype):
    """The rows on the GPU and their values, which the type holds exactly."""
    d = cuda(z, np.float64).to(DTYPES[dtype])
    assert np.array_equal(d.double().cpu().numpy(), z)
    return d


def reach(z, tau):
    """D of every word, and the error of the row's ln of its sum."""
    D = np.where(np.isneginf(z), 0.0, (z.max() - z) / tau)
    return D, SUM + U * (L.softmax(z, tau) * (4 * D + 16)).sum()


def check_distill(z, ids, vals, y, dtype, tau, alpha, n=None, scale=2.0 ** -13, grad=True, at=0.0, teacher_at=0.0):
    """One call over the rows z against the oracle.  n: the teacher's lse [rows] (fp32 values) or None.  at, teacher_at: what the
    rows and the lists (n = None) have in common, which changes nothing and which the oracle does without (far enough from zero its 64 bits hold no difference of logits either)."""
    rows, V = z.shape
    tau = float(np.float32(tau))
    d = rows_of(z, dtype)
    out = torch.full((rows, V), 7.0, dtype=d.dtype, device="cuda") if grad else None
    loss = binding.rnnlm_distill_loss(d, cuda(ids, np.int32), cuda(vals, np.float32), cuda(n, np.float32), cuda(y, np.int32), None, tau, alpha,
                                      scale, dlogits=out).double().cpu().numpy()
    g = out.double().cpu().numpy() if grad else None
    half = torch.finfo(DTYPES[dtype]).eps / 2
    a32 = float(np.float32(alpha))
    z, vals = z - at, vals.astype(np.float64) - teacher_at
    for r in range(rows):
        yr = -1 if y is None else int(y[r])
        nr = None if n is None else float(np.float32(n[r]))
        want, gr = L.distill(z[r], ids[r], vals[r], nr, yr, 1.0, tau, a32, scale)
        there = ids[r] >= 0
        t = vals[r][there] / tau
        norm = L.lse(t) if nr is None else nr
        p, spread = np.exp(t - norm), (t.max() - t) if len(t) else t
        # e^(t - t_max), its sum and the factor in front of it
        p_err = U * (4 * spread.max(initial=0.0) + 16 + 2 * (abs(t.max(initial=norm) - norm) if nr is not None else len(t)))
        D, ln_err = reach(z[r], tau)
        D1, ln_err1 = reach(z[r], 1.0)
        gap = np.abs(t - norm) + np.abs(z[r][ids[r][there]] / tau - L.lse(z[r], tau))
        tol = a32 * tau * tau * (p * (gap * p_err + ln_err)).sum()
        tol += (1 - a32) * ln_err1 if yr >= 0 else 0.0
        tol += 2 * U * abs(want) + 2.0 ** -40
        assert abs(loss[r] - want) <= tol, (r, loss[r], want, tol)
        if g is None:
            continue
        mass = np.zeros(V)
        np.add.at(mass, ids[r][there], p)
        size = a32 * tau * (p.sum() * L.softmax(z[r], tau) * (ln_err + p_err + U * (4 * D + 32)) + mass * (p_err + 8 * U))
        if yr >= 0 and a32 < 1:
            size += (1 - a32) * L.softmax(z[r]) * (ln_err1 + U * (8 * D1 + 32))
            size[yr] += 8 * U
        bound = scale * size + half * np.abs(gr) * (1 + 2.0 ** -9) + 1e-37
        bad = ~(np.abs(g[r] - gr) <= bound)
        assert not bad.any(), (r, np.nonzero(bad)[0][:5], g[r][bad][:5], gr[bad][:5], bound[bad][:5])
        if nr is None and alpha == 1.0 and dtype == "fp32":  # what the list takes off is what the row adds
            assert abs(g[r].sum()) <= scale * 2 * tau * (ln_err + p_err + 64 * U), g[r].sum()


# ---- rows far from zero -----------------------------------------------------------------------------------------------
def far_rows(rows, V, at, step, seed):
    """Logits around `at` in whole steps, which the type holds there."""
    rng = np.random.default_rng(seed)
    return at + step * np.round(rng.normal(0.0, 2.0, (rows, V)) / step)


def far_lists(rows, V, K, at, step, seed):
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.permutation(V)[:K] for _ in range(rows)])
    return ids, (at + step * np.round(rng.normal(0.0, 2.0, (rows, K)) / step)).astype(np.float32), rng.integers(0, V, rows)


FAR = [("fp32", 2.0 ** 14, 2.0 ** -9), ("fp32", -2.0 ** 14 + 32, 2.0 ** -10), ("fp32", 2.0 ** 20, 0.125), ("fp32", 2.0 ** 21, 0.25), ("fp32", -2.0 ** 23 + 64, 0.5),
       ("bf16", 256.0, 2.0), ("bf16", 2.0 ** 14, 128.0)]


@pytest.mark.parametrize("dtype,at,step", FAR)
@pytest.mark.parametrize("rows,V", [(3, 1203), (1030, 200), (2, 20011), (2, 70001)])
def test_distill_gradients_of_rows_far_from_zero(rows, V, dtype, at, step):
    z = far_rows(rows, V, at, step, V)
    ids, vals, y = far_lists(rows, V, 9, 0.0, 0.125, 1)
    d = rows_of(z, dtype)
    half = torch.finfo(DTYPES[dtype]).eps / 2
    for tau, alpha in ((1.0, 0.5), (1.5, 1.0), (2.0, 0.5), (1.5, 0.5), (0.7, 0.5)):
        tau = float(np.float32(tau))
        out = torch.empty_like(d)
        binding.rnnlm_distill_loss(d, cuda(ids, np.int32), cuda(vals), None, cuda(y, np.int32), None, tau, alpha, dlogits=out)
        got = out.double().cpu().numpy()
        for r in range(min(rows, 5)):
            _, g = L.distill(z[r], ids[r], vals[r], None, int(y[r]), 1.0, tau, alpha)
            D, err = reach(z[r], tau)
            D1, err1 = reach(z[r], 1.0)
            t = vals[r].astype(np.float64) / tau
            p_err = U * (4 * (t.max() - t.min()) + 16 + 2 * len(t) + 4 * np.abs(t).max())
            bound = alpha * tau * L.softmax(z[r], tau) * (err + p_err + U * (4 * D + 32)) + (1 - alpha) * L.softmax(z[r]) * (err1 + U * (8 * D1 + 32))
            np.add.at(bound, ids[r], alpha * tau * L.softmax(t) * (p_err + 8 * U))
            bound[y[r]] += (1 - alpha) * 8 * U
            bound += half * np.abs(g) * (1 + 2.0 ** -9)
            bad = ~(np.abs(got[r] - g) <= bound)
            assert not bad.any(), (tau, alpha, r, np.nonzero(bad)[0][:5], got[r][bad][:5], g[bad][:5], bound[bad][:5])
            if alpha == 1.0 and dtype == "fp32":
                assert abs(got[r].sum()) <= 2 * tau * (err + p_err + 64 * U)


@pytest.mark.parametrize("dtype,at,step", FAR)
@pytest.mark.parametrize("rows,V", [(3, 1203), (2, 20011)])
@pytest.mark.parametrize("grad", [True, False])
def test_distill_losses_of_rows_far_from_zero(rows, V, grad, dtype, at, step):
    """Students' and teachers' rows, each as far from zero as it likes: the losses do not change."""
    z = far_rows(rows, V, at, step, V)
    for teacher_at in (0.0, 2.0 ** 12, -2.0 ** 17):
        ids, vals, y = far_lists(rows, V, 9, teacher_at, 0.125, 1)
        for tau, alpha in ((1.0, 0.5), (1.5, 1.0), (2.0, 0.5), (0.7, 0.0)):
            check_distill(z, ids, vals, y, dtype, tau, alpha, grad=grad)
            n = np.float32(np.float64(vals.max(1)) / np.float32(tau) + 0.75)
            check_distill(z, ids, vals, y, dtype, tau, alpha, n, grad=grad)


@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_a_list_of_far_logits_at_the_lowest_temperature(dtype):
    """Logits of 4096 over 0.001: a list's probabilities hang on differences, not on what they are taken from."""
    z = far_rows(2, 1203, 0.0, 0.5, 3)
    ids, vals, y = far_lists(2, 1203, 6, 4096.0, 2.0 ** -10, 4)
    vals = (4096.0 + np.arange(6)[None] * 2.0 ** -10).repeat(2, 0).astype(np.float32)
    check_distill(z, ids, vals, y, dtype, 1e-3, 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [9, 1203, 20011])
@pytest.mark.parametrize("at", [-2.0 ** 40, 2.0 ** 60, -2.0 ** 127])
def test_distill_losses_of_rows_beyond_64_bits(at, V, dtype):
    """Half a row is masked, the others are equal: the losses hang on how many there are, whatever they are."""
    z = np.full((2, V), at)
    z[:, V // 2 + 1:] = -np.inf
    ids, y = np.array([[0, 1, V // 2], [1, 0, V // 2]]), np.array([1, V // 2])
    for teacher_at in (0.0, at):
        vals = np.full((2, 3), teacher_at, np.float32)
        vals[1, 0] = -np.inf
        ids[1, 0] = -1
        for tau, alpha in ((1.0, 0.5), (1.5, 1.0), (2.0, 0.5), (0.7, 0.0)):
            for grad in (True, False):
                check_distill(z, ids, vals, y, dtype, tau, alpha, grad=grad, at=at, teacher_at=teacher_at)


@pytest.mark.parametrize("dtype,at,step", FAR)
@pytest.mark.parametrize("V", [5, 1203, 20011, 70001, 200003])
def test_top_logits_sums_of_rows_far_from_zero(V, dtype, at, step):
    """The logarithm of the sum is rounded once, at its own size."""
    z = far_rows(2, V, at, step, V)
    z[1, : V // 2] = -np.inf
    d = cuda(z).to(DTYPES[dtype])
    for tau in (1.0, 1.3, 1.5, 0.7, 3.5, 0.03, 150.0):
        tau = float(np.float32(tau))
        lse = binding.rnnlm_top_logits(d, 2, tau)[2].double().cpu().numpy()
        for r in range(2):
            want = L.lse(z[r], tau)
            assert abs(lse[r] - want) <= U * abs(want) * (1 + 2.0 ** -8) + reach(z[r], tau)[1], (tau, r, lse[r], want)


# ---- rows of fewer words than a load holds ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 2, 3, 7, 9])
@pytest.mark.parametrize("at", [-2.0 ** 23, -2.0 ** 40, -2.0 ** 127, 2.0 ** 23])
def test_distill_of_a_few_words_far_from_zero(at, V, dtype):
    z = np.full((3, V), at)
    z[1] += np.arange(V) % 2 * (2.0 ** 16 if dtype == "bf16" else 1.0) if abs(at) == 2.0 ** 23 else 0.0  # (whole steps of the type)
    z[2, V // 2:] = z[2].max()
    ids, vals, y = np.arange(2)[None].repeat(3, 0) % V, np.array([[0.0, 1.0]] * 3, np.float32), np.array([0, V - 1, -1])
    for tau, alpha in ((1.0, 0.5), (2.0, 0.5), (4.0, 0.25), (2.0, 1.0)):
        for grad in (True, False):
            check_distill(z, ids, vals, y, dtype, tau, alpha, grad=grad, at=at)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 3, 7])
def test_distill_of_a_few_words_at_the_lowest_temperature(V, dtype):
    """-2^13 / 0.001 is beyond the references' range: every word has 1 / V (the loss at tau is tested with the rows far from zero)."""
    z = torch.full((2, V), -(2.0 ** 13), dtype=DTYPES[dtype], device="cuda")
    out = torch.empty_like(z)
    ids = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    loss = binding.rnnlm_distill_loss(z, ids, torch.zeros(2, 1, device="cuda"), tau=1e-3, dlogits=out)
    tau = float(np.float32(1e-3))
    want = np.full(V, tau / V)
    want[0] -= tau
    assert np.abs(out.double().cpu().numpy() - want).max() <= tau * (2.0 ** -9 if dtype == "bf16" else 64 * U)
    assert bool(torch.isfinite(loss).all())


# ---- NaNs of either kind ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,K", [(7, 3), (300, 40), (2050, 256), (5000, 40), (20011, 256), (70001, 64), (150001, 200), (400003, 20)])
def test_top_logits_of_rows_that_hold_signalling_nans(V, K, dtype):
    """They rank as masked words do, wherever in a load they stand: behind the greatest words, in front of them, or anywhere."""
    rng = np.random.default_rng(V)
    z = rng.normal(0.0, 3.0, (4, V))
    if dtype == "bf16":
        z = torch.as_tensor(z).to(torch.bfloat16).double().numpy()
    else:
        z = z.astype(np.float32).astype(np.float64)
    nan = rng.random((4, V)) < 0.02
    great = np.argsort(-z, 1)[:, : K + 5]
    for r, step in ((0, 1), (1, -1)):
        nan[r, np.clip(great[r] + step, 0, V - 1)] = True
        nan[r, great[r]] = False
    nan[2] = rng.random(V) < 0.3
    nan[3] = True
    nan[3, great[3][:2]] = False  # fewer numbers than asked for
    d = torch.as_tensor(z).to(DTYPES[dtype])
    bits = d.view(torch.int32 if dtype == "fp32" else torch.int16).clone()
    pos, neg = (0x7f800001, 0xff812345 - 2 ** 32) if dtype == "fp32" else (0x7f81, 0xff83 - 2 ** 16)
    bits[torch.as_tensor(nan)] = pos
    bits[torch.as_tensor(nan & (rng.random((4, V)) < 0.5))] = neg
    d = bits.cuda().view(DTYPES[dtype])
    ids, vals, lse = binding.rnnlm_top_logits(d, K)
    assert torch.isnan(lse).tolist() == nan.any(1).tolist()
    z[nan] = -np.inf
    for r in range(4):
        i, v, _ = L.top(z[r], K)
        assert np.array_equal(ids[r].cpu().numpy(), i), (r, np.nonzero(ids[r].cpu().numpy() != i)[0][:5])
        assert np.array_equal(vals[r].double().cpu().numpy(), v)


# ---- sums near the end of the range -----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V", [(2, 5008), (1030, 1008), (2, 70008)])
def test_distill_of_a_row_whose_great_words_come_late(rows, V, dtype):
    """The first words are 60 below the last ones: at tau = 2 sums of exponentials and of their squares relative to the first are
    some 2^45 and 2^88, and the gradient of the labels a quotient by them, at a small factor."""
    z = np.zeros((rows, V))
    z[:, V - 3:] = 60.0
    ids, vals = np.stack([[V - 1, 5, V - 2]] * rows), np.array([[1.0, 0.5, 0.25]] * rows, np.float32)
    y = np.full(rows, V - 3)
    for tau, alpha in ((2.0, 0.5), (2.0, 0.0), (1.0, 0.5), (1.5, 0.5)):
        check_distill(z[:3], ids[:3], vals[:3], y[:3], dtype, tau, alpha, scale=2.0 ** -60)
        if rows > 3:
            check_distill(z, ids, vals, y, dtype, tau, alpha, scale=2.0 ** -60)




@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("slots", [512, 2560, 8192, 16384, 25600])
def test_sums_of_waves_that_are_in_range_and_their_sum_is_not(slots, dtype):
    """Two words of 87.5 for every wave of a workgroup, behind its first loads: 2^127.2 a wave, more than the type holds together."""
    n = 4 if dtype == "fp32" else 8
    for threads in (256, 512, 1024):
        if slots < 2 * threads:
            continue
        z = np.zeros((2, slots * n))
        for wave in range(threads // 64):
            first = (threads + wave * 64) * n
            z[:, first: first + 2] = 87.5
        ids, vals, y = np.array([[3, threads * n]] * 2), np.array([[0.0, 1.0]] * 2, np.float32), np.array([threads * n + 1, 0])
        for tau, alpha in ((1.0, 0.5), (1.0, 1.0)):
            check_distill(z, ids, vals, y, dtype, tau, alpha)
        z2 = 2.0 * z  # (tau = 2: the same exponentials, their squares out of range)
        check_distill(z2, ids, vals, y, dtype, 2.0, 1.0)
        for rows, tau in ((z, 1.0), (z2, 2.0)):
            lse = binding.rnnlm_top_logits(rows_of(rows, dtype), 5, tau)[2].double().cpu().numpy()
            want = 87.5 + np.log(threads // 32)
            assert np.abs(lse - want).max() <= U * want + SUM, (threads, lse, want)


# ---- verification at temperatures far below a step of the logits ------------------------------------------------------
@pytest.mark.parametrize("V", [5, 1001, 20011, 100003])
@pytest.mark.parametrize("at", [1.5 * 2.0 ** 23, -1.5 * 2.0 ** 23, 1.5 * 2.0 ** 22, 2.0 ** 20, 1000.0])
def test_verify_where_a_step_of_the_type_is_many_temperatures(at, V):
    """tau = 0.001 and fp32 logits whose neighbours lie 1, 0.5, 0.125, 2^-14 apart: a step is hundreds of tau, or none."""
    rng = np.random.default_rng(V)
    step = float(np.spacing(np.float32(abs(at))))
    K, B = 2, 4
    target = at - step * rng.integers(0, 4, (K + 1, B, V))
    target[:, :, rng.integers(0, V, 3)] = at
    draft = target[:K] - step * (rng.random((K, B, V)) < 0.5)
    draft[:, :, 0] = at
    drafts = np.array([[rng.choice(np.nonzero(draft[i, b] == at)[0]) for b in range(B)] for i in range(K)])
    u = rng.random((K + 1, B)).astype(np.float32)
    tau = float(np.float32(1e-3))
    for q in (draft, None):
        n, tokens = binding.rnnlm_verify_drafts(rows_of(target, "fp32"), cuda(drafts, np.int32), cuda(u), None if q is None else rows_of(q, "fp32"),
                                                None, tau, tau)
        for b in range(B):
            want = L.verify(target[:, b], drafts[:, b], u[:, b], None if q is None else q[:, b], None, tau, tau)
            assert int(n[b]) == want[0] and tokens[:, b].tolist() == want[1].tolist(), (b, int(n[b]), tokens[:, b], want)
