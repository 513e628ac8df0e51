"""The operators on arrays of logits, through the binding, against the fp64 oracle (oracle/logits.py).

Tolerances.  An exponential e^{(z - m) / tau} is 2^t with t = z c + b in fp32: c, b and the sum are each rounded, |z| and |m|
over tau at most Z, so |dt| <= 2^-24 * 4 Z log2 e and the exponential is off by at most 2^-24 * 4 Z relative, plus one unit
(2^-23) of the hardware's exponential.  A thread adds at most 26 * 8 + 1 terms one after the other (2^-24 each), a tree of at
most 6 + 16 sums follows, and rescaling a running sum costs another rounding each 32 terms: SUM below.  A logarithm of such a
sum has that as an absolute error.  Outputs are rounded once: eps / 2 of their type."""
import numpy as np
import pytest
import torch

from oracle import logits as L
from paper_1502_00512_amd import binding

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SUM = (26 * 8 + 1 + 22 + 2 + 8) * 2.0 ** -24  # relative error of a sum of positive terms, apart from its terms'


def row_err(z, tau):
    """Bound of the error of a row's lse, and relative error of a softmax value of it."""
    z = z[np.isfinite(z)]
    Z = np.abs(z).max() / tau if len(z) else 0.0
    return SUM + 2.0 ** -24 * (8 * Z + 4)


def place(z, dtype, pad=0):
    """The rows on the GPU, pad elements of NaN between them; and their values as the type holds them."""
    rows, V = z.shape
    buf = torch.full((rows, V + pad), float("nan"), dtype=DTYPES[dtype], device="cuda")
    buf[:, :V] = torch.as_tensor(z)
    return buf[:, :V], buf[:, :V].float().cpu().numpy().astype(np.float64)


def patterns(kind, rows, V, seed):
    rng = np.random.default_rng(seed)
    z = rng.normal(0.0, 3.0, (rows, V))
    if kind == "equal":
        z[:] = 1.5
    elif kind == "masked":
        z[:] = -np.inf
    elif kind == "few":  # fewer words than asked for
        z[rng.random((rows, V)) < 0.98] = -np.inf
    elif kind == "rising":
        z = np.sort(z, 1)
    elif kind == "falling":
        z = -np.sort(-z, 1)
    elif kind == "ties":
        z = np.round(z)
    elif kind == "zeros":
        z = np.where(rng.random((rows, V)) < 0.5, 0.0, -0.0)
    elif kind == "nan":
        z[rng.random((rows, V)) < 0.05] = np.nan
    elif kind == "infinite":
        z[:, V // 2] = np.inf
    elif kind == "clustered":  # all the large ones next to each other
        z[:, : min(V, 300)] += 40.0
    elif kind == "steep":  # far apart: later words dwarf the earlier ones
        z = np.linspace(-200.0, 250.0, V)[None] + z
    elif kind == "offset":  # far from zero altogether
        z += 3e4
    elif kind == "all lowest":  # a mask that leaves nothing, of the type's lowest value
        z[:] = -3e38
    elif kind == "huge":
        z *= 1e30
    elif kind == "lowest":  # masks of the type's lowest value
        z[rng.random((rows, V)) < 0.9] = -3e38
    return z


# ---- top logits -------------------------------------------------------------------------------------------------------
def check_top(z, K, tau, dtype, pad):
    d, ref = place(z, dtype, pad)
    ids, vals, lse = binding.rnnlm_top_logits(d, K, tau)
    ids, vals, lse = ids.cpu().numpy(), vals.cpu().numpy(), lse.cpu().numpy().astype(np.float64)
    for r in range(len(z)):
        i, v, n = L.top(ref[r], K, tau)
        assert np.array_equal(ids[r], i), (r, np.nonzero(ids[r] != i)[0][:5])
        assert np.array_equal(vals[r].astype(np.float64), v)
        if np.isfinite(n):
            assert abs(lse[r] - n) <= row_err(ref[r], tau) + 2.0 ** -24 * abs(n), (lse[r], n)
        else:
            assert np.array_equal(lse[r], n, equal_nan=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V,K,pad", [(1, 1, 1, 0), (3, 2, 2, 1), (2, 7, 3, 0), (5, 8, 8, 3), (4, 9, 1, 0), (3, 100, 100, 5),
                                          (40, 1000, 17, 0), (2, 4097, 256, 1), (1, 33278, 100, 0), (600, 1500, 256, 7), (2, 70001, 64, 0)])
def test_top_logits_sizes(rows, V, K, pad, dtype):
    check_top(patterns("normal", rows, V, V + K), K, 1.3, dtype, pad)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["equal", "masked", "few", "rising", "falling", "ties", "zeros", "nan", "infinite", "clustered", "lowest", "steep", "offset", "all lowest", "huge"])
@pytest.mark.parametrize("V,K", [(300, 256), (5000, 40), (20011, 256)])
def test_top_logits_patterns(V, K, kind, dtype):
    check_top(patterns(kind, 3, V, 7), K, 1.0, dtype, 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["equal", "masked", "few", "ties", "nan", "clustered", "rising", "lowest"])
@pytest.mark.parametrize("slots,K", [(5001, 60), (9001, 256), (11001, 9), (18001, 256)])
def test_top_logits_of_wide_rows(slots, K, kind, dtype):
    check_top(patterns(kind, 2, slots * (4 if dtype == "fp32" else 8) - 3, 11), K, 1.0, dtype, 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["normal", "ties", "few"])
@pytest.mark.parametrize("V", [257, 500, 512, 513, 1000, 1031, 2047, 2050, 4099, 8200])
def test_top_logits_long_lists_of_short_rows(V, kind, dtype):
    for K in (64, 129, 256):
        check_top(patterns(kind, 3, V, V + K), K, 1.0, dtype, 1)


@pytest.mark.parametrize("dtype", DTYPES)
def test_top_logits_of_many_rows_in_one_chunk_and_of_the_widest_vocabulary(dtype):
    check_top(patterns("normal", 700, 9000, 1), 31, 0.7, dtype, 0)  # a chunk a row
    check_top(patterns("normal", 300, 45007 if dtype == "fp32" else 90007, 3), 20, 1.0, dtype, 0)  # chunks
    check_top(patterns("ties", 2, 1 << 20, 2), 256, 1.0, dtype, 0)
    check_top(patterns("clustered", 1, (1 << 20) - 3, 2), 256, 1.0, dtype, 1)


# ---- distillation -----------------------------------------------------------------------------------------------------
def lists(rows, V, K, seed, ragged):
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.permutation(V)[:K] if K <= V else rng.integers(0, V, K) for _ in range(rows)]).astype(np.int32)
    vals = rng.normal(0.0, 3.0, (rows, K)).astype(np.float32)
    y = rng.integers(0, V, rows).astype(np.int32)
    w = np.ones(rows, np.float32)
    if ragged:
        ids[rng.random((rows, K)) < 0.3] = -1
        ids[0] = -1  # no list at all
        if K > 2:
            ids[-1, 2] = ids[-1, 0]  # a word twice
            vals[-1, 1] = -np.inf
            y[-1] = max(ids[-1, 0], 0)  # and the label is on the list
        y[rng.random(rows) < 0.3] = -1
        w = rng.choice([0.0, 1.0, 0.5, -2.0], rows).astype(np.float32)
    return ids, vals, y, w


def check_distill(z, ids, vals, y, w, dtype, pad=0, tau=1.0, alpha=0.5, scale=0.125, own=True, grad="apart"):
    rows, V = z.shape
    d, ref = place(z, dtype, pad)
    cuda = lambda a: None if a is None else torch.as_tensor(a).cuda()  # noqa: E731
    n = None if own else np.array([L.lse(np.append(v / np.float64(tau), 0.5)) for v in vals.astype(np.float64)], np.float32)
    out = dict(apart=lambda: torch.full((rows, V + 3), 7.0, dtype=d.dtype, device="cuda")[:, :V], inplace=lambda: d, none=lambda: None)[grad]()
    total, flag = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    loss = binding.rnnlm_distill_loss(d, cuda(ids), cuda(vals), cuda(n), cuda(y), cuda(w), tau, alpha, scale, dlogits=out, sum_loss=total,
                                      range_flag=flag)
    got = loss.cpu().numpy().astype(np.float64)
    g = out.float().cpu().numpy().astype(np.float64) if out is not None else None
    w_ = np.ones(rows) if w is None else w
    eps = torch.finfo(DTYPES[dtype]).eps / 2
    for r in range(rows):
        if w_[r] == 0.0:
            assert got[r] == 0.0 and (g is None or (g[r] == 0.0).all())
            continue
        yr = -1 if y is None else int(y[r])
        nr = None if n is None else float(n[r])
        l, gr = L.distill(ref[r], ids[r], vals[r], nr, yr, float(w_[r]), tau, alpha, scale)
        if abs(l) > float(torch.finfo(torch.float32).max):  # a label's or a listed word's logit at the type's lowest value
            l = np.copysign(np.inf, l)
        there = (ids[r] >= 0) & (ids[r] < V) & np.isfinite(vals[r])
        t = vals[r][there].astype(np.float64) / tau
        norm = nr if nr is not None else (L.lse(t) if len(t) else 0.0)
        p = np.exp(t - norm)
        # a list's probability: its argument is rounded twice, and (own sum) so are the others'
        p_err = 2.0 ** -24 * (4 * np.abs(t).max() + 8) if len(t) else 0.0
        err, err1 = row_err(ref[r], tau), row_err(ref[r], 1.0)
        if not np.isfinite(l):
            assert np.array_equal(got[r], l, equal_nan=True)
        else:
            zk = ref[r][ids[r][there]] / tau
            gap = np.abs(t) + np.abs(zk) + np.abs(norm) + np.abs(L.lse(ref[r], tau)) if len(t) else np.zeros(0)
            gap = np.where(p > 0, gap, 0.0)
            tol = alpha * tau * tau * ((p * (err + p_err)).sum() + (p * gap).sum() * (p_err + 2.0 ** -23))
            tol += (1 - alpha) * (err1 + 2.0 ** -22 * np.abs(ref[r][np.isfinite(ref[r])]).max(initial=0.0)) if yr >= 0 else 0.0
            tol = abs(w_[r]) * (tol + 2.0 ** -40) + 2.0 ** -23 * abs(l)
            assert abs(got[r] - l) <= tol, (r, got[r], l, tol)
        if g is not None:
            mass = np.zeros(V)
            np.add.at(mass, ids[r][there], p)
            size = alpha * tau * (p.sum() * L.softmax(ref[r], tau) * (err + p_err + 2.0 ** -22) + mass * (p_err + 2.0 ** -21))
            if yr >= 0 and alpha < 1:
                size += (1 - alpha) * (L.softmax(ref[r]) * (err1 + 2.0 ** -22))
                size[yr] += 2.0 ** -22
            tol = abs(scale * w_[r]) * size + eps * np.abs(gr) * (1 + 1e-3) + 1e-37
            assert np.isfinite(gr).all()
            bad = ~(np.abs(g[r] - gr) <= tol)
            assert not bad.any(), (r, np.nonzero(bad)[0][:5], g[r][bad][:5], gr[bad][:5], tol[bad][:5])
    if np.isfinite(got).all():
        assert float(total) == pytest.approx(got.sum(), rel=1e-12, abs=1e-12)
    return flag


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V,K,pad", [(1, 1, 1, 0), (2, 3, 2, 1), (3, 8, 8, 0), (3, 9, 4, 2), (5, 250, 8, 0), (4, 1000, 257, 0), (3, 2049, 64, 7),
                                          (2, 8191, 1024, 0), (2, 20000, 10, 0), (2, 33278, 100, 1), (2, 70001, 64, 0), (1, 120007, 32, 0),
                                          (1, 300001, 16, 0)])
def test_distill_sizes(rows, V, K, pad, dtype):
    check_distill(patterns("normal", rows, V, V), *lists(rows, V, K, V + 1, False), dtype, pad, tau=2.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("slots", [200, 500, 1000, 1500, 2048, 3000, 4000, 6000, 8100, 10000, 12700, 18000, 25500, 25700])
def test_distill_widths(slots, dtype):
    V = slots * (4 if dtype == "fp32" else 8) + 1
    check_distill(patterns("normal", 3, V, slots), *lists(3, V, 30, slots, True), dtype, tau=1.0 if slots % 3 else 2.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["normal", "steep", "lowest", "huge"])
@pytest.mark.parametrize("slots,K", [(30, 20), (127, 1024), (255, 64), (511, 100)])
def test_distill_many_short_rows(slots, K, kind, dtype):
    V = slots * (4 if dtype == "fp32" else 8) + 3
    for tau, grad in ((2.0, "inplace"), (1.5, "apart"), (1.0, "apart")):
        check_distill(patterns(kind, 1025, V, slots), *lists(1025, V, K, slots, tau != 1.0), dtype, 1, tau, grad=grad)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0])
@pytest.mark.parametrize("kind", ["equal", "steep", "falling", "clustered", "lowest", "late", "offset", "all lowest", "huge"])
@pytest.mark.parametrize("V", [1203, 9001, 70001])
def test_distill_patterns(V, kind, tau, dtype):
    z = patterns("normal" if kind == "late" else kind, 2, V, 5)
    ids, vals, y, w = lists(2, V, 9, 4, False)
    if kind == "falling":
        z *= 60.0
    if kind == "late":  # only the last words are left, far below zero
        z[:, : V - 300] = -np.inf
        z[:, V - 300:] -= 500.0
        ids, y = V - 1 - ids % 300, V - 1 - y % 300
    check_distill(z, ids.astype(np.int32), vals, y.astype(np.int32), w, dtype, tau=tau)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("grad", ["apart", "inplace", "none"])
@pytest.mark.parametrize("tau,alpha,own", [(1.0, 0.5, True), (2.0, 0.3, False), (0.5, 1.0, True), (3.0, 0.0, False), (1.0, 1.0, False)])
def test_distill_ragged_lists(tau, alpha, own, grad, dtype):
    check_distill(patterns("normal", 9, 1203, 5), *lists(9, 1203, 21, 6, True), dtype, 3 if grad == "apart" else 0, tau, alpha, own=own, grad=grad)


@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_masked_words(dtype):
    z = patterns("few", 4, 700, 3)
    ids, vals, y, w = lists(4, 700, 12, 4, False)
    for r in range(3):  # the list and the label within what is left
        z[r, ids[r]] = z[r, y[r]] = 1.0
    z[0, ids[0, 0]] = -np.inf  # a listed word without probability: infinite loss, a gradient all the same
    ids[3] = -1
    y[3] = -1
    z[3] = -np.inf  # nothing left, nothing asked
    check_distill(z, ids, vals, y, w, dtype, tau=1.5)
    z[3, :] = -np.inf
    ids[3, 0] = 5  # an empty row that the list gives mass
    check_distill(z, ids, vals, y, w, dtype, tau=1.5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("grad", ["apart", "inplace"])
def test_distill_positions_without_weight_hold_anything(grad, dtype):
    z = patterns("normal", 5, 333, 3)
    ids, vals, y, w = lists(5, 333, 12, 4, False)
    z[1], z[3, 7], vals[1], w[1], w[3] = np.nan, np.inf, np.nan, 0.0, 0.0
    check_distill(z, ids, vals, y, w, dtype, 0, 2.0, grad=grad)


def test_distill_ids_out_of_range_count_as_absent_and_are_reported():
    z, (ids, vals, y, w) = patterns("normal", 3, 50, 1), lists(3, 50, 6, 2, False)
    assert int(check_distill(z, ids, vals, y, w, "fp32")) == 0
    ids[1, 3], y[2] = 50, 2 ** 31 - 1
    d, ref = place(z, "fp32")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.empty_like(d)
    loss = binding.rnnlm_distill_loss(d, torch.as_tensor(ids).cuda(), torch.as_tensor(vals).cuda(), None, torch.as_tensor(y).cuda(), None, 1.0, 0.5,
                                      dlogits=out, range_flag=flag)
    assert int(flag) == 1
    for r in range(3):
        l, g = L.distill(ref[r], ids[r], vals[r], None, int(y[r]), 1.0, 1.0, 0.5)
        assert float(loss[r]) == pytest.approx(l, rel=1e-5) and np.abs(out[r].cpu().numpy() - g).max() < 1e-6


def test_distill_a_nan_stays_in_its_row():
    z, (ids, vals, y, w) = patterns("normal", 3, 500, 1), lists(3, 500, 6, 2, False)
    z[1, 100] = np.nan
    d, _ = place(z, "fp32")
    out = torch.empty_like(d)
    loss = binding.rnnlm_distill_loss(d, torch.as_tensor(ids).cuda(), torch.as_tensor(vals).cuda(), None, torch.as_tensor(y).cuda(), None, 1.0, 0.5, dlogits=out)
    assert torch.isnan(loss).tolist() == [False, True, False]
    assert bool(torch.isfinite(out[0]).all()) and bool(torch.isfinite(out[2]).all()) and bool(torch.isnan(out[1]).all())


def test_distill_a_nan_in_a_list_stays_in_its_row():
    z, (ids, vals, y, w) = patterns("normal", 3, 500, 1), lists(3, 500, 6, 2, False)
    vals[1, 4] = np.nan
    vals[2, 4], ids[2, 4] = np.nan, -1  # of an absent entry: nobody's
    d, _ = place(z, "fp32")
    out = torch.empty_like(d)
    for n in (None, torch.full((3,), 9.0, device="cuda")):
        loss = binding.rnnlm_distill_loss(d, torch.as_tensor(ids).cuda(), torch.as_tensor(vals).cuda(), n, torch.as_tensor(y).cuda(), None, 1.0, 0.5, dlogits=out)
        assert torch.isnan(loss).tolist() == [False, True, False]
        assert bool(torch.isfinite(out[0]).all()) and bool(torch.isfinite(out[2]).all()) and bool(torch.isnan(out[1]).all())


def test_distill_gradient_is_the_loss_difference():
    """Against differences of the call's own losses: fp32 losses of about 4 to 2^-22, steps of 2^-5, third derivatives below 1."""
    rng = np.random.default_rng(2)
    V, tau, alpha, h = 20, 2.0, 0.6, 2.0 ** -5
    z = rng.normal(size=V).astype(np.float32)
    ids, vals = np.array([3, 7, 3, 11], np.int32), rng.normal(size=4).astype(np.float32)
    rows = np.concatenate([z[None], z + h * np.eye(V, dtype=np.float32), z - h * np.eye(V, dtype=np.float32)])
    n = len(rows)
    rep = lambda a: torch.as_tensor(np.repeat(a[None], n, 0)).cuda()  # noqa: E731
    out = torch.empty(n, V, device="cuda")
    loss = binding.rnnlm_distill_loss(torch.as_tensor(rows).cuda(), rep(ids), rep(vals), None, torch.full((n,), 7, dtype=torch.int32, device="cuda"),
                                      None, tau, alpha, dlogits=out).double().cpu().numpy()
    diff = (loss[1: V + 1] - loss[V + 1:]) / (2 * h)
    assert np.abs(diff - out[0].cpu().numpy()).max() <= 2 * 4 * 2.0 ** -22 / (2 * h) + h * h / 6


# ---- verification -----------------------------------------------------------------------------------------------------
def check_verify(target, drafts, u, draft=None, lengths=None, tau=1.0, tau_d=1.0, dtype="fp32", pad=0):
    K1, B, V = target.shape
    tau, tau_d = float(np.float32(tau)), float(np.float32(tau_d))  # as the call gets them: a drawn word may hang on 1e-9
    t, ref = place(target.reshape(-1, V), dtype, pad)
    q = qref = None
    if draft is not None:
        q, qref = place(draft.reshape(-1, V), dtype, 0)
        q, qref = q.unflatten(0, (K1 - 1, B)), qref.reshape(K1 - 1, B, V)
    cuda = lambda a, dt: None if a is None else torch.as_tensor(np.asarray(a, dt)).cuda()  # noqa: E731
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    n, tokens = binding.rnnlm_verify_drafts(t.unflatten(0, (K1, B)), cuda(drafts, np.int32), cuda(u, np.float32), q, cuda(lengths, np.int32), tau, tau_d,
                                            range_flag=flag)
    n, tokens, ref = n.cpu().numpy(), tokens.cpu().numpy(), ref.reshape(K1, B, V)
    for b in range(B):
        want = L.verify(ref[:, b], [] if drafts is None else drafts[:, b], np.float32(u[:, b]), None if draft is None else qref[:, b],
                        None if lengths is None else lengths[b], tau, tau_d)
        assert n[b] == want[0] and tokens[:, b].tolist() == want[1].tolist(), (b, n[b], tokens[:, b], want)
    return n, tokens, int(flag)


def texts(K, B, V, seed, close=0.5):
    rng = np.random.default_rng(seed)
    target = rng.normal(0.0, 2.0, (K + 1, B, V))
    draft = target[:K] + close * rng.normal(size=(K, B, V))
    q = np.exp(draft - draft.max(2, keepdims=True)) if K else draft
    drafts = np.array([[rng.choice(V, p=q[i, b] / q[i, b].sum()) for b in range(B)] for i in range(K)], np.int32).reshape(K, B)
    return target, draft, drafts, rng.random((K + 1, B)), rng.integers(0, K + 1, B)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("K,B,V,pad", [(1, 1, 1, 0), (2, 3, 2, 1), (3, 5, 7, 0), (4, 2, 100, 0), (8, 37, 1001, 3), (2, 300, 260, 0), (5, 2, 33278, 1),
                                       (3, 1, 100000, 0), (40, 2, 60, 0), (1, 1100, 20011, 0)])
def test_verify_sizes(K, B, V, pad, with_draft, dtype):
    target, draft, drafts, u, lengths = texts(K, B, V, K + B + V)
    n = check_verify(target, drafts, u, draft if with_draft else None, None, 1.0, 1.0, dtype, pad)[0]
    check_verify(target, drafts, u, draft if with_draft else None, lengths, 0.8, 1.25, dtype, pad)
    if with_draft and K * B >= 30:
        assert 0 < n.mean() < K  # both outcomes occur


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,V", [(1, 1), (3, 5000), (200, 33), (2, (1 << 20))])
def test_verify_without_drafts_draws_from_the_row(B, V, dtype):
    rng = np.random.default_rng(B)
    check_verify(rng.normal(0, 2, (1, B, V)), None, rng.random((1, B)), dtype=dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["equal", "steep", "offset", "all lowest", "lowest", "huge", "ties"])
@pytest.mark.parametrize("V", [900, 50001])
def test_verify_patterns(V, kind, dtype):
    K, B = 2, 3
    target, draft = (patterns(kind, n * B, V, s).reshape(n, B, V) for n, s in ((K + 1, 1), (K, 2)))
    rng = np.random.default_rng(3)
    drafts = np.array([[rng.choice(np.argsort(draft[i, b])[-20:]) for b in range(B)] for i in range(K)], np.int32)
    for d in (draft, None):
        check_verify(target, drafts, rng.random((K + 1, B)) * 0.5, d, None, 1.0, 2.0, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [515, 40007])
def test_verify_masked_rows_and_rows_that_are_no_numbers(V, dtype):
    K, B = 2, 10
    target, draft, drafts, u, _ = texts(K, B, V, 11)
    target[:, 0] = -np.inf                    # nothing left: no draft accepted, no word
    target[0, 1, 17] = np.nan
    target[0, 2, drafts[0, 2]] = -np.inf      # the draft is masked
    target[:, 3, 2:] = -np.inf                # two words left
    target[:, 3, :2] = 0.0
    drafts[:, 3] = 0
    target[:, 4], draft[:, 4] = 0.25, 0.25    # both flat: every draft accepted
    target[0, 5, 3] = np.inf
    target[:, 6, ::2] = -3e38                 # the lowest values of the type
    draft[:, 7], target[:, 7] = -np.inf, -np.inf
    draft[:, 7, 9] = target[:, 7, 9] = 0.0    # one word left in both, and it is the draft
    drafts[:, 7] = 9
    draft[:, 8] = -np.inf                     # a drafter without a word
    draft[0, 9, 7], u[0, 9] = np.nan, 0.9
    n, tokens, _ = check_verify(target, drafts, u, draft, dtype=dtype)
    assert tokens[:, 0].tolist() == tokens[:, 1].tolist() == tokens[:, 5].tolist() == [-1, -1, -1]
    assert n[4] == K and tokens[:, 7].tolist() == [9, 9, 9]
    check_verify(target, drafts, u, None, dtype=dtype)


@pytest.mark.parametrize("V", [1000, 20000, 100003])
def test_verify_numbers_at_the_ends(V):
    K, B = 1, 6
    target, draft, drafts, u, _ = texts(K, B, V, 4)
    u[:, :2], u[:, 2:4] = 0.0, np.float32(1.0) - np.float32(2.0 ** -24)
    check_verify(target, drafts, u, draft)
    check_verify(target, drafts, u, None)
    # a probability of exactly a half against a half: not accepted
    z = np.full((2, 1, 4), -np.inf)
    z[:, :, :2] = 0.0
    assert check_verify(z, np.zeros((1, 1), np.int32), np.array([[0.5], [0.2]]))[0].tolist() == [0]
    assert check_verify(z, np.zeros((1, 1), np.int32), np.array([[0.49999997], [0.2]]))[0].tolist() == [1]


@pytest.mark.parametrize("V", [3000, 33000, 100000])
def test_verify_a_draft_model_that_is_the_target(V):
    """Every draft of positive probability is accepted; one that is not drawn from the model's words leaves r = 0: p itself."""
    K, B = 2, 4
    target, draft, drafts, u, _ = texts(K, B, V, 3, 0.0)
    assert check_verify(target, drafts, u, draft)[0].tolist() == [K] * B
    target[0, :, drafts[0]] = draft[0, :, drafts[0]] = -np.inf
    assert check_verify(target, drafts, u, draft)[0].tolist() == [0] * B


def test_verify_drafts_out_of_range_and_lengths_beyond_the_batch():
    target, draft, drafts, u, _ = texts(3, 4, 90, 8)
    drafts[0, 1], drafts[1, 2], drafts[2, 3] = 90, -5, 2 ** 31 - 1
    u[:3] = 0.0  # every other draft is accepted
    assert check_verify(target, drafts, u, draft, [9, 9, 3, 2])[2] == 1
    assert check_verify(target, drafts, u, draft, [-4, 0, 1, 2])[2] == 0  # behind the texts' own drafts: not looked at
    check_verify(target, drafts, u, None, [9, 9, 3, 2])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tau", [1e-3, 1e3])
@pytest.mark.parametrize("V", [1203, 20011, 90001])
def test_temperatures_at_the_ends(V, tau, dtype):
    tau = float(np.float32(tau))
    z = patterns("normal", 4, V, V)
    check_top(z, 20, tau, dtype, 1)
    ids, vals, y, w = lists(4, V, 20, 3, False)
    for alpha in (0.5, 1.0):
        check_distill(z, ids, vals, y, w, dtype, tau=tau, alpha=alpha)
    target, draft, drafts, u, lengths = texts(2, 3, V, V)
    check_verify(target, drafts, u, draft, lengths, tau, tau, dtype)
    check_verify(target, drafts, u, draft, None, 1.0, tau, dtype)


# ---- streams, graphs, workspaces --------------------------------------------------------------------------------------
def test_calls_follow_their_stream_and_can_be_captured():
    """The three calls one after the other in a graph, replayed on new inputs with eager work between, against eager calls."""
    rng = np.random.default_rng(9)
    M, V, K, B, D = 12, 5003, 20, 4, 2
    z = torch.empty(M, V, device="cuda", dtype=torch.bfloat16)
    s = torch.empty(M, V, device="cuda", dtype=torch.bfloat16)
    u = torch.empty(D + 1, B, device="cuda")
    drafts = torch.empty(D, B, dtype=torch.int32, device="cuda")
    y = torch.empty(M, dtype=torch.int32, device="cuda")

    def refill(i):
        z.copy_(torch.as_tensor(rng.normal(0, 2, (M, V)))), s.copy_(torch.as_tensor(rng.normal(0, 2, (M, V))))
        u.copy_(torch.as_tensor(rng.random((D + 1, B)))), drafts.copy_(torch.as_tensor(rng.integers(0, V, (D, B))))
        y.copy_(torch.as_tensor(rng.integers(0, V, M)))

    def calls(out):
        binding.rnnlm_top_logits(z, K, 2.0, out["ids"], out["vals"], out["lse"], out["w1"])
        binding.rnnlm_distill_loss(s, out["ids"], out["vals"], out["lse"], y, None, 2.0, 0.5, 1.0 / M, out["loss"], out["d"], out["sum"])
        binding.rnnlm_verify_drafts(z.view(D + 1, B, V), drafts, u, s[: D * B].view(D, B, V), None, 1.0, 1.0, out["n"], out["tokens"], out["w2"])

    def fresh():
        e = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
        i32 = torch.int32
        return dict(ids=e(M, K, dtype=i32), vals=e(M, K), lse=e(M), w1=e(1 << 20, dtype=torch.uint8), w2=e(1 << 20, dtype=torch.uint8), loss=e(M),
                    d=e(M, V, dtype=torch.bfloat16), sum=e(1, dtype=torch.float64), n=e(B, dtype=i32), tokens=e(D + 1, B, dtype=i32))

    refill(0)
    kept = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(kept)  # (the first call outside of a capture)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(kept)
    for i in range(4):
        refill(i)
        graph.replay()
        eager = fresh()
        calls(eager)
        torch.cuda.synchronize()
        for k in kept:
            if k not in ("w1", "w2"):
                assert torch.equal(kept[k], eager[k]), (i, k)


def test_calls_on_two_streams_at_once():
    M, V, K, B, D = 300, 20011, 150, 20, 4
    i32 = torch.int32

    def make(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        z = torch.randn(M, V, device="cuda", generator=g).bfloat16()
        return dict(z=z, u=torch.rand(D + 1, B, device="cuda", generator=g), d=torch.empty_like(z),
                    drafts=torch.randint(0, V, (D, B), device="cuda", generator=g, dtype=i32))

    def calls(s):
        ids, vals, lse = binding.rnnlm_top_logits(s["z"], K)
        loss = binding.rnnlm_distill_loss(s["z"], ids, vals, lse, dlogits=s["d"])
        n, tokens = binding.rnnlm_verify_drafts(s["z"][: (D + 1) * B].view(D + 1, B, V), s["drafts"], s["u"], s["z"][M - D * B:].view(D, B, V))
        return [ids, vals, lse, loss, s["d"].clone(), n, tokens]

    states = [make(1), make(2)]
    alone = [calls(s) for s in states]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k in (0, 1):
            with torch.cuda.stream(streams[k]):
                got[k].append(calls(states[k]))
    torch.cuda.synchronize()
    for k in (0, 1):
        for turn in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(alone[k], turn))


def test_rows_behind_and_between_are_left_as_they_were():
    V, pad, M = 130, 6, 5
    for dtype in DTYPES.values():
        z = torch.randn(M, V, device="cuda").to(dtype)
        buf = torch.full((M + 2, V + pad), 3.0, dtype=dtype, device="cuda")
        ids = torch.randint(0, V, (M, 4), device="cuda", dtype=torch.int32)
        binding.rnnlm_distill_loss(z, ids, torch.randn(M, 4, device="cuda"), dlogits=buf[1: M + 1, :V])
        assert bool((buf[0] == 3).all() and (buf[M + 1] == 3).all() and (buf[1: M + 1, V:] == 3).all())
        assert not bool((buf[1: M + 1, :V] == 3).any())


@pytest.mark.parametrize("V", [700, 5001])
def test_rows_further_apart_than_32_bits_reach(V):
    ld, M = (1 << 30) + 1, 5
    buf = torch.empty((M - 1) * ld + V, device="cuda", dtype=torch.bfloat16)  # 8.6 GB: the last row starts behind 2^32 elements
    far = buf.as_strided((M, V), (ld, 1))
    near = torch.randn(M, V, device="cuda").bfloat16()
    far.copy_(near)
    got, want = binding.rnnlm_top_logits(far, 30), binding.rnnlm_top_logits(near, 30)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    drafts, u = torch.randint(0, V, (2, 1), device="cuda", dtype=torch.int32), torch.rand(3, 1, device="cuda")
    got = binding.rnnlm_verify_drafts(far[:3, None], drafts, u, far[3:, None])
    assert all(torch.equal(a, b) for a, b in zip(got, binding.rnnlm_verify_drafts(near[:3, None], drafts, u, near[3:, None])))
    ids, vals, lse = want
    loss, loss2 = binding.rnnlm_distill_loss(far, ids, vals, lse, dlogits=far), binding.rnnlm_distill_loss(near, ids, vals, lse, dlogits=near)
    assert torch.equal(loss, loss2) and torch.equal(far, near)


def test_same_inputs_same_bits():
    z = torch.randn(50, 3001, device="cuda").to(torch.bfloat16)
    ids, vals, lse = binding.rnnlm_top_logits(z, 200)
    first = None
    for _ in range(3):
        d = torch.empty_like(z)
        got = [*binding.rnnlm_top_logits(z, 200), binding.rnnlm_distill_loss(z, ids, vals, lse, tau=1.0, dlogits=d), d]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_empty_batches():
    z = torch.empty(0, 40, device="cuda")
    ids, vals, lse = binding.rnnlm_top_logits(z, 3)
    total = torch.ones(1, dtype=torch.float64, device="cuda")
    loss = binding.rnnlm_distill_loss(z, ids, vals, lse, dlogits=torch.empty_like(z), sum_loss=total)
    assert ids.shape == (0, 3) and loss.shape == (0,) and float(total) == 0.0


def test_the_binding_refuses():
    z = torch.zeros(4, 10, device="cuda")
    i = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    v = torch.zeros(4, 2, device="cuda")
    bad = [
        lambda: binding.rnnlm_top_logits(z.half(), 2), lambda: binding.rnnlm_top_logits(z.t(), 2), lambda: binding.rnnlm_top_logits(z, 11),
        lambda: binding.rnnlm_top_logits(z[:, ::2], 2), lambda: binding.rnnlm_top_logits(z[:1].expand(4, 10), 2),
        lambda: binding.rnnlm_top_logits(z, 2, ids=i.long()), lambda: binding.rnnlm_top_logits(z, 2, lse=torch.zeros(3, device="cuda")),
        lambda: binding.rnnlm_distill_loss(z, i[:3], v), lambda: binding.rnnlm_distill_loss(z, i, v.double()),
        lambda: binding.rnnlm_distill_loss(z, i, v, alpha=0.5), lambda: binding.rnnlm_distill_loss(z, i, v, dlogits=z.bfloat16()),
        lambda: binding.rnnlm_distill_loss(z, i, v, dlogits=z[:3]), lambda: binding.rnnlm_distill_loss(z, i, v, tau=0.0),
        lambda: binding.rnnlm_distill_loss(z, i.cpu(), v), lambda: binding.rnnlm_distill_loss(z.view(-1)[:36].view(4, 9), i, v, dlogits=z.view(-1)[4:].view(4, 9)),
        lambda: binding.rnnlm_verify_drafts(z.view(2, 2, 10), None, v[:2]), lambda: binding.rnnlm_verify_drafts(z.view(2, 2, 10), i[:1], v[:1]),
        lambda: binding.rnnlm_verify_drafts(z.view(2, 2, 10), i[:1], v[:2], z.view(2, 2, 10)),
        lambda: binding.rnnlm_verify_drafts(z.view(2, 2, 10), i[:1], v[:2], workspace=torch.zeros(8, dtype=torch.uint8, device="cuda")),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(binding.RnnlmError):
            call()
            print("not refused:", k)
    torch.cuda.synchronize()
