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
