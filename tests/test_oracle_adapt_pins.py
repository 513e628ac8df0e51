"""The oracle of the operators that adapt a trained model, against closed forms and differences."""
import numpy as np
import pytest

from oracle import adapt as A


def difference(f, z, h=1e-6):
    d = np.zeros(z.shape)
    for i in np.ndindex(*z.shape):
        up, down = z.copy(), z.copy()
        up[i] += h
        down[i] -= h
        d[i] = (f(up) - f(down)) / (2 * h)
    return d


def test_policy_by_hand():
    # two words of equal probability, drawn when the word had probability 1/4: rho = 2, clipped at 1.2 for good words only
    z, y = np.zeros((3, 2)), [0, 1, 0]
    loss, logp, dz, _ = A.policy(z, y, [1.0, -1.0, 0.0], old=np.log([0.25] * 3))
    assert np.allclose(logp, np.log(0.5), rtol=1e-15)
    assert np.allclose(loss, [-1.2, 2.0, 0.0], rtol=1e-14)
    assert np.allclose(dz, [[0, 0], [-1.0, 1.0], [0, 0]], atol=1e-14)
    # the reference gives the word probability 1: d = ln 2
    loss, _, dz, _ = A.policy(z[:1], y[:1], [0.0], ref=[0.0], beta=3.0)
    assert np.allclose(loss, 3 * (1 - np.log(2)), rtol=1e-14) and np.allclose(dz, [[-1.5, 1.5]], rtol=1e-14)


@pytest.mark.parametrize("tau,beta,old", [(1.0, 0.0, True), (0.7, 0.1, True), (1.3, 0.2, False)])
def test_policy_gradient(tau, beta, old):
    rng = np.random.default_rng(1)
    rows, V = 12, 7
    z, y = rng.normal(size=(rows, V)) * 2, rng.integers(-1, V, rows)
    logp = A.policy(z, y, np.zeros(rows), tau=tau)[1]
    o, ref, adv, w = logp + rng.normal(size=rows) * 0.4, logp + rng.normal(size=rows), rng.normal(size=rows), rng.random(rows)
    w[3] = 0.0
    kw = dict(ref=ref, weight=w, tau=tau, lo=0.2, hi=0.3, beta=beta)
    dz = A.policy(z, y, adv, old=o if old else None, scale=0.25, **kw)[2]
    # on-policy: the gradient is the one at old = l, held fixed
    f = lambda x: 0.25 * A.policy(x, y, adv, old=o if old else logp, **kw)[0].sum()  # noqa: E731
    assert np.abs(dz - difference(f, z)).max() < 1e-7


def test_preference_by_hand():
    # one position a text, two words: S = ln(p), r = ln(0.8 / 0.2) - (0.1 - 0.3)
    z = np.log([[[0.8, 0.2], [0.2, 0.8]]])
    y = np.array([[0, 0]])
    loss, S, dz, r, _ = A.preference(z, y, ref=[0.1, 0.3], beta=0.5)
    assert np.allclose(S, np.log([0.8, 0.2]), rtol=1e-14) and np.allclose(r, np.log(4) + 0.2, rtol=1e-14)
    x = 0.5 * (np.log(4) + 0.2)
    assert np.allclose(loss, -np.log(1 / (1 + np.exp(-x))), rtol=1e-14)
    g = -0.5 / (1 + np.exp(x))
    assert np.allclose(dz, [[[0.2 * g, -0.2 * g], [-0.8 * g, 0.8 * g]]], rtol=1e-13)
    assert np.allclose(A.preference(z, y, kind="squared", beta=0.5)[0], (np.log(4) - 1.0) ** 2, rtol=1e-14)
    assert np.allclose(A.preference(z, y, kind="hinge", beta=0.5)[0], 1 - 0.5 * np.log(4), rtol=1e-14)


@pytest.mark.parametrize("kind,smoothing", [("logistic", 0.0), ("logistic", 0.2), ("squared", 0.0), ("hinge", 0.0)])
@pytest.mark.parametrize("mean", [False, True])
def test_preference_gradient(kind, smoothing, mean):
    rng = np.random.default_rng(2)
    T, P, V = 4, 3, 5
    z, y = rng.normal(size=(T, 2 * P, V)) * 2, rng.integers(-1, V, (T, 2 * P))
    y[:, 1] = -1
    kw = dict(ref=rng.normal(size=2 * P), weight=np.array([1.0, 0.5, 2.0]), kind=kind, beta=0.3, smoothing=smoothing, mean=mean)
    dz = A.preference(z, y, scale=0.5, **kw)[2]
    assert np.abs(dz - difference(lambda x: 0.5 * A.preference(x, y, **kw)[0].sum(), z)).max() < 1e-7


@pytest.mark.parametrize("kind", ["logistic", "squared", "hinge"])
def test_preference_without_a_number(kind):
    # both texts of pair 0 hold a masked word: r = -inf + inf; pair 1 is as by itself
    z, y = np.zeros((2, 4, 3)), np.zeros((2, 4), int)
    z[0, 0, 0] = z[1, 2, 0] = -np.inf
    loss, S, dz, r, g = A.preference(z, y, kind=kind)
    assert S[0] == -np.inf and S[2] == -np.inf and np.isnan(r[0]) and np.isnan(loss[0]) and np.isnan(g[0])
    assert not dz[0, 0].any() and not dz[1, 2].any() and np.isnan(dz[1, 0]).all() and np.isnan(dz[0, 2]).all()
    alone = A.preference(z[:, [1, 3]], y[:, [1, 3]], kind=kind)
    assert loss[1] == alone[0][0] and np.array_equal(dz[:, [1, 3]], alone[2])


def test_adapter_gradient():
    rng = np.random.default_rng(3)
    M, K, N, R, n = 5, 4, 6, 2, 3
    x, down, up, base = rng.normal(size=(M, K)), rng.normal(size=(n, R, K)), rng.normal(size=(n, N, R)), rng.normal(size=(M, N))
    ids, scale, dout = np.array([0, 2, -1, 0, 9]), np.array([0.5, 1.0, 2.0]), rng.normal(size=(M, N))
    out, inner = A.adapter_forward(x, down, up, ids, scale, base)
    assert np.array_equal(out[2], base[2]) and np.array_equal(out[4], base[4]) and not inner[[2, 4]].any()
    assert np.allclose(out[1], base[1] + 2.0 * up[2] @ down[2] @ x[1], rtol=1e-13)
    ddown, dup, dx = A.adapter_backward(dout, x, inner, down, up, ids, scale)
    assert not ddown[1].any() and not dup[1].any()
    assert np.abs(ddown - difference(lambda d: (dout * A.adapter_forward(x, d, up, ids, scale)[0]).sum(), down)).max() < 1e-7
    assert np.abs(dup - difference(lambda u: (dout * A.adapter_forward(x, down, u, ids, scale)[0]).sum(), up)).max() < 1e-7
    assert np.abs(dx - difference(lambda v: (dout * A.adapter_forward(v, down, up, ids, scale)[0]).sum(), x)).max() < 1e-7
