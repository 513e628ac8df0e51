"""Pins of the oracle of the operators on logits: closed forms, worked examples, differences, and the property that
verification is there for (accepted and drawn words are distributed as the target's)."""
import numpy as np
import pytest

from oracle import logits as L


def test_lse_and_top_by_hand():
    z = np.array([0.0, np.log(3.0), -np.inf, np.log(3.0)])
    assert L.lse(z) == pytest.approx(np.log(7.0))
    assert L.lse(z, 2.0) == pytest.approx(np.log(1.0 + 2.0 * np.sqrt(3.0)))
    ids, vals, n = L.top(z, 4)
    assert ids.tolist() == [1, 3, 0, 2] and vals[3] == -np.inf and n == pytest.approx(np.log(7.0))
    assert L.lse([-np.inf, -np.inf]) == -np.inf and np.isnan(L.lse([0.0, np.nan])) and np.isnan(L.lse([0.0, np.inf]))


def test_softmax_sums_to_one_wherever_the_logits_are():
    for z in ([1.0, 2.0, 3.0], [-3e38] * 7, [1e30, 1e30, -1e30], [5e4, 5e4 + 1.0, -np.inf]):
        assert L.softmax(z, 0.7).sum() == pytest.approx(1.0, abs=1e-15)
    assert L.softmax([-np.inf] * 3).tolist() == [0.0] * 3 and np.isnan(L.softmax([0.0, np.inf])).any() and np.isnan(L.softmax([np.nan, 0.0])).all()


def test_distillation_from_the_student_itself_costs_nothing():
    z = np.random.default_rng(0).normal(size=50)
    loss, grad = L.distill(z, np.arange(50), z, L.lse(z, 2.0), tau=2.0)
    assert abs(loss) < 1e-14 and np.abs(grad).max() < 1e-15


def test_hard_labels_alone_are_cross_entropy():
    z = np.array([0.0, np.log(2.0), np.log(5.0)])
    loss, grad = L.distill(z, [0], [0.0], y=2, alpha=0.0)
    assert loss == pytest.approx(-np.log(5.0 / 8.0))
    assert grad == pytest.approx(np.array([1, 2, -3]) / 8.0)


def test_repeated_words_and_masks():
    z = np.array([0.0, 0.0, -np.inf])
    a = L.distill(z, [0, 0, 1], [0.0, 0.0, 0.0])
    b = L.distill(z, [0, 1], [np.log(2.0), 0.0])
    assert a[1] == pytest.approx(b[1])
    loss, grad = L.distill(z, [2, 0], [0.0, 0.0])
    assert loss == np.inf and grad == pytest.approx([0.0, 0.5, -0.5])
    assert L.distill(np.full(3, np.nan), [0], [1.0], weight=0.0)[0] == 0.0


@pytest.mark.parametrize("tau,alpha,own_sum", [(1.0, 1.0, True), (2.0, 0.5, True), (0.7, 0.3, False), (3.0, 1.0, False)])
def test_gradient_is_the_loss_difference(tau, alpha, own_sum):
    rng = np.random.default_rng(3)
    V, K = 13, 5
    z, ids, vals = rng.normal(size=V), rng.choice(V, K, replace=False), rng.normal(size=K)
    ids[2] = ids[0]
    n = None if own_sum else L.lse(vals, tau) + 0.2
    kw = dict(n=n, y=4, weight=1.7, tau=tau, alpha=alpha)
    grad = L.distill(z, ids, vals, scale=0.25, **kw)[1]
    for v in range(V):
        e = np.zeros(V)
        e[v] = 1e-5
        d = (L.distill(z + e, ids, vals, **kw)[0] - L.distill(z - e, ids, vals, **kw)[0]) / 2e-5
        assert 0.25 * d == pytest.approx(grad[v], abs=1e-9)


def test_verification_by_hand():
    third = np.log(np.array([[1.0, 1.0, 1.0], [2.0, 1.0, 1.0]]))
    # one draft with probability 1/3 under the target and all mass of its own: accepted below 1/3
    assert L.verify(third, [1], [0.3, 0.6])[0] == 1 and L.verify(third, [1], [0.3, 0.6])[1].tolist() == [1, 1]
    n, tokens = L.verify(third, [1], [0.4, 0.6])  # rejected: word 0 or 2, half and half
    assert n == 0 and tokens.tolist() == [2, -1]
    n, tokens = L.verify(third, [1], [0.3, 0.2], length=0)
    assert n == 0 and tokens.tolist() == [0, -1]
    assert L.verify(third, [7], [0.0, 0.0])[0] == 0  # no such word


@pytest.mark.parametrize("with_draft", [True, False])
def test_words_are_distributed_as_the_target(with_draft):
    """Over the draft's draws and a fine grid of both numbers, the first word has the target's probabilities."""
    rng = np.random.default_rng(5)
    V, G = 5, 60
    target, draft = rng.normal(size=(2, V)), rng.normal(size=(1, V))
    q = L.softmax(draft[0]) if with_draft else np.eye(V)[2]
    got, grid = np.zeros(V), (np.arange(G) + 0.5) / G
    for d in range(V):
        if q[d] == 0.0:
            continue
        for u in grid:
            for r in grid:
                got[L.verify(target, [d], [u, r], draft if with_draft else None)[1][0]] += q[d] / G / G
    assert np.abs(got - L.softmax(target[0])).max() < 2.0 / G
