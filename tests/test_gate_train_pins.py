"""Pins of oracle/gate_train_oracle.py: differences, closed forms, brute force, planted mistakes (CPU)."""
import math

import numpy as np
import pytest

from oracle import gate_train_oracle as go
from oracle import moe_oracle as orc


def batch(T, E, k, seed):
    rng = np.random.default_rng([seed, T, E, k])
    scores = rng.standard_normal((T, E)).astype(np.float32)
    return rng, scores, orc.topk_select(scores, k)


def differences(f, s, eps=1e-6):
    s = np.asarray(s, dtype=np.float64)
    g = np.zeros_like(s)
    for i in np.ndindex(*s.shape):
        a, b = s.copy(), s.copy()
        a[i] += eps
        b[i] -= eps
        g[i] = (f(a) - f(b)) / (2 * eps)
    return g


def test_balance_loss_closed_forms():
    E, k = 8, 2
    even = np.array([[2 * i % E, (2 * i + 1) % E] for i in range(8)], dtype=np.int32)
    counts, prob_sum, loss = go.balance_loss(np.zeros((8, E)), even)
    assert counts.tolist() == [2] * E and np.allclose(prob_sum, 1.0) and loss == pytest.approx(1.0)
    # the same k experts take everything: E / k
    sharp = np.full((8, E), -50.0)
    sharp[:, :k] = 50.0
    hot = np.tile(np.arange(k, dtype=np.int32), (8, 1))
    assert go.balance_loss(sharp, hot)[2] == pytest.approx(E / k, rel=1e-12)
    assert go.balance_loss(sharp, hot, np.zeros(8))[2] == 0.0
    mask = np.array([1, 0, 1, 1, 0, 0, 1, 1])
    a = go.balance_loss(sharp[mask == 1], hot[mask == 1])
    b = go.balance_loss(np.where(mask[:, None] == 1, sharp, np.nan), hot, mask)
    assert a[0].tolist() == b[0].tolist() and a[2] == b[2]


@pytest.mark.parametrize("renorm", [0, 1])
def test_route_backward_against_differences(renorm):
    T, E, k = 4, 6, 3
    rng, scores, idx = batch(T, E, k, 1)
    dw = rng.standard_normal((T, k))
    counts = go.balance_loss(scores, idx)[0]

    def f(s):
        p = go.softmax(s)
        balance = E * k * (counts * p.sum(axis=0)).sum() / counts.sum() ** 2
        return (go.routing_weights(s, idx, renorm) * dw).sum() + 0.3 * balance

    got = go.route_backward(scores, idx, dw, counts, 0.3, renorm)
    assert np.abs(got - differences(f, scores)).max() < 1e-8
    # a softmax gradient adds up to nothing in every row
    assert np.abs(got.sum(axis=1)).max() < 1e-15
    # either part alone; a padded row is 0 whatever it holds
    both = go.route_backward(scores, idx, dw, None, 0, renorm) + go.route_backward(scores, idx, None, counts, 0.3, renorm)
    assert np.allclose(both, got, atol=1e-15)
    poisoned = scores.copy()
    poisoned[1] = np.nan
    mask = np.array([1, 0, 1, 1])
    padded = go.route_backward(poisoned, idx, dw, counts, 0.3, renorm, mask)
    assert not padded[1].any() and np.array_equal(padded[[0, 2, 3]], got[[0, 2, 3]])


def test_routing_weights_are_the_router_s():
    _, scores, idx = batch(50, 16, 4, 2)
    for renorm in (0, 1):
        ref = orc.routing_weights(scores, idx, renorm)
        assert np.allclose(go.routing_weights(scores, idx, renorm), ref, rtol=1e-6)


def test_distill_against_differences_and_closed_forms():
    T, E = 3, 5
    rng, scores, _ = batch(T, E, 2, 3)
    target = rng.standard_normal((T, E))
    loss, grad = go.gate_distill(scores, target)
    assert np.abs(grad - differences(lambda s: go.gate_distill(s, target)[0], scores)).max() < 1e-8
    assert loss > 0 and go.gate_distill(scores, scores)[0] == pytest.approx(0.0, abs=1e-15)
    assert go.gate_distill(scores, scores + 7.0)[0] == pytest.approx(0.0, abs=1e-14)     # a softmax sees differences only
    # one-hot target: cross entropy
    hot = np.full((T, E), -np.inf)
    hot[:, 2] = 0.0
    log_p = scores[:, 2] - np.log(np.exp(scores.astype(np.float64)).sum(axis=1))
    assert go.gate_distill(scores, hot)[0] == pytest.approx(-log_p.mean(), rel=1e-12)
    # two experts: p = 1 / (1 + e^-a)
    a, b = 0.7, -0.2
    p, q = 1 / (1 + math.exp(-a)), 1 / (1 + math.exp(-b))
    want = q * math.log(q / p) + (1 - q) * math.log((1 - q) / (1 - p))
    assert go.gate_distill(np.array([[a, 0.0]]), np.array([[b, 0.0]]))[0] == pytest.approx(want, rel=1e-12)
    # nothing left of a row, or of the batch
    off = np.full((1, E), -np.inf)
    loss0, grad0 = go.gate_distill(off, target[:1])
    assert loss0 == 0.0 and not grad0.any()
    assert go.gate_distill(scores, target, 1.0, np.zeros(T))[0] == 0.0


def test_gate_backward_against_differences():
    rng = np.random.default_rng(4)
    T, d, E = 3, 4, 5
    x, w, ds = rng.standard_normal((T, d)), rng.standard_normal((E, d)), rng.standard_normal((T, E))
    dw, db, dx = go.gate_backward(x, w, ds)
    assert np.abs(dw - differences(lambda v: float((x @ v.T * ds).sum()), w)).max() < 1e-8
    assert np.abs(dx - differences(lambda v: float((v @ w.T * ds).sum()), x)).max() < 1e-8
    assert np.abs(db - differences(lambda v: float(((x @ w.T + v) * ds).sum()), np.zeros((1, E)))[0]).max() < 1e-8
    mask = np.array([1, 0, 1])
    xm, dm = x.copy(), ds.copy()
    xm[1], dm[1] = np.nan, np.nan
    pw, pb, px = go.gate_backward(xm, w, dm, mask)
    keep = [0, 2]
    assert np.allclose(pw, ds[keep].T @ x[keep]) and np.allclose(pb, ds[keep].sum(axis=0)) and not px[1].any()


def test_clip_closed_forms():
    norm, out = go.clip_grads([np.array([3.0]), np.array([[4.0]])], 1.0)
    assert norm == 5.0 and out[0][0] == pytest.approx(0.6) and out[1][0, 0] == pytest.approx(0.8)
    norm, out = go.clip_grads([np.array([3.0]), np.array([4.0])], 5.0)
    assert norm == 5.0 and out[0][0] == 3.0
    norm, out = go.clip_grads([np.array([np.inf]), np.array([1.0])], 1.0)
    assert norm == np.inf and out[1][0] == 1.0
    assert go.clip_grads([], 1.0)[0] == 0.0
    big = np.full(3, 1e30, dtype=np.float32)           # squares beyond fp32
    assert go.clip_grads([big], 1.0)[0] == pytest.approx(math.sqrt(3) * float(big[0]))


def test_planted_mistakes_are_seen():
    T, E, k = 4, 6, 3
    rng, scores, idx = batch(T, E, k, 5)
    dw = rng.standard_normal((T, k))
    right = go.route_backward(scores, idx, dw, None, 0, 1)
    # the renormalised gradient without the renormalisation, and one that forgets the inner sum
    w = go.routing_weights(scores, idx, 1)
    forgets = np.zeros((T, E))
    np.put_along_axis(forgets, idx.astype(np.int64), w * dw, axis=1)
    assert np.abs(go.route_backward(scores, idx, dw, None, 0, 0) - right).max() > 1e-2
    assert np.abs(forgets - right).max() > 1e-2
    # a mean over all tokens instead of those that count
    mask = np.array([1, 1, 0, 0])
    target = rng.standard_normal((T, E))
    loss, _ = go.gate_distill(scores, target, 1.0, mask)
    assert loss == pytest.approx(go.gate_distill(scores[:2], target[:2])[0], rel=1e-14)
    assert abs(loss * mask.sum() / T - loss) > 1e-3


def test_nan_scores_are_seen():
    rng = np.random.default_rng(6)
    for table in (0, 1):
        for row in ([np.nan] * 4, [0.3, np.nan, 1.0, -2.0], [-np.inf, np.nan, -np.inf, -np.inf]):
            tables = [rng.standard_normal((3, 4)) for _ in range(2)]
            tables[table][1] = row
            loss, grad = go.gate_distill(*tables)
            assert math.isnan(loss) and np.isnan(grad[1]).all() and np.isfinite(grad[[0, 2]]).all()
            assert np.isfinite(go.gate_distill(*tables, 1.0, np.array([1, 0, 1]))[0])
    assert np.isnan(go.balance_loss(np.array([[np.nan, 1.0]]), np.zeros((1, 1), dtype=np.int32))[1]).all()
