"""Pins of the oracle's score-row operators: known values, identities, and derivatives against differences (no GPU)."""
import math

import numpy as np
import pytest

from oracle import boost as ob
from oracle import scores as osc


def test_known_values():
    r = osc.log_probs([[math.log(1.0), math.log(2.0), math.log(1.0)]], labels=[2], k=4)
    assert r["lse"][0] == pytest.approx(math.log(4.0))
    assert r["logp"][0] == pytest.approx(math.log(0.25))
    assert r["rank"][0] == 2  # after class 1, and after class 0 of the same score
    assert r["entropy"][0] == pytest.approx(1.5 * math.log(2.0))
    assert r["top_id"][:, 0].tolist() == [1, 0, 2, -1]
    assert r["top_logp"][0, 0] == pytest.approx(math.log(0.5)) and r["top_logp"][3, 0] == -np.inf


def test_excluded_classes():
    r = osc.log_probs([[-np.inf, 3.0, -np.inf], [-np.inf] * 3], labels=[0, 1], k=2)
    assert r["lse"].tolist() == [3.0, -np.inf] and r["entropy"].tolist() == [0.0, 0.0]
    assert r["logp"].tolist() == [-np.inf, -np.inf] and r["rank"].tolist() == [1, 1]
    assert r["top_id"].tolist() == [[1, -1], [-1, -1]]


def test_temperature_divides_the_scores():
    a = np.random.default_rng(0).normal(size=(3, 7))
    x, y = osc.log_probs(a, T=2.5, k=3, labels=[0, 1, 6]), osc.log_probs(a / 2.5, k=3, labels=[0, 1, 6])
    for name in ("lse", "entropy", "logp", "top_logp"):
        assert np.allclose(x[name], y[name], rtol=1e-12)
    assert np.array_equal(x["top_id"], y["top_id"])


def lists(rng, n, d, k):
    ids = np.stack([rng.permutation(max(d, k))[:k] for _ in range(n)], 1).astype(np.int32)
    ids[ids >= d] = -1
    return ids, rng.normal(size=(k, n)) * 2


def test_a_full_list_at_temperature_one_is_the_cross_entropy_of_soft_labels():
    rng = np.random.default_rng(1)
    n, d = 4, 6
    F, Z = rng.normal(size=(n, d)), rng.normal(size=(n, d))
    ids = np.tile(np.arange(d, dtype=np.int32)[:, None], (1, n))
    _, g, h = osc.distill(F, ids, Z.T, kind="logits")
    p, q = np.exp(F), np.exp(Z)
    p, q = p / p.sum(1, keepdims=True), q / q.sum(1, keepdims=True)
    assert np.allclose(g, p - q) and np.allclose(h, p * (1 - p))


def test_all_weight_on_the_label_is_the_softmax_loss():
    rng = np.random.default_rng(2)
    F, y = rng.normal(size=(5, 4)), np.array([0, 3, 1, 2, 2], dtype=np.int32)
    ids, vals = lists(rng, 5, 4, 3)
    loss, g, h = osc.distill(F, ids, vals, T=3.0, w=1.0, labels=y)
    g0, h0 = ob.softmax_ce_derivatives(F, y)
    assert np.allclose(loss, ob.softmax_ce_loss(F, y)) and np.allclose(g, g0) and np.allclose(h, h0)


@pytest.mark.parametrize("kind", ["logits", "log_probs"])
@pytest.mark.parametrize("T,w", [(1.0, 0.0), (2.0, 0.3), (0.5, 1.0)])
def test_derivatives_against_differences(kind, T, w):
    rng = np.random.default_rng(3)
    n, d, k = 3, 5, 4
    F, y = rng.normal(size=(n, d)), np.array([1, -1, 4], dtype=np.int32)
    ids, vals = lists(rng, n, d, k)
    ids[0, 1], ids[1, 0] = -1, ids[2, 0]  # an unused place; one class twice
    vals[0, 1] = np.nan
    if kind == "log_probs":
        vals = -np.abs(np.nan_to_num(vals)) - 1.0
    loss, g, h = osc.distill(F, ids, vals, T=T, w=w, labels=y, kind=kind)
    eps = 1e-5
    for j in range(d):
        P, M = F.copy(), F.copy()
        P[:, j] += eps
        M[:, j] -= eps
        lp, gp, _ = osc.distill(P, ids, vals, T=T, w=w, labels=y, kind=kind)
        lm, gm, _ = osc.distill(M, ids, vals, T=T, w=w, labels=y, kind=kind)
        # central differences: error eps^2 times a third derivative (below 10 here) plus fp64 rounding over eps
        assert np.allclose((lp - lm) / (2 * eps), g[:, j], atol=1e-8)
        assert np.allclose((gp - gm)[:, j] / (2 * eps), h[:, j], atol=1e-8)


def test_rows_without_label_and_list_are_zero():
    loss, g, h = osc.distill([[1.0, 2.0]], np.array([[-1], [2]]), np.array([[np.nan], [1.0]]), T=2.0, w=0.5, labels=[-1])
    assert loss[0] == 0 and not g.any() and not h.any()
