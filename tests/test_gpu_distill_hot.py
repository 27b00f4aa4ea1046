"""The distillation loss at high temperatures: its terms are about T^2 log d and more, what they add up to is of the size
of the scores' and values' squared differences.

Bounds against the fp64 oracle, u = 2^-24, D the spread of a row's scores over T, the loss T^2 (1 - w) L + w (...):
* sum_j exp(x_j), x_j = (a_j - m) / T: with 1 + x taken exactly, phi(x) = exp(x) - 1 - x carries 3u in x (twice that in
  phi), its polynomial and the sum of 16 terms 20u: 26u phi, phi <= x^2 / 2; where |x| > 1/2, exp(x) carries
  (5 |x| + 17) u.  The running maximum moves by D in all, each move with an exponential of the same kind: 6u D^2 more or
  13u D more.  So log s is off by at most u 40 D^2 for D <= 1/2, else by u (20 D + 30).
* q_t: exp((v_t - v_max) / T) is off by r_t = 12u x^2 / 2, or (5 |x| + 4) u where |x| > 1/2; for log probabilities r_t =
  (3 |v_t| + 4) u.  L changes by at most sum_t q_t r_t (1 + |log q_t - log p_t| + |L|).
* exponentials below 2^-126 are 0, as documented: each place lacks at most 2^-126 (1 + |log q_t - log p_t| + |L|).
* what is 64 bits: 2^-50 of the magnitudes; (1 - w) T^2, w and the result are rounded: 3u |loss|.
* the label's term: log sum exp in fp32 as elsewhere, u (d / 16 + 30 + 3 E|z|) + 8u (log s1 + |z_y|).
A factor of 2 on the whole for second-order terms.
"""
import numpy as np
import pytest
import torch

from oracle import scores as osc

pytestmark = pytest.mark.gpu

import gpu_util as gu  # noqa: E402
from paper_2211_12858_amd import _lib as L  # noqa: E402
from paper_2211_12858_amd.driver import workspace  # noqa: E402
from test_gpu_distill import run  # noqa: E402

U = 2.0 ** -24


def bound(F, ids, vals, T, w, y, kind, loss):
    n, d = F.shape
    a = F.astype(np.float64)
    tol = np.zeros(n)
    for i in range(n):
        q, lq = osc.teacher_probs(ids[:, i], vals[:, i], d, T, kind)
        on = q > 0
        lp = osc.log_softmax(a[i], T)
        D = np.ptp(a[i][np.isfinite(a[i])]) / T
        Q = q.sum()
        diff = lq[on] - lp[ids[on, i]]
        if kind == "logits":
            x = (vals[on, i].max() - vals[on, i].astype(np.float64)) / T if on.any() else np.zeros(0)
            r = U * np.where(x <= 0.5, 6 * x * x, 5 * x + 4)
        else:
            r = U * (3 * np.abs(vals[on, i].astype(np.float64)) + 4)
        L = (q[on] * diff).sum()
        tol[i] = Q * U * (40 * D * D if D <= 0.5 else 20 * D + 30) + (q[on] * r * (1 + np.abs(diff) + abs(L))).sum()
        tol[i] += 2.0 ** -126 * (1 + np.abs(diff) + abs(L)).sum()
        tol[i] += 2.0 ** -50 * (Q * np.log(d) + Q * D + (q[on] * np.abs(lq[on])).sum())
        tol[i] *= (1.0 - w) * T * T
        if w and 0 <= y[i] < d:
            z = a[i] - a[i].max()
            p = np.exp(z)
            tol[i] += w * U * (d / 16 + 30 + 3 * (p * np.abs(z))[p > 0].sum() / p.sum()
                               + 8 * (np.log(p.sum()) + np.abs(z[y[i]])))
    return 2 * (tol + 3 * U * np.abs(loss))


def teacher_lists(rng, F, k, T, kind, noise):
    """The k best classes of a teacher whose scores are the student's with noise."""
    n, d = F.shape
    z = F + (rng.normal(size=(n, d)) * noise).astype(np.float32)
    ids = np.argsort(-z, axis=1, kind="stable")[:, :k]
    v = np.take_along_axis(z, ids, axis=1)
    if kind == "log_probs":
        x = z.astype(np.float64) / T
        m = x.max(axis=1, keepdims=True)
        lse = m + np.log(np.exp(x - m).sum(axis=1, keepdims=True))
        v = (v.astype(np.float64) / T - lse).astype(np.float32)
    return np.ascontiguousarray(ids.T.astype(np.int32)), np.ascontiguousarray(v.T.astype(np.float32))


def one(F, ids, vals, T, w, y, kind, some=slice(None)):
    fwd, got = run(F, ids, vals, T, w, y, kind)
    ys = None if y is None else y[some]
    want, _, _ = osc.distill(F[some], ids[:, some], vals[:, some], T, w, ys, kind)
    tol = bound(F[some], ids[:, some], vals[:, some], T, w, ys, kind, want)
    for name, loss in (("forward", fwd[some]), ("gradients", got["loss"][some])):
        off = np.abs(loss - want)
        assert np.all(off <= tol), (name, T, off.max(), tol[off.argmax()], want[off.argmax()])
    return fwd[some], want, tol


@pytest.mark.parametrize("T", [5.0, 20.0, 100.0, 1000.0, 10_000.0])
@pytest.mark.parametrize("kind,w", [("logits", 0.0), ("logits", 0.3), ("log_probs", 0.0)])
@pytest.mark.parametrize("n,d,k", [(1, 1, 1), (70, 2, 2), (300, 10, 10), (257, 50, 50), (64, 64, 64), (65, 100, 10),
                                   (33, 700, 20), (40, 1024, 64), (70, 1100, 64), (3, 9001, 64), (2, 65_535, 20)])
def test_hot(n, d, k, kind, w, T):
    print("case: hot", n, d, k, kind, w, T, flush=True)
    rng = np.random.default_rng(n + d + k)
    F = rng.normal(size=(n, d)).astype(np.float32)
    ids, vals = teacher_lists(rng, F, k, T, kind, 0.5)
    ids[k // 2:, 5::9], vals[k // 2:, 5::9] = -1, np.nan
    y = None
    if w:
        y = rng.integers(-1, d + 1, n).astype(np.int32)
    fwd, want, tol = one(F, ids, vals, T, w, y, kind)
    if kind == "logits":
        assert np.all(fwd >= -tol)
    if kind == "logits" and k == d and not w and T >= 20.0:
        # the whole teacher: what the bound allows is one of the squared spread, whatever T is.  D and x are at most
        # spread / T <= 1/2 here, |log q - log p| and |L| at most 1, so 40 D^2 + 6 x^2 (1 + 1 + 1) <= 58 (spread / T)^2;
        # 3u |loss|, |loss| <= spread^2; fp64's part is 2^-50 T^2 (2 log d + 2)
        full = np.all(ids >= 0, axis=0)
        spread = np.maximum(np.ptp(F, axis=1), np.ptp(vals, axis=0))
        assert np.all(tol[full] <= (2 * 61 * U * spread ** 2 + 2.0 ** -48 * T * T * (1 + np.log(d)))[full])


@pytest.mark.parametrize("T", [6.0, 300.0])
@pytest.mark.parametrize("n,d,k", [(100_003, 41, 1), (150_001, 10, 3), (30_011, 300, 5), (20_001, 1500, 16)])
def test_many_rows(n, d, k, T):
    print("case: hot", n, d, k, T, flush=True)
    rng = np.random.default_rng(n)
    F = rng.normal(size=(n, d)).astype(np.float32)
    ids = ((rng.integers(0, d, n)[None, :] + np.arange(k)[:, None] * (d // k)) % d).astype(np.int32)
    vals = rng.normal(size=(k, n)).astype(np.float32)
    y = rng.integers(-1, d, n).astype(np.int32)
    some = np.unique(np.concatenate([[0, 63, 64, n - 65, n - 64, n - 2, n - 1], rng.integers(0, n, 200)]))
    a, _, _ = one(F, ids, vals, T, 0.2, y, "logits", some)
    b, _, _ = one(F, ids, vals, T, 0.2, y, "logits", some)
    assert np.array_equal(a, b)


@pytest.mark.parametrize("T", [20.0, 1000.0])
@pytest.mark.parametrize("kind", ["logits", "log_probs"])
@pytest.mark.parametrize("d", [10, 300, 1500])
def test_far_scores_and_excluded_classes(d, kind, T):
    """Spreads of up to many T, rising columns (the running maximum moves with every step), excluded classes."""
    rng = np.random.default_rng(d)
    n, k = 150, 10
    F = (rng.normal(size=(n, d)) * np.array([1.0, 30.0, 3000.0])[np.arange(n) % 3, None]).astype(np.float32)
    F[50:100] = np.sort(F[50:100], axis=1)
    F[100:] += np.float32(5000.0)
    ids, vals = teacher_lists(rng, F, k, T, kind, 1.0)
    F[::2, 0] = -np.inf
    F[1::2, d // 2] = np.finfo(np.float32).min
    hit = (ids == np.where(np.arange(n) % 2 == 0, 0, d // 2)[None, :])
    ids[hit], vals[hit] = -1, np.nan
    low = F.copy()
    low[~(low > -1e30)] = -1e6 * T  # of probability 0 in fp64 as well
    fwd, got = run(F, ids, vals, T, 0.0, None, kind)
    want, _, _ = osc.distill(low, ids, vals, T, 0.0, None, kind)
    tol = bound(np.where(low > -1e6 * T, low, -np.inf), ids, vals, T, 0.0, None, kind, want)
    for loss in (fwd, got["loss"]):
        assert np.all(np.abs(loss - want) <= tol)
    ids[0, 0], vals[0, 0] = 0, 0.0  # an excluded class as a target
    F[2] = -np.inf                  # every class
    ids[:, 4], vals[:, 4] = -1, np.nan  # no place
    fwd, got = run(F, ids, vals, T, 0.0, None, kind)
    for loss in (fwd, got["loss"]):
        assert loss[0] == np.inf and loss[2] == np.inf and loss[4] == 0.0


def test_forward_and_gradient_calls_agree():
    rng = np.random.default_rng(1)
    for n, d, k in ((100_003, 60, 1), (500, 60, 9), (70, 900, 9), (70, 1300, 9)):
        F = rng.normal(size=(n, d)).astype(np.float32)
        ids, vals = rng.integers(0, d, (k, n)).astype(np.int32), rng.normal(size=(k, n)).astype(np.float32)
        fwd, got = run(F, ids, vals, 50.0, 0.0, None, "logits")
        assert np.array_equal(fwd, got["loss"])
        # the other outputs do not depend on whether the loss is asked for
        _, part = run(F, ids, vals, 50.0, 0.0, None, "logits", loss=False)
        for name in part:
            assert np.array_equal(part[name], got[name]), name


@pytest.mark.parametrize("n,d,k,ld", [(70, 20, 5, 3), (65, 700, 9, 5), (5, 3001, 6, 3), (70, 9, 3, (1 << 27) + 1)])
def test_strides_and_offsets_past_32_bits(n, d, k, ld):
    rng = np.random.default_rng(n + d)
    F = rng.normal(size=(n, d)).astype(np.float32)
    ids, vals = teacher_lists(rng, F, k, 50.0, "logits", 0.5)
    plain, _ = run(F, ids, vals, 50.0, 0.0, None, "logits")
    fwd, got = run(F, ids, vals, 50.0, 0.0, None, "logits", ld=ld)
    assert np.array_equal(fwd, plain) and np.array_equal(got["loss"], plain)


@pytest.mark.parametrize("d", [5, 100, 1600])
def test_nan_and_inf_stay_in_their_row(d):
    rng = np.random.default_rng(d)
    F = rng.normal(size=(70, d)).astype(np.float32)
    ids, vals = teacher_lists(rng, F, 5, 10.0, "logits", 0.5)
    y = rng.integers(0, d, 70).astype(np.int32)
    want, _ = run(F, ids, vals, 10.0, 0.3, y, "logits")
    F[3, 0], F[64, d - 1], F[69, 2], vals[1, 20] = np.nan, np.inf, np.nan, np.nan
    fwd, _ = run(F, ids, vals, 10.0, 0.3, y, "logits")
    keep = np.setdiff1d(np.arange(70), [3, 20, 64, 69])
    assert np.array_equal(fwd[keep], want[keep])


@pytest.mark.parametrize("n,d", [(300, 100), (200, 1500)])
def test_captured_and_replayed(n, d):
    """Replayed on changed scores between eager work; one workspace each for the graph and the eager calls."""
    print("case: hot graph", n, d, flush=True)
    rng = np.random.default_rng(d)
    F0 = rng.normal(size=(n, d)).astype(np.float32)
    ids, vals = teacher_lists(rng, F0, 5, 20.0, "log_probs", 0.5)
    M, idd, vd = torch.zeros((d, n), device=gu.DEV), gu.up(ids), gu.up(vals)
    loss, G = torch.zeros(n, device=gu.DEV), torch.zeros((d, n), device=gu.DEV)
    ws = workspace(L.sb_workspace_bytes(L.SB_CALL_DISTILL, n=n, d=d, k=5), gu.DEV)

    def call():
        L.sb_distill_gradients(M, n, d, n, 20.0, 0.0, None, 1, 5, idd, vd, n, loss, G, n, None, 0, None, None, ws, ws.numel())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    gu.sync()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for rep in range(3):
        F = rng.normal(size=(n, d)).astype(np.float32)
        M.copy_(gu.up(np.ascontiguousarray(F.T)))
        g.replay()
        gu.sync()
        _, eager = run(F, ids, vals, 20.0, 0.0, None, "log_probs", hess=False, row=False, norms=False)
        assert np.array_equal(loss.cpu().numpy(), eager["loss"]) and np.array_equal(G.cpu().numpy(), eager["G"]), rep
