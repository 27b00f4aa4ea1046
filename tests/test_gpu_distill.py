"""sb_distill_loss and sb_distill_gradients against the fp64 oracle, and the booster that learns from a teacher.

Bounds, u = 2^-24, second-order terms and the oracle's own roundings in a factor of 2 on the whole:
z = a - m has one rounding, z / T two more, an exponential at most 4u, a sum of d terms S = d/16 + 24 adds deep, so
with E over the student's distribution eps(p_j) = u (S + 16 + 3 |z_j| / T + 3 E|z| / T); a teacher's probability
eps(q_t) = u (k + 16 + 3 |v_t - v_max| / T) (the list's own values are exact); the products and sums of g, h and the
loss add at most (k + 8) u of the magnitudes that they add.
"""
import numpy as np
import pytest
import torch

from oracle import scores as osc

pytestmark = pytest.mark.gpu

import gpu_util as gu  # noqa: E402
from paper_2211_12858_amd import _lib as L  # noqa: E402
from paper_2211_12858_amd.driver import workspace  # noqa: E402

U = 2.0 ** -24
MARK = 12345.0


def up_cm(X, ld):
    """(rows, cols) host array as a column-major device matrix of the given leading dimension; gaps hold NaN or -1."""
    n, d = X.shape
    fill = float("nan") if X.dtype == np.float32 else 12345
    M = torch.full((d, ld), fill, dtype=torch.float32 if X.dtype == np.float32 else torch.int32, device=gu.DEV)
    M[:, :n] = gu.up(np.ascontiguousarray(X.T))
    return M


def run(F, t_id, t_val, T, w, labels, kind, hess=True, row=True, norms=True, loss=True, ld=0, stream=None):
    """(forward loss, dict of the gradient call's outputs); ld: added to every leading dimension."""
    n, d = F.shape
    k = t_id.shape[0]
    lf, lt, lg, lh = (n + ld * i for i in (1, 2, 3, 4))
    Fd, idd, vd = up_cm(F, lf), up_cm(np.ascontiguousarray(t_id.T), lt), up_cm(np.ascontiguousarray(t_val.T), lt)
    y = None if labels is None else gu.up(labels)
    ws = workspace(L.sb_workspace_bytes(L.SB_CALL_DISTILL, n=n, d=d, k=k), gu.DEV)
    fwd = torch.full((n,), MARK, device=gu.DEV)
    L.sb_distill_loss(Fd, n, d, lf, T, w, y, L.TEACHER[kind], k, idd, vd, lt, fwd, ws, ws.numel(), stream)
    o = {"G": torch.full((d, lg), MARK, device=gu.DEV)}
    if hess:
        o["hess"] = torch.full((d, lh), MARK, device=gu.DEV)
    if row:
        o["h_row"] = torch.full((n,), MARK, device=gu.DEV)
    if norms:
        o["norm2"] = torch.full((d,), MARK, dtype=torch.float64, device=gu.DEV)
    if loss:
        o["loss"] = torch.full((n,), MARK, device=gu.DEV)
    L.sb_distill_gradients(Fd, n, d, lf, T, w, y, L.TEACHER[kind], k, idd, vd, lt, o.get("loss"), o["G"], lg,
                           o.get("hess"), lh, o.get("h_row"), o.get("norm2"), ws, ws.numel(), stream)
    gu.sync()
    got = {name: t.cpu().numpy() for name, t in o.items()}
    for name in ("G", "hess"):
        if name in got:
            assert np.all(got[name][:, n:] == MARK), "rows behind the last one are left as they were"
            got[name] = got[name][:, :n]
    return fwd.cpu().numpy(), got


def check(F, t_id, t_val, T, w, labels, kind, fwd, got, rows=None):
    n, d = F.shape
    if "norm2" in got:
        G = got["G"].astype(np.float64)
        # fp64 sums of the stored values: n adds of one rounding each
        assert np.allclose(got["norm2"], (G * G).sum(axis=1), rtol=1e-12, atol=0.0)
    rows = np.arange(n) if rows is None else rows
    F, t_id, t_val = F[rows].astype(np.float64), t_id[:, rows], t_val[:, rows]
    labels = None if labels is None else labels[rows]
    k = t_id.shape[0]
    loss, g, h = osc.distill(F, t_id, t_val, T, w, labels, kind)
    S = d / 16 + 24
    z = F - F.max(axis=1, keepdims=True)
    tl, tg, th, lt = np.zeros(len(rows)), np.zeros_like(g), np.zeros_like(g), np.zeros(len(rows))

    def student(temp):
        p = np.exp(z / temp)
        s = p.sum(axis=1, keepdims=True)
        p /= s
        ez = (p * np.abs(z)).sum(axis=1, keepdims=True) / temp
        return p, U * (S + 16 + 3 * np.abs(z) / temp + 3 * ez), np.abs(np.log(s[:, 0])), U * (S + 6 + 3 * ez[:, 0])

    pT, eT, lsT, dT = student(T)
    p1, e1, ls1, d1 = student(1.0)
    for i in range(len(rows)):
        q, lq = osc.teacher_probs(t_id[:, i], t_val[:, i], d, T, kind)
        on = q > 0
        v = t_val[on, i].astype(np.float64)
        dv = (v.max() - v) / T if kind == "logits" and on.any() else 0.0
        eq = np.zeros(k)
        eq[on] = U * (k + 16 + 3 * dv)
        Q, B = q.sum(), (1.0 - w) * T
        eQ = (q * eq).sum() / max(Q, 1e-300) + U * (k + 4)
        A = w if labels is not None and 0 <= labels[i] < d else 0.0
        # magnitudes that meet in g, h and the loss, with their relative errors
        tg[i] += A * p1[i] * e1[i] + B * Q * pT[i] * (eT[i] + eQ)
        mag = A * p1[i] + B * Q * pT[i]
        th[i] = A * p1[i] * 2 * e1[i] + (1.0 - w) * Q * pT[i] * (2 * eT[i] + eQ)
        tl[i] += A * (d1[i] + 4 * U * ls1[i]) + B * T * Q * (dT[i] + 4 * U * lsT[i] + eQ * lsT[i])
        lmag = A * ls1[i] + B * T * Q * lsT[i]
        for t in np.nonzero(on)[0]:
            c = t_id[t, i]
            tg[i, c] += B * q[t] * eq[t]
            mag[c] += B * q[t]
            tl[i] += B * T * q[t] * (abs(lq[t]) * eq[t] + eq[t]) + B * q[t] * abs(z[i, c]) * eq[t]
            lmag += B * T * q[t] * abs(lq[t]) + B * q[t] * abs(z[i, c])
        if A:
            mag[labels[i]] += A
            lmag += A * abs(z[i, labels[i]])
        tg[i] += U * (k + 8) * mag
        th[i] += 8 * U * h[i]
        tl[i] += U * (k + 8) * lmag
        lt[i] = lmag
    # exponentials below 2^-126 of the row's largest are 0, as documented: p lacks at most 2^-126, g at most
    # (w + (1 - w) T Q) 2^-126 and h no more, Q <= 64 here
    tiny = 2.0 ** -126 * (1 + 64 * T)

    def close(name, gotv, want, tol):
        bad = ~(np.abs(gotv.astype(np.float64) - want) <= 2 * tol + tiny)
        assert not bad.any(), (name, np.argwhere(bad)[:5], gotv[bad][:5], want[bad][:5], tol[bad][:5])

    close("G", got["G"].T[rows], g, tg)
    if "hess" in got:
        close("hess", got["hess"].T[rows], h, th)
    if "h_row" in got:
        close("h_row", got["h_row"][rows], h.mean(axis=1), th.mean(axis=1) + U * (S + 4) * h.mean(axis=1))
    # the loss adds d terms target * z as well, all but k + 1 of them zero
    close("forward loss", fwd[rows], loss, tl)
    if "loss" in got:
        close("loss", got["loss"][rows], loss, tl)
    return g, h


def inputs(rng, n, d, k, kind, spread=2.0, labelled=True):
    """Student scores, a teacher's lists (rows with all, some and no places used; unused ones hold NaN) and labels."""
    F = (rng.normal(size=(n, d)) * spread).astype(np.float32)
    ids = np.empty((k, n), dtype=np.int32)
    for i in range(n):
        ids[:, i] = rng.permutation(d)[:k] if k <= d else rng.integers(0, d, k)
    vals = np.sort(rng.normal(size=(k, n)) * 2, axis=0)[::-1].astype(np.float32)
    if kind == "log_probs":
        vals = (vals - np.log(np.exp(vals.astype(np.float64)).sum(axis=0)) - rng.random(n)).astype(np.float32)
    for i in range(n):
        r = rng.random()
        used = 0 if r < 0.1 else (k + 1) // 2 if r < 0.25 else k
        ids[used:, i] = rng.choice([-1, d, -2 ** 31, 2 ** 31 - 1], k - used)
        vals[used:, i] = rng.choice([np.nan, np.inf, -np.inf, 5.0], k - used)
    y = None
    if labelled:
        y = rng.integers(0, d, n).astype(np.int32)
        y[rng.random(n) < 0.1] = -1
        y[rng.random(n) < 0.05] = d
    return F, np.ascontiguousarray(ids), np.ascontiguousarray(vals), y


# From one row and one class on; around the column widths of a wave and of a block, lists longer than the classes, odd
# row counts; each with both kinds of teacher and with labels, without, and at one temperature and two.
@pytest.mark.parametrize("kind,T,w", [("logits", 1.0, 0.5), ("logits", 2.0, 0.3), ("log_probs", 0.7, 0.0),
                                      ("log_probs", 1.0, 1.0)])
@pytest.mark.parametrize("n,d,k", [(1, 1, 1), (1, 1, 64), (3, 2, 2), (64, 5, 8), (65, 8, 3), (130, 9, 64), (63, 16, 5),
                                   (257, 17, 10), (64, 24, 7), (100, 25, 12), (40, 28, 64), (70, 32, 32), (129, 33, 6),
                                   (66, 57, 9), (200, 64, 40), (77, 100, 10), (33, 104, 64), (64, 113, 5), (31, 128, 20),
                                   (97, 203, 33), (50, 480, 64), (65, 512, 10), (64, 513, 64), (33, 640, 12),
                                   (63, 1000, 32), (32, 1024, 64), (5, 1025, 3), (70, 1100, 64), (9, 2500, 10),
                                   (3, 9001, 64), (2, 65_535, 20)])
def test_shapes(n, d, k, kind, T, w):
    print("case: distill", n, d, k, kind, T, w, flush=True)
    rng = np.random.default_rng(n * 1000 + d + k)
    F, ids, vals, y = inputs(rng, n, d, k, kind, labelled=w > 0)
    check(F, ids, vals, T, w, y, kind, *run(F, ids, vals, T, w, y, kind))


@pytest.mark.parametrize("n,d,k,kind,T,w", [(200_003, 10, 3, "logits", 1.0, 0.5), (150_001, 30, 30, "log_probs", 2.0, 0.2),
                                            (100_007, 100, 10, "logits", 2.0, 0.3), (30_011, 300, 64, "logits", 1.5, 0.0),
                                            (20_001, 600, 8, "log_probs", 1.0, 0.0), (12_345, 1000, 32, "logits", 4.0, 0.1),
                                            (9_001, 1500, 16, "logits", 2.0, 0.5), (100_003, 370, 9, "logits", 2.0, 0.4),
                                            (100_001, 41, 1, "log_probs", 1.0, 0.0),
                                            (100_031, 1030, 10, "logits", 0.8, 0.0)])
def test_many_rows(n, d, k, kind, T, w):
    print("case: distill", n, d, k, kind, T, w, flush=True)
    rng = np.random.default_rng(n + d + k)
    F = (rng.normal(size=(n, d)) * 2).astype(np.float32)
    ids = ((rng.integers(0, d, n)[None, :] + np.arange(k)[:, None] * (d // k)) % d).astype(np.int32)
    vals = (rng.normal(size=(k, n)) - (4.0 if kind == "log_probs" else 0.0)).astype(np.float32)
    ids[k // 2:, ::7] = -1
    ids[:, ::31] = -1
    y = rng.integers(-1, d, n).astype(np.int32) if w > 0 else None
    rows = np.unique(np.concatenate([[0, 63, 64, n - 65, n - 64, n - 2, n - 1], rng.integers(0, n, 300)]))
    fwd, got = run(F, ids, vals, T, w, y, kind)
    check(F, ids, vals, T, w, y, kind, fwd, got, rows)
    fwd2, got2 = run(F, ids, vals, T, w, y, kind)
    assert np.array_equal(fwd, fwd2)
    for name in got:
        assert np.array_equal(got[name], got2[name]), name


@pytest.mark.parametrize("n,d,k", [(70, 20, 5), (65, 100, 10), (31, 700, 9), (5, 3001, 6)])
def test_strides(n, d, k):
    rng = np.random.default_rng(d)
    F, ids, vals, y = inputs(rng, n, d, k, "logits")
    check(F, ids, vals, 2.0, 0.4, y, "logits", *run(F, ids, vals, 2.0, 0.4, y, "logits", ld=3))


@pytest.mark.parametrize("d", [3, 40, 300, 900, 2000])
def test_a_class_listed_more_than_once(d):
    rng = np.random.default_rng(d)
    n, k = 66, 12
    F, _, vals, y = inputs(rng, n, d, k, "logits")
    ids = rng.integers(0, 3, (k, n)).astype(np.int32)  # three classes for twelve places
    vals = rng.normal(size=(k, n)).astype(np.float32)
    y[:] = 1  # which is among them
    check(F, ids, vals, 2.0, 0.5, y, "logits", *run(F, ids, vals, 2.0, 0.5, y, "logits"))


@pytest.mark.parametrize("kind", ["logits", "log_probs"])
@pytest.mark.parametrize("d", [6, 100, 1500])
def test_empty_rows_are_zero(d, kind):
    """No label and no used place, or only values of -inf: no gradient, no hessian, no loss, whatever unused places hold."""
    rng = np.random.default_rng(d)
    n, k = 130, 5
    F, ids, vals, y = inputs(rng, n, d, k, kind)
    ids[:, :64], vals[:, :64], y[:64] = -1, np.nan, -1
    vals[:, 100], ids[:, 100], y[100] = -np.inf, 0, d
    fwd, got = run(F, ids, vals, 2.0, 0.3, y, kind)
    for i in list(range(64)) + [100]:
        assert fwd[i] == 0 and got["loss"][i] == 0 and got["h_row"][i] == 0
        assert not got["G"][:, i].any() and not got["hess"][:, i].any()
    check(F, ids, vals, 2.0, 0.3, y, kind, fwd, got)


@pytest.mark.parametrize("d", [7, 100, 600, 1400])
def test_far_scores(d):
    rng = np.random.default_rng(d)
    F, ids, vals, y = inputs(rng, 40, d, 5, "logits", spread=300.0)
    vals[:, :20] *= 500.0
    for T in (0.01, 1.0, 1000.0):
        check(F, ids, vals, T, 0.5, y, "logits", *run(F, ids, vals, T, 0.5, y, "logits"))


@pytest.mark.parametrize("n,d", [(70, 8), (70, 60), (65, 300), (40, 900), (5, 1600)])
@pytest.mark.parametrize("T,w", [(1.0, 0.4), (2.0, 0.4), (3.0, 0.0)])
def test_excluded_classes(n, d, T, w):
    """A score of -inf is one so low that its probability is 0 in fp64 as well; a target on it makes the loss +inf."""
    rng = np.random.default_rng(d)
    F, ids, vals, y = inputs(rng, n, d, 5, "logits")
    out = rng.random((n, d)) < 0.3
    for i in range(n):  # no target is excluded, but those of the last rows
        used = (ids[:, i] >= 0) & (ids[:, i] < d)
        out[i, ids[used, i]] = False
        out[i, 0] = False
        if 0 <= y[i] < d:
            out[i, y[i]] = False
    ids[0, n - 3:], vals[0, n - 3:] = d - 1, 1.0
    out[n - 3:, d - 1] = True
    out[n - 2] = True  # every class
    X, low = np.where(out, np.float32(-np.inf), F), np.where(out, np.float32(-1e4), F)
    fwd, got = run(X, ids, vals, T, w, y, "logits")
    hit = np.arange(n - 3, n)
    assert np.all(fwd[hit] == np.inf) and np.all(got["loss"][hit] == np.inf)
    _, g, h = osc.distill(X[hit], ids[:, hit], vals[:, hit], T, w, y[hit], "logits")
    # q eps(q) <= u (5 + 16 + 3 * 13), p eps(p) <= u (25 + 16 + 6 * 7) where p is near 1, less for more classes; g adds
    # them with w and (1 - w) T, h has p eps(p) twice
    assert np.allclose(got["G"].T[hit], g, rtol=0, atol=256 * U * max(T, 1.0))
    assert np.allclose(got["hess"].T[hit], h, rtol=0, atol=256 * U)
    assert not got["hess"][:, n - 2].any() and got["h_row"][n - 2] == 0
    keep = np.arange(n - 3)
    check(low, ids, vals, T, w, y, "logits", fwd, got, keep)


@pytest.mark.parametrize("d", [30, 400])
def test_excluded_classes_in_many_rows(d):
    rng = np.random.default_rng(d)
    n, k = 100_003, 1
    F = rng.normal(size=(n, d)).astype(np.float32)
    ids, vals = rng.integers(0, d // 2, (k, n)).astype(np.int32), rng.normal(size=(k, n)).astype(np.float32)
    ids[0, n - 1] = d - 1
    low = F.copy()
    low[:, d // 2:] = -1e4
    F[:, d // 2:] = -np.inf
    F[n - 2] = -np.inf
    ids[0, n - 2] = -1
    fwd, got = run(F, ids, vals, 2.0, 0.0, None, "logits")
    assert fwd[n - 1] == np.inf and fwd[n - 2] == 0 and got["loss"][n - 1] == np.inf and got["loss"][n - 2] == 0
    check(low, ids, vals, 2.0, 0.0, None, "logits", fwd, got, np.concatenate([np.arange(200), np.arange(n - 70, n - 2)]))


@pytest.mark.parametrize("d", [5, 100, 700, 1600])
def test_nan_and_inf_stay_in_their_row(d):
    rng = np.random.default_rng(d)
    F, ids, vals, y = inputs(rng, 70, d, 5, "logits")
    _, want = run(F, ids, vals, 2.0, 0.3, y, "logits", norms=False)
    bad = F.copy()
    bad[3, 0], bad[64, d - 1], bad[69, 2] = np.nan, np.inf, np.nan
    fwd, got = run(bad, ids, vals, 2.0, 0.3, y, "logits", norms=False)
    keep = np.setdiff1d(np.arange(70), [3, 64, 69])
    for name in want:
        assert np.array_equal(got[name][..., keep], want[name][..., keep]), name


@pytest.mark.parametrize("d", [12, 100, 700, 1600])
def test_outputs_are_optional(d):
    rng = np.random.default_rng(d)
    F, ids, vals, y = inputs(rng, 100, d, 4, "logits")
    _, whole = run(F, ids, vals, 2.0, 0.3, y, "logits")
    for off in ("hess", "row", "norms", "loss"):
        _, part = run(F, ids, vals, 2.0, 0.3, y, "logits", **{off: False})
        for name in part:
            assert np.array_equal(part[name], whole[name]), (off, name)


@pytest.mark.parametrize("d", [4, 60, 1300])
def test_gradient_is_the_differences_of_the_loss(d):
    """Central differences of the forward loss at 2^-6: the loss carries about 2^-22 of its size, the quotient
    2^-22 * 2^5 * loss + eps^2 times a third derivative (below 1 here, T = 1)."""
    rng = np.random.default_rng(d)
    n, k, eps = 3, 4, 2.0 ** -6
    F, _, vals, _ = inputs(rng, n, d, k, "logits", spread=1.0)
    ids = np.stack([rng.permutation(d)[:k] if d >= k else rng.integers(0, d, k) for _ in range(n)], 1).astype(np.int32)
    vals = np.nan_to_num(vals, nan=0.0, posinf=0.0, neginf=0.0)
    y = rng.integers(0, d, n).astype(np.int32)
    fwd, got = run(F, ids, vals, 1.0, 0.5, y, "logits")
    for j in rng.permutation(d)[:6]:
        P, M = F.copy(), F.copy()
        P[:, j] += eps
        M[:, j] -= eps
        step = P[:, j].astype(np.float64) - M[:, j]
        lp, _ = run(P, ids, vals, 1.0, 0.5, y, "logits")
        lm, _ = run(M, ids, vals, 1.0, 0.5, y, "logits")
        num = (lp.astype(np.float64) - lm) / step
        assert np.all(np.abs(num - got["G"][j]) <= 2.0 ** -17 * (1 + np.abs(fwd)) * (1 + d / 256) + eps * eps)


def test_offsets_past_32_bits():
    rng = np.random.default_rng(6)
    n, d, k = 70, 9, 3
    F, ids, vals, y = inputs(rng, n, d, k, "logits")
    check(F, ids, vals, 2.0, 0.5, y, "logits", *run(F, ids, vals, 2.0, 0.5, y, "logits", ld=(1 << 27) + 1))


@pytest.mark.parametrize("n,d", [(300, 130), (65, 513), (40, 576)])
def test_a_leading_dimension_of_2_to_the_24(n, d):
    rng = np.random.default_rng(7)
    k = 6
    F, ids, vals, y = inputs(rng, n, d, k, "logits")
    check(F, ids, vals, 2.0, 0.5, y, "logits", *run(F, ids, vals, 2.0, 0.5, y, "logits", ld=(1 << 24) // 4 + 100))


@pytest.mark.parametrize("n,d", [(300, 100), (500, 700), (200, 1500)])
def test_captured_and_replayed(n, d):
    """Two calls in one graph with a workspace each, replayed on changed scores between eager work."""
    print("case: graph", n, d, flush=True)
    rng = np.random.default_rng(d)
    k, T, w = 5, 2.0, 0.3
    _, ids, vals, y = inputs(rng, n, d, k, "logits")
    idd, vd, yd = gu.up(ids), gu.up(vals), gu.up(y)
    Fs = [torch.zeros((d, n), device=gu.DEV) for _ in range(2)]
    outs = [dict(loss=torch.zeros(n, device=gu.DEV), G=torch.zeros((d, n), device=gu.DEV),
                 hess=torch.zeros((d, n), device=gu.DEV), h_row=torch.zeros(n, device=gu.DEV),
                 norm2=torch.zeros(d, dtype=torch.float64, device=gu.DEV)) for _ in range(2)]
    wss = [workspace(L.sb_workspace_bytes(L.SB_CALL_DISTILL, n=n, d=d, k=k), gu.DEV) for _ in range(2)]

    def call(i):
        o = outs[i]
        L.sb_distill_gradients(Fs[i], n, d, n, T, w, yd, 0, k, idd, vd, n, o["loss"], o["G"], n, o["hess"], n, o["h_row"],
                               o["norm2"], wss[i], wss[i].numel())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(0)
    torch.cuda.current_stream().wait_stream(side)
    gu.sync()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(0)
        call(1)
    for rep in range(3):
        hosts = [rng.normal(size=(n, d)).astype(np.float32) for _ in range(2)]
        for M, F in zip(Fs, hosts):
            M.copy_(gu.up(np.ascontiguousarray(F.T)))
        g.replay()
        gu.sync()
        for o, F in zip(outs, hosts):
            _, eager = run(F, ids, vals, T, w, y, "logits")
            for name in eager:
                assert np.array_equal(o[name].cpu().numpy(), eager[name]), (rep, name)


def test_two_streams_at_once():
    rng = np.random.default_rng(11)
    n, d, k = 500, 1200, 7
    F, ids, vals, y = inputs(rng, n, d, k, "logits")
    _, want = run(F, ids, vals, 2.0, 0.3, y, "logits")
    Fd, idd, vd, yd = gu.up(np.ascontiguousarray(F.T)), gu.up(ids), gu.up(vals), gu.up(y)
    streams = [torch.cuda.Stream() for _ in range(2)]
    G = [torch.zeros((d, n), device=gu.DEV) for _ in streams]
    n2 = [torch.zeros(d, dtype=torch.float64, device=gu.DEV) for _ in streams]
    ws = [workspace(L.sb_workspace_bytes(L.SB_CALL_DISTILL, n=n, d=d, k=k), gu.DEV) for _ in streams]
    gu.sync()
    for _ in range(5):
        for i, s in enumerate(streams):
            L.sb_distill_gradients(Fd, n, d, n, 2.0, 0.3, yd, 0, k, idd, vd, n, None, G[i], n, None, 0, None, n2[i], ws[i],
                                   ws[i].numel(), s)
    gu.sync()
    for i in range(2):
        assert np.array_equal(G[i].cpu().numpy(), want["G"]) and np.array_equal(n2[i].cpu().numpy(), want["norm2"])
