"""sb_log_probs against the fp64 oracle.

Classes and ranks have to be equal; the real outputs are held to bounds of their own arithmetic, u = 2^-24:
z_j = (a_j - m) / T is formed from three roundings (|dz| <= 3u |z|), e_j = exp(z_j) by an exponential of at most 4u,
and sums of d terms in groups of at most 16 + d/16 adds, S = d/16 + 24 with the joins.  With the means E over p,
    eps_s = u (S + 6 + 3 E|z|) bounds the relative error of s, and so the absolute one of log s, to which the logarithm
    adds 4u |log s|;
    eps_t = u ((S + 10) E|z| + 6 E z^2) that of t / s.
The factor is 2 on the whole, for the second-order terms.
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
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
MARK = 12345.0  # what outputs hold before the call


def run(F, order="col", dtype="f32", T=1.0, labels=None, k=0, ld_f=None, ld_top=None, shift=0, outputs=True, stream=None):
    """F (n, d) host array -> dict of host outputs.  ld_f: leading dimension (the gaps hold NaN); shift: elements
    between the allocation and the matrix."""
    n, d = F.shape
    rows = d if order == "row" else n
    cols = n if order == "row" else d
    ld = rows if ld_f is None else ld_f
    buf = torch.full((shift + cols * ld,), float("nan"), dtype=TORCH[dtype], device=gu.DEV)
    M = buf[shift:].view(cols, ld)
    M[:, :rows] = gu.up(np.ascontiguousarray(F if order == "row" else F.T)).to(TORCH[dtype])
    ld_top = n if ld_top is None else ld_top
    out = {}
    if outputs:
        for name in ("lse", "entropy") + (("logp",) if labels is not None else ()):
            out[name] = torch.full((n,), MARK, dtype=torch.float32, device=gu.DEV)
        if labels is not None:
            out["rank"] = torch.full((n,), 12345, dtype=torch.int32, device=gu.DEV)
    if k:
        out["top_id"] = torch.full((k, ld_top), 12345, dtype=torch.int32, device=gu.DEV)
        out["top_logp"] = torch.full((k, ld_top), MARK, dtype=torch.float32, device=gu.DEV)
    y = None if labels is None else gu.up(labels)
    ws = workspace(L.sb_workspace_bytes(L.SB_CALL_LOG_PROBS, n=n, d=d, k=k), gu.DEV)
    gu.sync()
    L.sb_log_probs(M, L.DTYPE[dtype], L.SB_ROW_MAJOR if order == "row" else L.SB_COLUMN_MAJOR, n, d, ld, T, y,
                   out.get("logp"), out.get("rank"), out.get("lse"), out.get("entropy"), k, out.get("top_id"),
                   out.get("top_logp"), ld_top, ws, ws.numel(), stream)
    gu.sync()
    got = {name: t.cpu().numpy() for name, t in out.items()}
    for name in ("top_id", "top_logp"):
        if name in got:
            assert np.all(got[name][:, n:] == 12345), "places behind the last row are left as they were"
            got[name] = got[name][:, :n]
    return got


def rounded(F, dtype):
    return torch.from_numpy(np.ascontiguousarray(F, dtype=np.float32)).to(TORCH[dtype]).float().numpy()


def bounds(F, T):
    """Per row: m, eps_s + what log s adds, the bound of t / s, and log s."""
    F = F.astype(np.float64)
    m = F.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        z = np.where(np.isneginf(F), 0.0, (F - np.where(np.isneginf(m), 0.0, m)) / T)
        e = np.where(np.isneginf(F), 0.0, np.exp(z))
    s = np.maximum(e.sum(axis=1), 1e-300)
    e1, e2 = (e * np.abs(z)).sum(axis=1) / s, (e * z * z).sum(axis=1) / s
    S = F.shape[1] / 16 + 24
    ls = np.abs(np.log(s))
    return m[:, 0], U * (S + 6 + 3 * e1) + 4 * U * ls, U * ((S + 10) * e1 + 6 * e2), ls


def check(F, got, T, labels, k, rows=None):
    """got against the oracle on the given rows (all by default)."""
    rows = np.arange(F.shape[0]) if rows is None else rows
    F = F[rows]
    labels = None if labels is None else labels[rows]
    want = osc.log_probs(F, T, labels, k)
    got = {name: v[..., rows] for name, v in got.items()}
    m, ds, dt, ls = bounds(F, T)
    mt = np.where(np.isneginf(m), 0.0, np.abs(m)) / T

    def close(name, tol):
        g, w = got[name].astype(np.float64), want[name]
        # infinities, and what no fp32 value but they can stand for: past the largest one by half its step
        w = np.where(np.abs(w) >= 2.0 ** 128 - 2.0 ** 103, np.copysign(np.inf, w), w)
        same = g == w
        with np.errstate(invalid="ignore"):
            bad = ~(same | (np.abs(g - w) <= 2 * tol + 2.0 ** -140))
        assert not bad.any(), (name, np.argwhere(bad)[:5], g[bad][:5], w[bad][:5])

    if "lse" in got:
        close("lse", ds + 4 * U * mt + U * np.abs(np.where(np.isfinite(want["lse"]), want["lse"], 0.0)))
        close("entropy", ds + dt + U * (ls + want["entropy"]))
    if labels is not None and "logp" in got:
        lp = np.where(np.isfinite(want["logp"]), np.abs(want["logp"]), 0.0)
        close("logp", ds + 4 * U * (lp + ls))
        assert np.array_equal(got["rank"], want["rank"])
    if k:
        assert np.array_equal(got["top_id"], want["top_id"])
        lp = np.where(np.isfinite(want["top_logp"]), np.abs(want["top_logp"]), 0.0)
        close("top_logp", ds + 4 * U * (lp + ls))


def labels_of(rng, n, d):
    y = rng.integers(0, d, n).astype(np.int32)
    y[rng.random(n) < 0.1] = -1
    y[rng.random(n) < 0.05] = d
    return y


CASES = [("col", "f32"), ("row", "f32"), ("row", "f16"), ("row", "bf16")]


# From one row and one class on; around the chunks of columns, the widths at which another kernel takes the rows,
# lists shorter and longer than the classes, odd row counts.
@pytest.mark.parametrize("order,dtype", CASES)
@pytest.mark.parametrize("n,d,k", [(1, 1, 1), (1, 1, 64), (2, 3, 5), (1, 1000, 5), (63, 2, 1), (64, 15, 4), (65, 16, 16),
                                   (130, 17, 0), (257, 33, 33), (300, 64, 10), (129, 65, 64), (77, 100, 10),
                                   (200, 104, 8), (70, 128, 9), (64, 129, 32), (33, 255, 17), (40, 513, 20),
                                   (31, 1000, 32), (17, 1024, 64), (9, 1025, 3), (10, 2047, 20), (6, 4099, 64),
                                   (5, 8191, 5), (4, 8192, 12), (3, 8193, 40), (3, 30_011, 50), (2, 65_535, 64),
                                   (1, 65_535, 1)])
def test_shapes(order, dtype, n, d, k):
    print("case: log_probs", order, dtype, n, d, k, flush=True)
    rng = np.random.default_rng(n * 1000 + d + k)
    F = rounded(rng.normal(size=(n, d)) * 3, dtype)  # 16-bit scores have equal ones in every row
    y = labels_of(rng, n, d)
    T = [1.0, 2.0, 0.37][(n + d) % 3]
    check(F, run(F, order, dtype, T, y, k), T, y, k)


# Rows by the thousand: every row tile and grid stride, checked on a sample of rows that has the last ones.
@pytest.mark.parametrize("order,dtype", CASES)
@pytest.mark.parametrize("n,d,k", [(200_003, 5, 3), (150_001, 30, 8), (100_007, 100, 10), (70_001, 40, 40),
                                   (20_011, 257, 16), (9_001, 1000, 10)])
def test_many_rows(order, dtype, n, d, k):
    print("case: log_probs", order, dtype, n, d, k, flush=True)
    rng = np.random.default_rng(n + d + k)
    F = rounded(rng.normal(size=(n, d)).astype(np.float32) * 2, dtype)
    y = labels_of(rng, n, d)
    rows = np.unique(np.concatenate([[0, 63, 64, n - 65, n - 64, n - 2, n - 1], rng.integers(0, n, 400)]))
    check(F, run(F, order, dtype, 1.5, y, k), 1.5, y, k, rows)


# Leading dimensions past the matrix (the gaps hold NaN), matrices that start off a vector's alignment, lists with a
# leading dimension of their own.
# Several rows per wave and block in turn, at each width of a row's threads: 2048 blocks of four waves up to 1024 and
# 4096 classes, 1024 up to 16384, 512 or 256 beyond.  Every third row holds few different scores, so that its
# candidates outnumber their places, next to rows whose do not.
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,d,k", [(9001, 700, 10), (9003, 100, 33), (8200, 641, 64), (2050, 1025, 12), (8300, 1100, 40),
                                   (1100, 4097, 5), (1040, 4500, 64), (515, 16_385, 20), (600, 16_390, 64),
                                   (300, 20_001, 33), (520, 5000, 0)])
def test_rows_in_turn(dtype, n, d, k):
    print("case: log_probs row", dtype, n, d, k, flush=True)
    rng = np.random.default_rng(n + d + k)
    F = rng.normal(size=(n, d)).astype(np.float32) * 3
    F[::3] = rng.integers(0, 3, F[::3].shape)
    F = rounded(F, dtype)
    y = labels_of(rng, n, d)
    rows = np.unique(np.concatenate([np.arange(6), np.arange(n - 6, n), rng.integers(0, n, 60)]))
    check(F, run(F, "row", dtype, 2.0, y, k), 2.0, y, k, rows)


# Lists of every length class and both sides of the rules that choose lanes, waves, and the column splits and how many
# lanes join them.
@pytest.mark.parametrize("order,n,d,k", [("row", 160 * 40 - 1, 40, 5), ("row", 160 * 40, 40, 5), ("row", 102_400, 640, 3),
                                         ("row", 102_560, 641, 3), ("row", 20_000, 90, 14), ("row", 20_000, 90, 17),
                                         ("row", 20_000, 90, 48), ("row", 20_000, 90, 1), ("row", 20_000, 90, 0),
                                         ("col", 5000, 8 * 64 - 1, 9), ("col", 5000, 8 * 64, 13), ("col", 1000, 9 * 64, 20),
                                         ("col", 1000, 16 * 64, 64), ("col", 700, 17 * 64, 12), ("col", 64, 64 * 64, 33),
                                         ("col", 64, 65_535, 64), ("col", 60_000, 130, 33), ("col", 60_000, 130, 32),
                                         ("col", 43_000, 200, 64), ("col", 131_009, 130, 16), ("col", 131_073, 130, 16)])
def test_both_sides_of_the_rules(order, n, d, k):
    print("case: log_probs", order, n, d, k, flush=True)
    rng = np.random.default_rng(n + d + k)
    F = rng.normal(size=(n, d)).astype(np.float32)
    F[1::2] = np.round(F[1::2])
    y = labels_of(rng, n, d)
    rows = np.unique(np.concatenate([np.arange(6), np.arange(n - 6, n), rng.integers(0, n, 150)]))
    check(F, run(F, order, "f32", 0.7, y, k), 0.7, y, k, rows)


# Scores in ascending order make every class enter the list, in descending order only the first ones.
@pytest.mark.parametrize("order,dtype", CASES)
@pytest.mark.parametrize("n,d,k", [(70, 300, 20), (20_000, 100, 64), (20_000, 100, 10), (40, 3000, 64)])
@pytest.mark.parametrize("up", [True, False])
def test_sorted_scores(order, dtype, n, d, k, up):
    F = rounded(np.tile(np.arange(d, dtype=np.float32) * (0.25 if up else -0.25), (n, 1)), dtype)
    rows = np.array([0, 1, 63, n - 2, n - 1]) % n
    check(F, run(F, order, dtype, 1.0, None, k), 1.0, None, k, rows)


@pytest.mark.parametrize("order,dtype", CASES)
@pytest.mark.parametrize("n,d,pad,shift", [(70, 50, 1, 0), (70, 50, 3, 1), (33, 1001, 5, 3), (5, 9001, 7, 5), (130, 8, 8, 7),
                                           (1, 2051, 13, 1), (3, 40_003, 2, 6)])
def test_strides_and_alignment(order, dtype, n, d, pad, shift):
    rng = np.random.default_rng(n + d)
    F = rounded(rng.normal(size=(n, d)) * 2, dtype)
    y = labels_of(rng, n, d)
    got = run(F, order, dtype, 1.0, y, 7, ld_f=(d if order == "row" else n) + pad, ld_top=n + 3, shift=shift)
    check(F, got, 1.0, y, 7)


# Equal scores: whole rows of them, a few values only, both zeros; the lower class comes first.
@pytest.mark.parametrize("order,dtype", CASES)
@pytest.mark.parametrize("n,d,k", [(5, 40, 16), (3, 1000, 64), (130, 100, 10), (2, 9000, 64), (2, 65_535, 10)])
def test_ties(order, dtype, n, d, k):
    rng = np.random.default_rng(d)
    F = rng.integers(-2, 3, (n, d)).astype(np.float32)
    F[0] = 0.0
    F[1] = np.where(rng.random(d) < 0.5, 0.0, -0.0)
    y = labels_of(rng, n, d)
    check(F, run(F, order, dtype, 1.0, y, k), 1.0, y, k)


# Excluded classes: none left, one left, fewer left than places; the type's lowest values are ordinary scores.
@pytest.mark.parametrize("order,dtype", CASES)
@pytest.mark.parametrize("n,d,k", [(6, 12, 5), (70, 100, 10), (7, 1000, 20), (6, 20_000, 64)])
def test_excluded_classes(order, dtype, n, d, k):
    rng = np.random.default_rng(d + 1)
    F = rounded(rng.normal(size=(n, d)) * 2, dtype)
    F[0] = -np.inf
    F[1] = -np.inf
    F[1, d - 1] = 3.0
    F[2, rng.random(d) < 0.9] = -np.inf
    F[3, : d // 2] = -np.inf
    F[4] = float(torch.finfo(TORCH[dtype]).min)
    F[5] = -np.inf
    F[5, d // 3] = float(torch.finfo(TORCH[dtype]).min)
    y = labels_of(rng, n, d)
    y[:6] = [0, d - 1, 1, 0, d // 2, 0]
    check(F, run(F, order, dtype, 1.0, y, k), 1.0, y, k)


@pytest.mark.parametrize("order,dtype", CASES)
@pytest.mark.parametrize("d", [20, 1000, 9000])
def test_far_scores(order, dtype, d):
    """Scores far apart and far from zero: no overflow, and the order of equal 32-bit differences is kept."""
    rng = np.random.default_rng(d)
    F = rounded(rng.normal(size=(9, d)) * 300, dtype)
    F[1] = rounded(F[1] * 20, dtype)
    y = labels_of(rng, 9, d)
    for T in (1e-4, 0.05, 1e4):
        check(F, run(F, order, dtype, T, y, 9), T, y, 9)


# Scores whose size leaves few bits for their differences, and masks of the type's lowest value, some of which leave a
# row nothing else.
@pytest.mark.parametrize("order,dtype", CASES)
@pytest.mark.parametrize("d", [20, 700, 1500, 9000, 20_000])
@pytest.mark.parametrize("T", [0.01, 1.0, 100.0])
def test_large_scores_and_lowest_values(order, dtype, d, T):
    rng = np.random.default_rng(d)
    n, low = 40, torch.finfo(TORCH[dtype]).min
    F = rng.normal(size=(n, d)).astype(np.float32) * 3
    F[::4] += np.float32({"f32": 3e7, "f16": 3e4, "bf16": 1e9}[dtype])
    F[1::4][rng.random(F[1::4].shape) < 0.5] = low
    F[2] = F[9] = low
    F[6] = -np.inf
    F[6, d // 2] = low
    F[10, : d // 2] = -np.inf
    F = rounded(F, dtype)
    y = labels_of(rng, n, d)
    check(F, run(F, order, dtype, T, y, 12), T, y, 12)


@pytest.mark.parametrize("order,dtype", CASES)
@pytest.mark.parametrize("d", [3, 100, 1500, 9000])
def test_nan_and_inf_stay_in_their_row(order, dtype, d):
    rng = np.random.default_rng(d)
    F = rounded(rng.normal(size=(70, d)), dtype)
    y = rng.integers(0, d, 70).astype(np.int32)
    F[3, d // 2] = np.nan
    F[66, 0] = np.inf
    got = run(F, order, dtype, 1.0, y, 2)
    for i in (3, 66):
        for name in ("lse", "entropy", "logp"):
            assert np.isnan(got[name][i]), (name, i)
        assert np.all((got["top_id"][:, i] >= -1) & (got["top_id"][:, i] < d))
    check(F, got, 1.0, y, 2, np.setdiff1d(np.arange(70), [3, 66]))


@pytest.mark.parametrize("order,dtype", CASES)
@pytest.mark.parametrize("d", [3, 100, 1001, 9001])
def test_ranks_and_classes_of_nan_rows_are_in_range(order, dtype, d):
    rng = np.random.default_rng(d)
    n, k = 70, 20
    F = rounded(rng.normal(size=(n, d)), dtype)
    F[::2, rng.integers(0, d, 5)] = np.nan
    F[1::4] = np.nan
    F[3::4, d - 1] = np.inf
    y = np.full(n, d - 1, dtype=np.int32)
    F[0::8, d - 1] = np.nan  # the given class itself
    got = run(F, order, dtype, 1.0, y, k)
    assert got["rank"].min() >= 0 and got["rank"].max() < d
    assert got["top_id"].min() >= -1 and got["top_id"].max() < d
    assert np.isnan(got["lse"]).all() and np.isnan(got["logp"]).all() and np.isnan(got["entropy"]).all()


@pytest.mark.parametrize("order", ["col", "row"])
def test_outputs_are_optional(order):
    rng = np.random.default_rng(4)
    F = rng.normal(size=(100, 37)).astype(np.float32)
    y = labels_of(rng, 100, 37)
    whole = run(F, order, labels=y, k=6)
    assert np.array_equal(run(F, order, k=6, outputs=False)["top_id"], whole["top_id"])
    part = run(F, order)
    assert np.array_equal(part["lse"], whole["lse"]) and np.array_equal(part["entropy"], whole["entropy"])


def test_same_result_every_time_and_in_both_orders():
    rng = np.random.default_rng(5)
    F = rng.normal(size=(501, 1300)).astype(np.float32)
    y = labels_of(rng, 501, 1300)
    for order in ("col", "row"):
        a, b = run(F, order, labels=y, k=30), run(F, order, labels=y, k=30)
        for name in a:
            assert np.array_equal(a[name], b[name])
    assert np.array_equal(run(F, "col", k=30)["top_id"], run(F, "row", k=30)["top_id"])


def test_offsets_past_32_bits():
    """A column-major matrix and a row-major one whose last elements lie past 2^32 bytes and 2^31 elements."""
    rng = np.random.default_rng(6)
    F = rng.normal(size=(300, 9)).astype(np.float32)
    y = labels_of(rng, 300, 9)
    check(F, run(F, "col", labels=y, k=4, ld_f=(1 << 28) + 5), 1.0, y, 4)
    F = rng.normal(size=(9, 300)).astype(np.float32)
    y = labels_of(rng, 9, 300)
    check(F, run(F, "row", labels=y, k=4, ld_f=(1 << 28) + 5), 1.0, y, 4)


@pytest.mark.parametrize("order,n,d", [("col", 300, 100), ("row", 300, 100), ("col", 20, 5000), ("row", 20, 5000)])
def test_captured_and_replayed(order, n, d):
    """Two calls captured into one graph with a workspace each, replayed on changed scores between eager work."""
    print("case: graph", order, n, d, flush=True)
    k = 5
    rng = np.random.default_rng(d)
    y = labels_of(rng, n, d)
    yd = gu.up(y)
    shape = (n, d) if order == "row" else (d, n)
    A, B = (torch.zeros(shape, device=gu.DEV) for _ in range(2))
    outs = [dict(logp=torch.zeros(n, device=gu.DEV), rank=torch.zeros(n, dtype=torch.int32, device=gu.DEV),
                 lse=torch.zeros(n, device=gu.DEV), entropy=torch.zeros(n, device=gu.DEV),
                 top_id=torch.zeros((k, n), dtype=torch.int32, device=gu.DEV), top_logp=torch.zeros((k, n), device=gu.DEV))
            for _ in range(2)]
    wss = [workspace(L.sb_workspace_bytes(L.SB_CALL_LOG_PROBS, n=n, d=d, k=k), gu.DEV) for _ in range(2)]

    def call(M, o, ws):
        L.sb_log_probs(M, L.SB_F32, L.SB_ROW_MAJOR if order == "row" else L.SB_COLUMN_MAJOR, n, d,
                       d if order == "row" else n, 1.0, yd, o["logp"], o["rank"], o["lse"], o["entropy"], k, o["top_id"],
                       o["top_logp"], n, ws, ws.numel())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(A, outs[0], wss[0])
    torch.cuda.current_stream().wait_stream(side)
    gu.sync()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(A, outs[0], wss[0])
        call(B, outs[1], wss[1])
    for rep in range(3):
        Fs = [rng.normal(size=(n, d)).astype(np.float32) for _ in range(2)]
        for M, F in zip((A, B), Fs):
            M.copy_(gu.up(np.ascontiguousarray(F if order == "row" else F.T)))
        g.replay()
        gu.sync()
        for o, F in zip(outs, Fs):
            got = {name: t.cpu().numpy() for name, t in o.items()}
            check(F, got, 1.0, y, k)
            eager = run(F, order, labels=y, k=k)
            for name in got:
                assert np.array_equal(got[name], eager[name]), (rep, name)


def test_two_streams_at_once():
    rng = np.random.default_rng(8)
    F = [rng.normal(size=(40, 6000)).astype(np.float32) for _ in range(2)]
    want = [run(f, "col", k=9) for f in F]
    M = [gu.up(np.ascontiguousarray(f.T)) for f in F]
    tid = [torch.zeros((9, 40), dtype=torch.int32, device=gu.DEV) for _ in F]
    tlp = [torch.zeros((9, 40), device=gu.DEV) for _ in F]
    ws = [workspace(L.sb_workspace_bytes(L.SB_CALL_LOG_PROBS, n=40, d=6000, k=9), gu.DEV) for _ in F]
    streams = [torch.cuda.Stream() for _ in F]
    gu.sync()
    for _ in range(5):
        for i, s in enumerate(streams):
            L.sb_log_probs(M[i], 0, 0, 40, 6000, 40, 1.0, None, None, None, None, None, 9, tid[i], tlp[i], 40, ws[i],
                           ws[i].numel(), s)
    gu.sync()
    for i in range(2):
        assert np.array_equal(tid[i].cpu().numpy(), want[i]["top_id"])
        assert np.array_equal(tlp[i].cpu().numpy(), want[i]["top_logp"])


def test_refused_calls_leave_the_outputs_alone():
    lse = torch.full((4,), MARK, device=gu.DEV)
    F = torch.zeros((3, 4), device=gu.DEV)
    with pytest.raises(L.SBError):
        L.sb_log_probs(F, 0, 0, 4, 3, 4, 0.0, None, None, None, lse, None, 0, None, None, 0, None, 0)
    gu.sync()
    assert torch.all(lse == MARK)
