"""Which listed places are targets: an excluded class (score -inf) makes the loss +inf where its q_t is above 0, and adds
nothing where q_t = exp((v_t - v_max) / T) (or exp(v_t)) is below 2^-126, wherever in the list the largest value stands.

The same rows go through every kernel (rows in registers, a wave per tile of many rows, column ranges), which have to
agree; exp(-87) is above 2^-126 = exp(-87.34) and exp(-88) is below it, each by far more than the roundings of the gap.
"""
import numpy as np
import pytest

from oracle import scores as osc

pytestmark = pytest.mark.gpu

from test_gpu_distill import check, run  # noqa: E402


@pytest.mark.parametrize("kind", ["logits", "log_probs"])
@pytest.mark.parametrize("n,d", [(100_003, 400), (500, 30), (500, 400), (500, 900), (500, 1600)])
@pytest.mark.parametrize("T,w", [(0.01, 0.0), (1.0, 0.9), (2.0, 0.4)])
def test_excluded_places_below_others(n, d, T, w, kind):
    """Place 0 lists an excluded class; the largest value comes `gap` above it, in the second group of eight places,
    with others on the way up."""
    print("case: targets", n, d, T, w, kind, flush=True)
    rng = np.random.default_rng(d)
    k = 10
    gaps = np.array([0.0, 0.5, 40.0, 87.0, 88.0, 120.0, 200.0, 2000.0])[np.arange(n) % 8]
    F = rng.normal(size=(n, d)).astype(np.float32)
    ids = ((rng.integers(0, d, n)[None, :] + np.arange(k)[:, None] * (d // k)) % d).astype(np.int32)
    scale = T if kind == "logits" else 1.0
    vals = np.empty((k, n), dtype=np.float32)
    vals[0] = -gaps * scale
    vals[1:9] = -gaps * scale * np.linspace(0.9, 0.1, 8)[:, None]
    vals[9] = 0.0
    rows = np.arange(n)
    low = F.copy()
    F[rows, ids[0]] = -np.inf
    low[rows, ids[0]] = -1e4 * max(T, 1.0)  # its probability is 0 in fp64 as well
    y = ids[9].copy() if w else None
    fwd, got = run(F, ids, vals, T, w, y, kind)
    hit = gaps < 87.5
    for name, loss in (("forward", fwd), ("gradients", got["loss"])):
        assert np.all(loss[hit] == np.inf), (name, np.unique(gaps[hit][loss[hit] != np.inf]))
        assert np.all(np.isfinite(loss[~hit])), (name, np.unique(gaps[~hit][~np.isfinite(loss[~hit])]))
    off = vals.copy()
    off[0, ~hit] = -np.inf  # q of 0 by definition
    some = rows[~hit][:300]
    check(low[some], ids[:, some], off[:, some], T, w, None if y is None else y[some], kind, fwd[some],
          {name: got[name][..., some] for name in ("G", "hess", "h_row", "loss")})


@pytest.mark.parametrize("n", [100_003, 300])
def test_rising_values(n):
    """Values in rising order, far apart and near, no class excluded: the list's order does not matter."""
    rng = np.random.default_rng(5)
    d, k = 1000, 25
    F = (rng.normal(size=(n, d)) * 2).astype(np.float32)
    ids = ((rng.integers(0, d, n)[None, :] + np.arange(k)[:, None] * 40) % d).astype(np.int32)
    vals = np.sort(rng.normal(size=(k, n)), axis=0).astype(np.float32)
    vals[:, ::3] *= 100.0
    some = np.arange(300)
    fwd, _ = run(F, ids, vals, 0.5, 0.0, None, "logits", hess=False, row=False, norms=False)
    back, _ = run(F, ids[::-1].copy(), vals[::-1].copy(), 0.5, 0.0, None, "logits", hess=False, row=False, norms=False)
    want, _, _ = osc.distill(F[some], ids[:, some], vals[:, some], 0.5, 0.0, None, "logits")
    # a few hundred roundings (sums 1000/16 + 24 deep, 25 places, exponents of up to 40 by three roundings) of T^2 times
    # log s and the values' and scores' differences
    size = 0.25 * (np.log(d) + 2.0 * (np.ptp(vals[:, some], axis=0) + np.ptp(F[some], axis=1)))
    for got in (fwd[some], back[some]):
        assert np.all(np.abs(got - want) <= 512 * 2.0 ** -24 * size)
