"""Refusals of the calls on score rows, on the host before any device work (no GPU)."""
import os

import pytest

from paper_2211_12858_amd import build as sb_build

FAKE = 0x100000  # non-NULL address that is never dereferenced (validation fails first)
BIG = 1 << 40    # far from FAKE
ARG, SHAPE, UNSUPPORTED = 1, 2, 3


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(sb_build.LIB):
        sb_build.build()
    from paper_2211_12858_amd import _lib
    _lib.load()
    return _lib


def code(L, fn, kw):
    with pytest.raises(L.SBError) as e:
        fn(*kw.values())
    assert fn.__name__ in L.sb_last_error()
    return e.value.code


def lp_args(**kw):
    a = dict(F=FAKE, dtype=0, order=0, n=10, d=5, ld_f=10, temperature=1.0, labels=FAKE, logp=FAKE, rank=FAKE, lse=FAKE,
             entropy=FAKE, k=3, top_id=FAKE, top_logp=FAKE, ld_top=10, ws=None, ws_bytes=0, stream=0)
    assert set(kw) <= set(a)
    return dict(a, **kw)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(order=2), UNSUPPORTED),
    (dict(dtype=1), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),  # column-major scores are fp32
    (dict(F=None), ARG), (dict(n=0), ARG), (dict(n=2**31), ARG), (dict(n=-1), ARG), (dict(d=0), ARG),
    (dict(d=65536), ARG), (dict(k=-1), ARG), (dict(k=65), ARG),
    (dict(temperature=0.0), ARG), (dict(temperature=-1.0), ARG), (dict(temperature=float("nan")), ARG),
    (dict(temperature=float("inf")), ARG), (dict(temperature=1e-5), ARG), (dict(temperature=1e5), ARG),
    (dict(labels=None), ARG), (dict(labels=None, logp=None), ARG), (dict(labels=None, rank=None), ARG),
    (dict(top_id=None), ARG), (dict(top_logp=None), ARG),
    (dict(logp=None, rank=None, lse=None, entropy=None, k=0), ARG),
    (dict(ld_f=9), SHAPE), (dict(order=1, ld_f=4), SHAPE), (dict(ld_f=2**62), SHAPE), (dict(ld_top=9), SHAPE),
    (dict(ld_top=2**62), SHAPE), (dict(F=FAKE + 2), SHAPE), (dict(order=1, dtype=1, F=FAKE + 1), SHAPE),
])
def test_log_probs_refusals(L, kw, want):
    assert code(L, L.sb_log_probs, lp_args(**kw)) == want


def distill_args(**kw):
    a = dict(F=FAKE, n=10, d=5, ld_f=10, temperature=1.0, hard_weight=0.5, labels=FAKE, teacher=0, k=3, t_id=FAKE,
             t_val=FAKE, ld_t=10, loss=FAKE, ws=None, ws_bytes=0, stream=0)
    assert set(kw) <= set(a)
    return dict(a, **kw)


def gradient_args(**kw):
    a = dict(F=FAKE, n=10, d=5, ld_f=10, temperature=1.0, hard_weight=0.5, labels=FAKE, teacher=0, k=3, t_id=FAKE,
             t_val=FAKE, ld_t=10, loss=FAKE, G=BIG, ld_g=10, hess=2 * BIG, ld_hess=10, h_row=FAKE, norm2=FAKE, ws=None,
             ws_bytes=0, stream=0)
    assert set(kw) <= set(a)
    return dict(a, **kw)


@pytest.mark.parametrize("kw,want", [
    (dict(teacher=2), UNSUPPORTED), (dict(teacher=-1), UNSUPPORTED), (dict(F=None), ARG), (dict(t_id=None), ARG),
    (dict(t_val=None), ARG), (dict(n=0), ARG), (dict(n=2**31), ARG), (dict(d=0), ARG), (dict(d=65536), ARG),
    (dict(k=0), ARG), (dict(k=65), ARG), (dict(temperature=0.0), ARG), (dict(temperature=float("nan")), ARG),
    (dict(temperature=2e4), ARG), (dict(hard_weight=-0.1), ARG), (dict(hard_weight=1.1), ARG),
    (dict(hard_weight=float("nan")), ARG), (dict(labels=None), ARG), (dict(ld_f=9), SHAPE), (dict(ld_t=9), SHAPE),
    (dict(ld_f=2**62), SHAPE), (dict(ld_t=2**62), SHAPE), (dict(F=FAKE + 1), SHAPE), (dict(t_id=FAKE + 2), SHAPE),
    (dict(t_val=FAKE + 2), SHAPE),
])
def test_distill_refusals(L, kw, want):
    assert code(L, L.sb_distill_loss, distill_args(**kw)) == want
    assert code(L, L.sb_distill_gradients, gradient_args(**kw)) == want


def test_distill_loss_needs_its_output(L):
    assert code(L, L.sb_distill_loss, distill_args(loss=None)) == ARG


@pytest.mark.parametrize("kw,want", [
    (dict(G=None), ARG), (dict(ld_g=9), SHAPE), (dict(ld_hess=9), SHAPE), (dict(ld_g=2**62), SHAPE),
    (dict(ld_hess=2**62), SHAPE), (dict(G=FAKE), SHAPE), (dict(G=FAKE + 4 * 49), SHAPE), (dict(hess=FAKE), SHAPE),
    (dict(hess=BIG + 4 * 49), SHAPE), (dict(G=FAKE + 2), SHAPE),
])
def test_distill_gradients_refusals(L, kw, want):
    assert code(L, L.sb_distill_gradients, gradient_args(**kw)) == want


def test_workspace_sizes(L):
    for call, lo in ((L.SB_CALL_LOG_PROBS, 0), (L.SB_CALL_DISTILL, 1)):
        for k in (lo, 64):
            for n in (1, 2**31 - 1):
                for d in (1, 65535):
                    assert 0 <= L.sb_workspace_bytes(call, n=n, d=d, k=k) < 2**50
        for kw in (dict(n=0, d=5, k=3), dict(n=2**31, d=5, k=3), dict(n=5, d=0, k=3), dict(n=5, d=65536, k=3),
                   dict(n=5, d=5, k=lo - 1), dict(n=5, d=5, k=65)):
            with pytest.raises(L.SBError):
                L.sb_workspace_bytes(call, **kw)


def test_workspaces_are_checked(L):
    n, d, k = 200_000, 40, 3
    need = L.sb_workspace_bytes(L.SB_CALL_DISTILL, n=n, d=d, k=k)
    if need:
        kw = dict(n=n, d=d, ld_f=n, ld_t=n, ld_g=n, ld_hess=n)
        assert code(L, L.sb_distill_gradients, gradient_args(**kw)) == ARG  # NULL
        assert code(L, L.sb_distill_gradients, gradient_args(**kw, ws=FAKE, ws_bytes=need - 1)) == ARG
        assert code(L, L.sb_distill_gradients, gradient_args(**kw, ws=FAKE + 64, ws_bytes=need)) == SHAPE
    need = L.sb_workspace_bytes(L.SB_CALL_LOG_PROBS, n=100, d=65535, k=k)
    if need:
        kw = dict(n=100, d=65535, ld_f=100, ld_top=100, k=k)
        assert code(L, L.sb_log_probs, lp_args(**kw)) == ARG
        assert code(L, L.sb_log_probs, lp_args(**kw, ws=FAKE, ws_bytes=need - 1)) == ARG
        assert code(L, L.sb_log_probs, lp_args(**kw, ws=FAKE + 64, ws_bytes=need)) == SHAPE
