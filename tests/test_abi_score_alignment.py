"""Refusals of misaligned labels and outputs of the calls on score rows, on the host before any device work (no GPU).

Every address here overlaps nothing else, so that no other check can be the one that refuses it."""
import pytest

from test_abi_scores import BIG, FAKE, SHAPE, L, code, distill_args, gradient_args, lp_args  # noqa: F401 (L: fixture)


@pytest.mark.parametrize("off", [1, 2])
@pytest.mark.parametrize("name", ["labels", "logp", "rank", "lse", "entropy", "top_id", "top_logp"])
def test_log_probs(L, name, off):  # noqa: F811
    for kw in (dict(), dict(order=1, ld_f=5)):
        assert code(L, L.sb_log_probs, lp_args(**{name: 3 * BIG + off}, **kw)) == SHAPE
        assert name in L.sb_last_error()


@pytest.mark.parametrize("off", [1, 2])
@pytest.mark.parametrize("name", ["labels", "loss"])
def test_distill_loss(L, name, off):  # noqa: F811
    assert code(L, L.sb_distill_loss, distill_args(**{name: 3 * BIG + off})) == SHAPE
    assert name in L.sb_last_error()


@pytest.mark.parametrize("name,off", [(name, off) for name in ("labels", "loss", "G", "hess", "h_row", "norm2")
                                      for off in (1, 2)] + [("norm2", 4)])
def test_distill_gradients(L, name, off):  # noqa: F811
    assert code(L, L.sb_distill_gradients, gradient_args(**{name: 3 * BIG + off})) == SHAPE
    assert name in L.sb_last_error()


def test_what_is_not_given_is_not_checked(L):  # noqa: F811
    """Missing outputs are fine: the refusal is the workspace's."""
    assert code(L, L.sb_distill_gradients, gradient_args(loss=None, hess=None, h_row=None, norm2=None)) != SHAPE
