"""A teacher and its student together: a booster (or a network's logits) answers, another booster learns from the answers.

The student's steps against the oracle's: derivatives, leaf values from the stored hessians and the update, on the tree
that the device grew.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import boost as ob
from oracle import scores as osc
from workloads import make_inputs, workload

pytestmark = pytest.mark.gpu

import gpu_util as gu  # noqa: E402
from paper_2211_12858_amd.driver import Booster, log_probs  # noqa: E402


def booster(loss, wl, bins, F0=None):
    return Booster(bins, wl.n_bins, wl.d, loss, "top_outputs", 4, wl.depth, lam=1.0, lr=0.3, device=gu.DEV, F0=F0)


@pytest.mark.parametrize("T,w", [(1.0, 0.0), (2.0, 0.4)])
def test_student_of_a_booster(T, w):
    wl = workload("mc2m_rs5", n=3_000, m=12, d=9, depth=4)
    inp = make_inputs(wl)
    y = gu.up(inp.y)
    teacher = booster("softmax", wl, inp.bins)
    teacher.set_target(y)
    for _ in range(4):
        teacher.step()
    said = teacher.log_probs(labels=y, k=5, temperature=T)
    want = osc.log_probs(teacher.F.cpu().numpy().T, T, inp.y, 5)
    assert np.array_equal(said.top_id.cpu().numpy(), want["top_id"])
    assert np.array_equal(said.rank.cpu().numpy(), want["rank"])
    # 9 classes: far fewer than 64 roundings of 2^-24 relative to values below 8
    assert np.allclose(said.logp.cpu().numpy(), want["logp"], atol=2.0 ** -15)
    student = booster("distill", wl, inp.bins)
    student.set_teacher(said.top_id, said.top_logp, "log_probs", T, y if w else None, w)
    ids, vals = said.top_id.cpu().numpy(), said.top_logp.cpu().numpy()
    F = np.zeros((wl.n, wl.d), dtype=np.float32)
    for r in range(3):
        student.step()
        gu.sync()
        _, g, h = osc.distill(F, ids, vals, T, w, inp.y, "log_probs")
        # 9 terms a sum and 5 places a list: below 64 roundings of values below 2 T
        assert np.allclose(student.G.cpu().numpy().T, g, atol=2.0 ** -17 * T)
        assert np.allclose(student.hess.cpu().numpy().T, h, atol=2.0 ** -18)
        tree = student.ss.tree()
        V = oracle.leaf_values(student.G.cpu().numpy().T, tree["row_idx"], tree["leaf_off"], 1.0,
                               hess=student.hess.cpu().numpy().T)
        assert np.allclose(student.pending.cpu().numpy(), V, rtol=1e-6, atol=1e-7)
        F = ob.update_predictions(F, tree["row_idx"], tree["leaf_off"], student.pending.cpu().numpy(), student.lr)
        loss = student.distill_loss()
        assert student.pending is None and np.array_equal(student.F.cpu().numpy(), F.T)
        want_loss, _, _ = osc.distill(F, ids, vals, T, w, inp.y, "log_probs")
        # terms of at most 2 T^2 log 9 + ..., below 64 roundings of 16 T^2
        assert np.allclose(loss.cpu().numpy(), want_loss, atol=2.0 ** -14 * T * T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_student_of_a_network(dtype):
    """Row-major logits of the network's type, every second column of a wider matrix left out by the leading dimension."""
    wl = workload("mc2m_rs5", n=2_001, m=8, d=40, depth=3)
    inp = make_inputs(wl)
    g = torch.Generator(device=gu.DEV)
    g.manual_seed(3)
    wide = (torch.randn((wl.n, 53), generator=g, device=gu.DEV) * 3).to(dtype)
    logits = wide[:, :wl.d]
    said = log_probs(logits, k=10, temperature=2.0, order="row")
    a = logits.float().cpu().numpy()
    want = osc.log_probs(a, 2.0, None, 10)
    assert said.logp is None and said.rank is None
    assert np.array_equal(said.top_id.cpu().numpy(), want["top_id"])
    student = booster("distill", wl, inp.bins)
    student.set_teacher(said.top_id, said.top_logp, "log_probs", 2.0)
    student.step()
    gu.sync()
    _, gr, _ = osc.distill(np.zeros((wl.n, wl.d)), said.top_id.cpu().numpy(), said.top_logp.cpu().numpy(), 2.0, 0.0, None,
                           "log_probs")
    # 40 terms a sum, 10 places a list: below 128 roundings of values below 2 T
    assert np.allclose(student.G.cpu().numpy().T, gr, atol=2.0 ** -15)


def test_another_stream():
    """Outputs and workspace belong to the stream that the work runs on."""
    F = torch.randn((300, 2_000), device=gu.DEV)
    want = log_probs(F, k=6)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (s, s.cuda_stream):
        got = [log_probs(F, k=6, stream=stream) for _ in range(4)]
        s.synchronize()
        for r in got:
            assert torch.equal(r.top_id, want.top_id) and torch.equal(r.lse, want.lse)


def test_refusals():
    F = torch.zeros((4, 6), device=gu.DEV)
    with pytest.raises(ValueError):
        log_probs(F, order="rows")
    with pytest.raises(ValueError):
        log_probs(F.t())
    with pytest.raises(ValueError):
        log_probs(F.double())
    with pytest.raises(ValueError):
        log_probs(F, labels=torch.zeros(4, dtype=torch.int32, device=gu.DEV))
    with pytest.raises(ValueError):
        log_probs(F, labels=torch.zeros(6, dtype=torch.int64, device=gu.DEV))
    bins = np.zeros((6, 3), dtype=np.uint8)
    b = Booster(bins, 4, 4, "distill", "identity", 4, 1, device=gu.DEV)
    ids, vals = torch.zeros((2, 6), dtype=torch.int32, device=gu.DEV), torch.zeros((2, 6), device=gu.DEV)
    for call in (b.step, b.distill_loss, lambda: b.set_target(ids[0]), lambda: b.set_teacher(ids, vals.double()),
                 lambda: b.set_teacher(ids[:, :5], vals[:, :5]), lambda: b.set_teacher(ids, vals, hard_weight=0.5),
                 lambda: b.set_teacher(ids, vals, labels=ids[0][:5])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        Booster(bins, 4, 4, "softmax", "identity", 4, 1, device=gu.DEV).set_teacher(ids, vals)
