"""A booster's lists and workspace stay until the work that reads them is done, on whatever stream it runs."""
import contextlib

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import gpu_util as gu  # noqa: E402
from paper_2211_12858_amd import driver  # noqa: E402
from paper_2211_12858_amd.driver import Booster  # noqa: E402


@pytest.mark.parametrize("raw", [False, True])
def test_set_teacher_while_a_call_is_on_its_way(raw):
    """The stream is held back by earlier work, the lists are replaced before it comes to them, and what they were
    released for takes other values."""
    rng = np.random.default_rng(2)
    n, d, k = 4_000, 40, 8
    b = Booster(rng.integers(0, 16, (n, 4)).astype(np.uint8), 16, d, "distill", "top_outputs", 3, 2, device=gu.DEV,
                F0=gu.up(rng.normal(size=(d, n)).astype(np.float32)))
    ids = np.stack([rng.permutation(d)[:k] for _ in range(n)], 1).astype(np.int32)
    vals = rng.normal(size=(k, n)).astype(np.float32)
    y = rng.integers(0, d, n).astype(np.int32)

    def teach():
        b.set_teacher(gu.up(ids), gu.up(vals), "logits", 2.0, gu.up(y), 0.3)

    teach()
    b.gradients()
    want_G, want_norm2, want_loss = b.G.clone(), b.norm2.clone(), b.distill_loss()
    gu.sync()
    b.set_teacher(torch.zeros((1, n), dtype=torch.int32, device=gu.DEV), torch.zeros((1, n), device=gu.DEV), "logits")
    teach()
    gu.sync()
    s = torch.cuda.Stream()
    big = torch.randn((8192, 8192), device=gu.DEV)
    with torch.cuda.stream(s):
        for _ in range(20):  # some tens of milliseconds
            big = big @ big * 1e-4
    stream = s.cuda_stream if raw else s
    b.gradients(stream=stream)
    loss = b.distill_loss(stream=stream)
    assert not s.query(), "the stream was not held back for long enough to show anything"
    b.set_teacher(torch.zeros((1, n), dtype=torch.int32, device=gu.DEV), torch.zeros((1, n), device=gu.DEV), "logits")
    # every block that the old lists may have been released into
    taken = [torch.zeros((k, n), dtype=torch.int32, device=gu.DEV) for _ in range(12)]
    taken += [torch.zeros(n, dtype=torch.int32, device=gu.DEV) for _ in range(12)]
    torch.cuda.current_stream().synchronize()
    s.synchronize()
    assert torch.equal(b.G, want_G) and torch.equal(b.norm2, want_norm2) and torch.equal(loss, want_loss)
    del taken


@pytest.mark.parametrize("d", [40, 1100])
def test_captured_and_replayed(d):
    """Derivatives and loss in one graph, replayed on changed scores between eager work and other lists."""
    print("case: captured", d, flush=True)
    rng = np.random.default_rng(d)
    n, k = 700, 6
    bins = rng.integers(0, 16, (n, 4)).astype(np.uint8)
    a, b = (Booster(bins, 16, d, "distill", "top_outputs", 3, 2, device=gu.DEV) for _ in range(2))
    lists = [(gu.up(rng.integers(0, d, (k, n)).astype(np.int32)), gu.up(rng.normal(size=(k, n)).astype(np.float32)))
             for _ in range(2)]
    y = gu.up(rng.integers(0, d, n).astype(np.int32))
    for x in (a, b):
        x.set_teacher(*lists[0], "logits", 2.0, y, 0.3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.gradients()
    torch.cuda.current_stream().wait_stream(side)
    gu.sync()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.gradients()
        loss = a.distill_loss()
    for rep in range(4):
        F = gu.up(rng.normal(size=(d, n)).astype(np.float32))
        a.F.copy_(F)
        b.F.copy_(F)
        if rep == 2:
            a.set_teacher(*lists[1], "logits")  # the graph goes on with the lists that it was captured with
        g.replay()
        b.gradients()
        want = b.distill_loss()
        gu.sync()
        assert torch.equal(a.G, b.G) and torch.equal(a.hess, b.hess) and torch.equal(a.norm2, b.norm2), rep
        assert torch.equal(loss, want), rep


def test_a_held_update_goes_where_the_call_goes(monkeypatch):
    """The held update and the call that reads its scores run on one device and stream, whichever are current outside."""
    rng = np.random.default_rng(4)
    n, d = 500, 12
    b = Booster(rng.integers(0, 16, (n, 4)).astype(np.uint8), 16, d, "distill", "top_outputs", 3, 2, device=gu.DEV)
    b.set_teacher(gu.up(rng.integers(0, d, (3, n)).astype(np.int32)), gu.up(rng.normal(size=(3, n)).astype(np.float32)))
    inside, kept_on = [], driver._on

    @contextlib.contextmanager
    def on(device, stream):
        with kept_on(device, stream):
            inside.append(device)
            yield
            inside.pop()

    updates, kept = [], driver.L.sb_update_predictions

    def update(*args):
        updates.append(list(inside))
        return kept(*args)

    monkeypatch.setattr(driver, "_on", on)
    monkeypatch.setattr(driver.L, "sb_update_predictions", update)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for call in (b.gradients, b.distill_loss, b.log_probs):
        for stream in (None, s, s.cuda_stream):
            gu.sync()
            b.step()
            gu.sync()
            call(stream=stream)
            assert b.pending is None
    gu.sync()
    assert len(updates) == 9 and all(u and u[0] == b._F.device for u in updates)


def test_only_what_the_loss_uses_is_allocated(monkeypatch):
    rng = np.random.default_rng(4)
    bins = rng.integers(0, 16, (300, 4)).astype(np.uint8)
    asked, kept = [], driver.L.sb_workspace_bytes
    monkeypatch.setattr(driver.L, "sb_workspace_bytes", lambda call, **kw: asked.append(call) or kept(call, **kw))
    other = {driver.L.SB_CALL_GRADIENTS, driver.L.SB_CALL_UPDATE_AND_GRADIENTS}
    for loss in ("softmax", "sigmoid"):
        asked.clear()
        Booster(bins, 16, 12, loss, "top_outputs", 3, 2, device=gu.DEV)
        assert other <= set(asked)
    asked.clear()
    b = Booster(bins, 16, 12, "distill", "top_outputs", 3, 2, device=gu.DEV)
    b.set_teacher(torch.zeros((2, 300), dtype=torch.int32, device=gu.DEV), torch.zeros((2, 300), device=gu.DEV))
    for _ in range(2):
        b.step()
    b.flush()
    gu.sync()
    assert not other & set(asked)
