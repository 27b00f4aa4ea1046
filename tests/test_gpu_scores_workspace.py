"""Row-major scores need no workspace, whatever sb_workspace_bytes gives for column-major ones of the same sizes."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import gpu_util as gu  # noqa: E402
from paper_2211_12858_amd import _lib as L  # noqa: E402
from paper_2211_12858_amd import driver  # noqa: E402


@pytest.mark.parametrize("n,d,k", [(1, 1000, 5), (70, 640, 10), (100, 20_000, 64)])
def test_row_major_without_workspace(n, d, k):
    assert L.sb_workspace_bytes(L.SB_CALL_LOG_PROBS, n=n, d=d, k=k) > 0
    F = torch.randn((n, d), device=gu.DEV)
    lse, entropy = torch.empty(n, device=gu.DEV), torch.empty(n, device=gu.DEV)
    top_id, top_logp = torch.empty((k, n), dtype=torch.int32, device=gu.DEV), torch.empty((k, n), device=gu.DEV)
    L.sb_log_probs(F, L.SB_F32, L.SB_ROW_MAJOR, n, d, d, 1.0, None, None, None, lse, entropy, k, top_id, top_logp, n, None, 0)
    want = driver.log_probs(F, k=k, order="row")
    assert torch.equal(top_id, want.top_id) and torch.equal(top_logp, want.top_logp) and torch.equal(lse, want.lse)
    with pytest.raises(L.SBError):  # the column-major call does need it
        L.sb_log_probs(F, L.SB_F32, L.SB_COLUMN_MAJOR, n, d, n + (n == 1), 1.0, None, None, None, lse, entropy, k, top_id,
                       top_logp, n, None, 0)


def test_no_workspace_is_allocated_for_row_major_scores(monkeypatch):
    F = torch.randn((100, 20_000), device=gu.DEV)
    asked = []
    kept = driver.workspace
    monkeypatch.setattr(driver, "workspace", lambda nbytes, dev: asked.append(nbytes) or kept(nbytes, dev))
    driver.log_probs(F, k=20, order="row")
    assert not any(asked)
    driver.log_probs(F.t().contiguous(), k=20)
    assert any(asked)
