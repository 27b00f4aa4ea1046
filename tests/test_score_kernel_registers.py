"""Vector registers of the kernels on score rows, as the compiler reports them for the package's own flags (no GPU): rows
and lists are held in registers, and one that spills goes through memory in an inner loop.  The distillation kernel of
32-row tiles is left out: it spills some two dozen of its 128 once per tile, not per score.
"""
import pytest

from test_kernel_registers import spilled_registers


@pytest.mark.parametrize("source,kernels", [
    ("sb_logprob.hip", {"k_cols_by_lane<": 8, "k_rows_by_lane<": 24, "k_join<": 3, "k_row_in_block<": 18}),
    ("sb_distill.hip", {"k_distill_regs<64": 18, "k_loss_by_lane<": 2, "k_distill_stats<": 2, "k_distill_rows<": 4,
                        "k_distill_range<": 4}),
])
def test_no_spilled_registers(source, kernels, tmp_path):
    spilled = spilled_registers(source, tmp_path)
    for kernel, instances in kernels.items():
        of = {n: v for n, v in spilled.items() if n.startswith(kernel)}
        assert len(of) == instances, (kernel, sorted(of))
        assert all(v == 0 for v in of.values()), of
