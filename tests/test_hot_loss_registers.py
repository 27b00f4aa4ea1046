"""Vector registers of the kernels of the loss at high temperatures, as the compiler reports them (no GPU)."""
from test_kernel_registers import spilled_registers


def test_no_spilled_registers(tmp_path):
    spilled = spilled_registers("sb_distill.hip", tmp_path)
    of = {n: v for n, v in spilled.items() if n.startswith("k_hot_")}
    assert len(of) == 4 and not any(of.values()), of
