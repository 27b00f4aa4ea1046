"""Spilled vector registers of the distillation kernel of 32-row tiles (513 to 1024 classes), as the compiler reports them
(no GPU): 16 waves leave 128 registers to a lane that holds 32 scores, and what spills does so once per tile.  More than
this would be the scores' addresses, formed ahead of the loads and held.
"""
from test_kernel_registers import spilled_registers


def test_32_row_tiles(tmp_path):
    spilled = spilled_registers("sb_distill.hip", tmp_path)
    of = {n: v for n, v in spilled.items() if n.startswith("k_distill_regs<32")}
    assert len(of) == 12, sorted(of)
    assert all(v <= 40 for v in of.values()), of
