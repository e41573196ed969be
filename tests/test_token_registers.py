"""Registers of the kernels of trees, weights and moved rows, from the compiler's
metadata and assembly (CPU only), as for the kernels of attention of token chunks."""
import pytest

import test_extend_registers as registers

pytestmark = registers.pytestmark

MORE = {"weigh_kernels.hip": 20, "compact_kernels.hip": 0, "tree_kernels.hip": 0}


@pytest.mark.parametrize("src", sorted(MORE))
def test_these_too(src, tmp_path, monkeypatch):
    monkeypatch.setitem(registers.SPILLS, src, MORE[src])
    registers.test_step_loops_stay_in_registers(src, tmp_path)
