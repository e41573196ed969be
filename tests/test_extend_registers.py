"""Registers of the kernels of attention of token chunks, from the compiler's
metadata and assembly (CPU only): no kernel keeps its arguments in scratch memory,
and the blocks of matrix products in their step loops reload nothing from there (a
scratch reload comes with a wait for the loads in flight)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_24506_amd import build

pytestmark = pytest.mark.skipif(not os.path.exists(build.HIPCC) and shutil.which("hipcc") is None, reason="no hipcc")

SPILLS = {"extend_rows.hip": 20, "extend_mla.hip": 20, "extend_kernels.hip": 0, "rope_kernels.hip": 0}


@pytest.mark.parametrize("src", sorted(SPILLS))
def test_step_loops_stay_in_registers(src, tmp_path):
    out = tmp_path / "k.s"
    subprocess.run([build.HIPCC, *build.DEVICE_FLAGS, *build.KERNEL_FLAGS, *build.COMMON, "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, src), "-o", str(out)], check=True, capture_output=True, text=True)
    text = out.read_text()
    kernels = re.findall(r"^(_ZN2cp\w*kernel\w*):.*?^\.Lfunc_end", text, flags=re.M | re.S)
    assert kernels
    meta = text[text.index("amdhsa.kernels:"):]
    spilled = {m.group(1): int(m.group(2)) for m in
               re.finditer(r"\.symbol:\s+(\w+)\.kd.*?\.vgpr_spill_count:\s+(\d+)", meta, flags=re.S)}
    assert set(kernels) <= set(spilled)
    for name in kernels:
        assert spilled[name] <= SPILLS[src], (name, spilled[name])
        body = re.search(r"^" + name + r":(.*?)^\.Lfunc_end", text, flags=re.M | re.S).group(1)
        for block in re.split(r"^\.LBB\w+:", body, flags=re.M):
            if len(re.findall(r"\bv_mfma", block)) >= 16:  # eight or more products of a step
                assert len(re.findall(r"\bscratch_", block)) == 0, name
