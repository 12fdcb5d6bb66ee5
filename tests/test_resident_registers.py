"""Registers of the norms, and of the products in the types that test_packed_registers.py does not look at, as the compiler reports them: none goes to memory."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2312_11514_amd import build

# (kernels of a source: norms by pieces, 8 bits and norm; products by group, zero points and form)
KERNELS = {"norm_f32.hip": 4 * 2 * 3, "norm_f16.hip": 4 * 2 * 3, "norm_bf16.hip": 4 * 2 * 3, "packed_f32.hip": 3 * 2 * (3 + 3),
           "packed_f16.hip": 3 * 2 * 3 + 2 * (16 + 16 + 13), "packed_i8.hip": 3 * 2 * 3 + 2 * (16 + 16 + 13)}


@pytest.mark.parametrize("source", KERNELS)
def test_kernels_fit_their_registers(source):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("no hipcc")
    text = subprocess.run([hipcc, *build.flags_of(source), "--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-c", "-o", os.devnull,
                           os.path.join(build.HERE, "csrc", source)], capture_output=True, text=True, check=True).stderr
    kernels, name = {}, None
    for key, value in re.findall(r"remark: .*?([A-Za-z][A-Za-z ]*?)(?: \[[^\]]*\])?: (\S+)", text):
        if key == "Function Name":
            name = value
        elif name:
            kernels.setdefault(name, {})[key] = value
    assert len(kernels) == KERNELS[source], sorted(kernels)
    assert all(v["VGPRs Spill"] == "0" and v["ScratchSize"] == "0" for v in kernels.values()), [k for k, v in kernels.items() if v["ScratchSize"] != "0"]
