"""Registers of the products of weights in 4 bits, as the compiler reports them: none goes to memory, and forms for many rows leave some for four waves on a
SIMD, which their arithmetic needs."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2312_11514_amd import build


@pytest.mark.parametrize("source", ["packed_bf16.hip", "packed_i8_groups.hip"])
def test_products_fit_their_registers(source):
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
    few, many = ([v for k, v in kernels.items() if kind in k] for kind in ("k_packed_few", "k_packed_many"))
    assert len(few) == 3 * 2 * 3 and len(many) == 2 * (16 + 16 + 13)
    assert all(v["VGPRs Spill"] == "0" for v in few + many), [(k, v["VGPRs Spill"]) for k, v in kernels.items() if v.get("VGPRs Spill") != "0"]
    assert all(int(v["VGPRs"]) + int(v["AGPRs"]) <= 512 // 4 for v in many)
