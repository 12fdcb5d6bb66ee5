"""Registers of the attention over pages, as the compiler reports them: forms whose workgroups have eight waves fit two of them on a SIMD, and
no register goes to memory in a form for exactly so many dimensions."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2312_11514_amd import build


@pytest.mark.parametrize("source", ["kv_attend_f16_2.hip", "kv_attend_bf16_4.hip"])
def test_forms_of_several_tiles_fit_their_registers(source):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("no hipcc")
    text = subprocess.run([hipcc, *build.flags_of(source), "--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-c", "-o", os.devnull,
                           os.path.join(build.HERE, "csrc", source)], capture_output=True, text=True, check=True).stderr
    kernels, name = {}, None
    for key, value in re.findall(r"remark: .*?([A-Za-z][A-Za-z ]*?)(?: \[[^\]]*\])?: (\S+)", text):
        if key == "Function Name":
            name = re.search(r"k_kv_attendI(?:DF16_|DF16b|f)Li(\d+)ELb(\d)ELi(\d)ELi(\d)EE", value)
        elif name:
            kernels.setdefault(tuple(int(v) for v in name.groups()), {})[key] = value
    assert kernels
    for (dim, exact, tiles, waves), got in kernels.items():
        if exact and tiles * dim <= 256:
            assert got["VGPRs Spill"] == "0", (dim, tiles, waves, got)
        if waves == 8:
            assert int(got["Occupancy"]) >= 2, (dim, tiles, waves, got)
    assert {(128, 1, 2, 8), (64, 1, 2, 8)} <= set(kernels) or {(64, 1, 4, 8), (128, 1, 4, 4)} <= set(kernels)
