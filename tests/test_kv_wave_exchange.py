"""What lanes of a wave hand to one another in LDS without a barrier among the waves: the compiled kernels keep the order of it (the hardware does by
itself, the compiler where it is told to)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2312_11514_amd import build


@pytest.mark.parametrize("source", ["kv_attend_bf16_1.hip", "kv_attend_f16_2.hip", "kv_attend_f32_4.hip"])
def test_exchanges_inside_a_wave_are_ordered(source):
    """One before parts are added (which ones, by the first lane), and, with several tiles, one before positions are looked at one by one (what a row
    sees, by the lanes of the first group)."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("no hipcc")
    text = subprocess.run([hipcc, *build.flags_of(source), "--offload-device-only", "-S", "-o", "-", os.path.join(build.HERE, "csrc", source)],
                          capture_output=True, text=True, check=True).stdout
    kernels = re.findall(r"^_ZN3lif11k_kv_attendI(?:DF16_|DF16b|f)Li(\d+)ELb(\d)ELi(\d)ELi(\d)EE\w*:(.*?)^\.Lfunc_end", text, re.M | re.S)
    assert kernels
    for dim, exact, tiles, waves, body in kernels:
        assert body.count("wave barrier") >= (2 if int(tiles) > 1 else 1), (source, dim, exact, tiles, waves)
