"""A form of the attention that is not compiled is an error, and not a call that does nothing (behind the stand-in for the HIP runtime of
test_launches.py)."""
import ctypes as C
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
WIDTHS = (8, 32, 64, 72, 80, 96, 104, 128, 200, 256)


def child_forms(lib):
    """Every (type, tiles, head_dim, waves) by the launch itself: what it says, and how many launches there were."""
    seen = []
    for element in ("f16", "bf16", "f32"):
        for tiles in (1, 2, 4):
            name = "launch_attend_%s_%d" % (element, tiles)
            launch = getattr(lib.lib, "_ZN3lif%d%sERKNS_10AttendArgsEiiP12ihipStream_t" % (len(name), name))
            launch.restype, launch.argtypes = C.c_bool, [C.c_void_p, C.c_int, C.c_int, C.c_void_p]
            for dim in WIDTHS:
                for waves in (4, 8, 5):
                    args = (C.c_int32 * 256)(*[dim] * 256)             # head_dim among them; nothing is looked up on the host
                    said, got = lib.launches(lambda: launch(C.addressof(args), 1, waves, None))
                    seen.append((element, tiles, dim, waves, bool(said), len(got)))
    return seen


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    stub = str(tmp_path_factory.getbasetemp() / "hip_host_stub_kv_forms.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", stub, os.path.join(HERE, "hip_host_stub.cpp")], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads(r.stdout.splitlines()[-1])


def test_a_launch_says_whether_it_launched(forms):
    for *form, said, launches in forms:
        assert said == (launches == 1) and launches <= 1, form
    assert not any(said for _, _, _, waves, said, _ in forms if waves == 5)
    by = {tuple(f[:4]): f[4] for f in forms}
    assert by["f16", 1, 64, 8] and by["f32", 4, 128, 4] and by["bf16", 2, 256, 4]
    assert not by["f16", 4, 256, 4] and not by["f32", 4, 72, 4] and not by["bf16", 2, 200, 4]


if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(HERE))
    from tests.test_launches import Library
    print(json.dumps(child_forms(Library(sys.argv[1]))))
