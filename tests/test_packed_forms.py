"""A form of the products that is not compiled is an error, and not a call that does nothing; and the rule asks for none (behind the stand-in for the HIP
runtime of test_launches.py)."""
import ctypes as C
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.dirname(HERE))
from tests.packed_forms import form_names, forms  # noqa: E402

TYPES = ("f32", "f16", "bf16", "i8", "i8_groups")


class Product(C.Structure):
    """ProductArgs of lif_packed_few.h"""
    _fields_ = [(n, C.c_void_p) for n in ("codes", "groups")] + [(n, C.c_int32) for n in ("n_out", "n_in", "group", "in_tiles", "n_groups", "gap")] + \
        [(n, C.c_void_p) for n in ("x", "out", "x_scales", "bias")] + [(n, C.c_int64) for n in ("x_stride", "out_stride")] + \
        [(n, C.c_int32) for n in ("rows", "x_groups", "out_type")]


def child_forms(lib, count):
    """Every (type, form, group, zeros) by the launch itself: what it says, and how many launches there were."""
    seen = []
    for kind in TYPES:
        name = "launch_product_" + kind
        launch = getattr(lib.lib, "_ZN3lif%d%sERKNS_11ProductArgsENS_10PackedFormEbP12ihipStream_t" % (len(name), name))
        launch.restype, launch.argtypes = C.c_bool, [C.c_void_p, C.c_int, C.c_bool, C.c_void_p]
        for group in (32, 64, 128, 256):
            args = Product(n_out=1000, n_in=512, group=group, in_tiles=4, n_groups=512 // group, rows=100, x_stride=512, out_stride=1000, x_groups=1)
            for form in range(count + 1):
                for zeros in (False, True):
                    said, got = lib.launches(lambda: launch(C.addressof(args), form, zeros, None))
                    seen.append((kind, form, group, zeros, bool(said), len(got)))
    return seen


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    stub = str(tmp_path_factory.getbasetemp() / "hip_host_stub_packed_forms.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", stub, os.path.join(HERE, "hip_host_stub.cpp")], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub, str(len(form_names()))], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    return [tuple(v) for v in json.loads(r.stdout.splitlines()[-1])]


def test_a_launch_says_whether_it_launched(launched):
    names = form_names() + ["beyond the last"]
    by = {}
    for kind, form, group, zeros, said, launches in launched:
        assert said == (launches == 1) and launches <= 1, (kind, names[form], group, zeros)
        by.setdefault((kind, names[form], group), set()).add(said)
    assert all(len(v) == 1 for v in by.values())            # (zero points change nothing in that)
    assert by["f16", "outs128_rows64", 32] == by["f32", "outs64_rows16", 64] == by["i8_groups", "few4", 128] == {True}
    assert by["bf16", "outs64_rows64", 32] == by["f32", "outs48_rows48", 64] == by["f16", "outs64_rows16", 128] == by["f16", "few4", 256] == {False}
    assert not any(True in by[kind, "beyond the last", group] for kind in TYPES for group in (32, 64, 128))


def test_the_rule_asks_for_forms_that_are_there(launched, tmp_path):
    there = {(kind, form_names()[form], group) for kind, form, group, _, said, _ in launched if said}
    counts = [(rows, n_in, n_out) for rows in (1, 4, 5, 8, 9, 16, 17, 24, 33, 40, 48, 60, 64, 65, 97, 128, 200, 300, 512, 777, 1024, 5000, 1 << 19)
              for n_in in (8, 128, 712, 1528, 4096, 5128, 11008, 65536) for n_out in (1, 45, 300, 1024, 2061, 4096, 6157, 8205, 11008, 12557, 16397, 18176, 50001, 1 << 20)]
    asked = [(*c, group, f32) for c in counts for group in (32, 64, 128) for f32 in (False, True)]
    seen = set()
    for (_, _, _, group, f32), name in zip(asked, forms(tmp_path, asked)):
        for kind in TYPES[:1] if f32 else TYPES[1:]:
            assert (kind, name, group) in there, (kind, name, group)
        seen.add(name)
    assert seen == set(form_names())


if __name__ == "__main__":
    from tests.test_launches import Library
    print(json.dumps(child_forms(Library(sys.argv[1]), int(sys.argv[2]))))
