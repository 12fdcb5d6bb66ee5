"""What add_norm and the packed weights launch, looked at without a GPU (behind the stand-in for the HIP runtime of test_launches.py): grids and blocks fit
what the kernels assume, every form that a rule can choose is there, and the rule takes the forms that its comment says."""
import ctypes as C
import json
import os
import random
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
SIZES = {0: 4, 1: 2, 2: 2}


def _handle(lib, **c):
    b = lib.b
    cfg, h = b.LifPackedConfig(**c), C.c_void_p()
    buf = b.LifPackedBuffers(1 << 36, 1 << 38, lib.lib.lif_packed_code_bytes(C.byref(cfg)), lib.lib.lif_packed_group_bytes(C.byref(cfg)))
    assert lib.lib.lif_packed_create(C.byref(cfg), C.byref(buf), C.byref(h)) == 0, lib.lib.lif_last_error_string()
    return h


def child_multiply(lib, seed, n):
    rng, forms = random.Random(seed), set()
    for _ in range(n):
        n_out, n_in, group, zeros, dtype = int(2 ** rng.uniform(0, 20)), 8 * int(2 ** rng.uniform(0, 13)), rng.choice((32, 64, 128)), rng.choice((0, 1)), rng.choice((0, 1, 2))
        h = _handle(lib, n_out=n_out, n_in=n_in, group=group, zeros=zeros, dtype=dtype)
        for rows in [1, 4, 5, 8, 9, 16, 17, 1 << 19] + [int(2 ** rng.uniform(0, 19)) for _ in range(4)]:
            eight = rng.choice((0, 0, 1, 2))
            far = 1 << 42                                  # (arrays that do not overlap)
            r = lib.b.LifPackedRows(x=far, x_scales=2 * far if eight else None, out=3 * far, x_stride=n_in, out_stride=n_out, n_rows=rows,
                                    x_group=group if eight == 2 else 0)
            rc, got = lib.launches(lambda: lib.lib.lif_packed_multiply(h, C.byref(r), None))
            case = (n_out, n_in, group, zeros, dtype, rows, eight)
            assert rc == 0 and len(got) == 1, (case, rc, got)
            kernel, grid, block, lds, _ = got[0]
            assert lds == 0 and 0 < grid < 2 ** 32, case
            tiles = -(-n_out // 16)
            few = re.search(r"k_packed_fewI(\w+?)Li(\d+)ELb(\d)ELi(\d)ELi(\d)ELi(\d)EE", kernel)
            many = re.search(r"k_packed_manyI(\w+?)Li(\d+)ELb(\d)ELi(\d)ELi(\d)ELi(\d)EE", kernel)
            m = few or many
            groups = -(-n_in // group)
            element = "NS_7ByGroupE" if eight == 2 and groups > 1 else "a" if eight else ("f", "DF16_", "DF16b")[dtype]
            assert (m[1], int(m[2]), int(m[3])) == (element, group, zeros), (case, kernel)
            if few:
                quads, waves = int(m[4]), int(m[6])
                assert block == 64 * waves and grid == tiles * -(-rows // 16) and (quads == 4 or rows <= 4 * quads), (case, kernel, grid)
                forms.add(("few", element == "f", quads))
            else:
                nt, wn, wk = (int(m[i]) for i in (4, 5, 6))
                assert rows > 16 and block == 64 * wn * wk <= 1024 and grid == -(-tiles // wn) * -(-rows // (16 * nt)), (case, kernel, grid)
                forms.add(("many", element == "f", nt, wn, wk))
        lib.lib.lif_packed_destroy(h)
    return sorted(map(str, forms))


def child_norm(lib, seed, n):
    rng, forms = random.Random(seed), set()
    for _ in range(n):
        width, rows, dtype = 8 * int(2 ** rng.uniform(0, 13)), rng.choice((1, 2, 100, 1023, 1024, 5000, 1 << 19)), rng.choice((0, 1, 2))
        eight, far = rng.choice((0, 1)), 1 << 40
        a = lib.b.LifNormRows(x=far, out=2 * far, scales=3 * far if eight else None, x_stride=width, out_stride=width, n_rows=rows, width=width, dtype=dtype,
                              norm=rng.choice((0, 1, 2)), group=rng.choice((0, 32, 128)) if eight else 0, eps=1e-5)
        rc, got = lib.launches(lambda: lib.lib.lif_add_norm(C.byref(a), None))
        case = (width, rows, dtype, eight, a.norm)
        assert rc == 0 and len(got) == 1, (case, rc, got, lib.lib.lif_last_error_string())
        kernel, grid, block, lds, _ = got[0]
        m = re.search(r"k_add_normI(DF16_|DF16b|f)Li(\d)ELb(\d)ELi(\d)EE", kernel)
        pieces = int(m[2])
        assert (m[1], int(m[3]), int(m[4])) == (("f", "DF16_", "DF16b")[dtype], eight, a.norm), (case, kernel)
        # a piece of 8 for every thread, no wave without one
        assert grid == rows and block % 64 == 0 and 64 <= block <= 1024 and block * pieces * 8 >= width > (block - 64) * pieces * 8, (case, kernel, block)
        forms.add(pieces)
    return sorted(forms)


def child_make(lib):
    seen = []
    for n_out, n_in in ((1, 8), (17, 136), (4096, 4096), (1 << 20, 65536)):
        for dtype in (0, 1, 2):
            for zeros in (0, 1):
                h = _handle(lib, n_out=n_out, n_in=n_in, group=64, zeros=zeros, dtype=dtype)
                tiles, call, far = -(-n_out // 16) * -(-n_in // 128), lib.lib, 1 << 42        # (arrays beyond those of the matrix)
                for f in (lambda: call.lif_packed_quantize(h, far, n_in, None), lambda: call.lif_packed_dequantize(h, far, n_in, None),
                          lambda: call.lif_packed_pack(h, far, far, far if zeros else None, None)):
                    rc, got = lib.launches(f)
                    assert rc == 0 and [(g, b) for _, g, b, _, _ in got] == [(min(tiles, 2048), 256)], (n_out, n_in, got)
                    seen.append(got[0][0])
                lib.lib.lif_packed_destroy(h)
    return len(set(seen))


@pytest.fixture(scope="module")
def child(tmp_path_factory):
    stub = str(tmp_path_factory.getbasetemp() / "hip_host_stub_packed.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", stub, os.path.join(HERE, "hip_host_stub.cpp")], check=True)

    def run(what, *args):
        r = subprocess.run([sys.executable, os.path.abspath(__file__), stub, what] + [json.dumps(a) for a in args], capture_output=True, text=True,
                           timeout=300)
        assert r.returncode == 0, r.stderr[-3000:]
        return json.loads(r.stdout.splitlines()[-1])

    return run


def test_products(child):
    forms = child("multiply", 1, 500)
    few = {"('few', %s, %d)" % (f32, q) for f32 in (False, True) for q in (1, 2, 4)}
    many = {"('many', False, %d, %d, %d)" % f for f in ((1, 2, 4), (1, 2, 8), (2, 2, 4), (2, 2, 8), (2, 3, 5), (2, 4, 4), (2, 4, 2), (3, 3, 4), (3, 4, 2), (4, 4, 4), (4, 4, 2), (4, 5, 3), (2, 6, 2), (4, 6, 2),
                                                          (3, 7, 2), (4, 8, 1))}
    many |= {"('many', True, %d, %d, %d)" % f for f in ((1, 2, 4), (1, 4, 2), (4, 8, 1))}
    assert set(forms) == few | many, sorted(set(forms) ^ (few | many))


def test_norms(child):
    assert child("norm", 2, 400) == [1, 2, 4, 8]


def test_making_weights(child):
    assert child("make") == 3 * 2 + 3 + 1


@pytest.mark.parametrize("tiles,in_tiles,rows,f32,group,form", [
    (256, 32, 1, 0, 128, "few4"), (256, 32, 5, 0, 128, "few8"), (256, 32, 16, 0, 128, "few16"), (64, 32, 64, 0, 128, "few16"), (256, 32, 24, 0, 128, "outs32_rows16"),
    (256, 86, 24, 0, 128, "outs32_rows16_16"), (256, 32, 60, 0, 32, "outs32_rows32"), (256, 86, 60, 0, 32, "outs32_rows32_16"), (688, 32, 24, 0, 128, "outs48_rows32"),
    (688, 32, 48, 0, 128, "outs48_rows48"), (256, 32, 128, 0, 128, "outs64_rows32_16"), (1537, 32, 17, 0, 128, "outs64_rows32"), (257, 32, 97, 0, 32, "outs64_rows48"),
    (385, 32, 97, 0, 64, "outs64_rows64_16"), (688, 32, 256, 0, 64, "outs64_rows64"), (385, 32, 97, 0, 32, "outs64_rows32"), (1136, 36, 48, 0, 64, "outs80_rows64"),
    (1136, 32, 32, 0, 128, "outs96_rows32"), (688, 32, 256, 0, 32, "outs96_rows64"), (1376, 32, 48, 0, 64, "outs112_rows48"), (256, 32, 777, 0, 128, "outs128_rows64"),
    (3126, 32, 512, 0, 128, "outs128_rows64"), (64, 32, 64, 1, 64, "few16"), (256, 32, 128, 1, 64, "outs64_rows16"), (3126, 32, 512, 1, 64, "outs128_rows64")])
def test_the_rule(tmp_path, tiles, in_tiles, rows, f32, group, form):
    source = tmp_path / "rule.cpp"
    header = os.path.join(os.path.dirname(HERE), "paper_2312_11514_amd", "csrc", "lif_packed_form.h")
    source.write_text('#include "%s"\nint main() { return lif::packed_form(%d, %d, %d, %s, %d) == lif::PackedForm::%s ? 0 : 1; }\n' %
                      (header, tiles, in_tiles, rows, "true" if f32 else "false", group, form))
    subprocess.run(["g++", "-std=c++17", "-o", str(tmp_path / "rule"), str(source)], check=True)
    assert subprocess.run([str(tmp_path / "rule")]).returncode == 0


if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(HERE))
    from tests.test_launches import Library
    print(json.dumps(globals()["child_" + sys.argv[2]](Library(sys.argv[1]), *map(json.loads, sys.argv[3:]))))
