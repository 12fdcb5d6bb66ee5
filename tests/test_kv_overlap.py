"""Queries and outputs of attention and of rows of a cache that share memory: rows that are the same ones are fine, any other overlap is refused (behind the stand-in for
the HIP runtime of test_launches.py)."""
import ctypes as C
import json
import os
import random
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
SIZES = {0: 4, 1: 2, 2: 2}


def _cache(lib, dtype, heads, dim):
    b, p = lib.b, lib.p
    cfg = b.LifKvConfig(layers=1, heads=heads, kv_heads=1, head_dim=dim, page_tokens=16, pages=64, max_seqs=8, max_pages=8, max_tokens=8, dtype=dtype,
                        rotary_dim=0, norm_eps=1e-5, rotary_scale=1.0, scale=0.1)
    size, h = lib.lib.lif_kv_workspace_bytes(C.byref(cfg)), C.c_void_p()
    buf = b.LifKvBuffers(p, p, p, p, p, p, None, p, size)
    assert lib.lib.lif_kv_create(C.byref(cfg), C.byref(buf), C.byref(h)) == 0
    return h


def _shares(a, a_step, b, b_step, rows, size):
    taken = set()
    for r in range(rows):
        taken.update(range(a + r * a_step, a + r * a_step + size, 16))
    return any(x in taken for r in range(rows) for x in range(b + r * b_step, b + r * b_step + size, 16))


def _calls(lib, seed, launch):
    """[refused or not, what every byte says] of calls with random places and strides, most of them close to one another"""
    rng, seen, p = random.Random(seed), [], lib.p + (1 << 24)
    for _ in range(4000):
        dtype, heads, dim = rng.choice((0, 1, 2)), rng.choice((1, 2, 3)), rng.choice((8, 24))
        e, width = SIZES[dtype], heads * dim
        each = 16 // e
        batch, tokens = rng.randint(1, 4), rng.randint(1, 5)
        stride = lambda: (width + each - 1) // each * each + each * rng.choice((0, 0, 1, 5, 2 * width // each, 40))
        q_stride = stride()
        out_stride = q_stride if rng.random() < 0.6 else stride()
        at = 16 * rng.choice((0, 0, 1, -1, width * e // 16, -width * e // 16, rng.randint(-300, 300), q_stride * e // 16, 4000))
        h = _cache(lib, dtype, heads, dim)
        rc, got = lib.launches(launch(h, p, p + at, q_stride, out_stride, batch, tokens, heads * dim))
        lib.lib.lif_kv_destroy(h)
        rows = batch * tokens
        same = at == 0 and (q_stride == out_stride or rows == 1)
        bad = not same and _shares(p, q_stride * e, p + at, out_stride * e, rows, width * e)
        assert (rc, len(got)) == ((1, 0) if bad else (0, 1)), (dtype, heads, dim, batch, tokens, q_stride, out_stride, at, rc, got)
        seen.append((bool(bad), same, q_stride == out_stride))
    return [sum(s[0] and not s[2] for s in seen), sum(s[0] and s[2] for s in seen), sum(s[1] for s in seen), sum(not s[0] and not s[1] for s in seen)]


def child_attend(lib, seed):
    def launch(h, q, out, q_stride, out_stride, batch, tokens, _):
        query = lib.b.LifKvQuery(q=q, out=out, q_stride=q_stride, out_stride=out_stride, batch=batch, n_tokens=tokens)
        return lambda: lib.lib.lif_kv_attend(h, 0, C.byref(query), None)
    return _calls(lib, seed, launch)


def child_append(lib, seed):
    def launch(h, q, out, q_stride, out_stride, batch, tokens, width):
        k = lib.p + (1 << 30)
        rows = lib.b.LifKvRows(q=q, k=k, v=k, q_out=out, q_stride=q_stride, k_stride=width, v_stride=width, q_out_stride=out_stride, batch=batch,
                               n_tokens=tokens)
        return lambda: lib.lib.lif_kv_append(h, 0, C.byref(rows), None)
    return _calls(lib, seed, launch)


@pytest.fixture(scope="module")
def child(tmp_path_factory):
    stub = str(tmp_path_factory.getbasetemp() / "hip_host_stub_kv_overlap.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", stub, os.path.join(HERE, "hip_host_stub.cpp")], check=True)

    def run(what, *args):
        r = subprocess.run([sys.executable, os.path.abspath(__file__), stub, what] + [json.dumps(a) for a in args], capture_output=True, text=True,
                           timeout=300)
        assert r.returncode == 0, r.stderr[-3000:]
        return json.loads(r.stdout.splitlines()[-1])

    return run


def test_outputs_that_overlap_queries(child):
    assert all(n >= 200 for n in child("attend", 1))


def test_turned_queries_that_overlap_queries(child):
    assert all(n >= 200 for n in child("append", 2))


if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(HERE))
    from tests.test_launches import Library
    print(json.dumps(globals()["child_" + sys.argv[2]](Library(sys.argv[1]), *map(json.loads, sys.argv[3:]))))
