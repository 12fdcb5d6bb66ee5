"""What the calls of the key-value cache launch, looked at without a GPU (behind the stand-in for the HIP runtime of test_launches.py): grids and
blocks fit what the kernels assume, and the workspace holds what the workgroups of any attention call may leave in it."""
import ctypes as C
import json
import os
import random
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
PARTS_MOST = 2048                                          # workgroups of a call that may leave parts
HEAD_DIMS = (8, 24, 32, 40, 64, 80, 88, 96, 112, 128, 136, 200, 256)


def _pad(dim):
    return next(p for p in (32, 64, 80, 96, 128, 256) if dim <= p and (p != 80 or dim == 80))


def _cache(lib, **c):
    b, p = lib.b, lib.p
    cfg = b.LifKvConfig(**dict(dict(layers=2, page_tokens=16, pages=1000, max_seqs=64, rotary_dim=0, norm_eps=1e-5, rotary_scale=1.0, scale=0.1), **c))
    size = lib.lib.lif_kv_workspace_bytes(C.byref(cfg))
    assert size, c
    buf, h = b.LifKvBuffers(p, p, p, p, p, p, None, p, size), C.c_void_p()
    assert lib.lib.lif_kv_create(C.byref(cfg), C.byref(buf), C.byref(h)) == 0, lib.lib.lif_last_error_string()
    return h, size


def child_attend(lib, seed, n):
    rng = random.Random(seed)
    forms = set()
    for _ in range(n):
        kv_heads, share, dim = rng.choice((1, 2, 5, 8, 32)), rng.choice((1, 1, 2, 4, 7, 16, 71)), rng.choice(HEAD_DIMS)
        most, dtype, pages = rng.choice((1, 1, 5, 8, 60, 256)), rng.choice((0, 1, 2)), int(2 ** rng.uniform(0, 17))
        h, size = _cache(lib, heads=kv_heads * share, kv_heads=kv_heads, head_dim=dim, max_pages=pages, max_tokens=most, dtype=dtype)
        for _ in range(8):
            batch, tokens, expected = rng.choice((1, 2, 7, 64, 200, 1024)), rng.randint(1, most), rng.choice((0, 0, 100, 3000, 10 ** 6))
            assert lib.lib.lif_kv_set_expected_tokens(h, expected) == 0
            wide = kv_heads * share * dim
            q = lib.b.LifKvQuery(q=lib.p, out=lib.p, q_stride=wide, out_stride=wide, batch=batch, n_tokens=tokens)
            rc, got = lib.launches(lambda: lib.lib.lif_kv_attend(h, 0, C.byref(q), None))
            case = (kv_heads, share, dim, most, dtype, pages, batch, tokens, expected)
            if rc:                                         # more steps than are counted in 32 bits
                assert not got and batch * kv_heads * (pages * 16 / (64 if dtype == 0 else 128) + 2) > 2 ** 30, case
                continue
            assert len(got) == 1, (case, got)
            kernel, grid, block, lds, _ = got[0]
            form = re.search(r"k_kv_attendI(DF16_|DF16b|f)Li(\d+)ELb(\d)ELi(\d)ELi(\d)EE", kernel)
            element, pad, full, tiles, waves = form[1], int(form[2]), int(form[3]), int(form[4]), int(form[5])
            assert element == ("f", "DF16_", "DF16b")[dtype] and pad == _pad(dim) and full == (pad == dim), (case, kernel)
            rows = tokens * share
            blocks = -(-rows // (16 * tiles))
            assert block == 64 * waves and lds == 0 and grid % blocks == 0 and 0 < grid < 2 ** 31, (case, got)
            # tiles are in use: no block of rows is empty, and most rows are there
            assert 16 * tiles * blocks < rows + 16 * tiles and (blocks == 1 or tiles == 1 or 4 * 16 * tiles * blocks <= 5 * (rows + 15)), (case, kernel)
            if grid // blocks > 1:                         # workgroups that share an item leave parts, of two kinds
                assert grid <= PARTS_MOST, (case, grid)
                assert 4 * grid * min(rows, 16 * tiles) * (pad + 4) * 4 + 4 * PARTS_MOST * 4 <= size, (case, grid, size)
            forms.add((full, tiles, waves))
        lib.lib.lif_kv_destroy(h)
    return sorted(forms)


def child_append(lib, seed, n):
    rng = random.Random(seed)
    for _ in range(n):
        kv_heads, share, dim, dtype = rng.choice((1, 2, 5, 8, 32)), rng.choice((1, 1, 2, 4, 71)), rng.choice(HEAD_DIMS), rng.choice((0, 1, 2))
        most, heads, each = rng.choice((1, 5, 64, 256)), kv_heads * share, 4 if dtype == 0 else 8
        h, _ = _cache(lib, heads=heads, kv_heads=kv_heads, head_dim=dim, max_pages=100, max_tokens=most, dtype=dtype, norm=rng.choice((0, 1, 2)))
        for _ in range(6):
            batch, tokens = rng.choice((1, 3, 64, 1024)), rng.randint(1, most)
            r = lib.b.LifKvRows(q=lib.p, k=lib.p, v=lib.p, q_out=lib.p, q_stride=heads * dim, q_out_stride=heads * dim, k_stride=kv_heads * dim,
                                v_stride=kv_heads * dim, batch=batch, n_tokens=tokens)
            rc, got = lib.launches(lambda: lib.lib.lif_kv_append(h, 1, C.byref(r), None))
            assert rc == 0 and len(got) == 1, (rc, got)
            kernel, grid, block, lds, _ = got[0]
            case = (kv_heads, share, dim, dtype, batch, tokens, grid)
            lanes = 1
            while lanes * each < dim:
                lanes *= 2
            pieces = (tokens + each - 2) // each + 1       # that a row's tokens may lie in, wherever they begin
            value_blocks = -(-kv_heads * dim * (4 if dtype == 0 else 2) // (4 * 256))
            assert "k_kv_append" in kernel and block == 256 and lds == 0 and grid % batch == 0, case
            of_heads = grid // batch - pieces * value_blocks
            assert of_heads > 0 and of_heads % tokens == 0, case
            per = of_heads // tokens                       # workgroups of a token: no more than have heads at once
            assert 1 <= per <= -(-(heads + kv_heads) // (256 // lanes)), case
        lib.lib.lif_kv_destroy(h)
    return n


def child_pages(lib):
    seen = {}
    for seqs in (1, 256, 257, 1024):
        h, _ = _cache(lib, heads=4, kv_heads=4, head_dim=64, max_pages=100, max_tokens=1, dtype=1, max_seqs=seqs)
        p, call = lib.p, lib.lib
        seen[seqs] = {name: [[k[:k.find("E")] if k else k, g, b] for k, g, b, _, _ in lib.launches(f)[1]] for name, f in (
            ("reserve", lambda: call.lif_kv_reserve(h, p, None)), ("truncate", lambda: call.lif_kv_truncate(h, p, None)),
            ("fork", lambda: call.lif_kv_fork(h, p, p, seqs, None)), ("compact", lambda: call.lif_kv_compact(h, None)))}
        call.lif_kv_destroy(h)
    return seen


@pytest.fixture(scope="module")
def child(tmp_path_factory):
    stub = str(tmp_path_factory.getbasetemp() / "hip_host_stub_kv.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", stub, os.path.join(HERE, "hip_host_stub.cpp")], check=True)

    def run(what, *args):
        r = subprocess.run([sys.executable, os.path.abspath(__file__), stub, what] + [json.dumps(a) for a in args], capture_output=True, text=True,
                           timeout=300)
        assert r.returncode == 0, r.stderr[-3000:]
        return json.loads(r.stdout.splitlines()[-1])

    return run


def test_attention_launches_fit_workspace_and_kernels(child):
    forms = child("attend", 1, 400)
    assert [[1, 1, 4], [1, 1, 8], [1, 2, 8], [1, 4, 4], [1, 4, 8]] == [f for f in forms if f[0] and f != [1, 2, 4]], forms
    assert {(f[1], f[2]) for f in forms if not f[0]} >= {(1, 4), (1, 8), (2, 4), (2, 8)}, forms


def test_append_launches(child):
    assert child("append", 2, 200) == 200


def test_page_calls_launch_what_their_plans_assume(child):
    """A thread of the planning workgroup per slot; one launch for a reservation and a truncation, two where pages are copied after a plan"""
    for seqs, calls in child("pages").items():
        threads = 256 if int(seqs) <= 256 else 1024
        assert [b for _, _, b in calls["reserve"]] == [threads] and calls["reserve"][0][1] > 1
        assert [(g, b) for _, g, b in calls["truncate"]] == [(int(seqs), 256)]
        for name in ("fork", "compact"):
            (_, g0, b0), (_, g1, b1) = calls[name]
            assert (g0, b0, b1) == (1, threads, 256) and g1 > int(seqs), (name, calls[name])


if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(HERE))
    from tests.test_launches import Library
    print(json.dumps(globals()["child_" + sys.argv[2]](Library(sys.argv[1]), *map(json.loads, sys.argv[3:]))))
