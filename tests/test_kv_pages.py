"""The page calls of the key-value cache against the oracle: which page goes where, what is copied, what refuses."""
import random

import numpy as np
import pytest
import torch

import paper_2312_11514_amd as lif
from oracle.kv_oracle import PagedOracle
from tests.kv_harness import ints
from workloads.device import require_gpu

pytestmark = pytest.mark.gpu


def _cache(pages, max_seqs, max_pages, page=16, layers=2, kv_heads=2, dtype="f16", head_dim=8):
    require_gpu()
    kv = lif.KVCache(layers=layers, heads=kv_heads, kv_heads=kv_heads, head_dim=head_dim, page_tokens=page, pages=pages, max_seqs=max_seqs,
                     max_pages=max_pages, dtype=dtype)
    # every page is told apart by its number, in every layer's first and last element of keys and values
    stamp = torch.arange(pages, device="cuda", dtype=torch.float32) % 1000
    for l in range(layers):
        kv.k[l] = (stamp + l).view(-1, 1, 1, 1).to(kv.k.dtype)
        kv.v[l] = (stamp + 3 * l + 1).view(-1, 1, 1, 1, 1).to(kv.v.dtype)
    return kv, PagedOracle(pages, max_seqs, max_pages, page), (kv.k.clone(), kv.v.clone())


def _compare(kv, o, first, what):
    st = kv.state()
    assert st["error"] == o.error, (what, st, o.error)
    assert kv.lengths.tolist() == o.lengths, what
    assert kv.fresh.tolist() == o.fresh, what
    assert kv.table.tolist() == o.table(), what
    assert kv.refs.tolist() == o.refs(), what
    assert st["used_pages"] == o.used(), what
    assert st["moved_pages"] == o.moved, what
    # contents: of the pages in use, every one is a copy of the page it came from
    held = sorted({p for t in o.tables for p in t})
    if held:
        came = [o.content[p][1] for p in held]
        assert torch.equal(kv.k[:, held], first[0][:, came]), what
        assert torch.equal(kv.v[:, held], first[1][:, came]), what


@pytest.mark.parametrize("seed,pages,seqs,width,page", [(1, 40, 5, 12, 16), (2, 200, 40, 9, 32), (3, 64, 3, 64, 16), (4, 65, 7, 30, 256),
                                                         (5, 300, 1000, 3, 16), (6, 1, 2, 1, 16), (7, 5000, 33, 700, 16)])
def test_random_calls(seed, pages, seqs, width, page):
    kv, o, first = _cache(pages, seqs, width, page)
    _compare(kv, o, first, "reset")
    rng = random.Random(seed)
    seen = set()
    for step in range(60):
        call = rng.choice(["reserve", "reserve", "reserve", "truncate", "fork", "fork", "compact"])
        if o.error and rng.random() < 0.5:
            call = "truncate"
        if call == "reserve":
            most = max(1, pages * page * 2 // (seqs * 3))
            counts = [rng.choice([0, 1, 5, rng.randint(-3, most)]) if rng.random() < 0.7 else 0 for _ in range(seqs)]
            o.reserve(counts)
            kv.reserve(ints(counts))
        elif call == "truncate":
            to = [rng.choice([-1, -1, 0, 0, rng.randint(0, n + 3), n]) for n in o.lengths]
            o.truncate(to)
            kv.truncate(ints(to))
        elif call == "fork":
            empty = [s for s in range(seqs) if o.lengths[s] == 0]
            dst = rng.sample(empty, min(len(empty), rng.randint(1, 4))) or [0]
            src = [rng.randrange(seqs) for _ in dst]
            if rng.random() < 0.1:
                dst[0] = rng.randrange(-1, seqs + 1)
            o.fork(src, dst)
            kv.fork(ints(src), ints(dst))
        else:
            o.compact()
            kv.compact()
        seen.add((call, o.error))
        _compare(kv, o, first, (seed, step, call))
    assert len(seen) >= 4, seen


def test_tokens_behind_a_shared_page_get_a_copy():
    kv, o, first = _cache(8, 3, 4)
    for call in (lambda c: c.reserve([40, 0, 0]), lambda c: c.fork([0], [1]), lambda c: c.fork([0], [2]),
                 lambda c: c.truncate([20, 20, 32]),                        # into the second page, which all three hold
                 lambda c: c.reserve([1, 2, 0]),                            # the first two get copies, the third keeps the page
                 lambda c: c.truncate([17, 17, 17]),
                 lambda c: c.reserve([1, 1, 1])):
        call(o)
        call(_Gpu(kv))
        _compare(kv, o, first, "shared")
    # both holders of a page leave it at once: it is free again
    kv, o, first = _cache(4, 2, 2)
    for call in (lambda c: c.reserve([16, 0]), lambda c: c.fork([0], [1]), lambda c: c.truncate([5, 5]), lambda c: c.reserve([1, 1])):
        call(o)
        call(_Gpu(kv))
        _compare(kv, o, first, "left")
    assert o.moved == 2 and o.used() == 2


class _Gpu:
    def __init__(self, kv):
        self.kv = kv

    def reserve(self, c):
        self.kv.reserve(ints(c))

    def truncate(self, c):
        self.kv.truncate(ints(c))

    def fork(self, s, d):
        self.kv.fork(ints(s), ints(d))


def test_a_call_that_does_not_fit_changes_nothing_and_later_ones_wait_for_a_truncation():
    kv, o, first = _cache(4, 3, 3)
    g = _Gpu(kv)
    g.reserve([40, 10, 0])
    o.reserve([40, 10, 0])
    _compare(kv, o, first, "full")
    for counts in ([0, 0, 1], [0, 39, 0], [2 ** 31 - 1, 0, 0]):             # no page; no column; more than a table holds
        g.reserve(counts)
        o.reserve(counts)
        assert o.error == lif.binding.LIF_CAPACITY
        _compare(kv, o, first, counts)
        g.reserve([1, 0, 0])                                                # (nothing)
        kv.compact()
        g.fork([0], [2])
        _compare(kv, o, first, "waits")
        g.truncate([-1, -1, -1])
        o.truncate([-1, -1, -1])
    g.reserve([8, 0, 0])
    o.reserve([8, 0, 0])
    _compare(kv, o, first, "goes on")
    for src, dst in (([0, 0], [2, 2]), ([0], [1]), ([3], [2]), ([0], [-1])):
        g.fork(src, dst)
        o.fork(src, dst)
        assert o.error == lif.binding.LIF_INVALID_ARG
        _compare(kv, o, first, (src, dst))
        g.truncate([-1, -1, -1])
        o.truncate([-1, -1, -1])


def test_adopted_tables():
    kv, o, first = _cache(70, 4, 5)
    table = np.full((4, 5), -7, np.int32)
    table[0, :3], table[2, :1], table[3, :2] = [69, 3, 64], [3], [0, 63]
    kv.table.copy_(torch.from_numpy(table))
    kv.lengths.copy_(ints([33, 0, 16, 32]))
    kv.fresh.copy_(ints([1, 0, 16, 0]))
    kv.adopt()
    o.tables, o.lengths, o.fresh = [[69, 3, 64], [], [3], [0, 63]], [33, 0, 16, 32], [1, 0, 16, 0]
    _compare(kv, o, first, "adopted")
    kv.compact()
    o.compact()
    _compare(kv, o, first, "compact")
    g = _Gpu(kv)
    g.reserve([20, 1, 1, 1])
    o.reserve([20, 1, 1, 1])
    _compare(kv, o, first, "reserve")
    for bad in ("length", "fresh", "page"):
        if bad == "length":
            kv.lengths[1] = 81
        elif bad == "fresh":
            kv.lengths[1] = 3
            kv.fresh[1] = 4
        else:
            kv.fresh[1] = 0
            kv.table[1, 0] = 70
        kv.adopt()
        assert kv.state()["error"] == lif.binding.LIF_BAD_STATE, bad
        kv.truncate(ints([0] * 4))
        assert kv.state()["error"] == lif.binding.LIF_BAD_STATE, bad
    kv.reset()
    assert kv.state() == {"used_pages": 0, "error": 0, "moved_pages": 0}
    assert kv.table.eq(-1).all() and kv.refs.eq(0).all() and kv.lengths.eq(0).all() and kv.fresh.eq(0).all()


@pytest.mark.parametrize("dtype,kv_heads,head_dim,page", [("f16", 1, 8, 16), ("f32", 3, 72, 32), ("bf16", 8, 128, 16), ("f32", 5, 256, 256)])
def test_every_byte_of_a_page_moves(dtype, kv_heads, head_dim, page):
    """Pages of 256 bytes to 1.25 MiB, whole and not a multiple of what a workgroup copies at once"""
    kv, o, _ = _cache(6, 3, 3, page, layers=3, kv_heads=kv_heads, dtype=dtype, head_dim=head_dim)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    kv.k.normal_(generator=gen)
    kv.v.normal_(generator=gen)
    first = kv.k.clone(), kv.v.clone()
    g = _Gpu(kv)
    for c in (o, g):
        c.reserve([page, page + 3, 2 * page])
        c.truncate([0, -1, -1])
    _compare(kv, o, first, "before")
    kv.compact()
    o.compact()
    assert o.moved == 1
    _compare(kv, o, first, "compact")
    for c in (o, g):
        c.fork([1], [0])
    _compare(kv, o, first, "fork")
    # what nothing was copied to is as it was
    untouched = [p for p in range(6) if o.content[p] == ("initial", p)]
    assert torch.equal(kv.k[:, untouched], first[0][:, untouched]) and torch.equal(kv.v[:, untouched], first[1][:, untouched])


def test_a_step_of_page_calls_in_a_graph():
    """Captured once, replayed with other contents of the argument arrays and eager calls in between."""
    kv, o, first = _cache(64, 4, 16)
    counts, to = ints([0] * 4), ints([-1] * 4)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        kv.reserve(counts)
        kv.truncate(to)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.reserve(counts)
        kv.truncate(to)
        kv.compact()
    rng = random.Random(3)
    for step in range(6):
        c, t = [rng.randint(0, 40) for _ in range(4)], [rng.choice([-1, 0, 17, 33]) for _ in range(4)]
        counts.copy_(ints(c))
        to.copy_(ints(t))
        graph.replay()
        o.reserve(c)
        o.truncate(t)
        o.compact()
        _compare(kv, o, first, step)
        empty = [s for s in range(4) if o.lengths[s] == 0]
        if empty:
            _Gpu(kv).fork([3], empty[:1])
            o.fork([3], empty[:1])
            _compare(kv, o, first, (step, "fork"))
