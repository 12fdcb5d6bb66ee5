"""Attention over the pages against the oracle in fp64, with bounds that follow from the arithmetic."""
import numpy as np
import pytest
import torch

import paper_2312_11514_amd as lif
from oracle import kv_oracle as O
from tests.kv_harness import DTYPES, UNIT, build, ints

pytestmark = pytest.mark.gpu


def _check(out, lse, ref, dtype, n, d, tag):
    """out: one rounding to E; weights rounded to E (fp32: not); scores are fp32 sums of d products, and a weight is as good as its exponent; the
    sums over n weights and n products are fp32."""
    want, want_lse, size, reach = ref
    u = UNIT[dtype]
    score = (d + 4) * 2.0 ** -24 * reach + 2.0 ** -20
    part = (u if dtype != "f32" else 0.0) + 2 * score + 2 * (n + 8) * 2.0 ** -24
    tiny = {"f16": 2.0 ** -24, "bf16": 2.0 ** -133, "f32": 2.0 ** -149}[dtype]
    bound = u * np.abs(want) + part[..., None] * size + tiny
    err = np.abs(out - want)
    assert (err <= bound).all(), (tag, float((err - bound).max()), np.unravel_index(np.argmax(err - bound), err.shape))
    none = np.isinf(want_lse)
    assert (np.isneginf(lse) == none).all(), tag
    limit = score + 2 * (n + 8) * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(none, 0, want_lse)) + 2.0 ** -20
    assert (np.abs(np.where(none, 0, lse) - np.where(none, 0, want_lse)) <= limit).all(), tag


def _run(lengths, fresh, *, heads, kv_heads, head_dim, page, dtype, tokens, window=0, starts=None, tree=None, seed=1, slots=None, peaked=1.0,
         max_seqs=None, max_pages=0, change=None, stride=0, expected=0):
    kv, rows = build(lengths, fresh, kv_heads=kv_heads, head_dim=head_dim, page=page, dtype=dtype, seed=seed, heads=heads, max_tokens=tokens,
                     slots=slots, max_seqs=max_seqs, max_pages=max_pages)
    kv.set_expected_tokens(expected)
    rng = np.random.default_rng(seed + 1)
    b = len(lengths)
    wide = torch.from_numpy(peaked * rng.standard_normal((b, tokens, heads * head_dim + stride), dtype=np.float32)).to(DTYPES[dtype]).cuda()
    q = wide[..., :heads * head_dim].unflatten(-1, (heads, head_dim))
    back = torch.full((b, tokens, heads * head_dim + 2 * stride), 7.0, dtype=DTYPES[dtype], device="cuda")
    out = back[..., :heads * head_dim].unflatten(-1, (heads, head_dim))
    lse = torch.full((b, tokens, heads), 7.0, device="cuda")
    if change:
        change(kv, rows, q)
    words = None if tree is None else torch.tensor([[w - (1 << 64) if w >> 63 else w for w in ws] for ws in tree], dtype=torch.int64, device="cuda")
    call = lambda o, l: kv.attend(1, q, o, lse=l, window=window, starts=ints(starts) if starts else None, tree=words,
                                  slots=ints(slots) if slots else None)
    call(out, lse)
    assert kv.state()["error"] == 0
    got, got_lse, qn = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    scale = float(np.float32(head_dim ** -0.5))
    for i, (n, f) in enumerate(zip(lengths, fresh)):
        f = min(f, tokens)
        tag = (i, n, f, dtype, heads, kv_heads, head_dim)
        assert (got[i, f:] == 0).all() and np.isneginf(got_lse[i, f:]).all(), tag
        if f == 0:
            continue
        see = O.visible(n, f, starts[i] if starts else 0, window, tree[i] if tree else None)
        ref = O.attend(qn[i, :f], rows[i][0], rows[i][1], see, scale)
        _check(got[i, :f], got_lse[i, :f], ref, dtype, n, head_dim, tag)
    if stride:
        assert back[..., heads * head_dim:].eq(7).all()
    # a second call: the same bits
    again, again_lse = torch.zeros_like(back)[..., :heads * head_dim].unflatten(-1, (heads, head_dim)), torch.zeros_like(lse)
    call(again, again_lse)
    assert torch.equal(out, again) and torch.equal(lse, again_lse)
    return kv, got


SHAPES = [  # dtype, heads, kv_heads, head_dim, page
    ("f16", 4, 4, 128, 16), ("f16", 71, 1, 64, 16), ("bf16", 8, 2, 128, 32), ("f32", 4, 4, 80, 16), ("bf16", 4, 4, 80, 64),
    ("f32", 8, 1, 128, 16), ("f16", 3, 3, 96, 16), ("f16", 4, 2, 256, 32), ("f32", 2, 2, 256, 16), ("bf16", 5, 1, 32, 128),
    ("f32", 6, 2, 64, 256), ("f16", 2, 2, 8, 16), ("bf16", 20, 5, 112, 16), ("f32", 3, 1, 24, 32), ("f16", 40, 1, 40, 16),
    ("bf16", 33, 1, 256, 16), ("f32", 35, 1, 200, 16),
]


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,page", SHAPES)
def test_one_token_at_every_kind_of_length(dtype, heads, kv_heads, head_dim, page):
    lengths = [1, 0, 2, 15, 16, 17, 31, 33, 64, 127, 128, 129, 255, 300]
    _run(lengths, [min(1, n) for n in lengths], heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, dtype=dtype, tokens=1)


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,page", SHAPES)
def test_several_tokens_window_starts_and_trees(dtype, heads, kv_heads, head_dim, page):
    lengths, fresh = [5, 40, 0, 150, 3, 64, 200], [5, 3, 0, 5, 3, 4, 1]
    kw = dict(heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, dtype=dtype, tokens=5, stride=16)
    _run(lengths, fresh, **kw)
    _run(lengths, fresh, window=7, **kw)
    _run(lengths, fresh, window=1, **kw)
    _run(lengths, fresh, starts=[2, 39, 0, 33, 3, 64, 500], **kw)                 # some see nothing, some only themselves
    tree = [[1, 3, 5, 9, 19], [1, 2, 7, 0, 0], [0] * 5, [0, 1, 2, 3, 31], [1, 1, 1, 1, 1], [1 << 63 | 1, 3, 7, 15, 31], [0xffffffffffffffff] * 5]
    _run(lengths, fresh, tree=tree, **kw)
    _run(lengths, fresh, tree=tree, window=60, starts=[0, 5, 0, 149, 1, 0, 190], slots=[6, 2, 8, 0, 3, 1, 5], max_seqs=9, **kw)


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,tokens", [("f16", 4, 4, 64, 64), ("bf16", 8, 2, 128, 33), ("f32", 2, 1, 64, 256),
                                                                  ("f16", 6, 1, 32, 100), ("bf16", 2, 1, 256, 40)])
def test_many_tokens(dtype, heads, kv_heads, head_dim, tokens):
    _run([tokens, 300 + tokens, 7, 450], [tokens, tokens, 7, max(1, tokens // 2)], heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=16, dtype=dtype,
         tokens=tokens)


# How many rows a workgroup takes together goes by the rows and the steps: by the hint where there is one, else by what a full table would make of
# them.  Wide tables with a hint of many tokens, and without.
LARGE = [("f16", 8, 1, 128), ("bf16", 8, 2, 128), ("f32", 8, 1, 128), ("f16", 9, 1, 64), ("f32", 8, 2, 64), ("bf16", 6, 1, 80), ("f32", 9, 1, 80),
         ("f16", 8, 1, 96), ("f32", 8, 1, 96), ("bf16", 8, 1, 32), ("f32", 8, 1, 32), ("f16", 8, 1, 256), ("f32", 8, 1, 256), ("bf16", 8, 1, 112),
         ("f32", 9, 1, 40), ("f16", 8, 1, 200), ("f16", 9, 1, 24)]


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim", LARGE)
@pytest.mark.parametrize("tokens", [4, 6, 11, 16])
@pytest.mark.parametrize("expected", [1 << 21, 0])
def test_rows_together(dtype, heads, kv_heads, head_dim, tokens, expected):
    lengths, fresh = [tokens, 700, 0, 150, 33, 2100], [tokens, tokens, 0, tokens - 1, 2, tokens]
    kw = dict(heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=16, dtype=dtype, tokens=tokens, max_pages=1 << 17,
              expected=expected)
    _run(lengths, fresh, **kw)
    rng = np.random.default_rng(tokens)
    tree = [[int(w) | 1 << j if j else 1 for j, w in enumerate(rng.integers(0, 1 << tokens, tokens))] for _ in lengths]
    _run(lengths, fresh, tree=tree, window=600, starts=[0, 5, 0, 149, 1, 40], **kw)


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,tokens", [("f16", 71, 1, 64, 20), ("f32", 40, 1, 32, 30), ("bf16", 40, 2, 128, 40),
                                                                  ("bf16", 71, 1, 64, 256)])
@pytest.mark.parametrize("max_pages,expected", [(0, 0), (1 << 17, 0), (1 << 17, 1 << 21)])
def test_many_blocks_of_rows(dtype, heads, kv_heads, head_dim, tokens, max_pages, expected):
    _run([tokens + 130, 0, tokens, 1200], [tokens, 0, tokens // 2, tokens], heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=16, dtype=dtype,
         tokens=tokens, max_pages=max_pages, expected=expected)


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,tokens", [("f16", 8, 4, 128, 9), ("bf16", 24, 4, 64, 3), ("f32", 8, 4, 64, 9)])
def test_rows_together_by_the_lengths(dtype, heads, kv_heads, head_dim, tokens):
    """A batch with many steps and no hint; two long sequences among short ones"""
    rng = np.random.default_rng(5)
    lengths = [int(n) for n in rng.integers(0, 40, 700)]
    lengths[100], lengths[601] = 9000, 4001
    _run(lengths, [min(tokens, n) for n in lengths], heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=16, dtype=dtype, tokens=tokens, max_pages=4096)


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,tokens", [("f16", 8, 2, 128, 1), ("bf16", 8, 2, 128, 5), ("f16", 71, 1, 64, 1), ("f32", 6, 1, 80, 12)])
@pytest.mark.parametrize("expected", [1, 100, 3000, 1 << 30])
def test_hints_that_do_not_fit(dtype, heads, kv_heads, head_dim, tokens, expected):
    _run([5000, 40, 0, 700], [tokens, tokens, 0, tokens], heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=32, dtype=dtype, tokens=tokens,
         expected=expected, max_pages=1 << 16)


@pytest.mark.parametrize("batch", [1, 70, 300, 1024])
def test_batches(batch):
    rng = np.random.default_rng(batch)
    lengths = [int(v) for v in rng.integers(0, 90, batch)]
    lengths[batch // 3] = 700
    _run(lengths, [min(1, n) for n in lengths], heads=2, kv_heads=1, head_dim=32, page=16, dtype="f16", tokens=1,
         slots=[int(s) for s in rng.permutation(batch)])


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim", [("f16", 2, 1, 64), ("bf16", 4, 2, 128), ("f32", 1, 1, 80)])
def test_one_long_sequence_beside_short_ones(dtype, heads, kv_heads, head_dim):
    """Parts of an item from many workgroups"""
    _run([9001, 3, 77, 20000], [1, 1, 1, 1], heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=32, dtype=dtype, tokens=1, peaked=2.0)
    _run([12345], [3], heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=16, dtype=dtype, tokens=4, window=9999)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("heads,max_pages,size", [(1, 0, 1.6), (1, 0, 0.8), (70, 1 << 18, 1.6), (70, 1 << 18, 0.8)])
def test_many_small_weights_beside_a_large_one(dtype, heads, max_pages, size):
    """One key towers above 6000 others, which together still count: their weights are below what fp16 holds without a bias."""
    n, d = 6000, 64

    def change(kv, rows, q):
        keys, values = rows[0]
        keys *= 0.05
        keys[0, 17] = q[0, 0, 0].double().cpu().numpy() * size
        keys[:] = torch.from_numpy(keys).to(DTYPES[dtype]).double().numpy()
        values[0, :] = np.abs(values[0])
        from tests.kv_harness import put
        pages = kv.table[0, :-(-n // 16)].tolist()
        put(kv, 1, pages, torch.from_numpy(keys).to(DTYPES[dtype]), torch.from_numpy(values).to(DTYPES[dtype]))

    _run([n], [1], heads=heads, kv_heads=1, head_dim=d, page=16, dtype=dtype, tokens=1, change=change, peaked=1.3, max_pages=max_pages,
         expected=max_pages * 16)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("max_pages", [0, 1 << 18])
def test_what_a_token_does_not_see_never_reaches_it(dtype, bad, max_pages):
    """Keys and values that are not finite at positions before `starts`, behind a window, of later tokens and of other branches of a tree."""
    for heads, kv_heads, d in ((2, 1, 64), (4, 1, 128), (24, 1, 40), (6, 1, 128), (10, 1, 64)):
        tree = [[1, 3, 5, 11, 21]]
        spots = [(0, 36), (0, 38), (0, 39)]                       # the second, fourth and fifth of five new tokens, among others

        def change(kv, rows, q):
            for _, j in spots:
                page = int(kv.table[0, j // 16])
                kv.k[1, page, :, j % 16] = bad
                e = kv.v.shape[5]
                kv.v[1, page, :, j % 16 // e, :, j % 16 % e] = bad
            for j in (0, 1, 2, 12):
                page = int(kv.table[0, j // 16])
                kv.k[1, page, :, j % 16] = bad
                e = kv.v.shape[5]
                kv.v[1, page, :, j % 16 // e, 1:5, j % 16 % e] = bad

        for starts, window in (([13], 0), (None, 24)):
            for t in (None, tree):
                kv, rows = build([40], [5], kv_heads=kv_heads, head_dim=d, page=16, dtype=dtype, seed=4, heads=heads, max_pages=max_pages)
                kv.set_expected_tokens(max_pages * 16)
                change(kv, rows, None)
                q = torch.randn(1, 5, heads, d, device="cuda").to(DTYPES[dtype])
                out, lse = torch.empty_like(q), torch.empty(1, 5, heads, device="cuda")
                words = torch.tensor(t, dtype=torch.int64, device="cuda") if t else None
                kv.attend(1, q, out, lse=lse, window=window, starts=ints(starts) if starts else None, tree=words)
                see = O.visible(40, 5, starts[0] if starts else 0, window, t[0] if t else None)
                got, got_lse = out[0].double().cpu().numpy(), lse[0].double().cpu().numpy()
                touched = {36, 38, 39, 0, 1, 2, 12}
                for u in range(5):
                    if touched & set(np.nonzero(see[u])[0].tolist()):
                        assert not np.isfinite(got[u]).all(), (u, t, starts)
                        continue
                    ref = O.attend(q[0, u:u + 1].double().cpu().numpy(), np.nan_to_num(rows[0][0]), np.nan_to_num(rows[0][1]), see[u:u + 1],
                                   float(np.float32(d ** -0.5)))
                    _check(got[u:u + 1], got_lse[u:u + 1], ref, dtype, 40, d, (u, t, starts))
                    assert np.isfinite(got[u]).all()


def test_a_value_that_is_not_finite_reaches_the_rows_that_see_it():
    """... with its sign, and only its own dimension"""
    for dtype, heads, max_pages in (("f16", 2, 0), ("f32", 2, 0), ("f16", 9, 1 << 18), ("f32", 17, 1 << 18)):
        kv, rows = build([40], [3], kv_heads=1, head_dim=64, page=16, dtype=dtype, seed=4, heads=heads, max_pages=max_pages)
        kv.set_expected_tokens(max_pages * 16)
        page, e = int(kv.table[0, 2]), kv.v.shape[5]
        j = 38                                                     # the second of three new tokens
        kv.v[1, page, 0, j % 16 // e, 11, j % 16 % e] = -float("inf")
        q = torch.randn(1, 3, heads, 64, device="cuda").to(DTYPES[dtype])
        out = torch.empty_like(q)
        kv.attend(1, q, out)
        others = [d for d in range(64) if d != 11]
        assert out[..., others].isfinite().all() and out[0, 0].isfinite().all()
        assert torch.isneginf(out[0, 1:, :, 11]).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_query_that_is_not_a_number_stays_one(dtype):
    kv, _ = build([50, 60], [1, 1], kv_heads=2, head_dim=64, page=16, dtype=dtype, seed=4, heads=4)
    q = torch.randn(2, 1, 4, 64, device="cuda").to(DTYPES[dtype])
    clean, out = torch.empty_like(q), torch.empty_like(q)
    kv.attend(1, q, clean)
    q[0, 0, 2, 5] = float("nan")
    kv.attend(1, q, out)
    assert out[0, 0, 2].isnan().all()
    assert torch.equal(out[1], clean[1]) and torch.equal(out[0, 0, [0, 1, 3]], clean[0, 0, [0, 1, 3]])


def test_pages_beyond_32_bits():
    """A pool of more than 4 GiB of keys, and elements beyond 2^31: the pages at its end"""
    page, kv_heads, d = 256, 4, 128
    pages = 4200000000 // (page * kv_heads * d) // 2 * 2 + 17000
    kv = lif.KVCache(layers=1, heads=4, kv_heads=kv_heads, head_dim=d, page_tokens=page, pages=pages, max_seqs=2, max_pages=4, dtype="f16")
    assert kv.k.numel() > 2 ** 32
    rng = np.random.default_rng(2)
    table = torch.full((2, 4), -1, dtype=torch.int32)
    table[0, :3] = torch.tensor([pages - 1, 0, pages - 3])
    kv.table.copy_(table)
    kv.lengths.copy_(ints([700, 0]))
    kv.fresh.copy_(ints([1, 0]))
    kv.adopt()
    from tests.kv_harness import get, put
    keys, values = (torch.from_numpy(rng.standard_normal((kv_heads, 700, d), dtype=np.float32)).half() for _ in range(2))
    kv.k[0, pages - 1].fill_(float("nan"))
    put(kv, 0, [pages - 1, 0, pages - 3], keys, values)
    new = torch.from_numpy(rng.standard_normal((3, 1, 1, 4, d), dtype=np.float32)).half().cuda()
    q, out = torch.empty_like(new[0]), torch.empty_like(new[0])
    kv.append(0, new[0], new[1], new[2], q, slots=ints([0]))
    assert torch.equal(q, new[0])
    k, v = get(kv, 0, [pages - 1, 0, pages - 3])
    keys[:, 699], values[:, 699] = new[1, 0, 0].cpu(), new[2, 0, 0].cpu()
    assert torch.equal(k[:, :700], keys) and torch.equal(v[:, :700], values)
    kv.attend(0, q, out, slots=ints([0]))
    lse = torch.zeros(1, 1, 4, device="cuda")
    kv.attend(0, q, out, lse=lse, slots=ints([0]))
    ref = O.attend(q[0].double().cpu().numpy(), keys.double().numpy(), values.double().numpy(), np.ones((1, 700), bool), float(np.float32(d ** -0.5)))
    _check(out[0].double().cpu().numpy(), lse[0].double().cpu().numpy(), ref, "f16", 700, d, "far pages")
    kv.fork(ints([0]), ints([1]))                                 # and a copy of the last one
    kv.truncate(ints([-1, -1]))
    kv.compact()
    k2, v2 = get(kv, 0, kv.table[1, :3].tolist())
    assert torch.equal(k2[:, :700], keys) and torch.equal(v2[:, :700], values)


def test_in_a_graph_with_lengths_that_grow():
    """A decode step of two layers captured once: reserve, append, attend; replayed, every result equal to the eager one."""
    from tests.kv_harness import require_gpu
    require_gpu()
    make = lambda: lif.KVCache(layers=2, heads=4, kv_heads=2, head_dim=64, page_tokens=16, pages=64, max_seqs=3, max_pages=16, dtype="bf16")
    a, b = make(), make()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    x = torch.randn(2, 3, 3, 1, 4, 64, generator=gen, device="cuda").bfloat16()
    counts, outs = ints([1, 1, 1]), torch.zeros(2, 2, 3, 1, 4, 64, dtype=torch.bfloat16, device="cuda")

    def step(kv, out):
        kv.reserve(counts)
        for l in range(2):
            q = torch.empty_like(x[l, 0])
            kv.append(l, x[l, 0], x[l, 1, :, :, :2], x[l, 2, :, :, :2], q)
            kv.attend(l, q, out[l])

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(a, outs[0])
    torch.cuda.synchronize()
    a.reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, outs[0])
    for t in range(40):
        x.normal_(generator=gen)
        graph.replay()
        step(b, outs[1])
        assert torch.equal(outs[0], outs[1]), t
        assert a.lengths.tolist() == [t + 1] * 3


def test_on_a_stream_of_its_own():
    kv, rows = build([500, 40], [1, 1], kv_heads=2, head_dim=64, page=16, dtype="f16", seed=4, heads=4)
    q = torch.randn(2, 1, 4, 64, device="cuda").half()
    here, there = torch.empty_like(q), torch.empty_like(q)
    kv.attend(1, q, here)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        kv.attend(1, q, there)
    stream.synchronize()
    assert torch.equal(here, there)


def test_more_new_tokens_than_the_call_has_rows_for():
    """The call's are the first of them"""
    kv, rows = build([30], [6], kv_heads=1, head_dim=32, page=16, dtype="f32", seed=4, heads=2, max_tokens=6)
    q = torch.randn(1, 6, 2, 32, device="cuda")
    all_six, four = torch.empty_like(q), torch.empty(1, 4, 2, 32, device="cuda")
    kv.attend(1, q, all_six)
    kv.attend(1, q[:, :4], four)
    assert torch.allclose(all_six[:, :4], four, atol=1e-5, rtol=0)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("size", [30.0, 3e3, 6e4])
def test_scores_of_any_size(dtype, size):
    """Queries and keys as large as the type holds: scores up to 10^10, whose differences decide.  Per sequence one key wins by far, and the result is
    its value; lengths that go through several waves, workgroups and rescalings."""
    lengths, d, heads = [40, 700, 3000], 64, 4
    kv, rows = build(lengths, [1] * 3, kv_heads=2, head_dim=d, page=16, dtype=dtype, seed=8, heads=heads)
    from tests.kv_harness import put
    rng = np.random.default_rng(9)
    q = torch.from_numpy(np.sign(rng.standard_normal((3, 1, heads, d))) * size).to(DTYPES[dtype]).cuda()
    want = np.zeros((3, 1, heads, d))
    for i, n in enumerate(lengths):
        keys = rng.uniform(-0.5, 0.5, (2, n, d)) * size
        for g in range(2):                                 # the two query heads of a key head have the same direction
            q[i, 0, 2 * g + 1] = q[i, 0, 2 * g]
            at = int(rng.integers(n))
            keys[g, at] = np.sign(q[i, 0, 2 * g].float().cpu().numpy()) * size
            want[i, 0, 2 * g:2 * g + 2] = rows[i][1][g, at]
        put(kv, 1, kv.table[i, :-(-n // 16)].tolist(), torch.from_numpy(keys).to(DTYPES[dtype]), torch.from_numpy(rows[i][1]).to(DTYPES[dtype]))
    out, lse = torch.empty_like(q), torch.empty(3, 1, heads, device="cuda")
    kv.attend(1, q, out, lse=lse)
    # the winner's score is 64 size^2 / 8, the others' are at most half of it in size: 3600 behind for the smallest size, weights of e^-3600
    assert np.abs(out.double().cpu().numpy() - want).max() <= UNIT[dtype] * np.abs(want).max()
    score = float(torch.tensor(size).to(DTYPES[dtype])) ** 2 * d * float(np.float32(d ** -0.5))
    assert np.abs(lse.double().cpu().numpy() - score).max() <= score * (d + 4) * 2.0 ** -24 + 1e-5
