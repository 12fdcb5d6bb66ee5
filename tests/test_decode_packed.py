"""The example with its resident matrices in 4 bits, and one layer's calls in a row against the definitions: norms with the residual's addition, rows in
8 bits, projections, keys and values into their pages, attention."""
import numpy as np
import pytest
import torch

import paper_2312_11514_amd as lif
from oracle import packed_oracle as O
from tests.packed_harness import packed, random_weights, values

pytestmark = pytest.mark.gpu


def test_sequences_after_forks_truncation_and_compaction_equal_fresh_ones():
    from examples.decode import Decoder, main
    got = main(steps=5, dense=True, packed=True)
    assert got["pages"] < got["pages_before"] and got["moved"] > 0
    for slot, tokens in got["sequences"].items():
        fresh = Decoder(dense=True, packed=True)
        for at in range(0, len(tokens), 11):               # in pieces of another size, in another slot
            logits = fresh.step([tokens[at:at + 11] if s == 5 else [] for s in range(fresh.seqs)])[5][-1]
        scale = logits.abs().max()
        # as without 4 bits: sums in another order and a few roundings of 2^-11; and where that moves a row's element over a half, one of its 512 codes of 8
        # bits by a step, 1 / 127 of the largest element: 1 / (127 sqrt(512)) of a sum of 512
        assert (logits - got["logits"][slot]).abs().max() <= 2e-2 * scale, slot


@pytest.mark.parametrize("rows,dtype", [(1, "f16"), (5, "bf16"), (40, "f16"), (130, "f32")])
def test_half_a_layer_eager_and_replayed(rows, dtype):
    """x += out(attention(qkv(norm(x)))): each call against its definition on what the call before it has left, and replays against eager runs"""
    rng = np.random.default_rng(rows)
    heads, kv_heads, dim, d, group = 8, 2, 64, 520, 64
    width = (heads + 2 * kv_heads) * dim
    wq, wo = random_weights(rng, width, d, group, True), random_weights(rng, d, heads * dim, group, False)
    qkv_of, out_of = packed(*wq, group, True, dtype), packed(*wo, group, False, dtype)
    weight = torch.from_numpy(rng.uniform(0.5, 1.5, d).astype(np.float32)).cuda()
    x0, y0 = values(rng, (rows, d), dtype)[0], values(rng, (rows, d), dtype, 0.3)[0]
    x, y = x0.cuda(), y0.cuda()
    like = lambda *shape, t=x.dtype: torch.empty(rows, *shape, dtype=t, device="cuda")
    codes, scales, qkv, turned, mixed = like(d, t=torch.int8), like(-(-d // group), t=torch.float32), like(width), like(1, heads, dim), like(1, heads, dim)
    codes2, scales2, left = like(heads * dim, t=torch.int8), like(1, t=torch.float32), like(d)
    kv = lif.KVCache(layers=1, heads=heads, kv_heads=kv_heads, head_dim=dim, page_tokens=16, pages=rows, max_seqs=rows, max_pages=1, dtype=dtype)
    kv.reserve(torch.ones(rows, dtype=torch.int32, device="cuda"))
    q, k, v = (t.view(rows, 1, -1, dim) for t in qkv.split((heads * dim, kv_heads * dim, kv_heads * dim), -1))

    def calls():
        lif.add_norm(y, codes, weight=weight, residual=x, total=x, scales=scales, group=group)
        qkv_of.multiply(codes, qkv, scales=scales)
        kv.append(0, q, k, v, turned)
        kv.attend(0, turned, mixed)
        lif.add_norm(mixed.view(rows, -1), codes2, norm=lif.NORM_NONE, scales=scales2)
        out_of.multiply(codes2, left, scales=scales2)

    calls()
    torch.cuda.synchronize()
    h, n = O.sum_and_norm(y0.float().numpy(), x0.float().numpy(), "rms", 1e-5, weight.cpu().numpy())
    assert torch.equal(x.cpu(), torch.from_numpy(h).to(x.dtype))
    want, step = O.rows_in_8_bits(n, group)
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().double().numpy(), step)
    unit = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
    sums = lambda size, groups: (groups + 24) * 2.0 ** -23 * size                          # additions of groups, parts and scales in fp32
    ref, size = O.product(want * np.repeat(step, group, 1)[:, :d], *wq, group)
    assert (np.abs(qkv.cpu().double().numpy() - ref) <= 1.01 * (unit * np.abs(ref) + sums(size, 9)) + 1e-7).all()
    # one token a sequence sees itself alone: attention is its value, exactly
    share = heads // kv_heads
    assert torch.equal(mixed, v.repeat_interleave(share, 2))
    want2, step2 = O.rows_in_8_bits(mixed.float().cpu().numpy().reshape(rows, -1), 0)
    assert np.array_equal(codes2.cpu().numpy(), want2) and np.array_equal(scales2.cpu().double().numpy(), step2)
    ref2, size2 = O.product(want2 * step2, *wo, group)
    assert (np.abs(left.cpu().double().numpy() - ref2) <= 1.01 * (unit * np.abs(ref2) + sums(size2, 8)) + 1e-7).all()

    eager = left.clone()
    graph = torch.cuda.CUDAGraph()
    x.copy_(x0)
    with torch.cuda.graph(graph):
        calls()
    for i in range(3):
        x.copy_(x0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(left, eager) and torch.equal(x.cpu(), torch.from_numpy(h).to(x.dtype)), i
