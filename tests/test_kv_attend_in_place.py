"""Attention whose output takes the place of its queries: the same bits as with an output of its own."""
import pytest
import torch

from tests.kv_harness import DTYPES, build, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,tokens,max_pages", [
    ("f16", 8, 2, 128, 1, 0), ("f32", 6, 1, 80, 4, 0), ("bf16", 71, 1, 64, 1, 0), ("bf16", 8, 2, 128, 16, 1 << 17), ("f16", 24, 3, 64, 7, 1 << 17),
    ("f32", 16, 2, 64, 9, 1 << 17), ("f16", 40, 1, 40, 12, 1 << 17), ("bf16", 32, 2, 64, 60, 1 << 17), ("f16", 142, 2, 64, 20, 0)])
def test_in_place(dtype, heads, kv_heads, head_dim, tokens, max_pages):
    lengths = [tokens, 9001, 0, 300, 2100, 40 + tokens]
    fresh = [tokens, tokens, 0, max(1, tokens // 2), tokens, 1]
    slots = [4, 1, 5, 0, 2, 3]
    kv, _ = build(lengths, fresh, kv_heads=kv_heads, head_dim=head_dim, page=16, dtype=dtype, seed=2, heads=heads, max_tokens=tokens, slots=slots,
                  max_pages=max_pages)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    wide = torch.randn(6, tokens, heads * head_dim + 64, generator=gen, device="cuda").to(DTYPES[dtype])
    cut = lambda t: t[..., :heads * head_dim].unflatten(-1, (heads, head_dim))
    tree = torch.randint(0, 1 << tokens, (6, tokens), generator=gen, device="cuda") if tokens < 60 else None
    for expected in (0, 1, max_pages * 16):
        kv.set_expected_tokens(expected)
        for kw in ({}, {"window": 257, "starts": ints([0, 8000, 0, 7, 0, 1])}, {"tree": tree}):
            kw["slots"] = ints(slots)
            out = torch.empty_like(cut(wide))
            lse, lse2 = torch.empty(6, tokens, heads, device="cuda"), torch.empty(6, tokens, heads, device="cuda")
            kv.attend(1, cut(wide), out, lse=lse, **kw)
            for _ in range(3):
                same = wide.clone()
                kv.attend(1, cut(same), cut(same), lse=lse2, **kw)
                assert torch.equal(cut(same), out) and torch.equal(lse, lse2)
                assert torch.equal(same[..., heads * head_dim:], wide[..., heads * head_dim:])
