"""Draft trees in which the only new token of a sequence does not see itself: what its own key and value hold does not reach its output."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from tests.kv_harness import DTYPES, build
from tests.test_kv_attend import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("heads,head_dim,tokens,max_pages", [(1, 64, 1, 0), (4, 128, 1, 0), (6, 80, 3, 0), (24, 64, 2, 1 << 17), (40, 40, 1, 1 << 17),
                                                             (70, 64, 1, 1 << 17)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_one_new_token_that_does_not_see_itself(dtype, heads, head_dim, tokens, max_pages, bad):
    lengths = [1, 2, 17, 40, 700]
    for word in (0, 2, -2):                                # no bit; a bit of a token that is not there; all bits but its own
        kv, rows = build(lengths, [1] * 5, kv_heads=1, head_dim=head_dim, page=16, dtype=dtype, seed=3, heads=heads, max_tokens=tokens, max_pages=max_pages)
        kv.set_expected_tokens(max_pages * 16)
        e = kv.v.shape[5]
        for i, n in enumerate(lengths):
            page, at = int(kv.table[i, (n - 1) // 16]), (n - 1) % 16
            kv.k[1, page, :, at] = bad
            kv.v[1, page, :, at // e, :, at % e] = bad
        gen = torch.Generator(device="cuda")
        gen.manual_seed(5)
        q = torch.randn(5, tokens, heads, head_dim, generator=gen, device="cuda").to(DTYPES[dtype])
        tree = torch.full((5, tokens), word, dtype=torch.int64, device="cuda")
        out, lse = torch.empty_like(q), torch.empty(5, tokens, heads, device="cuda")
        kv.attend(1, q, out, lse=lse, tree=tree)
        got, got_lse, qn = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
        for i, n in enumerate(lengths):
            see = np.arange(n)[None, :] < n - 1
            ref = O.attend(qn[i, :1], rows[i][0], rows[i][1], see, float(np.float32(head_dim ** -0.5)))
            _check(got[i, :1], got_lse[i, :1], ref, dtype, n, head_dim, (n, word))
            assert (got[i, 1:] == 0).all() and np.isneginf(got_lse[i, 1:]).all()
