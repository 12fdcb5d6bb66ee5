"""Values as large as bf16 and fp32 hold: the mean of values is a value of that size, however many there are."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from tests.kv_harness import DTYPES, build, put
from tests.test_kv_attend import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e-30, 1e30, 1e36, 3e38])
@pytest.mark.parametrize("heads,kv_heads,tokens,max_pages", [(2, 2, 1, 0), (8, 1, 3, 0), (24, 1, 1, 1 << 17), (70, 1, 1, 1 << 17), (16, 1, 8, 1 << 17)])
def test_values_of_any_size(dtype, size, heads, kv_heads, tokens, max_pages):
    """Weights that are nearly equal, and ones of which some tower above the others; sequences of one position, of one workgroup, of many."""
    lengths, d = [1, 40, 20011], 64
    for peaked in (1e-3, 2.0):
        fresh = [min(tokens, n) for n in lengths]
        kv, rows = build(lengths, fresh, kv_heads=kv_heads, head_dim=d, page=16, dtype=dtype, seed=6, heads=heads, max_tokens=tokens, max_pages=max_pages)
        kv.set_expected_tokens(max_pages * 16)
        rng = np.random.default_rng(7)
        q = torch.from_numpy(peaked * rng.standard_normal((3, tokens, heads, d), dtype=np.float32)).to(DTYPES[dtype]).cuda()
        large = []
        for i, n in enumerate(lengths):
            values = torch.from_numpy(size * rng.uniform(0.5, 1.0, (kv_heads, n, d))).to(DTYPES[dtype])
            values[:, :, 1::2] *= -1
            put(kv, 1, kv.table[i, :-(-n // 16)].tolist(), torch.from_numpy(rows[i][0]).to(DTYPES[dtype]), values)
            large.append(values.double().numpy())
        out, lse = torch.empty_like(q), torch.empty(3, tokens, heads, device="cuda")
        kv.attend(1, q, out, lse=lse)
        got, got_lse, qn = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
        assert np.isfinite(got).all(), (size, peaked)
        for i, (n, f) in enumerate(zip(lengths, fresh)):
            ref = O.attend(qn[i, :f], rows[i][0], large[i], O.visible(n, f), float(np.float32(d ** -0.5)))
            # (in units of `size`: the bound's smallest term is a subnormal of the type)
            _check(got[i, :f] / size, got_lse[i, :f], (ref[0] / size, ref[1], ref[2] / size, ref[3]), dtype, n, d, (n, size, peaked))
