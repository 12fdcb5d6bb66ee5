"""add_norm: a row's result is the same bit for bit whatever the number of rows, also where its sums depend on their order."""
import numpy as np
import pytest
import torch

import paper_2312_11514_amd as lif
from oracle import packed_oracle as O
from tests.packed_harness import DTYPES, NORMS, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("dtype,width", [("f32", 264), ("f32", 1000), ("bf16", 1536), ("f32", 4544), ("f16", 4096), ("f32", 8192), ("f32", 8200), ("f32", 16384)])
def test_rows_of_outliers(dtype, width, norm):
    """Two large elements of opposite sign in a row of small ones: sums whose last bits are those of the large ones, in every order others"""
    rng = np.random.default_rng(width)
    rows = 1500
    x = rng.standard_normal((rows, width)).astype(np.float32)
    at = np.stack([rng.permutation(width)[:2] for _ in range(rows)])
    size = (1e4 if dtype == "f16" else 1e8) * rng.uniform(0.5, 1.5, rows).astype(np.float32)
    x[np.arange(rows), at[:, 0]], x[np.arange(rows), at[:, 1]] = size, -size
    x = torch.from_numpy(x).to(DTYPES[dtype]).cuda()
    call = lambda part, out, **more: lif.add_norm(part, out, norm=NORMS[norm], **more)
    want, got = torch.empty_like(x), torch.empty_like(x)
    call(x, want)
    for first, last in ((0, 1), (1, 1024), (1024, 1500)):
        call(x[first:last], got[first:last])
    assert torch.equal(got, want), (got != want).any(1).sum()
    codes, some = torch.empty(rows, width, dtype=torch.int8, device="cuda"), torch.empty(rows, width, dtype=torch.int8, device="cuda")
    scales, other = torch.empty(rows, 1, device="cuda"), torch.empty(rows, 1, device="cuda")
    call(x, codes, scales=scales)
    for first, last in ((0, 1), (1, 1024), (1024, 1500)):
        call(x[first:last], some[first:last], scales=other[first:last])
    assert torch.equal(some, codes) and torch.equal(other, scales)


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("rows,width", [(1030, 8), (1030, 40), (1030, 136), (1030, 264), (1030, 520), (1030, 1288), (1030, 4544), (1030, 8200), (2, 40008), (3, 65536)])
def test_codes_of_many_rows_and_of_wide_ones_bit_for_bit(rows, width, group):
    """Two pieces of a row to a thread, and eight"""
    for i, (dtype, norm) in enumerate([("f32", "layer"), ("bf16", "rms"), ("f16", "none")]):
        rng = np.random.default_rng(width + group + i)
        (x, xs), (r, rs) = values(rng, (rows, width), dtype), values(rng, (rows, width), dtype, 3.0)
        w, b = rng.uniform(0.5, 1.5, width).astype(np.float32), rng.standard_normal(width).astype(np.float32) if norm == "layer" else None
        out, total = torch.empty(rows, width, dtype=torch.int8, device="cuda"), r.cuda()
        scales = torch.empty(rows, -(-width // group) if group else 1, device="cuda")
        lif.add_norm(x.cuda(), out, norm=NORMS[norm], weight=torch.from_numpy(w).cuda(), bias=torch.from_numpy(b).cuda() if b is not None else None,
                     residual=total, total=total, scales=scales, group=group)
        h, y = O.sum_and_norm(xs, rs, norm, 1e-5, w if norm != "none" else None, b)
        codes, step = O.rows_in_8_bits(y, group)
        assert np.array_equal(scales.cpu().double().numpy(), step) and np.array_equal(out.cpu().numpy(), codes)
        assert torch.equal(total.cpu(), torch.from_numpy(h).to(DTYPES[dtype]))
