"""add_norm: a row's result is the same bit for bit whatever the number of rows, also where its sums depend on their order."""
import numpy as np
import pytest
import torch

import paper_2312_11514_amd as lif
from tests.packed_harness import DTYPES, NORMS

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
