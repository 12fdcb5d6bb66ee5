"""Offsets beyond 32 bits: matrices, rows and outputs of several gigabytes, their last parts against the same in small ones."""
import numpy as np
import pytest
import torch

import paper_2312_11514_amd as lif
from oracle import packed_oracle as O
from tests.packed_harness import packed, random_weights, values
from tests.test_packed_linear import bound_of
from workloads.device import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    require_gpu()
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows", [1, 40])
def test_a_matrix_of_eight_gigabytes(rows):
    rng = np.random.default_rng(31)
    n_in, n_out = 16384, 1 << 20
    codes, step, zero = random_weights(rng, 16, n_in, 128, True)
    small = packed(codes, step, zero, 128, True, "f16")
    big = lif.PackedLinear(n_out, n_in, group=128, zeros=True, dtype="f16")
    assert big.codes.numel() == 1 << 33
    big.codes.zero_()
    big.groups.zero_()
    for tile in (0, 40000, -1):
        big.codes.view(n_out // 16, -1)[tile] = small.codes
        big.groups.view(n_out // 16, -1)[tile] = small.groups
    x = values(rng, (rows, n_in), "f16")[0].cuda()
    out, want = torch.empty(rows, n_out, dtype=torch.float16, device="cuda"), torch.empty(rows, 16, dtype=torch.float16, device="cuda")
    big.multiply(x, out)
    small.multiply(x, want)
    y, size = O.product(x.cpu().double().numpy(), codes, step, zero, 128, middle=-64.0)
    for at in (0, 40000 * 16, n_out - 16):
        got = out[:, at:at + 16]                           # (of more rows another form takes it: sums in another order)
        assert rows > 1 or torch.equal(got, want)
        assert (np.abs(got.cpu().double().numpy() - y) <= bound_of(y, size, n_in, 128, "f16")).all()
    assert (out[:, 16:40000 * 16] == 0).all() and (out[:, 40000 * 16 + 16:-16] == 0).all()


def test_full_weights_of_eight_gigabytes():
    rng = np.random.default_rng(32)
    n_in, n_out = 4096, (1 << 20) - 7
    w = torch.zeros(n_out, n_in, dtype=torch.bfloat16, device="cuda")
    part = values(rng, (16, n_in), "bf16")[0].cuda()
    first = (n_out - 1) // 16 * 16                         # of the last tile
    w[:16] = part
    w[first:] = part[:n_out - first]
    big, small = lif.PackedLinear(n_out, n_in, group=64, zeros=True, dtype="bf16"), lif.PackedLinear(16, n_in, group=64, zeros=True, dtype="bf16")
    big.quantize(w)
    small.quantize(part)
    w.fill_(7.0)
    want = torch.empty_like(part)
    big.dequantize(w)
    small.dequantize(want)
    assert torch.equal(w[:16], want) and torch.equal(w[first:], want[:n_out - first]) and (w[16:first] == 0).all()


def test_rows_of_eight_gigabytes():
    """524288 rows, those of x and of the outputs; strides of the outputs beyond 32 bits with a few"""
    rng = np.random.default_rng(33)
    rows, n_in, n_out = 1 << 19, 8192, 20
    codes, step, zero = random_weights(rng, n_out, n_in, 64, False)
    m = packed(codes, step, zero, 64, False, "f16")
    x = torch.zeros(rows, n_in, dtype=torch.float16, device="cuda")
    some = values(rng, (8, n_in), "f16")[0]
    at = [0, 1, 262144, 300001, rows - 3, rows - 2, rows - 1, 77]
    x[at] = some.cuda()
    out = torch.empty(rows, n_out, dtype=torch.float16, device="cuda")
    m.multiply(x, out)
    y, size = O.product(some.double().numpy(), codes, step, zero, 64, middle=-64.0)
    assert (np.abs(out[at].cpu().double().numpy() - y) <= bound_of(y, size, n_in, 64, "f16")).all()
    rest = torch.ones(rows, dtype=torch.bool)
    rest[at] = False
    assert (out[rest.cuda()] == 0).all()
    del out
    wide = torch.empty(3 * (1 << 31), dtype=torch.float16, device="cuda")
    few = wide.as_strided((3, n_out), (1 << 31, 1))
    want = torch.empty(3, n_out, dtype=torch.float16, device="cuda")
    m.multiply(x[:3], few)
    m.multiply(x[:3], want)
    assert torch.equal(few, want)


def test_norms_of_eight_gigabytes():
    rng = np.random.default_rng(34)
    rows, width = 1 << 18, 16384
    x = torch.zeros(rows, width, dtype=torch.float16, device="cuda")
    some, weight = values(rng, (2, width), "f16")[0].cuda(), torch.from_numpy(rng.uniform(0.5, 1.5, width).astype(np.float32)).cuda()
    x[-2:] = some
    residual, total, out = torch.ones_like(x), torch.empty_like(x), torch.empty(rows, width, dtype=torch.int8, device="cuda")
    scales = torch.empty(rows, width // 32, device="cuda")
    lif.add_norm(x, out, weight=weight, residual=residual, total=total, scales=scales, group=32)
    want, t, s = torch.empty(2, width, dtype=torch.int8, device="cuda"), torch.empty_like(some), torch.empty(2, width // 32, device="cuda")
    lif.add_norm(some, want, weight=weight, residual=residual[:2], total=t, scales=s, group=32)
    assert torch.equal(out[-2:], want) and torch.equal(total[-2:], t) and torch.equal(scales[-2:], s)
    assert torch.equal(out[:-2], out[:1].expand(rows - 2, -1)) and (total[:-2] == 1).all()
