"""Scales of a checkpoint are kept, of any size: to 16 significant bits, and as they are where fp16 or bf16 holds them."""
import numpy as np
import pytest
import torch

import paper_2312_11514_amd as lif
from tests.packed_harness import nibbles

pytestmark = pytest.mark.gpu


def dequantized(codes, scales, group):
    m = lif.PackedLinear(*codes.shape, group=group, dtype="f32")
    m.pack(nibbles(codes).cuda(), torch.from_numpy(scales).cuda())
    out = torch.empty(codes.shape, device="cuda")
    m.dequantize(out)
    return m, out.cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scales_of_16_bit_types(dtype):
    """Every exponent, the largest ones and those below the normal numbers among them, of either sign"""
    bits = np.arange(-2 ** 15, 2 ** 15, 37).astype(np.int16)
    s = torch.from_numpy(bits).view(dtype).float().numpy()
    s = s[np.isfinite(s)][:, None]
    codes = np.random.default_rng(1).integers(0, 16, (len(s), 32))
    with np.errstate(over="ignore"):
        want = (codes - 8).astype(np.float32) * s              # 11 + 4 bits: exact, or infinite
    assert np.array_equal(dequantized(codes, s, 32)[1], want)


def test_scales_of_32_bits_are_rounded_to_16():
    """Half away from zero, to a multiple of 2^-141 at least; what is not finite, or would not be, is not a number"""
    rng = np.random.default_rng(2)
    s = (rng.uniform(-2, 2, 4000) * 2.0 ** rng.integers(-149, 127, 4000)).astype(np.float32)
    s[:6] = [np.inf, -np.inf, np.nan, np.finfo(np.float32).max, 2.0 ** -149, 0.0]
    codes = np.random.default_rng(3).integers(0, 16, (len(s), 32))
    wide = s.astype(np.float64)
    with np.errstate(all="ignore"):
        unit = np.exp2(np.maximum(np.frexp(wide)[1] - 16.0, -141.0))
        rounded = np.sign(wide) * np.floor(np.abs(wide) / unit + 0.5) * unit
        rounded[~(np.abs(wide) < np.inf) | (np.abs(rounded) >= 2.0 ** 128)] = np.nan
        want = ((codes - 8) * rounded[:, None]).astype(np.float32)
    assert np.isnan(want[:4]).all() and np.isfinite(rounded[4:]).all()
    assert np.array_equal(dequantized(codes, s[:, None], 32)[1], want, equal_nan=True)


@pytest.mark.parametrize("rows", [1, 40])
def test_products_with_small_scales(rows):
    """Scales of 2^-120 by rows of 2^100: 64 products, each exact, in whole numbers of 2^-20 below 2^24 times that"""
    n_out, n_in = 4101, 64
    rng = np.random.default_rng(rows)
    codes = rng.integers(0, 16, (n_out, n_in))
    s = np.full((n_out, 1), 2.0 ** -120, np.float32)
    m, _ = dequantized(codes, s, 64)
    x = rng.integers(-100, 101, (rows, n_in)) * 2.0 ** 100
    out = torch.empty(rows, n_out, device="cuda")
    m.multiply(torch.from_numpy(x.astype(np.float32)).cuda(), out)
    assert np.array_equal(out.cpu().double().numpy(), x @ ((codes - 8) * 2.0 ** -120).T)
