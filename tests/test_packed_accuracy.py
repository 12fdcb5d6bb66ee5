"""How far the sums of products are off before they are rounded to the type, seen through a bias that takes the answer off: the root of their mean square,
where a bound for each of them allows for every rounding at its worst."""
import numpy as np
import pytest
import torch

from oracle import packed_oracle as O
from tests.packed_harness import DTYPES, packed, random_weights

pytestmark = pytest.mark.gpu


def error_of_sums(rng, rows, n_in, n_out, group, zeros, dtype, offset):
    """Root mean square of (sum - answer) over that of the answers.  All rows are the same one, so that one bias fits them all: inputs of different sizes,
    `offset` of them common to all; weights as many above zero as below."""
    codes, step, zero = random_weights(rng, n_out, n_in, group, zeros)
    if zeros:
        zero = rng.integers(6, 10, zero.shape).astype(np.float64)
    middle = np.repeat(zero, group, 1)[:, :n_in]
    codes = middle + rng.integers(-6, 7, codes.shape)
    m = packed(codes, step, zero, group, zeros, dtype)
    x = torch.from_numpy(((rng.standard_normal((1, n_in)) + offset) * np.exp(0.7 * rng.standard_normal(n_in))).astype(np.float32)).to(DTYPES[dtype])
    y = O.product(x.double().numpy(), codes, step, zero, group)[0][0]
    bias = (-y).astype(np.float32)
    out = torch.empty(rows, n_out, dtype=DTYPES[dtype], device="cuda")
    m.multiply(x.cuda().repeat(rows, 1), out, bias=torch.from_numpy(bias).cuda())
    # the sum and the bias are within a factor of two of each other: their difference is exact, and is rounded relative to itself
    error = out.cpu().double().numpy() - (y + bias.astype(np.float64))
    return np.sqrt(np.mean(error ** 2) / np.mean(y ** 2))


@pytest.mark.parametrize("offset", [0.0, 0.2])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,n_out", [(1, 2048), (5, 512), (16, 512), (60, 4096), (130, 4096)])
def test_sums_are_no_further_off_than_one_addition_after_the_other(rows, n_out, dtype, group, zeros, offset):
    """n products of independent signs, added one after the other in fp32: the sum of k of them is about sqrt(k) of one, each addition is off by half a unit
    (2^-24 of the sum) at most and evenly spread, 2^-24 / sqrt(3): together 2^-24 sqrt(n^2 / 2 / 3) of one product, 2^-24 sqrt(n / 6) of the sum of n."""
    n_in = 11008
    far = error_of_sums(np.random.default_rng(rows + group), rows, n_in, n_out, group, zeros, dtype, offset)
    assert far <= 2.0 ** -24 * (n_in / 6) ** 0.5, far
