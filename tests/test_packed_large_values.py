"""Products of rows as large as their type holds: what is finite comes out finite, whatever the number of rows."""
import numpy as np
import pytest
import torch

from oracle import packed_oracle as O
from tests.packed_forms import few, forms
from tests.packed_harness import DTYPES, MIDDLE, packed, random_weights
from tests.test_packed_linear import bound_of

N_IN, N_OUT = 712, 4101
ROWS = [3, 16, 40, 150]


def test_rows_reach_both_kernels(tmp_path):
    got = {(r, f32): few(name) for f32 in (False, True) for r, name in zip(ROWS, forms(tmp_path, [(r, N_IN, N_OUT, 64, f32) for r in ROWS]))}
    assert got == {(r, f32): r <= 16 for r in ROWS for f32 in (False, True)}


def large_rows(rng, rows, dtype):
    """Rows of the largest values: all of one sign, of a sign for every 8, of any; between rows of small ones."""
    x = rng.uniform(0.5, 1.0, (rows, N_IN)) * 3.3e38
    x[1::4] *= np.repeat(rng.choice([-1.0, 1.0], (len(x[1::4]), N_IN // 8)), 8, 1)
    x[2::4] *= rng.choice([-1.0, 1.0], x[2::4].shape)
    x[3::4] = rng.standard_normal(x[3::4].shape)
    return torch.from_numpy(x.astype(np.float32)).to(DTYPES[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", ROWS)
def test_finite_results_of_large_neighbours(rows, dtype, group, zeros):
    rng = np.random.default_rng(rows + group)
    codes, step, zero = random_weights(rng, N_OUT, N_IN, group, zeros)
    step = step * 2.0 ** -12                               # answers: up to 712 products of 3.3e38 with 15 * 2^-12 * 1.5 / sqrt(712) = 1.5e38
    m = packed(codes, step, zero, group, zeros, dtype)
    x = large_rows(rng, rows, dtype)
    out = torch.empty(rows, N_OUT, dtype=DTYPES[dtype], device="cuda")
    m.multiply(x.cuda(), out)
    y, size = O.product(x.double().numpy(), codes, step, zero, group, middle=MIDDLE[dtype])
    assert np.abs(y).max() < 2e38
    got = out.cpu().double().numpy()
    assert np.isfinite(got).all(), np.unique(np.nonzero(~np.isfinite(got))[0])
    assert (np.abs(got - y) <= bound_of(y, size, N_IN, group, dtype)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", ROWS)
def test_finite_results_of_large_rows_and_zero_points(rows, dtype, group):
    """Zero points up to 255: a group's sum is up to 128 * 255 times the largest value before its step is applied"""
    rng = np.random.default_rng(rows + group)
    codes, step, zero = random_weights(rng, N_OUT, N_IN, group, True)
    zero = rng.integers(200, 256, zero.shape).astype(np.float64)
    step = step * 2.0 ** -17                               # answers: up to 712 products of 3.3e38 with 255 * 2^-17 * 1.5 / sqrt(712) = 2.6e37
    m = packed(codes, step, zero, group, True, dtype)
    x = large_rows(rng, rows, dtype)
    out = torch.empty(rows, N_OUT, dtype=DTYPES[dtype], device="cuda")
    m.multiply(x.cuda(), out)
    y, size = O.product(x.double().numpy(), codes, step, zero, group, middle=MIDDLE[dtype])
    assert np.abs(y).max() < 2e38
    got = out.cpu().double().numpy()
    assert np.isfinite(got).all(), np.unique(np.nonzero(~np.isfinite(got))[0])
    assert (np.abs(got - y) <= bound_of(y, size, N_IN, group, dtype)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", ROWS)
def test_small_rows(rows, dtype, zeros):
    """Rows of the smallest values: of x nothing above 2^-133 is lost, and of an addition within a group or of an output nothing above 2^-133 times the step
    (or once)"""
    rng = np.random.default_rng(rows)
    group = 64
    codes, step, zero = random_weights(rng, N_OUT, N_IN, group, zeros)
    step = step * 2.0 ** 8
    m = packed(codes, step, zero, group, zeros, dtype)
    x = torch.from_numpy((rng.standard_normal((rows, N_IN)) * 2.0 ** -122).astype(np.float32)).to(DTYPES[dtype])
    out = torch.empty(rows, N_OUT, dtype=DTYPES[dtype], device="cuda")
    m.multiply(x.cuda(), out)
    y, size = O.product(x.double().numpy(), codes, step, zero, group, middle=MIDDLE[dtype])
    additions = 3 * group if dtype == "f32" else group     # (three pieces of an fp32 element)
    lost = step.sum(1) * 2 * additions * 2.0 ** -133 + (step.shape[1] + 24) * 2.0 ** -133
    lost = lost + np.abs(O.weights_of(codes, step, zero, group)).sum(1) * 2.0 ** -133 * (dtype == "f32")
    got = out.cpu().double().numpy()
    assert np.abs(y).mean() > 2.0 ** -113 and (np.abs(got - y) <= bound_of(y, size, N_IN, group, dtype) + lost).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["row", "group"])
@pytest.mark.parametrize("group,zeros", [(32, False), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("rows", ROWS)
def test_finite_results_of_large_rows_in_8_bits(rows, group, zeros, kind):
    """Scales up to the largest of an fp32 row, 3.4e38 / 127"""
    rng = np.random.default_rng(rows + group)
    codes, step, zero = random_weights(rng, N_OUT, N_IN, group, zeros)
    if zeros:
        zero = rng.integers(200, 256, zero.shape).astype(np.float64)
    step = step * 2.0 ** -17                               # answers: as of test_finite_results_of_large_rows_and_zero_points
    m = packed(codes, step, zero, group, zeros, "f32")
    x = rng.integers(90, 128, (rows, N_IN)) * rng.choice([-1, 1], (rows, 1))
    x[2::4] *= rng.choice([-1, 1], x[2::4].shape)
    s = (rng.uniform(0.5, 1.0, (rows, step.shape[1] if kind == "group" else 1)) * 2.6e36).astype(np.float32)
    s[3::4] = 1e-3
    xs = x * np.repeat(s.astype(np.float64), group if kind == "group" else N_IN, 1)[:, :N_IN]
    out = torch.empty(rows, N_OUT, device="cuda")
    m.multiply(torch.from_numpy(x.astype(np.int8)).cuda(), out, scales=torch.from_numpy(s).cuda())
    y, size = O.product(xs, codes, step, zero, group, middle=MIDDLE["i8"])
    assert np.abs(y).max() < 2e38
    got = out.cpu().double().numpy()
    assert np.isfinite(got).all(), np.unique(np.nonzero(~np.isfinite(got))[0])
    assert (np.abs(got - y) <= bound_of(y, size, N_IN, group, "f32", True)).all()
