"""PackedLinear against its definition: packing, what the weights stand for, and products of rows of every type."""
import numpy as np
import pytest
import torch

import paper_2312_11514_amd as lif
from oracle import packed_oracle as O
from tests.packed_harness import DTYPES, MIDDLE, TINY, UNIT, at_stride, packed, random_weights, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n_out,n_in", [(1, 8), (16, 128), (17, 136), (33, 1288), (100, 40), (5, 4544)])
@pytest.mark.parametrize("zeros", [False, True])
def test_pack_keeps_codes_scales_and_zeros(n_out, n_in, group, zeros):
    rng = np.random.default_rng(n_out + n_in + group)
    codes, step, zero = random_weights(rng, n_out, n_in, group, zeros)
    if zeros:
        zero[0, 0], zero[-1, -1] = 255, 0
    for dtype in ("f32", "bf16"):
        m = packed(codes, step, zero, group, zeros, dtype)
        out, wide = at_stride(torch.zeros(n_out, n_in, dtype=DTYPES[dtype]), 16, -5.0)
        m.dequantize(out)
        want = torch.from_numpy(O.weights_of(codes, step, zero, group).astype(np.float32)).to(DTYPES[dtype])     # 11 + 8 bits: exact in fp32
        assert torch.equal(out.cpu(), want) and (wide[:, n_in:] == -5).all()


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n_out,n_in,group", [(1, 8, 32), (40, 128, 128), (17, 136, 64), (50, 1288, 32), (33, 4544, 128), (300, 512, 64)])
def test_quantize_bit_for_bit(n_out, n_in, group, dtype, zeros):
    rng = np.random.default_rng(n_out * n_in + group)
    w, ws = values(rng, (n_out, n_in), dtype)
    w += torch.linspace(-1, 1, n_out).to(w.dtype)[:, None]
    if n_out > 2:
        w[1], w[2, :8] = 0.0, 0.0
    ws = w.float().numpy()
    m = lif.PackedLinear(n_out, n_in, group=group, zeros=zeros, dtype=dtype)
    source, _ = at_stride(w, 16)
    m.quantize(source)
    out = torch.empty(n_out, n_in, dtype=DTYPES[dtype], device="cuda")
    m.dequantize(out)
    codes, step, zero = O.quantize(ws, group, zeros)
    want = torch.from_numpy(O.weights_of(codes, step, zero, group).astype(np.float32)).to(DTYPES[dtype])      # 16 + 4 bits: exact in fp32
    assert torch.equal(out.cpu(), want)
    # and no weight is further from what it stands for than half a step (a whole one where the zero point was rounded or the scale was rounded down)
    slack = (0.5 if not zeros else 1.0) * 1.001
    assert (np.abs(O.weights_of(codes, step, zero, group) - ws) <= slack * np.repeat(step, group, 1)[:, :n_in] + 1e-30).all()


@pytest.mark.parametrize("zeros", [False, True])
def test_quantize_ties_and_extremes(zeros):
    """Weights half way between two codes; groups that are zero, tiny, too large, or hold infinity or NaN"""
    group, rows = 32, []
    for e in (-100, -30, 0, 60):
        for m in (32768, 40001, 65535):
            step = m * 2.0 ** (e - 15)
            k = np.concatenate([[-7, 7, 0, 0], np.arange(-7, 7) + 0.5, np.arange(-7, 7) + 0.5])
            v = (k * step).astype(np.float32)
            v[18:] = np.nextafter(v[18:], np.float32(np.inf))
            rows.append(v)
    special = np.zeros((7, 32), np.float32)
    special[1] = 1e-37
    special[2, 5] = np.inf
    special[3, 9] = np.nan
    special[4] = np.linspace(-3e38, 3e38, 32)              # their difference is infinite
    special[5] = 5.0
    special[6] = -5.0
    w = np.concatenate([np.stack(rows), special])
    m = lif.PackedLinear(len(w), 32, group=group, zeros=zeros, dtype="f32")
    m.quantize(torch.from_numpy(w).cuda())
    out = torch.empty(len(w), 32, device="cuda")
    m.dequantize(out)
    with np.errstate(all="ignore"):
        codes, step, zero = O.quantize(w, group, zeros)
        want = O.weights_of(codes, step, zero, group).astype(np.float32)
    assert np.array_equal(out.cpu().numpy(), want, equal_nan=True)
    assert np.isnan(want[len(rows) + 2]).all() and np.isnan(want[len(rows) + 3]).all() and (want[len(rows) + 1] == 0).all()


def bound_of(y, size, n_in, group, dtype, whole=False):
    """An addition of the matrix cores or of the vector units is off by a unit of fp32 at most (2^-23 of what it leaves): those of a group (none, of whole
    numbers), of the groups, of the waves' parts and the bias, one for each product with a scale; then one rounding to the type."""
    additions = (0 if whole else 3 * group if dtype == "f32" else group) + -(-n_in // group) + 24
    return UNIT[dtype] * np.abs(y) + (1 + UNIT[dtype]) * additions * 2.0 ** -23 * size + TINY[dtype]


def check_product(rng, rows, n_in, n_out, group, zeros, dtype, bias=False, eight=None, extra=0, x_size=1.0):
    codes, step, zero = random_weights(rng, n_out, n_in, group, zeros)
    m = packed(codes, step, zero, group, zeros, dtype)
    b = rng.standard_normal(n_out).astype(np.float32) if bias else None
    scales = None
    if eight is None:
        x, xs = values(rng, (rows, n_in), dtype, x_size)
        xs = xs.astype(np.float64)
    else:
        groups = -(-n_in // group) if eight == "group" else 1
        x = torch.from_numpy(rng.integers(-127, 128, (rows, n_in)).astype(np.int8))
        s = rng.uniform(0.01, 1, (rows, groups)).astype(np.float32)
        xs = x.numpy().astype(np.float64) * np.repeat(s, group if eight == "group" else n_in, 1)[:, :n_in]
        scales = torch.from_numpy(s).cuda()
    xg, _ = at_stride(x, extra)
    out, wide = at_stride(torch.zeros(rows, n_out, dtype=DTYPES[dtype]), 1 + extra, -5.0)
    m.multiply(xg, out, bias=torch.from_numpy(b).cuda() if bias else None, scales=scales)
    torch.cuda.synchronize()
    y, size = O.product(xs, codes, step, zero, group, b, MIDDLE["i8" if eight else dtype])
    far = np.abs(out.cpu().double().numpy() - y) / bound_of(y, size, n_in, group, dtype, eight is not None)
    assert np.isfinite(far).all() and far.max() <= 1, (far.max(), np.unravel_index(far.argmax(), far.shape))
    assert (wide[:, n_out:] == -5).all()
    return m, xg, out


ROWS = [1, 2, 5, 15, 16, 17, 33, 64, 65, 130, 300]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", ROWS)
def test_products_by_rows(rows, dtype):
    for i, (n_in, n_out, group, zeros) in enumerate([(512, 64, 128, False), (1288, 37, 32, True), (136, 300, 64, True), (2560, 129, 64, False)]):
        check_product(np.random.default_rng(1000 * rows + i), rows, n_in, n_out, group, zeros, dtype, bias=i % 2 == 0, extra=8 * (i % 3))


@pytest.mark.parametrize("eight", ["row", "group"])
@pytest.mark.parametrize("rows", ROWS)
def test_products_of_rows_in_8_bits(rows, eight):
    for i, (n_in, n_out, group, zeros, dtype) in enumerate([(512, 64, 128, False, "f16"), (1288, 37, 32, True, "bf16"), (136, 300, 64, True, "f32"),
                                                            (2560, 129, 32, False, "f32"), (40, 20, 64, True, "f16")]):
        check_product(np.random.default_rng(1000 * rows + i), rows, n_in, n_out, group, zeros, dtype, bias=i % 2 == 1, eight=eight, extra=8 * (i % 3))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16", "i8"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n_in", [8, 24, 32, 40, 120, 128, 136, 1000, 1032, 4544])
def test_products_by_width(n_in, group, dtype):
    for rows in (1, 20, 70):
        check_product(np.random.default_rng(n_in + rows), rows, n_in, 45, group, rows == 20, "f16" if dtype == "i8" else dtype,
                      eight="group" if dtype == "i8" else None)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n_out", [1, 15, 16, 17, 31, 63, 64, 65, 127, 129, 1000])
def test_products_by_outputs(n_out, dtype):
    for rows in (1, 40, 200):
        check_product(np.random.default_rng(n_out + rows), rows, 264, n_out, 128, rows == 40, dtype, bias=True)


@pytest.mark.parametrize("dtype,rows,n_in,n_out", [("f16", 1, 16384, 4096), ("bf16", 8, 65536, 48), ("f32", 3, 11008, 1024), ("f16", 257, 4096, 2050),
                                                   ("bf16", 48, 4544, 4672), ("f16", 1, 1024, 50001)])
def test_large_products(dtype, rows, n_in, n_out):
    check_product(np.random.default_rng(rows), rows, n_in, n_out, 128, True, dtype)


# rows, outputs and inputs that the rule gives to each of its workgroups, by outputs and rows of them (groups of 32 have no 64 by 64 and no 80 by 64)
FORMS = {"32x16": (17, 2061, 712), "32x16_16": (17, 2061, 5128), "32x32": (17, 4109, 712), "32x32_16": (17, 4109, 5128), "48x32": (17, 11565, 712),
         "48x48": (33, 8205, 712), "64x32": (17, 12301, 136), "64x32_16": (33, 6157, 1528), "64x48": (33, 8205, 136), "64x64": (49, 8205, 136),
         "64x64_16": (97, 6157, 1528), "80x64": (33, 16397, 712), "96x32": (17, 16397, 712), "96x64": (97, 10253, 712), "112x48": (65, 12557, 712),
         "128x64": (97, 12301, 136)}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("kind,group,zeros", [("f16", 64, True), ("bf16", 32, False), ("f16", 128, False), ("row", 32, True), ("group", 64, True)])
def test_every_workgroup(kind, group, zeros, form):
    rows, n_out, n_in = FORMS[form]
    check_product(np.random.default_rng(n_out + n_in), rows, n_in, n_out, group, zeros, "bf16" if kind in ("row", "group") else kind, bias=True,
                  eight=kind if kind in ("row", "group") else None)


def test_largest_magnitudes():
    """fp32 rows up to the largest value, cut in pieces without an infinity; small ones beside them"""
    rng = np.random.default_rng(3)
    codes, step, zero = random_weights(rng, 20, 256, 64, False)
    m = packed(codes, step, zero, 64, False, "f32")
    x = torch.zeros(3, 256)
    x[0, 17], x[1, 200], x[2] = 3.4e38, -3.4028234e38, 1e-30
    out = torch.empty(3, 20, device="cuda")
    m.multiply(x.cuda(), out)
    y, size = O.product(x.double().numpy(), codes, step, zero, 64)
    fine = np.abs(y) < 3e38
    assert fine.any() and (np.abs(out.cpu().double().numpy() - y)[fine] <= bound_of(y, size, 256, 64, "f32")[fine]).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [5, 40, 150])
def test_rows_that_hold_nan_or_infinity_stay_by_themselves(dtype, rows):
    rng = np.random.default_rng(21)
    m, x, clean = check_product(rng, rows, 1288, 70, 64, True, dtype)
    clean = clean.clone()
    bad = [1, rows - 2]
    x[bad[0], 600], x[bad[1], 5] = float("nan"), float("inf")
    out = torch.empty(rows, 70, dtype=x.dtype, device="cuda")
    m.multiply(x, out)
    rest = [i for i in range(rows) if i not in bad]
    assert torch.equal(out[rest], clean[rest]) and out[bad[0]].isnan().all() and not out[bad[1]].isfinite().any()


def test_a_step_that_is_not_a_number_reaches_its_output_only():
    rng = np.random.default_rng(22)
    codes, step, zero = random_weights(rng, 40, 256, 64, False)
    step[7, 2] = np.nan
    for rows in (1, 30, 100):
        m = packed(codes, step, zero, 64, False, "f16")
        x, _ = values(rng, (rows, 256), "f16")
        out = torch.empty(rows, 40, dtype=torch.float16, device="cuda")
        m.multiply(x.cuda(), out)
        assert out[:, 7].isnan().all() and out[:, :7].isfinite().all() and out[:, 8:].isfinite().all()


@pytest.mark.parametrize("rows", [1, 20, 130])
def test_graph_replays_and_two_streams(rows):
    """A captured call replayed on new rows equals the eager one; two streams use one matrix at once"""
    rng = np.random.default_rng(23)
    codes, step, zero = random_weights(rng, 517, 1032, 128, True)
    m = packed(codes, step, zero, 128, True, "f16")
    x, out = torch.zeros(rows, 1032, dtype=torch.float16, device="cuda"), torch.empty(rows, 517, dtype=torch.float16, device="cuda")
    m.multiply(x, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.multiply(x, out)
    for _ in range(4):
        x.copy_(values(rng, (rows, 1032), "f16")[0])
        graph.replay()
        got = out.clone()
        m.multiply(x, out)
        torch.cuda.synchronize()
        assert torch.equal(got, out)
    xs = [values(rng, (rows, 1032), "f16")[0].cuda() for _ in range(2)]
    want = []
    for v in xs:
        m.multiply(v, out)
        want.append(out.clone())
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(out) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, v, o in zip(streams, xs, outs):
            with torch.cuda.stream(s):
                m.multiply(v, o)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_leading_dimensions_and_equal_results_for_equal_counts():
    rng = np.random.default_rng(24)
    m, x, out = check_product(rng, 24, 512, 130, 128, False, "bf16")
    cube = torch.empty(2, 3, 4, 130, dtype=torch.bfloat16, device="cuda")
    m.multiply(x.reshape(2, 3, 4, 512), cube)
    assert torch.equal(cube.view(24, 130), out)
