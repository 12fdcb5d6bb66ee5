"""add_norm against the definitions: the residual's addition, the norm of the sum, rows of the type or in 8 bits."""
import numpy as np
import pytest
import torch

import paper_2312_11514_amd as lif
from oracle import packed_oracle as O
from tests.packed_harness import DTYPES, NORMS, TINY, UNIT, at_stride, values

pytestmark = pytest.mark.gpu

# a lane's piece; pieces of one wave, of several, ragged; the largest row of one piece a thread, and of two, four and eight
WIDTHS = [8, 24, 72, 512, 520, 1288, 2048, 4096, 4544, 8192, 8200, 16384, 20008, 65536]


def inputs(rng, rows, width, dtype, residual):
    x, xs = values(rng, (rows, width), dtype)
    r, rs = values(rng, (rows, width), dtype, 3.0) if residual else (None, None)
    w, b = rng.uniform(0.5, 1.5, width).astype(np.float32), rng.standard_normal(width).astype(np.float32)
    return x, xs, r, rs, w, b


def run(x, r, norm, w, b, *, eps=1e-5, group=None, extra=0, total=True):
    """outputs (and scales) and totals of a call whose rows lie at a stride, and whether anything beside the rows changed"""
    xg, _ = at_stride(x, extra)
    rg = at_stride(r, 2 * extra)[0] if r is not None else None
    tg, t_wide = at_stride(torch.zeros_like(x), 3 * extra, -5.0) if r is not None and total else (None, None)
    out, o_wide = at_stride(torch.zeros(x.shape, dtype=torch.int8 if group is not None else x.dtype), extra, -5.0)
    scales = torch.full((len(x), -(-x.shape[1] // group) if group else 1), -1.0, device="cuda") if group is not None else None
    lif.add_norm(xg, out, norm=NORMS[norm], eps=eps, weight=torch.from_numpy(w).cuda() if w is not None else None,
                 bias=torch.from_numpy(b).cuda() if b is not None else None, residual=rg, total=tg, scales=scales, group=group or 0)
    torch.cuda.synchronize()
    for wide in (t_wide, o_wide):
        if wide is not None and extra:
            assert (wide[:, x.shape[1]:] == -5).all()
    return out.cpu(), scales.cpu() if scales is not None else None, tg.cpu() if tg is not None else None


def check_rows(got, y64, y32, h64, dtype, norm, w, b):
    """y is at most five fp32 roundings (sum, difference, 1 / root, their product, weight; bias) from the formula, relative to what they round, then one."""
    unit = 2.0 ** -24
    scale = np.abs(y32.astype(np.float64)) + 1e-300
    wide = np.abs(h64) * 0
    if norm != "none":
        d = h64 - (h64.mean(-1, keepdims=True) if norm == "layer" else 0)
        inv = 1 / np.sqrt((d * d).mean(-1, keepdims=True) + 1e-5)
        wide = (np.abs(h64) + 4 * np.abs(d)) * inv * (1 if w is None else np.abs(w)) + (0 if b is None else np.abs(b))
        # the sum's rounding moves mean and variance by no more than it moves the elements
        wide = wide + np.abs(h64).mean(-1, keepdims=True) * inv * (1 if w is None else np.abs(w)) + 2 * scale
    bound = UNIT[dtype] * np.abs(y64) + (1 + UNIT[dtype]) * unit * (2 * wide + np.abs(h64) * (norm == "none")) + TINY[dtype]
    assert (np.abs(got.double().numpy() - y64) <= bound).all(), np.max(np.abs(got.double().numpy() - y64) / bound)


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_widths(dtype, width):
    for i, (norm, residual, rows) in enumerate([("rms", True, 3), ("layer", True, 1), ("rms", False, 2), ("none", True, 2), ("layer", False, 1)]):
        rng = np.random.default_rng(100 * width + i)
        x, xs, r, rs, w, b = inputs(rng, rows, width, dtype, residual)
        b = b if norm == "layer" else None
        out, _, total = run(x, r, norm, w, b, extra=8 * (i % 3))
        h64, y64 = O.norm64(xs, rs, norm, 1e-5, w, b)
        h32, y32 = O.sum_and_norm(xs, rs, norm, 1e-5, w, b)
        if residual:
            assert torch.equal(total, torch.from_numpy(h32).to(DTYPES[dtype]))
        check_rows(out, y64, y32, h64, dtype, norm, w if norm != "none" else None, b)


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("width", [8, 40, 136, 512, 1288, 4096, 4544, 8200, 20008])
def test_codes_and_scales_bit_for_bit(width, group):
    for i, (dtype, norm) in enumerate([("f32", "rms"), ("f16", "layer"), ("bf16", "rms"), ("f16", "none")]):
        rng = np.random.default_rng(1000 * width + group + i)
        x, xs, r, rs, w, b = inputs(rng, 3, width, dtype, i != 3)
        b = b if norm == "layer" else None
        out, scales, total = run(x, r, norm, w, b, group=group, extra=8 * (i % 2))
        h, y = O.sum_and_norm(xs, rs, norm, 1e-5, w if norm != "none" else None, b)
        codes, step = O.rows_in_8_bits(y, group)
        assert np.array_equal(scales.double().numpy(), step)
        assert np.array_equal(out.numpy(), codes)
        if total is not None:
            assert torch.equal(total, torch.from_numpy(h).to(DTYPES[dtype]))


def test_halves_go_to_the_even_code():
    """Rows whose quotients are whole numbers and a half, exactly, for steps of many sizes; and their neighbours on both sides"""
    rows = []
    for e in (-100, -20, -3, 0, 5, 90):
        # 127 * 32768 / 2^15 = 127: a step of 2^e times a number of 16 bits
        for m in (32768, 32769, 50001, 65535):
            step = np.float32(m * 2.0 ** (e - 15))
            k = np.arange(-127, 127) + 0.5
            half = (k * np.float64(step)).astype(np.float32)
            assert (half.astype(np.float64) == k * np.float64(step)).all()
            row = np.concatenate([[np.float32(127 * np.float64(step))], half, np.nextafter(half, np.float32(np.inf)), np.nextafter(half, np.float32(-np.inf))])
            rows.append(np.pad(row, (0, -len(row) % 8)))
    x = torch.from_numpy(np.stack(rows).astype(np.float32))
    out, scales, _ = run(x, None, "none", None, None, group=0)
    codes, step = O.rows_in_8_bits(x.numpy(), 0)
    assert np.array_equal(scales.double().numpy(), step) and np.array_equal(out.numpy(), codes)


@pytest.mark.parametrize("group", [0, 32])
def test_zero_tiny_and_infinite_rows(group):
    width = 64
    x = torch.zeros(6, width)
    x[1] = 2.0 ** -111                                     # a step below 2^-110
    x[2, 3] = float("inf")
    x[3, 40] = float("nan")
    x[4] = torch.linspace(-1e38, 3e38, width)
    x[5] = -2.0 ** -100
    out, scales, _ = run(x, None, "none", None, None, group=group)
    codes, step = O.rows_in_8_bits(x.numpy(), group)
    assert np.array_equal(scales.double().numpy(), step, equal_nan=True)
    assert np.array_equal(out.numpy(), codes)
    assert scales[0].eq(0).all() and scales[1].eq(0).all() and scales[2].isnan().any() and scales[3].isnan().any() and scales[5].gt(0).all()


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_constant_and_zero_rows(norm):
    x = torch.zeros(3, 520)
    x[1] = 1234.5
    x[2] = 1e-3
    out, _, _ = run(x, None, norm, None, None)
    h64, y64 = O.norm64(x.numpy(), None, norm, 1e-5)
    assert torch.equal(out[0], torch.zeros(520))
    assert np.abs(out.double().numpy() - y64).max() <= 4 * 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_that_hold_nan_or_infinity_stay_by_themselves(dtype):
    rng = np.random.default_rng(5)
    x, _, r, _, w, b = inputs(rng, 5, 1288, dtype, True)
    clean = run(x, r, "rms", w, None)[0]
    x[1, 77], r[3, 1000] = float("nan"), float("inf")
    out = run(x, r, "rms", w, None)[0]
    assert torch.equal(out[[0, 2, 4]], clean[[0, 2, 4]])
    assert out[1].isnan().all() and out[3, 1000].isnan() and (out[3].float().nan_to_num(0.0) == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("where", ["total is residual", "total is x", "out is x", "out is residual", "both"])
def test_in_place(dtype, where):
    rng = np.random.default_rng(11)
    x, _, r, _, w, b = inputs(rng, 7, 4544, dtype, True)
    want, _, total = run(x, r, "layer", w, b)
    xg, rg = x.cuda(), r.cuda()
    out, tot = torch.empty_like(xg), torch.empty_like(xg)
    if where in ("total is residual", "both"):
        tot = rg
    if where == "total is x":
        tot = xg
    if where in ("out is x", "both"):
        out = xg
    if where == "out is residual":
        out = rg
    lif.add_norm(xg, out, norm=lif.NORM_LAYER, weight=torch.from_numpy(w).cuda(), bias=torch.from_numpy(b).cuda(), residual=rg, total=tot)
    assert torch.equal(out.cpu(), want) and torch.equal(tot.cpu(), total)


def test_parts_of_one_projections_rows():
    """x, residual, total and out as columns of one tensor: equal strides, nothing shared"""
    rng = np.random.default_rng(12)
    x, _, r, _, w, _ = inputs(rng, 9, 264, "f16", True)
    want, _, total = run(x, r, "rms", w, None)
    wide = torch.full((9, 4 * 264 + 8), 3.0, dtype=torch.float16, device="cuda")
    part = lambda i: wide[:, 264 * i:264 * (i + 1)]
    part(0).copy_(x)
    part(2).copy_(r)
    lif.add_norm(part(0), part(1), weight=torch.from_numpy(w).cuda(), residual=part(2), total=part(3))
    assert torch.equal(part(1).cpu(), want) and torch.equal(part(3).cpu(), total)
    assert torch.equal(part(0).cpu(), x) and torch.equal(part(2).cpu(), r) and (wide[:, -8:] == 3).all()


def test_many_rows_equal_few():
    """Rows do not depend on how many there are; leading dimensions are rows"""
    rng = np.random.default_rng(13)
    x, _, r, _, w, _ = inputs(rng, 4500, 2560, "bf16", True)
    out, _, total = run(x, r, "rms", w, None)
    codes, scales, _ = run(x, r, "rms", w, None, group=64)
    for at in (0, 1, 2047, 4499):
        few, _, t = run(x[at:at + 1], r[at:at + 1], "rms", w, None)
        c, s, _ = run(x[at:at + 1], r[at:at + 1], "rms", w, None, group=64)
        assert torch.equal(out[at:at + 1], few) and torch.equal(total[at:at + 1], t)
        assert torch.equal(codes[at:at + 1], c) and torch.equal(scales[at:at + 1], s)
    cube = x[:12].view(3, 4, 2560).cuda()
    got = torch.empty_like(cube)
    lif.add_norm(cube, got, weight=torch.from_numpy(w).cuda(), residual=r[:12].view(3, 4, 2560).cuda())
    assert torch.equal(got.cpu().view(12, -1), out[:12])


def test_graph_and_streams():
    rng = np.random.default_rng(14)
    x, _, r, _, w, _ = inputs(rng, 5, 4096, "f16", True)
    xg, rg, wg = x.cuda(), r.cuda(), torch.from_numpy(w).cuda()
    out, total = torch.empty_like(xg), torch.empty_like(xg)
    call = lambda: lif.add_norm(xg, out, weight=wg, residual=rg, total=total)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        a, b = values(rng, (5, 4096), "f16")[0], values(rng, (5, 4096), "f16", 3.0)[0]
        xg.copy_(a)
        rg.copy_(b)
        graph.replay()
        got, t = out.clone(), total.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(t, total)
