"""Products of 17 and more rows where the rows go through LDS (not those that share the kernel of few rows): every type, group and workgroup, widths that end
inside a tile, rows and scales that are not numbers.  Which form a product has is asked of the rule, so that no case moves to another kernel unnoticed."""
import numpy as np
import pytest
import torch

from oracle import packed_oracle as O
from tests.packed_forms import few, form_names, forms
from tests.packed_harness import DTYPES, MIDDLE, packed, random_weights, values
from tests.test_packed_linear import FORMS, bound_of, check_product

# fp32 rows: rows, outputs, inputs of each workgroup
F32 = {"outs32_rows16": (17, 2061, 712), "outs64_rows16": (40, 4101, 712), "outs128_rows64": (128, 11021, 264)}
WIDTHS = [8, 24, 40, 120, 136, 168, 1000, 1032, 4544]
WIDE = (20, 4101), (70, 2061)                              # rows, outputs
BAD = (40, 4101, 1288), (150, 2061, 1288)                  # rows, outputs, inputs


def test_cases_reach_their_kernels(tmp_path):
    asked = [(r, k, n, g, True) for r, n, k in F32.values() for g in (32, 64, 128)]
    assert forms(tmp_path, asked) == [name for name in F32 for _ in range(3)]
    assert set(F32) | {"few16"} == set(forms(tmp_path, [(r, k, n, 64, True) for r in (17, 40, 128, 777) for k in (128, 4096) for n in (16, 1024, 4096, 11008, 50000)]))
    asked = [(r, k, n, g, False) for r, n, k in FORMS.values() for g in (64, 128)]
    assert forms(tmp_path, asked) == ["outs%s_rows%s" % tuple(name.split("x")) for name in FORMS for _ in range(2)]
    assert {"outs%s_rows%s" % tuple(name.split("x")) for name in FORMS} | set(F32) | {"few4", "few8", "few16"} == set(form_names())
    asked = [(r, k, n, g, f32) for r, n in WIDE for k in WIDTHS for g in (32, 64, 128) for f32 in (False, True)]
    asked += [(r, k, n, g, f32) for r, n, k in BAD for g in (32, 64, 128) for f32 in (False, True)]
    assert not any(few(name) for name in forms(tmp_path, asked))


@pytest.mark.gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("form", F32)
def test_every_workgroup_of_fp32_rows(form, group, zeros):
    rows, n_out, n_in = F32[form]
    check_product(np.random.default_rng(n_out + group), rows, n_in, n_out, group, zeros, "f32", bias=zeros, extra=8 * zeros)


@pytest.mark.gpu
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("kind,group,zeros", [("bf16", 64, False), ("bf16", 128, False), ("bf16", 64, True), ("f16", 32, True), ("group", 32, False),
                                              ("group", 128, True), ("row", 64, False)])
def test_every_workgroup_of_other_kinds(kind, group, zeros, form):
    rows, n_out, n_in = FORMS[form]
    eight = kind if kind in ("row", "group") else None
    check_product(np.random.default_rng(n_out + n_in), rows, n_in, n_out, group, zeros, "f16" if eight else kind, eight=eight)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "row", "group"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n_in", WIDTHS)
def test_widths_that_end_inside_a_tile(n_in, group, kind):
    """What lies between the rows is not a number, and no answer sees it."""
    rng = np.random.default_rng(n_in + group)
    for (rows, n_out), zeros in zip(WIDE, (False, True)):
        codes, step, zero = random_weights(rng, n_out, n_in, group, zeros)
        eight = kind if kind in ("row", "group") else None
        dtype = "bf16" if eight else kind
        m = packed(codes, step, zero, group, zeros, dtype)
        scales = None
        if eight:
            xs, x_type = rng.integers(-127, 128, (rows, n_in)), torch.int8
            s = rng.uniform(0.01, 1, (rows, step.shape[1] if eight == "group" else 1)).astype(np.float32)
            scales = torch.from_numpy(s).cuda()
        else:
            xs, x_type = rng.standard_normal((rows, n_in)), DTYPES[dtype]
        wide = torch.full((rows, n_in + 24), -128 if eight else float("nan"), dtype=x_type, device="cuda")
        wide[:, :n_in] = torch.from_numpy(xs).to(x_type)
        xs = wide[:, :n_in].double().cpu().numpy()
        if eight:
            xs = xs * np.repeat(s.astype(np.float64), group if eight == "group" else n_in, 1)[:, :n_in]
        out = torch.empty(rows, n_out, dtype=DTYPES[dtype], device="cuda")
        m.multiply(wide[:, :n_in], out, scales=scales)
        y, size = O.product(xs, codes, step, zero, group, middle=MIDDLE["i8" if eight else dtype])
        assert (np.abs(out.cpu().double().numpy() - y) <= bound_of(y, size, n_in, group, dtype, eight is not None)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind,group,zeros", [("f32", 64, True), ("f32", 32, False), ("f16", 64, True), ("f16", 128, False), ("bf16", 64, True), ("bf16", 32, False),
                                              ("bf16", 128, False), ("group", 64, True), ("row", 32, False)])
@pytest.mark.parametrize("rows,n_out,n_in", BAD)
def test_rows_that_hold_nan_or_infinity_stay_by_themselves(rows, n_out, n_in, kind, group, zeros):
    rng = np.random.default_rng(rows + group)
    eight = kind if kind in ("row", "group") else None
    codes, step, zero = random_weights(rng, n_out, n_in, group, zeros)
    m = packed(codes, step, zero, group, zeros, "f16" if eight else kind)
    out = torch.empty(rows, n_out, dtype=DTYPES["f16" if eight else kind], device="cuda")
    clean, bad, scales = torch.empty_like(out), [1, rows - 2], None
    if eight:
        x = torch.from_numpy(rng.integers(-127, 128, (rows, n_in)).astype(np.int8)).cuda()
        scales = torch.from_numpy(rng.uniform(0.001, 0.1, (rows, step.shape[1] if eight == "group" else 1)).astype(np.float32)).cuda()
    else:
        x = values(rng, (rows, n_in), kind)[0].cuda()
    m.multiply(x, clean, scales=scales)
    if eight:
        scales[bad[0], -1], scales[bad[1], 0] = float("nan"), float("inf")
    else:
        x[bad[0], 600], x[bad[1], n_in - 1] = float("nan"), float("inf")
    m.multiply(x, out, scales=scales)
    rest = [i for i in range(rows) if i not in bad]
    assert clean.isfinite().all() and torch.equal(out[rest], clean[rest])
    assert out[bad[0]].isnan().all()
    # (times a weight of 0 infinity is not a number, times any other one it stays infinite)
    assert not out[bad[1]].isfinite().any()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "row", "group"])
@pytest.mark.parametrize("rows,n_out,n_in", BAD)
def test_a_step_that_is_not_a_number_reaches_its_output_only(rows, n_out, n_in, kind):
    rng = np.random.default_rng(rows)
    group, eight = 64, kind if kind in ("row", "group") else None
    codes, step, zero = random_weights(rng, n_out, n_in, group, True)
    step[7, 2], step[n_out - 1, -1] = np.nan, np.nan
    m = packed(codes, step, zero, group, True, "f16" if eight else kind)
    scales = None
    if eight:
        x = torch.from_numpy(rng.integers(-127, 128, (rows, n_in)).astype(np.int8)).cuda()
        scales = torch.full((rows, step.shape[1] if eight == "group" else 1), 0.01, device="cuda")
    else:
        x = values(rng, (rows, n_in), kind)[0].cuda()
    out = torch.empty(rows, n_out, dtype=DTYPES["f16" if eight else kind], device="cuda")
    m.multiply(x, out, scales=scales)
    rest = torch.ones(n_out, dtype=torch.bool)
    rest[[7, n_out - 1]] = False
    assert out[:, 7].isnan().all() and out[:, -1].isnan().all() and out[:, rest.cuda()].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_leading_dimensions_and_equal_results_for_equal_counts(dtype):
    rng = np.random.default_rng(24)
    rows, n_out, n_in = 24, 4101, 512
    m, x, out = check_product(rng, rows, n_in, n_out, 128, False, dtype)
    cube = torch.empty(2, 3, 4, n_out, dtype=DTYPES[dtype], device="cuda")
    m.multiply(x.reshape(2, 3, 4, n_in), cube)
    assert torch.equal(cube.view(rows, n_out), out)
