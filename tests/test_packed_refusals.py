"""What add_norm and the packed weights refuse: host code, no GPU needed."""
import ctypes as C
import os

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2312_11514_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2312_11514_amd.build import build_library
        build_library()
    binding.load_library()
    return binding


P, M = 1 << 32, 1 << 34                                   # of rows, of the matrix
CONFIG = dict(n_out=100, n_in=264, group=64, zeros=1, dtype=1)
NORM = dict(x=P, residual=P + (1 << 20), total=P + (2 << 20), out=P + (3 << 20), weight=P + (5 << 20), bias=P + (6 << 20), x_stride=264,
            residual_stride=264, total_stride=264, out_stride=264, n_rows=10, width=264, dtype=1, norm=2, group=0, eps=1e-5)
EIGHT = dict(scales=P + (4 << 20), group=64)
ROWS = dict(x=P, bias=P + (1 << 20), out=P + (2 << 20), x_stride=264, out_stride=100, n_rows=10, x_group=0)


def _refused(b, rc, *words):
    message = b.load_library().lif_last_error_string().decode()
    assert rc == b.LIF_INVALID_ARG and all(w in message for w in words), (rc, message)


def _handle(b, **changes):
    cfg = b.LifPackedConfig(**dict(CONFIG, **changes))
    lib, h = b.load_library(), C.c_void_p()
    buf = b.LifPackedBuffers(M, M + (1 << 30), lib.lif_packed_code_bytes(C.byref(cfg)), lib.lif_packed_group_bytes(C.byref(cfg)))
    assert lib.lif_packed_create(C.byref(cfg), C.byref(buf), C.byref(h)) == 0
    return lib, h


@pytest.mark.parametrize("change", [dict(n_out=0), dict(n_out=-1), dict(n_out=(1 << 20) + 1), dict(n_in=0), dict(n_in=4), dict(n_in=100), dict(n_in=65544),
                                    dict(group=0), dict(group=16), dict(group=256), dict(zeros=2), dict(zeros=-1), dict(dtype=3), dict(dtype=-1)])
def test_configurations(b, change):
    cfg, lib, h = b.LifPackedConfig(**dict(CONFIG, **change)), b.load_library(), C.c_void_p()
    assert lib.lif_packed_code_bytes(C.byref(cfg)) == 0 and lib.lif_packed_group_bytes(C.byref(cfg)) == 0
    buf = b.LifPackedBuffers(P, P, 1 << 40, 1 << 40)
    _refused(b, lib.lif_packed_create(C.byref(cfg), C.byref(buf), C.byref(h)), "configuration")


def test_sizes_and_buffers(b):
    lib, h = b.load_library(), C.c_void_p()
    cfg = b.LifPackedConfig(**CONFIG)
    codes, groups = lib.lif_packed_code_bytes(C.byref(cfg)), lib.lif_packed_group_bytes(C.byref(cfg))
    assert (codes, groups) == (112 * 384 // 2, 112 * 6 * 4)
    big = b.LifPackedConfig(n_out=1 << 20, n_in=65536, group=32, zeros=0, dtype=0)
    assert lib.lif_packed_code_bytes(C.byref(big)) == 1 << 35 and lib.lif_packed_group_bytes(C.byref(big)) == 1 << 33
    for buf in (b.LifPackedBuffers(None, P, codes, groups), b.LifPackedBuffers(P, None, codes, groups), b.LifPackedBuffers(P + 8, P, codes, groups),
                b.LifPackedBuffers(P, P + 4, codes, groups), b.LifPackedBuffers(P, P, codes - 1, groups), b.LifPackedBuffers(P, P, codes, groups - 1)):
        _refused(b, lib.lif_packed_create(C.byref(cfg), C.byref(buf), C.byref(h)))
    good = b.LifPackedBuffers(P, P, codes, groups)
    _refused(b, lib.lif_packed_create(None, C.byref(good), C.byref(h)), "null")
    _refused(b, lib.lif_packed_create(C.byref(cfg), None, C.byref(h)), "null")
    _refused(b, lib.lif_packed_create(C.byref(cfg), C.byref(good), None), "null")
    assert lib.lif_packed_code_bytes(None) == 0 and lib.lif_packed_group_bytes(None) == 0 and lib.lif_packed_destroy(None) == 0


@pytest.mark.parametrize("change,word", [
    (dict(x=None), "null"), (dict(out=None), "null"), (dict(residual=None), "residual"), (dict(dtype=3), "dtype"), (dict(norm=3), "norm"), (dict(norm=-1), "norm"),
    (dict(n_rows=0), "n_rows"), (dict(n_rows=-1), "n_rows"), (dict(n_rows=(1 << 19) + 1), "n_rows"), (dict(width=0), "width"), (dict(width=260), "width"),
    (dict(width=65544), "width"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"), (dict(group=32), "scales"),
    (dict(x=P + 2), "aligned"), (dict(residual=P + (1 << 20) + 8), "aligned"), (dict(total=P + (2 << 20) + 8), "aligned"), (dict(out=P + 8), "aligned"),
    (dict(weight=P + 2), "aligned"), (dict(bias=P + 2), "aligned"), (dict(x_stride=256), "stride"), (dict(x_stride=268), "stride"),
    (dict(residual_stride=0), "stride"), (dict(total_stride=-264), "stride"), (dict(out_stride=1 << 41), "stride"),
    # out one row behind x, total half a row into the residual, out over weight, total over out
    (dict(out=P + 528), "overlap"), (dict(total=P + (1 << 20) + 256), "overlap"), (dict(out=P + (5 << 20)), "overlap"), (dict(weight=P + (3 << 20) + 4), "overlap"),
    (dict(total=P + (3 << 20)), "overlap"), (dict(out=P, out_stride=272), "overlap"), (dict(total=P + (3 << 20) + 16), "overlap")])
def test_add_norm(b, change, word):
    args = b.LifNormRows(**dict(NORM, **change))
    _refused(b, b.load_library().lif_add_norm(C.byref(args), None), word)


@pytest.mark.parametrize("change,word", [
    (dict(group=16), "group"), (dict(group=256), "group"), (dict(group=-32), "group"), (dict(out=P + (3 << 20) + 4), "aligned"), (dict(scales=P + 2), "aligned"),
    (dict(out_stride=268), "stride"), (dict(out=P), "overlap"), (dict(scales=P + (3 << 20)), "overlap"), (dict(scales=P + (2 << 20) + 400), "overlap"),
    (dict(scales=P + 4), "overlap")])
def test_add_norm_in_8_bits(b, change, word):
    args = b.LifNormRows(**dict(NORM, **dict(EIGHT, **change)))
    _refused(b, b.load_library().lif_add_norm(C.byref(args), None), word)


@pytest.mark.parametrize("change,word", [
    (dict(x=None), "null"), (dict(out=None), "null"), (dict(n_rows=0), "n_rows"), (dict(n_rows=(1 << 19) + 1), "n_rows"), (dict(x_group=64), "x_group"),
    (dict(x_group=32, x_scales=P + (3 << 20)), "x_group"), (dict(x=P + 8), "aligned"), (dict(x_stride=256), "stride"), (dict(x_stride=268), "stride"),
    (dict(out=P + (2 << 20) + 1), "aligned"), (dict(out_stride=99), "out"), (dict(out_stride=1 << 41), "out"), (dict(bias=P + 2), "aligned"),
    (dict(x_scales=P + 2), "aligned"), (dict(out=P + 16), "overlap"), (dict(out=P), "overlap"), (dict(bias=P + (2 << 20) + 8), "overlap"),
    (dict(x_scales=P + (2 << 20) + 8), "overlap"), (dict(out=M + 100), "overlap"), (dict(out=M + (1 << 30) - 1998), "overlap"),
    (dict(x_stride=(1 << 22) + 8), "2^22")])
def test_multiply(b, change, word):
    lib, h = _handle(b)
    args = b.LifPackedRows(**dict(ROWS, **change))
    _refused(b, lib.lif_packed_multiply(h, C.byref(args), None), word)
    lib.lif_packed_destroy(h)


def test_out_between_the_rows_of_x_is_told_from_out_over_them(b):
    """Parts of one projection's rows: x has columns 0..263 of 512, out the 100 behind them, then 100 that begin inside x, then ones that reach the next row"""
    lib, h = _handle(b)
    for column, overlaps in ((264, False), (412, False), (256, True), (413, True)):
        args = b.LifPackedRows(**dict(ROWS, x_stride=512, out_stride=512, out=P + 2 * column, n_rows=0))
        rc = lib.lif_packed_multiply(h, C.byref(args), None)
        _refused(b, rc, "n_rows")                          # (nothing is launched here)
        args.n_rows = 10
        if overlaps:
            _refused(b, lib.lif_packed_multiply(h, C.byref(args), None), "overlap")
    lib.lif_packed_destroy(h)


def test_making_weights(b):
    lib, h = _handle(b)
    _refused(b, lib.lif_packed_quantize(None, P, 264, None), "null")
    _refused(b, lib.lif_packed_quantize(h, None, 264, None), "null")
    _refused(b, lib.lif_packed_quantize(h, P + 8, 264, None), "aligned")
    _refused(b, lib.lif_packed_quantize(h, P, 256, None), "stride")
    _refused(b, lib.lif_packed_quantize(h, P, 268, None), "stride")
    _refused(b, lib.lif_packed_dequantize(h, P + 4, 264, None), "aligned")
    _refused(b, lib.lif_packed_dequantize(h, P, 100, None), "stride")
    for at in (M, M + 16, M - 16, M + (1 << 30) + 32):
        _refused(b, lib.lif_packed_quantize(h, at, 264, None), "overlap")
        _refused(b, lib.lif_packed_dequantize(h, at, 264, None), "overlap")
        for arrays in ((at, P, P), (P, at, P), (P, P, at)):
            _refused(b, lib.lif_packed_pack(h, *arrays, None), "overlap")
    _refused(b, lib.lif_packed_pack(h, P, P, None, None), "zeros")
    _refused(b, lib.lif_packed_pack(h, None, P, P, None), "null")
    _refused(b, lib.lif_packed_pack(h, P + 2, P, P, None), "aligned")
    lib.lif_packed_destroy(h)
    lib, h = _handle(b, zeros=0)
    _refused(b, lib.lif_packed_pack(h, P, P, P, None), "zeros")
    _refused(b, lib.lif_packed_multiply(None, C.byref(b.LifPackedRows(**ROWS)), None), "null")
    _refused(b, lib.lif_packed_multiply(h, None, None), "null")
    _refused(b, lib.lif_add_norm(None, None), "null")
    lib.lif_packed_destroy(h)


def test_tensors_that_do_not_fit_are_refused_before_the_library_sees_them(b):
    import paper_2312_11514_amd as lif
    half = torch.zeros(3, 64, dtype=torch.float16)
    with pytest.raises(lif.LifError, match="current GPU"):
        lif.add_norm(half, torch.empty_like(half))
    for x in (half.double(), half.to(torch.int8), torch.tensor(1.0, dtype=torch.float16)):
        with pytest.raises(lif.LifError, match="x must be"):
            lif.add_norm(x, x.clone())
    with pytest.raises(lif.LifError, match="dtype"):
        lif.PackedLinear(16, 64, dtype="f64")
    for change in (dict(n_out=0), dict(n_in=20), dict(group=48)):
        with pytest.raises(lif.LifError, match="configuration"):
            lif.PackedLinear(**dict(dict(n_out=16, n_in=64, group=32), **change))


def test_row_strides(b):
    from paper_2312_11514_amd.packed import _stride
    t = torch.zeros(4, 6, 32)
    assert _stride(t, "t") == 32 and _stride(t[:, :, :16], "t") == 32 and _stride(t[0, :, :8], "t") == 32 and _stride(t[1, 2], "t") == 32
    assert _stride(t[:, 1, :], "t") == 192 and _stride(t[:, 2:3, :8], "t") == 192 and _stride(t[:1, 3:4, :8], "t") == 8
    import paper_2312_11514_amd as lif
    for bad in (t[:, :5], t.transpose(0, 1), t[..., ::2], t.transpose(1, 2)):
        with pytest.raises(lif.LifError, match="stride"):
            _stride(bad, "t")
