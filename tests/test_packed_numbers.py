"""Numbers that the C structures do not hold are the library's error, and not taken as others or as Python's: no GPU needed."""
import math

import pytest
import torch

import paper_2312_11514_amd as lif
from paper_2312_11514_amd import packed


@pytest.mark.parametrize("change", [dict(n_out=(1 << 32) + 16), dict(n_in=(1 << 32) + 64), dict(group=(1 << 32) + 32), dict(n_out=-(1 << 32) + 16), dict(n_out=16.0),
                                    dict(n_in="64"), dict(group=None)])
def test_sizes_of_a_matrix(change):
    with pytest.raises(lif.LifError, match="configuration"):
        lif.PackedLinear(**dict(dict(n_out=16, n_in=64, group=32), **change))


class Rows:
    """What the bindings ask of a tensor, of any number of rows"""

    def __init__(self, rows, width, dtype):
        self.shape, self.dtype = torch.Size((rows, width)), dtype

    def numel(self):
        return self.shape[0] * self.shape[1]

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0

    def data_ptr(self):
        return 1 << 32


@pytest.fixture
def on_a_gpu(monkeypatch):
    """The bindings with a device to be on, and no library that would launch"""
    if not packed._Torch.ready:
        packed._Torch.bind()
    monkeypatch.setattr(packed._Torch, "device", staticmethod(lambda: 0))
    monkeypatch.setattr(packed._b, "_stream", lambda: None)

    def add_norm(args, stream):                            # (an eps beyond fp32 is infinite there, which the library refuses)
        assert math.isinf(packed._NORM.unpack(args)[-1]), "the library was called"
        return lif.LIF_INVALID_ARG

    def multiply(handle, args, stream):
        raise AssertionError("the library was called")

    monkeypatch.setattr(packed._Torch, "add_norm", staticmethod(add_norm))
    monkeypatch.setattr(packed._Torch, "multiply", staticmethod(multiply))


@pytest.mark.parametrize("rows,more", [(1 << 31, {}), (4, dict(eps=1e300)), (4, dict(eps="small")), (4, dict(norm=1 << 31)), (4, dict(norm="rms")),
                                       (4, dict(group=1 << 40))])
def test_numbers_of_a_norm(on_a_gpu, rows, more):
    x = Rows(rows, 8, torch.float16)
    with pytest.raises(lif.LifError):
        lif.add_norm(x, Rows(rows, 8, torch.float16), **more)


def test_rows_of_a_product(on_a_gpu):
    m = object.__new__(lif.PackedLinear)
    m.n_out, m.n_in, m.group, m.row_groups, m.tdtype, m._gpu, m.handle = 16, 8, 32, 1, torch.float16, 0, None
    with pytest.raises(lif.LifError):
        m.multiply(Rows(1 << 31, 8, torch.float16), Rows(1 << 31, 16, torch.float16))


@pytest.mark.parametrize("codes,scales", [(None, torch.ones(16, 1)), (torch.zeros(16, 4, dtype=torch.uint8), None)])
def test_codes_and_scales_are_no_options(on_a_gpu, monkeypatch, codes, scales):
    m = object.__new__(lif.PackedLinear)
    m.n_out, m.n_in, m.group, m.row_groups, m.tdtype, m._gpu, m.handle = 16, 8, 32, 1, torch.float16, 0, None
    for t in (codes, scales):
        if t is not None:
            monkeypatch.setattr(t, "get_device", lambda: 0, raising=False)
    with pytest.raises(lif.LifError, match="must be given"):
        m.pack(codes, scales)
