"""Test-side glue of the packed weights and the norms: inputs, and codes as checkpoints hold them."""
from __future__ import annotations

import numpy as np
import torch

import paper_2312_11514_amd as lif

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}       # largest relative error of one rounding
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}    # smallest step of the type
NORMS = {"none": lif.NORM_NONE, "rms": lif.NORM_RMS, "layer": lif.NORM_LAYER}
MIDDLE = {"f32": 8.0, "f16": -64.0, "bf16": -128.0, "i8": 8.0}          # the code that counts nothing, at most


def values(rng, shape, dtype, size=1.0):
    """A tensor of the type on the CPU, and what it holds as float32."""
    t = (size * torch.from_numpy(rng.standard_normal(shape, dtype=np.float32))).to(DTYPES[dtype])
    return t, t.float().numpy()


def nibbles(codes):
    """[n, k] of 0..15 to uint8 [n, k / 2], the lower input in the lower half."""
    c = codes.astype(np.uint8)
    return torch.from_numpy(c[:, 0::2] | c[:, 1::2] << 4)


def random_weights(rng, n_out, n_in, group, zeros):
    """Codes 0..15, steps that 16 bits hold, zero points."""
    groups = -(-n_in // group)
    codes = rng.integers(0, 16, (n_out, n_in)).astype(np.float64)
    step = np.float16(rng.uniform(0.5, 1.5, (n_out, groups)) / n_in ** 0.5).astype(np.float64)
    zero = rng.integers(0, 16, (n_out, groups)).astype(np.float64) if zeros else np.full((n_out, groups), 8.0)
    return codes, step, zero


def packed(codes, step, zero, group, zeros, dtype):
    m = lif.PackedLinear(codes.shape[0], codes.shape[1], group=group, zeros=zeros, dtype=dtype)
    m.codes.fill_(0xa5)
    m.groups.fill_(-1)
    m.pack(nibbles(codes).cuda(), torch.from_numpy(step.astype(np.float32)).cuda(),
           torch.from_numpy(zero.astype(np.uint8)).cuda() if zeros else None)
    return m


def at_stride(t, extra, fill=7.0):
    """The same rows on the GPU at a larger stride; everything else holds `fill`."""
    wide = torch.full((t.shape[0], t.shape[1] + extra), fill, dtype=t.dtype, device="cuda")
    wide[:, :t.shape[1]] = t.cuda()
    return wide[:, :t.shape[1]], wide
