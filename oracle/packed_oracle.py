"""Norms with the residual's addition, weights in 4 bits and their products, in numpy: written from the definitions, shares no code with the HIP path."""
from __future__ import annotations

import numpy as np

F = np.float32


def sum_and_norm(x, residual, norm, eps, weight=None, bias=None):
    """The fixed chain of fp32 operations with sums in fp64: (h, y), float32."""
    h = x.astype(F) if residual is None else residual.astype(F) + x.astype(F)
    if norm == "none":
        return h, h
    wide = h.astype(np.float64)
    if norm == "layer":
        wide = wide - wide.mean(-1, keepdims=True)
    y = wide.astype(F) * (1.0 / np.sqrt((wide * wide).mean(-1, keepdims=True) + np.float64(F(eps)))).astype(F)
    if weight is not None:
        y = y * weight.astype(F)
    if bias is not None and norm == "layer":
        y = y + bias.astype(F)
    return h, y


def norm64(x, residual, norm, eps, weight=None, bias=None):
    """The same in 64 bits throughout."""
    h = x.astype(np.float64) + (0 if residual is None else residual.astype(np.float64))
    if norm == "none":
        return h, h
    d = h - (h.mean(-1, keepdims=True) if norm == "layer" else 0)
    y = d / np.sqrt((d * d).mean(-1, keepdims=True) + np.float64(F(eps)))
    y = y if weight is None else y * weight.astype(np.float64)
    return h, y if bias is None or norm != "layer" else y + bias.astype(np.float64)


def step_of(v):
    """fp32 to 16 significant bits, halves away from zero; below 2^-110: 0; infinite or not a number: not a number."""
    v = np.asarray(v, F)
    fraction, exponent = np.frexp(v.astype(np.float64))
    s = np.trunc(np.abs(fraction) * 2.0 ** 16 + 0.5) * np.sign(fraction) * np.exp2(exponent - 16.0)
    s = np.where(np.abs(s) < 2.0 ** -110, 0.0, s)
    return np.where(np.isfinite(v) & (np.abs(s) < 2.0 ** 128), s, np.nan)


def groups_of(a, group):
    """[rows, groups, group], zeros behind the last element."""
    a = np.asarray(a)
    pad = -a.shape[1] % group
    return np.pad(a, ((0, 0), (0, pad))).reshape(a.shape[0], -1, group)


def rows_in_8_bits(y, group):
    """y float32 [rows, width]: codes int8, scales float64 [rows, groups]."""
    parts = groups_of(y, group or y.shape[1])
    step = step_of(np.abs(parts).max(-1) * (F(1) / F(127)))
    with np.errstate(all="ignore"):
        codes = np.where(step[..., None] > 0, np.rint(parts.astype(np.float64) / step[..., None]), 0)      # halves to even
    return codes.astype(np.int8).reshape(len(y), -1)[:, :y.shape[1]], step


def quantize(w, group, zeros):
    """w float32 [n_out, n_in]: codes 0..15, steps and zero points [n_out, groups]."""
    parts = groups_of(w.astype(F), group)
    if zeros:
        low, high = np.minimum(parts, 0).min(-1), np.maximum(parts, 0).max(-1)
        step = step_of((high - low) * (F(1) / F(15)))
    else:
        step = step_of(np.abs(parts).max(-1) * (F(1) / F(7)))
    ok = step > 0
    with np.errstate(all="ignore"):
        zero = np.where(ok, np.clip(np.rint(-low.astype(np.float64) / step), 0, 15), 8) if zeros else np.full(step.shape, 8.0)
        codes = np.where(ok[..., None], np.rint(parts.astype(np.float64) / step[..., None]), 0) + zero[..., None]
    codes = np.clip(codes, 0, 15)
    return codes.reshape(len(w), -1)[:, :w.shape[1]], step, zero


def weights_of(codes, step, zero, group):
    """What they stand for, float64."""
    n = codes.shape[1]
    return (codes - np.repeat(zero, group, 1)[:, :n]) * np.repeat(step, group, 1)[:, :n]


def product(x, codes, step, zero, group, bias=None, middle=8.0):
    """(y, magnitude) in float64; the magnitude is what roundings of partial sums are relative to where codes are taken relative to `middle` and the
    rest comes off with the sum of x."""
    y = x.astype(np.float64) @ weights_of(codes, step, zero, group).T
    size = np.abs(x.astype(np.float64)) @ np.abs(weights_of(np.abs(codes - middle) + np.repeat(np.abs(zero - middle), group, 1)[:, :codes.shape[1]],
                                                            step, np.zeros_like(zero), group)).T
    return (y, size) if bias is None else (y + bias, size + np.abs(bias))
