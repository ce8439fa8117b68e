"""A cache in four bits and products of 8-bit integers, from their definitions.

The numbers of a group are defined by operations in 32 bits (see include/blendstep_bits.h), which numpy's float32 does; codes, and all that
is computed from them, are float64.
"""
from __future__ import annotations

import numpy as np


def _bf16_nearest(a):
    u = np.ascontiguousarray(a, dtype=np.float32).view(np.uint32)
    return ((u + ((u >> 16) & 1) + np.uint32(0x7FFF)) & np.uint32(0xFFFF0000)).view(np.float32)


def _bf16_above(a):
    """The smallest bf16 number that is not below a >= 0."""
    u = np.ascontiguousarray(a, dtype=np.float32).view(np.uint32)
    return ((u + np.uint32(0xFFFF)) & np.uint32(0xFFFF0000)).view(np.float32)


def kv4_numbers(v, group: int):
    """(scale, mid) of v [..., dh] float32: [..., dh / group] each, NaN where a group stands for NaN."""
    v = np.asarray(v, dtype=np.float32)
    v = v.reshape(v.shape[:-1] + (v.shape[-1] // group, group))
    bad = ~np.isfinite(v).all(axis=-1)
    v = np.where(bad[..., None], np.float32(0), v)
    lo, hi = v.min(axis=-1), v.max(axis=-1)
    with np.errstate(over="ignore", invalid="ignore"):
        bad |= ~np.isfinite(hi - lo)
        mid = _bf16_nearest(lo + np.float32(8) * ((hi - lo) / np.float32(15)))
        bad |= ~np.isfinite(mid)
        scale = np.maximum(_bf16_above(np.maximum((mid - lo) / np.float32(8), (hi - mid) / np.float32(7))), np.float32(2.0 ** -126))
    return np.where(bad, np.float32(np.nan), scale), np.where(bad, np.float32(0), mid)


def kv4_codes(v, scale, mid):
    """Codes 0 .. 15 of v [..., dh] (0 in groups that stand for NaN)."""
    v = np.asarray(v, dtype=np.float32)
    x = v.reshape(scale.shape + (v.shape[-1] // max(1, scale.shape[-1]),))
    with np.errstate(invalid="ignore"):
        c = np.rint((x - mid[..., None]).astype(np.float64) / scale[..., None]) + 8
    return np.clip(np.where(np.isnan(c), 0, c), 0, 15).astype(np.int64).reshape(v.shape)


def kv4_values(v, group: int):
    """(what is kept of v [..., dh] in float64, size): size [..., dh] is |mid| + |scale (c - 8)|, which bounds what rounding a factor of it can change."""
    scale, mid = kv4_numbers(v, group)
    part = np.repeat(scale.astype(np.float64), group, axis=-1) * (kv4_codes(v, scale, mid) - 8)
    mid = np.repeat(mid.astype(np.float64), group, axis=-1)
    return mid + part, np.abs(mid) + np.abs(part)


def w8_rows(x):
    """(integers, scale) of rows x [m, k]: scale = the greatest magnitude / 127, at least 2^-100 / 127, integers x / scale, all in float32; NaN for rows with a NaN or an infinity."""
    x = np.asarray(x, dtype=np.float32)
    most = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(len(x), dtype=np.float32)
    bad = ~np.isfinite(x).all(axis=1)
    scale = np.maximum(np.where(bad, np.float32(0), most), np.float32(2.0 ** -100)) / np.float32(127)
    with np.errstate(invalid="ignore"):
        q = np.clip(np.rint(np.where(bad[:, None], np.float32(0), x) / scale[:, None]), -127, 127).astype(np.int64)
    return q, np.where(bad, np.float32(np.nan), scale)


def w8_linear(x, w, scales):
    """x [m, k], w [n, k] integers, scales [n] -> [m, n] in float64."""
    q, s = w8_rows(x)
    return (q @ np.asarray(w, dtype=np.int64).T) * s[:, None].astype(np.float64) * np.asarray(scales, dtype=np.float64)[None, :]
