"""Plain references of the paged cache in 4 bits and of the per-head norms: loops
and numpy, from the documented formulas."""
from __future__ import annotations

import numpy as np

GROUP, MAX_SCALE = 32, 9216.0


def scale_value(byte):
    """What scale bytes stand for, in 64 bits: bits 7 to 14 of an fp16 number."""
    return (np.asarray(byte, np.uint16) << 7).view(np.float16).astype(np.float64)


def scale_byte(top):
    """The scale byte of a group with the largest magnitude `top` (a 32-bit float): the first whose value is
    at least fl(top / 7), by looking through all of them."""
    if not np.isfinite(top):
        return 255
    t = float(np.float32(top) / np.float32(7))
    for byte in range(226):
        if scale_value(byte) >= t:
            return byte
    return 225


def quantize(x):
    """(codes [..., d / 2], scales [..., d / 32]) of 32-bit rows."""
    x = np.asarray(x, np.float32)
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    with np.errstate(invalid="ignore"):
        top = np.abs(g).max(-1)
    seen = {t: scale_byte(np.float32(t)) for t in np.unique(top[~np.isnan(top)])}
    byte = np.array([255 if np.isnan(t) else seen[t] for t in top.reshape(-1)], np.uint8).reshape(top.shape)
    s = scale_value(byte).astype(np.float32)[..., None]
    with np.errstate(all="ignore"):
        y = np.where(s == 0, np.float32(0), g / s)
    c = np.where(np.isnan(s), 15.0, np.clip(np.rint(y), -7, 7) + 8).astype(np.uint8)
    c = c.reshape(x.shape)
    return c[..., 0::2] | (c[..., 1::2] << 4), byte


def values(codes, scales):
    """Rows [..., d] in 64 bits."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1).astype(np.float64) - 8
    s = scale_value(scales)
    return (c.reshape(*c.shape[:-1], -1, GROUP) * s[..., None]).reshape(c.shape)


def parts(pool, P, d):
    """Views of the codes [...][P][d / 2] and the scales [...][P][d / 32] of a pool (numpy or torch)."""
    cut = P * d // 2
    lead = tuple(pool.shape[:-1])
    if isinstance(pool, np.ndarray):
        return pool[..., :cut].reshape(*lead, P, d // 2), pool[..., cut:].reshape(*lead, P, d // GROUP)
    return pool[..., :cut].unflatten(-1, (P, d // 2)), pool[..., cut:].unflatten(-1, (P, d // GROUP))


def head_norm(x, w, eps, offset=0.0):
    """x [rows][heads][d] and w as 32-bit floats (the 16-bit operands widened): the documented 32-bit steps."""
    with np.errstate(all="ignore"):
        x = x.astype(np.float32)
        r = (1.0 / np.sqrt((x.astype(np.float64) ** 2).mean(-1, keepdims=True) + np.float64(np.float32(eps)))).astype(np.float32)
        return (x * r) * (np.float32(offset) + w.astype(np.float32))


def turn(x, pos, sections, theta):
    """x [rows][heads][d] (32 bits), pos [axes][rows]: the rotation in the documented 32-bit steps."""
    with np.errstate(all="ignore"):
        d = x.shape[2]
        axis = np.repeat(np.arange(len(sections)), sections)
        a = pos.astype(np.float64)[axis].T * theta ** (-2.0 * np.arange(d // 2) / d)
        c, s = (f(a).astype(np.float32)[:, None] for f in (np.cos, np.sin))
        lo, hi = x[..., :d // 2].astype(np.float32), x[..., d // 2:].astype(np.float32)
        return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)
