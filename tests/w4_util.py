"""The 4-bit matrices in plain numpy: order of the codes, their values, and the rounding by way of the oracle."""
import numpy as np

from oracle import capi

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=np.float64)
# E2M1's magnitudes as an 8-bit run-time format: the sign sits in bit 7 instead of bit 3
E2M1_DESC = capi.make_desc(8, 2, 1, 7, nan_code=8)


def padded(cols):
    return -(-cols // 128) * 128


def unpack(codes):
    """Stored bytes [rows, padded / 2] -> codes [rows, padded] in plain order."""
    rows, pitch = codes.shape
    words = np.ascontiguousarray(codes).view(np.uint32).reshape(rows, pitch // 64, 4, 4).transpose(0, 1, 3, 2).reshape(rows, -1)
    return ((words[:, :, None] >> (4 * np.arange(8, dtype=np.uint32))) & 15).astype(np.uint8).reshape(rows, -1)


def pack(plain):
    rows, n = plain.shape
    words = (plain.reshape(rows, -1, 8).astype(np.uint32) << (4 * np.arange(8, dtype=np.uint32))).sum(2, dtype=np.uint32)
    return np.ascontiguousarray(words.reshape(rows, n // 128, 4, 4).transpose(0, 1, 3, 2)).reshape(rows, -1).view(np.uint8)


def scale_values(scales, scale_fmt):
    """Scale bytes, or bfloat16 patterns in uint16, as binary64 values."""
    if scale_fmt == "e8m0":
        return np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (scales.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def values(codes, scales, group, scale_fmt):
    """What a stored matrix stands for, padding included, in binary64."""
    return GRID[unpack(codes)] * np.repeat(scale_values(scales, scale_fmt), group, axis=1)


def expect(x, group, scale_fmt, variant, k, seed, offset, src):
    """(plain codes, stored scales, plain float32 scale values) of a float32 matrix x that came from type `src`."""
    f = np.float32
    rows, cols = x.shape
    n = padded(cols)
    p = np.zeros((rows, n), dtype=f)
    p[:, :cols] = x
    g = p.reshape(rows, n // group, group)
    finite = np.where(np.isfinite(g), np.abs(g), f(0)).max(2)
    nan = np.isnan(g).any(2)
    if scale_fmt == "e8m0":
        _, e = np.frexp(finite)
        e = np.maximum(np.where(finite < f(2.0 ** -126), -127, e - 1 - 2), -127)
        stored = np.where(nan, 255, e + 127).astype(np.uint8)
        inv = np.ldexp(f(1), -e).astype(f)
        s = np.ldexp(1.0, e).astype(f)
    else:
        q = (finite * (f(1) / f(6))).view(np.uint32)
        s = ((q + np.uint32(0xFFFF)) & np.uint32(0xFFFF0000)).view(f)
        s = np.minimum(np.maximum(s, f(2.0 ** -126)), f(10880) if src == "fp16" else f(2.0 ** 125 * 1.328125))
        inv = f(1) / s
        stored = np.where(nan, 0x7FC0, s.view(np.uint32) >> 16).astype(np.uint16)
    with np.errstate(invalid="ignore"):
        y = (g * inv[:, :, None]).reshape(-1)
    y = np.where(np.isnan(y), f(0), y).astype(f)
    code8 = capi.fbsr_round_desc(y, E2M1_DESC, variant, k, seed, offset=offset)
    code = ((code8 & 7) | ((code8 >> 4) & 8)).reshape(g.shape)
    code[nan] = 0
    return code.reshape(rows, n), stored, np.where(nan, f(np.nan), s).astype(f)
