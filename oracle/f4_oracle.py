"""Microscaled 4-bit floating point in plain numpy, 64 bits: the format's values, the quantization rule, the packed buffer byte by byte, and the
products.  Written from the definitions in include/tman.h and the layout in csrc/f4.cuh; shares no code with the kernels.
"""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=np.float64)


def e4m3_values():
    """Value of every byte: sign, four exponent bits (bias 7), three mantissa bits; 0x7F and 0xFF are NaN, no infinities."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b >= 128, -v, v)


def e8m0_values():
    v = 2.0 ** (np.arange(256) - 127.0)
    v[255] = np.nan
    return v


def scale_values(scales, block):
    return (e8m0_values() if block == 32 else e4m3_values())[scales]


def nearest(v, grid):
    """Index of the entry of `grid` (ascending, 0 first) nearest to v >= 0: ties to the even index, the last entry at most."""
    hi = np.clip(np.searchsorted(grid, v), 1, len(grid) - 1)
    below, above = v - grid[hi - 1], grid[hi] - v
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return np.where(up, hi, hi - 1)


def quantize(x, block):
    """x float64 [rows][K] (values of fp16 or bf16).  Codes uint8 [rows][K] (one per byte), scales uint8 [rows][K/block], row scales [rows]."""
    rows, K = x.shape
    b = x.reshape(rows, K // block, block)
    fine = np.isfinite(b).all(-1)
    a = np.where(np.isfinite(b), np.abs(b), 0.0)
    r = np.ones(rows)
    if block == 32:
        top = a.max(-1)
        e = np.clip(np.frexp(np.where(top > 0, top, 1.0))[1] - 1 - 2, -127, 127)
        scales = np.where(top > 0, e + 127, 0).astype(np.uint8)
        unit = 2.0 ** (scales - 127.0)
        scales = np.where(fine, scales, 255).astype(np.uint8)
    else:
        m = a.max((1, 2))
        r = np.where(m > 0, 2.0 ** -126, 1.0)
        while (small := (m > 0) & (m > 2688.0 * r)).any():
            r = np.where(small, 2.0 * r, r)
        grid = e4m3_values()[:127]
        scales = nearest(a.max(-1) / (6.0 * r[:, None]), grid).astype(np.uint8)
        unit = grid[scales] * r[:, None]
        scales = np.where(fine, scales, 0x7F).astype(np.uint8)
    unit = unit[..., None]
    codes = nearest(np.where(unit > 0, a / np.where(unit > 0, unit, 1.0), 0.0), E2M1[:8]).astype(np.uint8)
    codes |= np.signbit(b).astype(np.uint8) << 3
    return codes.reshape(rows, K), scales, r


def values(codes, scales, row_scale, block):
    s = scale_values(scales, block)
    if block == 16:
        s = s * np.asarray(row_scale, dtype=np.float64)[:, None]
    return (E2M1[codes].reshape(codes.shape[0], -1, block) * s[..., None]).reshape(codes.shape)


def sections(rows, K, block):
    """Offsets of codes, scales, row scales, and the size."""
    up = lambda v: (v + 255) // 256 * 256
    tiles, units, h8 = -(-rows // 128), -(-K // 128), -(-rows // 8) * 8
    codes = 256
    scales = codes + up(units * 64 * h8)
    rowsc = scales + tiles * units * (512 if block == 32 else 1024)
    return codes, scales, rowsc, rowsc + (tiles * 512 if block == 16 else 0)


def pack(codes, scales, row_scale, block):
    """The packed buffer (uint8) of a matrix."""
    rows, K = codes.shape
    o_codes, o_scales, o_rows, total = sections(rows, K, block)
    out = np.zeros(total, dtype=np.uint8)
    out[:8] = np.frombuffer(b"TMANF4MX", dtype=np.uint8)
    out[8:24] = np.array([1, rows, K, block], dtype="<u4").view(np.uint8)
    out[24:56] = np.array([o_codes, o_scales, o_rows, total], dtype="<u8").view(np.uint8)
    halves, h8, tiles, sb = -(-K // 128), -(-rows // 8) * 8, -(-rows // 128), 512 if block == 32 else 1024
    r, k = np.meshgrid(np.arange(rows), np.arange(0, K, 2), indexing="ij")
    u = k // 256
    full = 2 * u + 1 < halves                      # units of 256 columns, the last perhaps of 128
    at = u * h8 * 128 + r // 8 * np.where(full, 1024, 512) + k % 256 // 32 * 128 + r % 8 * 16 + k % 32 // 2
    out[o_codes + at] = codes[:, 0::2] | (codes[:, 1::2] << 4)
    r, b = np.meshgrid(np.arange(rows), np.arange(K // block), indexing="ij")
    per = 128 // block
    u, half = b // per // 2, b // per % 2
    at = (u * tiles * 2 + r // 128 * np.where(2 * u + 1 < halves, 2, 1) + half) * sb + b % per // 4 * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4
    out[o_scales + at] = scales
    if block == 16:
        out[o_rows:o_rows + 4 * rows] = np.asarray(row_scale, dtype="<f4").view(np.uint8)
    return out
