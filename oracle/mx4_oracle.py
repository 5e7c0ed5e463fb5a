"""NumPy oracle of the MXFP4 format, its product and the RMS norm in front of
it, written from the definitions and sharing no code with the GPU path.

MXFP4 (OCP Microscaling Formats v1.0): blocks of 32 elements share a scale
2^e (byte e + 127, 255 for NaN) with e = floor(log2 max|x|) - 2, at least
-127; an element is the E2M1 number nearest to x / 2^e, of two equally near
the one with the even code, magnitudes above 6 as 6.
"""
from __future__ import annotations

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def round_bf16(a):
    """fp32 array rounded to bf16 (ties to even), as fp32."""
    u = np.ascontiguousarray(a, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16
    return (r & 0xFFFFFFFF).astype(np.uint32).view(np.float32).reshape(np.shape(a))


def quantize(x):
    """(codes uint8 [n, d/2], scales uint8 [n, d/32]) of finite or non-finite
    rows x [n, d]; arithmetic in fp64 (exact for fp32 inputs)."""
    x = np.asarray(x, np.float64)
    n, d = x.shape
    b = x.reshape(n, d // BLOCK, BLOCK)
    bad = ~np.isfinite(b).all(2)
    f = np.where(bad[..., None], 0.0, b)
    amax = np.abs(f).max(2)
    e = np.where(amax > 0, np.frexp(amax)[1] - 1 - 2, -127)     # frexp: amax = m 2^k, m in [1/2, 1)
    e = np.maximum(e, -127)
    u = np.abs(f) / np.exp2(e.astype(np.float64))[..., None]
    dist = np.abs(u[..., None] - LEVELS)
    best = dist.min(-1, keepdims=True)
    cand = dist == best
    first = cand.argmax(-1)
    last = 7 - cand[..., ::-1].argmax(-1)
    idx = np.where((first != last) & (first % 2 == 1), last, first)
    code = (idx + 8 * np.signbit(f)).astype(np.uint8)
    code[bad] = 0
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    code = code.reshape(n, d)
    return code[:, 0::2] | (code[:, 1::2] << 4), scales


def dequantize(codes, scales):
    """fp64 values of codes [..., d/2] and scales [..., d/32]."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = LEVELS[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.exp2(scales.astype(np.float64) - 127.0)
    s[scales == 255] = np.nan
    return v * np.repeat(s, BLOCK, axis=-1)


def linear(codes_x, scales_x, codes_w, scales_w):
    """(y, sum of |products|) in fp64."""
    x, w = dequantize(codes_x, scales_x), dequantize(codes_w, scales_w)
    return x @ w.T, np.abs(x) @ np.abs(w).T


def linear_grouped(codes_x, scales_x, offsets, codes_w, scales_w, m, row_ids=None):
    """As linear by experts; rows outside all experts are NaN."""
    d_out = codes_w.shape[1]
    y, a = np.full((m, d_out), np.nan), np.full((m, d_out), np.nan)
    for g in range(codes_w.shape[0]):
        rows = np.arange(offsets[g], offsets[g + 1])
        if rows.size:
            src = rows if row_ids is None else np.asarray(row_ids)[rows]
            y[rows], a[rows] = linear(codes_x[src], scales_x[src], codes_w[g], scales_w[g])
    return y, a


def rmsnorm(x, weight, residual=None, eps=1e-6):
    """(h, y) in fp64 throughout; y = 0 where the mean of squares and eps are."""
    h = np.asarray(x, np.float64)
    if residual is not None:
        h = h + np.asarray(residual, np.float64)
    v = (h * h).mean(1, keepdims=True) + eps
    r = np.where(v > 0, 1.0 / np.sqrt(np.where(v > 0, v, 1.0)), 0.0)
    return h, h * np.asarray(weight, np.float64) * r


def rmsnorm_f32(x, weight, residual=None, eps=1e-6):
    """(h, y) with the stated fp32 roundings: h = fl(x + residual), the sum
    of squares in fp64, r and y rounded to fp32."""
    h = np.asarray(x, np.float32)
    if residual is not None:
        h = h + np.asarray(residual, np.float32)
    h64 = h.astype(np.float64)
    v = (h64 * h64).sum(1, keepdims=True) / h.shape[1] + eps
    with np.errstate(divide="ignore"):
        r = np.where(v > 0, 1.0 / np.sqrt(v), 0.0).astype(np.float32)
    return h, (h * np.asarray(weight, np.float32)) * r


def quantize_int8(y):
    """Per-row int8 codes and scales of fp32 y, each step rounded to fp32."""
    y = np.asarray(y, np.float32)
    amax = np.abs(y).max(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        inv = np.where(amax > 0, np.float32(127) / amax, np.float32(0)).astype(np.float32)
    q = np.clip(np.rint(y * inv), -127, 127).astype(np.int8)
    return q, (amax / np.float32(127))[:, 0]
