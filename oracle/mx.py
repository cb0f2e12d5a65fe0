"""Microscaled matrices in 64 bits: quantise, dequantise, product, norm and gate, from their definitions.

Test infrastructure only, numpy; shares no code with the CUDA library or its binding.
"""
from __future__ import annotations

import numpy as np

# every magnitude of the types, in the order of their codes
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])


def magnitudes(bits: int) -> np.ndarray:
    return E4M3 if bits == 8 else E2M1


def scale_index(rows: int, K: int) -> np.ndarray:
    """Byte of row r's group g in the tiled scales, int64 [rows][K / 32]."""
    r, g = np.arange(rows)[:, None], np.arange(K // 32)[None]
    return ((r // 128) * (K // 128) + g // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + g % 4


def scale_bytes(rows: int, K: int) -> int:
    return -(-rows // 128) * 128 * K // 32


def tiled(exps: np.ndarray, K: int, fill: int = 0) -> np.ndarray:
    """Scale bytes [rows][K / 32] in their layout; bytes of rows behind the last are `fill`."""
    out = np.full(scale_bytes(len(exps), K), fill, np.uint8)
    out[scale_index(len(exps), K)] = exps
    return out


def nearest(a: np.ndarray, bits: int) -> np.ndarray:
    """Codes of the magnitudes nearest to a >= 0, ties to the even code."""
    mags = magnitudes(bits)
    mids = (mags[1:] + mags[:-1]) / 2                    # exact
    code = np.searchsorted(mids, a)                      # mids[code - 1] < a <= mids[code]
    tie = (code < len(mids)) & (a == mids[np.minimum(code, len(mids) - 1)]) & (code % 2 == 1)
    return code + tie


def quantize(v: np.ndarray, bits: int):
    """fp64 [rows][K] -> (codes as the type's bytes or packed nibbles, scale bytes [rows][K / 32])."""
    mags = magnitudes(bits)
    g = v.reshape(len(v), -1, 32)
    amax = np.abs(g).max(2)
    bad = ~np.isfinite(amax)
    a = np.where(bad | (amax == 0), 1.0, amax)
    e = np.frexp(a)[1] - 1 - (8 if bits == 8 else 2)
    e = np.where(a > np.ldexp(mags[-1], e), e + 1, e)
    e = np.where(amax == 0, 0, np.maximum(e, -127))
    with np.errstate(invalid="ignore"):
        scaled = np.where(bad[..., None], 0.0, np.ldexp(np.where(bad[..., None], 0.0, g), -e[..., None]))
    code = nearest(np.abs(scaled), bits).astype(np.uint8)
    sign = (np.signbit(scaled) & ~bad[..., None]).astype(np.uint8)
    code = (code | sign << (bits - 1)).reshape(v.shape)
    if bits == 4:
        code = code[:, 0::2] | code[:, 1::2] << 4
    return code, np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes: np.ndarray, exps: np.ndarray, bits: int) -> np.ndarray:
    """fp64 values [rows][K] of codes and scale bytes [rows][K / 32]."""
    if bits == 4:
        codes = np.stack((codes & 15, codes >> 4), 2).reshape(len(codes), -1)
    top = 1 << (bits - 1)
    mag = np.append(E4M3, np.nan) if bits == 8 else E2M1
    v = np.where(codes & top, -1.0, 1.0) * mag[codes & (top - 1)]
    s = np.where(exps == 255, np.nan, np.ldexp(1.0, exps.astype(int) - 127))
    return v * np.repeat(s, 32, 1)


def product(x: np.ndarray, w: np.ndarray):
    """(x @ w.T, |x| @ |w|.T) of fp64 values."""
    return x @ w.T, np.abs(x) @ np.abs(w).T


def half(v: np.ndarray) -> np.ndarray:
    """fp64 -> fp16, one rounding."""
    with np.errstate(over="ignore"):
        return v.astype(np.float16)


def norm(x, residual, gain, eps: float):
    """(h fp16, gain * h / sqrt(mean(h^2) + eps) fp64) of fp16 rows."""
    h = x if residual is None else half(x.astype(np.float64) + residual.astype(np.float64))
    d = h.astype(np.float64)
    v = d / np.sqrt(np.mean(d * d, 1, keepdims=True) + eps)
    return h, v if gain is None else v * gain.astype(np.float64)


def silu(gate_up: np.ndarray) -> np.ndarray:
    K = gate_up.shape[1] // 2
    g, u = gate_up[:, :K].astype(np.float64), gate_up[:, K:].astype(np.float64)
    with np.errstate(over="ignore"):
        return g / (1 + np.exp(-g)) * u


def wrong_groups(codes, exps, v, bits: int, delta, tiny: float = 0.0) -> np.ndarray:
    """Groups of codes and scale bytes that are not the nearest of values within v (1 +- delta) +- tiny:
    a scale that such an amax does not have, or a code further from v than the nearest by more than
    twice that.  delta: a number, or one for each value."""
    delta = np.broadcast_to(delta, v.shape).reshape(len(v), -1, 32)
    mags = magnitudes(bits)
    g = v.reshape(len(v), -1, 32)
    q = values(codes, np.where(exps == 255, 127, exps), bits).reshape(g.shape)
    amax = np.abs(g).max(2)
    bad = ~np.isfinite(amax)
    s = np.ldexp(1.0, exps.astype(int) - 127)
    d = delta.max(2)
    lo, hi = amax * (1 - d) - tiny, amax * (1 + d) + tiny
    fits = (mags[-1] * s >= lo) & ((mags[-1] * s / 2 < hi) | (exps == 0))
    fits |= (lo <= 0) & (exps == 127) & (q == 0).all(2)
    g0 = np.where(bad[..., None], 0.0, g)
    near = mags[nearest(np.abs(g0) / s[..., None], bits)] * s[..., None]
    off = np.abs(q - g0) > np.abs(near - np.abs(g0)) + 2 * (delta * np.abs(g0) + tiny)
    nan_ok = (exps == 255) & (q == 0).all(2)
    return np.where(bad, ~nan_ok, ~fits | off.any(2) | (exps == 255))
