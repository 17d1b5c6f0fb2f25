"""CPU oracle of the microscaled forward: quantization of rows to MXFP4 and MXFP8,
products of their values, the norm with quantized rows, and attention over caches
in MXFP4, in float64 (formats: oracle/codec_ref.py, of which this is a form over
whole arrays; a CPU test holds the two to the same codes).

TEST INFRASTRUCTURE ONLY, like `polestar_ref`.
"""

from __future__ import annotations

import numpy as np

from oracle.codec_ref import FORMATS, _grid

NAN_SCALE = 255


def quantize(v: np.ndarray, fmt: str) -> tuple[np.ndarray, np.ndarray]:
    """Rows [..., n] (float64) -> codes [..., n] (ints) and scale bytes [..., n / 32].
    A block with a NaN or an infinity: byte 255, zero codes."""
    v = np.asarray(v, np.float64)
    eb, mb, _, emax, _ = FORMATS[fmt]
    vals, codes = _grid(fmt)
    blk = v.reshape(*v.shape[:-1], -1, 32)
    bad = ~np.isfinite(blk).all(axis=-1)
    blk = np.where(bad[..., None], 0.0, blk)
    amax = np.abs(blk).max(axis=-1)
    _, e = np.frexp(amax)
    e = np.where(amax > 0, np.maximum(e - 1 - emax, -127), -127)
    a = np.abs(np.ldexp(blk, -e[..., None]))
    mid = (vals[1:] + vals[:-1]) / 2
    lo = np.searchsorted(mid, a, side="left")                       # at a middle: the lower one
    tie = (lo < len(mid)) & (a == mid[np.minimum(lo, len(mid) - 1)]) & (codes[lo] % 2 == 1)
    i = lo + tie
    c = codes[i] | np.where((blk < 0) & (vals[i] > 0), 1 << (eb + mb), 0)
    return c.reshape(v.shape), np.where(bad, NAN_SCALE, e + 127)


def values(codes: np.ndarray, scales: np.ndarray, fmt: str) -> np.ndarray:
    """Codes [..., n] and scale bytes [..., n / 32] -> float64 values (NaN for the byte 255)."""
    eb, mb, bias, _, _ = FORMATS[fmt]
    codes = np.asarray(codes, np.int64)
    mag = codes & ((1 << (eb + mb)) - 1)
    ex, m = mag >> mb, (mag & ((1 << mb) - 1)) / 2.0 ** mb
    x = np.where(ex == 0, m * 2.0 ** (1 - bias), (1 + m) * np.exp2(ex - bias))
    x = np.where(codes >> (eb + mb) & 1, -x, x).reshape(*codes.shape[:-1], -1, 32)
    s = np.where(scales == NAN_SCALE, np.nan, np.exp2(np.asarray(scales, np.float64) - 127))
    return (x * s[..., None]).reshape(codes.shape)


def pack(codes: np.ndarray, fmt: str) -> np.ndarray:
    """Codes [..., n] -> bytes."""
    if fmt == "mxfp8":
        return codes.astype(np.uint8)
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(b: np.ndarray, fmt: str) -> np.ndarray:
    """Bytes -> codes [..., n]."""
    b = np.asarray(b, np.int64)
    if fmt == "mxfp8":
        return b
    return np.stack((b & 15, b >> 4), axis=-1).reshape(*b.shape[:-1], -1)


def held(b: np.ndarray, scales: np.ndarray, fmt: str) -> np.ndarray:
    """Values of packed bytes and scale bytes."""
    return values(unpack(b, fmt), scales, fmt)


def rmsnorm(x: np.ndarray, gain: np.ndarray | None, eps: float) -> np.ndarray:
    """x / sqrt(mean x^2 + eps) * gain, float64 (eps as the float32 that the call passes)."""
    x = np.asarray(x, np.float64)
    h = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + float(np.float32(eps)))
    return h if gain is None else h * np.asarray(gain, np.float64)


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, length: int, scale: float):
    """One sequence and query head: q [n][hd], k and v [seq][hd], float64 ->
    out [n][hd], lse [n], and sum_j p_j |v_j| [n][hd] and max_j sum |q k_j| scale [n] for tolerances."""
    n, hd = q.shape
    if length == 0:
        return np.zeros((n, hd)), np.full(n, -np.inf), np.zeros((n, hd)), np.zeros(n)
    k, v = k[:length], v[:length]
    s = q @ k.T * scale
    m = s.max(axis=1, keepdims=True)
    p = np.exp(s - m)
    z = p.sum(axis=1, keepdims=True)
    p = p / z
    return p @ v, (m + np.log(z))[:, 0], p @ np.abs(v), (np.abs(q) @ np.abs(k).T).max(axis=1) * scale
