"""fp64 restatement of the 8-bit paged cache: e4m3 codes, block scales, the
record layout, appending and causal attention, token by token in numpy."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 16


def e4m3_values() -> np.ndarray:
    """The 256 values of the code: sign, 4 exponent bits (bias 7), 3 fraction bits; all ones is NaN."""
    out = np.zeros(256)
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        v = math.nan if c & 127 == 127 else (f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10))
        out[c] = -v if c & 128 else v
    return out


VALUES = e4m3_values()
_POSITIVE = VALUES[:127]


def e4m3_codes(x) -> np.ndarray:
    """Nearest codes of |x| <= 448, ties to the even code; NaN and infinities give the NaN code."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a, "left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    d_hi, d_lo = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isfinite(x), code + 128 * np.signbit(x), 127)
    return code.astype(np.uint8)


def scale_for(amax: float) -> float:
    """Smallest 2^e, e >= -126, with amax <= 448 * 2^e."""
    if amax == 0:
        return 2.0 ** -126
    e = max(-126, math.ceil(math.log2(amax / 448)) - 1)
    while 448 * 2.0 ** e < amax:
        e += 1
    return 2.0 ** e


def v_byte(t: int) -> int:
    return 4 * ((t % 8) // 2) + 2 * (t // 8) + t % 2


def record_bytes(hd: int) -> int:
    return 2 * BLOCK * hd + 32


def pack_record(k_codes, v_codes, k_scale: float, v_scale: float) -> np.ndarray:
    """k_codes, v_codes: uint8 [16, hd] -> the record's bytes."""
    hd = k_codes.shape[1]
    rec = np.zeros(record_bytes(hd), np.uint8)
    t, d = np.arange(BLOCK)[:, None], np.arange(hd)[None]
    rec[(t // 8 * (hd // 16) + d // 16) * 128 + t % 8 * 16 + d % 16] = k_codes
    rec[BLOCK * hd + d * 16 + 4 * ((t % 8) // 2) + 2 * (t // 8) + t % 2] = v_codes
    rec[-32:-24] = np.array([k_scale, v_scale], np.float32).view(np.uint8)
    return rec


def unpack_record(rec):
    """The record's (k_codes, v_codes [16, hd], k_scale, v_scale)."""
    hd = (len(rec) - 32) // 32
    t = np.arange(BLOCK)
    k = rec[:BLOCK * hd].reshape(2, hd // 16, 8, 16)[t // 8, :, t % 8].reshape(BLOCK, hd)
    v = rec[BLOCK * hd:2 * BLOCK * hd].reshape(hd, BLOCK)[:, [v_byte(i) for i in t]].T
    s = np.ascontiguousarray(rec[-32:-24]).view(np.float32)
    return k, v, float(s[0]), float(s[1])


def rope(x, angles) -> np.ndarray:
    """Rotate-half RoPE of x [..., hd] with angles [..., hd / 2, 2] (cos, sin)."""
    h = x.shape[-1] // 2
    a, b, c, s = x[..., :h], x[..., h:], angles[..., 0], angles[..., 1]
    return np.concatenate((a * c - b * s, b * c + a * s), -1)


def append_block(old, first: int, k, v):
    """One block: old = (k_codes, v_codes, k_scale, v_scale) or None, new rows k, v [n, hd] from token `first` on.
    Returns the block's (k_codes, v_codes, k_scale, v_scale); tokens behind the new rows are zeros."""
    out = []
    for i, x in enumerate((k, v)):
        x = np.asarray(x, np.float64)
        finite = np.abs(x[np.isfinite(x)])
        scale = scale_for(float(finite.max()) if finite.size else 0.0)
        codes = np.zeros((BLOCK, x.shape[1]), np.uint8)
        if first > 0:
            scale = max(scale, old[2 + i])
            codes[:first] = e4m3_codes(VALUES[old[i][:first]] * (old[2 + i] / scale))
        codes[first:first + len(x)] = e4m3_codes(x / scale)
        out.append((codes, scale))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def attention(q, k, v, scale: float):
    """q [R, hq, hd] of the last R of n tokens, k, v [n, hk, hd]: (out [R, hq, hd], lse [R, hq], weight [R, hq, hd]:
    the softmax average of |v|, which roundings of the probabilities are relative to)."""
    (R, hq, hd), (n, hk) = q.shape, k.shape[:2]
    out, lse, mag = np.zeros((R, hq, hd)), np.full((R, hq), -np.inf), np.zeros((R, hq, hd))
    for i in range(R):
        seen = n - R + i + 1
        if seen <= 0:
            continue
        for h in range(hq):
            g = h // (hq // hk)
            s = k[:seen, g] @ q[i, h] * scale
            m = s.max()
            p = np.exp(s - m)
            lse[i, h] = m + math.log(p.sum()) if not np.isnan(p.sum()) else math.nan
            out[i, h] = p @ v[:seen, g] / p.sum()
            mag[i, h] = p @ np.abs(v[:seen, g]) / p.sum()
    return out, lse, mag
