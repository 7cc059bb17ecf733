"""Plain forms, in 64 bits, of what a model does with resident units: tokens
into and out of KV pages, attention over shared prefixes, adapters beside a
projection.  Inputs are the stored bits; results are float64 with the sums of
magnitudes that error bounds are derived from.
"""
from __future__ import annotations

import numpy as np

BF16, F16, E4M3 = 1, 2, 3
HALF_STEP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, E4M3: 2.0 ** -4}


def _e4m3_values():
    code = np.arange(128)
    e, m = code >> 3, code & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[127] = np.nan
    return np.concatenate([v, -v])


E4M3_VALUES = _e4m3_values()


def to_bits(x, kind):
    """float array -> uint16 bits of the 16-bit type, nearest even."""
    x = np.asarray(x, dtype=np.float32)
    if kind == F16:
        with np.errstate(over="ignore"):
            return x.astype(np.float16).view(np.uint16)
    u = np.ascontiguousarray(x).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r)


def from_bits(u, kind):
    """Stored bits -> float64 (uint16 of a 16-bit type, uint8 codes of e4m3)."""
    if kind == E4M3:
        return E4M3_VALUES[u]
    if kind == F16:
        return np.ascontiguousarray(u).view(np.float16).astype(np.float64)
    return (np.asarray(u).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def e4m3_scale(x):
    """Scale of rows x [..., dim] (float64 of 16-bit values): the largest finite
    magnitude over 448, as the 32-bit division gives it, at least 2^-126."""
    a = np.abs(x)
    a = np.where(np.isfinite(a), a, 0.0).max(-1).astype(np.float32)
    return np.maximum(a / np.float32(448), np.float32(2.0 ** -126))


def e4m3_half_step(q):
    """Half the distance between e4m3 values around q (saturating at 448)."""
    a = np.clip(np.abs(q), 2.0 ** -6, 448.0)
    return 2.0 ** (np.floor(np.log2(a)) - 4)


def positions(row_off, lens):
    """Per row of the batch: its request and its agent's token (may be negative)."""
    row_off = np.asarray(row_off, dtype=np.int64)
    rows = np.diff(row_off)
    request = np.repeat(np.arange(len(rows)), rows)
    i = np.arange(row_off[-1]) - row_off[request]
    return request, np.asarray(lens, dtype=np.int64)[request] - rows[request] + i


def attention(q, keys, values, seen, scale):
    """One request's rows: q [rows, heads, per, dim]; keys and values [tokens,
    heads, dim]; seen [rows, tokens].  Returns out, lse and per output the sums
    that errors scale with: sum w |v| and the largest |v|; per row the largest
    scale * sum |q k| over what it sees."""
    rows, heads, per, dim = q.shape
    keys, values = np.where(seen.any(0)[:, None, None], keys, 0), \
        np.where(seen.any(0)[:, None, None], values, 0)
    if keys.shape[0] == 0:
        z = np.zeros(q.shape)
        return z, np.full(q.shape[:3], -np.inf), z, z, np.zeros(q.shape[:3])
    score = np.einsum("rhgd,thd->rhgt", q, keys) * scale
    size = np.einsum("rhgd,thd->rhgt", np.abs(q), np.abs(keys)) * abs(scale)
    score = np.where(seen[:, None, None, :], score, -np.inf)
    top = score.max(-1)
    ref = np.where(np.isfinite(top), top, 0.0)
    w = np.exp(score - ref[..., None])
    total = w.sum(-1)
    with np.errstate(divide="ignore"):
        lse = ref + np.log(total)                    # -infinity where nothing is seen
    w = w / np.where(total == 0, 1.0, total)[..., None]
    out = np.einsum("rhgt,thd->rhgd", w, values)
    mag = np.einsum("rhgt,thd->rhgd", w, np.abs(values))
    big = np.broadcast_to(np.abs(values).max(0)[None, :, None, :], out.shape)
    return out, lse, mag, big, np.where(seen[:, None, None, :], size, 0.0).max(-1)


def adapter(x, a, b, base, scale):
    """out = base + scale * B (A x) for rows x [rows, n_in]; also |scale| sum |B| |A x|
    and |scale| sum |B| (sum |A| |x|)."""
    low = x @ a.T
    return (base + scale * (low @ b.T), abs(scale) * (np.abs(low) @ np.abs(b).T),
            abs(scale) * ((np.abs(x) @ np.abs(a).T) @ np.abs(b).T))


def e4m3_encode(q):
    """Codes of 32-bit quotients, to nearest with ties to the even code,
    saturating; NaN to NaN."""
    q = np.asarray(q, dtype=np.float64)
    a = np.minimum(np.abs(q), 448.0)
    v = E4M3_VALUES[:127]
    hi = np.clip(np.searchsorted(v, np.where(np.isnan(a), 0, a)), 1, 126)
    lo = hi - 1
    up, down = v[hi] - a, a - v[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isnan(q), 127, code)
    return (code | (np.signbit(q) << 7)).astype(np.uint8)


def stored(x, kind):
    """What a cache of this kind holds after 16-bit rows x (in 64 bits) were written."""
    if kind != E4M3:
        return x
    s = e4m3_scale(x)[..., None]
    return from_bits(e4m3_encode(x.astype(np.float32) / s), E4M3) * s.astype(np.float64)
