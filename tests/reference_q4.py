"""Plain restatement, in 64 bits, of rotary positions, of the 4-bit rows and of attention over them: what the tests of these operators
compare with.  numpy only."""
import numpy as np

SCALE = 1.0 / np.sqrt(128.0)


def bits(x):
    """float array -> bf16 bit patterns, round to nearest even"""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    nan = np.isnan(np.asarray(x, np.float32))
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(nan, np.uint16(0x7FC0), r)


def number(b16):
    return (np.asarray(b16, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def to_bf16_number(x):
    """RNE of 64-bit numbers to the 8 bits of bf16 (normal range and below)"""
    m, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e, -125) - 8)
    return np.round(x / step) * step


def quantise(rows):
    """bf16 bits [..., 128] -> (values they stand for, scale [..., 2], low [..., 2]) in 64 bits"""
    with np.errstate(invalid="ignore"):
        x = number(rows).reshape(rows.shape[:-1] + (2, 64))
        low, high = x.min(-1), x.max(-1)
        bad = ~np.isfinite(x).all(-1)
        scale = to_bf16_number(np.where(bad, 0.0, high - low) / 15.0)
        code = np.zeros_like(x)
        for k in range(15):
            # (the border is exact in 64 bits, a difference x - low need not be: numbers may lie 2^100 apart)
            code += (x > low[..., None] + (k + 0.5) * scale[..., None]) & (scale[..., None] > 0)
        values = low[..., None] + code * scale[..., None]
        values[bad] = np.nan
    return values.reshape(rows.shape), scale, low


def turn(x, positions, axis, inv_freq, adjacent):
    """x [B, n, heads, 128] numbers, positions [B, n, n_axes] -> turned, in 64 bits"""
    phi = positions[..., axis].astype(np.float64) * inv_freq      # [B, n, 64]
    c, s = np.cos(phi)[:, :, None], np.sin(phi)[:, :, None]
    y = np.empty_like(x)
    if adjacent:
        p, q = x[..., 0::2], x[..., 1::2]
        y[..., 0::2], y[..., 1::2] = p * c - q * s, q * c + p * s
    else:
        p, q = x[..., :64], x[..., 64:]
        y[..., :64], y[..., 64:] = p * c - q * s, q * c + p * s
    return y


def attend(q, K, V, seen, scale=SCALE):
    """q [R, 128], K, V [n, 128], seen [R, n] -> out [R, 128], lse [R], sum of p |v| / sum of p [R, 128]"""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        logits = np.where(seen, q @ K.T * scale, -np.inf) if K.shape[0] else np.full((q.shape[0], 0), -np.inf)
        out, lse, spread = np.zeros_like(q), np.full(q.shape[0], -np.inf), np.zeros_like(q)
        for r in range(q.shape[0]):
            m = logits[r].max() if logits.shape[1] else -np.inf
            if m == -np.inf:
                continue
            p = np.exp(logits[r] - m)
            used = p != 0
            out[r], spread[r] = p[used] @ V[used] / p.sum(), p[used] @ np.abs(V[used]) / p.sum()
            lse[r] = m + np.log(p.sum())
    return out, lse, spread
