"""Plain fp64 CPU oracle of the 8-bit cache and the 4-bit weights (numpy only; used by tests).

Formats: e4m3 (OCP, no infinities) and e2m1 values with a power-of-two scale per block, held as exponent + 127.  A block's
exponent is the smallest with which its largest finite magnitude stays within the largest value of the format (448, 6), kept in
[-100, 120]; values are rounded to nearest, ties to the even code, those beyond the largest code to that.  With the exponent 120 the
largest code of the cache is 240: the next, 256, would stand for 2^128, which bf16 does not hold.  Pins:
tests/test_oracle_lowbit.py, tests/test_oracle_lowbit_range.py."""
import numpy as np

from . import kvra_oracle as orc

BLOCK, GROUP = 64, 32
E_MIN, E_MAX = -100, 120

# magnitude of code 0, 1, ...: e4m3 has 4 exponent bits (bias 7) and 3 mantissa bits, code 127 is NaN; e2m1 2 (bias 1) and 1
E4M3 = np.array([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])
E2M1 = np.array([m / 2 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1) for e in range(4) for m in range(2)])


def exponent(peak, most):
    """The smallest e with peak <= most * 2^e, kept within bounds (E_MIN for a peak of 0)."""
    peak = np.asarray(peak, dtype=np.float64)
    e = np.floor(np.log2(np.maximum(peak, 1e-300) / most)).astype(np.int64) - 1     # off by one at most: counted up below
    for _ in range(3):
        e += peak > most * 2.0 ** e
    return np.clip(np.where(peak > 0, e, E_MIN), E_MIN, E_MAX)


def nearest(x, values):
    """Index of the nearest of `values` (rising from 0) to |x|, ties to the even index; sign bit on top."""
    a = np.minimum(np.abs(x), values[-1])
    hi = np.clip(np.searchsorted(values, a), 1, len(values) - 1)
    below, above = a - values[hi - 1], values[hi] - a
    code = np.where((below < above) | ((below == above) & (hi % 2 == 1)), hi - 1, hi)
    return code | (np.signbit(x).astype(np.int64) * (128 if len(values) == 127 else 8))


def e4m3_codes(x, e):
    """x * 2^-e as e4m3 bytes; what is not finite is NaN."""
    e = np.asarray(e, dtype=np.float64)
    most = np.where(e >= E_MAX, 240.0, E4M3[-1])
    with np.errstate(invalid="ignore"):
        code = nearest(np.clip(np.where(np.isfinite(x), x, 0.0) * 2.0 ** -e, -most, most), E4M3)
    return np.where(np.isfinite(x), code, 127 | np.signbit(x) * 128).astype(np.uint8)


def e4m3_values(codes):
    c = codes.astype(np.int64)
    v = np.append(E4M3, np.nan)[c & 127]
    return np.where(c > 127, -v, v)


def append_rows(cache, scale, new, prefix):
    """Rows prefix .. of a cache (uint8 [capacity, heads, d]) and its scales (uint8 [blocks, heads]) take `new` (fp64), in place."""
    c, heads, _ = new.shape
    for b in range(prefix // BLOCK, (prefix + c + BLOCK - 1) // BLOCK):
        lo, hi = max(prefix, b * BLOCK), min(prefix + c, (b + 1) * BLOCK)
        rows = new[lo - prefix:hi - prefix]
        e = exponent(np.where(np.isfinite(rows), np.abs(rows), 0.0).max(axis=(0, 2)), 448.0)
        if lo > b * BLOCK:                                 # rows were there: the scale does not shrink, they follow it
            old = scale[b].astype(np.int64) - 127
            e = np.maximum(e, old)
            held = e4m3_values(cache[b * BLOCK:lo]) * 2.0 ** old[None, :, None]
            cache[b * BLOCK:lo] = e4m3_codes(held, e[None, :, None])
        cache[lo:hi] = e4m3_codes(rows, e[None, :, None])
        scale[b] = e + 127


def cache_values(cache, scale):
    e = np.repeat(scale.astype(np.int64) - 127, BLOCK, axis=0)[:cache.shape[0]]
    return e4m3_values(cache) * 2.0 ** e[..., None]


def rotate(x, prefix, base):
    return x if base is None or base <= 0 else orc.rope(x, np.arange(prefix, prefix + x.shape[0]), base)


def pack(w):
    """Codes [n, k/2] (first of a pair in the low bits) and scales [n, k/32] of w [n, k] (fp64)."""
    n, k = w.shape
    g = w.reshape(n, k // GROUP, GROUP)
    good = np.isfinite(g).all(axis=2)
    e = np.where(good, exponent(np.where(good[..., None], np.abs(g), 0.0).max(axis=2), 6.0), 128)
    code = nearest(np.where(good[..., None], g, 0.0) * 2.0 ** -e[..., None].astype(np.float64), E2M1).reshape(n, k // 2, 2)
    return (code[..., 0] | code[..., 1] << 4).astype(np.uint8), (e + 127).astype(np.uint8)


def unpack(codes, scales):
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[0], -1).astype(np.int64)
    v = np.where(c > 7, -E2M1[c & 7], E2M1[c & 7])
    factor = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(factor, GROUP, axis=1)


def linear(x, codes, scales, codes2=None, scales2=None, residual=None):
    """(result, sum of the magnitudes of the products it is made of: what its rounding errors are counted against)."""
    w = unpack(codes, scales)
    y, a = x @ w.T, np.abs(x) @ np.abs(w).T
    if codes2 is not None:
        w2 = unpack(codes2, scales2)
        u, b = x @ w2.T, np.abs(x) @ np.abs(w2).T
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-y))
        # d silu / dy is at most 1.1; the exponential's own error is counted with the products'
        return y * s * u, 1.1 * a * np.abs(u) + np.abs(y * s) * b
    return (y, a) if residual is None else (y + residual, a + np.abs(residual))


def attention(q, k, v, prefix, scale):
    """(softmax(scale q k^T) v, sum of weight * |v|, largest sum of |terms| of a row's scores); q [c, H, d], k and v
    [prefix + c, Hkv, d] in fp64, key j visible to row r iff j <= prefix + r."""
    c, H, d = q.shape
    G = H // k.shape[1]
    out, mass, reach = np.empty((c, H, d)), np.empty((c, H, d)), np.empty((c, H, 1))
    visible = np.arange(prefix + c)[None, :] <= np.arange(prefix, prefix + c)[:, None]
    for h in range(H):
        K, V = k[:, h // G], v[:, h // G]
        s = np.where(visible, scale * (q[:, h] @ K.T), -np.inf)
        reach[:, h, 0] = np.where(visible, scale * (np.abs(q[:, h]) @ np.abs(K).T), 0.0).max(axis=1)
        w = np.exp(s - s.max(axis=1, keepdims=True))
        w /= w.sum(axis=1, keepdims=True)
        out[:, h], mass[:, h] = w @ V, w @ np.abs(V)
    return out, mass, reach
