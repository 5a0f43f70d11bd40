"""Plain statements, in 64 bits, of what the calls of a 4-bit cache and of eviction answer (no library code)."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6.0])
GROUP = 32


def bf16(x):
    """Nearest bfloat16, as float64."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    r = (u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000)
    return r.view(np.float32).astype(np.float64)


def pack(x):
    """Codes [.., D] (0 .. 15) and scale bytes [.., D / 32] of rows of float values."""
    x = np.asarray(x, dtype=np.float64)
    x = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    top = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    e = np.full(top.shape, -125)
    for k in range(-125, 126):  # the smallest with top <= 7 * 2^e
        e = np.where(np.where(bad, 0.0, top) > 7 * 2.0 ** (k - 1), k, e)
    y = np.where(bad[..., None], 0.0, np.abs(x)) / (2.0 ** e)[..., None]
    code = np.zeros(y.shape, dtype=np.int64)
    for i in range(1, 8):
        middle = (GRID[i - 1] + GRID[i]) / 2
        code = np.where((y > middle) | ((y == middle) & (i % 2 == 0)), i, code)
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(x))
    return code.reshape(*code.shape[:-2], code.shape[-2] * GROUP), np.where(bad, 255, e + 127)


def values(code, byte):
    x = GRID[code % 8] * np.where(code >= 8, -1.0, 1.0)
    f = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return x * np.repeat(f, GROUP, -1)


def to_bytes(code):
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def from_bytes(codes):
    c = codes.astype(np.int64)
    return np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], 2 * c.shape[-1])


def evict(tally, pos, known, before, L, keep, first, recent, slack):
    """One head of one sequence.  (pairs of rows (from, to), positions of rows 0 .. keep - 1) or None where nothing changes."""
    if L <= keep + slack:
        return None
    where = [int(pos[t]) if t < known else before + t - known for t in range(L)]
    total = before + L - known
    safe = [p < first or p >= total - recent for p in where]
    rank = sorted(range(L), key=lambda t: (not safe[t], 0.0 if safe[t] else (np.inf if np.isnan(tally[t]) else -float(tally[t]) if tally[t] != -np.inf else 1e300), t))
    # (NaN last, -inf before it, any other value before that)
    stays = set(rank[:keep])
    holes = [t for t in range(keep) if t not in stays]
    movers = [t for t in range(keep, L) if t in stays]
    assert len(holes) == len(movers)
    pairs = list(zip(movers, holes))
    at = where[:keep]
    for a, b in pairs:
        at[b] = where[a]
    return pairs, at


def attention(q, k, v, scale):
    """q [G, D] over rows k, v [T, D]: outputs, log-sum-exps, weights [G, T], and what rounding errors scale with: sum p |v|, the largest |score|
    that the terms of a score can add up to."""
    z = q @ k.T * scale
    if k.shape[0] == 0:
        return np.zeros_like(q), np.full(len(q), -np.inf), z, np.zeros_like(q), np.zeros(len(q))
    m = z.max(1, keepdims=True)
    p = np.exp(z - m)
    s = p.sum(1, keepdims=True)
    p = p / s
    return p @ v, (m + np.log(s))[:, 0], p, p @ np.abs(v), (np.abs(q) @ np.abs(k).T * abs(scale)).max(1)


def rounding(z_most, T, D):
    """Relative error of a weight: a score's D products and sums and its scaling to base 2 (2^-24 of the terms' magnitudes each, both in the score and in the
    maximum or log-sum-exp it is held against), the exponential (2^-22), and the sums over up to T tokens (2^-24 each)."""
    return 2 * (D + 4) * 2.0 ** -24 * z_most + 2.0 ** -22 + (T + 64) * 2.0 ** -24
