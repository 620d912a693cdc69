"""Oracle: the paged 4-bit key/value cache and the attention over it (serving of concurrent episodes, Appendix A).

Test infrastructure only: the GPU library never imports this module.

A record holds 128 tokens of one key/value head:
  * keys: e2m1 codes [token][64 bytes] along the head dimension, low half first; every 32 elements share
    2^(b - 127) with b - 127 = floor(log2 max) - 2, one more where max is at least 1.75 powers of two,
    at least -100 and at most 125; byte b of block i of token t at [i][t % 16][t / 16];
  * values: e2m1 codes [element][64 bytes] along the tokens in the order `POS`; every token has a scale
    max / 6 rounded up to 6 significant bits, between 2^-100 and 1.3125 2^125, as bfloat16 in that order.
Codes are the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code, the sign kept on zeros. A block or
row with an infinity or a NaN has codes 0 and the scale NaN (byte 255).
The quotient max / 6 and the quotients that are coded are float32 roundings; the rest is exact.
"""
import numpy as np

PAGE, DH, RECORD = 128, 128, 17152
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
POS = np.array([16 * ((p >> 2) & 7) + 4 * (p >> 5) + (p & 3) for p in range(PAGE)])  # token of a position


def codes(x):
    """e2m1 codes of x (float64 values)."""
    a = np.minimum(np.abs(x), 6.0)
    hi = np.clip(np.searchsorted(GRID, a), 1, 7)
    lo = hi - 1
    up, down = GRID[hi] - a, a - GRID[lo]
    mag = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (mag + 8 * np.signbit(x)).astype(np.uint8)


def values(c):
    return np.where(c & 8, -1.0, 1.0) * GRID[c & 7]


def quant_k(k):
    """k [..., 128] -> codes, bytes [..., 4], held values."""
    x = np.asarray(k, np.float64).reshape(*k.shape[:-1], 4, 32)
    top = np.abs(x).max(-1)
    bad = ~np.isfinite(top)
    m, e = np.frexp(np.where(bad, 1.0, top))  # m in [1/2, 1)
    e = np.where(top == 0, -100, np.clip(e - 3 + (m >= 0.875), -100, 125))
    s = np.ldexp(1.0, e)[..., None]
    c = np.where(bad[..., None], 0, codes(np.where(bad[..., None], 0.0, x) / s)).astype(np.uint8)
    held = np.where(bad[..., None], np.nan, values(c) * s)
    return c.reshape(k.shape), np.where(bad, 255, e + 127).astype(np.uint8), held.reshape(k.shape)


def quant_v(v):
    """v [..., 128] -> codes, scales [...] (float32), held values."""
    x = np.asarray(v, np.float32)
    top = np.abs(x).max(-1)
    bad = ~np.isfinite(top)
    m, e = np.frexp((np.where(bad, 1.0, top).astype(np.float32) / np.float32(6.0)).astype(np.float64))
    s = np.clip(np.ldexp(np.ceil(m * 64.0), e - 6), 2.0 ** -100, 1.3125 * 2.0 ** 125).astype(np.float32)
    c = np.where(bad[..., None], 0, codes((np.where(bad[..., None], 0, x) / s[..., None]).astype(np.float64))).astype(np.uint8)
    held = np.where(bad[..., None], np.nan, values(c) * s[..., None].astype(np.float64))
    return c, np.where(bad, np.float32(np.nan), s).astype(np.float32), held


def _pack(c):
    return (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)


def _unpack(b):
    return np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], -1)


def store(cache, table_row, kv_head, first, k, v):
    """Write rows k, v [n, 128] of one head at positions first .. into cache [pages, kv_heads, RECORD] (bytes)."""
    ck, ek, _ = quant_k(k)
    cv, sv, _ = quant_v(v)
    place = np.argsort(POS)
    for i in range(len(k)):
        p = first + i
        if p < 0:
            continue
        rec = cache[table_row[p // PAGE], kv_head]
        t = p % PAGE
        rec[t * 64:t * 64 + 64] = _pack(ck[i])
        for b in range(4):
            rec[16384 + b * 128 + (t % 16) * 8 + t // 16] = ek[i, b]
        pos = int(place[t])
        rows = rec[8192:16384].reshape(DH, 64)
        sh = 4 * (pos & 1)
        rows[:, pos // 2] = (rows[:, pos // 2] & (0xF0 >> sh)) | (cv[i] << sh)
        bits = sv[i:i + 1].view(np.uint32)[0] >> 16 if np.isfinite(sv[i]) else 0x7FC0
        rec[16896 + 2 * pos:16898 + 2 * pos] = np.array([bits & 255, bits >> 8], np.uint8)


def load(cache, table_row, kv_head, length):
    """(K, V) [length, 128] float64 that the cache stands for."""
    K, V = np.zeros((length, DH)), np.zeros((length, DH))
    place = np.argsort(POS)
    for p0 in range(0, length, PAGE):
        rec = cache[table_row[p0 // PAGE], kv_head]
        n = min(PAGE, length - p0)
        t = np.arange(n)
        ck = values(_unpack(rec[:8192].reshape(PAGE, 64)))[:n].reshape(n, 4, 32)
        b = rec[16384:16896].reshape(4, 16, 8)[:, t % 16, t // 16].T.astype(np.float64)
        with np.errstate(over="ignore"):
            K[p0:p0 + n] = np.where((b == 255)[..., None], np.nan, ck * (2.0 ** (b - 127))[..., None]).reshape(n, DH)
        cv = values(_unpack(rec[8192:16384].reshape(DH, 64)))[:, place[:n]].T
        s = (rec[16896:].view(np.uint16)[place[:n]].astype(np.uint32) << 16).view(np.float32).astype(np.float64)
        V[p0:p0 + n] = cv * s[:, None]
    return K, V


def attend(q, K, V, last, scale):
    """One query [128] over positions <= last: (o, lse, sum p |v|, bound of the scores' sums of magnitudes)."""
    if last < 0:
        return np.zeros(DH), -np.inf, np.zeros(DH), 0.0
    k, v = K[:last + 1], V[:last + 1]
    s = scale * (k @ q)
    m = s.max()
    e = np.exp(s - m)
    p = e / e.sum()
    return p @ v, m + np.log(e.sum()), p @ np.abs(v), float(np.max(np.abs(s))) + scale * float((np.abs(k) @ np.abs(q)).max())
