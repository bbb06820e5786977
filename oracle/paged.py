"""The operators on a paged cache in fp64, from their definitions (include/blink.h). Oracle code: test infrastructure only.

A cache is a flat uint8 array. 16 bits: halves, keys [block][kv head][token][dim], then values [block][kv head][dim][token].
4 bits: per (block, kv head) codes of the keys, codes of the values, scales of the keys, scales of the values (e2m1 codes, one
power-of-two scale per 32 dimensions of a token).
"""
import numpy as np

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])
E_MIN, E_MAX = -23, 13


def cache_bytes(n_blocks, nkv, hd, bits):
    return n_blocks * nkv * hd * (64 if bits == 16 else 17)


def encode4(x):
    """x [..., hd] fp64 -> (codes [..., hd] 0..15, scale bytes [..., hd/32])."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(g).max(axis=-1)
    fine = np.isfinite(g).all(axis=-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.ceil(np.log2(np.where(fine & (top > 0), top, 1.0) / 7.0)).astype(int)     # 3.5 < top / 2^e <= 7
    e = np.where(top / 2.0 ** e <= 3.5, e - 1, np.where(top / 2.0 ** e > 7.0, e + 1, e))  # (the logarithm's own rounding)
    e = np.where(fine & (top > 0), np.clip(e, E_MIN, E_MAX), E_MIN)
    y = np.where(fine[..., None], g, 0.0) * 2.0 ** -e[..., None]
    a = np.abs(y)
    d = np.abs(a[..., None] - LEVELS[:8])
    near = d.min(axis=-1, keepdims=True)
    tie = d == near                                              # of two equally near codes the even one
    even = np.arange(8) % 2 == 0
    c = np.where((tie & even).any(axis=-1), np.argmax(tie & even, axis=-1), np.argmax(tie, axis=-1))
    c = np.where(fine[..., None], c | (np.signbit(y).astype(int) << 3), 0)
    return c.reshape(x.shape), np.where(fine, e + 127, 255).astype(np.uint8)


def decode4(codes, scales):
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return LEVELS[codes] * np.repeat(s, 32, axis=-1)


def half(x):
    """Round to nearest halves, saturating; NaN stays."""
    with np.errstate(over="ignore"):
        return np.clip(x, -65504.0, 65504.0).astype(np.float16)


class Cache:
    """View of a cache's bytes; put() stores a token as the operator does, get() reads tokens as fp64."""

    def __init__(self, data, n_blocks, nkv, hd, bits):
        self.n_blocks, self.nkv, self.hd, self.bits, self.data = n_blocks, nkv, hd, bits, data
        if bits == 16:
            kv = data.view(np.float16).reshape(2, n_blocks, nkv, 16 * hd)
            self.k, self.v = kv[0].reshape(n_blocks, nkv, 16, hd), kv[1].reshape(n_blocks, nkv, hd, 16)
        else:
            rec = data.reshape(n_blocks, nkv, 17 * hd)
            self.kc, self.vc = rec[..., :8 * hd], rec[..., 8 * hd:16 * hd]
            self.ks, self.vs = rec[..., 16 * hd:16 * hd + hd // 2], rec[..., 16 * hd + hd // 2:]

    def _value_at(self, off):
        """Byte of the pair of dimensions i of a token's value, for all i."""
        i, w = np.arange(self.hd // 2), self.hd // 32
        return ((off // 4 * 16 + i // w) * 4 + off % 4) * w + i % w

    def put(self, slot, k, v):
        """k, v [nkv][hd]: fp64 keys, values."""
        if slot < 0 or slot // 16 >= self.n_blocks:
            return
        b, o, hd = slot // 16, slot % 16, self.hd
        if self.bits == 16:
            self.k[b, :, o], self.v[b, :, :, o] = half(k), half(v)
            return
        g = np.arange(hd // 32) * 16 + o
        c, s = encode4(k)
        self.kc[b, :, o * (hd // 2):(o + 1) * (hd // 2)] = c[:, ::2] | c[:, 1::2] << 4
        self.ks[b][:, g] = s
        c, s = encode4(v)
        self.vc[b][:, self._value_at(o)] = c[:, ::2] | c[:, 1::2] << 4
        self.vs[b][:, g] = s

    def get(self, slot):
        b, o, hd = slot // 16, slot % 16, self.hd
        if self.bits == 16:
            return self.k[b, :, o].astype(np.float64), self.v[b, :, :, o].astype(np.float64)
        g = np.arange(hd // 32) * 16 + o
        two = lambda c: np.stack((c & 15, c >> 4), axis=-1).reshape(self.nkv, hd)      # noqa: E731
        return (decode4(two(self.kc[b, :, o * (hd // 2):(o + 1) * (hd // 2)]), self.ks[b][:, g]),
                decode4(two(self.vc[b][:, self._value_at(o)]), self.vs[b][:, g]))


def norm_rope(x, gain, eps, table, positions):
    """x [T][heads][hd] fp64; table [rows][hd/2][2]."""
    if gain is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * gain
    c, s = table[positions, :, 0][:, None].astype(np.float64), table[positions, :, 1][:, None].astype(np.float64)
    a, b = np.split(x, 2, axis=-1)
    return np.concatenate((a * c - b * s, b * c + a * s), axis=-1)


def visible(p, window, sinks):
    """The positions that a query at position p sees."""
    j = np.arange(max(0, p + 1))
    return j[(j > p - window) | (j < sinks)] if window else j


def attention(q, cache, tables, lens, cu, window=0, sinks=0, scale=1.0):
    """q [T][nq][hd] fp64. Returns (out, spread): spread[t][h][d] = sum p |v|, the scale of rounding errors; rows of no sequence NaN."""
    T, nq, hd = q.shape
    G = nq // cache.nkv
    out, spread = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for s in range(len(lens)):
        n = cu[s + 1] - cu[s]
        kv = {}
        for t in range(n):
            js = visible(int(lens[s]) - n + t, window, sinks)
            js = [j for j in js if 0 <= tables[s][j // 16] < cache.n_blocks]
            o = out[cu[s] + t], spread[cu[s] + t]
            if not js:
                o[0][:], o[1][:] = 0, 0
                continue
            for j in js:
                if j not in kv:
                    kv[j] = cache.get(int(tables[s][j // 16]) * 16 + j % 16)
            K, V = np.stack([kv[j][0] for j in js]), np.stack([kv[j][1] for j in js])
            for h in range(nq):
                with np.errstate(invalid="ignore"):
                    x = K[:, h // G] @ q[cu[s] + t, h] * scale
                    p = np.exp(x - x.max())
                    p /= p.sum()
                    o[0][h] = (p[:, None] * V[:, h // G]).sum(axis=0)
                    o[1][h] = (p[:, None] * np.abs(V[:, h // G])).sum(axis=0)
    return out, spread
