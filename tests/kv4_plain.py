"""The cache in 4 bits and attention over it in plain numpy, 64 bits, one definition after the other (include/fvar.h)."""
import numpy as np

GROUP = 32
SCALES = np.array([(8 + c % 8) * 2.0 ** (c // 8 - 23) for c in range(256)])


def quantise(x):
    """x [..., D] -> (numbers u [..., D] in 1..15, scale bytes [..., D / 32])."""
    g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (-1, GROUP))
    g = np.where(np.isnan(g), 0.0, g)
    top = np.abs(g).max(-1)
    byte = np.minimum(np.searchsorted(7.5 * SCALES, top), 255)          # the first scale that is large enough
    q = np.minimum(np.floor(np.abs(g) / SCALES[byte][..., None] + 0.5), 7.0)
    return (8 + np.sign(g) * q).astype(np.uint8).reshape(x.shape), byte.astype(np.uint8)


def values(u, byte):
    g = u.astype(np.float64).reshape(byte.shape + (GROUP,)) - 8.0
    return (g * SCALES[byte][..., None]).reshape(u.shape)


def pack(u):
    """u [..., D] -> codes [..., D / 2]."""
    w = u.astype(np.uint32).reshape(u.shape[:-1] + (-1, 8))
    word = sum(w[..., j] << np.uint32(4 * (j // 2) + 16 * (j % 2)) for j in range(8)).astype("<u4")
    return np.ascontiguousarray(word).view(np.uint8).reshape(u.shape[:-1] + (-1,))


def unpack(codes):
    word = np.ascontiguousarray(codes).view("<u4")
    return np.stack([(word >> np.uint32(4 * (j // 2) + 16 * (j % 2))) & 15 for j in range(8)], -1).reshape(codes.shape[:-1] + (-1,)).astype(np.uint8)


def attention(q, K, V, L, limits=None):
    """q [B][r][H * D], K, V [B][Hkv][>= L][D] -> (result [B][r][H * D], (sum of weight x |value|, sum of weight x 16 steps), bound of a
    score's error [B][r][H]).

    A score is a sum of D products in fp32 of queries with the numbers u of the cache, 0 to 15, less 8 times the sum of the
    queries, times the groups' scales s: every term is at most 16 s |q|, and 16 s <= 16 / 7 of the group's greatest value (which is 7 s).
    (D + 8) steps of 2^-23 of the sum of these, where a sum may be cut instead of rounded; the sums of the queries are taken in 24 bits."""
    B, r, _ = q.shape
    Hkv, D = K.shape[1], K.shape[3]
    H = q.shape[2] // D
    out, mag, wide, err = np.zeros((B, r, H, D)), np.zeros((B, r, H, D)), np.zeros((B, r, H, D)), np.zeros((B, r, H))
    for b in range(B):
        n = np.full(r, L) if limits is None else np.clip(limits[b], 0, L)
        for h in range(H):
            k, v = K[b, h // (H // Hkv), :L], V[b, h // (H // Hkv), :L]
            x = q[b, :, h * D : (h + 1) * D]
            s = x @ k.T / np.sqrt(D)
            s[np.arange(L)[None, :] >= n[:, None]] = -np.inf
            some = n > 0
            w = np.zeros_like(s)
            w[some] = np.exp(s[some] - s[some].max(-1, keepdims=True))
            w[some] /= w[some].sum(-1, keepdims=True)
            out[b, :, h], mag[b, :, h] = w @ v, w @ np.abs(v)
            if L:
                steps = [np.repeat(np.abs(y).reshape(L, -1, GROUP).max(-1), GROUP, -1) * (16.0 / 7.0) for y in (k, v)]
                wide[b, :, h] = w @ steps[1]
                err[b, :, h] = (D + 8) * 2.0 ** -23 * (np.abs(x) @ steps[0].T).max(-1) / np.sqrt(D)
    return out.reshape(B, r, H * D), (mag.reshape(B, r, H * D), wide.reshape(B, r, H * D)), err


def bound(out, mags, err, L, D):
    """How far a bf16 result of the kernels may be off.  With A = sum of weight x |value|: each weight is rounded to bf16 once
    (2^-8 of A), for few rows once more after its product with a group's scale, and the result once (2^-8 of it).  A score is off by err, then
    comes one product with log2(e) / sqrt(D), one subtraction of the maximum (2^-23 of the scores each, within twice err) and an exp2 of
    2^-22: every weight off by a factor within 1 +- (2 err + 2^-21), and the sum of the weights too.  The weighted sum itself is the difference
    of two sums of terms of at most 16 steps, in L / 8 + 64 steps (keys come eight or more at a time, and ranges of keys are joined)."""
    mag, wide = mags
    e = np.repeat(err, mag.shape[-1] // err.shape[-1], -1)
    off = (2 * 2.0 ** -8 + 2.0 ** -16 + 2 * (2 * e + 2.0 ** -21)) * mag + 2 * (L / 8 + 64) * 2.0 ** -23 * wide
    return off + 2.0 ** -8 * (np.abs(out) + off) + 1e-30
