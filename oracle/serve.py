"""Serving operators around the hot path (oracle; TEST INFRASTRUCTURE ONLY).

Dense attention of packed prompts, the 4-bit cache's format and the log
probabilities of a row of logits, written from their definitions in float64.
"""
import numpy as np

BLOCK = 32
# E2M1 (two exponent bits, one mantissa bit, no infinities): the codes 0..7
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def packed_attention(Q, K, V, cu, scale, causal=True):
    """Q [Hq, T, D], K, V [Hkv, T, D] -> [Hq, T, D]: each token's softmax over the
    tokens of its own sequence up to itself (or all of them); zeros outside."""
    Hq, T, D = Q.shape
    G = Hq // K.shape[0]
    out = np.zeros((Hq, T, D))
    for a, b in zip(cu[:-1], cu[1:]):
        for h in range(Hq):
            s = np.asarray(Q[h, a:b], np.float64) @ np.asarray(K[h // G, a:b], np.float64).T * scale
            for i in range(b - a):
                n = i + 1 if causal else b - a
                w = np.exp(s[i, :n] - s[i, :n].max())
                out[h, a + i] = w @ np.asarray(V[h // G, a:a + n], np.float64) / w.sum()
    return out


def quantise(x):
    """Codes (0..15, one per value) and scale bytes of x [.., D].

    A block of 32 dimensions shares 2^e, e the least integer in [-124, 125] with
    no magnitude above 7 * 2^e; magnitudes go to the nearest E2M1 value of
    x / 2^e, halfway to the even code, above 6 to 6.  Byte e + 127; 255 and codes 0
    where the block holds a NaN or an infinity."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], -1, BLOCK)
    codes = np.zeros(b.shape, np.uint8)
    scales = np.zeros(b.shape[:-1], np.uint8)
    for i in np.ndindex(scales.shape):
        if not np.isfinite(b[i]).all():
            scales[i] = 255
            continue
        e = -124
        while e < 125 and np.abs(b[i]).max() > 7 * 2.0**e:
            e += 1
        scales[i] = e + 127
        gap = np.abs(np.minimum(np.abs(b[i]) / 2.0**e, 6.0)[:, None] - E2M1)
        tie = gap == gap.min(1, keepdims=True)
        even = tie & (np.arange(8) % 2 == 0)
        codes[i] = np.where(tie.sum(1) > 1, even.argmax(1), tie.argmax(1)) + 8 * np.signbit(b[i])
    return codes.reshape(x.shape), scales


def values(codes, scales):
    """The values of codes [.., D] under scale bytes [.., D / 32]."""
    v = np.where(codes >= 8, -1.0, 1.0) * E2M1[codes & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, BLOCK, axis=-1)


def pack(codes):
    """Two codes a byte, the even dimension in the low half."""
    return codes[..., 0::2] | codes[..., 1::2] << 4


def unpack(b):
    return np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], -1)


def logprobs(x, targets, top_k):
    """log p of targets [n] (negative: 0; past the end: NaN), entropy, and the top_k
    (ids, log p) of one row of logits x [V]."""
    x = np.asarray(x, np.float64)
    ids = np.full(top_k, -1, np.int64)
    top = np.full(top_k, -np.inf)
    order = np.lexsort((np.arange(len(x)), -np.where(np.isnan(x), np.inf, x), ~np.isnan(x)))
    order = order[~(x[order] == -np.inf)][:top_k]
    if (x == -np.inf).all():
        y, ent = x, 0.0
    else:
        with np.errstate(invalid="ignore", divide="ignore"):
            y = x - x.max()
            y = y - np.log(np.exp(y).sum())
            p = np.exp(y)
            ent = -np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, y)).sum()
    ids[:len(order)] = order
    top[:len(order)] = y[order]
    lp = np.array([0.0 if t < 0 else np.nan if t >= len(x) else y[t] for t in targets])
    return lp, ent, ids, top
