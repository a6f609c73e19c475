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


def page_places(table, page, pages):
    """Row (page, slot) of every position that a row of the block table names, -1 where
    its entry names no page: [len(table) * page, 2]."""
    j = np.arange(len(table) * page)
    p = np.asarray(table, np.int64)[j // page]
    return np.where(((p >= 0) & (p < pages))[:, None], np.stack([p, j % page], 1), -1)


def paged_attention(Q, Kp, Vp, table, cu, start, window, sink, scale):
    """Q [Hq, T, D], Kp, Vp [pages, Hkv, page, D] -> [Hq, T, D]: the token at position p
    over the positions j <= p with j > p - window or j < sink that have a page; zeros where
    there are none and for tokens whose position has no place."""
    Q, Kp, Vp = (np.asarray(x, np.float64) for x in (Q, Kp, Vp))
    Hq, T, D = Q.shape
    pages, Hkv, page, _ = Kp.shape
    out = np.zeros((Hq, T, D))
    for b, (a, z) in enumerate(zip(cu[:-1], cu[1:])):
        at = page_places(table[b], page, pages)
        for t in range(max(a, 0), min(z, T)):
            p = int(start[b]) + t - max(a, 0)
            if not 0 <= p < len(at):
                continue
            j = np.arange(p + 1)
            j = j[((j > p - window) | (j < sink)) & (at[:p + 1, 0] >= 0)]
            if len(j) == 0:
                continue
            for h in range(Hq):
                g = h // (Hq // Hkv)
                k, v = (x[at[j, 0], g, at[j, 1]] for x in (Kp, Vp))
                with np.errstate(invalid="ignore", over="ignore"):
                    s = k @ Q[h, t] * scale
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    # a weight may be 0 here where it is not in truth
                    fin = np.isfinite(v)
                    out[h, t] = w @ np.where(fin, v, 0.0) + np.where(fin, 0.0, v).sum(0)
    return out


def w4_tiles(codes, scales):
    """Codes [N, K] and scale bytes [N, ceil(K / 32)] in the layout of the 4-bit weights: tiles of
    16 outputs and 128 inputs, element by element."""
    N, K = codes.shape
    n, k = -(-N // 16), -(-K // 128)
    C = np.zeros((n, k, 4, 16, 16), np.uint8)
    S = np.zeros((n, -(-K // 512), 4, 16, 4), np.uint8)
    for r in range(16 * n):
        for i in range(128 * k):
            if r < N and i < K:
                C[r // 16, i // 128, i % 128 // 32, r % 16, i % 32 // 2] |= int(codes[r, i]) << (4 * (i % 2))
            if i % 32 == 0:
                S[r // 16, i // 512, i % 128 // 32, r % 16, i // 128 % 4] = scales[r, i // 32] if r < N and i < K else 3
    return C, S
