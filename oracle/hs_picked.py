"""Plain numpy forms, in 64 bits, of the operators that pick tiles for each query: bounds of the keys, scores, the choice, and attention over
listed tiles.  Test infrastructure; shares no code with the HIP path."""
import numpy as np

TILE = 64


def tile_bounds(K_bits, held):
    """K_bits uint16 [B, Hkv, L, D] (zeros where pruned), held bool [B, Hkv, T].  Bit patterns [B, Hkv, T, 2, D] of the smallest and largest, by
    sign and magnitude; zeros where not held."""
    B, H, L, D = K_bits.shape
    x = K_bits.reshape(B, H, L // TILE, TILE, D).astype(np.int64)
    # place of a pattern on one line: -NaN .. -0 are -0x8000 .. -1 (the larger the magnitude the lower), +0 .. +NaN 0 .. 0x7fff
    line = np.where(x >= 0x8000, 0x7fff - x, x)
    both = np.stack([line.min(3), line.max(3)], axis=3)
    bits = np.where(both < 0, 0x7fff - both, both)
    return np.where(held[..., None, None], bits, 0).astype(np.uint16)


def query_scores(Q, low, high, held, positions=None):
    """Q [B, Hq, Lq, D], low, high [B, Hkv, T, D] float64.  Scores [B, Hkv, Lq, T] and the sum of the magnitudes that the largest is made of (the
    largest such sum of the heads)."""
    B, Hq, Lq, D = Q.shape
    H, T = low.shape[1], low.shape[2]
    G = Hq // H
    out, size = np.full((B, H, Lq, T), -np.inf), np.zeros((B, H, Lq, T))
    with np.errstate(invalid="ignore"):
        for b in range(B):
            for hq in range(Hq):
                h = hq // G
                for i in range(Lq):
                    q = Q[b, hq, i]
                    terms = np.maximum(q, 0.0) * high[b, h] + np.minimum(q, 0.0) * low[b, h]
                    s = terms.sum(-1)
                    s = np.where(np.isnan(s), np.inf, s)
                    out[b, h, i] = np.maximum(out[b, h, i], s)
                    size[b, h, i] = np.maximum(size[b, h, i], np.abs(terms).sum(-1))
    open_ = np.broadcast_to(held[:, :, None, :], out.shape).copy()
    if positions is not None:
        open_ &= np.arange(T)[None, :] * TILE <= np.asarray(positions)[:, None]
    return np.where(open_, out, -np.inf), size


def pick_tiles(scores, n, first, last):
    """scores float32 [..., T] -> int32 [..., n]."""
    flat = scores.reshape(-1, scores.shape[-1])
    out = np.full((flat.shape[0], n), -1, dtype=np.int32)
    for r, s in enumerate(flat):
        s = [np.inf if x != x else float(x) for x in s]
        there = [t for t, x in enumerate(s) if x > -np.inf]
        ends = set(there[:first]) | set(there[max(0, len(there) - last):] if last else [])
        rest = sorted((t for t in there if t not in ends), key=lambda t: (-s[t], t))
        take = sorted(sorted(ends) + rest[:max(0, n - len(ends))])
        out[r, :len(take)] = take
    return out.reshape(scores.shape[:-1] + (n,))


def listed_attention(Q, K, V, lists, held, scale, positions=None, tail_k=None, tail_v=None, tail_lens=None, weight=2.0 ** -16):
    """Q [B, Hq, Lq, D], K, V [B, Hkv, L, D] float64, lists int [B, Hkv, Lq, n].  Returns O, LSE and for each a bound on its error in the arithmetic of a
    matrix product with 32-bit sums: a score is a sum of D exact products, off by at most D steps of 2^-24 of the sum of their
    magnitudes (twice that where sums are cut, not rounded); scale and exponent each by 2^-24 of the argument; an exponential by 2^-22; a weight that
    multiplies a value by `weight` (two terms of 8 bits or more: 2^-16; one of 11 bits, half a step of fp16: 2^-11); each sum of n terms by n 2^-24, and by as much again where parts are joined."""
    B, Hq, Lq, D = Q.shape
    H, T = K.shape[1], K.shape[2] // TILE
    G = Hq // H
    O, LSE = np.zeros((B, Hq, Lq, D)), np.full((B, Hq, Lq), -np.inf)
    o_tol, l_tol = np.zeros((B, Hq, Lq, D)), np.zeros((B, Hq, Lq))
    e = 2.0 ** -24
    for b in range(B):
        for h in range(H):
            for i in range(Lq):
                tiles = sorted({int(t) for t in lists[b, h, i] if 0 <= t < T and held[b, h, t]})
                tokens = np.array([64 * t + j for t in tiles for j in range(64) if positions is None or 64 * t + j <= positions[i]], dtype=np.int64)
                k, v = K[b, h, tokens], V[b, h, tokens]
                if tail_k is not None:
                    m = min(max(int(tail_lens[b]), 0), 64)
                    k, v = np.concatenate([k, tail_k[b, h, :m]]), np.concatenate([v, tail_v[b, h, :m]])
                if len(k) == 0:
                    continue
                for g in range(h * G, (h + 1) * G):
                    q = Q[b, g, i]
                    s = scale * (k @ q)
                    m = s.max()
                    p = np.exp(s - m)
                    O[b, g, i], LSE[b, g, i] = p @ v / p.sum(), m + np.log(p.sum())
                    off = scale * 2 * D * e * (np.abs(k) @ np.abs(q)).max() + 4 * e * np.abs(s).max() * 1.5
                    size = p @ np.abs(v) / p.sum()
                    o_tol[b, g, i] = size * (2 * off + weight + 2.0 ** -21 + 4 * len(k) * e)
                    l_tol[b, g, i] = off + 2.0 ** -21 + 4 * e * abs(LSE[b, g, i]) + 4 * len(k) * e
    return O, LSE, o_tol, l_tol
