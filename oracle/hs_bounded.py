"""Plain numpy forms, in 64 bits, of the operators around a bounded cache: rotary positions, attention mass, eviction of tiles in place
and the choice of tokens.  Test infrastructure; shares no code with the HIP path."""
import math

import numpy as np


def rope_angles(rot_dim, base, scaling="plain", factor=1.0, low=0.0, high=0.0, trained=0):
    """theta of each pair and the gain."""
    i = np.arange(rot_dim // 2, dtype=np.float64)
    theta, gain = base ** (-2.0 * i / rot_dim), 1.0
    if scaling == "linear":
        theta = theta / factor
    elif scaling == "stretch":
        theta = (base * factor ** (rot_dim / (rot_dim - 2.0))) ** (-2.0 * i / rot_dim)
    elif scaling == "bands":
        s = np.clip((trained * theta / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        theta = s * theta + (1 - s) * theta / factor
    elif scaling == "ramp":
        def pair(turns):
            return rot_dim * math.log(trained / (2 * math.pi * turns)) / (2 * math.log(base))
        a = max(0.0, math.floor(pair(high)))
        b = max(min(rot_dim - 1.0, math.ceil(pair(low))), a + 0.001)
        s = 1.0 - np.clip((i - a) / (b - a), 0.0, 1.0)
        theta = s * theta + (1 - s) * theta / factor
        gain = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    return theta, gain


def rope(x, positions, theta, gain, pairs):
    """x [B, n, heads, D] float64, positions [B, n] -> rotated, and the sum of the magnitudes that each output is made of."""
    r = 2 * len(theta)
    a = positions.astype(np.float64)[:, :, None, None] * theta
    c, s = gain * np.cos(a), gain * np.sin(a)
    first = np.arange(0, r, 2) if pairs else np.arange(r // 2)
    second = first + (1 if pairs else r // 2)
    u, v = x[..., first], x[..., second]
    y, size = x.copy(), np.zeros_like(x)
    y[..., first], y[..., second] = u * c - v * s, u * s + v * c
    size[..., first] = size[..., second] = gain * (np.abs(u) + np.abs(v))
    return y, size


def attention_mass(Q, K, lse, held, scale, causal, q_start):
    """Q [B, Hq, Lq, D], K [B, Hkv, L, D] float64 (zeros where pruned), lse [B, Hq, Lq], held [B, Hkv, L / 64].  Returns what each token
    gets [B, Hkv, L] and a bound on its error in 32-bit arithmetic: a score is a sum of D exact products (each of the D additions off by
    at most 2^-24 of the sum of magnitudes), its argument of the exponential is off by at most 2^-24 of each factor and of the result, an
    exponential by 2^-22, a sum of m terms by m 2^-24."""
    B, Hq, Lq, D = Q.shape
    Hkv, L = K.shape[1], K.shape[2]
    G = Hq // Hkv
    out, tol = np.zeros((B, Hkv, L)), np.zeros((B, Hkv, L))
    e = 2.0 ** -24
    at = np.arange(L)
    for b in range(B):
        for h in range(Hkv):
            seen_tile = np.repeat(held[b, h], 64)
            k = np.where(seen_tile[:, None], K[b, h], 0.0)
            for g in range(G):
                q, ls = Q[b, h * G + g], lse[b, h * G + g].astype(np.float64)
                use = np.isfinite(ls)
                q, ls, i = q[use], ls[use], np.arange(Lq)[use]
                seen = np.broadcast_to(seen_tile, (len(i), L)).copy()
                if causal:
                    seen &= at[None, :] <= (q_start + i)[:, None]
                kk = np.where(np.isfinite(k), k, 0.0)      # a key that is not finite is seen by no query that counts
                s = q @ kk.T * scale
                p = np.where(seen, np.exp(np.where(seen, s - ls[:, None], -np.inf)), 0.0)
                size = np.abs(q) @ np.abs(kk).T * scale
                rel = (D + 1) * e * size + 4 * e * (np.abs(s) + np.abs(ls)[:, None]) + 4 * e
                out[b, h] += p.sum(0)
                tol[b, h] += (p * (rel + Lq * G * e)).sum(0)
    return out, tol


def evict(k_map, v_map, mass, keep, first, last, flag=1 << 30):
    """Maps [rows, T] after the eviction, and per row the moves {pool: [(from, to)]}, pools "k_dense", "k_sparse", "v_dense", "v_sparse"."""
    k_map, v_map = k_map.copy(), v_map.copy()
    moves = []
    for r in range(len(k_map)):
        held = [t for t in range(k_map.shape[1]) if k_map[r, t]]
        may = held[first:max(first, len(held) - last)]
        n = len(held) - int(keep[r])

        def rank(t):
            m = float(mass[r, t])
            return (0, 0.0, t) if math.isnan(m) else (1, m, t)

        drop = set(sorted(may, key=rank)[:max(0, n)])
        row = {}
        for name, m in (("k", k_map[r]), ("v", v_map[r])):
            for kind, sign in (("dense", 1), ("sparse", -1)):
                slots = {(abs(int(m[t])) & ~flag) - 1: t for t in held if int(m[t]) * sign > 0}
                left = len([t for t in slots.values() if t not in drop])
                holes = sorted(s for s, t in slots.items() if t in drop and s < left)
                movers = sorted(s for s, t in slots.items() if t not in drop and s >= left)
                assert len(holes) == len(movers)
                row[f"{name}_{kind}"] = list(zip(movers, holes))
                for frm, to in zip(movers, holes):
                    t = slots[frm]
                    m[t] = sign * ((to + 1) | (abs(int(m[t])) & flag))
        for t in drop:
            k_map[r, t] = v_map[r, t] = 0
        moves.append(row)
    return k_map, v_map, moves


def keep_tokens(weight, length, keep, first, last):
    """Indices of the tokens of one row that are kept, ascending."""
    n = min(length, len(weight))
    if n <= keep:
        return list(range(n))

    def rank(t):
        w = float(weight[t])
        return (1, 0.0, t) if math.isnan(w) else (0, -w, t)

    rest = sorted(range(first, n - last), key=rank)[:keep - first - last]
    return sorted(list(range(first)) + rest + list(range(n - last, n)))
