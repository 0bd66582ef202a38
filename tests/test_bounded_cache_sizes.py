"""The operators around a bounded cache at the sizes where another kernel or another share of the work is chosen: held tiles numbered by the workgroups
(attention mass), rows in parts of every length (choice of tokens), counts near what a launch holds.  Plain forms in 64 bits on the device."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2604_16864_amd import binding as hb

gpu = pytest.mark.gpu
D, TILE = 128, 64
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _bits(t):
    return t.detach().contiguous().view(torch.int16)


# ---------------------------------------------------------------------------------------------------------------------
# attention mass of many queries where tiles may be missing
# ---------------------------------------------------------------------------------------------------------------------
def _states(kinds, B, Hkv, T, g):
    """Tile states: row 0 holds nothing, row 1 one tile, row 2 (or the last) all of them, the others a number that is no multiple of 4."""
    s = torch.zeros((B * Hkv, T), dtype=torch.int8)
    for r in range(B * Hkv):
        n = {0: 0, 1: 1, 2: T}.get(r, max(1, (2 * T // 5) // 4 * 4 + 1 + r % 3)) if B * Hkv > 2 else (T // 4 // 4 * 4 + 3, T)[r]
        at = torch.randperm(T, generator=g)[:min(n, T)]
        s[r, at] = torch.tensor(kinds, dtype=torch.int8)[torch.randint(0, len(kinds), (len(at),), generator=g)]
    s = s.reshape(B, Hkv, T).numpy()
    v = np.where(s == hb.SKIP, hb.SKIP, hb.SPARSE24).astype(np.int8)
    return s, v


def _mass_64(Q, K, lse, held, causal, q_start):
    """What each token gets [B, Hkv, L], and the error of the scores' way there: a score is a sum of D exact products (D + 1 roundings of
    the sum of magnitudes at most), the argument of the exponential is off by 4 2^-24 of each of its two parts, an exponential by 4 2^-24."""
    B, Hq, Lq, _ = Q.shape
    Hkv, L = K.shape[1], K.shape[2]
    G, e, scale = Hq // Hkv, 2.0 ** -24, 1 / math.sqrt(D)
    out, tol = (torch.zeros((B, Hkv, L), dtype=torch.float64, device="cuda") for _ in range(2))
    at = torch.arange(L, device="cuda")
    for b in range(B):
        for hq in range(Hq):
            h = hq // G
            seen_tile = held[b, h].repeat_interleave(TILE)
            for i in range(0, Lq, 512):
                q, ls = Q[b, hq, i:i + 512].double(), lse[b, hq, i:i + 512].double()[:, None]
                s = torch.matmul(q, K[b, h].double().t()) * scale
                size = torch.matmul(q.abs(), K[b, h].double().abs().t()) * scale
                seen = seen_tile & torch.isfinite(ls)
                if causal:
                    seen = seen & (at <= q_start + i + torch.arange(len(q), device="cuda")[:, None])
                p = torch.where(seen, torch.exp(s - ls), 0.0)
                out[b, h] += p.sum(0)
                tol[b, h] += torch.where(seen, p * ((D + 1) * e * size + 4 * e * (s.abs() + ls.abs()) + 4 * e), 0.0).sum(0)
    return out, tol


@gpu
@pytest.mark.parametrize("kinds", [(hb.SPARSE24,), (hb.DENSE,), (hb.DENSE, hb.SPARSE24)], ids=["2:4", "dense", "mixed"])
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("B,Hkv,G,T,Lq,causal,ranges", [
    (2, 2, 4, 601, 60, True, 1),        # 604 workgroups, a row's last group of one tile
    (1, 1, 3, 2051, 77, False, 1),      # 513, and more tiles than one walk over the map looks at; 32 columns are 10 queries and 2 to spare
    (1, 2, 8, 2050, 31, True, 1),       # a second walk of two tiles
    (2, 2, 4, 21, 1300, True, 22),      # 528 in ranges of 7 blocks, queries before the first tile's end
    (1, 3, 1, 130, 2000, False, 6),     # 594 in ranges of 10 blocks of 32 queries of one head
    (4, 1, 4, 299, 4000, True, 28),     # 8400 in ranges of 17 blocks
])
def test_mass_where_held_tiles_are_numbered(B, Hkv, G, T, Lq, causal, ranges, dtype, kinds):
    """Calls of more than 512 workgroups, in one range of the queries and in several: rows that hold nothing, one tile, some and all; every element of
    the output and of the workspace is written, missing tiles get what they had."""
    L, t = T * TILE, TYPES[dtype]
    sh = hb.make_shape(B, Hkv * G, Hkv, L, dtype=t)
    g, gd = torch.Generator().manual_seed(T + Lq), torch.Generator(device="cuda").manual_seed(T + Lq)
    s, v = _states(kinds, B, Hkv, T, g)
    K = torch.randn((B, Hkv, L, D), generator=gd, device="cuda").to(t)
    kv = hb.compress_kv(sh, hb.make_policy(state_k=s, state_v=v), K, K)
    assert not kv.uniform
    held = kv.k_map != 0
    assert torch.equal(held.cpu(), torch.from_numpy(s != hb.SKIP))
    Ku, _ = hb.unpack_kv(sh, kv)
    Q = torch.randn((B, Hkv * G, Lq, D), generator=gd, device="cuda").to(t)
    lse = torch.randn((B, Hkv * G, Lq), generator=gd, device="cuda") + math.log(L)
    lse[:, :, Lq // 3] = -math.inf                       # queries that do not count, one in every head
    q_start = L - Lq
    if not causal:
        q_start = 0
    elif Lq > TILE:
        q_start = min(q_start, 40)                       # what lies behind the last query is seen by none
    want, tol = _mass_64(Q, Ku, lse, held, causal, q_start)
    for per_token in (False, True):
        need = hb.attn_mass_workspace_bytes(sh, Lq, causal, per_token)
        sizes = (B, Hkv, L if per_token else T)
        out_bytes = 4 * B * Hkv * sizes[2]
        n_ranges = max(1, need // out_bytes)
        # tokens: as many as 64 MiB hold
        assert n_ranges == min(ranges, max(1, (64 << 20) // out_bytes)) and n_ranges * B * Hkv * ((T + 3) // 4) > 512
        w, e = (want, tol) if per_token else (x.reshape(B, Hkv, T, TILE).sum(-1) for x in (want, tol))
        # terms of a sum are added to it one after the other a block of queries and a range of them at a time, before that and after it by at most 20 more
        depth = (Lq + 32 // G - 1) // (32 // G) + 20
        e = e + depth * 2.0 ** -24 * w
        before = torch.rand(sizes, generator=gd, device="cuda")
        ws = torch.full((max(16, need),), 0xff, dtype=torch.uint8, device="cuda")          # NaN
        for decay in (0.0, 0.75):
            got = hb.attn_mass(sh, Q, lse, kv, mass=before, out=torch.full_like(before, math.nan), per_token=per_token, causal=causal, q_start=q_start,
                               decay=decay, workspace=ws.clone())
            full = w + decay * before.double()
            err = (got.double() - full).abs()
            assert bool((err <= e + 2 * 2.0 ** -24 * (full + decay * before.double()) + 1e-37).all()), (per_token, decay, float(err.max()))
            old = torch.zeros_like(before) if decay == 0.0 else before * decay
            gone = ~(held if not per_token else held.repeat_interleave(TILE, -1))
            assert torch.equal(got[gone], old[gone])
        mine = before.clone()
        assert hb.attn_mass(sh, Q, lse, kv, mass=mine, per_token=per_token, causal=causal, q_start=q_start, decay=0.75) is mine
        assert torch.equal(mine, got)


# ---------------------------------------------------------------------------------------------------------------------
# choice of tokens: rows in parts of every length
# ---------------------------------------------------------------------------------------------------------------------
def _kept(w, keep, first, last):
    """Tokens of one row that are kept, ascending (numpy, no NaN; the lower token first among equals)."""
    n = len(w)
    if n <= keep:
        return np.arange(n)
    rest = first + np.argsort(-w[first:n - last], kind="stable")[:keep - first - last]
    return np.concatenate([np.arange(first), np.sort(rest), np.arange(n - last, n)])


@gpu
@pytest.mark.parametrize("kind", ["spread", "alike", "one bin"])
@pytest.mark.parametrize("B,Hkv,n,ragged", [
    (1, 1, 400000, False),     # 64 parts of 6400 tokens
    (5, 4, 70003, True),       # 51 parts of 1536
    (2, 9, 9001, True),        # 9 parts of 1024
    (8, 8, 131071, False),     # 16 parts of 8192
    (8, 8, 262144, True),      # 16 parts of 16384: the most that a part counts, and its keys are read again in every pass
    (2, 2, 262145, False),     # 64 parts of 4352
])
def test_keep_tokens_in_parts_of_every_length(B, Hkv, n, ragged, kind):
    sh = hb.make_shape(B, Hkv, Hkv, TILE)
    g = torch.Generator(device="cuda").manual_seed(n)
    K = torch.randn((1, 1, n, D), generator=g, device="cuda").bfloat16().expand(B, Hkv, n, D)      # heads share their vectors
    x = torch.rand((B, Hkv, n), generator=g, device="cuda")
    w = {"spread": torch.exp(3.0 * x - 9.0), "alike": torch.full_like(x, 0.25), "one bin": 1.0 + x / 8}[kind]
    lens = [n - 7919 * b if b % 3 else n for b in range(B)] if ragged else [n] * B
    lens = [max(1, m) for m in lens]
    wn = w.cpu().numpy()
    for keep, first, last in ((n // 16, 4, 32), (n - n // 3, 0, 1)):
        ko, vo, index = hb.keep_tokens(sh, K, K, w, keep, first=first, last=last, lens=torch.tensor(lens, dtype=torch.int32, device="cuda") if ragged else None)
        got = index.cpu().numpy()
        for b in range(B):
            for h in range(Hkv):
                t = _kept(wn[b, h, :lens[b]], keep, first, last)
                assert (got[b, h, :len(t)] == t).all() and (got[b, h, len(t):] == -1).all(), (keep, b, h)
        for b, h in ((0, 0), (B - 1, Hkv - 1)):
            i = index[b, h].long()
            there = (i >= 0)[:, None]
            want = torch.where(there, _bits(K[b, h])[i.clamp(min=0)], 0)
            assert torch.equal(_bits(ko[b, h]), want) and torch.equal(_bits(vo[b, h]), want)
        del ko, vo, index


# ---------------------------------------------------------------------------------------------------------------------
# counts near what a launch holds
# ---------------------------------------------------------------------------------------------------------------------
@gpu
def test_rope_of_more_tokens_than_four_a_workgroup_hold():
    """2^26 tokens and more (17 GB of queries of one head): a grid of 4 tokens a workgroup would have 2^32 threads.  All tokens are the same vector."""
    n = (1 << 26) + 1005
    sh, rope = hb.make_shape(1, 1, 1, TILE), hb.make_rope()
    x = torch.randn((1, 1, 1, D), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").bfloat16()
    out = torch.empty((1, 1, n, D), dtype=torch.bfloat16, device="cuda")
    hb.rope_qkv(sh, rope, q=x.expand(1, n, 1, D), positions=-9, q_out=out)
    for first in (0, (1 << 25) - 1000, (1 << 26) - 1000, n - 2000):
        part, _, _ = hb.rope_qkv(sh, rope, q=x.expand(1, 2000, 1, D), positions=first - 9)
        assert torch.equal(_bits(out[:, :, first:first + 2000]), _bits(part)), first


def _one(token=D):
    return C.byref(hb.HsView(4096, 0, D, token))


def test_rope_refuses_more_tokens_than_a_launch_holds():
    """(Addresses here are never read.)"""
    rope = hb.make_rope()
    for B, n in ((1, (1 << 29) - 31), (2, 1 << 28), (1, 2 ** 31 - 1)):
        sh = hb.make_shape(B, 1, 1, TILE)
        out = C.byref(hb.HsView(4096, D, D, D))
        assert hb.lib().hs_rope_qkv(C.byref(sh), C.byref(rope), n, None, 0, _one(0), out, None, None, None, None, None, 0, 0, None) == -2, (B, n)


def test_keep_tokens_refuses_more_rows_than_a_launch_holds():
    """(Addresses here are never read.)"""
    sh = hb.make_shape(1, 2, 2, TILE)
    K = C.byref(hb.HsView(4096, 0, 100 * D, D))
    for keep in ((1 << 28) - 15, 1 << 28, 1 << 30):
        assert hb.lib().hs_keep_tokens(C.byref(sh), 100, K, K, 4096, None, None, keep, 0, 0, 4096, 4096, 4096, 4096, None) == -2, keep


def test_mass_refuses_more_tiles_than_a_launch_holds():
    """Caches of positions for 2^26 tiles in a batch row's kv heads, nearly all of them missing.  (Addresses here are never read.)"""
    kv = C.byref(hb.HsKV(k_map=4096, v_map=4096))
    for Hkv, L, Lq, causal in ((8, 1 << 29, 8, 1), (64, 1 << 26, 1, 1), (3, 2 ** 31 - 64, 200, 0)):
        sh = hb.make_shape(1, Hkv, Hkv, L)
        Q = C.byref(hb.HsView(4096, 0, 1024 * D, D))
        assert hb.lib().hs_attn_mass(C.byref(sh), Lq, 0, 0.0, causal, Q, 4096, None, kv, None, 0, None, 0, None, 0, 1.0, None, 4096, 4096, None) == -2, (Hkv, L)


def test_binding_refuses_numbers_that_are_no_int32():
    """Numbers whose lower 32 bits would be another call's: refused before the tensors are looked at."""
    sh, rope = hb.make_shape(1, 4, 2, 128), hb.make_rope()
    q, k = torch.zeros((1, 3, 4, D), dtype=torch.bfloat16), torch.zeros((1, 3, 2, D), dtype=torch.bfloat16)
    kv, Q, lse, mass = hb.PackedKV(sh, [0, 0, 2, 0, 2], "cpu"), q.transpose(1, 2), torch.zeros(1, 4, 3), torch.zeros(1, 2, 2)
    tail, one, one_lse = torch.zeros((1, 2, TILE, D), dtype=torch.bfloat16), torch.zeros((1, 4, D), dtype=torch.bfloat16), torch.zeros(1, 4)
    K, w = k.transpose(1, 2), torch.zeros(1, 2, 3)
    for big in ((1 << 32) + 1, 1 << 31, -(1 << 31) - 1):
        for call in (lambda: hb.make_rope(rot_dim=big), lambda: hb.make_rope(trained=big), lambda: hb.rope_qkv(sh, rope, q, positions=big),
                     lambda: hb.rope_qkv(sh, rope, None, k, rows=big), lambda: hb.attn_mass(sh, Q, lse, kv, q_start=big),
                     lambda: hb.attn_mass(sh, one, one_lse, kv, tail_k=tail, tail_len=big, tail_tile=0), lambda: hb.attn_mass(sh, one, one_lse, kv, tail_k=tail, tail_len=1, tail_tile=big),
                     lambda: hb.attn_mass_workspace_bytes(sh, big), lambda: hb.evict_tiles(sh, kv, mass, big), lambda: hb.evict_tiles(sh, kv, mass, 1, first=big),
                     lambda: hb.evict_tiles(sh, kv, mass, 1, last=big), lambda: hb.keep_tokens(sh, K, K, w, big), lambda: hb.keep_tokens(sh, K, K, w, 2, first=big),
                     lambda: hb.keep_tokens(sh, K, K, w, 2, last=big), lambda: hb.rope_qkv(sh, rope, q[:, :1].expand(1, (1 << 31) + 5, 4, D))):
            with pytest.raises(hb.HsError, match="32-bit"):
                call()


# ---------------------------------------------------------------------------------------------------------------------
# evicted caches of many tiles, captured calls of long rows
# ---------------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("sk,sv,B,Hkv,T,keep", [(1.0, 1.0, 1, 8, 1024, 300), (0.5, 1.0, 2, 4, 512, 130), (0.97, 0.5, 1, 2, 2500, 2000), (1.0, 1.0, 16, 8, 40, 7)])
def test_attention_over_a_large_cache_after_eviction(sk, sv, B, Hkv, T, keep):
    """Slots in no order, pools that say nothing is skipped: decode (tiles by range and by count, with a tail and without) and prefill give the bits of a cache
    into which only the remaining tiles were packed, in order, with pools of the same sizes."""
    G, L = 4, T * TILE
    gd = torch.Generator(device="cuda").manual_seed(T)
    K, V = (torch.randn((B, Hkv, L, D), generator=gd, device="cuda").bfloat16() for _ in range(2))
    sh = hb.make_shape(B, Hkv * G, Hkv, L)
    kv = hb.compress_kv(sh, hb.make_policy(sparse_frac_k=sk, sparse_frac_v=sv), K, V)
    states = [np.where(m > 0, hb.DENSE, hb.SPARSE24).astype(np.int8) for m in (kv.k_map.cpu().numpy(), kv.v_map.cpu().numpy())]
    hb.evict_tiles(sh, kv, torch.rand((B, Hkv, T), generator=gd, device="cuda"), keep, first=1, last=4)
    gone = (kv.k_map == 0).cpu().numpy()
    assert (gone.sum(-1) == T - keep).all()
    slots = kv.k_map[0, 0].cpu().numpy()
    slots = -slots[slots < 0]
    assert (np.sort(slots) == np.arange(1, len(slots) + 1)).all() and (np.diff(slots) < 0).any()
    for s in states:
        s[gone] = hb.SKIP
    fresh = hb.PackedKV(sh, kv.counts, "cuda")
    pol = hb.make_policy(state_k=states[0], state_v=states[1])
    hb.compress_kv(sh, pol, K, V, out=fresh)
    hb.check_state_flag(pol)
    Q = torch.randn((B, Hkv * G, 192, D), generator=gd, device="cuda").bfloat16()
    tk, tv = (torch.randn((B, Hkv, TILE, D), generator=gd, device="cuda").bfloat16() for _ in range(2))
    for Lq in (64, 192):
        for a, b in zip(hb.prefill_attn(sh, Q[:, :, :Lq].contiguous(), kv), hb.prefill_attn(sh, Q[:, :, :Lq].contiguous(), fresh)):
            assert torch.equal(a, b)
    q = Q[:, :, 0].contiguous()
    for extra in (dict(), dict(tail_k=tk, tail_v=tv, tail_len=33)):
        for a, b in zip(hb.decode_attn(sh, q, kv, **extra), hb.decode_attn(sh, q, fresh, **extra)):
            assert torch.equal(a, b)
    lse = torch.full((B, Hkv * G, 192), math.log(keep * TILE), device="cuda")
    for per_token in (False, True):
        assert torch.equal(hb.attn_mass(sh, Q, lse, kv, per_token=per_token), hb.attn_mass(sh, Q, lse, fresh, per_token=per_token))


@gpu
def test_captured_calls_of_long_rows_replay():
    """Rows in parts, held tiles numbered in several ranges, many tiles dropped: captured once, replayed with other inputs, eager work between the replays."""
    B, Hkv, G, T, n, Lq = 2, 2, 4, 150, 30000, 1000
    L = T * TILE
    gd = torch.Generator(device="cuda").manual_seed(3)
    sh = hb.make_shape(B, Hkv * G, Hkv, L)
    K = torch.randn((B, Hkv, n, D), generator=gd, device="cuda").bfloat16()
    kv = hb.compress_kv(sh, hb.make_policy(sparse_frac_k=0.5), K[:, :, :L], K[:, :, L:2 * L])
    kv.uniform = 0
    Q, lse = torch.empty((B, Hkv * G, Lq, D), dtype=torch.bfloat16, device="cuda"), torch.empty((B, Hkv * G, Lq), device="cuda")
    w, mass = torch.empty((B, Hkv, n), device="cuda"), torch.empty((B, Hkv, T), device="cuda")
    bufs = [t for t in (kv.k_dense, kv.k_nnz, kv.k_meta, kv.k_map, kv.v_dense, kv.v_nnz, kv.v_meta, kv.v_map) if t is not None]
    backup = [t.clone() for t in bufs]
    assert hb.attn_mass_workspace_bytes(sh, Lq) > mass.nbytes

    def fill():
        Q.normal_(generator=gd), lse.uniform_(8.0, 10.0, generator=gd), w.exponential_(generator=gd), mass.uniform_(generator=gd)
        for t, b in zip(bufs, backup):
            t.copy_(b)

    def calls():
        hb.attn_mass(sh, Q, lse, kv, mass=mass, decay=0.5)
        kept = hb.keep_tokens(sh, K, K, w, 2000, first=4, last=32)
        hb.evict_tiles(sh, kv, mass, 60, first=1, last=2)
        return [mass, *kept, *bufs]

    fill()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    fill()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for _ in range(4):
        fill()
        before = mass.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        mass.copy_(before)
        for t, b in zip(bufs, backup):
            t.copy_(b)
        for a, b in zip(got, calls()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()
