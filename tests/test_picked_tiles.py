"""The operators that pick tiles for each query: bounds of the keys, scores, the choice, attention over listed tiles.  GPU tests hold the library
against oracle/hs_picked.py (64 bits); refusals are looked at on the CPU."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import hs_picked as ref
from paper_2604_16864_amd import binding as hb

gpu = pytest.mark.gpu
D, TILE = 128, 64
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _f64(t):
    return t.detach().double().cpu().numpy()


def _bits(t):
    return t.detach().contiguous().view(torch.int16).cpu()


def _ubits(t):
    return _bits(t).numpy().view(np.uint16)


def _i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


POLICIES = {"2:4": dict(), "dense": dict(sparse_frac_k=0.0, sparse_frac_v=0.0), "dense keys": dict(sparse_frac_k=0.0), "dense values": dict(sparse_frac_v=0.0),
            "half": dict(sparse_frac_k=0.5, sparse_frac_v=0.5), "some": dict(skip_frac=0.3), "some of half": dict(skip_frac=0.4, sparse_frac_k=0.5, sparse_frac_v=0.5)}


def _cache(B, Hq, Hkv, T, dtype, policy, seed, spoil=None):
    """A shape, its packed cache, and the keys and values that it holds, in 64 bits, with what is held."""
    t = TYPES[dtype]
    sh = hb.make_shape(B, Hq, Hkv, T * TILE, dtype=t)
    g = _gen(seed)
    K, V = torch.randn((B, Hkv, T * TILE, D), generator=g).to(t), torch.randn((B, Hkv, T * TILE, D), generator=g).to(t)
    if spoil is not None:
        spoil(K, V)
    kv = hb.compress_kv(sh, hb.make_policy(**POLICIES[policy]) if isinstance(policy, str) else policy, K.cuda(), V.cuda())
    Ku, Vu = hb.unpack_kv(sh, kv)
    return sh, kv, Ku, Vu, (kv.k_map != 0).cpu().numpy()


# ---------------------------------------------------------------------------------------------------------------------
# bounds of the keys
# ---------------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("policy", sorted(POLICIES))
@pytest.mark.parametrize("B,Hkv,T", [(1, 1, 1), (2, 3, 7), (1, 2, 70)])
def test_bounds(B, Hkv, T, policy, dtype):
    sh, kv, K, _, held = _cache(B, Hkv * 2, Hkv, T, dtype, policy, 5 * T + B)
    want = ref.tile_bounds(_ubits(K), held)
    assert (_ubits(hb.tile_bounds(sh, kv)) == want).all()
    # a part of the tiles leaves the others
    out = torch.full((B, Hkv, T, 2, D), 7.0, dtype=TYPES[dtype], device="cuda")
    a, n = T // 3, max(1, T // 2)
    assert hb.tile_bounds(sh, kv, a, n, out=out) is out
    got = _ubits(out)
    assert (got[:, :, a:a + n] == want[:, :, a:a + n]).all()
    rest = torch.cat([out[:, :, :a], out[:, :, a + n:]], dim=2)
    assert bool((rest == 7.0).all())
    assert (_ubits(hb.tile_bounds(sh, kv, a))[:, :, a:] == want[:, :, a:]).all()
    part = _ubits(hb.tile_bounds(sh, kv, a, n))
    assert (part[:, :, a:a + n] == want[:, :, a:a + n]).all() and not part[:, :, :a].any() and not part[:, :, a + n:].any()


@gpu
@pytest.mark.parametrize("policy", ["2:4", "dense", "some of half"])
def test_bounds_of_one_tile_of_each_sequence(policy):
    B, Hkv, T = 5, 2, 9
    sh, kv, K, _, held = _cache(B, 4, Hkv, T, "bf16", policy, 3)
    want = ref.tile_bounds(_ubits(K), held)
    out = torch.full((B, Hkv, T, 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
    tiles = [0, 8, -1, 9, 4]
    hb.tile_bounds(sh, kv, _i32(tiles), out=out)
    for b, t in enumerate(tiles):
        for other in range(T):
            if other == t:
                assert (_ubits(out[b, :, t]) == want[b, :, t]).all(), b
            else:
                assert bool((out[b, :, other] == 7.0).all()), (b, other)
    new = _ubits(hb.tile_bounds(sh, kv, _i32([2, 2, 2, 2, 2])))
    assert (new[:, :, 2] == want[:, :, 2]).all() and not new[:, :, 3:].any() and not new[:, :, :2].any()


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("policy", ["2:4", "dense"])
def test_bounds_of_every_bit_pattern(policy, dtype):
    """All 65536 patterns of a 16-bit type among the keys, infinities, NaN and zeros of both signs included."""
    def spoil(K, V):
        every = torch.randperm(65536, generator=_gen(1)).to(torch.int32).to(torch.int16).view(TYPES[dtype])
        K.view(-1)[:65536] = every

    sh, kv, K, _, held = _cache(1, 2, 1, 9, dtype, policy, 8, spoil)
    want = ref.tile_bounds(_ubits(K), held)
    assert (_ubits(hb.tile_bounds(sh, kv)) == want).all()
    assert np.isnan(_f64(torch.from_numpy(want.view(np.int16)).view(TYPES[dtype]))).any()


# ---------------------------------------------------------------------------------------------------------------------
# scores
# ---------------------------------------------------------------------------------------------------------------------
def _close_scores(got, want, size):
    """A score is a sum of 128 exact products (of the 256 one factor is zero in half): each of the additions off by at most a step of 2^-23 of
    the sum of the magnitudes, cut or rounded."""
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want)
    assert ((got == want) | (off <= 128 * 2.0 ** -23 * size)).all(), np.nanmax(off)


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("B,G,Hkv,T,Lq", [(1, 1, 1, 1, 1), (1, 4, 2, 16, 1), (2, 7, 3, 17, 1), (1, 8, 2, 130, 1), (1, 1, 2, 5, 2), (2, 3, 1, 33, 16), (1, 8, 1, 20, 17),
                                          (1, 4, 2, 3, 150), (1, 5, 1, 301, 33)])
def test_scores(B, G, Hkv, T, Lq, dtype):
    t = TYPES[dtype]
    g = _gen(T + Lq)
    sh = hb.make_shape(B, G * Hkv, Hkv, T * TILE, dtype=t)
    Q = torch.randn((B, G * Hkv, Lq, D), generator=g).to(t)
    mid, reach = torch.randn((B, Hkv, T, 1, D), generator=g), torch.rand((B, Hkv, T, 2, D), generator=g)
    bounds = (mid + reach * torch.tensor([-2.0, 2.0])[:, None]).to(t)
    k_map = (torch.rand((B, Hkv, T), generator=g) < 0.7).to(torch.int32) * -3
    low, high = _f64(bounds[:, :, :, 0]), _f64(bounds[:, :, :, 1])
    for causal, at in ((False, None), (True, None), (True, (T * TILE - Lq) // 3)):
        first = T * TILE - Lq if at is None else at
        for m in (None, k_map):
            held = np.ones((B, Hkv, T), bool) if m is None else (m != 0).numpy()
            want, size = ref.query_scores(_f64(Q), low, high, held, first + np.arange(Lq) if causal else None)
            got = hb.query_scores(sh, Q.cuda(), bounds.cuda(), None if m is None else m.cuda(), causal=causal, q_start=at)
            assert tuple(got.shape) == (B, Hkv, Lq, T)
            _close_scores(_f64(got), want, size)
    if Lq == 1:  # without a token axis
        assert torch.equal(hb.query_scores(sh, Q[:, :, 0].cuda(), bounds.cuda(), k_map.cuda())[:, :, None], hb.query_scores(sh, Q.cuda(), bounds.cuda(), k_map.cuda(), causal=False))


@gpu
def test_scores_bound_every_key():
    """No key of a tile scores more than its bound, whatever the tiles are."""
    for dtype in sorted(TYPES):
        sh, kv, K, _, held = _cache(2, 8, 2, 11, dtype, "some of half", 4)
        Q = torch.randn((2, 8, 3, D), generator=_gen(9)).to(TYPES[dtype])
        s = _f64(hb.query_scores(sh, Q.cuda(), hb.tile_bounds(sh, kv), kv.k_map, causal=False))
        q, k = _f64(Q).reshape(2, 2, 4, 3, D), _f64(K).reshape(2, 2, 11, TILE, D)
        real = np.einsum("bhgid,bhtjd->bhgitj", q, k).max((2, 5))
        size = np.einsum("bhgid,bhtjd->bhgitj", np.abs(q), np.abs(k)).max((2, 5))
        assert (np.where(held[:, :, None], real - 128 * 2.0 ** -23 * 4 * size, -np.inf) <= s).all()
        assert (s[np.broadcast_to(~held[:, :, None], s.shape)] == -np.inf).all()


@gpu
def test_scores_of_infinities_and_nan():
    """What cannot be ruled out scores +inf; other tiles, heads and queries keep their scores."""
    sh = hb.make_shape(1, 2, 1, 20 * TILE)
    g = _gen(5)
    Q, bounds = torch.randn((1, 2, 18, D), generator=g).bfloat16(), torch.randn((1, 1, 20, 2, D), generator=g).bfloat16()
    Q[0, :, :, 3], Q[0, :, :, 5], Q[0, :, :, 11] = 1.0, -2.0, 0.0
    bounds[0, 0, 2, 1, 3] = math.nan        # a NaN bound
    bounds[0, 0, 4, 1, 3] = math.inf        # reached
    bounds[0, 0, 6, 0, 5] = -math.inf       # reached from below
    bounds[0, 0, 8, 1, 11] = math.inf       # times zero
    bounds[0, 0, 10, :, 3] = -math.inf      # both, and a positive query: ruled out
    Q[0, 1, 17, 20] = math.nan              # the second head of the last query
    want, size = ref.query_scores(_f64(Q), _f64(bounds[:, :, :, 0]), _f64(bounds[:, :, :, 1]), np.ones((1, 1, 20), bool))
    for q, w, z in ((Q, want, size), (Q[:, :, 5:6], want[:, :, 5:6], size[:, :, 5:6]), (Q[:, :, 17:], want[:, :, 17:], size[:, :, 17:])):
        got = _f64(hb.query_scores(sh, q.cuda(), bounds.cuda(), causal=False))
        assert not np.isnan(got).any() and (np.isinf(got) == np.isinf(w)).all() and (got[np.isinf(w)] == w[np.isinf(w)]).all()
        fine = np.isfinite(w)
        _close_scores(got[fine], w[fine], z[fine])
    assert (want[0, 0, 0, [2, 4, 6, 8]] == math.inf).all() and (want[0, 0, 17] == math.inf).all()


# ---------------------------------------------------------------------------------------------------------------------
# the choice
# ---------------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("T,Lq", [(1, 1), (2, 3), (63, 2), (64, 1), (65, 5), (256, 1), (257, 2), (512, 3), (777, 40), (1024, 1), (1025, 1), (2048, 2), (2049, 1),
                                  (8192, 1), (8193, 1), (16384, 1), (16385, 1), (65536, 1)])
def test_pick(T, Lq):
    g = _gen(T)
    sh = hb.make_shape(2, 2, 2, T * TILE)
    s = (torch.randn((2, 2, Lq, T), generator=g) * 4).half().float()       # many are equal
    s[0, :, :, torch.rand(T, generator=g) < 0.3] = -math.inf
    s[1, 0, 0] = -math.inf
    s[1, 1] = torch.randn((Lq, T), generator=g)
    for n, first, last in ((1, 0, 0), (5, 1, 4), (32, 1, 4), (3, 3, 0), (4, 0, 4), (max(1, T // 2), 0, 0), (T + 7, 2, 2), (max(1, T - 1), 0, 0)):
        got = hb.pick_tiles(sh, s.cuda(), n, first, last)
        assert (got.cpu().numpy() == ref.pick_tiles(s.numpy(), n, first, last)).all(), (n, first, last)
    flat = s[:, :, 0].contiguous().cuda()
    assert (hb.pick_tiles(sh, flat, 4).cpu().numpy() == ref.pick_tiles(s[:, :, 0].numpy(), 4, 0, 0)).all()


@gpu
@pytest.mark.parametrize("T,Lq", [(90, 190), (300, 190), (700, 190), (1500, 190), (3000, 190), (1, 400), (64, 400), (65, 400), (128, 400), (129, 1400), (256, 1400)])
def test_pick_for_many_queries(T, Lq):
    """More than 512, 1024 and 4096 rows, which other numbers of threads take."""
    g = _gen(T)
    sh = hb.make_shape(1, 3, 3, T * TILE)
    s = (torch.randn((1, 3, Lq, T), generator=g) * 4).half().float()
    s[0, 0, 0, ::3], s[0, 0, 1, ::2], s[0, 0, 2], s[0, 0, 3], s[0, 0, 4] = math.nan, math.inf, 2.5, -math.inf, torch.where(torch.rand(T, generator=g) < 0.5, 0.0, -0.0)
    s[torch.rand(s.shape, generator=g) < 0.2] = -math.inf
    for n, first, last in ((24, 1, 4), (1, 0, 0), (max(3, T // 2), 3, 0), (5, 1, 4)):
        assert (hb.pick_tiles(sh, s.cuda(), n, first, last).cpu().numpy() == ref.pick_tiles(s.numpy(), n, first, last)).all(), (n, first, last)


@gpu
@pytest.mark.parametrize("kind", ["alike", "two values", "zeros of both signs", "special", "none", "near"])
@pytest.mark.parametrize("T", [40, 100, 1000, 5000, 20000])
def test_pick_of_special_scores(T, kind):
    g = _gen(T)
    s = {"alike": torch.full((1, 1, 3, T), -2.5), "two values": (torch.rand((1, 1, 3, T), generator=g) < 0.1).float(),
         "zeros of both signs": torch.where(torch.rand((1, 1, 3, T), generator=g) < 0.5, 0.0, -0.0), "none": torch.full((1, 1, 3, T), -math.inf),
         "near": 1.0 + torch.randint(0, 60, (1, 1, 3, T), generator=g) * 2.0 ** -23}.get(kind)
    if s is None:
        s = torch.randn((1, 1, 3, T), generator=g)
        x = torch.rand((1, 1, 3, T), generator=g)
        s[x < 0.02], s[(x > 0.1) & (x < 0.12)], s[(x > 0.2) & (x < 0.4)], s[(x > 0.5) & (x < 0.51)] = math.nan, math.inf, -math.inf, 3.4e38
        s[(x > 0.6) & (x < 0.61)], s[(x > 0.7) & (x < 0.71)] = -3.4e38, 1e-45
    sh = hb.make_shape(1, 1, 1, T * TILE)
    for n, first, last in ((1, 0, 0), (17, 1, 4), (T // 3, 0, 0), (T // 40 + 1, 0, 1)):
        assert (hb.pick_tiles(sh, s.cuda(), n, first, last).cpu().numpy() == ref.pick_tiles(s.numpy(), n, first, last)).all(), (n, first, last)


def _unranked(kind, T, g):
    """Three rows of scores whose finite ones span no width that 32 bits hold, or that have none."""
    s = torch.full((3, T), {"nan": math.nan}.get(kind, math.inf))
    if kind == "inf and nan":
        s[torch.rand((3, T), generator=g) < 0.5] = math.nan
    elif kind == "wide":
        s = (torch.rand((3, T), generator=g) * 2 - 1) * 3.4e38
        s[:, 7], s[:, 11] = -3.4e38, 3.4e38
    elif kind == "alike":
        s[:] = 1.5
    s[1, torch.rand(T, generator=g) < 0.1] = -math.inf
    return s


@gpu
@pytest.mark.parametrize("first,last", [(0, 0), (1, 4)])
@pytest.mark.parametrize("kind", ["inf", "nan", "inf and nan", "wide", "alike"])
@pytest.mark.parametrize("T", [72, 100, 300, 600, 1000, 2000, 4000, 5000, 10000, 20000])
def test_pick_of_scores_without_a_width(T, kind, first, last):
    """Any number left to take by score, those about the most that are ranked one against all (64) among them; nothing is written behind the lists."""
    rows = _unranked(kind, T, _gen(T))
    for Lq in (3, 600):
        sh = hb.make_shape(1, 1, 1, T * TILE)
        s = rows.repeat(Lq // 3, 1)[None, None].contiguous().cuda()
        for rest in sorted({1, 2, 63, 64, 65, 66, 67, 128, 129, T // 2}):
            n = rest + first + last
            space = torch.full((Lq * n + 2 * T + 128,), 77, dtype=torch.int32, device="cuda")
            out = space[64:64 + Lq * n].view(1, 1, Lq, n)
            got = hb.pick_tiles(sh, s, n, first, last, out=out).cpu().numpy()[0, 0]
            want = ref.pick_tiles(rows.numpy(), n, first, last)
            assert (got.reshape(-1, 3, n) == want).all(), (Lq, rest)
            assert bool((space[:64] == 77).all()) and bool((space[64 + Lq * n:] == 77).all()), (Lq, rest)


# ---------------------------------------------------------------------------------------------------------------------
# attention over listed tiles
# ---------------------------------------------------------------------------------------------------------------------
def _lists(B, Hkv, Lq, T, n, seed):
    """Lists of n entries: tiles in any order, some twice, some numbers that are no tiles."""
    g = _gen(seed)
    x = torch.randint(0, T, (B, Hkv, Lq, n), generator=g)
    x = torch.where(torch.rand(x.shape, generator=g) < 0.1, torch.randint(-5, 0, x.shape, generator=g), x)
    return torch.where(torch.rand(x.shape, generator=g) < 0.1, T + torch.randint(0, 1 << 30, x.shape, generator=g), x).to(torch.int32)


def _close_attention(got_o, got_lse, want, dtype, what=""):
    O, LSE, o_tol, l_tol = want
    u = torch.finfo(dtype).eps / 2
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    o, lse = _f64(got_o), _f64(got_lse)
    assert np.isfinite(o).all(), what
    off = np.abs(o - O) - (u * np.abs(O) + (1 + u) * o_tol + tiny)
    assert (off <= 0).all(), (what, off.max())
    none = np.isinf(LSE)
    assert (lse[none] == -np.inf).all() and (o[none] == 0).all(), what
    assert (np.abs(lse[~none] - LSE[~none]) <= l_tol[~none]).all(), what


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("policy", sorted(POLICIES))
@pytest.mark.parametrize("B,G,Hkv,T,Lq,n", [(1, 1, 1, 1, 1, 1), (2, 4, 2, 9, 1, 5), (1, 8, 1, 40, 1, 70), (1, 7, 2, 12, 5, 6), (2, 3, 2, 6, 70, 3), (1, 2, 4, 33, 2, 20),
                                            (1, 5, 1, 8, 301, 4), (2, 1, 2, 7, 90, 30)])
def test_listed_attention(B, G, Hkv, T, Lq, n, policy, dtype):
    sh, kv, K, V, held = _cache(B, G * Hkv, Hkv, T, dtype, policy, 7 * T + n)
    Q = torch.randn((B, G * Hkv, Lq, D), generator=_gen(n)).to(TYPES[dtype])
    lists = _lists(B, Hkv, Lq, T, n, 3 * n)
    lists[:, :, Lq // 2 + 1:Lq // 2 + 3] = -1          # queries with no tile at all
    first = T * TILE - Lq
    for causal, at, scale in ((False, None, 0.0), (True, None, 0.0), (True, first // 2, 0.02)):
        pos = (first if at is None else at) + np.arange(Lq) if causal else None
        want = ref.listed_attention(_f64(Q), _f64(K), _f64(V), lists.numpy(), held, scale or D ** -0.5, pos, weight=2.0 ** (-16 if B * Hkv * Lq <= 300 else -11))
        o, lse = hb.listed_attn(sh, Q.cuda(), kv, lists.cuda(), causal=causal, q_start=at, scale=scale)
        _close_attention(o, lse, want, TYPES[dtype], (causal, at))
    if Lq == 1:
        o1, lse1 = hb.listed_attn(sh, Q[:, :, 0].cuda(), kv, lists[:, :, 0].contiguous().cuda())
        o, lse = hb.listed_attn(sh, Q.cuda(), kv, lists.cuda(), causal=False)
        assert torch.equal(_bits(o1), _bits(o[:, :, 0])) and torch.equal(lse1, lse[..., 0])


@gpu
@pytest.mark.parametrize("policy", ["2:4", "dense", "some of half"])
@pytest.mark.parametrize("B,n", [(1, 3), (3, 20), (70, 6), (300, 4)])
def test_listed_attention_with_a_dense_tail(B, n, policy):
    """Tails of every length, by themselves too, of few and of many sequences."""
    T, Hkv, G = 8, 1, 4
    sh, kv, K, V, held = _cache(B, G * Hkv, Hkv, T, "bf16", policy, n)
    g = _gen(B)
    Q, tk, tv = torch.randn((B, G, D), generator=g).bfloat16(), torch.randn((B, Hkv, TILE, D), generator=g).bfloat16(), torch.randn((B, Hkv, TILE, D), generator=g).bfloat16()
    lens = torch.randint(-3, 70, (B,), generator=g, dtype=torch.int32)
    lens[0] = 0
    lists = _lists(B, Hkv, 1, T, n, B)[:, :, 0].contiguous()
    lists[B // 2] = -1
    tk[0], tv[0] = math.nan, math.inf      # no token of it is valid
    for x in (lens, 17):
        want = ref.listed_attention(_f64(Q)[:, :, None], _f64(K), _f64(V), lists.numpy()[:, :, None], held, D ** -0.5, None, _f64(tk), _f64(tv),
                                    lens.numpy() if x is lens else np.full(B, 17))
        o, lse = hb.listed_attn(sh, Q.cuda(), kv, lists.cuda(), tail_k=tk.cuda(), tail_v=tv.cuda(), tail_len=x.cuda() if x is lens else x)
        if x is not lens:                  # the first sequence sees its NaN
            assert bool(torch.isnan(o[0]).all()) and bool(torch.isnan(lse[0]).all())
            o[0], lse[0] = 0.0, -math.inf
            want = tuple(w.copy() for w in want)
            want[0][0], want[1][0], want[2][0] = 0.0, -np.inf, 0.0
        _close_attention(o[:, :, None], lse[:, :, None], want, torch.bfloat16, x)


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("policy", sorted(POLICIES))
def test_lists_are_sets(policy, dtype):
    """The order of a list, tiles named again and numbers that are no tiles do not change a bit."""
    B, Hkv, T, n = 2, 2, 30, 24
    sh, kv, _, _, _ = _cache(B, 8, Hkv, T, dtype, policy, 11)
    Q = torch.randn((B, 8, D), generator=_gen(2)).to(TYPES[dtype]).cuda()
    g = _gen(12)
    base = torch.stack([torch.randperm(T, generator=g)[:10] for _ in range(B * Hkv)]).reshape(B, Hkv, 10)
    sorted_ = torch.cat([base.sort(-1).values, torch.full((B, Hkv, n - 10), -1)], -1).to(torch.int32)
    mixed = torch.cat([base, base[..., :7], torch.full((B, Hkv, 7), T)], -1)[..., torch.randperm(n, generator=g)].to(torch.int32)
    a, b = hb.listed_attn(sh, Q, kv, sorted_.cuda()), hb.listed_attn(sh, Q, kv, mixed.contiguous().cuda())
    assert torch.equal(_bits(a[0]), _bits(b[0])) and torch.equal(a[1], b[1])


@gpu
@pytest.mark.parametrize("policy", ["2:4", "dense", "dense keys", "dense values", "half"])
@pytest.mark.parametrize("far", [(), (0,), (3, 4), (1, 5, 9), tuple(range(12))])
@pytest.mark.parametrize("Lq", [1, 5, 310])
def test_value_tiles_in_either_encoding(Lq, far, policy):
    """bf16 caches whose value tiles are held in fp16 encoding, but for some of values that fp16 does not hold."""
    def spoil(K, V):
        for t in far:
            V[:, :, t * TILE:(t + 1) * TILE] *= 2.0 ** -20
    T = 12
    sh, kv, K, V, held = _cache(1, 4, 1, T, "bf16", policy, 13, spoil)
    assert {t for t in range(T) if not int(kv.v_map[0, 0, t].abs()) & hb.MAP_F16} >= set(far)
    Q = torch.randn((1, 4, Lq, D), generator=_gen(2)).bfloat16()
    lists = torch.tensor([9, 0, 3, 1, 4, 11, 5], dtype=torch.int32).expand(1, 1, Lq, 7).contiguous()
    lists[:, :, ::2] = lists[:, :, ::2].sort(-1).values
    want = ref.listed_attention(_f64(Q), _f64(K), _f64(V), lists.numpy(), held, D ** -0.5, weight=2.0 ** (-16 if Lq <= 300 else -11))
    o, lse = hb.listed_attn(sh, Q.cuda(), kv, lists.cuda(), causal=False)
    _close_attention(o, lse, want, torch.bfloat16)


@gpu
def test_two_calls_at_once():
    """Two streams, each with its own lists and workspace, over one cache."""
    sh, kv, _, _, _ = _cache(2, 8, 2, 60, "bf16", "half", 23)
    g = _gen(24)
    Q = [torch.randn((2, 8, D), generator=g).bfloat16().cuda() for _ in range(2)]
    bounds = hb.tile_bounds(sh, kv)

    def step(q):
        return hb.listed_attn(sh, q, kv, hb.pick_tiles(sh, hb.query_scores(sh, q, bounds, kv.k_map), 30, 1, 4))
    want = [step(q) for q in Q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(step(Q[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for o, lse in got[i]:
            assert torch.equal(o, want[i][0]) and torch.equal(lse, want[i][1])


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("policy", ["2:4", "dense", "dense keys", "dense values", "some of half"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("Lq", [130, 170])
def test_unseen_tokens_do_not_touch_results(Lq, bad, policy, dtype):
    """Keys and values that are no numbers: in tiles that are not listed, and behind a causal query within its tile.  Queries by themselves, and in
    company (more than 300 of them)."""
    T = 6
    sh, clean, _, _, _ = _cache(1, 4, 2, T, dtype, policy, 6)
    states = [torch.where(m == 0, hb.SKIP, torch.where(m > 0, hb.DENSE, hb.SPARSE24)).to(torch.int8) for m in (clean.k_map, clean.v_map)]

    def spoil(K, V):
        for x in (K, V):
            x[:, :, 2 * TILE:3 * TILE:3] = bad       # a tile that no list names
            x[:, :, 4 * TILE + 21:] = bad            # behind the last query
    policy2 = hb.make_policy(state_k=states[0], state_v=states[1])
    sh, dirty, K, V, held = _cache(1, 4, 2, T, dtype, policy2, 6, spoil)
    Q = torch.randn((1, 4, Lq, D), generator=_gen(1)).to(TYPES[dtype])
    lists = torch.tensor([0, 1, 3, 4, 5], dtype=torch.int32).expand(1, 2, Lq, 5).contiguous()
    at = 4 * TILE + 21 - Lq
    o, lse = hb.listed_attn(sh, Q.cuda(), dirty, lists.cuda(), q_start=at)
    want = ref.listed_attention(_f64(Q), np.nan_to_num(_f64(K), nan=0.0, posinf=0.0, neginf=0.0), np.nan_to_num(_f64(V), nan=0.0, posinf=0.0, neginf=0.0), lists.numpy(), held,
                                D ** -0.5, at + np.arange(Lq), weight=2.0 ** (-16 if 2 * Lq <= 300 else -11))
    _close_attention(o, lse, want, TYPES[dtype])
    # a query that sees one: NaN, or what infinities give
    o, lse = hb.listed_attn(sh, Q[:, :, :1].cuda(), dirty, lists[:, :, :1].contiguous().cuda(), q_start=4 * TILE + 21)
    if math.isnan(bad) and bool(held[0, 0, 4]):
        assert bool(torch.isnan(o[0, :2]).all()) and bool(torch.isnan(lse[0, :2]).all())


@gpu
@pytest.mark.parametrize("G", [1, 2, 3, 7])
@pytest.mark.parametrize("policy", ["2:4", "dense", "half"])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_tiles_of_neighbouring_queries_do_not_touch_results(bad, policy, G):
    """Queries that do not list a tile whose keys and values are no numbers, between others that do."""
    T, Lq, Hkv = 7, 160, 2

    def spoil(K, V):
        K[:, 0, 2 * TILE:3 * TILE] = bad
        V[:, :, 2 * TILE + 5:3 * TILE:4] = bad
    _, clean, _, _, _ = _cache(1, G * Hkv, Hkv, T, "bf16", policy, 6)
    states = [torch.where(m > 0, hb.DENSE, hb.SPARSE24).to(torch.int8) for m in (clean.k_map, clean.v_map)]
    sh, kv, K, V, held = _cache(1, G * Hkv, Hkv, T, "bf16", hb.make_policy(state_k=states[0], state_v=states[1]), 6, spoil)
    Q = torch.randn((1, G * Hkv, Lq, D), generator=_gen(1)).bfloat16()
    lists = torch.full((1, Hkv, Lq, 4), -1, dtype=torch.int32)
    lists[..., :3] = torch.tensor([6, 0, 3])
    lists[:, :, ::3, 3] = 2
    o, lse = hb.listed_attn(sh, Q.cuda(), kv, lists.cuda(), causal=False)
    zero = [np.nan_to_num(_f64(x), nan=0.0, posinf=0.0, neginf=0.0) for x in (K, V)]
    want = ref.listed_attention(_f64(Q), *zero, np.where(lists.numpy() == 2, -1, lists.numpy()), held, D ** -0.5, weight=2.0 ** -11)
    rest = np.arange(Lq) % 3 != 0
    _close_attention(o[:, :, rest], lse[:, :, rest], tuple(x[:, :, rest] for x in want), torch.bfloat16)
    assert not bool(torch.isfinite(o[:, :, ::3].float()).all(-1).any())


@gpu
@pytest.mark.parametrize("policy", ["dense", "dense keys"])
@pytest.mark.parametrize("Lq", [30, 320])
def test_large_values(Lq, policy):
    """Values whose weighted sums stay below 2^128 where no weight passes 2^8, and do not where weights reach 2^15: tiles 4 to 11 score some 6.2 binades more than
    the first four, which those of a wave begin with."""
    T, B, Hkv, G = 12, 1, 4, 4

    def spoil(K, V):
        K.mul_(0.2)
        K[:, :, 4 * TILE:] += 0.38             # 128 channels and queries of about 1, a scale of 128 ** -0.5: 4.3 more
        V.copy_((1.0 + 0.3 * V.float().abs()) * 2.0 ** 109)
    sh, kv, K, V, held = _cache(B, G * Hkv, Hkv, T, "bf16", policy, 41, spoil)
    Q = (1.0 + 0.1 * torch.randn((B, G * Hkv, Lq, D), generator=_gen(42))).bfloat16()
    lists = torch.arange(T, dtype=torch.int32).expand(B, Hkv, Lq, T).contiguous()
    want = ref.listed_attention(_f64(Q), _f64(K), _f64(V), lists.numpy(), held, D ** -0.5)
    o, lse = hb.listed_attn(sh, Q.cuda(), kv, lists.cuda(), causal=False)
    _close_attention(o, lse, want, torch.bfloat16)


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("policy", ["2:4", "dense", "half"])
@pytest.mark.parametrize("G,Hkv,Lq", [(1, 16, 133), (3, 8, 82), (4, 8, 66), (8, 4, 66)])
def test_steep_scores(G, Hkv, Lq, policy, dtype):
    """Scores that rise and fall by a hundred binades from tile to tile, by few for some queries and by many for others, several tiles a wave: the running reference
    moves often, for columns that do not see the tile too, and lags behind by up to 7 binades."""
    T, n = 16, 9
    sizes = torch.tensor([0.05, 0.3, 0.8, 2.0, 4.0, 1.0, 0.1, 6.0, 0.5, 3.0, 0.2, 8.0, 0.02, 5.0, 7.0, 1.5])

    def spoil(K, V):
        K.mul_(sizes.repeat_interleave(TILE)[:, None].to(K.dtype))
    sh, kv, K, V, held = _cache(1, G * Hkv, Hkv, T, dtype, policy, 51, spoil)
    g = _gen(52)
    Q = (torch.randn((1, G * Hkv, Lq, D), generator=g) * torch.exp(torch.rand((1, G * Hkv, Lq, 1), generator=g) * 3.4 - 2.3)).to(TYPES[dtype])
    lists = torch.rand((1, Hkv, Lq, T), generator=g).argsort(-1)[..., :n].to(torch.int32).contiguous()
    for causal in (False, True):
        pos = T * TILE - Lq + np.arange(Lq) if causal else None
        want = ref.listed_attention(_f64(Q), _f64(K), _f64(V), lists.numpy(), held, D ** -0.5, pos, weight=2.0 ** -11)
        # weights below the normal numbers of fp16 are off by half a step of 2^-24, the largest one is 2^8 at least
        want[2][:] += 64 * n * 2.0 ** -33 * np.abs(_f64(V)).max()
        o, lse = hb.listed_attn(sh, Q.cuda(), kv, lists.cuda(), causal=causal)
        _close_attention(o, lse, want, TYPES[dtype], causal)


@gpu
@pytest.mark.parametrize("T,n", [(3000, 40), (9000, 9), (65536, 5)])
def test_many_queries_on_long_rows(T, n):
    """Rows of more tiles than the bit maps of 16 queries hold: against single queries, whose lists they are."""
    Lq = 310
    sh = hb.make_shape(1, 2, 1, T * TILE)
    small = hb.make_shape(1, 2, 1, 8 * TILE)
    K = torch.randn((1, 1, 8 * TILE, D), generator=_gen(3)).bfloat16().cuda()
    few = hb.compress_kv(small, hb.make_policy(), K, K)
    kv = hb.PackedKV(sh, [T - 8, 0, 8, 0, 8], "cuda")          # slots that repeat: a valid cache to read
    kv.k_nnz, kv.k_meta, kv.v_nnz, kv.v_meta = few.k_nnz, few.k_meta, few.v_nnz, few.v_meta
    slots = -(torch.arange(T, dtype=torch.int32, device="cuda") % 8 + 1)
    kv.k_map, kv.v_map = slots.repeat(1, 1, 1), slots.repeat(1, 1, 1) - (few.v_map[0, 0, 0].abs() & hb.MAP_F16)
    Q = torch.randn((1, 2, Lq, D), generator=_gen(4)).bfloat16().cuda()
    lists = torch.randint(0, T, (1, 1, Lq, n), generator=_gen(5), dtype=torch.int32).cuda()
    lists[..., 0] = T - 1
    o, lse = hb.listed_attn(sh, Q, kv, lists, causal=False)
    for i in range(Lq):
        o1, lse1 = hb.listed_attn(sh, Q[:, :, i], kv, lists[:, :, i].contiguous())
        assert (o[:, :, i].float() - o1.float()).abs().max().item() <= 4 * 2.0 ** -8 * o1.float().abs().max().item(), i
        assert (lse[:, :, i] - lse1).abs().max().item() <= 1e-4, i


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("policy", sorted(POLICIES))
def test_all_tiles_listed_is_attention(policy, dtype):
    """Lists that name every tile give what decode and prefill attention give, to the tolerance of both."""
    B, Hkv, T, Lq = 2, 2, 10, 64
    sh, kv, K, V, held = _cache(B, 8, Hkv, T, dtype, policy, 21)
    Q = torch.randn((B, 8, Lq, D), generator=_gen(4)).to(TYPES[dtype]).cuda()
    every = torch.arange(T, dtype=torch.int32).expand(B, Hkv, Lq, T).contiguous().cuda()
    u = torch.finfo(TYPES[dtype]).eps / 2
    for got, want, tol in ((hb.listed_attn(sh, Q, kv, every), hb.prefill_attn(sh, Q, kv), None),
                           (hb.listed_attn(sh, Q[:, :, 5].contiguous(), kv, every[:, :, 5].contiguous()), hb.decode_attn(sh, Q[:, :, 5].contiguous(), kv), None)):
        # both within the contract of attention: two roundings of 16 bits, and weights of 11 bits in prefill
        assert (got[0].float() - want[0].float()).abs().max().item() <= 8 * u * want[0].float().abs().max().item()
        assert (got[1] - want[1]).abs().max().item() <= 1e-4


@gpu
@pytest.mark.parametrize("n_tiles", [1030, 2100])
def test_lists_longer_than_a_pass(n_tiles):
    """More tiles than a workgroup lists at a time, in one share: against all of them in decode attention."""
    B, T = 260, n_tiles
    sh = hb.make_shape(B, 1, 1, T * TILE, dtype=torch.float16)
    # all sequences share the slots of few tiles' contents: a map whose slots repeat is a valid cache to read
    K = torch.randn((B, 1, 4 * TILE, D), generator=_gen(3)).half().cuda()
    small = hb.compress_kv(hb.make_shape(B, 1, 1, 4 * TILE, dtype=torch.float16), hb.make_policy(), K, K)
    kv = hb.PackedKV(sh, [T - 4, 0, 4, 0, 4], "cuda")
    kv.k_nnz, kv.k_meta, kv.v_nnz, kv.v_meta = small.k_nnz, small.k_meta, small.v_nnz, small.v_meta
    slots = -(torch.arange(T, dtype=torch.int32, device="cuda") % 4 + 1)
    kv.k_map, kv.v_map = slots.repeat(B, 1, 1), slots.repeat(B, 1, 1)
    Q = torch.randn((B, 1, D), generator=_gen(6)).half().cuda()
    every = torch.arange(T - 1, -1, -1, dtype=torch.int32, device="cuda").repeat(B, 1, 1)
    a, b = hb.listed_attn(sh, Q, kv, every), hb.decode_attn(sh, Q, kv)
    assert (a[0].float() - b[0].float()).abs().max().item() <= 4 * 2.0 ** -11 * b[0].float().abs().max().item()
    assert (a[1] - b[1]).abs().max().item() <= 1e-4


def _repeated(sh, small, T):
    """A cache of T tiles a row whose slots are those of a small one, over and over: a valid cache to read."""
    kv = hb.PackedKV(sh, [T - 4, 0, 4, 0, 4], "cuda")
    kv.k_nnz, kv.k_meta, kv.v_nnz, kv.v_meta = small.k_nnz, small.k_meta, small.v_nnz, small.v_meta
    at = torch.arange(T, dtype=torch.int32, device="cuda") % 4
    kv.k_map, kv.v_map = (m[:, :, :1].repeat(1, 1, T) - at for m in (small.k_map, small.v_map))
    return kv


def _attention_over_copies(Q, K, V, lists, scale, weight):
    """Attention of Q [B, Hq, Lq, D] over a cache whose tile t holds what tile t % 4 of K, V [B, Hkv, 256, D] holds, in 64 bits: a token of the four stands for as many
    as the list has copies of its tile.  O, LSE and bounds on their error as in the oracle."""
    B, Hq, Lq, _ = Q.shape
    H = K.shape[1]
    O, LSE, o_tol, l_tol = np.zeros(Q.shape), np.zeros(Q.shape[:3]), np.zeros(Q.shape), np.zeros(Q.shape[:3])
    e = 2.0 ** -24
    for b in range(B):
        for hq in range(Hq):
            h = hq // (Hq // H)
            copies = np.stack([np.bincount(np.unique(x) % 4, minlength=4) for x in lists[b, h]]).repeat(TILE, axis=-1)
            k, v = np.where(copies.any(0)[:, None], K[b, h], 0.0), np.where(copies.any(0)[:, None], V[b, h], 0.0)
            s = np.where(copies > 0, scale * (Q[b, hq] @ k.T), -np.inf)
            m = s.max(-1, keepdims=True)
            p = copies * np.exp(s - m)
            total, count = p.sum(-1, keepdims=True), copies.sum(-1)
            O[b, hq], LSE[b, hq] = p @ v / total, (m + np.log(total))[:, 0]
            off = scale * 2 * D * e * (np.abs(Q[b, hq]) @ np.abs(k).T).max(-1) + 4 * e * np.where(copies > 0, np.abs(s), 0.0).max(-1) * 1.5
            o_tol[b, hq] = p @ np.abs(v) / total * (2 * off + weight + 2.0 ** -21 + 4 * count * e)[:, None]
            l_tol[b, hq] = off + 2.0 ** -21 + 4 * e * np.abs(LSE[b, hq]) + 4 * count * e
    return O, LSE, o_tol, l_tol


@gpu
@pytest.mark.parametrize("bad", [None, math.nan, math.inf])
def test_neighbouring_queries_over_more_tiles_than_a_pass(bad):
    """Up to 16 queries in company that list some 2200 or 2400 tiles among them, in one share: three passes of 1024.  With values that are no numbers in tiles that two of three
    queries do not list, which are done again one by one."""
    B, Hkv, T, Lq, n = 4, 2, 3000, 301, 300
    g = _gen(61)
    K, V = torch.randn((B, Hkv, 4 * TILE, D), generator=g).bfloat16(), torch.randn((B, Hkv, 4 * TILE, D), generator=g).bfloat16()
    if bad is not None:
        V[:, :, 3 * TILE + 5::7] = bad
    few = hb.compress_kv(hb.make_shape(B, Hkv, Hkv, 4 * TILE), hb.make_policy(sparse_frac_k=0.0, sparse_frac_v=0.0), K.cuda(), V.cuda())
    sh = hb.make_shape(B, Hkv, Hkv, T * TILE)
    kv = hb.PackedKV(sh, [T - 4, 4, 0, 4, 0], "cuda")         # slots that repeat: a valid cache to read
    kv.k_dense, kv.v_dense = few.k_dense, few.v_dense
    kv.k_map, kv.v_map = (m.repeat(1, 1, T // 4) for m in (few.k_map, few.v_map))
    Q = torch.randn((B, Hkv, Lq, D), generator=g).bfloat16()
    lists = torch.randint(0, T, (B, Hkv, Lq, n), generator=g)
    clean = np.arange(Lq) % 3 != 0 if bad is not None else np.ones(Lq, bool)
    if bad is not None:
        lists[:, :, clean] -= (lists[:, :, clean] % 4 == 3).long()
    lists = lists.to(torch.int32)
    for first in (0, 4, 32):                                  # the tiles of the first, of a middle and of a late workgroup
        assert len(np.unique(lists[0, 0, first * 4:first * 4 + 16].numpy())) > 2 * 1024
    assert hb.listed_attn_workspace_bytes(sh, Lq, n) == 0     # one share
    o, lse = hb.listed_attn(sh, Q.cuda(), kv, lists.cuda(), causal=False)
    want = _attention_over_copies(_f64(Q[:, :, clean]), _f64(K), _f64(V), lists[:, :, clean].numpy(), D ** -0.5, 2.0 ** -11)
    _close_attention(o[:, :, clean], lse[:, :, clean], want, torch.bfloat16)
    if bad is not None:
        assert not bool(torch.isfinite(o[:, :, ~clean].float()).all(-1).any())


@gpu
@pytest.mark.parametrize("B,n", [(200, 1100), (140, 2100), (300, 1500)])
def test_single_queries_over_more_tiles_than_a_pass(B, n):
    """Lists in any order of more than 1024 tiles, in one share: 8 waves, or 4."""
    T = 2400
    g = _gen(62)
    K, V = torch.randn((B, 1, 4 * TILE, D), generator=g).half(), torch.randn((B, 1, 4 * TILE, D), generator=g).half()
    small = hb.make_shape(B, 2, 1, 4 * TILE, dtype=torch.float16)
    few = hb.compress_kv(small, hb.make_policy(), K.cuda(), V.cuda())
    K, V = hb.unpack_kv(small, few)
    sh = hb.make_shape(B, 2, 1, T * TILE, dtype=torch.float16)
    kv = _repeated(sh, few, T)
    Q = torch.randn((B, 2, D), generator=g).half()
    lists = torch.stack([torch.randperm(T, generator=g)[:n] for _ in range(B)])[:, None].to(torch.int32).contiguous()
    assert hb.listed_attn_workspace_bytes(sh, 1, n) == 0
    o, lse = hb.listed_attn(sh, Q.cuda(), kv, lists.cuda())
    want = _attention_over_copies(_f64(Q)[:, :, None], _f64(K), _f64(V), lists.numpy()[:, :, None], D ** -0.5, 2.0 ** -16)
    _close_attention(o[:, :, None], lse[:, :, None], want, torch.float16)


@gpu
def test_bounds_and_scores_beyond_32_bits():
    """Bounds of more than 4 GiB: the last rows of tiles against those that they repeat."""
    B, Hkv, T = 20, 8, 60000
    sh = hb.make_shape(B, Hkv, Hkv, T * TILE)
    K = torch.randn((B, Hkv, 4 * TILE, D), generator=_gen(1)).bfloat16().cuda()
    few_shape = hb.make_shape(B, Hkv, Hkv, 4 * TILE)
    few = hb.compress_kv(few_shape, hb.make_policy(), K, K)
    kv = _repeated(sh, few, T)
    bounds, small = hb.tile_bounds(sh, kv), hb.tile_bounds(few_shape, few)
    assert bounds.numel() * 2 > 1 << 32
    for t in (0, 1, 30000, T - 1):
        assert torch.equal(_bits(bounds[:, :, t]), _bits(small[:, :, t % 4])), t
    Q = torch.randn((B, Hkv, D), generator=_gen(2)).bfloat16().cuda()
    s, want = hb.query_scores(sh, Q, bounds, kv.k_map), hb.query_scores(few_shape, Q, small)
    assert torch.equal(s, want.repeat(1, 1, T // 4))
    best = hb.pick_tiles(sh, s, 3)
    assert torch.equal(best, (want.argmax(-1, keepdim=True) + 4 * torch.arange(3, device="cuda")).int())


@gpu
@pytest.mark.parametrize("Lq", [1, 301])
def test_listed_attention_in_pools_beyond_32_bits(Lq):
    """Slots behind 4 GiB of either pool."""
    T, cap = 8, 600000
    sh = hb.make_shape(1, 4, 1, T * TILE)
    K = torch.randn((1, 1, T * TILE, D), generator=_gen(1)).bfloat16().cuda()
    near = hb.compress_kv(sh, hb.make_policy(), K, K)
    far = hb.PackedKV(sh, [0, 0, cap, 0, cap], "cuda")
    far.uniform = 0
    for name, size in (("k_nnz", 8192), ("k_meta", 1024), ("v_nnz", 8192), ("v_meta", 1024)):
        getattr(far, name)[-T * size:] = getattr(near, name)
    far.k_map, far.v_map = near.k_map - (cap - T), near.v_map - (cap - T)
    Q = torch.randn((1, 4, Lq, D), generator=_gen(2)).bfloat16().cuda()
    lists = torch.tensor([1, 4, 7], dtype=torch.int32, device="cuda").expand(1, 1, Lq, 3).contiguous()
    near.uniform = 0
    for a, b in zip(hb.listed_attn(sh, Q, far, lists, causal=False), hb.listed_attn(sh, Q, near, lists, causal=False)):
        assert torch.equal(a, b)
    assert torch.equal(_bits(hb.tile_bounds(sh, far)), _bits(hb.tile_bounds(sh, near)))


@gpu
def test_views_of_queries():
    """Strides of a projection's output, [B, Lq, Hq, D] within a wider tensor."""
    sh, kv, _, _, _ = _cache(2, 8, 2, 12, "bf16", "2:4", 5)
    wide = torch.randn((2, 9, 12, D), generator=_gen(5)).bfloat16().cuda()
    q = wide[:, :, 2:10].transpose(1, 2)
    bounds = hb.tile_bounds(sh, kv)
    s, s2 = hb.query_scores(sh, q, bounds), hb.query_scores(sh, q.contiguous(), bounds)
    assert torch.equal(s, s2)
    lists = hb.pick_tiles(sh, s, 4, 1, 1)
    for x, y in zip(hb.listed_attn(sh, q, kv, lists), hb.listed_attn(sh, q.contiguous(), kv, lists)):
        assert torch.equal(x, y)
    one, l1 = q[:, :, 3], lists[:, :, 3].contiguous()
    assert torch.equal(hb.query_scores(sh, one, bounds), hb.query_scores(sh, one.contiguous(), bounds))
    assert torch.equal(hb.listed_attn(sh, one, kv, l1)[0], hb.listed_attn(sh, one.contiguous(), kv, l1)[0])


# ---------------------------------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_serving_with_picked_tiles(dtype):
    """A prompt, then steps that append, bound, score, pick and attend, with evictions between them: every step against 64 bits."""
    t = TYPES[dtype]
    B, Hq, Hkv, T, prompt, n = 2, 8, 2, 14, 9, 4
    sh = hb.make_shape(B, Hq, Hkv, T * TILE, dtype=t)
    g = _gen(31)
    K, V = torch.randn((B, Hkv, T * TILE, D), generator=g).to(t).cuda(), torch.randn((B, Hkv, T * TILE, D), generator=g).to(t).cuda()
    states = torch.zeros((B, Hkv, T), dtype=torch.int8)
    states[:, :, :prompt] = hb.SPARSE24
    states[:, :, 0] = hb.DENSE
    kv = hb.PackedKV(sh, [0, 2, T, 2, T], "cuda")
    hb.compress_kv(sh, hb.make_policy(state_k=states.cuda(), state_v=states.cuda()), K, V, out=kv)
    bounds = hb.tile_bounds(sh, kv)
    mass = torch.rand((B, Hkv, T), generator=g).cuda()
    tail_k, tail_v = torch.zeros((B, Hkv, TILE, D), dtype=t, device="cuda"), torch.zeros((B, Hkv, TILE, D), dtype=t, device="cuda")
    for step in range(prompt, T):
        if step > prompt:                       # the tail of the last steps is full
            at = _i32([step - 1, -1 if step % 2 else step - 1])
            hb.append_tile(sh, kv, at, tail_k, tail_v)
            hb.tile_bounds(sh, kv, at, out=bounds)
        if step == prompt + 3:
            hb.evict_tiles(sh, kv, mass, 7, first=1, last=2)
        tail_k.copy_(K[:, :, step * TILE:(step + 1) * TILE])
        tail_v.copy_(V[:, :, step * TILE:(step + 1) * TILE])
        q = torch.randn((B, Hq, D), generator=g).to(t).cuda()
        scores = hb.query_scores(sh, q, bounds, kv.k_map)
        picked = hb.pick_tiles(sh, scores, n, first=1, last=1)
        lens = torch.randint(0, 65, (B,), generator=g, dtype=torch.int32)
        o, lse = hb.listed_attn(sh, q, kv, picked, tail_k=tail_k, tail_v=tail_v, tail_len=lens.cuda())
        Ku, Vu = hb.unpack_kv(sh, kv)
        held = (kv.k_map != 0).cpu().numpy()
        fresh = ref.tile_bounds(_ubits(Ku), held)
        assert (_ubits(bounds)[held] == fresh[held]).all(), step
        f = _f64(torch.from_numpy(fresh.view(np.int16)).view(t))
        want, size = ref.query_scores(_f64(q)[:, :, None], f[:, :, :, 0], f[:, :, :, 1], held)
        _close_scores(_f64(scores)[:, :, None], want, size)
        assert (picked.cpu().numpy() == ref.pick_tiles(scores.cpu().numpy(), n, 1, 1)).all()
        res = ref.listed_attention(_f64(q)[:, :, None], _f64(Ku), _f64(Vu), picked.cpu().numpy()[:, :, None], held, D ** -0.5, None, _f64(tail_k), _f64(tail_v), lens.numpy())
        _close_attention(o[:, :, None], lse[:, :, None], res, t, step)


def _chain(sh, kv, Q, bounds, tail, out):
    hb.tile_bounds(sh, kv, out=bounds)
    hb.query_scores(sh, Q, bounds, kv.k_map, out=out["scores"])
    hb.pick_tiles(sh, out["scores"], out["list"].shape[-1], 1, 2, out=out["list"])
    return hb.listed_attn(sh, Q, kv, out["list"], out=out["o"], lse=out["lse"], workspace=out["ws"], **tail)


def _chain_buffers(sh, n, with_tail):
    T = sh.L // TILE
    t = hb.torch_dtype(sh)
    return dict(scores=torch.empty((sh.B, sh.Hkv, T), device="cuda"), list=torch.empty((sh.B, sh.Hkv, n), dtype=torch.int32, device="cuda"),
                o=torch.empty((sh.B, sh.Hq, D), dtype=t, device="cuda"), lse=torch.empty((sh.B, sh.Hq), device="cuda"),
                ws=torch.empty(max(16, hb.listed_attn_workspace_bytes(sh, 1, n, with_tail)), dtype=torch.uint8, device="cuda"))


@gpu
def test_captured_steps_replay():
    """A step captured into a graph, replayed over changed queries, caches and tails beside eager work on buffers of its own."""
    sh, kv, _, _, _ = _cache(2, 8, 2, 40, "bf16", "some of half", 17)
    g = _gen(18)
    Q = torch.randn((2, 8, D), generator=g).bfloat16().cuda()
    tail = dict(tail_k=torch.randn((2, 2, TILE, D), generator=g).bfloat16().cuda(), tail_v=torch.randn((2, 2, TILE, D), generator=g).bfloat16().cuda(),
                tail_len=_i32([9, 33]))
    bounds, eager_bounds = hb.tile_bounds(sh, kv), hb.tile_bounds(sh, kv)
    a, b = _chain_buffers(sh, 12, True), _chain_buffers(sh, 12, True)
    _chain(sh, kv, Q, bounds, tail, a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _chain(sh, kv, Q, bounds, tail, a)
    for i in range(4):
        Q.copy_(torch.randn((2, 8, D), generator=g).bfloat16())
        tail["tail_len"].copy_(_i32([(i * 23) % 65, 64 - i]))
        kv.k_nnz.view(torch.int16)[i * 100:i * 100 + 64].neg_()
        for x in a.values():
            x.zero_()
        graph.replay()
        _chain(sh, kv, Q, eager_bounds, tail, b)
        torch.cuda.synchronize()
        assert torch.equal(_bits(bounds), _bits(eager_bounds)), i
        for name in ("scores", "list", "o", "lse"):
            assert torch.equal(a[name], b[name]), (i, name)


@gpu
def test_calls_go_to_the_current_stream_and_equal_calls_give_equal_bits():
    sh, kv, _, _, _ = _cache(3, 12, 3, 50, "fp16", "some of half", 19)
    Q = torch.randn((3, 12, 7, D), generator=_gen(1)).half().cuda()
    bounds = hb.tile_bounds(sh, kv)
    lists = hb.pick_tiles(sh, hb.query_scores(sh, Q, bounds, kv.k_map), 9, 1, 2)
    want = hb.listed_attn(sh, Q, kv, lists)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    big = torch.randn((4096, 4096), device="cuda")
    with torch.cuda.stream(side):
        late = torch.zeros_like(Q)
        for _ in range(20):
            big = big @ big * 1e-3
        late.copy_(Q)                      # behind the products: a call on another stream would read zeros
        got = hb.listed_attn(sh, late, kv, hb.pick_tiles(sh, hb.query_scores(sh, late, hb.tile_bounds(sh, kv), kv.k_map), 9, 1, 2))
    side.synchronize()
    for x, y in zip(want, got):
        assert torch.equal(x, y)
    for _ in range(3):
        for x, y in zip(want, hb.listed_attn(sh, Q, kv, lists)):
            assert torch.equal(x, y)


@gpu
def test_python_and_native_marshalling_give_the_same(monkeypatch):
    B, Hq, Hkv, T = 2, 8, 2, 10
    sh, kv, _, _, _ = _cache(B, Hq, Hkv, T, "bf16", "some", 2)
    g = _gen(3)
    Q, tk = torch.randn((B, Hq, 20, D), generator=g).bfloat16().cuda(), torch.randn((B, Hkv, TILE, D), generator=g).bfloat16().cuda()
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    took = []

    def calls():
        bounds = hb.tile_bounds(sh, kv)
        res = [bounds, hb.tile_bounds(sh, kv, 2, 3), hb.tile_bounds(sh, kv, one), hb.tile_bounds(sh, kv, one, out=bounds.clone()), hb.tile_bounds(sh, kv, 1, 2, out=bounds.clone())]
        s = hb.query_scores(sh, Q, bounds, kv.k_map)
        res += [s, hb.query_scores(sh, Q, bounds, causal=False), hb.query_scores(sh, Q[:, :, 3], bounds, kv.k_map), hb.query_scores(sh, Q, bounds, kv.k_map, q_start=70, out=torch.empty_like(s))]
        res += [hb.pick_tiles(sh, s, 4, 1, 1), hb.pick_tiles(sh, res[-2], 3), hb.pick_tiles(sh, s, 4, 1, 1, out=torch.empty((B, Hkv, 20, 4), dtype=torch.int32, device="cuda"))]
        res += list(hb.listed_attn(sh, Q, kv, res[-3])) + list(hb.listed_attn(sh, Q[:, :, 3], kv, res[-2], want_lse=False))
        p = hb.pick_tiles(sh, hb.query_scores(sh, Q[:, :, 1], bounds), 3)
        res += list(hb.listed_attn(sh, Q[:, :, 1], kv, p, tail_k=tk, tail_v=tk, tail_len=one * 9)) + list(hb.listed_attn(sh, Q[:, :, 1], kv, p, tail_k=tk, tail_v=tk, tail_len=5))
        return res

    class Seen:
        def __getattr__(self, name):
            fn = getattr(native, name)

            def call(*a):
                r = fn(*a)
                took.append((name, r is not None))
                return r
            return call

    native = hb._fast()
    monkeypatch.setattr(hb, "_native", Seen())
    by_native = calls()
    assert {n for n, _ in took} >= {"bounds", "scores", "pick", "listed"}
    # bounds of a part of the tiles into a new tensor are made by the Python code
    assert [name for name, ok in took if not ok] == ["bounds", "bounds"]
    none = type("None_", (), {n: staticmethod(lambda *a: None) for n in hb._NATIVE_CALLS})
    monkeypatch.setattr(hb, "_native", none)
    for a, b in zip(by_native, calls()):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))


# ---------------------------------------------------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------------------------------------------------
def test_refusals_on_the_host():
    """Arguments that the library refuses before it launches anything (addresses here are never read)."""
    L, sh = hb.lib(), hb.make_shape(2, 8, 2, 256)
    s, kv = C.byref(sh), hb.HsKV(k_map=4096, v_map=4096)
    big = C.byref(hb.make_shape(1, 1, 1, 65537 * 64))

    def view(data=4096, batch=1 << 20, head=1 << 14, token=D):
        return C.byref(hb.HsView(data, batch, head, token))

    def bounds(tile=0, n=4, tiles=None, cache=C.byref(kv), out=4096, shape=s):
        return L.hs_tile_bounds(shape, tile, n, tiles, cache, out, None)

    for bad, rc in ((dict(tile=-1), -1), (dict(tile=4), -1), (dict(n=0), -1), (dict(n=5), -1), (dict(tile=3, n=2), -1), (dict(n=2 ** 31 - 1, tile=2 ** 31 - 1), -1),
                    (dict(out=None), -1), (dict(out=4104), -1), (dict(cache=None), -1), (dict(shape=None), -1), (dict(shape=C.byref(hb.make_shape(2, 8, 2, 100))), -2),
                    (dict(shape=C.byref(hb.make_shape(64, 1024, 1024, 64 * 2048, dtype=0)), n=2048), -2)):
        assert bounds(**bad) == rc, bad

    def scores(Lq=8, q_start=0, causal=1, Q=view(), b=4096, k_map=None, out=4096, shape=s):
        return L.hs_query_scores(shape, Lq, q_start, causal, Q, b, k_map, out, None)

    for bad, rc in ((dict(Lq=0), -1), (dict(q_start=-1), -1), (dict(q_start=249), -1), (dict(Lq=300), -1), (dict(Q=None), -1), (dict(Q=view(data=4104)), -1), (dict(b=None), -1),
                    (dict(b=4104), -1), (dict(k_map=4098), -1), (dict(out=None), -1), (dict(out=4098), -1), (dict(Q=view(token=100)), -1), (dict(Q=view(head=-8)), -1),
                    (dict(Lq=(1 << 30) + 1, causal=0), -2), (dict(shape=C.byref(hb.make_shape(1024, 64, 63, 64))), -2)):
        assert scores(**bad) == rc, bad

    def pick(Lq=8, sc=4096, n=4, first=0, last=0, out=4096, shape=s):
        return L.hs_pick_tiles(shape, Lq, sc, n, first, last, out, None)

    for bad, rc in ((dict(Lq=0), -1), (dict(sc=None), -1), (dict(sc=4098), -1), (dict(out=None), -1), (dict(out=4097), -1), (dict(n=0), -1), (dict(first=-1), -1),
                    (dict(last=-1), -1), (dict(first=3, last=2), -1), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), -1), (dict(n=(1 << 20) + 1), -2), (dict(shape=big), -2),
                    (dict(Lq=1 << 20), -2)):
        assert pick(**bad) == rc, bad

    def listed(Lq=8, q_start=0, scale=0.0, causal=1, Q=view(), cache=C.byref(kv), lists=4096, n=4, tk=None, tv=None, tail_len=0, lens=None, o=4096, lse=None, ws=4096, shape=s):
        return L.hs_listed_attn(shape, Lq, q_start, scale, causal, Q, cache, lists, n, tk, tv, tail_len, lens, o, lse, ws, None)

    one = dict(Lq=1, causal=0)
    uniform = hb.HsKV(k_map=4096, v_map=4096, uniform=1)
    for bad, rc in ((dict(Lq=0), -1), (dict(q_start=-1), -1), (dict(q_start=249), -1), (dict(scale=-1.0), -1), (dict(scale=math.nan), -1), (dict(Q=None), -1), (dict(cache=None), -1),
                    (dict(lists=None), -1), (dict(lists=4098), -1), (dict(n=0), -1), (dict(o=None), -1), (dict(o=4097), -1), (dict(lse=4098), -1), (dict(tk=4096), -1),
                    (dict(tv=4096), -1), (dict(tk=4096, tv=4096), -2), (dict(one, tk=4096, tv=4096, tail_len=65), -1), (dict(one, tk=4096, tv=4096, tail_len=-1), -1),
                    (dict(one, tk=4104, tv=4096), -1), (dict(one, ws=None, n=64), -1), (dict(one, ws=4104, n=64), -1), (dict(cache=C.byref(uniform)), -1), (dict(shape=big), -2),
                    (dict(Lq=(1 << 30) + 1, causal=0), -2), (dict(Lq=1 << 22, causal=0), -2), (dict(n=(1 << 20) + 1), -2), (dict(Q=view(token=4)), -1)):
        assert listed(**bad) == rc, bad
    size = C.c_size_t(0)
    for bad in ((0, 4, C.byref(size)), (1, 0, C.byref(size)), (1, 4, None)):
        assert L.hs_listed_attn_workspace_bytes(s, bad[0], bad[1], 0, bad[2]) == -1
    assert hb.listed_attn_workspace_bytes(hb.make_shape(64, 32, 8, 65536), 1, 64, True) == 0
    assert L.hs_listed_attn_workspace_bytes(s, 1, (1 << 20) + 1, 0, C.byref(size)) == -2 and L.hs_listed_attn_workspace_bytes(big, 1, 4, 0, C.byref(size)) == -2
    for n in (1, 5, 1 << 20):
        for Lq in (1, 2, 100, 5000):
            assert 0 <= hb.listed_attn_workspace_bytes(sh, Lq, n) <= 16 << 20


def test_refusals_of_the_binding():
    """Tensors that are not where or what the call takes, numbers beyond 32 bits."""
    sh = hb.make_shape(1, 4, 2, 128)
    q = torch.zeros((1, 4, 3, D), dtype=torch.bfloat16)
    kv = hb.PackedKV(sh, [0, 0, 2, 0, 2], "cpu")
    bounds, lists = torch.zeros((1, 2, 2, 2, D), dtype=torch.bfloat16), torch.zeros((1, 2, 3, 1), dtype=torch.int32)
    wrong = (hb.HsError, AssertionError)
    for call in (lambda: hb.tile_bounds(sh, kv), lambda: hb.query_scores(sh, q, bounds), lambda: hb.pick_tiles(sh, torch.zeros((1, 2, 3, 2)), 1),
                 lambda: hb.listed_attn(sh, q, kv, lists), lambda: hb.pick_tiles(sh, torch.zeros((1, 2, 3, 2)), 1 << 32),
                 lambda: hb.listed_attn_workspace_bytes(sh, 1, 1 << 32)):
        with pytest.raises(wrong):
            call()


@gpu
def test_refusals_of_the_binding_on_the_device():
    sh, kv, _, _, _ = _cache(1, 4, 2, 6, "bf16", "2:4", 1)
    q = torch.zeros((1, 4, 3, D), dtype=torch.bfloat16, device="cuda")
    bounds = hb.tile_bounds(sh, kv)
    scores = hb.query_scores(sh, q, bounds)
    lists = hb.pick_tiles(sh, scores, 2)
    tail = torch.zeros((1, 2, TILE, D), dtype=torch.bfloat16, device="cuda")
    wrong = (hb.HsError, AssertionError)
    for call in (lambda: hb.tile_bounds(sh, kv, 6), lambda: hb.tile_bounds(sh, kv, -1), lambda: hb.tile_bounds(sh, kv, 0, 7), lambda: hb.tile_bounds(sh, kv, out=bounds[:, :1]),
                 lambda: hb.tile_bounds(sh, kv, out=bounds.half()), lambda: hb.query_scores(sh, q.half(), bounds), lambda: hb.query_scores(sh, q, bounds[:, :, :5]),
                 lambda: hb.query_scores(sh, q, bounds, kv.k_map[:, :, :5]), lambda: hb.query_scores(sh, q, bounds, q_start=400), lambda: hb.query_scores(sh, q[..., :64], bounds),
                 lambda: hb.pick_tiles(sh, scores, 0), lambda: hb.pick_tiles(sh, scores, 2, 1, 2), lambda: hb.pick_tiles(sh, scores[..., :5], 2), lambda: hb.pick_tiles(sh, scores.half(), 2),
                 lambda: hb.listed_attn(sh, q, kv, lists.long()), lambda: hb.listed_attn(sh, q, kv, lists[:, :, :2]), lambda: hb.listed_attn(sh, q, kv, lists, q_start=1 << 33),
                 lambda: hb.listed_attn(sh, q, kv, lists, tail_k=tail), lambda: hb.listed_attn(sh, q, kv, lists, tail_k=tail, tail_v=tail, tail_len=3),
                 lambda: hb.listed_attn(sh, q[:, :, 0], kv, lists[:, :, 0].contiguous(), tail_k=tail, tail_v=tail, tail_len=65),
                 lambda: hb.listed_attn(sh, q, kv, lists, scale=-1.0), lambda: hb.listed_attn(sh, q, kv, lists, out=torch.empty((1, 4, 2, D), dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(wrong):
            call()
