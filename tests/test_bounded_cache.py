"""The operators around a bounded cache: rotary positions, attention mass, eviction of tiles in place, choice of tokens.  GPU tests hold the
library against oracle/hs_bounded.py (64 bits); refusals are looked at on the CPU."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import hs_bounded as ref
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


# ---------------------------------------------------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------------------------------------------------
SCALINGS = {"plain": (hb.ROPE_PLAIN, {}), "linear": (hb.ROPE_LINEAR, dict(factor=4.0)), "stretch": (hb.ROPE_STRETCH, dict(factor=8.0)),
            "bands": (hb.ROPE_BANDS, dict(factor=8.0, low=1.0, high=4.0, trained=8192)),
            "ramp": (hb.ROPE_RAMP, dict(factor=16.0, low=1.0, high=32.0, trained=4096))}


def _rope(rot, pairs, scaling, base):
    kind, extra = SCALINGS[scaling]
    rope = hb.make_rope(rot_dim=rot, layout=hb.ROPE_PAIRS if pairs else hb.ROPE_HALVES, base=base, scaling=kind, **extra)
    return rope, ref.rope_angles(rot, base, scaling, **extra)


@pytest.mark.parametrize("scaling", sorted(SCALINGS))
@pytest.mark.parametrize("rot,base", [(128, 10000.0), (128, 500000.0), (64, 1e6), (16, 10000.0), (96, 150.0)])
def test_rope_plan_holds_the_angles(rot, base, scaling):
    """Turns per position in units of 2^-64: theta / 2 pi to the last bits of a double (a few roundings of 2^-53)."""
    rope, (theta, gain) = _rope(rot, False, scaling, base)
    assert (rope.rot_dim, rope.layout) == (rot, hb.ROPE_HALVES)
    assert abs(rope.gain - gain) <= 2.0 ** -23
    for i in range(64):
        want = theta[i] / (2 * math.pi) if i < rot // 2 else 0.0
        # pow(x, y) in two ways differs by a few units of the last place of its result times |y ln x|; a turn is a whole number of
        # units of 2^-64, so the nearest one is up to 2^-65 away
        assert abs(rope.turn[i] / 2.0 ** 64 - want) <= 2.0 ** -53 * 64 * want + 2.0 ** -65, i


def _close_rope(got, want, size, dtype, gain, what):
    """One rounding to 16 bits (half a step), and at most 8 2^-24 of the magnitudes that a value is made of: the angle in half turns is
    rounded to 24 bits (pi 2^-25 radians) and cut to 32 (pi 2^-32), sine and cosine are good to 2 units, gain, products and the sum are
    rounded once each."""
    u = torch.finfo(dtype).eps / 2
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    err = np.abs(got - want)
    assert np.isfinite(got).all(), what
    assert (err <= u * np.abs(want) + (1 + u) * 8 * 2.0 ** -24 * size + tiny).all(), (what, err.max())


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,n,rot,scaling", [(1, 32, 8, 1, 128, "plain"), (1, 1, 1, 1, 16, "plain"), (3, 14, 2, 77, 64, "ramp"), (2, 8, 8, 2, 96, "bands"),
                                                    (5, 4, 1, 1, 128, "stretch"), (64, 32, 8, 1, 128, "bands"), (1, 7, 1, 1000, 128, "linear"),
                                                    (2, 32, 8, 513, 32, "plain"), (1, 24, 3, 4100, 112, "bands")])
def test_rope(B, Hq, Hkv, n, rot, scaling, pairs, dtype):
    t = TYPES[dtype]
    rope, (theta, gain) = _rope(rot, pairs, scaling, 10000.0)
    g = _gen(B * 1000 + n)
    qkv = torch.randn((B, n, Hq + 2 * Hkv, D), generator=g).to(t).cuda()
    pos = torch.randint(-5000, 200000, (B, n), generator=g, dtype=torch.int32)
    sh = hb.make_shape(B, Hq, Hkv, TILE, dtype=t)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    qo, ko, vo = hb.rope_qkv(sh, rope, q, k, v, positions=pos.cuda())
    for name, x, y in (("q", q, qo), ("k", k, ko)):
        want, size = ref.rope(_f64(x), pos.numpy(), theta, gain, pairs)
        _close_rope(_f64(y.transpose(1, 2)), want, size, t, gain, name)
        assert torch.equal(_bits(y.transpose(1, 2)[..., rot:]), _bits(x[..., rot:])), name
    assert torch.equal(_bits(vo.transpose(1, 2)), _bits(v))
    # parts of it alone give the same bits
    assert torch.equal(_bits(hb.rope_qkv(sh, rope, q=q, positions=pos.cuda())[0]), _bits(qo))
    _, k2, none = hb.rope_qkv(sh, rope, k=k, positions=pos.cuda())
    assert none is None and torch.equal(_bits(k2), _bits(ko))


@gpu
@pytest.mark.parametrize("pairs", [False, True])
def test_rope_beyond_the_last_level_cache(pairs):
    """A call of more than 256 MB gives the bits of its parts."""
    sh = hb.make_shape(2, 32, 8, TILE)
    rope, _ = _rope(128, pairs, "bands", 500000.0)
    qkv = torch.randn((2, 8200, 48, D), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    pos = torch.arange(8200, dtype=torch.int32, device="cuda").repeat(2, 1) + 77
    whole = hb.rope_qkv(sh, rope, qkv[:, :, :32], qkv[:, :, 32:40], qkv[:, :, 40:], positions=pos)
    for i in range(0, 8200, 1025):
        x = qkv[:, i:i + 1025]
        part = hb.rope_qkv(sh, rope, x[:, :, :32], x[:, :, 32:40], x[:, :, 40:], positions=pos[:, i:i + 1025].contiguous())
        assert all(torch.equal(a[:, :, i:i + 1025], b) for a, b in zip(whole, part)), i


@gpu
@pytest.mark.parametrize("first", [0, 1, -1, 131071, (1 << 31) - 1, -(1 << 31)])
def test_rope_positions_near_and_far(first):
    """The angle of any int32 position is exact: positions that are a run from `first`, against 64 bits (whose own angle is off by 2^-53 of
    position times theta, at most 2^-22 radians at 2^31)."""
    sh = hb.make_shape(2, 2, 1, TILE)
    rope, (theta, gain) = _rope(128, False, "plain", 10000.0)
    n = 1 if abs(first) > 1 << 30 else 5
    q = torch.randn((2, n, 2, D), generator=_gen(3)).to(torch.bfloat16).cuda()
    out, _, _ = hb.rope_qkv(sh, rope, q=q, positions=first)
    pos = first + np.arange(n)[None, :].repeat(2, 0)
    want, size = ref.rope(_f64(q), pos, theta, gain, False)
    _close_rope(_f64(out.transpose(1, 2)), want, size * 4, torch.bfloat16, gain, first)


@gpu
def test_rope_zero_position_and_back():
    """At position 0 vectors come out bit for bit; a turn by p and one by -p leave a vector within two roundings."""
    sh = hb.make_shape(1, 4, 2, TILE)
    for pairs in (False, True):
        rope, _ = _rope(128, pairs, "plain", 10000.0)
        x = torch.randn((1, 9, 4, D), generator=_gen(4)).to(torch.bfloat16).cuda()
        assert torch.equal(_bits(hb.rope_qkv(sh, rope, q=x, positions=torch.zeros((1, 9), dtype=torch.int32, device="cuda"))[0].transpose(1, 2)), _bits(x))
        p = torch.arange(700, 709, dtype=torch.int32, device="cuda")[None]
        y = hb.rope_qkv(sh, rope, q=x, positions=p)[0].transpose(1, 2)
        z = hb.rope_qkv(sh, rope, q=y, positions=-p)[0].transpose(1, 2)
        # both channels of a pair are rounded (2^-8 of each), then turned back and rounded again
        r = _f64(x).reshape(1, 9, 4, 64, 2) if pairs else np.stack([_f64(x)[..., :64], _f64(x)[..., 64:]], -1)
        size = np.abs(r).sum(-1, keepdims=True)
        w = _f64(z).reshape(1, 9, 4, 64, 2) if pairs else np.stack([_f64(z)[..., :64], _f64(z)[..., 64:]], -1)
        assert (np.abs(w - r) <= 3 * 2.0 ** -8 * size).all()


@gpu
@pytest.mark.parametrize("n", [1, 3])
def test_rope_into_rows_of_the_tail(n):
    """New keys and values go to each sequence's own rows of the tail buffer; everything else in it stays."""
    B, Hq, Hkv = 6, 8, 2
    sh = hb.make_shape(B, Hq, Hkv, TILE, dtype=torch.float16)
    rope, _ = _rope(128, False, "plain", 10000.0)
    g = _gen(n)
    q, k, v = (torch.randn((B, n, h, D), generator=g).half().cuda() for h in (Hq, Hkv, Hkv))
    tk, tv = (torch.randn((B, Hkv, TILE, D), generator=g).half().cuda() for _ in range(2))
    rows = torch.tensor([0, 63, 5, -n, 64, 64 - n], dtype=torch.int32)       # two sequences take no part; with n = 3 one keeps its first token only
    pos = torch.randint(0, 5000, (B, n), generator=g, dtype=torch.int32).cuda()
    _, k_all, v_all = hb.rope_qkv(sh, rope, q, k, v, positions=pos)
    want_k, want_v = tk.clone(), tv.clone()
    for b in range(B):
        for i in range(n):
            r = int(rows[b]) + i
            if 0 <= r < TILE:
                want_k[b, :, r], want_v[b, :, r] = k_all[b, :, i], v_all[b, :, i]
    out = hb.rope_qkv(sh, rope, q, k, v, positions=pos, k_out=tk, v_out=tv, rows=rows.cuda())
    assert out[1] is tk and out[2] is tv
    assert torch.equal(_bits(tk), _bits(want_k)) and torch.equal(_bits(tv), _bits(want_v))


@gpu
def test_rope_strides_and_in_place():
    B, Hq, Hkv, n = 2, 6, 3, 21
    sh = hb.make_shape(B, Hq, Hkv, TILE)
    rope, _ = _rope(64, True, "linear", 10000.0)
    g = _gen(8)
    q, k = (torch.randn((B, n, h, D), generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hkv))
    pos = torch.arange(n, dtype=torch.int32, device="cuda").repeat(B, 1)
    qo, ko, vo = hb.rope_qkv(sh, rope, q, k, k, positions=pos)
    # head-major inputs, outputs inside larger tensors, values broadcast from one head
    big = torch.full((B, Hq, n + 7, 2 * D), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big[:, :, 3:3 + n, D:]
    hb.rope_qkv(sh, rope, q.transpose(1, 2).contiguous().transpose(1, 2), positions=0, q_out=out)
    assert torch.equal(_bits(out), _bits(qo))
    rest = big.clone()
    rest[:, :, 3:3 + n, D:] = 7.0
    assert bool((rest == 7.0).all())
    one = k[:, :, :1].expand(B, n, Hkv, D)
    _, k1, v1 = hb.rope_qkv(sh, rope, None, k, one, positions=0)
    assert torch.equal(_bits(k1), _bits(ko)) and torch.equal(_bits(v1), _bits(one.transpose(1, 2)))
    hb.rope_qkv(sh, rope, q, positions=0, q_out=q.transpose(1, 2))           # in place
    assert torch.equal(_bits(q.transpose(1, 2)), _bits(qo))
    assert torch.equal(_bits(vo.transpose(1, 2)), _bits(k))


# ---------------------------------------------------------------------------------------------------------------------
# attention mass
# ---------------------------------------------------------------------------------------------------------------------
def _cache(B, Hkv, L, dtype, policy, seed, plant=None):
    """A packed cache, its keys as it holds them (64 bits) and the tiles that it holds."""
    t = TYPES[dtype]
    g = _gen(seed)
    K, V = (torch.randn((B, Hkv, L, D), generator=g).to(t) for _ in range(2))
    if plant is not None:
        plant(K)
    Hq = Hkv
    sh = hb.make_shape(B, Hq, Hkv, L, dtype=t)
    if policy.get("states"):
        T = L // TILE
        s = torch.randint(0, 3, (B, Hkv, T), generator=g).numpy().astype(np.int8)
        s[0, 0] = hb.SKIP                                                     # a row that holds nothing
        v = np.where(s == 0, 0, torch.randint(1, 3, (B, Hkv, T), generator=g).numpy()).astype(np.int8)
        pol = hb.make_policy(state_k=s, state_v=v)
    else:
        pol = hb.make_policy(**policy)
    kv = hb.compress_kv(sh, pol, K.cuda(), V.cuda())
    Ku, _ = hb.unpack_kv(sh, kv)
    return kv, _f64(Ku), kv.k_map.cpu().numpy() != 0, g


POLICIES = {"2:4": dict(), "dense": dict(sparse_frac_k=0.0, sparse_frac_v=0.0), "half": dict(sparse_frac_k=0.5, skip_frac=0.25), "states": dict(states=True)}


def _mass_case(B, Hkv, G, L, Lq, dtype, policy, causal, q_start, seed, plant=None):
    kv, K, held, g = _cache(B, Hkv, L, dtype, POLICIES[policy], seed, plant)
    sh = hb.make_shape(B, Hkv * G, Hkv, L, dtype=TYPES[dtype])
    Q = torch.randn((B, Hkv * G, Lq, D), generator=g).to(TYPES[dtype])
    # plausible log-sum-exps, not tied to these scores: the operator takes them as they are
    lse = torch.randn((B, Hkv * G, Lq), generator=g) + math.log(L)
    return kv, K, held, sh, Q, lse


def _tiles(x):
    return x.reshape(*x.shape[:2], -1, TILE).sum(-1)


def _check_mass(got, want, tol, before, decay, per_token, what):
    if not per_token:
        want, tol = _tiles(want), _tiles(tol) + TILE * 2.0 ** -24 * _tiles(want)
    old = 0.0 if before is None or decay == 0 else decay * _f64(before)
    want = want + old
    err = np.abs(_f64(got) - want)
    assert (err <= tol + 2 * 2.0 ** -24 * (np.abs(want) + np.abs(old)) + 1e-37).all(), (what, err.max())


@gpu
@pytest.mark.parametrize("policy", sorted(POLICIES))
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("B,Hkv,G,L,Lq,causal", [(1, 1, 1, 64, 1, False), (2, 2, 4, 640, 1, False), (1, 3, 7, 320, 1, True), (1, 2, 8, 1024, 16, True),
                                                 (2, 1, 4, 448, 100, True), (1, 1, 5, 192, 192, True), (1, 2, 1, 128, 33, False), (1, 8, 4, 2048, 77, True),
                                                 (1, 1, 2, 64, 1000, False), (3, 1, 3, 1280, 640, True)])
def test_mass(B, Hkv, G, L, Lq, causal, dtype, policy):
    q_start = L - Lq
    kv, K, held, sh, Q, lse = _mass_case(B, Hkv, G, L, Lq, dtype, policy, causal, q_start, 5 * L + Lq)
    want, tol = ref.attention_mass(_f64(Q), K, lse.numpy(), held, 1 / math.sqrt(D), causal, q_start)
    Qd, ld = Q.cuda(), lse.cuda()
    for per_token in (False, True):
        got = hb.attn_mass(sh, Qd, ld, kv, per_token=per_token, causal=causal)
        _check_mass(got, want, tol, None, 1.0, per_token, "new")
        before = torch.rand(got.shape, generator=_gen(1)).cuda()
        for decay in (0.0, 0.75, 1.0):
            add = hb.attn_mass(sh, Qd, ld, kv, mass=before, out=torch.full_like(before, math.nan), per_token=per_token, causal=causal, decay=decay)
            _check_mass(add, want, tol, before, decay, per_token, decay)
        mine = before.clone()
        assert hb.attn_mass(sh, Qd, ld, kv, mass=mine, per_token=per_token, causal=causal) is mine         # in place, the same bits
        assert torch.equal(mine, add)


@gpu
@pytest.mark.parametrize("q_start,Lq", [(0, 1), (0, 65), (63, 2), (100, 200), (37, 283)])
def test_mass_of_queries_inside_the_cache(q_start, Lq):
    kv, K, held, sh, Q, lse = _mass_case(2, 2, 3, 320, Lq, "bf16", "half", True, q_start, q_start)
    want, tol = ref.attention_mass(_f64(Q), K, lse.numpy(), held, 0.125, True, q_start)
    for per_token in (False, True):
        got = hb.attn_mass(sh, Q.cuda(), lse.cuda(), kv, per_token=per_token, causal=True, q_start=q_start, scale=0.125)
        _check_mass(got, want, tol, None, 1.0, per_token, q_start)


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("policy", ["2:4", "dense", "half"])
def test_mass_is_the_column_sum_of_the_attention_it_follows(dtype, policy):
    """With the LSE that prefill and decode return the weights of a query add up to 1: those of all to the number of queries (each LSE is off by
    at most 1e-4, the parity tests' bound)."""
    B, Hkv, G, L = 1, 2, 4, 1024
    kv, K, held, sh, Q, _ = _mass_case(B, Hkv, G, L, 256, dtype, policy, True, L - 256, 77)
    _, lse = hb.prefill_attn(sh, Q.cuda(), kv)
    got = hb.attn_mass(sh, Q.cuda(), lse, kv)
    assert np.allclose(_f64(got).sum(-1), G * 256, rtol=3e-4)
    want, tol = ref.attention_mass(_f64(Q), K, lse.cpu().numpy(), held, 1 / math.sqrt(D), True, L - 256)
    _check_mass(got, want, tol, None, 1.0, False, "prefill")
    q = Q[:, :, -1].contiguous().cuda()
    _, lse1 = hb.decode_attn(sh, q, kv)
    got = hb.attn_mass(sh, q, lse1, kv)
    assert np.allclose(_f64(got).sum(-1), G, rtol=3e-4)
    # views: the last queries of the prompt
    part = hb.attn_mass(sh, Q.cuda()[:, :, -32:], lse[:, :, -32:], kv)
    whole = hb.attn_mass(sh, Q[:, :, -32:].contiguous().cuda(), lse[:, :, -32:].contiguous(), kv)
    assert torch.equal(part, whole)


@gpu
@pytest.mark.parametrize("Lq", [1, 40])
@pytest.mark.parametrize("policy", ["2:4", "dense"])
def test_mass_of_queries_that_saw_nothing_and_of_keys_that_are_nan(policy, Lq):
    """Queries of LSE -inf, NaN and inf weigh nothing, whatever the keys hold; a key of NaN gives NaN only to a query of finite LSE that sees it."""
    def plant(K):
        K[0, 0, 100, 3] = math.nan
        K[0, 1, 5, 0] = math.inf
    kv, K, held, sh, Q, lse = _mass_case(1, 2, 2, 192, Lq, "bf16", policy, False, 0, 9, plant)
    lse[:] = math.nan                                    # what attention gives these queries
    lse[0, 0, 0], lse[0, 1, 0], lse[0, 2, 0] = -math.inf, math.inf, -math.inf
    for per_token in (False, True):
        got = hb.attn_mass(sh, Q.cuda(), lse.cuda(), kv, per_token=per_token, causal=False)
        assert bool((got == 0).all())
    if Lq > 1:                                           # queries in front of the NaN do not see it
        lse[:, :, :30] = 4.0
        got = hb.attn_mass(sh, Q.cuda(), lse.cuda(), kv, per_token=True, causal=True, q_start=60)
        want, tol = ref.attention_mass(_f64(Q), K, lse.numpy(), held, 1 / math.sqrt(D), True, 60)
        _check_mass(got[:, :1], want[:, :1], tol[:, :1], None, 1.0, True, "before the NaN")


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows", [False, True])
def test_mass_with_a_dense_tail(rows, dtype):
    """The tail's tokens count to the tile that they will be appended as."""
    B, Hkv, G, L = 5, 2, 4, 512
    T = L // TILE
    g = _gen(12)
    sh = hb.make_shape(B, Hkv * G, Hkv, L, dtype=TYPES[dtype])
    K, V = (torch.randn((B, Hkv, L, D), generator=g).to(TYPES[dtype]) for _ in range(2))
    n_held = [7, 3, 6, 1, 7] if rows else [6] * B
    s = np.zeros((B, Hkv, T), dtype=np.int8)
    for b, n in enumerate(n_held):
        s[b, :, :n] = hb.SPARSE24
    kv = hb.compress_kv(sh, hb.make_policy(state_k=s, state_v=s), K.cuda(), V.cuda())
    Ku, _ = hb.unpack_kv(sh, kv)
    tk, tv = (torch.randn((B, Hkv, TILE, D), generator=g).to(TYPES[dtype]) for _ in range(2))
    lens = [1, 64, 0, 37, 80] if rows else [17] * B
    tiles = [7, 3, 6, 1, -1] if rows else [6] * B                             # the last sequence's tail is left out
    tail_len = torch.tensor(lens, dtype=torch.int32, device="cuda") if rows else 17
    tail_tile = torch.tensor(tiles, dtype=torch.int32, device="cuda") if rows else 6
    q = torch.randn((B, Hkv * G, D), generator=g).to(TYPES[dtype]).cuda()
    _, lse = hb.decode_attn(sh, q, kv, tail_k=tk.cuda(), tail_v=tv.cuda(), tail_len=tail_len)
    Q64 = _f64(q)[:, :, None]
    want, tol = ref.attention_mass(Q64, _f64(Ku), lse.cpu().numpy()[:, :, None], s != 0, 1 / math.sqrt(D), False, 0)
    for b in range(B):
        n = min(lens[b], TILE)
        if n == 0 or not 0 <= tiles[b] < T:
            continue
        k = np.zeros((1, Hkv, TILE, D))
        k[0, :, :n] = _f64(tk)[b, :, :n]
        w, e = ref.attention_mass(Q64[b:b + 1], k, lse.cpu().numpy()[b:b + 1, :, None], np.ones((1, Hkv, 1), bool), 1 / math.sqrt(D), False, 0)
        at = tiles[b] * TILE
        want[b, :, at:at + n] += w[0, :, :n]
        tol[b, :, at:at + n] += e[0, :, :n]
    before = torch.rand((B, Hkv, T), generator=g).cuda()
    for per_token in (False, True):
        old = before if not per_token else before.repeat_interleave(TILE, -1).contiguous()
        got = hb.attn_mass(sh, q, lse, kv, mass=old, out=torch.empty_like(old), per_token=per_token, decay=0.5, tail_k=tk.cuda(), tail_len=tail_len,
                           tail_tile=tail_tile)
        _check_mass(got, want, tol, old, 0.5, per_token, "tail")
    if not rows:
        assert np.allclose((_f64(got) - 0.5 * _f64(old)).sum(-1), G, rtol=3e-4)


@gpu
@pytest.mark.parametrize("per_token", [False, True])
def test_mass_of_a_long_prompt_against_64_bits_on_the_device(per_token):
    """Sizes at which the queries are cut into ranges and at which they are not, a row of which is held against float64 on the GPU."""
    for B, Hkv, G, L, Lq in ((1, 8, 4, 4096, 4096), (1, 1, 8, 8192, 2500), (2, 8, 2, 16384, 300)):
        sh = hb.make_shape(B, Hkv * G, Hkv, L)
        g = torch.Generator(device="cuda").manual_seed(L)
        K, Q = torch.randn((B, Hkv, L, D), generator=g, device="cuda").bfloat16(), torch.randn((B, Hkv * G, Lq, D), generator=g, device="cuda").bfloat16()
        kv = hb.compress_kv(sh, hb.make_policy(), K, K)
        Ku, _ = hb.unpack_kv(sh, kv)
        lse = torch.empty((B, Hkv * G, Lq), device="cuda")
        at = torch.arange(L, device="cuda")
        b, h = B - 1, Hkv - 1
        want, size = torch.zeros(L, dtype=torch.float64, device="cuda"), torch.zeros(L, dtype=torch.float64, device="cuda")
        lse.fill_(-math.inf)                             # the other kv heads' queries are left out
        for j in range(h * G, (h + 1) * G):
            s = torch.matmul(Q[b, j].double(), Ku[b, h].double().t()) / math.sqrt(D)
            s.masked_fill_(at > (L - Lq + torch.arange(Lq, device="cuda"))[:, None], -math.inf)
            lse[b, j] = torch.logsumexp(s, -1).float()
            p = torch.exp(s - lse[b, j].double()[:, None])
            want += p.sum(0)
            size += torch.where(p > 0, p * (s.abs() + lse[b, j].double().abs()[:, None] + 1.0), 0.0).sum(0)
        got = hb.attn_mass(sh, Q, lse, kv, per_token=per_token).double()
        if not per_token:
            want, size = want.reshape(-1, TILE).sum(-1), size.reshape(-1, TILE).sum(-1)
        # arguments of the exponential: products of magnitude 11 at most, 4 2^-24 of each factor and 129 2^-24 of the score's parts (about
        # 11 times the spread of a score, which is 1); sums of up to 2^15 terms, each partial sum off by half a unit: 2^-24 sqrt of them in the mean
        tol = size * (4 + 129 / 2) * 2.0 ** -24 + want * 2.0 ** -15 * 2.0 ** -2
        assert bool(((got[b, h] - want).abs() <= tol).all()), (L, Lq, ((got[b, h] - want).abs() / tol).max())
        got[b, h] = 0
        assert bool((got == 0).all())


# ---------------------------------------------------------------------------------------------------------------------
# eviction of tiles
# ---------------------------------------------------------------------------------------------------------------------
def _random_cache(B, Hkv, T, held, sk, sv, seed, shuffle=False, room=0):
    """A cache of random bytes: `held` tiles of each row (an int or one number per row), share sk / sv of them 2:4."""
    rng = np.random.default_rng(seed)
    rows = B * Hkv
    held = np.broadcast_to(np.asarray(held), (rows,))
    maps, caps = [], []
    tiles = [np.sort(rng.permutation(T)[:n]) for n in held]
    for x, share in ((0, sk), (1, sv)):
        m = np.zeros((rows, T), dtype=np.int32)
        for r in range(rows):
            sparse = rng.random(len(tiles[r])) < share
            for sign, pick in ((1, tiles[r][~sparse]), (-1, tiles[r][sparse])):
                slots = np.arange(1, len(pick) + 1)
                m[r, pick] = sign * (rng.permutation(slots) if shuffle else slots)
            if x == 1:
                flagged = tiles[r][rng.random(len(tiles[r])) < 0.5]
                m[r, flagged] += np.sign(m[r, flagged]) * hb.MAP_F16
        plain = np.where(x == 1, np.sign(m) * (np.abs(m) & ~hb.MAP_F16), m)
        caps += [int(max(0, plain.max())) + room, int(max(0, -plain.min())) + room]
        maps.append(m)
    sh = hb.make_shape(B, Hkv, Hkv, T * TILE)
    kv = hb.PackedKV(sh, [0] + caps, "cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    for name in ("k_dense", "k_nnz", "k_meta", "v_dense", "v_nnz", "v_meta"):
        t = getattr(kv, name)
        if t is not None:
            t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    kv.k_map.copy_(torch.from_numpy(maps[0]).reshape(B, Hkv, T))
    kv.v_map.copy_(torch.from_numpy(maps[1]).reshape(B, Hkv, T))
    return sh, kv, maps


POOLS = {"k_dense": (("k_dense", 16384),), "k_sparse": (("k_nnz", 8192), ("k_meta", 1024)), "v_dense": (("v_dense", 16384),),
         "v_sparse": (("v_nnz", 8192), ("v_meta", 1024))}


def _pool(kv, name, rows, size):
    t = getattr(kv, name)
    return None if t is None else t.view(rows, -1, size)


def _check_evict(sh, kv, maps, mass, keep, first, last, call):
    rows, T = sh.B * sh.Hkv, sh.L // TILE
    want = {n: _pool(kv, n, rows, s).cpu().clone() for p in POOLS.values() for n, s in p if getattr(kv, n) is not None}
    k, v, moves = ref.evict(maps[0], maps[1], mass.reshape(rows, T), np.broadcast_to(np.asarray(keep).reshape(-1), (rows,)), first, last)
    for r, row in enumerate(moves):
        for pool, pairs in row.items():
            for n, _ in POOLS[pool]:
                for frm, to in pairs:
                    want[n][r, to] = want[n][r, frm]
    call()
    assert (kv.k_map.cpu().numpy().reshape(rows, T) == k).all()
    assert (kv.v_map.cpu().numpy().reshape(rows, T) == v).all()
    for n, w in want.items():
        assert torch.equal(getattr(kv, n).view(w.shape).cpu(), w), n
    return k, v


@gpu
@pytest.mark.parametrize("B,Hkv,T,held,sk,sv", [(1, 1, 1, 1, 1.0, 1.0), (1, 2, 5, 5, 1.0, 0.0), (2, 3, 70, 50, 0.5, 0.5), (2, 2, 300, 300, 0.0, 1.0),
                                                (1, 2, 256, 200, 0.97, 0.9), (1, 1, 1025, 900, 0.5, 1.0), (2, 1, 1500, 700, 0.2, 0.6), (1, 2, 4200, 300, 0.9, 0.8)])
@pytest.mark.parametrize("shuffle", [False, True])
def test_evict(B, Hkv, T, held, sk, sv, shuffle):
    for keep, first, last in ((1, 0, 0), (max(1, held - 1), 1, 4), (max(1, held // 4), 1, 4), (max(1, held // 2), 0, 3), (3, 2, 7), (held, 0, 0), (held + 5, 9, 9),
                              (1, held, 0), (2, 0, held + 3)):
        sh, kv, maps = _random_cache(B, Hkv, T, held, sk, sv, 100 * T + keep, shuffle)
        mass = np.random.default_rng(keep).random((B, Hkv, T)).astype(np.float32)
        _check_evict(sh, kv, maps, mass, keep, first, last, lambda: hb.evict_tiles(sh, kv, torch.from_numpy(mass).cuda(), keep, first=first, last=last))
        assert kv.uniform == 0


@gpu
def test_evict_ties_zeros_nan_and_infinities():
    B, Hkv, T = 2, 2, 90
    values = np.array([0.0, -0.0, 1.0, 1.0, np.nan, np.inf, -np.inf, 3e-45, -2.0], dtype=np.float32)
    for keep in (80, 60, 45, 20, 5):
        sh, kv, maps = _random_cache(B, Hkv, T, T, 0.5, 0.5, keep, True)
        mass = values[np.random.default_rng(keep).integers(0, len(values), (B, Hkv, T))]
        _check_evict(sh, kv, maps, mass, keep, 1, 2, lambda: hb.evict_tiles(sh, kv, torch.from_numpy(mass).cuda(), keep, first=1, last=2))


@gpu
def test_evict_rows_of_their_own_length_and_budget():
    """Rows hold and keep different numbers of tiles, one of them none; rooms beyond the slots in use; a second eviction goes on from the first."""
    B, Hkv, T = 3, 2, 130
    sh, kv, maps = _random_cache(B, Hkv, T, [130, 0, 1, 64, 65, 100], 0.6, 0.3, 5, room=3)
    for step, keep in enumerate(([40, 5, 1, 64, 1, -3], [30, 5, 1, 7, 1, 1])):
        mass = np.random.default_rng(step).random((B, Hkv, T)).astype(np.float32)
        ws = torch.randint(0, 256, (hb.workspace_bytes(sh, hb.OP_EVICT),), dtype=torch.uint8, device="cuda")
        budget = torch.tensor(keep, dtype=torch.int32, device="cuda").reshape(B, Hkv)
        maps = _check_evict(sh, kv, maps, mass, np.maximum(keep, 1), 2, 1,
                            lambda: hb.evict_tiles(sh, kv, torch.from_numpy(mass).cuda(), budget, first=2, last=1, workspace=ws))


@gpu
def test_evict_the_longest_row():
    T = 65536
    sh, kv, maps = _random_cache(1, 1, T, 2000, 1.0, 1.0, 6)
    mass = np.random.default_rng(1).random((1, 1, T)).astype(np.float32)
    _check_evict(sh, kv, maps, mass, 700, 1, 4, lambda: hb.evict_tiles(sh, kv, torch.from_numpy(mass).cuda(), 700, first=1, last=4))


@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("sk,sv", [(1.0, 1.0), (0.5, 1.0), (0.0, 0.5)])
def test_a_cache_after_eviction_is_a_cache(sk, sv, dtype):
    """Unpacking, attention, re-packing, mass and a further eviction see the cache that packing only the remaining tiles would have made."""
    B, Hkv, G, L = 2, 2, 4, 1536
    T, t = L // TILE, TYPES[dtype]
    g = _gen(31)
    K, V = (torch.randn((B, Hkv, L, D), generator=g).to(t).cuda() for _ in range(2))
    sh = hb.make_shape(B, Hkv * G, Hkv, L, dtype=t)
    kv = hb.compress_kv(sh, hb.make_policy(sparse_frac_k=sk, sparse_frac_v=sv), K, V)
    K0, V0 = hb.unpack_kv(sh, kv)
    states = [np.where(m > 0, hb.DENSE, np.where(m < 0, hb.SPARSE24, hb.SKIP)).astype(np.int8) for m in (kv.k_map.cpu().numpy(), kv.v_map.cpu().numpy())]
    mass = torch.rand((B, Hkv, T), generator=g)
    hb.evict_tiles(sh, kv, mass.cuda(), 9, first=1, last=2)
    gone = (kv.k_map == 0).cpu()
    assert bool(((~gone).sum(-1) == 9).all()) and torch.equal(gone, (kv.v_map == 0).cpu())
    keep = (~gone).repeat_interleave(TILE, -1).cuda()  # chooses rows; a product with 0 would make -0 of a negative value
    Ku, Vu = hb.unpack_kv(sh, kv)
    assert torch.equal(_bits(Ku[keep]), _bits(K0[keep])) and torch.equal(_bits(Vu[keep]), _bits(V0[keep]))
    for s in states:
        s[gone.numpy()] = hb.SKIP
    pol = hb.make_policy(state_k=states[0], state_v=states[1])
    fresh = hb.PackedKV(sh, kv.counts, "cuda")
    hb.compress_kv(sh, pol, K, V, out=fresh)
    hb.check_state_flag(pol)
    q = torch.randn((B, Hkv * G, 128, D), generator=g).to(t).cuda()
    for a, b in zip(hb.prefill_attn(sh, q, kv), hb.prefill_attn(sh, q, fresh)):
        assert torch.equal(a, b)
    d = q[:, :, 0].contiguous()
    for a, b in zip(hb.decode_attn(sh, d, kv), hb.decode_attn(sh, d, fresh)):
        assert torch.equal(a, b)
    lse = torch.full((B, Hkv * G, 128), 6.0, device="cuda")
    assert torch.equal(hb.attn_mass(sh, q, lse, kv), hb.attn_mass(sh, q, lse, fresh))
    one, other = (hb.recompress_kv(sh, x, hb.make_policy(dense_first_tiles=1, dense_last_tiles=1)) for x in (kv, fresh))
    assert torch.equal(one.k_map, other.k_map) and torch.equal(one.v_map, other.v_map)
    for a, b in zip(hb.unpack_kv(sh, one), hb.unpack_kv(sh, other)):
        assert torch.equal(_bits(a[keep]), _bits(b[keep]))
    # the last tile, dropped from every row by a mass of its own, comes back through an append
    lightest = torch.ones_like(mass)
    lightest[..., T - 1] = 0
    hb.evict_tiles(sh, kv, lightest.cuda(), 8)
    assert bool((kv.k_map[..., T - 1] == 0).all()) and bool(((kv.k_map != 0).sum(-1) == 8).all())
    over = torch.zeros(1, dtype=torch.int32, device="cuda")
    if sk == sv == 1.0:  # pools of one kind have the room in every row
        hb.append_tile(sh, kv, T - 1, K[:, :, -TILE:], V[:, :, -TILE:], overflow=over)
        assert int(over) == 0
        for a, b in zip(hb.unpack_kv(sh, kv), (K0, V0)):
            assert torch.equal(_bits(a[:, :, -TILE:]), _bits(b[:, :, -TILE:]))
    hb.evict_tiles(sh, kv, mass.cuda(), 4)
    assert int((kv.k_map != 0).sum(-1).max()) == 4


# ---------------------------------------------------------------------------------------------------------------------
# choice of tokens
# ---------------------------------------------------------------------------------------------------------------------
def _check_keep(sh, K, V, w, keep, first, last, lens):
    ko, vo, idx = hb.keep_tokens(sh, K, V, w, keep, first=first, last=last, lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"))
    n, wn = K.shape[2], w.cpu().numpy()
    for b in range(sh.B):
        m = n if lens is None else max(0, min(n, lens[b]))
        for h in range(sh.Hkv):
            t = ref.keep_tokens(wn[b, h], m, keep, first, last)
            assert idx[b, h].tolist() == t + [-1] * (keep - len(t)), (b, h)
            at = torch.tensor(t, dtype=torch.long, device="cuda")
            for x, y in ((K, ko), (V, vo)):
                assert torch.equal(_bits(y[b, h, :len(t)]), _bits(x[b, h, at]))
                assert not bool(_bits(y[b, h, len(t):]).any())


@gpu
@pytest.mark.parametrize("B,Hkv,n", [(1, 1, 1), (2, 3, 65), (1, 2, 1000), (3, 1, 1025), (2, 2, 5000)])
def test_keep_tokens(B, Hkv, n):
    for keep, first, last in ((1, 0, 0), (max(1, n // 10), 0, 0), (max(9, n // 3), 4, 5), (n, 0, 0), (n + 3, 2, 1), (7, 3, 4), (max(1, n - 1), 0, 0)):
        sh = hb.make_shape(B, Hkv, Hkv, TILE, dtype=torch.float16)
        g = _gen(n + keep)
        K, V = (torch.randn((B, Hkv, n, D), generator=g).half().cuda() for _ in range(2))
        w = torch.rand((B, Hkv, n), generator=g).cuda()
        _check_keep(sh, K, V, w, keep, first, last, None)
        _check_keep(sh, K, V, w, keep, first, last, [n, 0, 3 * n // 4][:B] if B > 1 else [n // 2])


@gpu
def test_keep_tokens_ties_zeros_nan_and_infinities():
    values = torch.tensor([0.0, -0.0, 1.0, 1.0, math.nan, math.inf, -math.inf, 3e-45, -2.0])
    sh = hb.make_shape(2, 4, 2, TILE)
    for n, keep in ((300, 40), (300, 100), (300, 290), (1500, 1000), (1500, 200)):
        g = _gen(keep)
        K, V = (torch.randn((2, 2, n, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        w = values[torch.randint(0, len(values), (2, 2, n), generator=g)].cuda()
        _check_keep(sh, K, V, w, keep, 1, 2, None)
    w = torch.full((2, 2, 1500), 0.25, device="cuda")                           # all alike
    _check_keep(sh, K, V, w, 200, 0, 0, [1500, 900])


@gpu
@pytest.mark.parametrize("kind", ["spread", "alike", "two values", "mostly zeros", "one bin", "special"])
def test_keep_tokens_of_rows_in_parts(kind):
    """Rows long enough to be ranked in parts: weights that differ, that are all or mostly the same, that share their upper bits (more of
    them than the list of a bin holds, and fewer), and ones that are not numbers."""
    sh = hb.make_shape(3, 2, 1, TILE)
    g = _gen(6)
    for n, keeps in ((4097, (1, 2000, 4096)), (30000, (300, 20000, 29999)), (32769, (70, 32768)), (70000, (50, 69000)), (140000, (9000,))):
        K, V = (torch.randn((3, 1, n, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        x = torch.rand((3, 1, n), generator=g)
        w = {"spread": torch.exp(4 * torch.randn((3, 1, n), generator=g)), "alike": torch.full((3, 1, n), 0.25), "two values": 1.0 + (x > 0.7).float(),
             "mostly zeros": torch.where(x > 0.9, x, 0.0), "one bin": 1.0 + x / 8, "special": torch.where(x > 0.5, x, torch.where(x > 0.3, math.nan, torch.where(x > 0.1, -math.inf, -x)))}[kind]
        for keep in keeps:
            _check_keep(sh, K, V, w.cuda(), keep, min(keep // 3, 40), min(keep // 3, 70), [n, n // 2 + 7, keep + 1])
    _check_keep(sh, K, V, w.cuda(), 400, 150, 250, None)                        # none but the ends
    _check_keep(sh, K, V, w.cuda(), 140000, 1, 2, [140000, 0, 139999])          # all of them


@gpu
def test_keep_tokens_of_views_and_long_rows():
    sh = hb.make_shape(1, 2, 2, TILE)
    g = torch.Generator(device="cuda").manual_seed(4)
    n = 70001
    fused = torch.randn((1, n + 5, 6, D), generator=g, device="cuda").bfloat16()
    K, V = fused[:, 5:, 1:3].transpose(1, 2), fused[:, 2:2 + n, 3:5].transpose(1, 2)
    w = torch.exp(3 * torch.randn((1, 3, n + 9), generator=g, device="cuda"))[:, 1:, 4:4 + n]
    _check_keep(sh, K, V, w, 5000, 64, 256, None)


@gpu
@pytest.mark.parametrize("n,alike", [(600001, False), (600001, True), (1 << 20, False)])
def test_keep_tokens_of_the_longest_rows(n, alike):
    sh = hb.make_shape(1, 1, 1, TILE)
    g = torch.Generator(device="cuda").manual_seed(n)
    K = torch.randn((1, 1, n, D), generator=g, device="cuda").bfloat16()
    w = torch.full((1, 1, n), 3.0, device="cuda") if alike else torch.rand((1, 1, n), generator=g, device="cuda")
    _check_keep(sh, K, K, w, 1000, 4, 32, None)


# ---------------------------------------------------------------------------------------------------------------------
# together, captured, refused
# ---------------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_serving_with_a_bounded_cache(dtype):
    """A prompt's best tokens become the cache, then every step rotates its token into the tail, attends, gathers the tiles' weight, and every 64
    steps the tail is appended and the lightest tile dropped.  At every step the call's output is that of plain attention over the
    tokens that the cache and the tail hold then."""
    t = TYPES[dtype]
    B, Hq, Hkv, n, keep, budget = 2, 8, 2, 700, 256, 5
    G, cap = Hq // Hkv, 8 * TILE
    g = _gen(20)
    rope = hb.make_rope(base=10000.0)
    sh = hb.make_shape(B, Hq, Hkv, cap, dtype=t)
    proj = torch.randn((B, n, Hq + 2 * Hkv, D), generator=g).to(t).cuda()
    # prompt: rotated, attended to densely in whole tiles, weighed by its last 48 queries, cut down to its `keep` best tokens
    whole = n // TILE * TILE
    q, k, v = hb.rope_qkv(sh, rope, proj[:, :, :Hq], proj[:, :, Hq:Hq + Hkv], proj[:, :, Hq + Hkv:])
    ps = hb.make_shape(B, Hq, Hkv, whole, dtype=t)
    pk = hb.compress_kv(ps, hb.make_policy(sparse_frac_k=0.0, sparse_frac_v=0.0), k[:, :, :whole], v[:, :, :whole])
    _, lse = hb.prefill_attn(ps, q[:, :, :whole].contiguous(), pk)
    w = hb.attn_mass(ps, q[:, :, whole - 48:whole], lse[:, :, -48:], pk, per_token=True)
    ko, vo, idx = hb.keep_tokens(sh, k[:, :, :whole], v[:, :, :whole], w, keep, first=4, last=32)
    assert bool((idx[:, :, 1:] > idx[:, :, :-1]).all()) and bool((idx[:, :, -32:] == torch.arange(whole - 32, whole, device="cuda")).all())
    # a cache with room for 8 tiles of positions and budget + 1 slots
    states = np.zeros((B, Hkv, 8), dtype=np.int8)
    states[:, :, :keep // TILE] = hb.SPARSE24
    full_k, full_v = (torch.zeros((B, Hkv, cap, D), dtype=t, device="cuda") for _ in range(2))
    full_k[:, :, :keep], full_v[:, :, :keep] = ko, vo
    kv = hb.PackedKV(sh, [0, 0, budget + 1, 0, budget + 1], "cuda")
    hb.compress_kv(sh, hb.make_policy(state_k=states, state_v=states), full_k, full_v, out=kv)
    tail_k, tail_v = (torch.zeros((B, Hkv, TILE, D), dtype=t, device="cuda") for _ in range(2))
    mass = torch.zeros((B, Hkv, 8), device="cuda")
    next_tile, tail_len = keep // TILE, 0
    for step in range(3 * TILE + 5):
        x = torch.randn((B, 1, Hq + 2 * Hkv, D), generator=g).to(t).cuda()
        q1, _, _ = hb.rope_qkv(sh, rope, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], positions=n + step, k_out=tail_k, v_out=tail_v, rows=tail_len)
        tail_len += 1
        q1 = q1[:, :, 0]
        O, lse1 = hb.decode_attn(sh, q1, kv, tail_k=tail_k, tail_v=tail_v, tail_len=tail_len)
        before = mass.clone()
        hb.attn_mass(sh, q1, lse1, kv, mass=mass, tail_k=tail_k, tail_len=tail_len, tail_tile=next_tile, causal=False)
        assert np.allclose(_f64(mass - before).sum(-1), G, rtol=1e-3)
        if step % 16 == 0 or tail_len == TILE:
            Ku, Vu = hb.unpack_kv(sh, kv)
            held = (kv.k_map != 0).repeat_interleave(TILE, -1)
            for b in range(B):
                for h in range(Hkv):
                    kk = torch.cat([Ku[b, h][held[b, h]], tail_k[b, h, :tail_len]]).double()
                    vv = torch.cat([Vu[b, h][held[b, h]], tail_v[b, h, :tail_len]]).double()
                    qq = q1[b, h * G:(h + 1) * G].double()
                    want = _f64(torch.softmax(qq @ kk.t() / math.sqrt(D), -1) @ vv)
                    err = np.abs(_f64(O[b, h * G:(h + 1) * G]) - want)
                    assert err.max() <= 1e-2 * np.abs(want).max() and err.mean() <= 2.5e-3 * np.abs(want).mean()
        if tail_len == TILE:
            over = torch.zeros(1, dtype=torch.int32, device="cuda")
            hb.append_tile(sh, kv, next_tile, tail_k, tail_v, overflow=over)
            assert int(over) == 0
            hb.evict_tiles(sh, kv, mass, budget, first=1, last=1)
            held = kv.k_map != 0
            assert int(held.sum(-1).max()) <= budget and bool(held[..., 0].all()) and bool(held[..., next_tile].all())
            next_tile, tail_len = next_tile + 1, 0


@gpu
def test_captured_calls_replay():
    """Each call captured once and replayed with other inputs in the same buffers, eager work between the replays; two captured graphs with
    workspaces of their own."""
    B, Hq, Hkv, L = 2, 8, 2, 1024
    T = L // TILE
    sh = hb.make_shape(B, Hq, Hkv, L)
    rope = hb.make_rope()
    g = torch.Generator(device="cuda").manual_seed(1)

    def normal(*sizes):
        return torch.randn(sizes, generator=g, device="cuda").bfloat16()

    K, V, x = normal(B, Hkv, L, D), normal(B, Hkv, L, D), normal(B, 1, Hq + 2 * Hkv, D)
    kv = hb.compress_kv(sh, hb.make_policy(sparse_frac_k=0.5), K, V)
    kv.uniform = 0
    backup = (kv.k_map.clone(), kv.v_map.clone())
    pools = {n: getattr(kv, n).clone() for p in POOLS.values() for n, _ in p if getattr(kv, n) is not None}
    tk, tv, pos = normal(B, Hkv, TILE, D), normal(B, Hkv, TILE, D), torch.full((B, 1), 5, dtype=torch.int32, device="cuda")
    rows = torch.zeros(B, dtype=torch.int32, device="cuda")
    mass, Qp, lse = torch.rand((B, Hkv, T), generator=g, device="cuda"), normal(B, Hq, 200, D), torch.full((B, Hq, 200), 7.0, device="cuda")
    w = torch.rand((B, Hkv, L), generator=g, device="cuda")
    ws_m = torch.empty(max(16, hb.attn_mass_workspace_bytes(sh, 200)), dtype=torch.uint8, device="cuda")
    ws_e = torch.empty(hb.workspace_bytes(sh, hb.OP_EVICT), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(mass)

    def calls():
        q1, _, _ = hb.rope_qkv(sh, rope, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], positions=pos, k_out=tk, v_out=tv, rows=rows)
        hb.attn_mass(sh, Qp, lse, kv, mass=mass, out=out, workspace=ws_m)
        kept = hb.keep_tokens(sh, K, V, w, 100, first=3, last=7)
        hb.evict_tiles(sh, kv, out, 6, first=1, last=2, workspace=ws_e)
        return [q1, tk, tv, out, *kept, kv.k_map, kv.v_map]

    def reset():
        kv.k_map.copy_(backup[0]), kv.v_map.copy_(backup[1])
        for n, p in pools.items():
            getattr(kv, n).copy_(p)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for i in range(4):
        x.copy_(normal(*x.shape)), Qp.copy_(normal(*Qp.shape)), pos.fill_(1000 * i + 3), rows.fill_(i)
        lse.uniform_(5.0, 9.0), w.uniform_(), mass.uniform_()
        reset()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        reset()
        for a, b in zip(got, calls()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


@gpu
def test_calls_go_to_the_current_stream_and_equal_calls_give_equal_bits():
    sh = hb.make_shape(1, 8, 2, 4096)
    g = torch.Generator(device="cuda").manual_seed(2)
    K, Q = torch.randn((1, 2, 4096, D), generator=g, device="cuda").bfloat16(), torch.randn((1, 8, 1111, D), generator=g, device="cuda").bfloat16()
    kv = hb.compress_kv(sh, hb.make_policy(), K, K)
    lse = torch.full((1, 8, 1111), 8.0, device="cuda")
    want = hb.attn_mass(sh, Q, lse, kv)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    late = torch.zeros_like(Q)
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        late.copy_(Q)
        got = hb.attn_mass(sh, late, lse, kv)          # reads what the copy in front of it on this stream wrote
        index = hb.keep_tokens(sh, K, K, hb.attn_mass(sh, late, lse, kv, per_token=True), 50)[2]
    s.synchronize()
    assert torch.equal(got, want)
    for _ in range(3):
        assert torch.equal(hb.attn_mass(sh, Q, lse, kv), want)
        assert torch.equal(hb.keep_tokens(sh, K, K, hb.attn_mass(sh, Q, lse, kv, per_token=True), 50)[2], index)


@gpu
def test_python_and_native_marshalling_give_the_same(monkeypatch):
    B, Hq, Hkv, L = 2, 8, 2, 512
    sh = hb.make_shape(B, Hq, Hkv, L)
    g = torch.Generator(device="cuda").manual_seed(3)
    K, Q = torch.randn((B, Hkv, L, D), generator=g, device="cuda").bfloat16(), torch.randn((B, Hq, 70, D), generator=g, device="cuda").bfloat16()
    tk = torch.randn((B, Hkv, TILE, D), generator=g, device="cuda").bfloat16()
    lse, rope = torch.full((B, Hq, 70), 6.0, device="cuda"), hb.make_rope(layout=hb.ROPE_PAIRS)
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    took = []

    def calls():
        kv = hb.compress_kv(sh, hb.make_policy(), K, K)
        res = list(hb.rope_qkv(sh, rope, Q.transpose(1, 2), K[:, :, :70].transpose(1, 2), K[:, :, :70].transpose(1, 2), positions=9, rows=0))
        res += list(hb.rope_qkv(sh, rope, None, K[:, :, :1].transpose(1, 2), None, k_out=tk.clone(), rows=one))[1:2]
        res += [hb.attn_mass(sh, Q, lse, kv), hb.attn_mass(sh, Q, lse, kv, per_token=True, q_start=100, scale=0.3, decay=0.5)]
        res += [hb.attn_mass(sh, Q[:, :, 0], lse[:, :, 0], kv, tail_k=tk, tail_len=one, tail_tile=3), hb.attn_mass(sh, Q[:, :, 1], lse[:, :, 1], kv, tail_k=tk, tail_len=5, tail_tile=one)]
        res += list(hb.keep_tokens(sh, K, K, res[-3], 40, first=1, last=2, lens=one * 300))
        hb.evict_tiles(sh, kv, res[4], 3, first=1)
        hb.evict_tiles(sh, kv, res[4], torch.ones((B, Hkv), dtype=torch.int32, device="cuda"))
        return res + [kv.k_map, kv.v_map, kv.k_nnz, kv.v_nnz]

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
    assert all(ok for name, ok in took if name in ("rope", "mass", "evict", "keep")) and {n for n, _ in took} >= {"rope", "mass", "evict", "keep"}
    none = type("None_", (), {n: staticmethod(lambda *a: None) for n in hb._NATIVE_CALLS})
    monkeypatch.setattr(hb, "_native", none)
    for a, b in zip(by_native, calls()):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))


def test_rope_plan_refusals():
    ok = dict(rot_dim=64, layout=0, scaling=hb.ROPE_RAMP, trained=4096, base=1e4, factor=4.0, low=1.0, high=32.0)
    L, out = hb.lib(), hb.HsRope()
    assert L.hs_rope_plan(C.byref(hb.HsRopeParams(**ok)), C.byref(out)) == 0
    for bad, rc in ((dict(rot_dim=0), -2), (dict(rot_dim=24), -2), (dict(rot_dim=144), -2), (dict(layout=2), -1), (dict(scaling=5), -1), (dict(scaling=-1), -1),
                    (dict(base=1.0), -1), (dict(base=math.nan), -1), (dict(base=math.inf), -1), (dict(factor=0.0), -1), (dict(factor=math.nan), -1),
                    (dict(trained=0), -1), (dict(low=0.0), -1), (dict(high=1.0), -1), (dict(high=math.inf), -1)):
        assert L.hs_rope_plan(C.byref(hb.HsRopeParams(**dict(ok, **bad))), C.byref(out)) == rc, bad
    assert L.hs_rope_plan(None, C.byref(out)) == -1 and L.hs_rope_plan(C.byref(hb.HsRopeParams(**ok)), None) == -1
    with pytest.raises(hb.HsError):
        hb.make_rope(rot_dim=20)


def test_refusals_on_the_host():
    """Arguments that the library refuses before it launches anything (addresses here are never read)."""
    L, sh, rope = hb.lib(), hb.make_shape(2, 8, 2, 256), hb.make_rope()
    s, r = C.byref(sh), C.byref(rope)

    def view(data=4096, batch=1 << 20, head=1 << 14, token=D):
        return C.byref(hb.HsView(data, batch, head, token))

    def qkv(n=4, q=view(), qo=view(), k=view(), ko=view(), v=view(), vo=view(), n_rows=64, shape=s, plan=r):
        return L.hs_rope_qkv(shape, plan, n, None, 0, q, qo, k, ko, v, vo, None, 0, n_rows, None)

    bad_plan = hb.HsRope()
    for bad, rc in ((dict(n=0), -1), (dict(q=None), -1), (dict(qo=None), -1), (dict(ko=None), -1), (dict(vo=None), -1), (dict(k=None, ko=None), -1),
                    (dict(q=None, qo=None, k=None, ko=None, v=None, vo=None), -1), (dict(n_rows=0), -1), (dict(q=view(data=4104)), -1), (dict(q=view(data=None)), -1),
                    (dict(k=view(token=132)), -1), (dict(qo=view(head=64)), -1), (dict(vo=view(token=0)), -1), (dict(q=view(batch=-8)), -1), (dict(plan=None), -1),
                    (dict(plan=C.byref(bad_plan)), -1), (dict(shape=C.byref(hb.make_shape(2, 8, 2, 256, D=64))), -2), (dict(n=1 << 30), -2)):
        assert qkv(**bad) == rc, bad

    kv = hb.HsKV(k_map=4096, v_map=4096)
    size = C.c_size_t(0)

    def mass(Lq=8, q_start=0, scale=0.0, causal=1, Q=view(), lse=4096, cache=C.byref(kv), tail=None, tail_len=0, lens=None, decay=1.0, before=None, out=4096, ws=None,
             shape=s):
        return L.hs_attn_mass(shape, Lq, q_start, scale, causal, Q, lse, None, cache, tail, tail_len, lens, 0, None, 0, decay, before, out, ws, None)

    for bad, rc in ((dict(Lq=0), -1), (dict(q_start=-1), -1), (dict(q_start=249), -1), (dict(Lq=300), -1), (dict(scale=-1.0), -1), (dict(scale=math.nan), -1), (dict(Q=None), -1),
                    (dict(lse=None), -1), (dict(lse=4098), -1), (dict(out=None), -1), (dict(out=4097), -1), (dict(before=4098), -1), (dict(cache=None), -1),
                    (dict(decay=-1.0), -1), (dict(decay=math.nan), -1), (dict(decay=math.inf), -1), (dict(tail=4096), -2), (dict(tail=4096, Lq=1), -2),
                    (dict(tail=4096, Lq=1, causal=0, tail_len=65), -1), (dict(tail=4096, Lq=1, causal=0, tail_len=-1), -1), (dict(tail=4104, Lq=1, causal=0), -1),
                    (dict(Q=view(token=100)), -1), (dict(shape=C.byref(hb.make_shape(2, 8, 2, 100))), -2)):
        assert mass(**bad) == rc, bad
    assert L.hs_attn_mass_workspace_bytes(s, 0, 1, 0, C.byref(size)) == -1 and L.hs_attn_mass_workspace_bytes(s, 8, 1, 0, None) == -1
    for Lq in (1, 2, 100, 5000, 1 << 20):
        for big in (hb.make_shape(1, 1, 1, 64), hb.make_shape(1, 32, 8, 32768), hb.make_shape(16, 32, 8, 131072)):
            for per_token in (0, 1):
                assert 0 <= hb.attn_mass_workspace_bytes(big, Lq, True, per_token) <= 64 << 20
                assert Lq > 1 or hb.attn_mass_workspace_bytes(big, Lq, True, per_token) == 0

    def evict(m=4096, keep=3, keeps=None, first=0, last=0, ws=4096, cache=C.byref(kv), shape=s):
        return L.hs_evict_tiles(shape, cache, m, keep, keeps, first, last, ws, None)

    uniform = hb.HsKV(k_map=4096, v_map=4096, uniform=1)
    for bad, rc in ((dict(m=None), -1), (dict(m=4098), -1), (dict(keep=0), -1), (dict(first=-1), -1), (dict(last=-1), -1), (dict(ws=None), -1), (dict(ws=4098), -1),
                    (dict(cache=None), -1), (dict(cache=C.byref(uniform)), -1), (dict(shape=C.byref(hb.make_shape(1, 1, 1, 65537 * 64))), -2)):
        assert evict(**bad) == rc, bad

    def keep(n=100, K=view(), V=view(), w=4096, n_keep=10, first=0, last=0, ko=4096, vo=4096, idx=4096, ws=4096):
        return L.hs_keep_tokens(s, n, K, V, w, None, None, n_keep, first, last, ko, vo, idx, ws, None)

    for bad, rc in ((dict(n=0), -1), (dict(K=None), -1), (dict(V=None), -1), (dict(w=None), -1), (dict(w=4097), -1), (dict(n_keep=0), -1), (dict(first=-1), -1),
                    (dict(last=-1), -1), (dict(first=6, last=5), -1), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), -1), (dict(ko=None), -1), (dict(vo=4104), -1),
                    (dict(idx=None), -1), (dict(n=(1 << 20) + 1), -2), (dict(ws=4104), -1), (dict(n=100000, ws=None), -1), (dict(K=view(token=4)), -1)):
        assert keep(**bad) == rc, bad


def test_refusals_of_counts_near_the_end_of_32_bits():
    """Queries that all lie at one address (stride 0) may be as many as an int counts, and so may rows of padding: what the kernels' sums cannot hold is refused."""
    L, sh = hb.lib(), hb.make_shape(1, 8, 2, 256)
    one, kv, size = C.byref(hb.HsView(4096, 0, D, 0)), C.byref(hb.HsKV(k_map=4096, v_map=4096)), C.c_size_t(0)
    for Lq in ((1 << 30) + 1, 2 ** 31 - 1):
        assert L.hs_attn_mass(C.byref(sh), Lq, 0, 0.0, 0, one, 4096, None, kv, None, 0, None, 0, None, 0, 1.0, None, 4096, 4096, None) == -2
        assert L.hs_attn_mass_workspace_bytes(C.byref(sh), Lq, 0, 0, C.byref(size)) == -2
        assert L.hs_keep_tokens(C.byref(sh), 100, one, one, 4096, None, None, Lq, 0, 0, 4096, 4096, 4096, 4096, None) == -2
    assert L.hs_attn_mass_workspace_bytes(C.byref(sh), 1 << 30, 0, 0, C.byref(size)) == 0


def test_refusals_of_the_binding():
    """Tensors that are not where or what the call takes."""
    sh, rope = hb.make_shape(1, 4, 2, 128), hb.make_rope()
    q, k = torch.zeros((1, 3, 4, D), dtype=torch.bfloat16), torch.zeros((1, 3, 2, D), dtype=torch.bfloat16)
    kv = hb.PackedKV(sh, [0, 0, 2, 0, 2], "cpu")
    wrong = (hb.HsError, AssertionError)
    for call in (lambda: hb.rope_qkv(sh, rope, q, k, k), lambda: hb.rope_qkv(sh, rope), lambda: hb.rope_qkv(sh, rope, None, None, k),
                 lambda: hb.attn_mass(sh, q.transpose(1, 2), torch.zeros(1, 4, 3), kv), lambda: hb.evict_tiles(sh, kv, torch.zeros(1, 2, 2), 1),
                 lambda: hb.keep_tokens(sh, k.transpose(1, 2), k.transpose(1, 2), torch.zeros(1, 2, 3), 2)):
        with pytest.raises(wrong):
            call()
