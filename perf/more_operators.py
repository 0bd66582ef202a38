"""Attention of each query over the tiles that a cheap score picks for it, as cases that can be timed and checked: per tile of the packed
cache the smallest and the largest key in every channel, from these what a query can score at most in a tile, the choice of each query's
tiles, and attention over the tiles chosen.

`prepare` makes inputs from a seed on the GPU, `run` is one call: with `own` the framework's, otherwise the same in elementary torch
operations; `exact` is the definition in 64 bits.

Fields of a case: op; B, Hq, Hkv, dtype; T tiles of 64 tokens a sequence; and
  bounds  keys (2:4, dense, mixed), skip (share of the tiles not held), step (one tile of each sequence, at its own place; else all)
  scores  Lq queries (1: a decode step; more: the last tokens of the cache, causal), skip
  pick    Lq, skip, n tiles picked, first, last (tiles that are always picked)
  attn    Lq, n, keys, values (2:4, dense, mixed), tail (tokens beyond the packed ones, on average half a tile)
"""
import math

import torch

own = False

D, TILE = 128, 64
SINK, WINDOW = 1, 4            # tiles that are always picked: 64 and 256 tokens


def _case(name, op, **kw):
    return dict(dict(B=1, Hq=32, Hkv=8, dtype="bf16"), name=name, op=op, **kw)


def listed():
    return [
        # every 64 steps of serving: the tile just appended to each of 16 sequences
        _case("bounds_step_b16", "bounds", B=16, T=256, keys="2:4", skip=0.0, step=True),
        # after a prompt of 32K tokens
        _case("bounds_prompt_32k", "bounds", T=512, keys="2:4", skip=0.0, step=False),
        # after four prompts of 64K tokens, keys dense
        _case("bounds_prompt_b4_64k", "bounds", B=4, dtype="fp16", T=1024, keys="dense", skip=0.0, step=False),
        # a decode step over a 32K cache
        _case("scores_step_32k", "scores", T=512, Lq=1, skip=0.0),
        # a decode step of 32 sequences at 128K, a quarter of the tiles dropped
        _case("scores_step_b32_128k", "scores", B=32, T=2048, Lq=1, skip=0.25),
        # the last 65 tokens of two prompts, seven heads a group
        _case("scores_window_b2", "scores", B=2, Hq=14, Hkv=2, dtype="fp16", T=777, Lq=65, skip=0.0),
        # that decode step's choice: 32 tiles of 512
        _case("pick_step_32k", "pick", T=512, Lq=1, skip=0.0, n=32, first=SINK, last=WINDOW),
        # 32 sequences at 128K: 64 tiles of 2048
        _case("pick_step_b32_128k", "pick", B=32, T=2048, Lq=1, skip=0.25, n=64, first=SINK, last=WINDOW),
        # each of the last 300 tokens of a prompt picks its own
        _case("pick_window_300", "pick", Hq=14, Hkv=2, T=777, Lq=300, skip=0.0, n=41, first=SINK, last=WINDOW),
        # a decode step over 32 tiles of a 32K cache and the tail
        _case("attn_step_32k", "attn", T=512, Lq=1, n=32, keys="2:4", values="2:4", tail=True),
        # a decode step of 16 sequences at 64K
        _case("attn_step_b16_64k", "attn", B=16, T=1024, Lq=1, n=64, keys="2:4", values="2:4", tail=True),
        # the last 65 tokens of two prompts, half of the keys' tiles dense
        _case("attn_window_b2", "attn", B=2, Hq=14, Hkv=2, dtype="fp16", T=777, Lq=65, n=41, keys="mixed", values="2:4", tail=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["bounds", "scores", "pick", "attn", "attn"])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16"]))
    c["Hkv"] = rng.choice([1, 2, 3, 4, 8, 8, 8])
    c["Hq"] = c["Hkv"] * rng.choice([1, 2, 3, 4, 4, 4, 5, 7, 8])
    c["B"] = rng.choice([1, 1, 2, 3, 4, 8, 13, 16])
    rows = c["B"] * c["Hkv"]
    if op == "bounds":
        c["keys"] = rng.choice(["2:4", "2:4", "dense", "mixed"])
        c["skip"] = rng.choice([0.0, 0.0, 0.25, 0.75])
        c["step"] = rng.random() < 0.3
        c["T"] = _log_int(rng, 1, min(2048, 32768 // rows))
        return c
    c["Lq"] = rng.choice([1, 1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 300)])
    if op == "attn":
        c["keys"], c["values"] = rng.choice(["2:4", "2:4", "dense", "mixed"]), rng.choice(["2:4", "2:4", "dense", "mixed"])
        c["T"] = _log_int(rng, 1, min(2048, 65536 // rows))
        c["n"] = _log_int(rng, 1, min(256, c["T"]))
        c["tail"] = c["Lq"] == 1 and rng.random() < 0.6
        while rows * c["Lq"] * c["n"] > 10000:
            if c["Lq"] > 1 and rng.random() < 0.5:
                c["Lq"] = max(1, c["Lq"] // 2)
            else:
                c["n"] = max(1, c["n"] // 2)
    else:
        c["skip"] = rng.choice([0.0, 0.0, 0.25, 0.75])
        c["T"] = _log_int(rng, 1, min(8192, 500000 // rows))
        while rows * c["Lq"] * c["T"] > 500000 and c["Lq"] > 1:
            c["Lq"] = max(1, c["Lq"] // 2)
    c["Lq"] = min(c["Lq"], c["T"] * TILE)
    if op == "pick":
        c["first"], c["last"] = rng.choice([(0, 0), (SINK, WINDOW), (SINK, WINDOW), (2, 0)])
        c["n"] = max(1, c["first"] + c["last"], _log_int(rng, 1, 256))
    return c


# ------------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------------
def _dtype(c):
    return torch.float16 if c["dtype"] == "fp16" else torch.bfloat16


def _gen(seed, k):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 16 + k)


def _normal(sizes, dtype, g):
    """Normal values, drawn one part of the first axis at a time (bounds the 32-bit intermediate)."""
    out = torch.empty(sizes, dtype=dtype, device="cuda")
    for i in range(sizes[0]):
        out[i] = torch.randn(sizes[1:], device="cuda", generator=g).to(dtype)
    return out


def _keys(c, g):
    """Keys [B, Hkv, T * 64, D]: some channels are larger than others and off zero, and tokens near each other alike."""
    B, H, T = c["B"], c["Hkv"], c["T"]
    size = torch.exp(0.5 * torch.randn((H, 1, D), device="cuda", generator=g))
    middle = torch.randn((H, 1, D), device="cuda", generator=g) * size
    out = torch.empty((B, H, T * TILE, D), dtype=_dtype(c), device="cuda")
    for b in range(B):
        near = torch.randn((H, T, 1, D), device="cuda", generator=g).expand(H, T, TILE, D).reshape(H, T * TILE, D)
        out[b] = (middle + size * (0.6 * near + 0.8 * torch.randn((H, T * TILE, D), device="cuda", generator=g))).to(out.dtype)
    return out


def _prune(x, sparse, along):
    """x [B, H, T * 64, D] with the two smaller of every four entries along the channels (-1) or the tokens (-2) of the tiles in
    sparse [B, H, T] set to zero; of equal magnitudes the lower place stays."""
    for b in range(x.shape[0]):
        y = x[b].transpose(-1, -2) if along == -2 else x[b]
        y = y.reshape(*y.shape[:-1], y.shape[-1] // 4, 4)
        m = y.abs()
        parts = []
        for j in range(4):
            larger = sum((m[..., i] > m[..., j]).to(torch.int8) if i > j else (m[..., i] >= m[..., j]).to(torch.int8) for i in range(4) if i != j)
            parts.append(torch.where(larger < 2, y[..., j], torch.zeros((), dtype=x.dtype, device="cuda")))
        y = torch.stack(parts, dim=-1).flatten(-2)
        y = y.transpose(-1, -2) if along == -2 else y
        x[b] = torch.where(sparse[b].repeat_interleave(TILE, dim=-1)[..., None], y, x[b])
    return x


def _kinds(c, kind, g):
    """Which tiles are 2:4 [B, H, T]."""
    share = {"2:4": 1.0, "dense": 0.0, "mixed": 0.5}[kind]
    return torch.rand((c["B"], c["Hkv"], c["T"]), generator=g, device="cuda") < share


def _held(c, g):
    return torch.rand((c["B"], c["Hkv"], c["T"]), generator=g, device="cuda") >= c["skip"]


def _prepare_bounds(c, seed):
    st = {"held": _held(c, _gen(seed, 1)), "k_sparse": _kinds(c, c["keys"], _gen(seed, 2))}
    st["K"] = _prune(_keys(c, _gen(seed, 0)), st["k_sparse"], -1)
    st["bounds"] = torch.zeros((c["B"], c["Hkv"], c["T"], 2, D), dtype=_dtype(c), device="cuda")
    if c["step"]:
        st["tiles"] = torch.randint(0, c["T"], (c["B"],), generator=_gen(seed, 3), device="cuda", dtype=torch.int32)
    return st


def _positions(c):
    """Positions of the queries: the last ones of the cache."""
    return torch.arange(c["T"] * TILE - c["Lq"], c["T"] * TILE, device="cuda")


def _prepare_scores(c, seed):
    B, H, T = c["B"], c["Hkv"], c["T"]
    g = _gen(seed, 0)
    size = torch.exp(0.5 * torch.randn((H, 1, D), device="cuda", generator=g))
    middle = torch.randn((H, 1, D), device="cuda", generator=g) * size + 0.6 * size * torch.randn((B, H, T, D), device="cuda", generator=g)
    low = middle - size * (1.5 + 0.6 * torch.rand((B, H, T, D), device="cuda", generator=g))
    high = middle + size * (1.5 + 0.6 * torch.rand((B, H, T, D), device="cuda", generator=g))
    st = {"bounds": torch.stack([low, high], dim=3).to(_dtype(c)), "Q": _normal((B, c["Hq"], c["Lq"], D), _dtype(c), _gen(seed, 1))}
    st["held"] = _held(c, _gen(seed, 2))
    return st


def _prepare_pick(c, seed):
    B, H, T, Lq = c["B"], c["Hkv"], c["T"], c["Lq"]
    # scores of neighbouring queries are alike; some are equal to the bit
    s = 40.0 + 10.0 * torch.randn((B, H, 1, T), generator=_gen(seed, 0), device="cuda")
    s = (s + 3.0 * torch.randn((B, H, Lq, T), generator=_gen(seed, 1), device="cuda")).to(torch.float16).float()
    open_ = _held(c, _gen(seed, 2))[:, :, None, :] & (torch.arange(T, device="cuda") * TILE <= _positions(c)[:, None])
    return {"scores": torch.where(open_, s, -math.inf)}


def _prepare_attn(c, seed):
    B, H, T, Lq, n = c["B"], c["Hkv"], c["T"], c["Lq"], c["n"]
    st = {"k_sparse": _kinds(c, c["keys"], _gen(seed, 2)), "v_sparse": _kinds(c, c["values"], _gen(seed, 3))}
    st["K"] = _prune(_keys(c, _gen(seed, 0)), st["k_sparse"], -1)
    st["V"] = _prune(_normal((B, H, T * TILE, D), _dtype(c), _gen(seed, 1)), st["v_sparse"], -2)
    st["Q"] = _normal((B, c["Hq"], Lq, D), _dtype(c), _gen(seed, 4))
    # each query's tiles: the ends, and others that its neighbours mostly pick too; in order, -1 where there are fewer
    s = torch.randn((B, H, 1, T), generator=_gen(seed, 5), device="cuda") + 0.3 * torch.randn((B, H, Lq, T), generator=_gen(seed, 6), device="cuda")
    s[..., :SINK] += 100.0
    at = _positions(c)[:, None] // TILE - torch.arange(T, device="cuda")          # tiles before the query's own
    s = s + torch.where(at < WINDOW, 50.0, 0.0)
    s = s.masked_fill(at < 0, -math.inf)
    best = s.topk(n, dim=-1)
    st["list"] = torch.where(best.values > -math.inf, best.indices, T).sort(dim=-1).values
    st["list"] = torch.where(st["list"] < T, st["list"], -1).to(torch.int32)
    if c["tail"]:
        st["tail_k"] = _keys(dict(c, T=1), _gen(seed, 7))
        st["tail_v"] = _normal((B, H, TILE, D), _dtype(c), _gen(seed, 8))
        st["tail_len"] = torch.randint(1, TILE, (B,), generator=_gen(seed, 9), device="cuda", dtype=torch.int32)
    return st


_PREPARE = {"bounds": _prepare_bounds, "scores": _prepare_scores, "pick": _prepare_pick, "attn": _prepare_attn}


def _handles(c, st):
    """What a program that uses the framework keeps beside its tensors."""
    from paper_2604_16864_amd import binding as hb
    st["shape"] = shape = hb.make_shape(c["B"], c["Hq"], c["Hkv"], c["T"] * TILE, dtype=_dtype(c))
    if c["op"] in ("bounds", "attn"):
        k, v = st["k_sparse"], st.get("v_sparse", st["k_sparse"])
        held = st.get("held", torch.ones_like(k))
        if bool(held.all()) and c["keys"] != "mixed" and c.get("values") != "mixed":
            policy = hb.make_policy(sparse_frac_k=float(c["keys"] == "2:4"), sparse_frac_v=float(c.get("values", c["keys"]) == "2:4"))
        else:
            states = [torch.where(held, torch.where(x, hb.SPARSE24, hb.DENSE), hb.SKIP).to(torch.int8).cpu().numpy() for x in (k, v)]
            policy = hb.make_policy(state_k=states[0], state_v=states[1])
        st["kv"] = hb.compress_kv(shape, policy, st["K"], st.get("V", st["K"]))
    elif c["op"] == "scores":
        st["k_map"] = None if c["skip"] == 0.0 else (st["held"].cumsum(-1) * st["held"]).to(torch.int32)


def prepare(case, seed):
    st = _PREPARE[case["op"]](case, seed)
    st["case"] = dict(case)
    if own:
        _handles(case, st)
    return st


# ------------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------------
def _run_bounds(c, st):
    if own:
        from paper_2604_16864_amd import binding as hb
        return hb.tile_bounds(st["shape"], st["kv"], tile=st["tiles"] if c["step"] else 0, out=st["bounds"])
    K = st["K"].view(c["B"], c["Hkv"], c["T"], TILE, D)
    if c["step"]:
        b, t = torch.arange(c["B"], device="cuda"), st["tiles"].long()
        k = K[b, :, t]
        both = torch.stack([k.amin(-2), k.amax(-2)], dim=-2)
        st["bounds"][b, :, t] = torch.where(st["held"][b, :, t][..., None, None], both, torch.zeros_like(both))
    else:
        both = torch.stack([K.amin(-2), K.amax(-2)], dim=-2)
        st["bounds"].copy_(torch.where(st["held"][..., None, None], both, torch.zeros_like(both)))
    return st["bounds"]


def _run_scores(c, st):
    one = c["Lq"] == 1
    if own:
        from paper_2604_16864_amd import binding as hb
        s = hb.query_scores(st["shape"], st["Q"][:, :, 0] if one else st["Q"], st["bounds"], st["k_map"])
        return s.unsqueeze(2) if one else s
    B, H, T, Lq = c["B"], c["Hkv"], c["T"], c["Lq"]
    q = st["Q"].float().view(B, H, -1, D)
    low, high = st["bounds"][:, :, :, 0].float(), st["bounds"][:, :, :, 1].float()
    s = torch.matmul(q.clamp(min=0.0), high.transpose(-1, -2)) + torch.matmul(q.clamp(max=0.0), low.transpose(-1, -2))
    s = s.view(B, H, -1, Lq, T).amax(2)
    open_ = st["held"][:, :, None, :] & (torch.arange(T, device="cuda") * TILE <= _positions(c)[:, None])
    return torch.where(open_, s, -math.inf)


def _run_pick(c, st):
    if own:
        from paper_2604_16864_amd import binding as hb
        return hb.pick_tiles(st["shape"], st["scores"], c["n"], first=c["first"], last=c["last"])
    s, T, n = st["scores"], c["T"], c["n"]
    open_ = s > -math.inf
    number = open_.cumsum(-1)                      # of the query's open tiles, from 1
    always = open_ & ((number <= c["first"]) | (number > number[..., -1:] - c["last"]))
    best = torch.where(always, math.inf, s).sort(dim=-1, descending=True, stable=True)
    index = torch.where(best.values > -math.inf, best.indices, T)[..., :n].sort(dim=-1).values
    if n > T:
        index = torch.nn.functional.pad(index, (0, n - T), value=T)
    return torch.where(index < T, index, -1).to(torch.int32)


def _run_attn(c, st):
    B, H, T, Lq, n, G = c["B"], c["Hkv"], c["T"], c["Lq"], c["n"], c["Hq"] // c["Hkv"]
    if own:
        from paper_2604_16864_amd import binding as hb
        tail = dict(tail_k=st["tail_k"], tail_v=st["tail_v"], tail_len=st["tail_len"]) if c["tail"] else {}
        if Lq == 1:
            o, lse = hb.listed_attn(st["shape"], st["Q"][:, :, 0], st["kv"], st["list"][:, :, 0], **tail)
            return o.unsqueeze(2), lse.unsqueeze(2)
        return hb.listed_attn(st["shape"], st["Q"], st["kv"], st["list"], **tail)
    o, lse = torch.empty_like(st["Q"]), torch.empty((B, c["Hq"], Lq), dtype=torch.float32, device="cuda")
    K, V = (st[x].view(B, H, T, TILE, D) for x in "KV")
    b, h = torch.arange(B, device="cuda")[:, None, None, None], torch.arange(H, device="cuda")[:, None, None]
    step = max(1, 16384 // (B * H * n))            # queries at a time: bounds what is gathered
    for i in range(0, Lq, step):
        m = min(step, Lq - i)
        q = st["Q"][:, :, i:i + m].float().view(B, H, G, m, D).transpose(2, 3)
        at = st["list"][:, :, i:i + m].long()
        token = (at[..., None] * TILE + torch.arange(TILE, device="cuda")).flatten(-2)
        seen = (token >= 0) & (token <= _positions(c)[i:i + m, None])
        k, v = (x[b, h, at.clamp(min=0)].flatten(3, 4).float() for x in (K, V))
        if c["tail"]:
            k, v = torch.cat([k, st["tail_k"][:, :, None].float()], dim=3), torch.cat([v, st["tail_v"][:, :, None].float()], dim=3)
            tail_seen = torch.arange(TILE, device="cuda") < st["tail_len"][:, None]
            seen = torch.cat([seen, tail_seen[:, None, None].expand(B, H, m, TILE)], dim=-1)
        s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(D)
        s = s.masked_fill(~seen[:, :, :, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        o[:, :, i:i + m] = (torch.matmul(p, v) / total).transpose(2, 3).reshape(B, -1, m, D).to(o.dtype)
        lse[:, :, i:i + m] = (top + torch.log(total))[..., 0].transpose(2, 3).reshape(B, -1, m)
    return o, lse


_RUN = {"bounds": _run_bounds, "scores": _run_scores, "pick": _run_pick, "attn": _run_attn}


def run(state):
    return _RUN[state["case"]["op"]](state["case"], state)


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
_SHARE = {"2:4": 1.0, "mixed": 0.5, "dense": 0.0}


def _tile_bytes(kind):
    return 9216 * _SHARE[kind] + 16384 * (1.0 - _SHARE[kind])


def work(case):
    c = case
    rows, T = c["B"] * c["Hkv"], c["T"]
    if c["op"] == "bounds":
        tiles = rows * (1 if c["step"] else T)
        return {"bytes": float(tiles * ((1.0 - c["skip"]) * _tile_bytes(c["keys"]) + 4 * D)), "flops": 2.0 * TILE * D * tiles}
    queries = rows * c["Lq"]
    if c["op"] == "scores":
        held = rows * T * (1.0 - c["skip"])
        pairs = queries * T * (1.0 - c["skip"]) * (c["Hq"] // c["Hkv"])
        return {"bytes": float(held * 4 * D + queries * T * 4 + c["B"] * c["Hq"] * c["Lq"] * D * 2), "flops": 4.0 * D * pairs}
    if c["op"] == "pick":
        return {"bytes": float(queries * 4 * (T + c["n"])), "flops": 0.0}
    # tiles that some query picks: all of one query's, and of many queries' at most what there is
    tiles = rows * min(T, c["n"] if c["Lq"] == 1 else c["n"] + T // 4)
    heads = c["B"] * c["Hq"] * c["Lq"]
    flops = 2.0 * D * TILE * c["n"] * heads * ((1.0 - 0.5 * _SHARE[c["keys"]]) + (1.0 - 0.5 * _SHARE[c["values"]]))
    tail = rows * TILE // 2 * D * 4 if c["tail"] else 0
    return {"bytes": float(tiles * (_tile_bytes(c["keys"]) + _tile_bytes(c["values"])) + tail + queries * 4 * c["n"] + heads * (4 * D + 4)), "flops": flops}


# ------------------------------------------------------------------------------------------------------------------
# the same from the definition, in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def _exact_bounds(c, st):
    out = torch.zeros(st["bounds"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        for t in ([int(st["tiles"][b])] if c["step"] else range(c["T"])):
            k = st["K"][b, :, t * TILE:(t + 1) * TILE].double().sort(dim=1).values
            held = st["held"][b, :, t, None].double()
            out[b, :, t, 0], out[b, :, t, 1] = k[:, 0] * held, k[:, -1] * held
    return out


def _exact_scores(c, st):
    B, H, T, Lq, G = c["B"], c["Hkv"], c["T"], c["Lq"], c["Hq"] // c["Hkv"]
    out = torch.full((B, H, Lq, T), -math.inf, dtype=torch.float64, device="cuda")
    step = max(1, 250000 // T)
    for b in range(B):
        for h in range(H):
            low, high = st["bounds"][b, h, :, 0].double(), st["bounds"][b, h, :, 1].double()
            for g in range(h * G, (h + 1) * G):
                for i in range(0, Lq, step):
                    q = st["Q"][b, g, i:i + step, None].double()
                    # channel by channel the larger of the two products
                    s = torch.maximum(q * low, q * high).sum(-1)
                    out[b, h, i:i + step] = torch.maximum(out[b, h, i:i + step], s)
            for i in range(Lq):
                out[b, h, i, (T * TILE - Lq + i) // TILE + 1:] = -math.inf
            out[b, h].masked_fill_(~st["held"][b, h], -math.inf)
    return out


def _exact_pick(c, st):
    out = torch.full((c["B"], c["Hkv"], c["Lq"], c["n"]), -1, dtype=torch.int32)
    scores = st["scores"].cpu()
    for b in range(c["B"]):
        for h in range(c["Hkv"]):
            for i in range(c["Lq"]):
                s = scores[b, h, i].tolist()
                there = [t for t in range(c["T"]) if s[t] > -math.inf]
                lead = there[:c["first"]]
                trail = there[max(len(lead), len(there) - c["last"]):]
                rest = sorted(there[len(lead):len(there) - len(trail)], key=lambda t: (-s[t], t))
                take = sorted((lead + trail + rest)[:c["n"]])
                out[b, h, i, :len(take)] = torch.tensor(take, dtype=torch.int32)
    return out.cuda()


def _exact_attn(c, st):
    """Row by row over the whole cache, with a mask of the tokens that the list names."""
    B, H, T, Lq, G = c["B"], c["Hkv"], c["T"], c["Lq"], c["Hq"] // c["Hkv"]
    L = T * TILE
    o = torch.zeros((B, c["Hq"], Lq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, c["Hq"], Lq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(H):
            k, v = st["K"][b, h].double(), st["V"][b, h].double()
            mask = torch.zeros((Lq, T + 1), dtype=torch.bool, device="cuda").scatter_(1, st["list"][b, h].long() % (T + 1), True)[:, :T]
            mask = mask.repeat_interleave(TILE, dim=1) & (torch.arange(L, device="cuda") <= torch.arange(L - Lq, L, device="cuda")[:, None])
            if c["tail"]:
                m = int(st["tail_len"][b])
                k, v = torch.cat([k, st["tail_k"][b, h, :m].double()]), torch.cat([v, st["tail_v"][b, h, :m].double()])
                mask = torch.cat([mask, torch.ones((Lq, m), dtype=torch.bool, device="cuda")], dim=1)
            for g in range(h * G, (h + 1) * G):
                s = torch.mm(st["Q"][b, g].double(), k.t()) * D ** -0.5
                s = torch.where(mask, s, -math.inf)
                lse[b, g] = torch.logsumexp(s, dim=-1)
                o[b, g] = torch.mm(torch.exp(s - lse[b, g][:, None]), v)
    return o, lse


_EXACT = {"bounds": _exact_bounds, "scores": _exact_scores, "pick": _exact_pick, "attn": _exact_attn}


def exact(case, seed):
    return _EXACT[case["op"]](case, _PREPARE[case["op"]](case, seed))
