// Bounds of the keys of every tile, channel by channel, and what a query can score at most in a tile.
#include "hs_common.h"

namespace {

typedef short s16x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// read past the caches: what is read once a call
__device__ __forceinline__ uint4 ld_past(const uint4* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
}

// Two 16-bit floating-point numbers as integers of the same order: -NaN < -inf < .. < -0 < +0 < .. < inf < +NaN.  Its own inverse.
__device__ __forceinline__ uint32_t order_of(uint32_t x) {
  const s16x2_t sign = __builtin_bit_cast(s16x2_t, x) >> (short)15;
  return x ^ (__builtin_bit_cast(uint32_t, sign) & 0x7fff7fffu);
}
__device__ __forceinline__ uint32_t lower(uint32_t x, uint32_t y) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2_t, x), __builtin_bit_cast(s16x2_t, y)));
}
__device__ __forceinline__ uint32_t upper(uint32_t x, uint32_t y) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2_t, x), __builtin_bit_cast(s16x2_t, y)));
}

// Two kept values (in the order of integers, where a pruned 0 is 0) into their places of four channels.
__device__ __forceinline__ uint2 spread(uint32_t kept, uint32_t at) {
  const uint64_t x = ((uint64_t)(kept & 0xffffu) << (16 * (at & 3u))) | ((uint64_t)(kept >> 16) << (16 * ((at >> 2) & 3u)));
  return make_uint2((uint32_t)x, (uint32_t)(x >> 32));
}

// One step of the reduction over the 16 lanes that hold a tile's tokens: each lane keeps half of its N words, joined with its partner's, and
// hands over the others.  CTRL pairs lanes that differ in `bit`.
template <int N, int CTRL>
__device__ __forceinline__ void halve(uint32_t* x, bool bit) {
#pragma unroll
  for (int i = 0; i < N / 2; i++) {
    const uint32_t keep = bit ? x[i + N / 2] : x[i], give = bit ? x[i] : x[i + N / 2];
    x[i] = lower(keep, (uint32_t)__builtin_amdgcn_mov_dpp((int)give, CTRL, 0xf, 0xf, true));
  }
}

// A wave per tile.  What bounds it: the load stream, past the caches in workgroups of one wave (32768 dense tiles 89.6 us, 6.2 TB/s; through them in workgroups of four 98.4; 4096 2:4 tiles of 38 MB
// 10.2 and 11.5, on other cards 8.9 to 10.0); of a 2:4 tile it issues some 740 vector
// instructions, 2900 clocks of a SIMD where the stream leaves it 4000.  Its keys are read in the pool's order: lane (a, r) holds tokens 16 m + r and 32 channels of each, as 16 pairs, over which it
// keeps the lowest and the highest; then the 16 lanes of a hand each other halves of them (lowest and inverted highest: 32 words), until each has
// 4 channels of one bound.
__global__ __launch_bounds__(64) void bounds_kernel(hs_kv_dev kv, int Hkv, int T, int tile, int n_tiles, const int32_t* __restrict__ tiles,
                                                    uint16_t* __restrict__ bounds) {
  const int l = threadIdx.x, a = l >> 4, r = l & 15;
  const int n = blockIdx.x, row = n / n_tiles;
  int t = tile + (n - row * n_tiles);
  if (tiles != nullptr) {
    t = tiles[row / Hkv];
    if (t < 0 || t >= T) return;
  }
  const int mk = __builtin_amdgcn_readfirstlane(kv.k_map[(int64_t)row * T + t]);
  uint16_t* out = bounds + ((int64_t)row * T + t) * (2 * HS_D);
  uint32_t x[32];  // [0 .. 15] lowest, [16 .. 31] highest
  int channel;     // of word 2 (r & 7) of either
  if (mk == 0) {
    *reinterpret_cast<uint2*>(out + 4 * l) = make_uint2(0, 0);
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; i++) { x[i] = 0x7fff7fffu; x[16 + i] = 0x80008000u; }
  if (mk > 0) {
    const uint4* p = reinterpret_cast<const uint4*>(kv.k_dense + ((int64_t)row * kv.cap_dense_k + (mk - 1)) * HS_TILE_DENSE_BYTES) + l;
#pragma unroll
    for (int m = 0; m < 4; m++)
#pragma unroll
      for (int s = 0; s < 4; s++) {
        const uint4 v = ld_past(p + 64 * (4 * m + s));
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const uint32_t o = order_of(w[e]);
          x[4 * s + e] = lower(x[4 * s + e], o);
          x[16 + 4 * s + e] = upper(x[16 + 4 * s + e], o);
        }
      }
    channel = 32 * ((r >> 1) & 3) + 8 * a + 4 * (r & 1);
  } else {
    const int64_t slot = (int64_t)row * kv.cap_sparse_k + (-mk - 1);
    const uint4* p = reinterpret_cast<const uint4*>(kv.k_nnz + slot * HS_TILE_NNZ_BYTES) + l;
    const uint4 at = ld_past(reinterpret_cast<const uint4*>(kv.k_meta + slot * HS_TILE_META_BYTES) + l);
    const uint32_t idx[4] = {at.x, at.y, at.z, at.w};
#pragma unroll
    for (int m = 0; m < 4; m++)
#pragma unroll
      for (int kb = 0; kb < 2; kb++) {
        const uint4 v = ld_past(p + 64 * (2 * m + kb));
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const uint2 o = spread(order_of(w[q]), idx[m] >> (16 * kb + 4 * q));
          const int i = 8 * kb + 2 * q;
          x[i] = lower(x[i], o.x);
          x[i + 1] = lower(x[i + 1], o.y);
          x[16 + i] = upper(x[16 + i], o.x);
          x[17 + i] = upper(x[17 + i], o.y);
        }
      }
    channel = 64 * ((r >> 2) & 1) + 16 * a + 4 * (r & 3);
  }
#pragma unroll
  for (int i = 16; i < 32; i++) x[i] = ~x[i];  // the highest as the lowest of the inverted
  halve<32, 0x140>(x, (r & 8) != 0);  // lanes of a row mirrored
  halve<16, 0x141>(x, (r & 4) != 0);  // of its halves
  halve<8, 0x4e>(x, (r & 2) != 0);    // two apart
  halve<4, 0xb1>(x, (r & 1) != 0);    // neighbours
  const uint32_t back = (r & 8) != 0 ? 0xffffffffu : 0u;
  *reinterpret_cast<uint2*>(out + (r >> 3) * HS_D + channel) = make_uint2(order_of(x[0] ^ back), order_of(x[1] ^ back));
}

// ---- scores ----
// sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c is a product over 256 terms: the bounds of 16 tiles are the A operand of the 16x16x32 matrix instruction
// as they lie in memory, the positive and the negative parts of the queries the B operand.  Products of 16-bit numbers are exact in the
// instruction, sums are held in 32 bits.
__device__ __forceinline__ float no_nan(float x) { return x == x ? x : INFINITY; }  // a tile that cannot be ruled out

__device__ __forceinline__ void parts_of(uint4 q, uint4& pos, uint4& neg) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  uint32_t p[4], n[4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const uint32_t sign = __builtin_bit_cast(uint32_t, __builtin_bit_cast(s16x2_t, w[i]) >> (short)15);
    p[i] = w[i] & ~sign;
    n[i] = w[i] & sign;
  }
  pos = make_uint4(p[0], p[1], p[2], p[3]);
  neg = make_uint4(n[0], n[1], n[2], n[3]);
}

template <bool F16>
__device__ __forceinline__ f32x4_t bound_product(const uint4 (&low)[4], const uint4 (&high)[4], const uint4 (&q)[4]) {
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int st = 0; st < 4; st++) {
    uint4 pos, neg;
    parts_of(q[st], pos, neg);
    s = hs_elem<F16>::mma(high[st], pos, s);
    s = hs_elem<F16>::mma(low[st], neg, s);
  }
  return s;
}
__device__ __forceinline__ void load_query(uint4 (&v)[4], const uint16_t* q, int a) {
#pragma unroll
  for (int st = 0; st < 4; st++) v[st] = *reinterpret_cast<const uint4*>(q + 32 * st + 8 * a);
}

// What of a row's 16 tiles from t0 on is needed: the bounds of tile t0 + l % 16, unless it is SKIP (m == 0).
struct TileBounds {
  uint4 low[4], high[4];
  __device__ __forceinline__ void load(const uint16_t* row, int t0, int m, int l) {
    const uint16_t* p = row + (int64_t)(t0 + (l & 15)) * (2 * HS_D) + 8 * (l >> 4);
#pragma unroll
    for (int st = 0; st < 4; st++) {
      low[st] = m != 0 ? *reinterpret_cast<const uint4*>(p + 32 * st) : make_uint4(0, 0, 0, 0);
      high[st] = m != 0 ? *reinterpret_cast<const uint4*>(p + HS_D + 32 * st) : make_uint4(0, 0, 0, 0);
    }
  }
};

// Four scores of one query, tiles t .. t + 3; held[i] == 0: SKIP, or behind the row.
__device__ __forceinline__ void store_scores(const hs_scores_args& g, int row, int query, int t, f32x4_t s, const int (&held)[4], bool wide) {
  float* to = g.scores + ((int64_t)row * g.Lq + query) * g.T + t;
  float x[4];
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = held[i] != 0 && (!g.causal || (int64_t)(t + i) * HS_BT <= (int64_t)g.q_start + query) ? s[i] : -INFINITY;
  if (wide) {
    if (t < g.T) *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (t + i < g.T) to[i] = x[i];
  }
}
__device__ __forceinline__ bool wide_scores(const hs_scores_args& g) { return (g.T & 3) == 0 && ((uintptr_t)g.scores & 15) == 0; }

// One query per sequence.  What bounds it: reading the bounds, 256 rows of 2048 tiles of which a quarter is SKIP 38 to 40 us, 5.2 TB/s (SKIP tiles read too 58); all of them held 48, 5.6 TB/s; 512 rows 91, 5.9 TB/s.
// Reads past the caches are no faster here (52, 100).
// grid = (tiles, rows); a wave has n_blocks (1 or 2) blocks of 16 tiles, both requested at once.  Columns are the
// group's heads, over again up to 16.
template <bool F16>
__global__ __launch_bounds__(256) void scores_one_kernel(hs_scores_args g, int n_blocks) {
  const int l = threadIdx.x & 63, a = l >> 4, c = l & 15, G = g.Hq / g.Hkv;
  const int t0 = 16 * n_blocks * (int)(blockIdx.x * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
  if (t0 >= g.T) return;
  const int row = blockIdx.y, b = row / g.Hkv, h = row - b * g.Hkv;
  int m = l < 16 * n_blocks && t0 + l < g.T;  // whether tile t0 + l is held
  if (g.k_map != nullptr && m != 0) m = g.k_map[(int64_t)row * g.T + t0 + l];
  uint4 q[4];
  load_query(q, g.q.p + b * g.q.sb + ((int64_t)h * G + c % G) * g.q.sh, a);
  const uint16_t* bounds = g.bounds + (int64_t)row * g.T * (2 * HS_D);
  const bool wide = wide_scores(g);
  auto load = [&](TileBounds& r, int k) { r.load(bounds, t0 + 16 * k, __shfl(m, 16 * k + c), l); };
  auto use = [&](const TileBounds& r, int k) {
    f32x4_t s = bound_product<F16>(r.low, r.high, q);
    int held[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      float x = no_nan(s[i]);
#define HS_JOIN(CTRL_) x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL_, 0xf, 0xf, true)));
      HS_JOIN(0x128) HS_JOIN(0x124) HS_JOIN(0x122) HS_JOIN(0x121)  // 8, 4, 2 and 1 lanes round the 16
#undef HS_JOIN
      s[i] = x;
      held[i] = __shfl(m, 16 * k + 4 * a + i);
    }
    if (c == 0) store_scores(g, row, 0, t0 + 16 * k + 4 * a, s, held, wide);
  };
  TileBounds first, second;
  load(first, 0);
  if (n_blocks > 1) load(second, 1);  // a block behind the row has no held tile and is not stored
  use(first, 0);
  if (n_blocks > 1) use(second, 1);
}

// More queries.  What bounds it: latency while queries are few (65 queries, 7 heads, 777 tiles, 4 rows: 6.3 us); heads known to the compiler are worth 0.6 of it, their products side by side.
// grid = (tiles, rows, ranges of the queries); a wave reads its 16 tiles once.  Columns are 16 queries, one head after the other, all heads'
// queries requested at once.
template <bool F16, int G>
__global__ __launch_bounds__(256) void scores_kernel(hs_scores_args g, int per_range) {
  const int l = threadIdx.x & 63, a = l >> 4, c = l & 15;
  const int t0 = 16 * (int)(blockIdx.x * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
  if (t0 >= g.T) return;
  const int row = blockIdx.y, b = row / g.Hkv, h = row - b * g.Hkv;
  const uint16_t* q = g.q.p + b * g.q.sb + (int64_t)h * G * g.q.sh;
  int m = t0 + c < g.T;
  if (g.k_map != nullptr && m != 0) m = g.k_map[(int64_t)row * g.T + t0 + c];
  TileBounds r;
  r.load(g.bounds + (int64_t)row * g.T * (2 * HS_D), t0, m, l);
  int held[4];
#pragma unroll
  for (int i = 0; i < 4; i++) held[i] = __shfl(m, 4 * a + i);
  const bool wide = wide_scores(g);
  const int q_first = (int)blockIdx.z * per_range, q_last = min(g.Lq, q_first + per_range);
  for (int q0 = q_first; q0 < q_last; q0 += 16) {
    const uint16_t* from = q + min(q0 + c, q_last - 1) * g.q.st;
    uint4 v[G][4];
#pragma unroll
    for (int k = 0; k < G; k++) load_query(v[k], from + k * g.q.sh, a);
    f32x4_t best = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int k = 0; k < G; k++) {
      const f32x4_t s = bound_product<F16>(r.low, r.high, v[k]);
#pragma unroll
      for (int i = 0; i < 4; i++) best[i] = fmaxf(best[i], no_nan(s[i]));
    }
    if (q0 + c < q_last) store_scores(g, row, q0 + c, t0 + 4 * a, best, held, wide);
  }
}

}  // namespace

hipError_t hs_launch_bounds(int B, int Hkv, int T, const hs_kv_dev& kv, int tile, int n_tiles, const int32_t* tiles, uint16_t* bounds, hipStream_t st) {
  const int64_t n = (int64_t)B * Hkv * n_tiles;
  hipLaunchKernelGGL(bounds_kernel, dim3((unsigned)n), dim3(64), 0, st, kv, Hkv, T, tile, n_tiles, tiles, bounds);
  return hipGetLastError();
}

hipError_t hs_launch_scores(const hs_scores_args& a, int dtype, hipStream_t st) {
  const int rows = a.B * a.Hkv, tile_blocks = (a.T + 15) / 16;
  const int64_t fixed = (int64_t)rows * tile_blocks;
  if (a.Lq == 1) {
    // blocks of a wave, us: 512 rows of 2048 tiles, 1: 93.9, 2: 91.6, 4: 97.0; 128 rows of 512, 9.5, 8.9, 10.0; 8 rows of 512, 3.0, 3.6, 4.9
    const int n = fixed >= 2048 ? 2 : 1;
    const int64_t per_row = (tile_blocks + n - 1) / n;
    const int waves = per_row * rows <= 1024 ? 1 : 4;
    const dim3 grid((unsigned)((per_row + waves - 1) / waves), (unsigned)rows), block(64 * waves);
    if (dtype == HS_FP16) hipLaunchKernelGGL((scores_one_kernel<true>), grid, block, 0, st, a, n);
    else hipLaunchKernelGGL((scores_one_kernel<false>), grid, block, 0, st, a, n);
    return hipGetLastError();
  }
  const int64_t blocks = ((int64_t)a.Lq + 15) / 16;
  int64_t ranges = 2048 / fixed;
  ranges = ranges < 1 ? 1 : (ranges > blocks ? blocks : ranges);
  const int per_range = (int)((blocks + ranges - 1) / ranges) * 16;
  ranges = ((int64_t)a.Lq + per_range - 1) / per_range;
  const int waves = fixed * ranges <= 1024 ? 1 : 4;
  const dim3 grid((unsigned)((tile_blocks + waves - 1) / waves), (unsigned)rows, (unsigned)ranges), block(64 * waves);
#define HS_SCORES(G_)                                                                                    \
  case G_:                                                                                               \
    if (dtype == HS_FP16) hipLaunchKernelGGL((scores_kernel<true, G_>), grid, block, 0, st, a, per_range); \
    else hipLaunchKernelGGL((scores_kernel<false, G_>), grid, block, 0, st, a, per_range);               \
    break
  switch (a.Hq / a.Hkv) { HS_SCORES(1); HS_SCORES(2); HS_SCORES(3); HS_SCORES(4); HS_SCORES(5); HS_SCORES(6); HS_SCORES(7); HS_SCORES(8); }
#undef HS_SCORES
  return hipGetLastError();
}
