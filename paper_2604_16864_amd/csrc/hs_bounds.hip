// Bounds of the keys of every tile, channel by channel, and what a query can score at most in a tile.
#include "hs_common.h"

namespace {

typedef short s16x2_t __attribute__((ext_vector_type(2)));

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

// A wave per tile.  Its keys are read in the pool's order: lane (a, r) holds tokens 16 m + r and 32 channels of each, as 16 pairs, over which it
// keeps the lowest and the highest; then the 16 lanes of a hand each other halves of them (lowest and inverted highest: 32 words), until each has
// 4 channels of one bound.
__global__ __launch_bounds__(64 * HS_BOUNDS_TILES) void bounds_kernel(hs_kv_dev kv, int n_rows, int Hkv, int T, int tile, int n_tiles,
                                                                      const int32_t* __restrict__ tiles, uint16_t* __restrict__ bounds) {
  const int l = threadIdx.x & 63, a = l >> 4, r = l & 15;
  const int n = blockIdx.x * HS_BOUNDS_TILES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = n / n_tiles;
  if (row >= n_rows) return;
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
        const uint4 v = p[64 * (4 * m + s)];
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
    const uint4 at = reinterpret_cast<const uint4*>(kv.k_meta + slot * HS_TILE_META_BYTES)[l];
    const uint32_t idx[4] = {at.x, at.y, at.z, at.w};
#pragma unroll
    for (int m = 0; m < 4; m++)
#pragma unroll
      for (int kb = 0; kb < 2; kb++) {
        const uint4 v = p[64 * (2 * m + kb)];
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
// ONE: one query per sequence; columns are the group's heads, over again up to 16.  Else columns are 16 queries, one head after the other.
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
__device__ __forceinline__ f32x4_t bound_product(const uint4 (&low)[4], const uint4 (&high)[4], const uint16_t* q, int a) {
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  uint4 v[4];
#pragma unroll
  for (int st = 0; st < 4; st++) v[st] = *reinterpret_cast<const uint4*>(q + 32 * st + 8 * a);
#pragma unroll
  for (int st = 0; st < 4; st++) {
    uint4 pos, neg;
    parts_of(v[st], pos, neg);
    s = hs_elem<F16>::mma(high[st], pos, s);
    s = hs_elem<F16>::mma(low[st], neg, s);
  }
  return s;
}

template <bool F16, bool ONE>
__global__ __launch_bounds__(256) void scores_kernel(hs_scores_args g, int64_t n_waves, int tile_blocks, int per_range) {
  const int l = threadIdx.x & 63, a = l >> 4, c = l & 15, G = g.Hq / g.Hkv;
  int64_t n = (int64_t)blockIdx.x * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (n >= n_waves) return;
  const int t0 = (int)(n % tile_blocks) * 16;
  n /= tile_blocks;
  const int row = (int)(n % ((int64_t)g.B * g.Hkv)), range = (int)(n / ((int64_t)g.B * g.Hkv));
  const int b = row / g.Hkv, h = row - b * g.Hkv;
  uint4 low[4], high[4];
  const uint16_t* p = g.bounds + ((int64_t)row * g.T + min(t0 + c, g.T - 1)) * (2 * HS_D) + 8 * a;
#pragma unroll
  for (int st = 0; st < 4; st++) {
    low[st] = *reinterpret_cast<const uint4*>(p + 32 * st);
    high[st] = *reinterpret_cast<const uint4*>(p + HS_D + 32 * st);
  }
  const int t = t0 + 4 * a, n_here = min(4, g.T - t);  // tiles of this lane's results
  int held[4];
#pragma unroll
  for (int i = 0; i < 4; i++) held[i] = i < n_here ? (g.k_map != nullptr ? g.k_map[(int64_t)row * g.T + t + i] : 1) : 0;
  const uint16_t* q = g.q.p + b * g.q.sb + (int64_t)h * G * g.q.sh;
  const bool wide = (g.T & 3) == 0 && ((uintptr_t)g.scores & 15) == 0;
  const int q_first = range * per_range, q_last = min(g.Lq, q_first + per_range);
  for (int q0 = q_first; q0 < q_last; q0 += ONE ? 1 : 16) {
    f32x4_t best = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    const int mine = ONE ? q0 : q0 + c;
    if constexpr (ONE) {
      best = bound_product<F16>(low, high, q + (c % G) * g.q.sh, a);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        float x = no_nan(best[i]);
#define HS_JOIN(CTRL_) x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL_, 0xf, 0xf, true)));
        HS_JOIN(0x128) HS_JOIN(0x124) HS_JOIN(0x122) HS_JOIN(0x121)  // 8, 4, 2 and 1 lanes round the 16
#undef HS_JOIN
        best[i] = x;
      }
    } else {
      for (int head = 0; head < G; head++) {
        const f32x4_t s = bound_product<F16>(low, high, q + head * g.q.sh + min(mine, g.Lq - 1) * g.q.st, a);
#pragma unroll
        for (int i = 0; i < 4; i++) best[i] = fmaxf(best[i], no_nan(s[i]));
      }
    }
    if (n_here <= 0 || (ONE ? c != 0 : mine >= q_last)) continue;
    float* to = g.scores + ((int64_t)row * g.Lq + mine) * g.T + t;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = held[i] != 0 && (!g.causal || (int64_t)(t + i) * HS_BT <= (int64_t)g.q_start + mine) ? best[i] : -INFINITY;
    if (wide) {
      *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++)
        if (i < n_here) to[i] = v[i];
    }
  }
}

struct ScoresPlan { int tile_blocks, per_range, threads; int64_t n_waves, blocks; };
ScoresPlan plan_scores(const hs_scores_args& a) {
  ScoresPlan p;
  p.tile_blocks = (a.T + 15) / 16;
  const int64_t fixed = (int64_t)p.tile_blocks * a.B * a.Hkv, blocks = ((int64_t)a.Lq + 15) / 16;
  int64_t ranges = 2048 / fixed;
  ranges = ranges < 1 ? 1 : (ranges > blocks ? blocks : ranges);
  p.per_range = (int)((blocks + ranges - 1) / ranges) * 16;
  ranges = ((int64_t)a.Lq + p.per_range - 1) / p.per_range;
  p.n_waves = fixed * ranges;
  p.threads = p.n_waves <= 1024 ? 64 : 256;
  p.blocks = (p.n_waves + p.threads / 64 - 1) / (p.threads / 64);
  return p;
}

}  // namespace

hipError_t hs_launch_bounds(int B, int Hkv, int T, const hs_kv_dev& kv, int tile, int n_tiles, const int32_t* tiles, uint16_t* bounds, hipStream_t st) {
  const int64_t n = (int64_t)B * Hkv * n_tiles;
  hipLaunchKernelGGL(bounds_kernel, dim3((unsigned)((n + HS_BOUNDS_TILES - 1) / HS_BOUNDS_TILES)), dim3(64 * HS_BOUNDS_TILES), 0, st, kv, B * Hkv, Hkv, T,
                     tile, n_tiles, tiles, bounds);
  return hipGetLastError();
}

int64_t hs_scores_blocks(const hs_scores_args& a) { return plan_scores(a).blocks; }

hipError_t hs_launch_scores(const hs_scores_args& a, int dtype, hipStream_t st) {
  const ScoresPlan p = plan_scores(a);
#define HS_SCORES(F16_, ONE_) \
  hipLaunchKernelGGL((scores_kernel<F16_, ONE_>), dim3((unsigned)p.blocks), dim3(p.threads), 0, st, a, p.n_waves, p.tile_blocks, p.per_range)
  if (dtype == HS_FP16) {
    if (a.Lq == 1) HS_SCORES(true, true); else HS_SCORES(true, false);
  } else {
    if (a.Lq == 1) HS_SCORES(false, true); else HS_SCORES(false, false);
  }
#undef HS_SCORES
  return hipGetLastError();
}
