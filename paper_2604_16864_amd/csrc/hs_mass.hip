// Attention weight that each tile (or token) of the packed cache gathers: the column sums of the softmax whose log-sum-exps a prefill or
// decode call returned, sum over queries i of exp(scale q_i . k_j - LSE_i).
//
// With the LSE known there is no running maximum and no second product: a tile's weight depends on its keys and on the queries alone.
// So a wave holds one tile's K operands in registers (the pools' byte order is that of the matrix instruction) and the queries pass by: S^T = K Q^T
// leaves tokens in rows and queries in columns, a lane adds up its 16 tokens of one column, and the 16 columns are joined at the end.
#include "hs_common.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
}

// K operands of one tile.  KM: 0 = 2:4, 1 = dense, 2 = either (mk < 0: 2:4)
template <int KM>
struct KTile {
  static constexpr int kN = KM == 0 ? 8 : 16;
  uint4 k[kN];
  uint4 idx;
};
template <int KM>
__device__ __forceinline__ void k_load(KTile<KM>& r, const hs_kv_dev& kv, int64_t row, int mk, int l) {  // mk != 0, wave-uniform
  r.idx = make_uint4(0, 0, 0, 0);
  if (KM == 0 || (KM == 2 && mk < 0)) {
    const int64_t slot = row * kv.cap_sparse_k + (-mk - 1);
    const uint4* p = reinterpret_cast<const uint4*>(kv.k_nnz + slot * (int64_t)HS_TILE_NNZ_BYTES) + l;
#pragma unroll
    for (int i = 0; i < 8; i++) r.k[i] = ld_stream(p + 64 * i);
    r.idx = ld_stream(reinterpret_cast<const uint4*>(kv.k_meta + slot * (int64_t)HS_TILE_META_BYTES) + l);
  } else {
    const int64_t slot = row * kv.cap_dense_k + (mk - 1);
    const uint4* p = reinterpret_cast<const uint4*>(kv.k_dense + slot * (int64_t)HS_TILE_DENSE_BYTES) + l;
#pragma unroll
    for (int i = 0; i < 16; i++) r.k[i % KTile<KM>::kN] = ld_stream(p + 64 * i);
  }
}
// S^T of the tile's 64 tokens and 16 queries: lane (a, c) holds tokens 16m + 4a + i of column c
template <bool F16, int KM>
__device__ __forceinline__ void scores(const KTile<KM>& r, bool sparse, const uint4 (&qb)[4], f32x4_t (&s)[4]) {
  typedef hs_elem<F16> E;
#pragma unroll
  for (int m = 0; m < 4; m++) s[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (KM == 0 || (KM == 2 && sparse)) {
    const int idx[4] = {(int)r.idx.x, (int)r.idx.y, (int)r.idx.z, (int)r.idx.w};
#pragma unroll
    for (int m = 0; m < 4; m++) s[m] = E::template smma<0>(r.k[2 * m], qb[0], qb[1], s[m], idx[m]);
#pragma unroll
    for (int m = 0; m < 4; m++) s[m] = E::template smma<1>(r.k[2 * m + 1], qb[2], qb[3], s[m], idx[m]);
  } else {
#pragma unroll
    for (int st = 0; st < 4; st++)
#pragma unroll
      for (int m = 0; m < 4; m++) s[m] = E::mma(r.k[(4 * m + st) % KTile<KM>::kN], qb[st], s[m]);
  }
}

// The value of another lane of the 16: c ^ 8, c ^ 7, c ^ 2, c ^ 1
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, true));
}
// v[e] summed over the 16 lanes of a row, lane c getting the sum of element e = c.  Every step a lane gives half of what it holds to a
// partner that gives it the other half: 15 sums instead of 64.
__device__ __forceinline__ float sum_columns(const float (&v)[16], int c) {
  float x[8], y[4], z[2];
  const bool b3 = c & 8, b2 = c & 4, b1 = c & 2, b0 = c & 1;
#pragma unroll
  for (int e = 0; e < 8; e++) x[e] = (b3 ? v[e + 8] : v[e]) + dpp<0x128>(b3 ? v[e] : v[e + 8]);  // row_ror:8
#pragma unroll
  for (int e = 0; e < 4; e++) y[e] = (b2 ? x[e + 4] : x[e]) + dpp<0x141>(b2 ? x[e] : x[e + 4]);  // row_half_mirror
#pragma unroll
  for (int e = 0; e < 2; e++) z[e] = (b1 ? y[e + 2] : y[e]) + dpp<0x4e>(b1 ? y[e] : y[e + 2]);   // quad_perm 2 3 0 1
  return (b0 ? z[1] : z[0]) + dpp<0xb1>(b0 ? z[0] : z[1]);                                       // quad_perm 1 0 3 2
}
// token of the tile whose sum sum_columns leaves in lane (a, c)
__device__ __forceinline__ int token_of(int a, int c) { return 16 * (c >> 2) + 4 * a + (c & 3); }

__device__ __forceinline__ float sum_wave(float x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

__device__ __forceinline__ float faded(const hs_mass_args& A, int64_t i) { return A.in == nullptr || A.decay == 0.f ? 0.f : A.decay * A.in[i]; }

// mass_out of one tile from the sum of each lane's token
__device__ __forceinline__ void put(const hs_mass_args& A, int64_t row, int t, float sum, int l) {
  if (A.per_token) {
    const int64_t i = (row * A.T + t) * HS_BT + token_of(l >> 4, l & 15);
    A.out[i] = faded(A, i) + sum;
  } else {
    sum = sum_wave(sum);
    const int64_t i = row * A.T + t;
    if (l == 0) A.out[i] = faded(A, i) + sum;
  }
}

// One query per head.  HBM-bound on the packed keys: a wave takes a tile, reads each of its bytes once, straight into operand registers.
// Columns are the group's heads.
template <bool F16, int KM>
__global__ __launch_bounds__(256) void mass_step_kernel(hs_mass_args A, hs_kv_dev kv, float scale_log2) {
  const int tid = threadIdx.x, l = tid & 63, a = l >> 4, c = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t = blockIdx.x * 4 + w, hkv = blockIdx.y, b = blockIdx.z;
  if (t >= A.T) return;
  const int G = A.Hq / A.Hkv;
  const int64_t row = (int64_t)b * A.Hkv + hkv;
  const int mk = __builtin_amdgcn_readfirstlane(kv.k_map[row * A.T + t]);
  KTile<KM> r;
  if (mk != 0) k_load(r, kv, row, mk, l);
  // the dense tail belongs to this tile?
  int tail_len = 0;
  if (A.tail_k != nullptr && t == (A.tail_tiles != nullptr ? A.tail_tiles[b] : A.tail_tile))
    tail_len = A.tail_lens != nullptr ? min(max(A.tail_lens[b], 0), HS_BT) : A.tail_len;
  tail_len = __builtin_amdgcn_readfirstlane(tail_len);
  const int64_t hq = (int64_t)hkv * G + (c < G ? c : 0);
  const uint16_t* q = A.q + b * A.q_sb + hq * A.q_sh + 8 * a;
  uint4 qb[4];
#pragma unroll
  for (int s = 0; s < 4; s++) qb[s] = c < G ? *reinterpret_cast<const uint4*>(q + 32 * s) : make_uint4(0, 0, 0, 0);
  const float lse = A.lse[b * A.l_sb + hq * A.l_sh];
  const bool counts = c < G && fabsf(lse) < INFINITY;
  const float lse2 = lse * kLog2e;
  float v[16];
#pragma unroll
  for (int e = 0; e < 16; e++) v[e] = 0.f;
  if (mk != 0) {
    f32x4_t s[4];
    scores<F16, KM>(r, mk < 0, qb, s);
#pragma unroll
    for (int e = 0; e < 16; e++) v[e] = counts ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 2][e & 3], scale_log2, -lse2)) : 0.f;
  }
  if (tail_len > 0) {
    typedef hs_elem<F16> E;
    const uint16_t* tk = A.tail_k + (row * HS_BT + c) * HS_D + 8 * a;
#pragma unroll
    for (int m = 0; m < 4; m++) {
      f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < 4; st++) {
        const uint4 kk = 16 * m + c < tail_len ? *reinterpret_cast<const uint4*>(tk + 16 * m * HS_D + 32 * st) : make_uint4(0, 0, 0, 0);
        s = E::mma(kk, qb[st], s);
      }
#pragma unroll
      for (int i = 0; i < 4; i++)
        if (counts && 16 * m + 4 * a + i < tail_len) v[4 * m + i] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale_log2, -lse2));
    }
  }
  put(A, row, t, sum_columns(v, c), l);
}

// ---- many queries ----
// The queries of a kv head's group are numbered query by query, the group's heads side by side (column f: query f / G, head f % G), and pass
// by in blocks of 32 columns: the B operand of the 32x32x16 matrix instruction, staged in LDS for the workgroup's four waves, which hold
// a tile of 64 tokens each.  2:4 tiles are expanded once into the dense form: they stay in registers for thousands of queries, the exponentials
// bound the kernel (16 a lane and 1024 scores; two half-empty sparse products would save matrix time that is not short and cost
// 16 moves to clear their accumulators), and beside the 32x32 form the vector ALU keeps more of its rate than beside the 16x16 ones.
//
// Matrix operands of 32x32x16: lane l = 32 hi + r holds row (column) r and 8 values of k; step (kb, u, half) takes channels
// 64 kb + 32 u + 16 hi + 8 half + e, in K and Q alike.  Result: column r, rows 8 (i / 4) + 4 hi + i % 4, i = 0..15.
typedef float f32x16_t __attribute__((ext_vector_type(16)));
template <bool F16>
__device__ __forceinline__ f32x16_t mma32(uint4 a, uint4 b, f32x16_t c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// A tile's operands k[row block][step], from wherever the pool's order has them.
__device__ __forceinline__ void k_operands(uint4 (&k)[2][8], const hs_kv_dev& kv, int64_t row, int mk, int l) {  // mk != 0, wave-uniform
  const int hi = l >> 5, r = l & 15, mr = (l >> 4) & 1;
  if (mk > 0) {
    const uint8_t* p = kv.k_dense + (row * kv.cap_dense_k + (mk - 1)) * (int64_t)HS_TILE_DENSE_BYTES;
#pragma unroll
    for (int R = 0; R < 2; R++)
#pragma unroll
      for (int s = 0; s < 8; s++) {  // s = 4 kb + 2 u + half: chunk 4 m + 2 kb + u, lane group 2 hi + half
        const int chunk = 4 * (2 * R + mr) + (s >> 1), lane = 16 * (2 * hi + (s & 1)) + r;
        k[R][s] = ld_stream(reinterpret_cast<const uint4*>(p + 1024 * chunk + 16 * lane));
      }
    return;
  }
  const int64_t slot = row * kv.cap_sparse_k + (-mk - 1);
  const uint8_t* p = kv.k_nnz + slot * (int64_t)HS_TILE_NNZ_BYTES;
  const uint8_t* pm = kv.k_meta + slot * (int64_t)HS_TILE_META_BYTES;
  uint4 kept[2][4];      // [row block][2 kb + u]: 16 channels
  uint32_t idx[2][2];    // [row block][u]: both kb
#pragma unroll
  for (int R = 0; R < 2; R++)
#pragma unroll
    for (int u = 0; u < 2; u++) {
      const int m = 2 * R + mr, lane = 16 * (2 * u + hi) + r;
#pragma unroll
      for (int kb = 0; kb < 2; kb++) kept[R][2 * kb + u] = ld_stream(reinterpret_cast<const uint4*>(p + 1024 * (2 * m + kb) + 16 * lane));
      idx[R][u] = *reinterpret_cast<const uint32_t*>(pm + 16 * lane + 4 * m);
    }
#pragma unroll
  for (int R = 0; R < 2; R++)
#pragma unroll
    for (int kb = 0; kb < 2; kb++)
#pragma unroll
      for (int u = 0; u < 2; u++) {
        const uint4 v = kept[R][2 * kb + u];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w}, where = idx[R][u] >> (16 * kb);
        uint32_t d[8];
#pragma unroll
        for (int q = 0; q < 4; q++) {  // two values into their places of four
          const uint32_t at = where >> (4 * q);
          const uint64_t x = ((uint64_t)(w[q] & 0xffffu) << (16 * (at & 3u))) | ((uint64_t)(w[q] >> 16) << (16 * ((at >> 2) & 3u)));
          d[2 * q] = (uint32_t)x;
          d[2 * q + 1] = (uint32_t)(x >> 32);
        }
        k[R][4 * kb + 2 * u] = make_uint4(d[0], d[1], d[2], d[3]);
        k[R][4 * kb + 2 * u + 1] = make_uint4(d[4], d[5], d[6], d[7]);
      }
}

// Direct loads into LDS, lane l's bytes to base + 16 l (4 l).  Inline assembly: the compiler would wait for all of them in front of any LDS
// read; they are waited for by count (landed) and a barrier instead.
typedef __attribute__((address_space(3))) void* lptr_t;
__device__ __forceinline__ void lds_load16(uint32_t base, const void* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(base), "v"((uint64_t)p) : "memory", "m0");
}
__device__ __forceinline__ void lds_load4(uint32_t base, const void* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(base), "v"((uint64_t)p) : "memory", "m0");
}

constexpr int kStages = 3;                        // a block is requested two blocks ahead
constexpr int kStageBytes = 8 * 1024 + 4 * 256;   // 8 steps of 64 lanes x 16 bytes, and a copy of the columns' LSE for each wave
constexpr int kGroup = 4;                         // tiles of a workgroup

template <bool F16, bool TOKEN>
__global__ __launch_bounds__(256, 2) void mass_kernel(hs_mass_args A, hs_kv_dev kv, float scale_log2) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[kStages * kStageBytes];
  const int tid = threadIdx.x, l = tid & 63, hi = l >> 5, r = l & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_groups = (A.T + kGroup - 1) / kGroup;
  const int hkv = blockIdx.x % A.Hkv, rest = blockIdx.x / A.Hkv, group = rest % n_groups, range = rest / n_groups, b = blockIdx.y;
  const int G = A.Hq / A.Hkv;
  const int64_t row = (int64_t)b * A.Hkv + hkv;
  const int t = kGroup * group + w;
  const bool mine = t < A.T;
  const int mk = mine ? __builtin_amdgcn_readfirstlane(kv.k_map[row * A.T + t]) : 0;
  // blocks of this workgroup: its range's, from the first with a query that sees its first tile on
  const int64_t columns = (int64_t)A.Lq * G;
  const int blocks = (int)((columns + 31) / 32);
  const int64_t first_query = A.causal ? max(0, HS_BT * kGroup * group - A.q_start) : 0;
  const int lo = max((int)((int64_t)blocks * range / A.n_ranges), (int)(first_query * G / 32)), hi_blk = (int)((int64_t)blocks * (range + 1) / A.n_ranges);
  float acc[2][16];
#pragma unroll
  for (int R = 0; R < 2; R++)
#pragma unroll
    for (int i = 0; i < 16; i++) acc[R][i] = 0.f;
  float tile_sum = 0.f;

  if (lo < hi_blk) {
    uint4 k[2][8];
    if (mk != 0) k_operands(k, kv, row, mk, l);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lptr_t)lds);
    // the lane's column of the next block to request
    const int64_t f0 = (int64_t)32 * lo + r;
    int qi = (int)(f0 / G), qg = (int)(f0 % G);
    const int step_i = 32 / G, step_g = 32 % G;
    const uint16_t* q0 = A.q + b * A.q_sb + (int64_t)hkv * G * A.q_sh + 16 * hi;
    const float* l0 = A.lse + b * A.l_sb + (int64_t)hkv * G * A.l_sh;
    auto request = [&](int stage) {
      const uint32_t at = lds0 + stage * kStageBytes;
      const int i = min(qi, A.Lq - 1);  // columns past the last read it again and weigh nothing
      const uint16_t* q = q0 + qg * A.q_sh + i * A.q_st;
      // steps w and w + 4: (kb, u, half) = (0, w / 2, w % 2) and (1, same)
      const uint16_t* qw = q + 32 * (w >> 1) + 8 * (w & 1);
      lds_load16(at + 1024 * w, qw);
      lds_load16(at + 1024 * (w + 4), qw + 64);
      lds_load4(at + 8192 + 256 * w, l0 + qg * A.l_sh + i);
      qi += step_i; qg += step_g;
      if (qg >= G) { qg -= G; qi++; }
    };
    const int n = hi_blk - lo;
    __builtin_amdgcn_s_waitcnt(0x0f70);  // the tile's own loads: only the requests below are counted from here on
    request(0);
    if (n > 1) request(1);
    int ci = (int)(f0 / G), cg = (int)(f0 % G);  // the lane's column of the block at hand
    int stage = 0;
    for (int blk = 0; blk < n; blk++) {
      if (blk + 1 < n) asm volatile("s_waitcnt vmcnt(3) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (blk + 2 < n) request(stage == 0 ? 2 : stage - 1);
      // visible: the block's last query sees the tile's first token
      const int64_t f_last = min(columns, (int64_t)32 * (lo + blk + 1)) - 1;
      const int i_first = __builtin_amdgcn_readfirstlane(ci), i_last = (int)(f_last / G);
      if (mk != 0 && (!A.causal || A.q_start + i_last >= HS_BT * t)) {
        const uint4* qs = reinterpret_cast<const uint4*>(lds + stage * kStageBytes);
        f32x16_t s[2];
#pragma unroll
        for (int R = 0; R < 2; R++)
#pragma unroll
          for (int i = 0; i < 16; i++) s[R][i] = 0.f;
#pragma unroll
        for (int st = 0; st < 8; st++) {
          const uint4 q = qs[64 * st + l];
#pragma unroll
          for (int R = 0; R < 2; R++) s[R] = mma32<F16>(k[R][st], q, s[R]);
        }
        const float lse = *reinterpret_cast<const float*>(lds + stage * kStageBytes + 8192 + 256 * w + 4 * l);
        const float lse2 = lse * kLog2e;
        const bool counts = ci < A.Lq && fabsf(lse) < INFINITY;
        const bool all_seen = !A.causal || A.q_start + i_first >= HS_BT * t + HS_BT - 1;
        float p[2][16];
        if (all_seen && __ballot(!counts) == 0ull) {
#pragma unroll
          for (int R = 0; R < 2; R++)
#pragma unroll
            for (int i = 0; i < 16; i++) p[R][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[R][i], scale_log2, -lse2));
        } else {
          const int last = A.causal ? A.q_start + ci - HS_BT * t : HS_BT;  // last token of the tile that the column sees
#pragma unroll
          for (int R = 0; R < 2; R++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
              const bool seen = counts && 32 * R + 8 * (i >> 2) + 4 * hi + (i & 3) <= last;
              p[R][i] = seen ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[R][i], scale_log2, -lse2)) : 0.f;
            }
        }
        if (TOKEN) {
#pragma unroll
          for (int R = 0; R < 2; R++)
#pragma unroll
            for (int i = 0; i < 16; i++) acc[R][i] += p[R][i];
        } else {  // a tree first: few roundings per block
#pragma unroll
          for (int d = 8; d >= 1; d >>= 1)
#pragma unroll
            for (int i = 0; i < d; i++) {
              p[0][i] += p[0][i + d];
              p[1][i] += p[1][i + d];
            }
          tile_sum += p[0][0] + p[1][0];
        }
      }
      ci += step_i; cg += step_g;
      if (cg >= G) { cg -= G; ci++; }
      stage = stage == kStages - 1 ? 0 : stage + 1;
    }
  }
  if (!mine) return;

  const int64_t rows = (int64_t)A.B * A.Hkv;
  if (TOKEN) {
    float x[16];
    const bool b4 = l & 16;
#pragma unroll
    for (int i = 0; i < 16; i++) x[i] = (b4 ? acc[1][i] : acc[0][i]) + __shfl_xor(b4 ? acc[0][i] : acc[1][i], 16);
    const float sum = sum_columns(x, l & 15);
    const int i = l & 15, token = 16 * (l & 16) / 8 + 8 * (i >> 2) + 4 * hi + (i & 3);
    const int64_t at = (row * A.T + t) * HS_BT + token;
    if (A.n_ranges == 1) A.out[at] = faded(A, at) + sum;
    else A.ws[range * rows * A.T * HS_BT + at] = sum;
  } else {
    const float sum = sum_wave(tile_sum);
    const int64_t at = row * A.T + t;
    if (l == 0) {
      if (A.n_ranges == 1) A.out[at] = faded(A, at) + sum;
      else A.ws[range * rows * A.T + at] = sum;
    }
  }
}

// Joins the ranges' sums.
__global__ __launch_bounds__(256) void mass_join_kernel(hs_mass_args A, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float sum = 0.f;
  for (int r = 0; r < A.n_ranges; r++) sum += A.ws[r * n + i];
  A.out[i] = faded(A, i) + sum;
}

}  // namespace

int hs_mass_ranges(int B, int Hq, int Hkv, int T, int Lq, int causal, int per_token) {
  (void)causal;
  if (Lq == 1) return 1;
  const int64_t rows = (int64_t)B * Hkv, groups = rows * ((T + kGroup - 1) / kGroup), blocks = ((int64_t)Lq * (Hq / Hkv) + 31) / 32;
  const int64_t out_bytes = rows * T * (per_token ? HS_BT : 1) * 4;
  int64_t n = (4096 + groups - 1) / groups;
  if (n > blocks / 16) n = blocks / 16;
  if (n * out_bytes > ((int64_t)64 << 20)) n = ((int64_t)64 << 20) / out_bytes;
  return n < 1 ? 1 : (int)n;
}

hipError_t hs_launch_mass(const hs_mass_args& a, const hs_kv_dev& kv, int dtype, hipStream_t st) {
  const float sl2 = (float)((double)a.scale * 1.4426950408889634);
  const bool f16 = dtype == HS_FP16;
  if (a.Lq == 1 && !a.causal) {
    const int km = kv.cap_dense_k == 0 ? 0 : (kv.cap_sparse_k == 0 ? 1 : 2);
    const dim3 grid((a.T + 3) / 4, a.Hkv, a.B);
#define HS_STEP(F_, KM_) hipLaunchKernelGGL((mass_step_kernel<F_, KM_>), grid, dim3(256), 0, st, a, kv, sl2)
    if (f16) { if (km == 0) HS_STEP(true, 0); else if (km == 1) HS_STEP(true, 1); else HS_STEP(true, 2); }
    else { if (km == 0) HS_STEP(false, 0); else if (km == 1) HS_STEP(false, 1); else HS_STEP(false, 2); }
#undef HS_STEP
    return hipGetLastError();
  }
  const dim3 grid((unsigned)((a.T + kGroup - 1) / kGroup) * a.n_ranges * a.Hkv, a.B);
#define HS_MASS(F_, T_) hipLaunchKernelGGL((mass_kernel<F_, T_>), grid, dim3(256), 0, st, a, kv, sl2)
  if (f16) { if (a.per_token) HS_MASS(true, true); else HS_MASS(true, false); }
  else { if (a.per_token) HS_MASS(false, true); else HS_MASS(false, false); }
#undef HS_MASS
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_ranges == 1) return e;
  const int64_t n = (int64_t)a.B * a.Hkv * a.T * (a.per_token ? HS_BT : 1);
  hipLaunchKernelGGL(mass_join_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a, n);
  return hipGetLastError();
}
