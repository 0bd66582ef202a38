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
// Columns are the group's heads.  8 rows of 512 2:4 tiles (37.8 MB) take 7.1 us, 64 rows of 2048 with half of them held (606 MB) 93 us, 6.5 TB/s.
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
// What bounds it: the vector ALU.  Per score it has a fused multiply-add, an exponential (two issue slots) and an addition.  In a 16K prompt, 32
// heads, 2:4 keys, 32 columns and a tile take 807 clocks of a SIMD; in 627 of them (78 %, by the counters) it issues 125 instructions and the 32
// exponentials' second slots, 4 clocks each: 552 are the scores' three instructions and 10 matrix ones, the rest addresses, limits and the blocks in
// which a query's view ends.  The matrix pipe is busy for 40 %.  The power limit holds the clock at 2.0 to 2.1 GHz.
// us, on one card: the prompt 813, per token 863; 4096 queries on 16K tokens, 2:4 keys per tile 369, per token 400, dense keys 478 and 500.  A barrier
// every two blocks, and the columns' LSE once, are worth 1 to 2 % of it.  Measured beside it, where the prompt took 800: two tiles a wave, for half
// of the reads of LDS and L2, 1005 (2 waves per SIMD instead of 3); the scheduler's own order, products first, 1155.
//
// The queries of a kv head's group pass by in blocks of 32 columns (32 / G queries, the group's G heads of each side by side), the B operand of
// the 32x32 matrix instructions, staged in LDS for the workgroup's four waves, which hold a tile of 64 tokens each.
//
// Matrix operands: lane l = 32 hi + r holds row (column) r.  Step (kb, u, p) takes 16 channels, 64 kb + 32 u + 16 p + 8 hi + e from lane group hi;
// a sparse step (kb, u) takes the 32 channels of p = 0 and 1: its B operand is that of the two dense steps, its A operand the
// kept values of the 16 channels 64 kb + 32 u + 16 hi, a piece of a 2:4 tile as the pool has it.
// Result: column r, rows 8 (i / 4) + 4 hi + i % 4, i = 0..15.
typedef float f32x16_t __attribute__((ext_vector_type(16)));
template <bool F16>
__device__ __forceinline__ f32x16_t mma32(uint4 a, uint4 b, f32x16_t c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
template <bool F16, int ABID>
__device__ __forceinline__ f32x16_t smma32(uint4 a, uint4 b0, uint4 b1, f32x16_t c, int idx) {
  const hs_u4x2 b{b0, b1};
  if constexpr (F16) return __builtin_amdgcn_smfmac_f32_32x32x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x16_t, b), c, idx, 0, ABID);
  else return __builtin_amdgcn_smfmac_f32_32x32x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x16_t, b), c, idx, 0, ABID);
}

// Two kept values into their places of four channels.
__device__ __forceinline__ uint2 spread(uint32_t kept, uint32_t at) {
  const uint64_t x = ((uint64_t)(kept & 0xffffu) << (16 * (at & 3u))) | ((uint64_t)(kept >> 16) << (16 * ((at >> 2) & 3u)));
  return make_uint2((uint32_t)x, (uint32_t)(x >> 32));
}

// A tile's operands, from wherever the pool's order has them, and its products with a block of queries x[step].
// DENSE: of a tile of either kind, 2:4 ones expanded.
template <bool F16, bool DENSE>
struct KTile32 {
  uint4 k[2][8];  // [row block][step 4 kb + 2 u + p]
  __device__ __forceinline__ void load(const hs_kv_dev& kv, int64_t row, int mk, int l) {  // mk != 0, wave-uniform
    const int hi = l >> 5, r = l & 15, mr = (l >> 4) & 1;
    if (mk > 0) {
      const uint8_t* p = kv.k_dense + (row * kv.cap_dense_k + (mk - 1)) * (int64_t)HS_TILE_DENSE_BYTES;
#pragma unroll
      for (int R = 0; R < 2; R++)
#pragma unroll
        for (int s = 0; s < 8; s++) {  // chunk 4 m + 2 kb + u, lane group 2 p + hi
          const int chunk = 4 * (2 * R + mr) + (s >> 1), lane = 16 * (2 * (s & 1) + hi) + r;
          k[R][s] = ld_stream(reinterpret_cast<const uint4*>(p + 1024 * chunk + 16 * lane));
        }
      return;
    }
    const int64_t slot = row * kv.cap_sparse_k + (-mk - 1);
    const uint8_t* pv = kv.k_nnz + slot * (int64_t)HS_TILE_NNZ_BYTES;
    const uint8_t* pm = kv.k_meta + slot * (int64_t)HS_TILE_META_BYTES;
    uint2 kept[2][8];      // channels 8 hi .. 8 hi + 7 of a piece
    uint32_t idx[2][4];    // [row block][2 u + p]: both kb
#pragma unroll
    for (int R = 0; R < 2; R++)
#pragma unroll
      for (int a = 0; a < 4; a++) {
        const int m = 2 * R + mr, lane = 16 * a + r;
#pragma unroll
        for (int kb = 0; kb < 2; kb++) kept[R][4 * kb + a] = *reinterpret_cast<const uint2*>(pv + 1024 * (2 * m + kb) + 16 * lane + 8 * hi);
        idx[R][a] = *reinterpret_cast<const uint32_t*>(pm + 16 * lane + 4 * m);
      }
#pragma unroll
    for (int R = 0; R < 2; R++)
#pragma unroll
      for (int s = 0; s < 8; s++) {
        const uint32_t at = idx[R][s & 3] >> (16 * (s >> 2) + 8 * hi);
        const uint2 lo4 = spread(kept[R][s].x, at), hi4 = spread(kept[R][s].y, at >> 4);
        k[R][s] = make_uint4(lo4.x, lo4.y, hi4.x, hi4.y);
      }
  }
  static constexpr int kSteps = 16;
  // step i of the products of x into s (both row blocks)
  __device__ __forceinline__ void step(int i, const uint4 (&x)[8], f32x16_t (&s)[2]) const {
    const f32x16_t zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int st = i >> 1, R = i & 1;
    s[R] = mma32<F16>(k[R][st], x[st], st == 0 ? zero : s[R]);
  }
};
// 2:4 tiles.  The sparse instruction adds to its accumulators in place: instead of clearing them (32 moves a block) the first 32 channels
// go through the dense one, expanded.
template <bool F16>
struct KTile32<F16, false> {
  uint4 first[2][2];     // [row block][p]: channels 0 .. 31
  uint4 k[2][3];         // [row block][sparse step 2 kb + u - 1]
  uint32_t idx[2][2];    // [row block][u]: both kb
  __device__ __forceinline__ void load(const hs_kv_dev& kv, int64_t row, int mk, int l) {  // mk < 0, wave-uniform
    const int hi = l >> 5, r = l & 15, mr = (l >> 4) & 1;
    const int64_t slot = row * kv.cap_sparse_k + (-mk - 1);
    const uint8_t* pv = kv.k_nnz + slot * (int64_t)HS_TILE_NNZ_BYTES;
    const uint8_t* pm = kv.k_meta + slot * (int64_t)HS_TILE_META_BYTES;
    uint2 kept[2][2];
    uint32_t at[2][2];
#pragma unroll
    for (int R = 0; R < 2; R++) {
      const int m = 2 * R + mr;
#pragma unroll
      for (int p = 0; p < 2; p++) {
        const int lane = 16 * p + r;
        kept[R][p] = *reinterpret_cast<const uint2*>(pv + 1024 * (2 * m) + 16 * lane + 8 * hi);
        at[R][p] = *reinterpret_cast<const uint32_t*>(pm + 16 * lane + 4 * m);
      }
#pragma unroll
      for (int s = 1; s < 4; s++) {  // 2 kb + u
        const int lane = 16 * (2 * (s & 1) + hi) + r;
        k[R][s - 1] = *reinterpret_cast<const uint4*>(pv + 1024 * (2 * m + (s >> 1)) + 16 * lane);
      }
#pragma unroll
      for (int u = 0; u < 2; u++) idx[R][u] = *reinterpret_cast<const uint32_t*>(pm + 16 * (16 * (2 * u + hi) + r) + 4 * m);
    }
#pragma unroll
    for (int R = 0; R < 2; R++)
#pragma unroll
      for (int p = 0; p < 2; p++) {
        const uint32_t w = at[R][p] >> (8 * hi);
        const uint2 lo4 = spread(kept[R][p].x, w), hi4 = spread(kept[R][p].y, w >> 4);
        first[R][p] = make_uint4(lo4.x, lo4.y, hi4.x, hi4.y);
      }
  }
  static constexpr int kSteps = 10;
  __device__ __forceinline__ void step(int i, const uint4 (&x)[8], f32x16_t (&s)[2]) const {
    const f32x16_t zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int st = i >> 1, R = i & 1;
    if (st < 2) s[R] = mma32<F16>(first[R][st], x[st], st == 0 ? zero : s[R]);
    else if (st == 2) s[R] = smma32<F16, 0>(k[R][0], x[2], x[3], s[R], (int)idx[R][1]);
    else if (st == 3) s[R] = smma32<F16, 1>(k[R][1], x[4], x[5], s[R], (int)idx[R][0]);
    else s[R] = smma32<F16, 1>(k[R][2], x[6], x[7], s[R], (int)idx[R][1]);
  }
};

// Direct loads into LDS, lane l's bytes to base + 16 l (4 l), from a uniform address + the lane's offset.  Inline assembly: the compiler would
// wait for all of them in front of any LDS read; they are waited for by count and a barrier instead.
typedef __attribute__((address_space(3))) void* lptr_t;
__device__ __forceinline__ void lds_load16(uint32_t base, const void* p, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(base), "v"(off), "s"((uint64_t)p) : "memory", "m0");
}
__device__ __forceinline__ void lds_load4(uint32_t base, const void* p, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(base), "v"(off), "s"((uint64_t)p) : "memory", "m0");
}

constexpr int kStages = 4;                        // two blocks are worked on while the next two are on their way
constexpr int kStageBytes = 8 * 1024 + 256;       // 32 columns of 256 bytes, and the columns' LSE (twice)
constexpr int kGroup = HS_MASS_TILES;
constexpr int kAhead = 2;                         // pairs of exponentials in front of a block's first products
// Products of a block beside the exponentials of the one before (two sets of scores), or one set and, for the registers that this frees, 3 waves per
// SIMD instead of 2 (dense keys, and 2:4 ones per token).  us, beside / one set, on one card: dense keys per tile, 4096 queries on 16K tokens 491 / 478, 512
// on 4 x 4K 79 / 78, a 2K prompt 36.7 / 31.7, a 16K one 1026 / 1021, 100 queries on 32K 39.1 / 39.3; per token 4096 queries 500 / 615, a 16K prompt 1048 / 1262
// (55 registers spilled; beside, one).  2:4 keys per tile, 3 waves either way: 4096 queries 369 / 365, 128 on 32K 37.7 / 36.5, 512 on 4 x 4K 65 / 62, a 16K
// prompt 813 / 826, a 2K one 29.2 / 31.6; per token 4096 queries 400 / 409, 128 on 32K 40.2 / 41.0, 512 on 4 x 4K 73 / 73, a 16K prompt 864 / 899, a 2K one
// 37.7 / 32.6.
constexpr bool beside(bool token, bool dense) { return token || !dense; }

// A block's 32 columns lie in LDS one after the other, the 16-byte chunks of column r exchanged by c -> c ^ (r & 15): loads from memory are of
// whole 256-byte vectors, 4 to an instruction (as matrix operands, 16 bytes of 64 vectors to an instruction, they cost 500 clocks a
// block), and reads of one chunk of 32 columns touch every bank alike.
template <bool F16, bool TOKEN, bool DENSE>
__global__ __launch_bounds__(256, beside(TOKEN, DENSE) ? 2 : 3) void mass_kernel(hs_mass_args A, hs_kv_dev kv, float scale_log2) {
  __shared__ __attribute__((aligned(256))) uint8_t lds[kStages * kStageBytes];
  const int tid = threadIdx.x, l = tid & 63, hi = l >> 5, r = l & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_groups = (A.T + kGroup - 1) / kGroup;
  const int hkv = blockIdx.x % A.Hkv, rest = blockIdx.x / A.Hkv, group = rest % n_groups, range = rest / n_groups, b = blockIdx.y;
  const int G = A.Hq / A.Hkv, Q = 32 / G;  // queries of a block
  const int64_t row = (int64_t)b * A.Hkv + hkv;
  const int64_t rows = (int64_t)A.B * A.Hkv;
  // The wave's tile: of the row's held ones number kGroup group + w (none: mk == 0, and no query sees it).  Where tiles may be missing the
  // workgroup numbers them, and its waves write the sums of 0 of the missing ones among the tiles kGroup group + w.
  int t = kGroup * group + w, t_first = kGroup * group, mk = 0;
  if (!A.numbered) {
    if (t < A.T) mk = __builtin_amdgcn_readfirstlane(kv.k_map[row * A.T + t]);
  } else {
    __shared__ int counts[8][4], found[kGroup][2];
    const int32_t* map = kv.k_map + row * A.T;
    if (t < A.T && map[t] == 0) {  // wave-uniform
      const int per = TOKEN ? HS_BT : 1;
      if (l < per) {
        const int64_t at = (row * A.T + t) * per + l;
        if (A.n_ranges == 1) A.out[at] = faded(A, at);
        else A.ws[range * rows * A.T * per + at] = 0.f;
      }
    }
    if (tid < kGroup) found[tid][0] = 0x7fffffff;
    int carried = 0;
    for (int base = 0; base < A.T && carried < kGroup * (group + 1); base += 2048) {
      int m[8];
#pragma unroll
      for (int j = 0; j < 8; j++) m[j] = base + 256 * j + tid < A.T ? map[base + 256 * j + tid] : 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const unsigned long long held = __ballot(m[j] != 0);
        if (l == 0) counts[j][w] = __builtin_popcountll(held);
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const unsigned long long held = __ballot(m[j] != 0);
        int before = carried;
#pragma unroll
        for (int k = 0; k < 4; k++) {
          if (k < w) before += counts[j][k];
          carried += counts[j][k];
        }
        const int number = before + __builtin_popcountll(held & ((1ull << l) - 1ull)) - kGroup * group;
        if (m[j] != 0 && number >= 0 && number < kGroup) { found[number][0] = base + 256 * j + tid; found[number][1] = m[j]; }
      }
    }
    __syncthreads();
    t_first = __builtin_amdgcn_readfirstlane(found[0][0]);
    if (t_first == 0x7fffffff) return;  // the whole workgroup: fewer tiles are held
    t = __builtin_amdgcn_readfirstlane(found[w][0]);
    mk = t != 0x7fffffff ? __builtin_amdgcn_readfirstlane(found[w][1]) : 0;
    if (mk == 0) t = A.T;
  }
  const bool mine = mk != 0 || (!A.numbered && t < A.T);
  // blocks of this workgroup: its range's, from the first with a query that sees its first tile on
  const int blocks = (A.Lq + Q - 1) / Q;
  const int lo = max((int)((int64_t)blocks * range / A.n_ranges), A.causal ? max(0, HS_BT * t_first - A.q_start) / Q : 0);
  const int n = (int)((int64_t)blocks * (range + 1) / A.n_ranges) - lo;
  float acc[2][16];
#pragma unroll
  for (int R = 0; R < 2; R++)
#pragma unroll
    for (int i = 0; i < 16; i++) acc[R][i] = 0.f;
  float tile_sum = 0.f;

  if (n > 0) {
    KTile32<F16, DENSE> tile;
    if (mk != 0) tile.load(kv, row, mk, l);
    // of these blocks, the first that the wave's tile has any query in, and the first from which on every query sees all of it
    const int vis = mk == 0 ? n : (A.causal ? max(0, max(0, HS_BT * t - A.q_start) / Q - lo) : 0);
    const int full = A.causal ? (max(0, HS_BT * t + HS_BT - 1 - A.q_start) + Q - 1) / Q - lo : 0;

    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lptr_t)lds);
    // What the lane loads of a block: chunk l % 16 of columns 8 w + l / 16 and the fourth behind it, and the LSE of column r.  Its offset from
    // the block's first query and head; columns beyond the block's (32 % G) take the first one.
    auto offset_of = [&](int column) -> uint32_t {
      const int i = column / G, g = column - i * G;
      return i < Q ? (uint32_t)(2 * (i * A.q_st + g * A.q_sh)) : 0u;
    };
    const int col0 = 8 * w + (l >> 4), col1 = col0 + 4;
    const uint32_t chunk0 = 16 * ((l & 15) ^ (col0 & 15)), chunk1 = 16 * ((l & 15) ^ (col1 & 15));
    const uint32_t off0 = offset_of(col0) + chunk0, off1 = offset_of(col1) + chunk1;
    const int my_i = r / G, my_g = r - my_i * G;  // the lane's column
    const uint32_t off_l = my_i < Q ? (uint32_t)(4 * (my_i + my_g * A.l_sh)) : 0u;
    const uint16_t* q = A.q + b * A.q_sb + (int64_t)hkv * G * A.q_sh + (int64_t)lo * Q * A.q_st;
    const float* ls = A.lse + b * A.l_sb + (int64_t)hkv * G * A.l_sh + (int64_t)lo * Q;
    const int64_t q_step = Q * A.q_st;
    const int n_whole = A.Lq / Q - lo;  // blocks before the one that ends inside
    auto request = [&](int blk, int stage) {
      const uint32_t at = lds0 + stage * kStageBytes;
      uint32_t o0 = off0, o1 = off1, ol = off_l;
      if (blk >= n_whole) {  // queries past the last: the first of the block again
        const int there = A.Lq - (lo + blk) * Q;
        if (col0 / G >= there) o0 = chunk0;
        if (col1 / G >= there) o1 = chunk1;
        if (my_i >= there) ol = 0;
      }
      lds_load16(at + 2048 * w, q, o0);
      lds_load16(at + 2048 * w + 1024, q, o1);
      if (w == (blk & 3)) lds_load4(at + 8192, ls, ol);
      q += q_step;
      ls += Q;
    };
    request(0, 0);
    if (n > 1) request(1, 1);

    int stage = kStages - 1;  // of the block last waited for
    // Waits for block blk (each one once, in order): for two at a time, and the two behind them are requested, into the stages that every wave
    // has left.
    auto wait_for = [&](int blk) {
      stage = (stage + 1) & (kStages - 1);
      if (blk & 1) return;
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (blk + 2 < n) request(blk + 2, stage ^ 2);
      if (blk + 3 < n) request(blk + 3, (stage ^ 2) + 1);
    };
    const uint32_t my_column = 256 * r + 16 * (hi ^ (r & 15)), my_lse = 8192 + 4 * l;
    auto fetch = [&](uint4 (&x)[8], float& lse) {
      const uint32_t at = stage * kStageBytes + my_column;
#pragma unroll
      for (int st = 0; st < 8; st++) x[st] = *reinterpret_cast<const uint4*>(lds + (at ^ (32 * st)));  // chunk 2 st + hi
      lse = *reinterpret_cast<const float*>(lds + stage * kStageBytes + my_lse);
    };
    // Columns past the last query and those whose LSE is not finite do not count, nor do tokens that a query does not see.  (Columns beyond the
    // block's are dropped with their lanes at the end.)
    auto weigh_seen = [&](const f32x16_t (&s)[2], float lse, int blk) {
      const int i0 = (lo + blk) * Q + my_i;
      const bool counts = fabsf(lse) < INFINITY && i0 < A.Lq;
      const int last = A.causal ? A.q_start + i0 - HS_BT * t : HS_BT;  // last token of the tile that the column sees
      const float lse2 = lse * kLog2e;
      float p[32];
#pragma unroll
      for (int e = 0; e < 32; e++) {
        const bool seen = counts && 32 * (e >> 4) + 8 * ((e & 15) >> 2) + 4 * hi + (e & 3) <= last;
        p[e] = seen ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 4][e & 15], scale_log2, -lse2)) : 0.f;
      }
      if (TOKEN) {
#pragma unroll
        for (int e = 0; e < 32; e++) acc[e >> 4][e & 15] += p[e];
      } else {
#pragma unroll
        for (int e = 4; e < 32; e++) p[e & 3] += p[e];
        tile_sum += (p[0] + p[1]) + (p[2] + p[3]);
      }
    };
    auto all_count = [&](float lse) { return __ballot(!(fabsf(lse) < INFINITY)) == 0ull; };
    // Where every query sees the whole tile and counts, the products of a block run beside the exponentials of the one before, which a wave
    // issues without waiting for either: a few scores a lane behind each matrix instruction, the first ones while the queries come
    // out of LDS.  The order is fixed by hand (left to the scheduler the products came first, one waiting for the other).
    auto both = [&](f32x16_t (&next)[2], float& lse_next, const f32x16_t (&cur)[2], float lse_cur) {
      uint4 x[8];
      fetch(x, lse_next);
      const float lse2 = lse_cur * kLog2e;
      float part[4] = {0.f, 0.f, 0.f, 0.f}, p[32];  // tiles: four sums per block first, few roundings
      auto sum = [&](int e) {
        if (TOKEN) acc[e >> 4][e & 15] += p[e];
        else part[e & 3] = e < 4 ? p[e] : part[e & 3] + p[e];
      };
      auto two = [&](int g) {  // scores 2 g and 2 g + 1; their sums behind the next pair's exponentials
#pragma unroll
        for (int e = 2 * g; e < 2 * g + 2; e++) p[e] = __builtin_fmaf(cur[e >> 4][e & 15], scale_log2, -lse2);
#pragma unroll
        for (int e = 2 * g; e < 2 * g + 2; e++) p[e] = __builtin_amdgcn_exp2f(p[e]);
        if (g > 0) { sum(2 * g - 2); sum(2 * g - 1); }
        __builtin_amdgcn_sched_barrier(0);
      };
      constexpr int kN = KTile32<F16, DENSE>::kSteps;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int g = 0; g < kAhead; g++) two(g);
#pragma unroll
      for (int i = 0; i < kN; i++) {
        tile.step(i, x, next);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = kAhead + (16 - kAhead) * i / kN; g < kAhead + (16 - kAhead) * (i + 1) / kN; g++) two(g);
      }
      sum(30); sum(31);
      if (!TOKEN) tile_sum += (part[0] + part[1]) + (part[2] + part[3]);
    };
    // the same scores without the products, tiles only
    auto weigh_all = [&](const f32x16_t (&s)[2], float lse) {
      const float lse2 = lse * kLog2e;
      float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 32; e++) part[e & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 4][e & 15], scale_log2, -lse2));
      tile_sum += (part[0] + part[1]) + (part[2] + part[3]);
    };
    f32x16_t s0[2], s1[2];
    float lse0, lse1;
    const int n_steady = min(n, n_whole) - 1;  // blocks that have a whole one behind them
    for (int blk = 0; blk < n;) {
      wait_for(blk);
      if (blk < vis) { blk++; continue; }
      {
        uint4 x[8];
        fetch(x, lse0);
#pragma unroll
        for (int i = 0; i < KTile32<F16, DENSE>::kSteps; i++) tile.step(i, x, s0);
      }
      if (beside(TOKEN, DENSE) && blk >= full) {
        for (;;) {
          if (blk >= n_steady || !all_count(lse0)) break;
          wait_for(blk + 1);
          both(s1, lse1, s0, lse0);
          blk++;
          if (blk >= n_steady || !all_count(lse1)) {
            s0[0] = s1[0]; s0[1] = s1[1]; lse0 = lse1;
            break;
          }
          wait_for(blk + 1);
          both(s0, lse0, s1, lse1);
          blk++;
        }
      }
      if (!beside(TOKEN, DENSE) && blk >= full && blk < n_whole && all_count(lse0)) {
        weigh_all(s0, lse0);
        blk++;
        continue;
      }
      weigh_seen(s0, lse0, blk);
      blk++;
    }
    if (my_i >= Q) {  // no column of any block
      tile_sum = 0.f;
#pragma unroll
      for (int e = 0; e < 32; e++) acc[e >> 4][e & 15] = 0.f;
    }
  }
  if (!mine) return;
  if (TOKEN) {
    float x[16];
    const bool b4 = l & 16;
#pragma unroll
    for (int i = 0; i < 16; i++) x[i] = (b4 ? acc[1][i] : acc[0][i]) + __shfl_xor(b4 ? acc[0][i] : acc[1][i], 16);
    const float sum = sum_columns(x, l & 15);
    const int i = l & 15, token = 2 * (l & 16) + 8 * (i >> 2) + 4 * hi + (i & 3);
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
  for (int r0 = 0; r0 < A.n_ranges; r0 += 16) {  // requested 16 at a time
    float x[16];
#pragma unroll
    for (int k = 0; k < 16; k++) x[k] = r0 + k < A.n_ranges ? A.ws[(r0 + k) * n + i] : 0.f;
#pragma unroll
    for (int k = 0; k < 16; k++) sum += x[k];
  }
  A.out[i] = faded(A, i) + sum;
}

}  // namespace

int hs_mass_ranges(int B, int Hq, int Hkv, int T, int Lq, int per_token) {
  if (Lq == 1) return 1;
  const int64_t rows = (int64_t)B * Hkv, groups = rows * ((T + kGroup - 1) / kGroup), queries = 32 / (Hq / Hkv), blocks = (Lq + queries - 1) / queries;
  const int64_t out_bytes = rows * T * (per_token ? HS_BT : 1) * 4;
  int64_t n = min((8192 + groups - 1) / groups, blocks / 16);
  n = max(n, min((512 + groups - 1) / groups, blocks / 4));
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
  // Tiles that may be missing: held ones are numbered (one pass over the row's map per workgroup, 2 us) where workgroups have much to do, or
  // there are more of them than fit the chip.
  hs_mass_args m = a;
  const int64_t workgroups = (int64_t)((a.T + kGroup - 1) / kGroup) * a.n_ranges * a.Hkv * a.B, queries = 32 / (a.Hq / a.Hkv);
  m.numbered = !kv.uniform && (workgroups > 512 || a.Lq / queries / a.n_ranges >= 16);
  const dim3 grid((unsigned)((a.T + kGroup - 1) / kGroup) * a.n_ranges * a.Hkv, a.B);
#define HS_MASS(F_, T_) \
  if (kv.cap_dense_k == 0) hipLaunchKernelGGL((mass_kernel<F_, T_, false>), grid, dim3(256), 0, st, m, kv, sl2); \
  else hipLaunchKernelGGL((mass_kernel<F_, T_, true>), grid, dim3(256), 0, st, m, kv, sl2)
  if (f16) { if (a.per_token) { HS_MASS(true, true); } else { HS_MASS(true, false); } }
  else { if (a.per_token) { HS_MASS(false, true); } else { HS_MASS(false, false); } }
#undef HS_MASS
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_ranges == 1) return e;
  const int64_t n = (int64_t)a.B * a.Hkv * a.T * (a.per_token ? HS_BT : 1);
  hipLaunchKernelGGL(mass_join_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a, n);
  return hipGetLastError();
}
