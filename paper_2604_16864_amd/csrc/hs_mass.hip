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

// Many queries.  A workgroup takes one tile and a range of the query blocks (16 queries of one head); its 4 waves take the
// blocks in turn.
template <bool F16, int KM>
__global__ __launch_bounds__(256) void mass_kernel(hs_mass_args A, hs_kv_dev kv, float scale_log2) {
  const int tid = threadIdx.x, l = tid & 63, a = l >> 4, c = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t = blockIdx.x % A.T, range = blockIdx.x / A.T, hkv = blockIdx.y, b = blockIdx.z;
  const int G = A.Hq / A.Hkv;
  const int64_t row = (int64_t)b * A.Hkv + hkv;
  const int mk = __builtin_amdgcn_readfirstlane(kv.k_map[row * A.T + t]);
  __shared__ float sm[4][64];
  float v[16];
#pragma unroll
  for (int e = 0; e < 16; e++) v[e] = 0.f;
  if (mk != 0) {
    KTile<KM> r;
    k_load(r, kv, row, mk, l);
    const int blocks = (A.Lq + 15) / 16;
    const int first_seen = A.causal ? max(0, HS_BT * t - A.q_start) / 16 : 0;  // block of the first query that sees the tile
    const int lo = max((int)((int64_t)blocks * range / A.n_ranges), first_seen), hi = (int)((int64_t)blocks * (range + 1) / A.n_ranges);
    for (int64_t n = w; n < (int64_t)(hi - lo) * G; n += 4) {
      const int blk = lo + (int)(n / G), g = (int)(n % G);
      const int i = 16 * blk + c;  // the column's query
      const int64_t hq = (int64_t)hkv * G + g;
      const bool there = i < A.Lq;
      const uint16_t* q = A.q + b * A.q_sb + hq * A.q_sh + (there ? i : 0) * A.q_st + 8 * a;
      uint4 qb[4];
#pragma unroll
      for (int s = 0; s < 4; s++) qb[s] = *reinterpret_cast<const uint4*>(q + 32 * s);
      const float lse = A.lse[b * A.l_sb + hq * A.l_sh + (there ? i : 0)];
      const bool counts = there && fabsf(lse) < INFINITY;
      const float lse2 = lse * kLog2e;
      const int last = A.causal ? A.q_start + i - HS_BT * t : HS_BT;  // last token of the tile that the query sees
      f32x4_t s[4];
      scores<F16, KM>(r, mk < 0, qb, s);
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const bool seen = counts && 16 * (e >> 2) + 4 * a + (e & 3) <= last;
        v[e] += seen ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 2][e & 3], scale_log2, -lse2)) : 0.f;
      }
    }
  }
  sm[w][l] = sum_columns(v, c);
  __syncthreads();
  if (w != 0) return;
  float sum = (sm[0][l] + sm[1][l]) + (sm[2][l] + sm[3][l]);
  if (A.n_ranges == 1) {
    put(A, row, t, sum, l);
    return;
  }
  const int64_t rows = (int64_t)A.B * A.Hkv;
  if (A.per_token) {
    A.ws[((range * rows + row) * A.T + t) * HS_BT + token_of(a, c)] = sum;
  } else {
    sum = sum_wave(sum);
    if (l == 0) A.ws[(range * rows + row) * A.T + t] = sum;
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
  const int64_t rows = (int64_t)B * Hkv, blocks = (int64_t)((Lq + 15) / 16) * (Hq / Hkv);
  const int64_t out_bytes = rows * T * (per_token ? HS_BT : 1) * 4;
  int64_t n = (2048 + rows * T - 1) / (rows * T);
  if (n > blocks / 16) n = blocks / 16;            // at least 4 blocks a wave
  if (n * out_bytes > ((int64_t)64 << 20)) n = ((int64_t)64 << 20) / out_bytes;
  return n < 1 ? 1 : (int)n;
}

hipError_t hs_launch_mass(const hs_mass_args& a, const hs_kv_dev& kv, int dtype, hipStream_t st) {
  const int km = kv.cap_dense_k == 0 ? 0 : (kv.cap_sparse_k == 0 ? 1 : 2);
  const float sl2 = (float)((double)a.scale * 1.4426950408889634);
  const bool f16 = dtype == HS_FP16;
#define HS_MASS_KM(KERNEL_, GRID_, KM_)                                                                              \
  do {                                                                                                               \
    if (f16) hipLaunchKernelGGL((KERNEL_<true, KM_>), GRID_, dim3(256), 0, st, a, kv, sl2);                          \
    else hipLaunchKernelGGL((KERNEL_<false, KM_>), GRID_, dim3(256), 0, st, a, kv, sl2);                             \
  } while (0)
#define HS_MASS(KERNEL_, GRID_)                                                                                      \
  do {                                                                                                               \
    const dim3 grid GRID_;                                                                                           \
    if (km == 0) HS_MASS_KM(KERNEL_, grid, 0); else if (km == 1) HS_MASS_KM(KERNEL_, grid, 1); else HS_MASS_KM(KERNEL_, grid, 2); \
  } while (0)
  if (a.Lq == 1 && !a.causal) {
    HS_MASS(mass_step_kernel, ((a.T + 3) / 4, a.Hkv, a.B));
    return hipGetLastError();
  }
  HS_MASS(mass_kernel, ((unsigned)a.T * a.n_ranges, a.Hkv, a.B));
#undef HS_MASS
#undef HS_MASS_KM
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_ranges == 1) return e;
  const int64_t n = (int64_t)a.B * a.Hkv * a.T * (a.per_token ? HS_BT : 1);
  hipLaunchKernelGGL(mass_join_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a, n);
  return hipGetLastError();
}
