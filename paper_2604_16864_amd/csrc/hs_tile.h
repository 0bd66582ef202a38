// One tile of the packed cache under a wave of queries: its operands, the softmax recurrence, the dense tail and the join of a workgroup's parts.
// Shared by decode attention and attention over listed tiles.
#pragma once
#include <type_traits>

#include "hs_common.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;


// streaming (non-temporal) 16-byte load: decode attention reads the packed cache once per call
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
}
template <bool STREAM>
__device__ __forceinline__ uint4 ld_tile(const uint4* p) {
  if constexpr (STREAM) return ld_stream(p); else return *p;
}



// four consecutive 16-bit outputs; O is the caller's and need not be aligned to more than its elements
__device__ __forceinline__ void store4(uint16_t* p, uint32_t lo, uint32_t hi, bool aligned8) {
  if (aligned8) {
    *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
  } else {
    p[0] = (uint16_t)lo; p[1] = (uint16_t)(lo >> 16); p[2] = (uint16_t)hi; p[3] = (uint16_t)(hi >> 16);
  }
}

// Operand registers of one tile (K and V), filled by tile_load and consumed by tile_compute.
// KM / VM: kind of the K / V tile, 0 = 2:4, 1 = dense (the kernel sorts its tiles by kind first).
template <int KM, int VM>
struct TileRegs {
  static_assert((KM == 0 || KM == 1) && (VM == 0 || VM == 1), "one kind per operand");
  static constexpr int kNK = KM == 0 ? 8 : 16;  // 16-byte chunks per lane: 2:4 tile 8, dense tile 16
  static constexpr int kNV = VM == 0 ? 8 : 16;
  uint4 k[kNK];
  uint4 v[kNV];
  uint4 km, vm;  // the lane's four 32-bit index words of the K / V tile
};

// WHAT: 1 = K alone, 2 = V alone, 3 = both.  STREAM: what is read is not read again soon.
template <int KM, int VM, int WHAT = 3, bool STREAM = true>
__device__ __forceinline__ void tile_load(TileRegs<KM, VM>& r, const hs_kv_dev& kv, int64_t row, int mk, int mv, int l) {  // mk, mv: wave-uniform
  mv = hs_map_plain(mv);
  if (WHAT & 1) r.km = make_uint4(0, 0, 0, 0);  // only 2:4 tiles carry index words
  if (WHAT & 2) r.vm = make_uint4(0, 0, 0, 0);
  constexpr bool k_sparse = KM == 0, v_sparse = VM == 0;
  if (!(WHAT & 1)) {
  } else if (k_sparse) {
    const int64_t slot = row * kv.cap_sparse_k + (-mk - 1);
    const uint4* p = reinterpret_cast<const uint4*>(kv.k_nnz + slot * (int64_t)HS_TILE_NNZ_BYTES) + l;
#pragma unroll
    for (int i = 0; i < 8; i++) r.k[i] = ld_tile<STREAM>(p + 64 * i);
    r.km = ld_tile<STREAM>(reinterpret_cast<const uint4*>(kv.k_meta + slot * (int64_t)HS_TILE_META_BYTES) + l);
  } else {
    const int64_t slot = row * kv.cap_dense_k + (mk - 1);
    const uint4* p = reinterpret_cast<const uint4*>(kv.k_dense + slot * (int64_t)HS_TILE_DENSE_BYTES) + l;
#pragma unroll
    for (int i = 0; i < 16; i++) r.k[i % TileRegs<KM, VM>::kNK] = ld_tile<STREAM>(p + 64 * i);
  }
  if (!(WHAT & 2)) {
  } else if (v_sparse) {
    const int64_t slot = row * kv.cap_sparse_v + (-mv - 1);
    const uint4* p = reinterpret_cast<const uint4*>(kv.v_nnz + slot * (int64_t)HS_TILE_NNZ_BYTES) + l;
#pragma unroll
    for (int i = 0; i < 8; i++) r.v[i] = ld_tile<STREAM>(p + 64 * i);
    r.vm = ld_tile<STREAM>(reinterpret_cast<const uint4*>(kv.v_meta + slot * (int64_t)HS_TILE_META_BYTES) + l);
  } else {
    const int64_t slot = row * kv.cap_dense_v + (mv - 1);
    const uint4* p = reinterpret_cast<const uint4*>(kv.v_dense + slot * (int64_t)HS_TILE_DENSE_BYTES) + l;
#pragma unroll
    for (int i = 0; i < 16; i++) r.v[i % TileRegs<KM, VM>::kNV] = ld_tile<STREAM>(p + 64 * i);
  }
}

// One tile: GEMM1 (S^T = K Q^T), online softmax, GEMM2 (O^T += V^T P^T).
// F16: element type of the cache (hs_elem).  A V tile of a bf16 cache may be stored in fp16
// encoding (HS_MAP_F16 in its map entry); the numerators then go into GEMM2 as fp16 too.  The
// running reference sits kShift = 8 binades under the running maximum, so that numerators reach
// 2^8 and what fp16 flushes to zero is below 2^-32 of the largest one (a context of 2^17 tokens
// then loses < 2^-15 of the sum).
// ENC: 0 = V tile in bf16, 1 = in fp16 (encoding bit, or an fp16 cache).
// limit(s): what of the scores is not seen (set to -inf there); lane holds tokens 16 m + 4 a + i of its column in s[m][i].
struct SeesAll { __device__ __forceinline__ void operator()(f32x4_t (&)[4]) const {} };
template <int KM, int VM, bool F16, int ENC, typename Limit = SeesAll>
__device__ __forceinline__ void tile_compute(const TileRegs<KM, VM>& r, const uint4 (&qb)[4], float scale_log2, int c,
                                             f32x4_t (&o)[8], float& m_run, float& l_run, Limit limit = Limit()) {
  constexpr bool k_sparse = KM == 0, v_sparse = VM == 0;
  constexpr int kNK = TileRegs<KM, VM>::kNK, kNV = TileRegs<KM, VM>::kNV;
  typedef hs_elem<F16> E;
  typedef hs_elem<true> E16;
  constexpr float kShift = 8.f;
  constexpr bool v_f16 = ENC == 1;
  f32x4_t s[4];
  const int kidx[4] = {(int)r.km.x, (int)r.km.y, (int)r.km.z, (int)r.km.w};
  const int vidx[4] = {(int)r.vm.x, (int)r.vm.y, (int)r.vm.z, (int)r.vm.w};
#pragma unroll
  for (int m = 0; m < 4; m++) s[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (k_sparse) {  // the 4 row blocks are independent chains
#pragma unroll
    for (int m = 0; m < 4; m++)
      s[m] = E::template smma<0>(r.k[2 * m], qb[0], qb[1], s[m], kidx[m]);
#pragma unroll
    for (int m = 0; m < 4; m++)
      s[m] = E::template smma<1>(r.k[2 * m + 1], qb[2], qb[3], s[m], kidx[m]);
  }
#pragma unroll
  for (int m = 0; m < 4; m++) {
    if (!k_sparse) {
#pragma unroll
      for (int st = 0; st < 4; st++)
        s[m] = E::mma(r.k[(4 * m + st) % kNK], qb[st], s[m]);
    }
  }
  limit(s);
  // online softmax for column c (log2 domain)
  const float m_prev = m_run;
  float mx = -INFINITY;
#pragma unroll
  for (int m = 0; m < 4; m++)
#pragma unroll
    for (int i = 0; i < 4; i++) mx = fmaxf(mx, s[m][i]);
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  m_run = fmaxf(m_prev, mx * scale_log2 - kShift);
  const float m_ref = m_run > -INFINITY ? m_run : 0.f;  // every score -inf so far: weights 0, not exp2(-inf + inf)
  const float alpha = __builtin_amdgcn_exp2f(m_prev - m_ref);  // 0 on the first tile
  float psum = 0.f;
  // P^T as the B operand: element 8h+4u+i of lane group a <- token 16(2h+u)+4a+i.
  // Columns < 8 carry bf16(p), columns >= 8 carry bf16(p - bf16(p)), so that the sum of
  // the two accumulator columns sees p to ~16 bits although the operand type is bf16.
  float p[4][4];
#pragma unroll
  for (int m = 0; m < 4; m++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      p[m][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[m][i], scale_log2, -m_ref));
      psum += p[m][i];
    }
  uint32_t pb[8];
  auto pack_as = [&](auto enc) {
    typedef hs_elem<decltype(enc)::value> EP;
#pragma unroll
    for (int m = 0; m < 4; m++) {
      const uint32_t hi0 = EP::pack2(p[m][0], p[m][1]), hi1 = EP::pack2(p[m][2], p[m][3]);
      const uint32_t lo0 = EP::pack2(p[m][0] - EP::lo_f32(hi0), p[m][1] - EP::hi_f32(hi0));
      const uint32_t lo1 = EP::pack2(p[m][2] - EP::lo_f32(hi1), p[m][3] - EP::hi_f32(hi1));
      pb[2 * m] = c < 8 ? hi0 : lo0;
      pb[2 * m + 1] = c < 8 ? hi1 : lo1;
    }
  };
  if (v_f16) pack_as(std::true_type{});
  else pack_as(std::false_type{});
  l_run = l_run * alpha + psum;
#pragma unroll
  for (int i = 0; i < 8; i++) o[i] *= alpha;
  const uint4 pb_lo = make_uint4(pb[0], pb[1], pb[2], pb[3]);  // dense step h = 0
  const uint4 pb_hi = make_uint4(pb[4], pb[5], pb[6], pb[7]);  // dense step h = 1
  if (v_f16) {
#pragma unroll
    for (int mb = 0; mb < 8; mb++) {
      if (v_sparse) {
        if (mb & 1) o[mb] = E16::template smma<1>(r.v[mb], pb_lo, pb_hi, o[mb], vidx[mb >> 1]);
        else o[mb] = E16::template smma<0>(r.v[mb], pb_lo, pb_hi, o[mb], vidx[mb >> 1]);
      } else {
        o[mb] = E16::mma(r.v[(2 * mb) % kNV], pb_lo, o[mb]);
        o[mb] = E16::mma(r.v[(2 * mb + 1) % kNV], pb_hi, o[mb]);
      }
    }
  } else {
#pragma unroll
    for (int mb = 0; mb < 8; mb++) {
      if (v_sparse) {
        if (mb & 1) o[mb] = E::template smma<1>(r.v[mb], pb_lo, pb_hi, o[mb], vidx[mb >> 1]);
        else o[mb] = E::template smma<0>(r.v[mb], pb_lo, pb_hi, o[mb], vidx[mb >> 1]);
      } else {
        o[mb] = E::mma(r.v[(2 * mb) % kNV], pb_lo, o[mb]);
        o[mb] = E::mma(r.v[(2 * mb + 1) % kNV], pb_hi, o[mb]);
      }
    }
  }
}

// Which tile forms (bit 0 K dense, bit 1 V dense, bit 2 V in bf16 encoding) a kernel instantiation can meet:
// KM / VM 0 = every tile 2:4, 1 = every tile dense, 2 = any mix; an fp16 cache has no bf16-encoded tiles.
template <int KM, int VM, bool F16>
__host__ __device__ constexpr bool form_allowed(int f) {
  return ((f & 1) ? KM != 0 : KM != 1) && ((f & 2) ? VM != 0 : VM != 1) && ((f & 4) ? !F16 : true);
}
// fn(std::integral_constant<int, f>) for every allowed form f except SKIP_FORM, in ascending order
template <int KM, int VM, bool F16, int SKIP_FORM, int F = 0, typename Fn>
__device__ __forceinline__ void static_for_forms(Fn&& fn) {
  if constexpr (F < 8) {
    if constexpr (F != SKIP_FORM && form_allowed<KM, VM, F16>(F)) fn(std::integral_constant<int, F>{});
    static_for_forms<KM, VM, F16, SKIP_FORM, F + 1>(fn);
  }
}

// The dense tail (at most one tile of not yet compressed tokens) as seen by the split kernel: `len` < 0 = the call has
// none; `lens` (device, [B], or NULL) replaces `len` per batch row, kept inside the tail buffer.
struct TailArgs {
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* lens;
  int len;
};

// Q^T of one (batch, kv head) row as the B operand: columns 0..G-1 and 8..8+G-1 both hold head column % 8 of the group
// (GEMM2 over the tiles gives the second copy the low-order half of P).  Head h of the group is at Q + (hq0 + h head_step) unit.
__device__ __forceinline__ void load_q(const uint16_t* __restrict__ Q, int64_t hq0, int64_t head_step, int unit, int G, int a, int c, uint4 (&qb)[4]) {
  const int head = c & 7;
  const bool valid = head < G;
  const uint16_t* q = Q + (hq0 + (valid ? head : 0) * head_step) * unit + 8 * a;
#pragma unroll
  for (int s = 0; s < 4; s++) qb[s] = valid ? *reinterpret_cast<const uint4*>(q + 32 * s) : make_uint4(0, 0, 0, 0);
}

// A wave's share of the dense tail of one row: tokens 16 q .. 16 q + 15 of the tail buffer, all query heads of the group, into the
// combine's slots (reference, sum, unnormalised O^T per column).  Everything it reads is requested at once; the scores come from
// the 16-bit matrix instruction like those of a dense tile, O^T from the 32-bit one, so that P keeps its 32 bits:
// its k is a lane group's token i (the accumulators of the scores are its B operand as they stand), its row r of block mb is channel
// 8 r + mb, so that a lane reads 8 consecutive channels of 4 tokens.  Tokens from tail_len on are not read.
// Latency-bound, one chain of load, products, exponentials, products.  The same on the vector ALU, with q and P in LDS, read
// the LDS once more per head and was the last to end: us a call, then / now, 8 rows of 256 tiles with a tail, 4 heads a row
// 14.1 / 12.5, 8 heads 16.1 / 12.8; 128 rows of 16 tiles 13.7 / 12.4, 15.9 / 12.8; 8 rows of 32 tiles 8.3 / 7.6, 10.1 / 7.6; with one
// head a row the same.
// AHEAD: the caller has raised the wave's priority, until its loads are requested.
template <bool F16, bool AHEAD>
__device__ __forceinline__ void tail_piece(const TailArgs& tail, int tail_len, int64_t row, int q, const uint4 (&qb)[4], float scale_log2,
                                           int l, float (&sm_o)[8][HS_D], float (&sm_m)[8], float (&sm_l)[8]) {
  typedef hs_elem<F16> E;
  const int a = l >> 4, c = l & 15, left = tail_len - 16 * q;  // left: wave-uniform
  float m = -INFINITY, sum = 0.f;
  f32x4_t o[8];
#pragma unroll
  for (int mb = 0; mb < 8; mb++) o[mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (left > 0) {
    const uint16_t* tk = tail.k + (row * HS_BT + 16 * q + c) * HS_D + 8 * a;
    const uint16_t* tv = tail.v + (row * HS_BT + 16 * q + 4 * a) * HS_D + 8 * c;
    uint4 kk[4], vv[4];
#pragma unroll
    for (int s = 0; s < 4; s++) kk[s] = c < left ? *reinterpret_cast<const uint4*>(tk + 32 * s) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; i++) vv[i] = 4 * a + i < left ? *reinterpret_cast<const uint4*>(tv + i * HS_D) : make_uint4(0, 0, 0, 0);
    if constexpr (AHEAD) { __builtin_amdgcn_sched_barrier(0); __builtin_amdgcn_s_setprio(0); }
    f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < 4; st++) s = E::mma(kk[st], qb[st], s);
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if (4 * a + i >= left) s[i] = -INFINITY;
      mx = fmaxf(mx, s[i]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    m = mx * scale_log2;
    const float ref = m > -INFINITY ? m : 0.f;  // every score -inf: weights 0, not exp2(-inf + inf)
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale_log2, -ref));
      sum += p[i];
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const uint32_t d[4] = {vv[i].x, vv[i].y, vv[i].z, vv[i].w};
#pragma unroll
      for (int mb = 0; mb < 8; mb++)
        o[mb] = __builtin_amdgcn_mfma_f32_16x16x4f32(mb & 1 ? E::hi_f32(d[mb >> 1]) : E::lo_f32(d[mb >> 1]), p[i], o[mb], 0, 0, 0);
    }
  }
  if (c < 8) {
    if (a == 0) { sm_m[c] = m; sm_l[c] = sum; }
#pragma unroll
    for (int i = 0; i < 4; i++) {
      float4* d = reinterpret_cast<float4*>(&sm_o[c][8 * (4 * a + i)]);
      d[0] = make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
      d[1] = make_float4(o[4][i], o[5][i], o[6][i], o[7][i]);
    }
  }
}
// Combines the N parts that the waves have left in LDS (and, with_tail, the tail's four behind them) and writes the row's partial of split
// `slot`, or (DIRECT) its O and LSE.  hq0: the row of O of the group's first head, head_rows: rows from a head to the next.  Thread = (head tid / 32, 4 channels).  part_m, part_l, part_o: 8 heads a part.
// TAIL: the dense tail's four parts may stand behind the N.
template <bool F16, bool DIRECT, int N, bool TAIL = DIRECT>
__device__ __forceinline__ void combine_parts(int tid, bool with_tail, int G, int64_t hq0, int64_t head_rows, const float (*part_m)[8], const float (*part_l)[8],
                                              const float (*part_o)[8][HS_D], int n_splits, int slot, float* __restrict__ ws_o,
                                              float* __restrict__ ws_l) {
  const int g = tid >> 5, ch = (tid & 31) * 4;
  if (g >= G) return;
  const int64_t hq = hq0 + g * head_rows;
  float mstar = -INFINITY;
#pragma unroll
  for (int k = 0; k < N; k++) mstar = fmaxf(mstar, part_m[k][g]);
  if (TAIL && with_tail) {
#pragma unroll
    for (int k = N; k < N + 4; k++) mstar = fmaxf(mstar, part_m[k][g]);
  }
  // a part without a reference has seen nothing (l and O are 0) or only NaN scores (l is NaN): neither is left out,
  // and only l == 0 is an empty split, so that a NaN reaches O and LSE however the tiles are divided
  const float mref = mstar > -INFINITY ? mstar : 0.f;
  float lsum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](int k) {
    const float f = __builtin_amdgcn_exp2f(part_m[k][g] - mref);
    lsum += f * part_l[k][g];
#pragma unroll
    for (int i = 0; i < 4; i++) acc[i] += f * part_o[k][g][ch + i];
  };
#pragma unroll
  for (int k = 0; k < N; k++) add(k);
  if (TAIL && with_tail) {
#pragma unroll
    for (int k = N; k < N + 4; k++) add(k);
  }
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
  const float lse = lsum == 0.f ? -INFINITY : (mstar + __builtin_amdgcn_logf(lsum)) * kLn2;
  if constexpr (DIRECT) {
    typedef hs_elem<F16> E;
    uint16_t* po = reinterpret_cast<uint16_t*>(ws_o) + hq * HS_D + ch;
    store4(po, E::pack2(acc[0] * inv, acc[1] * inv), E::pack2(acc[2] * inv, acc[3] * inv), ((uintptr_t)ws_o & 7) == 0);
    if (ws_l != nullptr && (tid & 31) == 0) ws_l[hq] = lse;
  } else {
    float* po = ws_o + (hq * n_splits + slot) * HS_D + ch;
    *reinterpret_cast<float4*>(po) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
    if ((tid & 31) == 0) ws_l[hq * n_splits + slot] = lse;
  }
}

}  // namespace
