// Rotary positions on the way from the projection into the cache: queries and keys are turned, queries, keys and values put where
// attention and the cache take them from, in one launch.
//
// Pair i of a vector at position p turns by p theta_i.  In units of 2^-64 turns that is p turn_i modulo 2^64, an integer product:
// no position is too far for it, and its upper 32 bits, read as a signed number, are the angle in half turns times 2^31 within
// 2^-31.  Products and sums are taken in 32-bit floating point and rounded once to the output's 16 bits.
//
// HBM-bound: every vector is read once and written once.  A vector is the work of 8 lanes, two 16-byte chunks each: the two chunks
// whose channels turn together (halves), or any two (pairs, and channels that do not turn).  A thread computes the
// sines and cosines of its 8 pairs once and then takes the heads of its token in turn.
#include "hs_common.h"

namespace {

// NT: past the caches
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <bool NT>
__device__ __forceinline__ uint4 load16(const uint16_t* p) {
  if constexpr (NT) return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
  else return *reinterpret_cast<const uint4*>(p);
}
template <bool NT>
__device__ __forceinline__ void store16(uint16_t* p, uint4 v) {
  if constexpr (NT) __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), reinterpret_cast<u32x4_t*>(p));
  else *reinterpret_cast<uint4*>(p) = v;
}

struct Angles { float c[8], s[8]; };

// PAIRS: neighbouring channels turn together.  chunk0, chunk1: the lane's 16-byte chunks of a vector.
template <bool F16, bool PAIRS>
__device__ __forceinline__ void turn(uint4& x, uint4& y, const Angles& an) {
  typedef hs_elem<F16> E;
  uint32_t u[4] = {x.x, x.y, x.z, x.w}, v[4] = {y.x, y.y, y.z, y.w};
  if (PAIRS) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float a = E::lo_f32(u[i]), b = E::hi_f32(u[i]), c = E::lo_f32(v[i]), d = E::hi_f32(v[i]);
      u[i] = E::pack2(a * an.c[i] - b * an.s[i], a * an.s[i] + b * an.c[i]);
      v[i] = E::pack2(c * an.c[4 + i] - d * an.s[4 + i], c * an.s[4 + i] + d * an.c[4 + i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float a0 = E::lo_f32(u[i]), a1 = E::hi_f32(u[i]), b0 = E::lo_f32(v[i]), b1 = E::hi_f32(v[i]);
      u[i] = E::pack2(a0 * an.c[2 * i] - b0 * an.s[2 * i], a1 * an.c[2 * i + 1] - b1 * an.s[2 * i + 1]);
      v[i] = E::pack2(a0 * an.s[2 * i] + b0 * an.c[2 * i], a1 * an.s[2 * i + 1] + b1 * an.c[2 * i + 1]);
    }
  }
  x = make_uint4(u[0], u[1], u[2], u[3]);
  y = make_uint4(v[0], v[1], v[2], v[3]);
}

// A workgroup has 32 places of 8 lanes: `tokens` (a power of two) consecutive tokens of the flattened [B, n], and for each of them 32 / tokens
// heads side by side; a thread takes the heads h0 + place / tokens + i 32 / tokens of its token, up to `per` of them.
template <bool F16, bool PAIRS, bool NT>
__global__ __launch_bounds__(256) void rope_kernel(hs_rope_args A, int tokens_log2, int per) {
  const int tid = threadIdx.x, j = tid & 7, place = tid >> 3;
  const int tokens = 1 << tokens_log2, step = 32 >> tokens_log2;
  const int64_t at = (int64_t)blockIdx.x * tokens + (place & (tokens - 1));
  if (at >= (int64_t)A.B * A.n) return;
  const int b = (int)(at / A.n), i = (int)(at - (int64_t)b * A.n);
  const int nq = A.q.p != nullptr ? A.Hq : 0, nk = A.k.p != nullptr ? A.Hkv : 0, nv = A.v.p != nullptr ? A.Hkv : 0;
  const int h_end = min(nq + nk + nv, (int)(blockIdx.y + 1) * per * step);
  int h = (int)blockIdx.y * per * step + (place >> tokens_log2);
  if (h >= h_end) return;
  const int P = A.rope.rot_dim >> 4;  // lanes below P hold channels that turn (halves)
  int c0, c1;                         // the lane's chunks of 8 channels
  bool turns0, turns1;
  if (PAIRS) {
    c0 = j; c1 = j + 8;
    turns0 = c0 < 2 * P; turns1 = c1 < 2 * P;
  } else {
    c0 = j < P ? j : P + j; c1 = j < P ? j + P : j + 8;
    turns0 = turns1 = j < P;
  }
  const int64_t row = (A.rows != nullptr ? (int64_t)A.rows[b] : (int64_t)A.first_row) + i;
  const bool row_ok = row >= 0 && row < A.n_rows;
  // the vector of head slot h: queries, then keys, then values
  auto source = [&](int h) -> const uint16_t* {
    const hs_vec_view& s = h < nq ? A.q : (h < nq + nk ? A.k : A.v);
    const int hh = h < nq ? h : (h < nq + nk ? h - nq : h - nq - nk);
    return s.p + b * s.sb + hh * s.sh + i * s.st;
  };
  const uint16_t* p = source(h);
  uint4 x = load16<NT>(p + 8 * c0), y = load16<NT>(p + 8 * c1);
  Angles an;
  {
    const int64_t pos = A.positions != nullptr ? (int64_t)A.positions[at] : (int64_t)A.first_position + i;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const int pair = PAIRS ? 4 * (e < 4 ? c0 : c1) + (e & 3) : 8 * j + e;
      const bool turns = PAIRS ? (e < 4 ? turns0 : turns1) : turns0;
      float s = 0.f, c = 1.f;
      if (turns) {
        const uint64_t phase = (uint64_t)pos * A.rope.turn[pair & 63];
        sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &s, &c);
        s *= A.rope.gain; c *= A.rope.gain;
      }
      an.s[e] = s; an.c[e] = c;
    }
  }
  for (;;) {
    const int next = h + step;
    const bool more = next < h_end;
    uint4 xn, yn;
    if (more) {
      const uint16_t* pn = source(next);
      xn = load16<NT>(pn + 8 * c0);
      yn = load16<NT>(pn + 8 * c1);
    }
    if (h < nq + nk && (turns0 || turns1)) {
      const uint4 y0 = y;
      turn<F16, PAIRS>(x, y, an);
      if (PAIRS && !turns1) y = y0;  // bits of channels that do not turn stay (NaN payloads, -0)
    }
    uint16_t* d;
    bool ok = true;
    if (h < nq) {
      d = A.qo.p + b * A.qo.sb + h * A.qo.sh + i * A.qo.st;
    } else {
      const hs_vec_view& o = h < nq + nk ? A.ko : A.vo;
      d = o.p + b * o.sb + (h < nq + nk ? h - nq : h - nq - nk) * o.sh + row * o.st;
      ok = row_ok;
    }
    if (ok) {
      store16<NT>(d + 8 * c0, x);
      store16<NT>(d + 8 * c1, y);
    }
    if (!more) return;
    x = xn; y = yn; h = next;
  }
}

}  // namespace

hipError_t hs_launch_rope(const hs_rope_args& a, int dtype, hipStream_t st) {
  const int64_t at = (int64_t)a.B * a.n;
  const int heads = (a.q.p ? a.Hq : 0) + (a.k.p ? a.Hkv : 0) + (a.v.p ? a.Hkv : 0);
  // Beyond the last-level cache (256 MB in all) past the caches, and 4 tokens a workgroup, whose vectors are read 8 heads at a time; below it
  // 32 tokens, written side by side.  us, 32 tokens plain / 4 tokens past the caches: 32768 tokens of 48 heads (805 MB) 202 / 159,
  // 4096 (101 MB) 22.3 / 27.2, 512 6.55 / 6.5.  (805 MB in 159 us are 5.05 TB/s, what a plain copy of 2 GiB reaches on the card, 4.98.)
  const bool past = at * heads * (2 * HS_D * 2) > (int64_t)256 << 20;
  int lg = 0;
  while (lg < (past ? 2 : HS_ROPE_MOST_LOG2) && (2 << lg) <= at) lg++;
  while ((at + (1 << lg) - 1) >> lg > HS_MAX_BLOCKS) lg++;  // from 2^26 tokens on; the caller has checked that 32 a workgroup do
  const int64_t blocks = (at + (1 << lg) - 1) >> lg;
  const int step = 32 >> lg;
  int per = (heads + step - 1) / step;
  const int64_t want = past ? 2048 : 4096;  // workgroups: 8 to 16 per compute unit
  const int64_t groups = blocks >= want ? 1 : (want + blocks - 1) / blocks;
  if (per > 1 && groups > 1) per = per > groups ? (int)((per + groups - 1) / groups) : 1;
  const dim3 grid((unsigned)blocks, (unsigned)((heads + per * step - 1) / (per * step)));
  const bool f16 = dtype == HS_FP16;
#define HS_ROPE(F_, P_)                                                                                     \
  do {                                                                                                      \
    if (past) hipLaunchKernelGGL((rope_kernel<F_, P_, true>), grid, dim3(256), 0, st, a, lg, per);          \
    else hipLaunchKernelGGL((rope_kernel<F_, P_, false>), grid, dim3(256), 0, st, a, lg, per);              \
  } while (0)
  if (a.rope.layout == HS_ROPE_PAIRS) {
    if (f16) HS_ROPE(true, true); else HS_ROPE(false, true);
  } else {
    if (f16) HS_ROPE(true, false); else HS_ROPE(false, false);
  }
#undef HS_ROPE
  return hipGetLastError();
}
