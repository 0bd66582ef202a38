// Ranking of 32-bit floating-point values by one workgroup: shared by the eviction of tiles and the choice of tokens.
#pragma once
#include "hs_common.h"

namespace {

// Order-preserving bit pattern: a < b as numbers <=> key(a) < key(b); zeros are equal, NaN is below everything.
__device__ __forceinline__ uint32_t rank_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);  // -0 + 0 = 0
  return x != x ? 0u : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
// What candidates are ranked by: the key, then the place.  No two are equal.
__device__ __forceinline__ uint64_t rank_of(uint32_t key, int place) { return (uint64_t)key << 32 | (uint32_t)place; }

// Lane movements inside the vector ALU (a lane shuffle goes through the LDS, some 100 clocks each): what a step brings from the lanes below, 0 where
// there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_below(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
// fn(from_below) for the six steps of an inclusive scan over the wave: lane 63 ends up with all 64
#define HS_WAVE_STEPS(STEP)                                                                                     \
  STEP(0x111, 0xf) STEP(0x112, 0xf) STEP(0x114, 0xf) STEP(0x118, 0xf) STEP(0x142, 0xa) STEP(0x143, 0xc)
// Inclusive sums over the lanes of a wave.
__device__ __forceinline__ int wave_upto(int x) {
#define HS_STEP(C_, R_) x += (int)from_below<C_, R_>((uint32_t)x);
  HS_WAVE_STEPS(HS_STEP)
#undef HS_STEP
  return x;
}
// All lanes' bits or-ed, in every lane.
__device__ __forceinline__ uint64_t wave_or(uint64_t v) {
  uint32_t lo = (uint32_t)v, hi = (uint32_t)(v >> 32);
#define HS_STEP(C_, R_) lo |= from_below<C_, R_>(lo); hi |= from_below<C_, R_>(hi);
  HS_WAVE_STEPS(HS_STEP)
#undef HS_STEP
  return (uint64_t)__builtin_amdgcn_readlane(hi, 63) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, 63);
}

// hist[0 .. 64 PER) counted by wave 0: bin and how many are in the bins in front of it, where the sum first reaches `count`.
struct Bin { int bin, below, in; };
template <int PER>
__device__ __forceinline__ void find_bin(const int* hist, int count, Bin* out) {  // wave 0 only
  const int l = threadIdx.x & 63;
  int c[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; i++) { c[i] = hist[PER * l + i]; sum += c[i]; }
  int below = wave_upto(sum) - sum;
#pragma unroll
  for (int i = 0; i < PER; i++) {
    if (below < count && count <= below + c[i]) *out = Bin{PER * l + i, below, c[i]};
    below += c[i];
  }
}

// An upper bound (inclusive) of the `count` smallest ranks, 1 <= count <= how many there are: each(fn) calls fn(rank) for every candidate of
// this thread.  Radix selection, 8 bits at a time, passing over bits that no two candidates differ in (weights that came out of a 16-bit
// format differ in few), until the bin found is taken whole.  Every thread takes part; three barriers a pass.
struct RankScratch { int hist[256]; Bin bin; unsigned long long any[16], all[16]; };
// The lowest rank of all (~0: no candidate).  One barrier.
template <int NT, typename Each>
__device__ __forceinline__ uint64_t smallest_rank(Each each, RankScratch* s) {
  unsigned long long low = ~0ull;
  each([&](uint64_t rank) { low = rank < low ? rank : low; });
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned long long other = __shfl_xor(low, d);
    low = other < low ? other : low;
  }
  if ((threadIdx.x & 63) == 0) s->any[threadIdx.x >> 6] = low;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT / 64; i++) low = s->any[i] < low ? s->any[i] : low;
  return low;
}
template <int NT, typename Each>
__device__ __forceinline__ uint64_t smallest_bound(int count, Each each, RankScratch* s) {
  constexpr int NW = NT / 64;
  const int tid = threadIdx.x, w = tid >> 6;
  unsigned long long any = 0ull, all = ~0ull;
  each([&](uint64_t rank) { any |= rank; all &= rank; });
  any = wave_or(any);
  all = ~wave_or(~all);
  if ((tid & 63) == 0) { s->any[w] = any; s->all[w] = all; }
  for (int i = tid; i < 256; i += NT) s->hist[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; i++) { any |= s->any[i]; all &= s->all[i]; }
  if (any == all) return any;  // one candidate
  const uint64_t differ = any ^ all;
  uint64_t prefix = all;   // bits found so far, and those that all have
  uint64_t known = ~differ;
  for (;;) {
    const uint64_t rest = ~known;  // its highest bit is the digit's highest
    const int top = 64 - __builtin_clzll(rest), low = top > 8 ? top - 8 : 0;
    const uint32_t digit = (1u << (top - low)) - 1u;
    const uint64_t above = top == 64 ? 0ull : ~0ull << top;
    each([&](uint64_t rank) {
      if (((rank ^ prefix) & above) == 0ull) atomicAdd(&s->hist[(uint32_t)(rank >> low) & digit], 1);
    });
    __syncthreads();
    if (tid < 64) find_bin<4>(s->hist, count, &s->bin);
    __syncthreads();
    const Bin b = s->bin;
    const uint64_t window = (uint64_t)digit << low;
    prefix = (prefix & ~window) | (uint64_t)(uint32_t)b.bin << low;
    known |= window;
    count -= b.below;
    // taken whole, or the last bits that differ: everything below is in
    if (b.in == count || known == ~0ull) return known == ~0ull ? prefix : (prefix & above) | (uint64_t)(uint32_t)b.bin << low | ~(above | window);
    for (int i = tid; i < 256; i += NT) s->hist[i] = 0;
    __syncthreads();
  }
}

}  // namespace
