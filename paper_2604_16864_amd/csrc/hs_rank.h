// Ranking of 32-bit floating-point values by one workgroup: shared by the eviction of tiles and the choice of tokens.
#pragma once
#include "hs_common.h"

namespace {

// Order-preserving bit pattern: a < b as numbers <=> key(a) < key(b); zeros are equal, NaN is below everything.
__device__ __forceinline__ uint32_t rank_key(float x) {
  if (x != x) return 0u;
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return b ^ (b & 0x80000000u ? 0xffffffffu : 0x80000000u);
}

// Prefix counts over a workgroup of NT threads: each thread's flag is numbered in thread order from `carried` on, which moves on
// by the count of all.  sm: NT / 64 ints.  Every thread takes part.
template <int NT>
__device__ __forceinline__ int number_of(bool flag, int& carried, int* sm) {
  constexpr int NW = NT / 64;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const unsigned long long vote = __ballot(flag);
  if (l == 0) sm[w] = __builtin_popcountll(vote);
  __syncthreads();
  int before = carried, all = 0;
#pragma unroll
  for (int i = 0; i < NW; i++) {
    if (i < w) before += sm[i];
    all += sm[i];
  }
  carried += all;
  __syncthreads();
  return before + __builtin_popcountll(vote & ((1ull << l) - 1ull));
}

// The `count` smallest (1 <= count <= how many there are) of the keys that `get` gives for places lo <= t < hi (false: no candidate): those below
// `key`, and of those equal to it the first `ties` by place.  Radix selection, a byte at a time.
// hist: 260 ints of LDS.  Every thread takes part.
struct Threshold { uint32_t key; int ties; };
template <int NT, typename Get>
__device__ __forceinline__ Threshold smallest(int lo, int hi, int count, Get get, int* hist) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0, mask = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += NT) hist[i] = 0;
    __syncthreads();
    for (int t = lo + tid; t < hi; t += NT) {
      uint32_t key;
      if (get(t, key) && (key & mask) == prefix) atomicAdd(&hist[(key >> shift) & 255u], 1);
    }
    __syncthreads();
    if (tid < 64) {  // lane l: bins 4 l .. 4 l + 3
      int bin[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; i++) { bin[i] = hist[4 * tid + i]; sum += bin[i]; }
      int upto = sum;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(upto, d);
        if (tid >= d) upto += x;
      }
      int below = upto - sum;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        if (below < count && count <= below + bin[i]) { hist[256] = 4 * tid + i; hist[257] = count - below; }
        below += bin[i];
      }
    }
    __syncthreads();
    prefix |= (uint32_t)hist[256] << shift;
    mask |= 255u << shift;
    count = hist[257];
    __syncthreads();
  }
  return Threshold{prefix, count};
}

}  // namespace
