// Choice of the tokens that go into a cache: per (batch, kv head) row the first, the last and of the others those of largest weight, in
// order of position.  One workgroup per row finds them; then their keys and values are gathered.
#include "hs_common.h"
#include "hs_rank.h"

namespace {

// One workgroup per row.  Weights are read three times, the last two from the L2: a histogram of the keys' upper 11 bits finds the bin that the
// last token kept falls into; that bin's tokens are listed in LDS and ranked there exactly (radix selection over key and place, so that ties go
// by place); then every wave writes the tokens kept of its own part of the row, behind those of the parts before it.
constexpr int kBins = 2048, kList = 4096;
template <int NT>
__global__ __launch_bounds__(NT) void keep_select_kernel(int Hkv, int n, const float* __restrict__ weight, int64_t w_sb, int64_t w_sh, const int32_t* __restrict__ lens,
                                                         int keep, int first, int last, int32_t* __restrict__ index) {
  constexpr int NW = NT / 64, U = 8;
  __shared__ int hist[kBins];
  __shared__ uint64_t list[kList];
  __shared__ RankScratch rank;
  __shared__ int taken[NW], chunk[NT / 64], n_list;
  __shared__ Bin found;
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const int b = blockIdx.x / Hkv, h = blockIdx.x % Hkv;
  weight += b * w_sb + h * w_sh;
  index += (int64_t)blockIdx.x * keep;
  const int len = lens != nullptr ? min(max(lens[b], 0), n) : n;
  if (len <= keep) {
    for (int i = tid; i < keep; i += NT) index[i] = i < len ? i : -1;
    return;
  }
  const int lo = first, hi = len - last, want = keep - first - last;  // first + last <= keep < len: 0 <= want < hi - lo
  // the wave's part of the candidates, whole strips of 64
  const int strips = (hi - lo + 63) / 64, s0 = (int)((int64_t)strips * w / NW), s1 = (int)((int64_t)strips * (w + 1) / NW);
  // fn(place, key, valid) of U strips at a time; the largest weights have the lowest keys
  auto part = [&](auto fn) {
    for (int s = s0; s < s1; s += U) {
      float x[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int t = lo + 64 * (s + u) + l;
        x[u] = s + u < s1 && t < hi ? weight[t] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int t = lo + 64 * (s + u) + l;
        fn(t, ~rank_key(x[u]), s + u < s1 && t < hi);
      }
    }
  };
  uint64_t bound = 0;  // of the ranks that are taken
  if (want > 0) {
    for (int i = tid; i < kBins; i += NT) hist[i] = 0;
    if (tid < NW) taken[tid] = 0;
    if (tid == 0) n_list = 0;
    __syncthreads();
    part([&](int, uint32_t key, bool valid) {
      const int bin = (int)(key >> 21);
      // lanes that share the first one's bin are counted at once: rows of equal weights would take 64 turns at one counter
      const unsigned long long there = __ballot(valid);
      if (there == 0ull) return;
      const int leader = __builtin_ctzll(there);
      const int its = __builtin_amdgcn_readlane(bin, leader);
      const unsigned long long alike = __ballot(valid && bin == its);
      if (l == leader) atomicAdd(&hist[its], __builtin_popcountll(alike));
      else if (valid && bin != its) atomicAdd(&hist[bin], 1);
    });
    __syncthreads();
    // the bin: sums of NT equal chunks first, then the chunk's bins by wave 0
    {
      constexpr int PER = kBins / NT;
      int sum = 0;
#pragma unroll
      for (int i = 0; i < PER; i++) sum += hist[PER * tid + i];
      const int upto = wave_upto(sum);
      if (l == 63) chunk[w] = upto;
      __syncthreads();
      int below = upto - sum;
#pragma unroll
      for (int k = 0; k < NW; k++)
        if (k < w) below += chunk[k];
#pragma unroll
      for (int i = 0; i < PER; i++) {
        const int c = hist[PER * tid + i];
        if (below < want && want <= below + c) found = Bin{PER * tid + i, below, c};
        below += c;
      }
    }
    __syncthreads();
    const Bin bin = found;
    const int rest = want - bin.below;  // of the bin's tokens
    // the wave's tokens that are taken for certain, and the list of the bin's
    int sure = 0;
    const bool whole = rest == bin.in, listed = bin.in <= kList;
    part([&](int t, uint32_t key, bool valid) {
      const int its = (int)(key >> 21);
      sure += __builtin_popcountll(__ballot(valid && (whole ? its <= bin.bin : its < bin.bin)));
      if (!whole && listed) {
        const bool mine = valid && its == bin.bin;
        const unsigned long long all = __ballot(mine);
        if (all != 0ull) {
          int at = 0;
          if (l == 0) at = atomicAdd(&n_list, __builtin_popcountll(all));
          at = __builtin_amdgcn_readfirstlane(at) + __builtin_popcountll(all & ((1ull << l) - 1ull));
          if (mine) list[at] = rank_of(key, t);
        }
      }
    });
    if (l == 0) taken[w] = sure;
    __syncthreads();
    if (whole) {
      bound = (uint64_t)(uint32_t)bin.bin << 53 | (~0ull >> 11);
    } else if (listed) {
      bound = smallest_bound<NT>(rest, [&](auto fn) {
        for (int i = tid; i < bin.in; i += NT) fn(list[i]);
      }, &rank);
      for (int i = tid; i < bin.in; i += NT) {
        const uint64_t r = list[i];
        if (r <= bound) {  // whose part it is: the last that begins at or before its strip
          const int strip = ((int)(uint32_t)r - lo) >> 6;
          int p = (int)(((int64_t)strip * NW) / strips);
          while (p + 1 < NW && (int)((int64_t)strips * (p + 1) / NW) <= strip) p++;
          atomicAdd(&taken[p], 1);
        }
      }
    } else {  // most weights alike: ranked where they are
      bound = smallest_bound<NT>(rest, [&](auto fn) {
        part([&](int t, uint32_t key, bool valid) {
          if (valid && (int)(key >> 21) == bin.bin) fn(rank_of(key, t));
        });
      }, &rank);
      int more = 0;
      part([&](int t, uint32_t key, bool valid) {
        more += __builtin_popcountll(__ballot(valid && (int)(key >> 21) == bin.bin && rank_of(key, t) <= bound));
      });
      if (l == 0) taken[w] += more;
    }
    __syncthreads();
  }
  for (int i = tid; i < first; i += NT) index[i] = i;
  for (int i = tid; i < last; i += NT) index[keep - last + i] = hi + i;
  if (want == 0) return;
  int at = first;
#pragma unroll
  for (int k = 0; k < NW; k++)
    if (k < w) at += taken[k];
  part([&](int t, uint32_t key, bool valid) {
    const bool take = valid && rank_of(key, t) <= bound;
    const unsigned long long all = __ballot(take);
    if (take) index[at + __builtin_popcountll(all & ((1ull << l) - 1ull))] = t;
    at += __builtin_popcountll(all);
  });
}

// 16 lanes a vector, 16 output rows a workgroup
__global__ __launch_bounds__(256) void keep_gather_kernel(int Hkv, int keep, hs_vec_view K, hs_vec_view V, const int32_t* __restrict__ index, uint16_t* __restrict__ K_out,
                                                          uint16_t* __restrict__ V_out) {
  const int row = blockIdx.y, b = row / Hkv, h = row % Hkv, c = threadIdx.x & 15;
  const int i = blockIdx.x * 16 + (threadIdx.x >> 4);
  if (i >= keep) return;
  const int64_t at = (int64_t)row * keep + i;
  const int t = index[at];
  uint4 k = make_uint4(0, 0, 0, 0), v = k;
  if (t >= 0) {
    k = *reinterpret_cast<const uint4*>(K.p + b * K.sb + h * K.sh + t * K.st + 8 * c);
    v = *reinterpret_cast<const uint4*>(V.p + b * V.sb + h * V.sh + t * V.st + 8 * c);
  }
  *reinterpret_cast<uint4*>(K_out + at * HS_D + 8 * c) = k;
  *reinterpret_cast<uint4*>(V_out + at * HS_D + 8 * c) = v;
}

}  // namespace

hipError_t hs_launch_keep(int B, int Hkv, int n, hs_vec_view K, hs_vec_view V, const float* weight, int64_t w_sb, int64_t w_sh, const int32_t* lens,
                          int keep, int first, int last, uint16_t* K_out, uint16_t* V_out, int32_t* index, hipStream_t st) {
  const int rows = B * Hkv;
  if (n <= 4096)
    hipLaunchKernelGGL((keep_select_kernel<256>), dim3(rows), dim3(256), 0, st, Hkv, n, weight, w_sb, w_sh, lens, keep, first, last, index);
  else
    hipLaunchKernelGGL((keep_select_kernel<1024>), dim3(rows), dim3(1024), 0, st, Hkv, n, weight, w_sb, w_sh, lens, keep, first, last, index);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(keep_gather_kernel, dim3((keep + 15) / 16, rows), dim3(256), 0, st, Hkv, keep, K, V, index, K_out, V_out);
  return hipGetLastError();
}
