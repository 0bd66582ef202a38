// Choice of the tiles that a query attends to, by their scores.
#include "hs_rank.h"

namespace {

__device__ __forceinline__ int bits_below(unsigned long long bits, int l) { return __builtin_popcountll(bits & ((1ull << l) - 1ull)); }

// Exclusive counts of the bits in front of each word, and of all in `total`: by wave 0; the caller's barriers around it.
__device__ __forceinline__ void count_words(const unsigned long long* bits, int n_words, int* before, int* total) {
  const int l = threadIdx.x & 63;
  int sum = 0;
  for (int i0 = 0; i0 < n_words; i0 += 64) {
    const int c = i0 + l < n_words ? __builtin_popcountll(bits[i0 + l]) : 0;
    const int upto = wave_upto(c);
    if (i0 + l < n_words) before[i0 + l] = sum + upto - c;
    sum += __builtin_amdgcn_readlane(upto, 63);
  }
  if (l == 0) *total = sum;
}

// One workgroup per query.  A thread holds PER scores, of tiles j NT + tid, in registers; a wave's 64 are one word of the row's bits.  Tiles that are
// open (score above -inf) are numbered to find the ends, the rest are ranked by (score falling, tile rising), and the chosen ones, numbered again, are
// written in their order.
template <int NT, int PER>
__global__ __launch_bounds__(NT) void pick_kernel(int T, const float* __restrict__ scores, int n_pick, int first, int last, int32_t* __restrict__ list) {
  constexpr int NW = NT / 64, kWords = NW * PER;
  __shared__ RankScratch scratch;
  __shared__ unsigned long long bits[kWords];
  __shared__ int before[kWords], total;
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const float* row = scores + (int64_t)blockIdx.x * T;
  int32_t* out = list + (int64_t)blockIdx.x * n_pick;
  uint32_t key[PER];  // rising where the score falls; ~0: not open
#pragma unroll
  for (int j = 0; j < PER; j++) {
    const int t = j * NT + tid;
    const float s = t < T ? row[t] : -INFINITY;
    key[j] = s > -INFINITY ? ~rank_key(s) : (s != s ? ~rank_key(INFINITY) : ~0u);
  }
#pragma unroll
  for (int j = 0; j < PER; j++) {
    const unsigned long long open = __ballot(key[j] != ~0u);
    if (l == 0) bits[j * NW + w] = open;
  }
  __syncthreads();
  if (tid < 64) count_words(bits, kWords, before, &total);
  __syncthreads();
  const int n_open = total;
  if (n_open > n_pick) {
    const int n_first = min(first, n_open), n_last = min(last, n_open - n_first), rest = n_pick - n_first - n_last;
    unsigned long long ends = 0ull;  // bit j: an end
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const int number = before[j * NW + w] + bits_below(bits[j * NW + w], l);
      if (key[j] != ~0u && (number < n_first || number >= n_open - n_last)) ends |= 1ull << j;
    }
    uint64_t bound = 0;
    if (rest > 0)
      bound = smallest_bound<NT>(rest, [&](auto fn) {
#pragma unroll
        for (int j = 0; j < PER; j++)
          if (key[j] != ~0u && !(ends >> j & 1ull)) fn(rank_of(key[j], j * NT + tid));
      }, &scratch);
    __syncthreads();  // the numbers are read
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const bool chosen = key[j] != ~0u && ((ends >> j & 1ull) || (rest > 0 && rank_of(key[j], j * NT + tid) <= bound));
      const unsigned long long word = __ballot(chosen);
      if (l == 0) bits[j * NW + w] = word;
    }
    __syncthreads();
    if (tid < 64) count_words(bits, kWords, before, &total);
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < PER; j++) {
    const unsigned long long word = bits[j * NW + w];
    if (word >> l & 1ull) out[before[j * NW + w] + bits_below(word, l)] = j * NT + tid;
  }
  for (int i = total + tid; i < n_pick; i += NT) out[i] = -1;
}

}  // namespace

hipError_t hs_launch_pick(int64_t rows, int T, const float* scores, int n_pick, int first, int last, int32_t* list, hipStream_t st) {
#define HS_PICK(NT_, PER_) hipLaunchKernelGGL((pick_kernel<NT_, PER_>), dim3((unsigned)rows), dim3(NT_), 0, st, T, scores, n_pick, first, last, list)
  if (T <= 256) HS_PICK(256, 1);
  else if (T <= 512) HS_PICK(256, 2);
  else if (T <= 1024) HS_PICK(256, 4);
  else if (T <= 2048) HS_PICK(256, 8);
  else if (T <= 8192) HS_PICK(1024, 8);
  else HS_PICK(1024, 64);
#undef HS_PICK
  return hipGetLastError();
}
