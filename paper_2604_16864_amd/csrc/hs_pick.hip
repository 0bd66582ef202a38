// Choice of the tiles that a query attends to, by their scores.
#include <limits.h>

#include "hs_rank.h"

namespace {

constexpr int kListed = 64;

__device__ __forceinline__ int bits_below(unsigned long long bits, int l) { return __builtin_popcountll(bits & ((1ull << l) - 1ull)); }

// Number of the first bit of each of a wave's words (word j NW + w of `bits`, in LDS, written before a barrier), and of all bits.  Up to 64 words every wave counts
// by itself; more are counted by wave 0 into `sm`, with two barriers.
template <int NW, int PER>
struct Numbers {
  static constexpr int kWords = NW * PER;
  static constexpr bool kShared = kWords > 64;
  int mine[kShared ? 1 : PER], total;
  const int* sm_;
  __device__ __forceinline__ void count(const unsigned long long* bits, int* sm, int w, int l) {
    if constexpr (!kShared) {
      const int c = l < kWords ? __builtin_popcountll(bits[l]) : 0, upto = wave_upto(c), front = upto - c;
#pragma unroll
      for (int j = 0; j < PER; j++) mine[j] = __builtin_amdgcn_readlane(front, j * NW + w);
      total = __builtin_amdgcn_readlane(upto, 63);
    } else {
      sm_ = sm;
      if (w == 0) {
        int sum = 0;
        for (int i0 = 0; i0 < kWords; i0 += 64) {
          const int c = __builtin_popcountll(bits[i0 + l]), upto = wave_upto(c);
          sm[i0 + l] = sum + upto - c;
          sum += __builtin_amdgcn_readlane(upto, 63);
        }
        if (l == 0) sm[kWords] = sum;
      }
      __syncthreads();
      total = sm[kWords];
    }
  }
  __device__ __forceinline__ int before(int j, int w) const {
    if constexpr (kShared) return sm_[j * NW + w]; else return mine[j];
  }
};

// Largest of the lanes' values, in lane 63.
__device__ __forceinline__ float wave_max_63(float x) {
#define HS_STEP(C_, R_) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), C_, R_, 0xf, false)));
  HS_WAVE_STEPS(HS_STEP)
#undef HS_STEP
  return x;
}

// What bounds all of this is latency: a row is a few kilobytes, read once, and a chain of steps that each wait for the one before.
// One workgroup per query.  A thread has PER scores, of tiles j NT + tid, in registers (of long rows it reads them anew for each pass); a wave's 64 are one
// word of the row's bits.  Tiles that are open (score above -inf) are numbered to find the ends.  The others are counted into bins of equal width between the
// largest and the smallest finite score; the bins above the one in which the count is reached are in, and of that one those with the best ranks (score
// falling, tile rising): each compared with all, where they are few, else by radix selection, which also takes scores whose width is not finite.  The chosen
// ones, numbered again, are written in their order.
template <int NT, int PER>
__global__ __launch_bounds__(NT) void pick_kernel(int T, const float* __restrict__ scores, int n_pick, int first, int last, int32_t* __restrict__ list) {
  constexpr int NW = NT / 64, kWords = NW * PER;
  constexpr bool LONG = PER > 16;
  constexpr int kBins = LONG ? 2048 : (NT * PER > 2048 ? 1024 : 256);
  __shared__ RankScratch scratch;
  __shared__ unsigned long long open_bits[kWords], chosen_bits[kWords], few[kListed];
  __shared__ int sm_before[kWords <= 64 ? 1 : kWords + 1], n_few;
  __shared__ __attribute__((aligned(16))) int hist[kBins];
  __shared__ float ends_of[2][NW];
  const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float* row = scores + (int64_t)blockIdx.x * T;
  int32_t* out = list + (int64_t)blockIdx.x * n_pick;
  auto load = [&](int j) -> float {
    const int t = j * NT + tid;
    const float x = t < T ? row[t] : -INFINITY;
    return x == x ? x : INFINITY;  // a tile that cannot be ruled out
  };
  const int n_each = LONG ? (T + 8 * NT - 1) / (8 * NT) * 8 : PER;
  float s[LONG ? 8 : PER];
  if constexpr (!LONG) {
#pragma unroll
    for (int j = 0; j < PER; j++) s[j] = load(j);
  }
  auto each = [&](auto fn) {  // fn(j, score)
    if constexpr (LONG) {
      for (int j0 = 0; j0 < n_each; j0 += 8) {
#pragma unroll
        for (int j = 0; j < 8; j++) s[j] = load(j0 + j);
#pragma unroll
        for (int j = 0; j < 8; j++) fn(j0 + j, s[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < PER; j++) fn(j, s[j]);
    }
  };
  for (int i = tid; i < kBins; i += NT) hist[i] = 0;
  if (tid == 0) n_few = 0;
  if (LONG)
    for (int i = NW * n_each + tid; i < kWords; i += NT) open_bits[i] = chosen_bits[i] = 0ull;
  float high = -INFINITY, low = -INFINITY;  // of the finite scores: the largest, and the largest of the negated
  each([&](int j, float x) {
    const unsigned long long open = __ballot(x > -INFINITY);
    if (x > -INFINITY && x < INFINITY) { high = fmaxf(high, x); low = fmaxf(low, -x); }
    if (l == 0) open_bits[j * NW + w] = open;
  });
  high = wave_max_63(high);
  low = wave_max_63(low);
  if (l == 63) { ends_of[0][w] = high; ends_of[1][w] = low; }
  __syncthreads();
  Numbers<NW, PER> number;
  number.count(open_bits, sm_before, w, l);
  const int n_open = number.total;
  const unsigned long long* picked = open_bits;
  if (n_open > n_pick) {
    const int n_first = min(first, n_open), n_last = min(last, n_open - n_first), rest = n_pick - n_first - n_last;
    unsigned long long is_open = 0ull, ranked = 0ull;  // bit j: open; and decided about by its score
    each([&](int j, float) {
      const unsigned long long open = open_bits[j * NW + w];
      const int at = number.before(j, w) + bits_below(open, l);
      if (open >> l & 1ull) {
        is_open |= 1ull << j;
        if (at >= n_first && at < n_open - n_last) ranked |= 1ull << j;
      }
    });
    high = ends_of[0][0];
    low = ends_of[1][0];
#pragma unroll
    for (int k = 1; k < NW; k++) { high = fmaxf(high, ends_of[0][k]); low = fmaxf(low, ends_of[1][k]); }
    const float width = high + low;  // finite; -inf where no score is finite; inf where it is beyond 32 bits
    const bool binned = width < INFINITY && width > -INFINITY && rest > 0;
    const float per = width > 0.f ? (float)(kBins - 1) / width : 0.f;
    // falls with the score, by rounding alike; infinite `per` (of a width below the normal numbers) leaves the first and the last bin
    auto bin_of = [&](float x) -> int {
      const float at = x < high ? (high - x) * per : 0.f;
      return at < (float)(kBins - 1) ? (int)at : kBins - 1;
    };
    auto rank = [&](int j, float x) { return rank_of(~rank_key(x), j * NT + tid); };
    // not binned: all that are ranked are in question, more of them than are left to take, and compared by radix selection whatever their number
    int bound_bin = 0, left = rest, in_bin = INT_MAX;
    if (binned) {
      each([&](int j, float x) { if (ranked >> j & 1ull) atomicAdd(&hist[bin_of(x)], 1); });
      __syncthreads();
      // each wave finds the bin by itself
      int c[kBins / 64], sum = 0;
#pragma unroll
      for (int i = 0; i < kBins / 64; i += 4) {
        const int4 v = *reinterpret_cast<const int4*>(&hist[kBins / 64 * l + i]);
        c[i] = v.x; c[i + 1] = v.y; c[i + 2] = v.z; c[i + 3] = v.w;
        sum += v.x + v.y + v.z + v.w;
      }
      const int upto = wave_upto(sum);
      int below = upto - sum, bin = 0, in = 0, need = 0;
      const int where = __builtin_ctzll(__ballot(upto >= rest));
#pragma unroll
      for (int i = 0; i < kBins / 64; i++) {
        if (below < rest && below + c[i] >= rest) { bin = kBins / 64 * l + i; in = c[i]; need = rest - below; }
        below += c[i];
      }
      bound_bin = __builtin_amdgcn_readlane(bin, where);
      in_bin = __builtin_amdgcn_readlane(in, where);
      left = __builtin_amdgcn_readlane(need, where);
    }
    auto in_question = [&](int j, float x) { return (ranked >> j & 1ull) && (!binned || bin_of(x) == bound_bin); };
    uint64_t bound = 0ull;  // of those in question, ranks up to it are in; not looked at where none is
    if (rest > 0 && left == in_bin) {
      bound = ~0ull;
    } else if (rest > 0 && in_bin <= kListed) {
      each([&](int j, float x) { if (in_question(j, x)) few[atomicAdd(&n_few, 1)] = rank(j, x); });
      __syncthreads();
      // each wave finds it by itself: the one with left - 1 better ones
      const uint64_t mine = l < in_bin ? few[l] : ~0ull;
      int better = 0;
      for (int i0 = 0; i0 < in_bin; i0 += 8) {
        uint64_t other[8];
#pragma unroll
        for (int i = 0; i < 8; i++) other[i] = few[min(i0 + i, in_bin - 1)];
#pragma unroll
        for (int i = 0; i < 8; i++) better += i0 + i < in_bin && other[i] < mine ? 1 : 0;
      }
      const int where = __builtin_ctzll(__ballot(l < in_bin && better == left - 1));
      bound = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), where) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)mine, where);
    } else if (rest > 0) {
      bound = smallest_bound<NT>(left, [&](auto fn) { each([&](int j, float x) { if (in_question(j, x)) fn(rank(j, x)); }); }, &scratch);
    }
    each([&](int j, float x) {
      bool in = is_open >> j & 1ull;
      if (ranked >> j & 1ull) {
        const int bin = binned ? bin_of(x) : bound_bin;
        in = rest > 0 && (bin < bound_bin || (bin == bound_bin && rank(j, x) <= bound));
      }
      const unsigned long long word = __ballot(in);
      if (l == 0) chosen_bits[j * NW + w] = word;
    });
    __syncthreads();
    number.count(chosen_bits, sm_before, w, l);
    picked = chosen_bits;
  }
#pragma unroll LONG ? 1 : PER
  for (int j = 0; j < n_each; j++) {
    const unsigned long long word = picked[j * NW + w];
    if (word >> l & 1ull) out[number.before(j, w) + bits_below(word, l)] = j * NT + tid;
  }
  for (int i = number.total + tid; i < n_pick; i += NT) out[i] = -1;
}

// Rows of few tiles: a wave per row, 64 PER tiles, nothing shared.  The bound is found bit by bit from the highest one that two ranked scores differ in: how
// many have a 0 there, by ballots; until a half is taken whole.
template <int PER>
__global__ __launch_bounds__(256) void pick_wave_kernel(int64_t rows, int T, const float* __restrict__ scores, int n_pick, int first, int last, int32_t* __restrict__ list) {
  const int l = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (r >= rows) return;
  const float* row = scores + r * T;
  int32_t* out = list + r * n_pick;
  uint32_t key[PER];  // rises where the score falls
  unsigned long long in[PER];
  int n_open = 0;
#pragma unroll
  for (int j = 0; j < PER; j++) {
    const int t = 64 * j + l;
    const float x = t < T ? row[t] : -INFINITY;
    key[j] = ~rank_key(x == x ? x : INFINITY);  // NaN: a tile that cannot be ruled out
    in[j] = __ballot(!(x == -INFINITY));
    n_open += __builtin_popcountll(in[j]);
  }
  if (n_open > n_pick) {
    const int n_first = min(first, n_open), n_last = min(last, n_open - n_first);
    int rest = n_pick - n_first - n_last;
    unsigned long long ranked[PER];
    uint32_t any = 0u, all = ~0u;
    int before = 0;
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const int at = before + bits_below(in[j], l);
      const bool mine = (in[j] >> l & 1ull) && at >= n_first && at < n_open - n_last;
      ranked[j] = __ballot(mine);
      before += __builtin_popcountll(in[j]);
      any |= mine ? key[j] : 0u;
      all &= mine ? key[j] : ~0u;
    }
    const uint64_t both = wave_or((uint64_t)any << 32 | (uint32_t)~all);
    any = (uint32_t)(both >> 32);
    all = ~(uint32_t)both;
    // keys from low on, span + 1 of them: those that the bound is among; rest: how many of them are taken.  All before low are.
    const uint32_t differ = any ^ all;
    const int bits = differ != 0u ? 32 - __builtin_clz(differ) : 0;
    uint32_t span = bits == 32 ? ~0u : (1u << bits) - 1u, low = all & ~span;
    bool whole = rest == 0;  // of those: all, or (rest == 0) none
    for (int b = bits - 1; b >= 0 && !whole; b--) {
      span >>= 1;
      int n = 0;
#pragma unroll
      for (int j = 0; j < PER; j++) n += __builtin_popcountll(__ballot(key[j] - low <= span) & ranked[j]);
      if (n < rest) {
        rest -= n;
        low += span + 1u;
      } else {
        whole = n == rest;
      }
    }
    int same = 0;
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const unsigned long long level = __ballot(key[j] >= low && key[j] - low <= span) & ranked[j], better = __ballot(key[j] < low) & ranked[j];
      const unsigned long long taken = __ballot((level >> l & 1ull) && same + bits_below(level, l) < rest);
      same += __builtin_popcountll(level);
      in[j] = (in[j] & ~ranked[j]) | (n_pick - n_first - n_last > 0 ? better | taken : 0ull);
    }
  }
  int number = 0;
#pragma unroll
  for (int j = 0; j < PER; j++) {
    if (in[j] >> l & 1ull) out[number + bits_below(in[j], l)] = 64 * j + l;
    number += __builtin_popcountll(in[j]);
  }
  for (int i = number + l; i < n_pick; i += 64) out[i] = -1;
}

}  // namespace

// Threads of a row: many hide the latency of the steps where rows are few, few leave more rows side by side.  us a call, replayed from a graph, 32 tiles of
// T picked, 256 / 512 / 1024 threads:
//   8 rows     T = 512   3.9 / 3.6 / 4.1    1000   4.9 / 4.1 / 4.3    2048   6.9 / 5.2 / 5.1    4096     - / 7.3 / 6.4
//   1024 rows  T = 512   5.1 / 5.9 / 12.3   1000   6.7 / 7.4 / 13.8   2048   9.4 / 10.0 / 16.8  4096     - / 16.6 / 23.3
// a workgroup / a wave for each:
//   8 rows     T = 64    3.3 / 2.9          128    3.3 / 3.6          200    3.4 / 4.2
//   2048 rows  T = 64    5.3 / 4.1          128    5.5 / 4.7          200    5.8 / 6.4
//   8192 rows  T = 64    12.6 / 6.7         128    13.6 / 8.5         200    14.5 / 11.2          512  19.5 / 20.9
hipError_t hs_launch_pick(int64_t rows, int T, const float* scores, int n_pick, int first, int last, int32_t* list, hipStream_t st) {
#define HS_PICK(NT_, PER_) hipLaunchKernelGGL((pick_kernel<NT_, PER_>), dim3((unsigned)rows), dim3(NT_), 0, st, T, scores, n_pick, first, last, list)
#define HS_PICK_WAVE(PER_) \
  hipLaunchKernelGGL((pick_wave_kernel<PER_>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, rows, T, scores, n_pick, first, last, list)
  const bool few = rows <= 512;
  if (T <= 64) HS_PICK_WAVE(1);
  else if (T <= 128 && rows > 1024) HS_PICK_WAVE(2);
  else if (T <= 256 && rows > 4096) HS_PICK_WAVE(4);
  else if (T <= 256) HS_PICK(256, 1);
  else if (T <= 512) { if (few) HS_PICK(512, 1); else HS_PICK(256, 2); }
  else if (T <= 1024) { if (few) HS_PICK(512, 2); else HS_PICK(256, 4); }
  else if (T <= 2048) HS_PICK(512, 4);
  else if (T <= 4096) { if (few) HS_PICK(1024, 4); else HS_PICK(512, 8); }
  else if (T <= 8192) HS_PICK(1024, 8);
  else if (T <= 16384) HS_PICK(1024, 16);
  else HS_PICK(1024, 64);
#undef HS_PICK
#undef HS_PICK_WAVE
  return hipGetLastError();
}
