// Choice of the tokens that go into a cache: per (batch, kv head) row the first, the last and of the others those of largest weight, in
// order of position.  Their indices are found by one workgroup per row (short rows) or by three launches of one per part of a row; then their
// keys and values are gathered.
#include "hs_common.h"
#include "hs_rank.h"

namespace {

constexpr int kBins = 2048;

// Counts a wave's keys by their upper bits; 64 alike at once: rows of equal weights would take 64 turns at one counter for every 64 tokens.
__device__ __forceinline__ void count_bins(int* hist, uint32_t key, bool valid) {
  const int bin = (int)(key >> 21);
  const int one = __builtin_amdgcn_readfirstlane(bin);
  if (__ballot(valid && bin == one) == ~0ull) {
    if ((threadIdx.x & 63) == 0) atomicAdd(&hist[one], 64);
  } else if (valid) {
    atomicAdd(&hist[bin], 1);
  }
}

// One workgroup per row.  Weights are read three times, the last two from the L2: a histogram of the keys' upper 11 bits finds the bin that the
// last token kept falls into; that bin's tokens are listed in LDS and ranked there exactly (radix selection over key and place, so that ties go
// by place); then every wave writes the tokens kept of its own part of the row, behind those of the parts before it.
constexpr int kList = HS_KEEP_SHORT;
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
    part([&](int, uint32_t key, bool valid) { count_bins(hist, key, valid); });
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
    const bool whole = rest == bin.in;
    part([&](int t, uint32_t key, bool valid) {
      const int its = (int)(key >> 21);
      sure += __builtin_popcountll(__ballot(valid && (whole ? its <= bin.bin : its < bin.bin)));
      if (!whole) {
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
    } else {
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

// ---- long rows ----
// A workgroup takes a part of a row's candidates, and what one has found the others read in the next launch: (1) a histogram per part of the
// keys' upper 11 bits; (2) every part adds the row's up, finds the bin that the last token kept falls into, and lists its own
// tokens of that bin; (3) every part ranks the row's list (the same in each), and writes the indices of its own tokens kept behind those
// of the parts before it.  At most 64 parts: what they have found is a lane each.  One workgroup a row spends 27 us per 32K tokens on its
// arithmetic alone.
// Latency-bound, three launches: 8 rows of 32K tokens 3.6 + 4.8 + 6.5 us, 32 rows of up to 128K 6.4 + 7.3 + 12.0, for weights whose logarithm has a spread
// of 2: their bin, a quarter of a power of two, holds about a thousand of 128K.  The narrower the weights, the more it holds, and lists beyond
// kLdsList are read from the L2 in every pass, bins beyond kLongList (unless their keys are all alike) leave every part to rank the whole row by loads that
// wait for each other.  us of the whole call, 32 rows of 128K tokens, 8192 / 32768 kept: spread 2 69 / 239, 1 74 / 254, 0.5 95 /
// 1045, 0.1 942 / 1151, uniform in 0 .. 1 883 / 1055, one bin 1020 / 1098, all alike 71 / 211; 8 rows of 32K, 4096 kept: 20.9, 22.3, 28.7, 34.8, 30.6, 128, 19.8.
constexpr int kParts = 64, kLongList = 8192, kLdsList = 2048;
constexpr int kCoarse = 64, kFine = kBins / kCoarse;  // a histogram's bins, also in sums of 32
struct KeepRow {            // per row, in the workspace
  int32_t bin, rest, in, unused;  // the bin, its tokens that are kept, its tokens
  int32_t sure[kParts], listed[kParts];  // of a part: tokens kept for certain, tokens of the bin
  uint32_t any[kParts], all[kParts];     // bits that any / all of a part's keys of the bin have
};
struct KeepWs {
  uint64_t* list;           // [rows][kLongList]
  KeepRow* head;            // [rows]
  uint16_t* coarse;         // [rows][parts][kCoarse]
  uint16_t* fine;           // [rows][parts][kBins]
};
// About 1024 workgroups where there are many rows (more of them rank more lists), parts of 1024 tokens at least.
static int keep_parts(int64_t rows, int n) {
  int64_t most = 1024 / rows;
  most = most < 16 ? 16 : (most > kParts ? kParts : most);
  const int by_size = (n + 1023) / 1024;
  return n > (1 << 18) ? kParts : (by_size < most ? by_size : (int)most);
}
static KeepWs keep_ws(void* ws, int64_t rows, int parts) {
  KeepWs k;
  k.list = reinterpret_cast<uint64_t*>(ws);
  k.head = reinterpret_cast<KeepRow*>(k.list + rows * kLongList);
  k.coarse = reinterpret_cast<uint16_t*>(k.head + rows);
  k.fine = k.coarse + rows * parts * kCoarse;
  return k;
}
struct KeepArgs {
  const float* weight;
  int64_t w_sb, w_sh;
  const int32_t* lens;
  int32_t* index;
  int Hkv, n, keep, first, last, size;  // size: tokens of a part
};
struct Part {
  const float* weight;
  int len, lo, hi, want, p0, p1, size;  // the part's tokens are p0 .. p1 - 1
  bool all_kept;
};
__device__ __forceinline__ Part part_of(const KeepArgs& A) {
  const int row = blockIdx.y, b = row / A.Hkv, h = row % A.Hkv;
  Part p;
  p.weight = A.weight + b * A.w_sb + h * A.w_sh;
  p.len = A.lens != nullptr ? min(max(A.lens[b], 0), A.n) : A.n;
  p.all_kept = p.len <= A.keep;
  p.lo = A.first; p.hi = p.len - A.last; p.want = A.keep - A.first - A.last;
  p.size = A.size;
  p.p0 = (int)min((int64_t)p.hi, p.lo + (int64_t)p.size * blockIdx.x);
  p.p1 = (int)min((int64_t)p.hi, (int64_t)p.p0 + p.size);
  return p;
}
// A part's keys, a wave a contiguous share: read once into registers (PER > 0, size <= 256 PER) or 8 strips at a time in every pass (PER == 0).
// 256 threads.
template <int PER>
struct PartKeys {
  const Part& p;
  int q0, q1;  // the lane's first token, the end of its wave's
  uint32_t key[PER > 0 ? PER : 1];
  __device__ __forceinline__ explicit PartKeys(const Part& part) : p(part) {
    const int share = p.size / 4;
    const int start = p.p0 + share * (int)(threadIdx.x >> 6);
    q0 = start + (int)(threadIdx.x & 63); q1 = min(p.p1, start + share);
    if constexpr (PER > 0) {
      float x[PER];
#pragma unroll
      for (int u = 0; u < PER; u++) x[u] = q0 + 64 * u < q1 ? p.weight[q0 + 64 * u] : 0.f;
#pragma unroll
      for (int u = 0; u < PER; u++) key[u] = ~rank_key(x[u]);
    }
  }
  // fn(place, key, valid); every lane takes part
  template <typename Fn>
  __device__ __forceinline__ void each(Fn fn) const {
    if constexpr (PER > 0) {
#pragma unroll
      for (int u = 0; u < PER; u++) fn(q0 + 64 * u, key[u], q0 + 64 * u < q1);
    } else {
      constexpr int U = 8;
      for (int t0 = q0; t0 - (int)(threadIdx.x & 63) < q1; t0 += 64 * U) {
        float x[U];
#pragma unroll
        for (int u = 0; u < U; u++) x[u] = t0 + 64 * u < q1 ? p.weight[t0 + 64 * u] : 0.f;
#pragma unroll
        for (int u = 0; u < U; u++) fn(t0 + 64 * u, ~rank_key(x[u]), t0 + 64 * u < q1);
      }
    }
  }
};

template <int PER>
__global__ __launch_bounds__(256) void keep_count_kernel(KeepArgs A, KeepWs ws) {
  __shared__ __attribute__((aligned(16))) int hist[kBins];
  const Part p = part_of(A);
  if (p.all_kept || p.want == 0) return;
  const PartKeys<PER> keys(p);
  for (int i = threadIdx.x; i < kBins; i += 256) hist[i] = 0;
  __syncthreads();
  keys.each([&](int, uint32_t key, bool valid) { count_bins(hist, key, valid); });
  __syncthreads();
  const int64_t part = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  uint32_t* fine = reinterpret_cast<uint32_t*>(ws.fine + part * kBins);
  for (int i = threadIdx.x; i < kBins / 2; i += 256) fine[i] = (uint32_t)hist[2 * i] | (uint32_t)hist[2 * i + 1] << 16;
  // sums of 32: a quarter of one a thread
  int sum = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) sum += hist[8 * threadIdx.x + i];
  sum += __builtin_amdgcn_mov_dpp(sum, 0xb1, 0xf, 0xf, true);  // lanes of four
  sum += __builtin_amdgcn_mov_dpp(sum, 0x4e, 0xf, 0xf, true);
  if ((threadIdx.x & 3) == 0) ws.coarse[part * kCoarse + (threadIdx.x >> 2)] = (uint16_t)sum;
}

template <int PER>
__global__ __launch_bounds__(256) void keep_list_kernel(KeepArgs A, KeepWs ws) {
  __shared__ int sums[8][kCoarse], n_list;
  __shared__ uint16_t fine[kParts][kFine];
  __shared__ uint32_t any4[4], all4[4];
  const Part p = part_of(A);
  if (p.all_kept || p.want == 0) return;
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6, mine = blockIdx.x, parts = gridDim.x;
  const int64_t row = blockIdx.y;
  const PartKeys<PER> keys(p);
  // the bin, by sums of 32 first: a lane a bin
  const uint16_t* coarse = ws.coarse + row * parts * kCoarse;
  const int own = coarse[mine * kCoarse + l];
  int sum = 0;
  {
    int v[kParts / 4];  // requested at once
#pragma unroll
    for (int k = 0; k < kParts / 4; k++) v[k] = w + 4 * k < parts ? coarse[(w + 4 * k) * kCoarse + l] : 0;
#pragma unroll
    for (int k = 0; k < kParts / 4; k++) sum += v[k];
  }
  sums[w][l] = sum;
  if (tid == 0) n_list = 0;
  __syncthreads();
  sum = sums[0][l] + sums[1][l] + sums[2][l] + sums[3][l];
  int upto = wave_upto(sum);
  const int group = __builtin_ctzll(__ballot(upto >= p.want));  // want is at most the number of candidates
  const int below_group = __builtin_amdgcn_readlane(upto - sum, group);
  int sure = l < group ? own : 0;
  __syncthreads();
  {
    const uint16_t* f = ws.fine + row * parts * kBins + group * kFine + (tid & 31);
    int s = 0;
    uint16_t v[kParts / 8];
#pragma unroll
    for (int k = 0; k < kParts / 8; k++) v[k] = (tid >> 5) + 8 * k < parts ? f[((tid >> 5) + 8 * k) * kBins] : (uint16_t)0;
#pragma unroll
    for (int k = 0; k < kParts / 8; k++) {
      fine[(tid >> 5) + 8 * k][tid & 31] = v[k];
      s += v[k];
    }
    sums[tid >> 5][tid & 31] = s;
  }
  __syncthreads();
  sum = 0;
  if (l < kFine) {
#pragma unroll
    for (int k = 0; k < 8; k++) sum += sums[k][l];
  }
  upto = below_group + wave_upto(sum);
  const int at_fine = __builtin_ctzll(__ballot(upto >= p.want));
  const Bin bin = {group * kFine + at_fine, __builtin_amdgcn_readlane(upto - sum, at_fine), __builtin_amdgcn_readlane(sum, at_fine)};
  if (l < at_fine) sure += fine[mine][l];
  sure = wave_upto(sure);  // lane 63's: tokens of the part in the bins before it
  const int listed = l < parts ? fine[l][at_fine] : 0;  // of part l
  const int listed_upto = wave_upto(listed);
  const int of_mine = __builtin_amdgcn_readlane(listed, mine);
  uint64_t* list = ws.list + row * kLongList + __builtin_amdgcn_readlane(listed_upto, mine) - of_mine;
  const bool write = bin.in <= kLongList;
  uint32_t any = 0u, all = ~0u;
  int n = 0;  // of the wave's tokens in the bin
  keys.each([&](int, uint32_t key, bool valid) {
    const bool in = valid && (int)(key >> 21) == bin.bin;
    n += __builtin_popcountll(__ballot(in));
    any |= in ? key : 0u;
    all &= in ? key : ~0u;
  });
  if (write && n != 0) {
    int at = 0;
    if (l == 0) at = atomicAdd(&n_list, n);
    at = __builtin_amdgcn_readfirstlane(at);
    keys.each([&](int t, uint32_t key, bool valid) {
      const bool in = valid && (int)(key >> 21) == bin.bin;
      const unsigned long long those = __ballot(in);
      if (in) list[at + __builtin_popcountll(those & ((1ull << l) - 1ull))] = rank_of(key, t);
      at += __builtin_popcountll(those);
    });
  }
  const uint64_t bits = wave_or((uint64_t)any << 32 | ~all);
  if (l == 0) { any4[w] = (uint32_t)(bits >> 32); all4[w] = ~(uint32_t)bits; }
  __syncthreads();
  if (tid == 63) {
    KeepRow* r = ws.head + row;
    if (mine == 0) { r->bin = bin.bin; r->rest = p.want - bin.below; r->in = bin.in; }
    r->sure[mine] = sure;
    r->listed[mine] = of_mine;
    r->any[mine] = any4[0] | any4[1] | any4[2] | any4[3];
    r->all[mine] = all4[0] & all4[1] & all4[2] & all4[3];
  }
}

template <int PER>
__global__ __launch_bounds__(256) void keep_take_kernel(KeepArgs A, KeepWs ws) {
  __shared__ uint64_t lds_list[kLdsList];
  __shared__ RankScratch rank;
  __shared__ int waves[4], more[4];
  const Part p = part_of(A);
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6, mine = blockIdx.x, parts = gridDim.x;
  const int64_t row = blockIdx.y;
  int32_t* index = A.index + row * A.keep;
  if (p.all_kept) {
    for (int i = 256 * mine + tid; i < A.keep; i += 256 * parts) index[i] = i < p.len ? i : -1;
    return;
  }
  for (int i = 256 * mine + tid; i < A.first; i += 256 * parts) index[i] = i;
  for (int i = 256 * mine + tid; i < A.last; i += 256 * parts) index[A.keep - A.last + i] = p.hi + i;
  if (p.want == 0) return;
  const PartKeys<PER> keys(p);
  const KeepRow* r = ws.head + row;
  const int bin = r->bin, rest = r->rest, in = r->in;
  const int sure = l < mine ? r->sure[l] : 0, listed = l < parts ? r->listed[l] : 0;  // of part l
  const uint64_t bits = wave_or(l < parts ? (uint64_t)r->any[l] << 32 | (uint32_t)~r->all[l] : 0ull);
  const uint32_t any = (uint32_t)(bits >> 32), all = ~(uint32_t)bits;
  int at = A.first + __builtin_amdgcn_readlane(wave_upto(sure), 63);
  const int bins_mine = __builtin_amdgcn_readlane(listed, mine), bins_before = __builtin_amdgcn_readlane(wave_upto(listed), mine) - bins_mine;
  // Which tokens of the bin are kept: all; or, their keys alike, the first `rest` by place, of which this part has `mine_of_bin`; or those up
  // to `bound` in the list.
  const bool alike = any == all;
  uint64_t bound = (uint64_t)(uint32_t)bin << 53 | (~0ull >> 11);
  int mine_of_bin = bins_mine;
  if (rest < in && alike) {
    mine_of_bin = min(max(rest - bins_before, 0), bins_mine);
    at += min(rest, bins_before);
  } else if (rest == in) {
    at += bins_before;
  } else {
    int kept_before = 0;
    if (in <= kLongList) {
      const uint64_t* list = ws.list + row * kLongList;
      if (in <= kLdsList) {
        for (int i = tid; i < in; i += 256) lds_list[i] = list[i];
        __syncthreads();
        list = lds_list;
      }
      bound = smallest_bound<256>(rest, [&](auto fn) {
        for (int i = tid; i < in; i += 256) fn(list[i]);
      }, &rank);
      for (int i = tid; i < bins_before; i += 256) kept_before += list[i] <= bound;  // the parts before this one have listed theirs first
    } else {  // more tokens in one bin than fit the list: every part ranks them where they are
      auto of_row = [&](int end, auto fn) {
        for (int t = p.lo + tid; t < end; t += 256) {
          const uint32_t key = ~rank_key(p.weight[t]);
          if ((int)(key >> 21) == bin) fn(rank_of(key, t));
        }
      };
      bound = smallest_bound<256>(rest, [&](auto fn) { of_row(p.hi, fn); }, &rank);
      of_row(p.p0, [&](uint64_t x) { kept_before += x <= bound; });
    }
    kept_before = wave_upto(kept_before);
    if (l == 63) more[w] = kept_before;
    __syncthreads();
    at += more[0] + more[1] + more[2] + more[3];
  }
  // two passes over the part: how many each wave takes, then their indices
  auto takes = [&](int t, uint32_t key, bool valid, int& of_bin) -> bool {
    if (!alike || rest == in) return valid && rank_of(key, t) <= bound;
    const bool in_bin = valid && (int)(key >> 21) == bin;
    const unsigned long long those = __ballot(in_bin);
    const bool take = valid && ((int)(key >> 21) < bin || (in_bin && of_bin + __builtin_popcountll(those & ((1ull << l) - 1ull)) < mine_of_bin));
    of_bin += __builtin_popcountll(those);
    return take;
  };
  const bool counted = alike && rest < in;
  int of_bin = 0;
  if (counted) {  // tokens of the bin in the waves before this one
    int n = 0;
    keys.each([&](int, uint32_t key, bool valid) { n += __builtin_popcountll(__ballot(valid && (int)(key >> 21) == bin)); });
    if (l == 0) more[w] = n;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; k++)
      if (k < w) of_bin += more[k];
  }
  int n = 0, ob = of_bin;
  keys.each([&](int t, uint32_t key, bool valid) { n += __builtin_popcountll(__ballot(takes(t, key, valid, ob))); });
  if (l == 0) waves[w] = n;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; k++)
    if (k < w) at += waves[k];
  ob = of_bin;
  keys.each([&](int t, uint32_t key, bool valid) {
    const bool take = takes(t, key, valid, ob);
    const unsigned long long those = __ballot(take);
    if (take) index[at + __builtin_popcountll(those & ((1ull << l) - 1ull))] = t;
    at += __builtin_popcountll(those);
  });
}

// 16 lanes a vector, 16 output rows a workgroup.  HBM-bound: 32 rows of 8192 tokens (268 MB read and written) 42 us, 6.3 TB/s.
__global__ __launch_bounds__(256) void keep_gather_kernel(int Hkv, int keep, hs_vec_view K, hs_vec_view V, const int32_t* __restrict__ index, uint16_t* __restrict__ K_out,
                                                          uint16_t* __restrict__ V_out) {
  const int row = blockIdx.y, b = row / Hkv, h = row % Hkv, c = threadIdx.x & 15;
  const int i = blockIdx.x * HS_KEEP_GATHERED + (threadIdx.x >> 4);
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

size_t hs_keep_ws_bytes(int64_t rows, int n) {
  if (n <= HS_KEEP_SHORT) return 0;
  return (size_t)rows * (kLongList * sizeof(uint64_t) + sizeof(KeepRow) + (size_t)keep_parts(rows, n) * (kCoarse + kBins) * sizeof(uint16_t));
}

hipError_t hs_launch_keep(int B, int Hkv, int n, hs_vec_view K, hs_vec_view V, const float* weight, int64_t w_sb, int64_t w_sh, const int32_t* lens,
                          int keep, int first, int last, uint16_t* K_out, uint16_t* V_out, int32_t* index, void* ws, hipStream_t st) {
  const int rows = B * Hkv;
  // us, one workgroup a row / parts, keys and values gathered: 8 rows of 3000 tokens 12.9 / 15.0, of 4096 13.4 / 15.1; 64 rows of 4096 16.4 / 18.3
  if (n <= 2048) {
    hipLaunchKernelGGL((keep_select_kernel<256>), dim3(rows), dim3(256), 0, st, Hkv, n, weight, w_sb, w_sh, lens, keep, first, last, index);
  } else if (n <= HS_KEEP_SHORT) {
    hipLaunchKernelGGL((keep_select_kernel<1024>), dim3(rows), dim3(1024), 0, st, Hkv, n, weight, w_sb, w_sh, lens, keep, first, last, index);
  } else {
    const int parts = keep_parts(rows, n), size = ((n + parts - 1) / parts + 255) / 256 * 256;  // at most 2^20 / 64: counts fit 16 bits
    const KeepArgs A{weight, w_sb, w_sh, lens, index, Hkv, n, keep, first, last, size};
    const KeepWs k = keep_ws(ws, rows, parts);
    const dim3 grid(parts, rows);
#define HS_KEEP(PER_)                                                                  \
  do {                                                                                 \
    hipLaunchKernelGGL((keep_count_kernel<PER_>), grid, dim3(256), 0, st, A, k);       \
    hipLaunchKernelGGL((keep_list_kernel<PER_>), grid, dim3(256), 0, st, A, k);        \
    hipLaunchKernelGGL((keep_take_kernel<PER_>), grid, dim3(256), 0, st, A, k);        \
  } while (0)
    if (size <= 256 * 4) HS_KEEP(4);
    else if (size <= 256 * 8) HS_KEEP(8);
    else if (size <= 256 * 16) HS_KEEP(16);
    else if (size <= 256 * 32) HS_KEEP(32);
    else HS_KEEP(0);
#undef HS_KEEP
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(keep_gather_kernel, dim3((keep + HS_KEEP_GATHERED - 1) / HS_KEEP_GATHERED, rows), dim3(256), 0, st, Hkv, keep, K, V, index, K_out, V_out);
  return hipGetLastError();
}
