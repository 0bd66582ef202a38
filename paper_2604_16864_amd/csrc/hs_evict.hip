// Eviction of tiles from a packed cache in place.
//
// Of a row's held tiles the ones of lowest mass are dropped, and each pool's used slots are made 0 .. n - 1 again with as few copies as that
// takes: of the remaining tiles only those whose slot is n or above move, the k-th of them (by slot) into the k-th freed slot below
// n.  Sources lie from n on and destinations below it, so the copies of a row do not depend on each other and run in any order.
#include "hs_common.h"
#include "hs_rank.h"

namespace {

// Moves of a row in the workspace: their number per pool (dense K, 2:4 K, dense V, 2:4 V), then source << 16 | destination, dense ones first,
// K's in the first half of the list and V's in the second.
__device__ __forceinline__ int32_t* row_ws(int32_t* ws, int64_t row, int T) { return ws + row * (4 + 2 * (int64_t)(T + 1)); }

template <int NT>
__device__ __forceinline__ void copy_slot(const uint8_t* pool, int64_t base, int bytes, uint32_t move) {
  const uint4* s = reinterpret_cast<const uint4*>(pool + (base + (move >> 16)) * bytes);
  uint4* d = reinterpret_cast<uint4*>(const_cast<uint8_t*>(pool) + (base + (move & 0xffffu)) * bytes);
  for (int i = threadIdx.x; i < bytes / 16; i += NT) d[i] = s[i];
}
// move i of a row: n0 of dense K, n1 of 2:4 K, n2 of dense V, then of 2:4 V
template <int NT>
__device__ __forceinline__ void copy_tile(const hs_kv_dev& kv, int64_t row, int T, const int32_t* my_ws, int i, int n0, int n1, int n2) {
  const uint32_t move = (uint32_t)my_ws[4 + (i < n0 + n1 ? i : (T + 1) + i - n0 - n1)];
  if (i < n0) {
    copy_slot<NT>(kv.k_dense, row * kv.cap_dense_k, HS_TILE_DENSE_BYTES, move);
  } else if (i < n0 + n1) {
    copy_slot<NT>(kv.k_nnz, row * kv.cap_sparse_k, HS_TILE_NNZ_BYTES, move);
    copy_slot<NT>(kv.k_meta, row * kv.cap_sparse_k, HS_TILE_META_BYTES, move);
  } else if (i < n0 + n1 + n2) {
    copy_slot<NT>(kv.v_dense, row * kv.cap_dense_v, HS_TILE_DENSE_BYTES, move);
  } else {
    copy_slot<NT>(kv.v_nnz, row * kv.cap_sparse_v, HS_TILE_NNZ_BYTES, move);
    copy_slot<NT>(kv.v_meta, row * kv.cap_sparse_v, HS_TILE_META_BYTES, move);
  }
}

// One workgroup per row.  A thread holds PER tiles in registers (PER > 0, T <= NT PER), or walks the row's maps (PER == 0).
// Latency-bound: a chain of a map read, prefix counts, the choice and the slots' bookkeeping, 9 barriers where one tile goes (128 rows of 1024
// tiles: 8.3 us, 1.7 of them the copies), 15 to 20 with a radix selection (32 rows of 1024 tiles down to 256: 9.7, 2.8 of them the selection).
// COPY: the row's moves are made here, too (few, by the host's count); otherwise they are listed for evict_move_kernel.
template <int NT, int PER, bool COPY>
__global__ __launch_bounds__(NT) void evict_kernel(int T, hs_kv_dev kv, const float* __restrict__ mass, int keep, const int32_t* __restrict__ keeps,
                                                   int first, int last, int32_t* __restrict__ ws) {
  extern __shared__ uint32_t lds[];
  constexpr int NW = NT / 64;
  __shared__ RankScratch rank;
  __shared__ int counts[NW], left[4], n_holes[4];
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const int64_t row = blockIdx.x;
  int32_t* const k_map = const_cast<int32_t*>(kv.k_map) + row * T;
  int32_t* const v_map = const_cast<int32_t*>(kv.v_map) + row * T;
  mass += row * T;
  int32_t* my_ws = row_ws(ws, row, T);
  const int words = (T + 31) / 32;
  // dense K, 2:4 K, dense V, 2:4 V
  uint32_t* const marks = lds;                                             // [4][words]
  uint16_t* const before = reinterpret_cast<uint16_t*>(lds + 4 * words);   // [4][words]
  uint32_t* const dropped = lds + 6 * words;                               // [words]
  const int room[4] = {min(T, kv.cap_dense_k), min(T, kv.cap_sparse_k), min(T, kv.cap_dense_v), min(T, kv.cap_sparse_v)};

  // The row's tiles: PER > 0 in registers, tile j NT + tid in place j.
  constexpr int kN = PER > 0 ? PER : 1;
  int mk[kN], mv[kN];
  uint32_t key[kN];
  auto tiles = [&](auto fn) {  // fn(tile, k entry, v entry, key) in ascending order of the tile
    if constexpr (PER > 0) {
#pragma unroll
      for (int j = 0; j < PER; j++) fn(j * NT + tid, mk[j], mv[j], key[j]);
    } else {
      for (int t = tid; t < (T + NT - 1) / NT * NT; t += NT) {
        const int a = t < T ? k_map[t] : 0;
        fn(t, a, a != 0 ? v_map[t] : 0, a != 0 ? rank_key(mass[t]) : 0u);
      }
    }
  };
  if constexpr (PER > 0) {
    float m[PER];
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const int t = j * NT + tid;
      mk[j] = t < T ? k_map[t] : 0;
      mv[j] = t < T ? v_map[t] : 0;
      m[j] = t < T ? mass[t] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < PER; j++) key[j] = rank_key(m[j]);
  }
  if (keeps != nullptr) keep = max(1, keeps[row]);
  for (int i = tid; i < 4 * words; i += NT) marks[i] = 0;
  for (int i = tid; i < words; i += NT) dropped[i] = 0;
  if (tid < 4) { left[tid] = 0; n_holes[tid] = 0; }

  // Tiles held, and where the candidates begin and end: behind the first `first` and in front of the last `last` of them.  The held tiles
  // as bits, whose counts number them.
  tiles([&](int t, int a, int, uint32_t) {
    const unsigned long long held = __ballot(a != 0);
    if (l < 2 && 2 * (t >> 6) + l < words) before[2 * (t >> 6) + l] = (uint16_t)__builtin_popcount((uint32_t)(held >> (32 * l)));  // for now: in the word itself
  });
  __syncthreads();
  // words in chunks of NT: counts in front of each
  int n = 0;
  for (int i0 = 0; i0 < words; i0 += NT) {
    const int i = i0 + tid, mine = i < words ? before[i] : 0;
    const int upto = wave_upto(mine);
    if (l == 63) counts[w] = upto;
    __syncthreads();
    int off = n;
#pragma unroll
    for (int k = 0; k < NW; k++) {
      if (k < w) off += counts[k];
      n += counts[k];
    }
    if (i < words) before[i] = (uint16_t)(off + upto - mine);  // at most 65535: fewer than T
    __syncthreads();
  }
  const int n_drop = min(n - keep, n - min(n, first) - min(n, last));  // may be negative
  if (n_drop <= 0) {  // the whole workgroup
    if (!COPY && tid < 4) my_ws[tid] = 0;
    return;
  }
  // a candidate's number among the held tiles: from `first` on, below n - last
  auto is_candidate = [&](int t, int a) -> bool {
    const unsigned long long held = __ballot(a != 0);  // of the wave's 64 tiles, which start at a multiple of 64
    if (a == 0) return false;
    const int word = 2 * (t >> 6);
    const int number = before[word] + __builtin_popcountll(held & ((1ull << l) - 1ull));
    return number >= first && number < n - last;
  };
  uint32_t cands = 0;  // PER > 0: a bit per place
  if constexpr (PER > 0) {
#pragma unroll
    for (int j = 0; j < PER; j++) cands |= is_candidate(j * NT + tid, mk[j]) ? 1u << j : 0u;
  }
  auto candidates = [&](auto fn) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int j = 0; j < PER; j++)
        if ((cands >> j) & 1u) fn(rank_of(key[j], j * NT + tid));
    } else {
      tiles([&](int t, int a, int, uint32_t ky) {
        if (is_candidate(t, a)) fn(rank_of(ky, t));
      });
    }
  };
  // one tile over, the usual case of a cache that grows by one: no selection
  const uint64_t bound = n_drop == 1 ? smallest_rank<NT>(candidates, &rank) : smallest_bound<NT>(n_drop, candidates, &rank);

  // what stays of each pool
  {
    int stay[4] = {0, 0, 0, 0}, j = 0;
    tiles([&](int t, int a, int b, uint32_t ky) {
      const bool cand = PER > 0 ? (cands >> j++) & 1u : is_candidate(t, a);
      const bool drop = cand && rank_of(ky, t) <= bound;
      const unsigned long long gone = __ballot(drop);
      if (l < 2 && 2 * (t >> 6) + l < words) dropped[2 * (t >> 6) + l] = (uint32_t)(gone >> (32 * l));
      stay[0] += __builtin_popcountll(__ballot(a > 0 && !drop));
      stay[1] += __builtin_popcountll(__ballot(a < 0 && !drop));
      stay[2] += __builtin_popcountll(__ballot(b > 0 && !drop));
      stay[3] += __builtin_popcountll(__ballot(b < 0 && !drop));
    });
    if (l < 4) atomicAdd(&left[l], l == 0 ? stay[0] : l == 1 ? stay[1] : l == 2 ? stay[2] : stay[3]);
  }
  __syncthreads();
  auto is_dropped = [&](int t) -> bool { return (dropped[t >> 5] >> (t & 31)) & 1u; };
  auto mark = [&](int m, int pool, bool drop) {
    const int slot = (abs(m) & ~HS_MAP_F16) - 1;
    if (slot < room[pool] && drop == (slot < left[pool])) atomicOr(&marks[pool * words + (slot >> 5)], 1u << (slot & 31));
  };
  tiles([&](int t, int a, int b, uint32_t) {
    if (a == 0) return;
    const bool drop = is_dropped(t);
    mark(a, a > 0 ? 0 : 1, drop);
    mark(b, b > 0 ? 2 : 3, drop);
  });
  __syncthreads();
  // marks in front of each word: a wave a pool
  if (w < 4) {
    int carried = 0;
    for (int i0 = 0; i0 < words; i0 += 64) {
      const int i = i0 + l;
      const uint32_t m = i < words ? marks[w * words + i] : 0u;
      const int upto = wave_upto(__builtin_popcount(m));
      if (i < words) {
        before[w * words + i] = (uint16_t)(carried + upto - __builtin_popcount(m));
        const int in_front = left[w] - 32 * i;  // slots of the word that the remaining tiles take
        const uint32_t h = in_front >= 32 ? m : (in_front <= 0 ? 0u : m & ((1u << in_front) - 1u));
        if (h != 0) atomicAdd(&n_holes[w], __builtin_popcount(h));
      }
      carried += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  __syncthreads();
  // the freed slots in order, in the list where the moves are going to be: dense, then 2:4
  auto list_of = [&](int pool) -> int32_t* { return my_ws + 4 + (pool >> 1) * (T + 1) + ((pool & 1) ? n_holes[pool - 1] : 0); };
  for (int pool = 0; pool < 4; pool++)
    for (int slot = tid; slot < left[pool]; slot += NT) {
      const int word = pool * words + (slot >> 5);
      const uint32_t m = marks[word], bit = 1u << (slot & 31);
      if (m & bit) list_of(pool)[before[word] + __builtin_popcount(m & (bit - 1u))] = slot;
    }
  __syncthreads();
  auto moved = [&](int m, int pool) -> int {  // the entry of a tile that stays
    const int slot = (abs(m) & ~HS_MAP_F16) - 1;
    if (slot >= room[pool] || slot < left[pool]) return m;
    const int word = pool * words + (slot >> 5);
    const int k = before[word] + __builtin_popcount(marks[word] & ((1u << (slot & 31)) - 1u)) - n_holes[pool];
    if (k < 0 || k >= n_holes[pool]) return m;  // slots that are not 0 .. n - 1: the tile stays
    int32_t* at = list_of(pool) + k;
    const int to = *at;
    *at = (int32_t)((uint32_t)slot << 16 | (uint32_t)to);
    const int entry = (to + 1) | (abs(m) & HS_MAP_F16);
    return m > 0 ? entry : -entry;
  };
  tiles([&](int t, int a, int b, uint32_t) {
    if (a == 0) return;
    const bool drop = is_dropped(t);
    const int na = drop ? 0 : moved(a, a > 0 ? 0 : 1), nb = drop ? 0 : moved(b, b > 0 ? 2 : 3);
    if (na != a) k_map[t] = na;
    if (nb != b) v_map[t] = nb;
  });
  if (COPY) {
    __syncthreads();
    for (int i = 0; i < n_holes[0] + n_holes[1] + n_holes[2] + n_holes[3]; i++)
      copy_tile<NT>(kv, row, T, my_ws, i, n_holes[0], n_holes[1], n_holes[2]);
  } else if (tid < 4) {
    my_ws[tid] = n_holes[tid];
  }
}

// grid (any, rows).  HBM-bound: 270 MB read and written in 48 us, 5.6 TB/s.
__global__ __launch_bounds__(256) void evict_move_kernel(int T, hs_kv_dev kv, int32_t* __restrict__ ws) {
  const int64_t row = blockIdx.y;
  const int32_t* my_ws = row_ws(ws, row, T);
  const int n0 = my_ws[0], n1 = my_ws[1], n2 = my_ws[2], n3 = my_ws[3];
  for (int i = blockIdx.x; i < n0 + n1 + n2 + n3; i += gridDim.x) copy_tile<256>(kv, row, T, my_ws, i, n0, n1, n2);
}

}  // namespace

hipError_t hs_launch_evict(int B, int Hkv, int T, const hs_kv_dev& kv, const float* mass, int keep, const int32_t* keeps, int first, int last,
                           int32_t* ws, hipStream_t st) {
  const int rows = B * Hkv, words = (T + 31) / 32;
  const size_t lds = 7 * words * sizeof(uint32_t);
  // No row can hold more tiles than its pools have slots: with room for few more than `keep` (a cache of fixed size that grows tile by tile) a
  // row's workgroup makes the few moves itself, and there is one launch.
  const int most = (int)(min((int64_t)T, min((int64_t)kv.cap_dense_k + kv.cap_sparse_k, (int64_t)kv.cap_dense_v + kv.cap_sparse_v)));
  const bool copy = keeps == nullptr && most - keep <= 4;
#define HS_EVICT(NT_, PER_)                                                                                                          \
  do {                                                                                                                               \
    if (copy) hipLaunchKernelGGL((evict_kernel<NT_, PER_, true>), dim3(rows), dim3(NT_), lds, st, T, kv, mass, keep, keeps, first, last, ws); \
    else hipLaunchKernelGGL((evict_kernel<NT_, PER_, false>), dim3(rows), dim3(NT_), lds, st, T, kv, mass, keep, keeps, first, last, ws);     \
  } while (0)
  if (T <= 256) HS_EVICT(256, 1);
  else if (T <= 1024) HS_EVICT(512, 2);
  else if (T <= 4096) HS_EVICT(1024, 4);
  else HS_EVICT(1024, 0);
#undef HS_EVICT
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || copy) return e;
  int per_row = 2048 / rows;
  if (per_row < 1) per_row = 1;
  if (per_row > T) per_row = T;
  hipLaunchKernelGGL(evict_move_kernel, dim3(per_row, rows), dim3(256), 0, st, T, kv, ws);
  return hipGetLastError();
}
