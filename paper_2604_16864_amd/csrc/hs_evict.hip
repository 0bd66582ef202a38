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

// one workgroup per row
template <int NT>
__global__ __launch_bounds__(NT) void evict_select_kernel(int T, int4 caps, int32_t* __restrict__ k_map, int32_t* __restrict__ v_map, const float* __restrict__ mass, int keep,
                                                          const int32_t* __restrict__ keeps, int first, int last, int32_t* __restrict__ ws) {
  extern __shared__ uint32_t lds[];
  __shared__ int hist[260], sm[NT / 64], bounds[2], left[4], n_holes[2];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  k_map += row * T; v_map += row * T; mass += row * T;
  int32_t* my_ws = row_ws(ws, row, T);
  const int words = (T + 31) / 32;
  uint32_t* dropped = lds;                        // a bit per tile
  uint32_t* marks[2] = {lds + words, lds + 2 * words};         // a bit per slot of the dense and the 2:4 pool
  uint32_t* before[2] = {lds + 3 * words, lds + 4 * words};    // marks in front of a word
  if (keeps != nullptr) keep = max(1, keeps[row]);

  // tiles held, and the places between which they may be dropped
  int n = 0;
  for (int t0 = 0; t0 < T; t0 += NT) {
    const int t = t0 + tid;
    number_of<NT>(t < T && k_map[t] != 0, n, sm);
  }
  const int n_drop = min(n - keep, n - min(n, first) - min(n, last));  // may be negative
  if (n_drop <= 0) {  // the whole workgroup
    if (tid < 4) my_ws[tid] = 0;
    return;
  }
  if (tid == 0) { bounds[0] = 0; bounds[1] = T; }
  if (tid < 4) left[tid] = 0;
  for (int i = tid; i < words; i += NT) dropped[i] = 0;
  __syncthreads();
  int seen = 0;
  for (int t0 = 0; t0 < T; t0 += NT) {
    const int t = t0 + tid;
    const bool held = t < T && k_map[t] != 0;
    const int number = number_of<NT>(held, seen, sm);
    if (held && number == first) bounds[0] = t;
    if (held && number == n - last) bounds[1] = t;
  }
  __syncthreads();
  const int lo = bounds[0], hi = bounds[1];
  auto candidate = [&](int t, uint32_t& key) -> bool {
    if (k_map[t] == 0) return false;
    key = rank_key(mass[t]);
    return true;
  };
  const Threshold th = smallest<NT>(lo, hi, n_drop, candidate, hist);
  int tie = 0;
  for (int t0 = 0; t0 < T; t0 += NT) {
    const int t = t0 + tid;
    const int mk = t < T ? k_map[t] : 0;
    const bool cand = mk != 0 && t >= lo && t < hi;
    const uint32_t key = cand ? rank_key(mass[t]) : 0xffffffffu;
    const int number = number_of<NT>(cand && key == th.key, tie, sm);
    const bool drop = cand && (key < th.key || (key == th.key && number < th.ties));
    if (drop) atomicOr(&dropped[t >> 5], 1u << (t & 31));
    if (mk != 0 && !drop) {
      atomicAdd(&left[mk > 0 ? 0 : 1], 1);
      atomicAdd(&left[v_map[t] > 0 ? 2 : 3], 1);
    }
  }
  __syncthreads();

  for (int x = 0; x < 2; x++) {  // K, then V
    int32_t* map = x == 0 ? k_map : v_map;
    int32_t* list = my_ws + 4 + x * (T + 1);
    const int room[2] = {min(T, x == 0 ? caps.x : caps.z), min(T, x == 0 ? caps.y : caps.w)};  // slots of the two pools
    for (int i = tid; i < 2 * words; i += NT) lds[words + i] = 0;
    if (tid < 2) n_holes[tid] = 0;
    __syncthreads();
    for (int t = tid; t < T; t += NT) {
      const int m = map[t];
      if (m == 0) continue;
      const bool drop = (dropped[t >> 5] >> (t & 31)) & 1u;
      const int kind = m > 0 ? 0 : 1, slot = (abs(m) & ~HS_MAP_F16) - 1;
      if (slot < room[kind] && drop == (slot < left[2 * x + kind])) atomicOr(&marks[kind][slot >> 5], 1u << (slot & 31));
    }
    __syncthreads();
    for (int kind = 0; kind < 2; kind++) {  // marks in front of each word
      int carried = 0;
      for (int i0 = 0; i0 < words; i0 += NT) {
        const int i = i0 + tid;
        int upto = i < words ? __builtin_popcount(marks[kind][i]) : 0;
        const int mine = upto, l = tid & 63;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int y = __shfl_up(upto, d);
          if (l >= d) upto += y;
        }
        if (l == 63) sm[tid >> 6] = upto;
        __syncthreads();
        int off = carried;
        for (int k = 0; k < NT / 64; k++) {
          if (k < (tid >> 6)) off += sm[k];
          carried += sm[k];
        }
        if (i < words) {
          before[kind][i] = off + upto - mine;
          const int in_front = left[2 * x + kind] - 32 * i;  // slots of the word that are kept for the remaining tiles
          const uint32_t m = in_front >= 32 ? marks[kind][i] : (in_front <= 0 ? 0u : marks[kind][i] & ((1u << in_front) - 1u));
          if (m != 0) atomicAdd(&n_holes[kind], __builtin_popcount(m));
        }
        __syncthreads();
      }
    }
    // the freed slots, in order
    for (int kind = 0; kind < 2; kind++)
      for (int i = tid; i < words; i += NT) {
        uint32_t m = marks[kind][i];
        int k = before[kind][i];
        while (m != 0) {
          const int slot = 32 * i + __builtin_ctz(m);
          m &= m - 1;
          if (slot < left[2 * x + kind]) list[(kind == 0 ? 0 : n_holes[0]) + k] = slot;
          k++;
        }
      }
    __syncthreads();
    for (int t = tid; t < T; t += NT) {
      const int m = map[t];
      if (m == 0) continue;
      if ((dropped[t >> 5] >> (t & 31)) & 1u) continue;
      const int kind = m > 0 ? 0 : 1, slot = (abs(m) & ~HS_MAP_F16) - 1;
      if (slot >= room[kind] || slot < left[2 * x + kind]) continue;
      const int k = before[kind][slot >> 5] + __builtin_popcount(marks[kind][slot >> 5] & ((1u << (slot & 31)) - 1u)) - n_holes[kind];
      if (k < 0 || k >= n_holes[kind]) continue;  // slots that are not 0 .. n - 1: the tile stays
      const int at = (kind == 0 ? 0 : n_holes[0]) + k, to = list[at];
      list[at] = (int32_t)((uint32_t)slot << 16 | (uint32_t)to);
      const int entry = (to + 1) | (abs(m) & HS_MAP_F16);
      map[t] = m > 0 ? entry : -entry;
    }
    __syncthreads();
    if (tid < 2) my_ws[2 * x + tid] = n_holes[tid];
    for (int t = tid; t < T; t += NT)
      if (x == 1 && ((dropped[t >> 5] >> (t & 31)) & 1u)) { k_map[t] = 0; v_map[t] = 0; }
    __syncthreads();
  }
}

__device__ __forceinline__ void copy_slot(uint8_t* pool, int64_t base, int bytes, uint32_t move, int tid) {
  const uint4* s = reinterpret_cast<const uint4*>(pool + (base + (move >> 16)) * bytes);
  uint4* d = reinterpret_cast<uint4*>(pool + (base + (move & 0xffffu)) * bytes);
  for (int i = tid; i < bytes / 16; i += 256) d[i] = s[i];
}

// grid (any, rows)
__global__ __launch_bounds__(256) void evict_move_kernel(int T, hs_kv_dev kv, int32_t* __restrict__ ws) {
  const int64_t row = blockIdx.y;
  const int32_t* my_ws = row_ws(ws, row, T);
  const int n0 = my_ws[0], n1 = my_ws[1], n2 = my_ws[2], n3 = my_ws[3], tid = threadIdx.x;
  for (int i = blockIdx.x; i < n0 + n1 + n2 + n3; i += gridDim.x) {
    if (i < n0 + n1) {
      const uint32_t move = (uint32_t)my_ws[4 + i];
      if (i < n0) {
        copy_slot((uint8_t*)kv.k_dense, row * kv.cap_dense_k, HS_TILE_DENSE_BYTES, move, tid);
      } else {
        copy_slot((uint8_t*)kv.k_nnz, row * kv.cap_sparse_k, HS_TILE_NNZ_BYTES, move, tid);
        copy_slot((uint8_t*)kv.k_meta, row * kv.cap_sparse_k, HS_TILE_META_BYTES, move, tid);
      }
    } else {
      const int j = i - n0 - n1;
      const uint32_t move = (uint32_t)my_ws[4 + (T + 1) + j];
      if (j < n2) {
        copy_slot((uint8_t*)kv.v_dense, row * kv.cap_dense_v, HS_TILE_DENSE_BYTES, move, tid);
      } else {
        copy_slot((uint8_t*)kv.v_nnz, row * kv.cap_sparse_v, HS_TILE_NNZ_BYTES, move, tid);
        copy_slot((uint8_t*)kv.v_meta, row * kv.cap_sparse_v, HS_TILE_META_BYTES, move, tid);
      }
    }
  }
}

}  // namespace

hipError_t hs_launch_evict(int B, int Hkv, int T, const hs_kv_dev& kv, const float* mass, int keep, const int32_t* keeps, int first, int last,
                           int32_t* ws, hipStream_t st) {
  const int rows = B * Hkv, words = (T + 31) / 32;
  const size_t lds = 5 * words * sizeof(uint32_t);
  const int4 caps = make_int4(kv.cap_dense_k, kv.cap_sparse_k, kv.cap_dense_v, kv.cap_sparse_v);
  if (T <= 1024)
    hipLaunchKernelGGL((evict_select_kernel<256>), dim3(rows), dim3(256), lds, st, T, caps, (int32_t*)kv.k_map, (int32_t*)kv.v_map, mass, keep, keeps, first, last, ws);
  else
    hipLaunchKernelGGL((evict_select_kernel<1024>), dim3(rows), dim3(1024), lds, st, T, caps, (int32_t*)kv.k_map, (int32_t*)kv.v_map, mass, keep, keeps, first, last, ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  int per_row = 2048 / rows;
  if (per_row < 1) per_row = 1;
  if (per_row > T) per_row = T;
  hipLaunchKernelGGL(evict_move_kernel, dim3(per_row, rows), dim3(256), 0, st, T, kv, ws);
  return hipGetLastError();
}
