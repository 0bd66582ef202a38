// Attention of every query over the tiles that its list names: the kernels of decode attention's tiles, handed out from a list.
#include "hs_tile.h"

namespace {

constexpr int kListCap = 1024;  // tiles listed in LDS at a time; longer shares take several passes

// Values of V of tokens behind `limit` (a token of the tile, the same for all columns) set to zero: their numerators are 0, which an infinity or
// NaN among them would make NaN.
template <int KM, int VM>
__device__ __forceinline__ void cut_values(TileRegs<KM, VM>& r, int limit, int a) {
  const uint32_t idx[4] = {r.vm.x, r.vm.y, r.vm.z, r.vm.w};
#pragma unroll
  for (int i = 0; i < TileRegs<KM, VM>::kNV; i++) {
    uint32_t v[4] = {r.v[i].x, r.v[i].y, r.v[i].z, r.v[i].w};
#pragma unroll
    for (int q = 0; q < 4; q++) {
      int t0, t1;  // tokens of the pair
      if (VM == 0) {
        const int g = 4 * (2 * (a >> 1) + (q & 1)) + 2 * (a & 1) + (q >> 1);
        const uint32_t at = idx[i >> 1] >> (16 * (i & 1) + 4 * q);
        t0 = 4 * g + (int)(at & 3u);
        t1 = 4 * g + (int)((at >> 2) & 3u);
      } else {
        t0 = 16 * (2 * (i & 1) + q / 2) + 4 * a + 2 * (q & 1);
        t1 = t0 + 1;
      }
      v[q] &= (t0 > limit ? 0u : 0xffffu) | (t1 > limit ? 0u : 0xffff0000u);
    }
    r.v[i] = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

// grid: n_splits workgroups for each query of each (batch, kv head) row, rows fastest, and behind them, for a tail that is a part of its own, one for
// each row.  A workgroup marks the tiles of its query's list in a bit map of the row (so that the order of a list, tiles named twice and
// numbers that are no tiles do not matter), numbers them, and takes the share [n s / S, n (s + 1) / S) of the numbers, its waves every NW-th of these.
template <int KM, int VM, bool F16, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2)))
void listed_kernel(hs_listed_args g, hs_kv_dev kv, int n_splits, int n_parts, float scale_log2, float* __restrict__ ws_o, float* __restrict__ ws_l) {
  constexpr bool DIRECT = NW == 8;
  constexpr int kParts = DIRECT ? NW + 4 : NW;
  extern __shared__ uint32_t sm_bits[];  // ceil(T / 32) words
  __shared__ __attribute__((aligned(16))) float sm_o[kParts][8][HS_D];
  __shared__ float sm_m[kParts][8], sm_l[kParts][8];
  __shared__ int sm_list[kListCap], sm_cnt[NW];
  const int tid = threadIdx.x, l = tid & 63, a = l >> 4, c = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = g.Hq / g.Hkv, T = g.T, BH = g.B * g.Hkv;
  int64_t n = blockIdx.x;
  const int row = (int)(n % BH);
  n /= BH;
  const int b = row / g.Hkv, h = row - b * g.Hkv;
  const TailArgs tail{g.tail_k, g.tail_v, g.tail_lens, g.tail_len};
  auto tail_length = [&]() -> int {
    return __builtin_amdgcn_readfirstlane(tail.lens != nullptr ? min(max(tail.lens[b], 0), HS_BT) : tail.len);
  };
  const bool is_tail = !DIRECT && n >= (int64_t)n_splits * g.Lq;
  const int i_q = is_tail ? 0 : (int)(n % g.Lq), split = is_tail ? n_parts - 1 : (int)(n / g.Lq);
  uint4 qb[4];
  load_q(g.q.p + b * g.q.sb + (int64_t)h * G * g.q.sh + i_q * g.q.st, 0, g.q.sh, 1, G, a, c, qb);
  if (is_tail) {
    tail_piece<F16, false>(tail, tail_length(), row, w, qb, scale_log2, l, sm_o[w], sm_m[w], sm_l[w]);
  } else {
    f32x4_t o[8];
#pragma unroll
    for (int i = 0; i < 8; i++) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;
    const int64_t pos = g.causal ? (int64_t)g.q_start + i_q : (int64_t)T * HS_BT;  // the last token seen
    const int32_t* list = g.list + ((int64_t)row * g.Lq + i_q) * g.n_list;
    const int n_words = (T + 31) / 32;
    for (int i = tid; i < n_words; i += 64 * NW) sm_bits[i] = 0u;
    __syncthreads();
    for (int i = tid; i < g.n_list; i += 64 * NW) {
      const int t = list[i];
      if (t >= 0 && t < T && (int64_t)t * HS_BT <= pos) atomicOr(&sm_bits[t >> 5], 1u << (t & 31));
    }
    __syncthreads();
    // words of this thread, in order
    const int per = (n_words + 64 * NW - 1) / (64 * NW), w0 = min(n_words, tid * per), w1 = min(n_words, w0 + per);
    int mine = 0;
    for (int i = w0; i < w1; i++) mine += __builtin_popcount(sm_bits[i]);
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int below = __shfl_up(upto, d);
      if (l >= d) upto += below;
    }
    if (l == 63) sm_cnt[w] = upto;
    __syncthreads();
    int first = upto - mine, n_all = 0;
#pragma unroll
    for (int k = 0; k < NW; k++) {
      if (k < w) first += sm_cnt[k];
      n_all += sm_cnt[k];
    }
    const int lo = (int)((int64_t)n_all * split / n_splits), hi = (int)((int64_t)n_all * (split + 1) / n_splits);

    auto form_of = [](int mk, int mv) -> int { return (mk > 0 ? 1 : 0) | (mv > 0 ? 2 : 0) | ((!F16 && !hs_map_f16(mv)) ? 4 : 0); };
    constexpr int kFirstForm = (KM == 1 ? 1 : 0) | (VM == 1 ? 2 : 0);
    // One sweep over the list's tiles of one form; wave w takes every NW-th.  Returns the set of forms that it met.
    auto sweep = [&](auto form_c, int n_list) -> unsigned {
      constexpr int kForm = decltype(form_c)::value;
      constexpr int KK = kForm & 1, VK = (kForm >> 1) & 1, kEnc = (kForm & 4) ? 0 : 1;
      constexpr int DEPTH = KK == 0 && VK == 0 ? 2 : 1;
      TileRegs<KK, VK> ring[DEPTH];
      int at[DEPTH];
      bool have[DEPTH];
      unsigned seen = 0;
      for (int base = w; base < n_list; base += 64 * NW) {
        const int i_mine = base + NW * l;
        int t_v = 0, mk_v = 0, mv_v = 0;
        if (i_mine < n_list) {
          t_v = sm_list[i_mine];
          mk_v = kv.uniform ? (KM == 0 ? -(t_v + 1) : t_v + 1) : kv.k_map[(int64_t)row * T + t_v];
          mv_v = kv.uniform && F16 ? (VM == 0 ? -(t_v + 1) : t_v + 1) : kv.v_map[(int64_t)row * T + t_v];
        }
        const int form_v = form_of(mk_v, mv_v);
        unsigned long long act = __ballot(mk_v != 0 && form_v == kForm);
#pragma unroll
        for (int f = 0; f < 8; f++)
          if (f != kForm && form_allowed<KM, VM, F16>(f)) seen |= (__ballot(mk_v != 0 && form_v == f) != 0ull ? 1u : 0u) << f;
        auto fetch = [&](int d) {
          have[d] = act != 0ull;
          if (have[d]) {
            const int i = __builtin_ctzll(act);
            act &= act - 1;
            at[d] = __builtin_amdgcn_readlane(t_v, i);
            tile_load<KK, VK>(ring[d], kv, row, __builtin_amdgcn_readlane(mk_v, i), __builtin_amdgcn_readlane(mv_v, i), l);
          }
        };
#pragma unroll
        for (int d = 0; d < DEPTH; d++) fetch(d);
        bool go = have[0];
        while (go) {
#pragma unroll
          for (int d = 0; d < DEPTH; d++) {
            if (go && have[d]) {  // in the order of issue: the first empty slot ends the round
              const int64_t limit = pos - (int64_t)at[d] * HS_BT;  // the last token of the tile that is seen
              if (limit < HS_BT - 1) {
                cut_values<KK, VK>(ring[d], (int)limit, a);
                tile_compute<KK, VK, F16, kEnc>(ring[d], qb, scale_log2, c, o, m_run, l_run, [&](f32x4_t (&s)[4]) {
#pragma unroll
                  for (int m = 0; m < 4; m++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                      if (16 * m + 4 * a + i > (int)limit) s[m][i] = -INFINITY;
                });
              } else {
                tile_compute<KK, VK, F16, kEnc>(ring[d], qb, scale_log2, c, o, m_run, l_run);
              }
              fetch(d);
            } else {
              go = false;
            }
          }
        }
      }
      return seen;
    };
    for (int r0 = lo; r0 < hi; r0 += kListCap) {  // the same trips in every thread
      const int r1 = min(hi, r0 + kListCap);
      int number = first;
      for (int i = w0; i < w1 && number < r1; i++) {
        uint32_t bits = sm_bits[i];
        while (bits != 0u && number < r1) {
          if (number >= r0) sm_list[number - r0] = 32 * i + __builtin_ctz(bits);
          bits &= bits - 1;
          number++;
        }
      }
      __syncthreads();
      const unsigned seen = sweep(std::integral_constant<int, kFirstForm>{}, r1 - r0);
      static_for_forms<KM, VM, F16, kFirstForm>([&](auto form_c) {
        if ((seen >> decltype(form_c)::value) & 1u) sweep(form_c, r1 - r0);
      });
      __syncthreads();  // the list is rewritten by the next pass
    }
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
#pragma unroll
    for (int i = 0; i < 8; i++)
#pragma unroll
      for (int j = 0; j < 4; j++) {  // column c + column c^8 (rotate by 8 inside the 16-lane row)
        const int other = __builtin_amdgcn_mov_dpp(__float_as_int(o[i][j]), 0x128, 0xf, 0xf, true);
        o[i][j] += __int_as_float(other);
      }
    if (c < 8) {
      if (a == 0) { sm_m[w][c] = m_run; sm_l[w][c] = l_run; }
#pragma unroll
      for (int mb = 0; mb < 8; mb++)
        *reinterpret_cast<float4*>(&sm_o[w][c][16 * mb + 4 * a]) = make_float4(o[mb][0], o[mb][1], o[mb][2], o[mb][3]);
    }
    if constexpr (DIRECT) {
      if (tail.len >= 0) {
        const int q = NW - 1 - w;
        if (q < 4) tail_piece<F16, false>(tail, tail_length(), row, q, qb, scale_log2, l, sm_o[NW + q], sm_m[NW + q], sm_l[NW + q]);
      }
    }
  }
  __syncthreads();
  combine_parts<F16, DIRECT, NW>(tid, tail.len >= 0, G, ((int64_t)b * g.Hq + h * G) * g.Lq + i_q, g.Lq, sm_m, sm_l, sm_o, n_parts, split, ws_o, ws_l);
}

template <int KM, int VM, int NW>
hipError_t launch(const hs_listed_args& a, const hs_kv_dev& kv, bool f16, int n_splits, int n_parts, float* wo, float* wl, hipStream_t st) {
  const int64_t blocks = (int64_t)a.B * a.Hkv * ((int64_t)a.Lq * n_splits + (NW == 4 && a.tail_len >= 0 ? 1 : 0));
  const size_t lds = (size_t)(a.T + 31) / 32 * 4;
  const float sl2 = a.scale * kLog2e;
  if (f16) hipLaunchKernelGGL((listed_kernel<KM, VM, true, NW>), dim3((unsigned)blocks), dim3(64 * NW), lds, st, a, kv, n_splits, n_parts, sl2, wo, wl);
  else hipLaunchKernelGGL((listed_kernel<KM, VM, false, NW>), dim3((unsigned)blocks), dim3(64 * NW), lds, st, a, kv, n_splits, n_parts, sl2, wo, wl);
  return hipGetLastError();
}

}  // namespace

int hs_listed_splits(int B, int Hkv, int Lq, int n_list) {
  const int64_t rows = (int64_t)B * Hkv * Lq;
  int64_t n = 512 / rows;
  if (n > (n_list + 3) / 4) n = (n_list + 3) / 4;
  return n < 1 ? 1 : (int)n;
}
int hs_listed_parts(int B, int Hkv, int Lq, int n_list, int with_tail) {
  const int n = hs_listed_splits(B, Hkv, Lq, n_list);
  return n == 1 ? 0 : n + (with_tail ? 1 : 0);
}

hipError_t hs_launch_listed(const hs_listed_args& a, const hs_kv_dev& kv, int dtype, hipStream_t st) {
  const int km = kv.cap_dense_k == 0 ? 0 : (kv.cap_sparse_k == 0 ? 1 : 2);
  const int vm = kv.cap_dense_v == 0 ? 0 : (kv.cap_sparse_v == 0 ? 1 : 2);
  const int n_splits = hs_listed_splits(a.B, a.Hkv, a.Lq, a.n_list), n_parts = hs_listed_parts(a.B, a.Hkv, a.Lq, a.n_list, a.tail_len >= 0);
  const bool direct = n_parts == 0;
  const int64_t rows = (int64_t)a.B * a.Hq * a.Lq;
  float* wo = direct ? reinterpret_cast<float*>(a.o) : a.ws;
  float* wl = direct ? a.lse : a.ws + (size_t)rows * n_parts * HS_D;
  hipError_t e = hipSuccess;
#define HS_GO(KM_, VM_)                                                                                    \
  e = direct ? launch<KM_, VM_, 8>(a, kv, dtype == HS_FP16, 1, 1, wo, wl, st)                              \
             : launch<KM_, VM_, 4>(a, kv, dtype == HS_FP16, n_splits, n_parts, wo, wl, st);                \
  break
  switch (km * 3 + vm) {
    case 0: HS_GO(0, 0);
    case 1: HS_GO(0, 1);
    case 2: HS_GO(0, 2);
    case 3: HS_GO(1, 0);
    case 4: HS_GO(1, 1);
    case 5: HS_GO(1, 2);
    case 6: HS_GO(2, 0);
    case 7: HS_GO(2, 1);
    default: HS_GO(2, 2);
  }
#undef HS_GO
  if (e != hipSuccess || direct) return e;
  return hs_launch_merge(rows, n_parts, wo, wl, a.o, a.lse, st, dtype);
}
