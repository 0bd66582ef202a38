// Attention of every query over the tiles that its list names: decode attention's work on a tile, with tiles handed out from a list.
// Included by the translation units that instantiate it: hs_listed.hip (tensors of one kind) and hs_listed_mixed.hip.
#pragma once
#include "hs_rank.h"
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

constexpr int kLaneEntries = 4;  // entries of a list that a lane can hold: lists of up to 256 are looked at in registers

// grid: n_splits workgroups for each query of each (batch, kv head) row, rows fastest.  A workgroup takes the share [n s / S, n (s + 1) / S) of the list's
// tiles in ascending order, each of its NW waves every NW-th of these.  Which tiles these are every wave finds by itself, in registers, where the list is what
// hs_pick_tiles writes: ascending, what is no tile (or begins behind a causal query) at its end.  Any other list is marked in a bit map of the row's tiles and
// numbered from there, so that order, tiles named twice and numbers between them that are no tiles do not matter.
// The tile that a causal query stands in is left out of this and done by the last workgroup's first wave, which has the fewest of the others, with the tokens behind the query cut off.  The dense
// tail has workgroups of its own behind all others, or, of a query that one workgroup does, is its first four waves' beginning.
// UNIFORM: as in decode attention, slot == tile and one kind per tensor; the K map is not read.  STREAM: tiles are read past the caches.
template <int KM, int VM, bool F16, bool UNIFORM, int NW, bool STREAM>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2)))
void listed_kernel(hs_listed_args g, hs_kv_dev kv, int n_splits, float scale_log2, float* __restrict__ ws_o, float* __restrict__ ws_l) {
  extern __shared__ uint32_t sm_bits[];  // ceil(T / 32) words
  __shared__ __attribute__((aligned(16))) float sm_o[NW + 4][8][HS_D];
  __shared__ float sm_m[NW + 4][8], sm_l[NW + 4][8];
  __shared__ int sm_list[kListCap], sm_cnt[NW];
  const int tid = threadIdx.x, l = tid & 63, a = l >> 4, c = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = g.Hq / g.Hkv, T = g.T, BH = g.B * g.Hkv;
  int64_t n = blockIdx.x;
  const int row = (int)(n % BH);
  n /= BH;
  const int b = row / g.Hkv, h = row - b * g.Hkv;
  const int i_q = (int)(n % g.Lq), split = (int)(n / g.Lq);
  const bool last_split = split == n_splits - 1;
  const int64_t pos = g.causal ? (int64_t)g.q_start + i_q : (int64_t)T * HS_BT - 1;  // the last token seen
  const int t_end = (int)((pos + 1) / HS_BT);  // tiles that are seen whole: those below
  const int t_cut = (pos + 1) % HS_BT != 0 ? t_end : -1;  // the one that is not, if any
  const int32_t* list = g.list + ((int64_t)row * g.Lq + i_q) * g.n_list;
  int entry[kLaneEntries];
#pragma unroll
  for (int j = 0; j < kLaneEntries; j++) entry[j] = 64 * j + l < g.n_list ? list[64 * j + l] : -1;
  uint4 qb[4];
  load_q(g.q.p + b * g.q.sb + (int64_t)h * G * g.q.sh + i_q * g.q.st, 0, g.q.sh, 1, G, a, c, qb);
  auto tail_part = [&](int q, int part) {
    const int tail_len = __builtin_amdgcn_readfirstlane(g.tail_lens != nullptr ? min(max(g.tail_lens[b], 0), HS_BT) : g.tail_len);
    tail_piece<F16, false>(TailArgs{g.tail_k, g.tail_v, nullptr, 0}, tail_len, row, q, qb, scale_log2, l, sm_o[part], sm_m[part], sm_l[part]);
  };
  const int64_t hq0 = ((int64_t)b * g.Hq + h * G) * g.Lq + i_q;
  const int n_parts = n_splits + (n_splits > 1 && g.tail_len >= 0 ? 1 : 0);
  if (split == n_splits) {  // the whole workgroup: the dense tail of a row, a part of its own
    if (w < 4) tail_part(w, w);
    __syncthreads();
    combine_parts<F16, false, 4>(tid, false, G, hq0, g.Lq, sm_m, sm_l, sm_o, n_parts, split, ws_o, ws_l);
    return;
  }
  const bool with_tail = n_splits == 1 && g.tail_len >= 0;
  if (with_tail && w < 4) tail_part(w, NW + w);

  f32x4_t o[8];
#pragma unroll
  for (int i = 0; i < 8; i++) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;

  // ---- which tiles ----
  int n_all = 0;          // tiles seen whole that the list names
  bool plain = g.n_list <= 64 * kLaneEntries, cut = false;
  {
    bool more = true;     // every entry so far is a tile
    int before = -1;
#pragma unroll
    for (int j = 0; j < kLaneEntries; j++) {
      if (64 * j < g.n_list) {
        const unsigned long long whole = __ballot(entry[j] >= 0 && entry[j] < t_end), half = __ballot(entry[j] == t_cut && t_cut >= 0);
        const unsigned long long good = whole | half;
        int low = __shfl_up(entry[j], 1);
        if (l == 0) low = before;
        before = __builtin_amdgcn_readlane(entry[j], 63);
        plain = plain && (good & (good + 1ull)) == 0ull && (more || good == 0ull) && __ballot((good >> l & 1ull) && low >= entry[j]) == 0ull;
        more = good == ~0ull;
        n_all += __builtin_popcountll(whole);
        cut = cut || half != 0ull;
      }
    }
  }
  int first = 0, w0 = 0, w1 = 0;  // of a list that is not plain: the number of this thread's first tile, and its words of the bit map
  if (!plain) {                   // the same in all waves
    const int n_words = (T + 31) / 32;
    for (int i = tid; i < n_words; i += 64 * NW) sm_bits[i] = 0u;
    __syncthreads();
    bool mine_cut = false;
    for (int i = tid; i < g.n_list; i += 64 * NW) {
      const int t = list[i];
      if (t >= 0 && t < t_end) atomicOr(&sm_bits[t >> 5], 1u << (t & 31));
      mine_cut |= t == t_cut && t_cut >= 0;
    }
    cut = __syncthreads_or(mine_cut) != 0;
    const int per = (n_words + 64 * NW - 1) / (64 * NW);
    w0 = min(n_words, tid * per);
    w1 = min(n_words, w0 + per);
    int mine = 0;
    for (int i = w0; i < w1; i++) mine += __builtin_popcount(sm_bits[i]);
    const int upto = wave_upto(mine);
    if (l == 63) sm_cnt[w] = upto;
    __syncthreads();
    first = upto - mine;
    n_all = 0;
#pragma unroll
    for (int k = 0; k < NW; k++) {
      if (k < w) first += sm_cnt[k];
      n_all += sm_cnt[k];
    }
  }
  const int lo = (int)((int64_t)n_all * split / n_splits), hi = (int)((int64_t)n_all * (split + 1) / n_splits);

  // ---- their attention ----
  auto form_of = [](int mk, int mv) -> int { return (mk > 0 ? 1 : 0) | (mv > 0 ? 2 : 0) | ((!F16 && !hs_map_f16(mv)) ? 4 : 0); };
  constexpr int kFirstForm = (KM == 1 ? 1 : 0) | (VM == 1 ? 2 : 0);
  // The tiles numbered [from, to); tile_of(i): tile number i.  A wave takes up to 64 of its own a round, one form after the other, so that no branch sits
  // between loads and products; forms that none has are passed over.
  // Tiles that are both 2:4 are two in flight.  A dense operand leaves the registers for one: the next one's K is requested as soon as the scores are made, its V
  // behind the products.
  // GUESS (uniform caches): a round's first tiles are requested by their numbers alone, beside the read of the map; one whose V turns out to be in the other
  // encoding is left to the other form.
  auto attend = [&](int from, int to, auto tile_of) {
    for (int base = from + (NW - 1 - w); base < to; base += 64 * NW) {  // from the last wave on: the first ones have the tail
      const int i_mine = base + NW * l, t_v = tile_of(min(i_mine, to - 1));
      int mk_v = 0, mv_v = 0;
      if (i_mine < to) {
        mk_v = UNIFORM ? (KM == 0 ? -(t_v + 1) : t_v + 1) : kv.k_map[(int64_t)row * T + t_v];
        mv_v = UNIFORM && F16 ? (VM == 0 ? -(t_v + 1) : t_v + 1) : kv.v_map[(int64_t)row * T + t_v];
      }
      auto tiles_of = [&](auto form_c, auto guess_c) {
        constexpr int kForm = decltype(form_c)::value;
        constexpr bool GUESS = decltype(guess_c)::value;
        constexpr int KK = kForm & 1, VK = (kForm >> 1) & 1, kEnc = (kForm & 4) ? 0 : 1;
        constexpr int DEPTH = KK == 0 && VK == 0 ? 2 : 1;
        TileRegs<KK, VK> ring[DEPTH];
        bool have[DEPTH], wrong[DEPTH];
        if (GUESS) {
#pragma unroll
          for (int d = 0; d < DEPTH; d++) {
            have[d] = base + NW * d < to;
            const int slot = __builtin_amdgcn_readlane(mk_v, d);
            if (have[d]) tile_load<KK, VK, 3, STREAM>(ring[d], kv, row, slot, KK == VK ? slot : -slot, l);
          }
        }
        unsigned long long act = __ballot(mk_v != 0 && form_of(mk_v, mv_v) == kForm);
        if (!GUESS && act == 0ull) return;
        auto next = [&](int& mk, int& mv) -> bool {
          if (act == 0ull) return false;
          const int i = __builtin_ctzll(act);
          act &= act - 1;
          mk = __builtin_amdgcn_readlane(mk_v, i);
          mv = __builtin_amdgcn_readlane(mv_v, i);
          return true;
        };
#pragma unroll
        for (int d = 0; d < DEPTH; d++) {
          wrong[d] = GUESS && !F16 && have[d] && !(act >> d & 1ull);
          if (!GUESS) {
            int mk = 0, mv = 0;
            have[d] = next(mk, mv);
            if (have[d]) tile_load<KK, VK, 3, STREAM>(ring[d], kv, row, mk, mv, l);
          }
        }
        if (GUESS) act &= ~((1ull << DEPTH) - 1ull);
        bool go = have[0];
        while (go) {
#pragma unroll
          for (int d = 0; d < DEPTH; d++) {
            if (go && have[d]) {  // in the order of issue: the first empty slot ends the round
              int mk = 0, mv = 0;
              const bool more = next(mk, mv);
              if (!wrong[d]) {
                if (DEPTH == 1) {
                  tile_compute<KK, VK, F16, kEnc>(ring[d], qb, scale_log2, c, o, m_run, l_run, [&](f32x4_t (&)[4]) {
                    if (more) tile_load<KK, VK, 1, STREAM>(ring[d], kv, row, mk, mv, l);
                  });
                  if (more) tile_load<KK, VK, 2, STREAM>(ring[d], kv, row, mk, mv, l);
                } else {
                  tile_compute<KK, VK, F16, kEnc>(ring[d], qb, scale_log2, c, o, m_run, l_run);
                }
              }
              if ((DEPTH > 1 || wrong[d]) && more) tile_load<KK, VK, 3, STREAM>(ring[d], kv, row, mk, mv, l);
              wrong[d] = false;
              have[d] = more;
            } else {
              go = false;
            }
          }
        }
      };
      tiles_of(std::integral_constant<int, kFirstForm>{}, std::integral_constant<bool, UNIFORM>{});
      static_for_forms<KM, VM, F16, kFirstForm>([&](auto form_c) { tiles_of(form_c, std::false_type{}); });
    }
  };
  if (plain) {
    attend(lo, hi, [&](int i) {
      int t = 0;
#pragma unroll
      for (int j = 0; j < kLaneEntries; j++) {
        const int x = __shfl(entry[j], i & 63);
        if (i >> 6 == j) t = x;
      }
      return t;
    });
  } else {
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
      attend(0, r1 - r0, [&](int i) { return sm_list[i]; });
      __syncthreads();  // the list is rewritten by the next pass
    }
  }
  if (cut && last_split && w == 0) {
    const int mk = __builtin_amdgcn_readfirstlane(kv.k_map[(int64_t)row * T + t_cut]), mv = __builtin_amdgcn_readfirstlane(kv.v_map[(int64_t)row * T + t_cut]);
    const int limit = (int)((pos + 1) % HS_BT) - 1;
    static_for_forms<KM, VM, F16, -1>([&](auto form_c) {
      constexpr int kForm = decltype(form_c)::value;
      constexpr int KK = kForm & 1, VK = (kForm >> 1) & 1, kEnc = (kForm & 4) ? 0 : 1;
      if (mk == 0 || form_of(mk, mv) != kForm) return;
      TileRegs<KK, VK> r;
      tile_load<KK, VK, 3, STREAM>(r, kv, row, mk, mv, l);
      cut_values<KK, VK>(r, limit, a);
      tile_compute<KK, VK, F16, kEnc>(r, qb, scale_log2, c, o, m_run, l_run, [&](f32x4_t (&s)[4]) {
#pragma unroll
        for (int m = 0; m < 4; m++)
#pragma unroll
          for (int i = 0; i < 4; i++)
            if (16 * m + 4 * a + i > limit) s[m][i] = -INFINITY;
      });
    });
  }

  // ---- join: lane groups, hi/lo columns, then the waves ----
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
  __syncthreads();
  if (n_splits == 1) combine_parts<F16, true, NW, true>(tid, with_tail, G, hq0, g.Lq, sm_m, sm_l, sm_o, 1, 0, ws_o, ws_l);
  else combine_parts<F16, false, NW>(tid, false, G, hq0, g.Lq, sm_m, sm_l, sm_o, n_parts, split, ws_o, ws_l);
}

template <int KM, int VM, bool UNIFORM>
hipError_t launch_listed(const hs_listed_args& a, const hs_kv_dev& kv, bool f16, hs_listed_plan p, float* wo, float* wl, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.B * a.Hkv * ((int64_t)a.Lq * p.splits + (p.splits > 1 && a.tail_len >= 0 ? 1 : 0)))), block(64 * p.waves);
  const size_t lds = (size_t)(a.T + 31) / 32 * 4;
  const float sl2 = a.scale * kLog2e;
#define HS_LISTED(F16_, NW_, STREAM_) \
  hipLaunchKernelGGL((listed_kernel<KM, VM, F16_, UNIFORM, NW_, STREAM_>), grid, block, lds, st, a, kv, p.splits, sl2, wo, wl)
#define HS_LISTED_AS(F16_)                                                                     \
  if (a.Lq == 1) { if (p.waves == 8) HS_LISTED(F16_, 8, true); else HS_LISTED(F16_, 4, true); } \
  else { if (p.waves == 8) HS_LISTED(F16_, 8, false); else HS_LISTED(F16_, 4, false); }
  if (f16) {
    HS_LISTED_AS(true)
  } else {
    HS_LISTED_AS(false)
  }
#undef HS_LISTED_AS
#undef HS_LISTED
  return hipGetLastError();
}

}  // namespace
