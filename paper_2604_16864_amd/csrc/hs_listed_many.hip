// Attention over listed tiles of more than one query a sequence: neighbouring queries share a workgroup, over the tiles that any of them picks.
#include "hs_listed_kernel.h"

namespace {
// Queries that stand side by side pick much the same tiles: up to 16 / G of them share a workgroup, their heads as the 16 columns of the products, over all tiles that
// one of their lists names.  A column whose query does not see a tile, or not all of it, has scores of -inf there.  What bounds it: a tile's chain of loads,
// products, exponentials and products, 1.05 us a tile for a wave alone on its SIMD (600 rows of 64 tiles, 4 heads, 2:4, 28 us: 150 workgroups, 24 tiles a wave), and the places of the workgroups:
// 2400 rows, 59 to 62 us, are 600 workgroups for 512 places (two a compute unit), 1.2 waves a SIMD on average; tiles come out of the L2 at 16 TB/s then, each for 16 columns, the vector ALU is active in 27 % of the
// time, the matrix cores in 9 %.  Three waves a SIMD spill (2400 rows 73 where two took 56).  With two, nothing spills where K or V is all 2:4; else 4
// (all dense) to 26 registers (both mixed) do in bf16, up to 9 in fp16: 2400 rows with half of both dense 79 us, all dense 87, in fp16 74 and 86.
// The numerators enter the second product in one term of 11 bits (a V tile in fp16 encoding), or two of 8 (bf16).
constexpr float kSlack = 7.f;  // numerators reach 2^15, which fp16 holds
template <int KM, int VM, bool F16, int ENC, typename Limit>
__device__ __forceinline__ void tile_compute_many(const TileRegs<KM, VM>& r, const uint4 (&qb)[4], float scale_log2, float slack, f32x4_t (&o)[8], float& m_run,
                                                  float& l_run, Limit limit) {
  constexpr int kNK = TileRegs<KM, VM>::kNK, kNV = TileRegs<KM, VM>::kNV;
  typedef hs_elem<F16> E;
  typedef hs_elem<ENC == 1> EV;
  constexpr float kShift = 8.f;  // as in tile_compute
  const int kidx[4] = {(int)r.km.x, (int)r.km.y, (int)r.km.z, (int)r.km.w};
  const int vidx[4] = {(int)r.vm.x, (int)r.vm.y, (int)r.vm.z, (int)r.vm.w};
  f32x4_t s[4];
#pragma unroll
  for (int m = 0; m < 4; m++) {
    s[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (KM == 0) {
      s[m] = E::template smma<0>(r.k[2 * m], qb[0], qb[1], s[m], kidx[m]);
      s[m] = E::template smma<1>(r.k[2 * m + 1], qb[2], qb[3], s[m], kidx[m]);
    } else {
#pragma unroll
      for (int st = 0; st < 4; st++) s[m] = E::mma(r.k[(4 * m + st) % kNK], qb[st], s[m]);
    }
  }
  limit(s);
  const float m_prev = m_run;
  float mx = -INFINITY;
#pragma unroll
  for (int m = 0; m < 4; m++)
#pragma unroll
    for (int i = 0; i < 4; i++) mx = fmaxf(mx, s[m][i]);
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  // The reference follows the maximum only when that has grown by more than `slack` binades: a row's tiles mostly leave it, and the accumulators, as they are.
  const float want = mx * scale_log2 - kShift;
  float alpha = 1.f;
  const bool moves = __ballot(want > m_prev + slack) != 0ull;
  if (moves) m_run = fmaxf(m_prev, want);
  const float m_ref = m_run > -INFINITY ? m_run : 0.f;  // nothing seen so far: weights 0, not exp2(-inf + inf)
  if (moves) alpha = __builtin_amdgcn_exp2f(m_prev - m_ref);
  float p[4][4], psum = 0.f;
#pragma unroll
  for (int m = 0; m < 4; m++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      p[m][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[m][i], scale_log2, -m_ref));
      psum += p[m][i];
    }
  l_run = l_run * alpha + psum;
  if (moves) {
#pragma unroll
    for (int i = 0; i < 8; i++) o[i] *= alpha;
  }
  uint32_t hi[8];
#pragma unroll
  for (int m = 0; m < 4; m++) {
    hi[2 * m] = EV::pack2(p[m][0], p[m][1]);
    hi[2 * m + 1] = EV::pack2(p[m][2], p[m][3]);
  }
  auto add = [&](const uint32_t (&pb)[8]) {
    const uint4 lo4 = make_uint4(pb[0], pb[1], pb[2], pb[3]), hi4 = make_uint4(pb[4], pb[5], pb[6], pb[7]);
#pragma unroll
    for (int mb = 0; mb < 8; mb++) {
      if (VM == 0) {
        if (mb & 1) o[mb] = EV::template smma<1>(r.v[mb], lo4, hi4, o[mb], vidx[mb >> 1]);
        else o[mb] = EV::template smma<0>(r.v[mb], lo4, hi4, o[mb], vidx[mb >> 1]);
      } else {
        o[mb] = EV::mma(r.v[(2 * mb) % kNV], lo4, o[mb]);
        o[mb] = EV::mma(r.v[(2 * mb + 1) % kNV], hi4, o[mb]);
      }
    }
  };
  add(hi);
  if (ENC == 0) {
#pragma unroll
    for (int m = 0; m < 4; m++)
#pragma unroll
      for (int u = 0; u < 2; u++)
        hi[2 * m + u] = EV::pack2(p[m][2 * u] - EV::lo_f32(hi[2 * m + u]), p[m][2 * u + 1] - EV::hi_f32(hi[2 * m + u]));
    add(hi);
  }
}

// grid: n_splits workgroups of 4 waves for each block of n_queries <= 16 / G queries of each row, rows fastest (so that the workgroups of a row meet on few XCDs, whose L2
// then has its tiles).  The lists are marked in a bit map of the row's tiles for each query and the tiles that one names are numbered: order,
// tiles named twice and numbers that are no tiles do not matter.
// A product with a numerator of 0 is NaN where the value is an infinity or NaN.  So where the accumulators end up with any, which is rare, the work is done again query by
// query, each over its own tiles alone and with the values behind it cut off.  Finite values near the end of bf16's range get there too, their sums times 2^15; the reference
// follows the maximum then, so that weights end at 2^8 and what single queries hold is held here.
template <int KM, int VM, bool F16>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void listed_many_kernel(hs_listed_args g, hs_kv_dev kv, int n_queries, int n_splits, float scale_log2, float* __restrict__ ws_o, float* __restrict__ ws_l) {
  constexpr int NW = 4;
  extern __shared__ uint32_t sm_bits[];  // [n_queries][n_words]
  __shared__ __attribute__((aligned(16))) float sm_o[NW][16][HS_D];
  __shared__ float sm_m[NW][16], sm_l[NW][16];
  __shared__ uint32_t sm_list[kListCap];  // tile | queries << 16
  __shared__ int sm_cnt[NW];
  const int tid = threadIdx.x, l = tid & 63, a = l >> 4, c = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = g.Hq / g.Hkv, T = g.T, BH = g.B * g.Hkv, n_blocks = (g.Lq + n_queries - 1) / n_queries;
  int64_t n = blockIdx.x;
  const int row = (int)(n % BH);
  n /= BH;
  const int b = row / g.Hkv, h = row - b * g.Hkv;
  const int i0 = (int)(n % n_blocks) * n_queries, split = (int)(n / n_blocks), n_here = min(n_queries, g.Lq - i0);
  const int mine = c / G, head = c - mine * G;  // this column's query and head
  const bool valid = mine < n_here;
  uint4 qb[4];
  {
    const uint16_t* q = g.q.p + b * g.q.sb + ((int64_t)h * G + head) * g.q.sh + (i0 + (valid ? mine : 0)) * g.q.st + 8 * a;
#pragma unroll
    for (int s = 0; s < 4; s++) qb[s] = valid ? *reinterpret_cast<const uint4*>(q + 32 * s) : make_uint4(0, 0, 0, 0);
  }
  // the last token that query k of the block sees
  auto sees = [&](int k) -> int { return g.causal ? g.q_start + i0 + k : T * HS_BT - 1; };

  // ---- which tiles ----
  const int n_words = (T + 31) / 32, n_units = n_words * 4;  // a thread counts units of 8 tiles
  for (int i = tid; i < n_here * n_words; i += 64 * NW) sm_bits[i] = 0u;
  __syncthreads();
  {
    // the lists of neighbouring queries lie behind each other
    const int32_t* list = g.list + ((int64_t)row * g.Lq + i0) * g.n_list;
    const int64_t entries = (int64_t)n_here * g.n_list;
    for (int64_t i1 = tid; i1 < entries; i1 += 4 * 64 * NW) {
      int t[4];
#pragma unroll
      for (int j = 0; j < 4; j++) t[j] = i1 + j * 64 * NW < entries ? list[i1 + j * 64 * NW] : -1;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        if (t[j] < 0) continue;
        const int k = (int)((uint32_t)(i1 + j * 64 * NW) / (uint32_t)g.n_list);
        if (t[j] <= sees(k) / HS_BT) atomicOr(&sm_bits[k * n_words + (t[j] >> 5)], 1u << (t[j] & 31));
      }
    }
  }
  __syncthreads();
  // which of a unit's 8 tiles each query names, and which any does
  auto unit = [&](int u, uint32_t (&of)[16]) -> uint32_t {
    uint32_t any = 0u;
#pragma unroll
    for (int k = 0; k < 16; k++) {
      of[k] = k < n_here ? sm_bits[k * n_words + (u >> 2)] >> (8 * (u & 3)) & 0xffu : 0u;
      any |= of[k];
    }
    return any;
  };
  const int per = (n_units + 64 * NW - 1) / (64 * NW), u0 = min(n_units, tid * per), u1 = min(n_units, u0 + per);
  int count = 0;
  for (int u = u0; u < u1; u++) {
    uint32_t of[16];
    count += __builtin_popcount(unit(u, of));
  }
  const int upto = wave_upto(count);
  if (l == 63) sm_cnt[w] = upto;
  __syncthreads();
  int first = upto - count, n_all = 0;
#pragma unroll
  for (int k = 0; k < NW; k++) {
    if (k < w) first += sm_cnt[k];
    n_all += sm_cnt[k];
  }
  const int lo = (int)((int64_t)n_all * split / n_splits), hi = (int)((int64_t)n_all * (split + 1) / n_splits);

  // ---- their attention ----
  auto form_of = [](int mk, int mv) -> int { return (mk > 0 ? 1 : 0) | (mv > 0 ? 2 : 0) | ((!F16 && !hs_map_f16(mv)) ? 4 : 0); };
  f32x4_t o[8];
  float m_run, l_run;
  int alone = -1;  // the query that is done by itself; -1: all at once
  for (;;) {
#pragma unroll
    for (int i = 0; i < 8; i++) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m_run = -INFINITY;
    l_run = 0.f;
    const float slack = alone < 0 ? kSlack : 0.f;
    const uint32_t active = alone < 0 ? (1u << n_here) - 1u : 1u << alone;
    const int sees_first = sees(alone < 0 ? 0 : alone);  // the least of those
    for (int r0 = lo; r0 < hi; r0 += kListCap) {         // the same trips in every thread
      const int r1 = min(hi, r0 + kListCap);
      int number = first;
      for (int u = u0; u < u1 && number < r1; u++) {
        uint32_t of[16], any = unit(u, of);
        while (any != 0u && number < r1) {
          const int bit = __builtin_ctz(any);
          if (number >= r0) {
            uint32_t who = 0u;
#pragma unroll
            for (int k = 0; k < 16; k++) who |= (of[k] >> bit & 1u) << k;
            sm_list[number - r0] = (uint32_t)(8 * u + bit) | who << 16;
          }
          any &= any - 1;
          number++;
        }
      }
      __syncthreads();
      for (int base = w; base < r1 - r0; base += 64 * NW) {  // up to 64 tiles of this wave a round
        const int i_mine = base + NW * l;
        int mk_v = 0, mv_v = 0;
        uint32_t e_v = 0u;
        if (i_mine < r1 - r0) {
          e_v = sm_list[i_mine];
          mk_v = kv.k_map[(int64_t)row * T + (e_v & 0xffffu)];
          mv_v = kv.v_map[(int64_t)row * T + (e_v & 0xffffu)];
        }
        static_for_forms<KM, VM, F16, -1>([&](auto form_c) {
          constexpr int kForm = decltype(form_c)::value;
          constexpr int KK = kForm & 1, VK = (kForm >> 1) & 1, kEnc = (kForm & 4) ? 0 : 1;
          unsigned long long act = __ballot(mk_v != 0 && form_of(mk_v, mv_v) == kForm && (e_v >> 16 & active) != 0u);
          if (act == 0ull) return;
          TileRegs<KK, VK> tile;
          int mk, mv, e;
          auto next = [&]() {
            const int i = __builtin_ctzll(act);
            act &= act - 1;
            mk = __builtin_amdgcn_readlane(mk_v, i);
            mv = __builtin_amdgcn_readlane(mv_v, i);
            e = __builtin_amdgcn_readlane((int)e_v, i);
          };
          next();
          tile_load<KK, VK, 3, false>(tile, kv, row, mk, mv, l);
          for (bool more = true; more;) {
            const int t = e & 0xffff;
            const uint32_t who = (uint32_t)e >> 16 & active;
            const bool whole = who == active && sees_first - t * HS_BT >= HS_BT - 1;
            const int limit = (who >> mine & 1u) ? sees(mine) - t * HS_BT : -1;  // the last token of the tile that this column sees
            if (alone >= 0 && !whole) cut_values<KK, VK>(tile, sees_first - t * HS_BT, a);
            more = act != 0ull;
            if (more) next();
            tile_compute_many<KK, VK, F16, kEnc>(tile, qb, scale_log2, slack, o, m_run, l_run, [&](f32x4_t (&s)[4]) {
              if (more) tile_load<KK, VK, 1, false>(tile, kv, row, mk, mv, l);
              if (whole) return;
#pragma unroll
              for (int m = 0; m < 4; m++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                  if (16 * m + 4 * a + i > limit) s[m][i] = -INFINITY;
            });
            if (more) tile_load<KK, VK, 2, false>(tile, kv, row, mk, mv, l);
          }
        });
      }
      __syncthreads();  // the list is rewritten by the next pass
    }
    if (alone < 0) {
      float z = 0.f;  // 0, or NaN
#pragma unroll
      for (int i = 0; i < 8; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) z += o[i][j] * 0.f;
      if (__syncthreads_or(z != 0.f)) {
        alone = 0;
        continue;
      }
    }
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
    if (alone < 0 || mine == alone) {
      if (a == 0) { sm_m[w][c] = m_run; sm_l[w][c] = l_run; }
#pragma unroll
      for (int mb = 0; mb < 8; mb++)
        *reinterpret_cast<float4*>(&sm_o[w][c][16 * mb + 4 * a]) = make_float4(o[mb][0], o[mb][1], o[mb][2], o[mb][3]);
    }
    if (alone < 0) break;
    if (++alone == n_here) break;
  }

  // ---- join the waves: thread = (column tid / 16, 8 channels) ----
  __syncthreads();
  const int col = tid >> 4, ch = (tid & 15) * 8, of = col / G;
  if (of >= n_here) return;
  const int64_t hq = ((int64_t)b * g.Hq + h * G + (col - of * G)) * g.Lq + i0 + of;
  float mstar = -INFINITY;
#pragma unroll
  for (int k = 0; k < NW; k++) mstar = fmaxf(mstar, sm_m[k][col]);
  const float mref = mstar > -INFINITY ? mstar : 0.f;  // a part without one has seen nothing, or only NaN scores: neither is left out
  float lsum = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < NW; k++) {
    const float f = __builtin_amdgcn_exp2f(sm_m[k][col] - mref);
    lsum += f * sm_l[k][col];
#pragma unroll
    for (int i = 0; i < 8; i++) acc[i] += f * sm_o[k][col][ch + i];
  }
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
  const float lse = lsum == 0.f ? -INFINITY : (mstar + __builtin_amdgcn_logf(lsum)) * kLn2;
#pragma unroll
  for (int i = 0; i < 8; i++) acc[i] *= inv;
  if (n_splits == 1) {
    typedef hs_elem<F16> E;
    uint16_t* po = reinterpret_cast<uint16_t*>(ws_o) + hq * HS_D + ch;
    const bool aligned8 = ((uintptr_t)ws_o & 7) == 0;
    store4(po, E::pack2(acc[0], acc[1]), E::pack2(acc[2], acc[3]), aligned8);
    store4(po + 4, E::pack2(acc[4], acc[5]), E::pack2(acc[6], acc[7]), aligned8);
    if (ws_l != nullptr && ch == 0) ws_l[hq] = lse;
  } else {
    float* po = ws_o + (hq * n_splits + split) * HS_D + ch;
    *reinterpret_cast<float4*>(po) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    *reinterpret_cast<float4*>(po + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
    if (ch == 0) ws_l[hq * n_splits + split] = lse;
  }
}

template <int KM, int VM>
hipError_t launch_many(const hs_listed_args& a, const hs_kv_dev& kv, bool f16, hs_listed_plan p, float* wo, float* wl, hipStream_t st) {
  const int64_t blocks = ((int64_t)a.Lq + p.queries - 1) / p.queries;
  const dim3 grid((unsigned)((int64_t)a.B * a.Hkv * blocks * p.splits)), block(256);
  const size_t lds = (size_t)p.queries * ((a.T + 31) / 32) * 4;
  const float sl2 = a.scale * kLog2e;
  if (f16) hipLaunchKernelGGL((listed_many_kernel<KM, VM, true>), grid, block, lds, st, a, kv, p.queries, p.splits, sl2, wo, wl);
  else hipLaunchKernelGGL((listed_many_kernel<KM, VM, false>), grid, block, lds, st, a, kv, p.queries, p.splits, sl2, wo, wl);
  return hipGetLastError();
}

}  // namespace

hipError_t hs_launch_listed_many(int km, int vm, const hs_listed_args& a, const hs_kv_dev& kv, bool f16, hs_listed_plan p, float* wo, float* wl, hipStream_t st) {
  switch (km * 3 + vm) {
    case 0: return launch_many<0, 0>(a, kv, f16, p, wo, wl, st);
    case 1: return launch_many<0, 1>(a, kv, f16, p, wo, wl, st);
    case 2: return launch_many<0, 2>(a, kv, f16, p, wo, wl, st);
    case 3: return launch_many<1, 0>(a, kv, f16, p, wo, wl, st);
    case 4: return launch_many<1, 1>(a, kv, f16, p, wo, wl, st);
    case 5: return launch_many<1, 2>(a, kv, f16, p, wo, wl, st);
    case 6: return launch_many<2, 0>(a, kv, f16, p, wo, wl, st);
    case 7: return launch_many<2, 1>(a, kv, f16, p, wo, wl, st);
    default: return launch_many<2, 2>(a, kv, f16, p, wo, wl, st);
  }
}
