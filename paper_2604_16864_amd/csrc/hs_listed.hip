// Attention over listed tiles: how a call is shared out, and its kernels for tensors with one kind of tile.
#include "hs_listed_kernel.h"

// Shares, us a call, replayed from a graph, 4 heads a row, 2:4, with a tail (x8: of 8 waves):
//   8 rows, lists of 8      1: 8.7  2: 7.7  x8 1: 7.6          32 rows of 64   1: 27.3  4: 14.3  6: 13.6  8: 13.8  16: 14.8
//   8 rows of 32            1: 16.7  4: 10.1  8: 8.5  16: 8.0  64 rows of 64   1: 29.3  2: 20.1  4: 18.9  8: 20.0
//   8 rows of 256           8: 19.4  16: 14.9  32: 14.2        128 rows of 64  1: 34.2  2: 29.7  4: 30.8  x8 1: 31.8
//   256 rows of 64          1: 50.7  2: 52.6  x8 1: 49.9       128 rows of 16  1: 13.1  2: 13.6  x8 1: 12.4
//   512 rows of 32          1: 51.3  2: 56.8  x8 1: 52.7       384 rows of 16  1: 23.9  2: 28.8  x8 1: 26.7
// So: about as many workgroups as compute units, with a tile at least for each of their waves; one workgroup without a join where rows are many or lists short,
// of 8 waves while every one has a compute unit to itself.  The shares do not depend on the tiles' kinds: the workspace's size follows from them.
// A step of single tokens reads past the caches: what it reads comes again with the next step, when the other layers' have gone through them.  128 rows of 64 tiles, 151 MB
// that are not in the last-level cache: 30.7 us, through the caches 34.9; 512 rows 94 and 108.  Queries that stand side by side pick much the same tiles, and
// read through the caches: 65 of them with 41 tiles each on 4 rows 22.2 us, past them 29.9.
// 256 of them with 64 each on 8 rows 20.2 with 4 waves, 17.5 with 8.
// Neighbouring queries in one workgroup, over all tiles that one of them picks (hs_listed_many.hip), against one by one, lists that differ in a third of their tiles:
// 32 rows 11.9 and 9.9, 128 rows 15.3 and 13.9, 256 rows 19.2 and 20.4, 320 rows 15.2 and 16.1 (dense 18.4 and 22.4; 8 heads a row, two queries a workgroup, 17.8 and
// 16.7), 384 rows 20.6 and 25.9, 600 rows 25.7 and 38.6, 2400 rows 56.0 and 111.
hs_listed_plan hs_plan_listed(int B, int Hq, int Hkv, int T, int Lq, int n_list) {
  hs_listed_plan p{1, 4, 1};
  int64_t rows = (int64_t)B * Hkv * Lq;
  if (Lq > 1 && rows > 300) {
    // as many neighbours as columns and 24 KB of bit maps hold
    const int columns = 16 / (Hq / Hkv), maps = 6144 / ((T + 31) / 32);
    p.queries = columns < maps ? columns : maps;
    if (p.queries > Lq) p.queries = Lq;
    rows = (int64_t)B * Hkv * (((int64_t)Lq + p.queries - 1) / p.queries);
  } else if (rows > 128 || n_list <= 8 || (rows > 64 && n_list <= 32)) {
    if (rows <= 256) p.waves = 8;
    return p;
  }
  const int by_rows = rows > 256 ? 1 : (int)(256 / rows), by_tiles = n_list / 4 + (n_list % 4 != 0);
  p.splits = by_rows < by_tiles ? by_rows : by_tiles;
  return p;
}

hipError_t hs_launch_listed(const hs_listed_args& a, const hs_kv_dev& kv, int dtype, hipStream_t st) {
  const int km = kv.cap_dense_k == 0 ? 0 : (kv.cap_sparse_k == 0 ? 1 : 2);
  const int vm = kv.cap_dense_v == 0 ? 0 : (kv.cap_sparse_v == 0 ? 1 : 2);
  const bool f16 = dtype == HS_FP16;
  const hs_listed_plan p = hs_plan_listed(a.B, a.Hq, a.Hkv, a.T, a.Lq, a.n_list);
  const bool direct = p.splits == 1;
  const int n_parts = p.splits + (a.tail_len >= 0 ? 1 : 0);
  const int64_t rows = (int64_t)a.B * a.Hq * a.Lq;
  float* wo = direct ? reinterpret_cast<float*>(a.o) : a.ws;
  float* wl = direct ? a.lse : a.ws + (size_t)rows * n_parts * HS_D;
  hipError_t e = hipSuccess;
#define HS_GO(KM_, VM_) \
  e = kv.uniform ? launch_listed<KM_, VM_, true>(a, kv, f16, p, wo, wl, st) : launch_listed<KM_, VM_, false>(a, kv, f16, p, wo, wl, st)
  if (p.queries > 1) e = hs_launch_listed_many(km, vm, a, kv, f16, p, wo, wl, st);
  else if (km == 2 || vm == 2) e = hs_launch_listed_mixed(km, vm, a, kv, f16, p, wo, wl, st);
  else if (km == 0 && vm == 0) HS_GO(0, 0);
  else if (km == 0) HS_GO(0, 1);
  else if (vm == 0) HS_GO(1, 0);
  else HS_GO(1, 1);
#undef HS_GO
  if (e != hipSuccess || direct) return e;
  return hs_launch_merge(rows, n_parts, wo, wl, a.o, a.lse, st, dtype);
}
