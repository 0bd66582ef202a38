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
// Neighbouring queries in one workgroup, over all tiles that one of them picks (hs_listed_many.hip), against one by one; 512 tiles a sequence, lists as perf/more_operators.py makes them (a
// quarter of a list differs from the neighbour's; four list 98 tiles of 64 each among them, two 80, sixteen 130), no tail.  One by one with 4 waves / with 8 (of 32 and 128 rows: of 4 in shares) / in company:
//   rows                           32                  128                 256                 260                 304                 384                 600                 2400
//   64 tiles, 4 heads   2:4        18.7  10.5  12.3    19.1  15.3  14.2    18.8  15.9  16.3    23.8  28.2  18.1    25.2  28.9  17.5    25.3  29.2  20.9    38.9  43.0  28.0    112  142  62
//                       dense      24.6  10.9  14.4    26.6  19.6  17.9    27.9  24.2  21.0    39.2  42.8  23.1    39.7  43.7  23.0    40.1  43.5  26.9    56.6  64.3  37.9    171  208  89
//   64 tiles, 1 head    2:4        19.1  10.3  12.1    20.1  15.9  14.2    20.2  15.8  14.4    24.1  28.4  14.7    25.4  28.8  15.3    25.4  29.1  15.7    38.6  42.5  17.2    110  139  35
//   64 tiles, 8 heads   2:4        17.9  10.8  12.6    18.4  15.1  15.1    19.3  16.5  19.0    23.9  28.3  24.2    25.2  28.9  23.5    25.5  29.5  24.1    39.5  43.3  32.8    116  145  80
//   16 tiles, 4 heads   2:4         8.5   8.8  11.6     8.6   9.9  12.4     8.7   8.3  12.4    10.1  13.6  12.8    10.9  14.4  12.9    11.0  14.5  13.9    16.3  20.9  14.3    43   66   28
//                       dense       9.3   8.9  12.9     9.5  10.2  13.2     9.5   9.5  13.5    13.1  16.7  14.6    13.4  17.1  14.5    13.6  17.2  15.7    19.7  25.0  17.6    51   80   36
//   16 tiles, 8 heads   2:4         8.5   9.0  11.5     8.5  10.3  12.2     8.7   8.5  13.2    10.2  13.8  12.2    11.0  14.9  12.4    11.1  15.0  12.4    16.5  21.8  15.7    44   69   38
// One border for all: long lists would share from about 128 rows on (260 of 64 tiles 23.8 one by one, 18.1 shared), short ones from about 500 (384 of 16 tiles 11.0, 13.9).
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
