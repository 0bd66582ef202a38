// Attention over listed tiles: its kernels for tensors with both kinds of tile.
#include "hs_listed_kernel.h"

hipError_t hs_launch_listed_mixed(int km, int vm, const hs_listed_args& a, const hs_kv_dev& kv, bool f16, hs_listed_plan p, float* wo, float* wl, hipStream_t st) {
  if (km == 2 && vm == 2) return launch_listed<2, 2, false>(a, kv, f16, p, wo, wl, st);
  if (km == 2) return vm == 0 ? launch_listed<2, 0, false>(a, kv, f16, p, wo, wl, st) : launch_listed<2, 1, false>(a, kv, f16, p, wo, wl, st);
  return km == 0 ? launch_listed<0, 2, false>(a, kv, f16, p, wo, wl, st) : launch_listed<1, 2, false>(a, kv, f16, p, wo, wl, st);
}
