// Choice of the tokens that go into a cache: per (batch, kv head) row the first, the last and of the others those of largest weight, in
// order of position.  One workgroup per row finds them; then their keys and values are gathered.
#include "hs_common.h"
#include "hs_rank.h"

namespace {

template <int NT>
__global__ __launch_bounds__(NT) void keep_select_kernel(int Hkv, int n, const float* __restrict__ weight, int64_t w_sb, int64_t w_sh, const int32_t* __restrict__ lens,
                                                         int keep, int first, int last, int32_t* __restrict__ index) {
  __shared__ int hist[260], sm[NT / 64];
  const int tid = threadIdx.x;
  const int b = blockIdx.x / Hkv, h = blockIdx.x % Hkv;
  weight += b * w_sb + h * w_sh;
  index += (int64_t)blockIdx.x * keep;
  const int len = lens != nullptr ? min(max(lens[b], 0), n) : n;
  if (len <= keep) {
    for (int i = tid; i < keep; i += NT) index[i] = i < len ? i : -1;
    return;
  }
  const int lo = first, hi = len - last, want = keep - first - last;  // first + last <= keep < len
  Threshold th{0, 0};
  if (want > 0)  // the largest by the complement of their keys
    th = smallest<NT>(lo, hi, want, [&](int t, uint32_t& key) -> bool { key = ~rank_key(weight[t]); return true; }, hist);
  int tie = 0, at = 0;
  for (int t0 = 0; t0 < len; t0 += NT) {
    const int t = t0 + tid;
    const bool cand = want > 0 && t >= lo && t < hi;
    const uint32_t key = cand ? ~rank_key(weight[t]) : 0xffffffffu;
    const int number = number_of<NT>(cand && key == th.key, tie, sm);
    const bool take = t < len && (t < lo || t >= hi || (cand && (key < th.key || (key == th.key && number < th.ties))));
    const int place = number_of<NT>(take, at, sm);
    if (take) index[place] = t;
  }
}

// 16 lanes a vector, 16 output rows a workgroup
__global__ __launch_bounds__(256) void keep_gather_kernel(int Hkv, int keep, hs_vec_view K, hs_vec_view V, const int32_t* __restrict__ index, uint16_t* __restrict__ K_out,
                                                          uint16_t* __restrict__ V_out) {
  const int row = blockIdx.y, b = row / Hkv, h = row % Hkv, c = threadIdx.x & 15;
  const int i = blockIdx.x * 16 + (threadIdx.x >> 4);
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

hipError_t hs_launch_keep(int B, int Hkv, int n, hs_vec_view K, hs_vec_view V, const float* weight, int64_t w_sb, int64_t w_sh, const int32_t* lens,
                          int keep, int first, int last, uint16_t* K_out, uint16_t* V_out, int32_t* index, hipStream_t st) {
  const int rows = B * Hkv;
  if (n <= 1024)
    hipLaunchKernelGGL((keep_select_kernel<256>), dim3(rows), dim3(256), 0, st, Hkv, n, weight, w_sb, w_sh, lens, keep, first, last, index);
  else
    hipLaunchKernelGGL((keep_select_kernel<1024>), dim3(rows), dim3(1024), 0, st, Hkv, n, weight, w_sb, w_sh, lens, keep, first, last, index);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(keep_gather_kernel, dim3((keep + 15) / 16, rows), dim3(256), 0, st, Hkv, keep, K, V, index, K_out, V_out);
  return hipGetLastError();
}
