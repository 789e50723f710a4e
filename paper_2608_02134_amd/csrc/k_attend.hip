// Attention of new tokens over the paged cache.
#include <algorithm>

#include "gmc_cache.h"
#include "gmc_device.h"

namespace gmc {

// One wave per query row and head, 64 keys at a time: lane j scores key j,
// then every lane adds the keys' value entries of its own columns.
template <typename T>
__global__ void __launch_bounds__(64) attend_row_kernel(CacheView c, AttendArgs a) {
  __shared__ float qs[256];
  const int i = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, h = hq / c.hg, lane = threadIdx.x;
  long long first;
  int n;
  new_rows(a.starts, a.max_new, a.rows, b, &first, &n);
  if (i >= n) return;
  const int len = cache_len(c, b);
  const int t = len - n + i;   // the row's own slot (negative: more rows than the cache holds)
  const T* q = static_cast<const T*>(a.q) + (first + i) * a.q_stride + hq * c.dh;
  for (int d = lane; d < c.dh; d += 64) qs[d] = to_f32(q[d]) * a.scale;
  __syncthreads();
  const T* kp = static_cast<const T*>(c.k);
  const T* vp = static_cast<const T*>(c.v);
  const int32_t* pos = c.slot_pos ? c.slot_pos + (static_cast<long long>(b) * c.hkv + h) * c.cap : nullptr;
  const int mine = t < 0 ? 0 : (pos ? pos[t] : t);
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 <= t; s0 += 64) {
    const int s = s0 + lane;
    long long row = s <= t ? cache_row(c, b, h, s) : -1;
    if (row >= 0 && a.window) {
      const int p = pos ? pos[s] : s;
      if (mine - p >= a.window && p >= a.sinks) row = -1;
    }
    float x = -INFINITY;
    if (row >= 0) {
      const T* k = kp + row * c.dh;
      x = 0.f;
      for (int d = 0; d < c.dh; ++d) x += qs[d] * to_f32(k[d]);
    }
    const float mn = fmaxf(m, wave_max(x));
    const float base = mn == -INFINITY ? 0.f : mn;
    const float p = row >= 0 ? expf(x - base) : 0.f;
    const float f = expf(m - base);
    l = l * f + wave_sum(p);
    for (int e = 0; e < 4; ++e) o[e] *= f;
    m = mn;
    for (int j = 0; j < 64; ++j) {
      const long long rj = __shfl(row, j);
      if (rj < 0) continue;
      const float pj = __shfl(p, j);
      for (int e = 0; e < 4; ++e)
        if (lane + 64 * e < c.dh) o[e] += pj * to_f32(vp[rj * c.dh + lane + 64 * e]);
    }
  }
  T* out = static_cast<T*>(a.out) + ((first + i) * c.hq + hq) * c.dh;
  for (int e = 0; e < 4; ++e)
    if (lane + 64 * e < c.dh) out[lane + 64 * e] = from_f32<T>(l == 0.f ? 0.f : o[e] / l);
  if (a.lse && lane == 0) a.lse[(first + i) * c.hq + hq] = l == 0.f ? -INFINITY : m + logf(l);
}

hipError_t launch_cache_attend(const CacheView& c, const AttendArgs& a, hipStream_t st) {
  const dim3 grid(a.max_new, c.hq, c.n_seq);
  if (c.dtype == 0)
    hipLaunchKernelGGL(attend_row_kernel<float>, grid, dim3(64), 0, st, c, a);
  else
    hipLaunchKernelGGL(attend_row_kernel<bf16_t>, grid, dim3(64), 0, st, c, a);
  return hipGetLastError();
}

}  // namespace gmc
