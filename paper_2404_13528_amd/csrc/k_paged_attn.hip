// Attention of one new token per request over a paged key / value cache.
#include "device_common.h"
#include "paged.h"

namespace sm {

// One wave per (request, query head), one key at a time: lane l holds features l, l + 64, ...
template <typename T>
__global__ __launch_bounds__(64) void paged_attn_kernel(PagedAttnArgs a) {
  const int r = blockIdx.y, h = blockIdx.x, lane = threadIdx.x, hk = h / (a.heads_q / a.heads_kv);
  const int len = min(max(a.lens[r], 0), a.max_pages * a.page);
  const T* q = (const T*)a.q + r * a.q_r + h * a.q_h;
  float qf[4], acc[4], m = -INFINITY, l = 0.f;
  for (int e = 0; e < 4; ++e) { qf[e] = lane + 64 * e < a.d ? Elem<T>::ld(q + lane + 64 * e) : 0.f; acc[e] = 0.f; }
  for (int j = 0; j < len; ++j) {
    const int pg = j / a.page, in = j - pg * a.page, id = a.table[r * a.pitch + pg];
    if (id < 0 || id >= a.n_pages) continue;
    const T* k = (const T*)a.k + id * a.k_page + in * a.k_t + hk * a.k_h;
    const T* v = (const T*)a.v + id * a.v_page + in * a.v_t + hk * a.v_h;
    float s = 0.f;
    for (int e = 0; e < 4; ++e) if (lane + 64 * e < a.d) s = fmaf(qf[e], Elem<T>::ld(k + lane + 64 * e), s);
    s = wave_sum(s) * a.scale;
    const float mn = fmaxf(m, s), f = m == -INFINITY ? 0.f : expf(m - mn), p = expf(s - mn);
    m = mn; l = l * f + p;
    for (int e = 0; e < 4; ++e) if (lane + 64 * e < a.d) acc[e] = fmaf(p, Elem<T>::ld(v + lane + 64 * e), acc[e] * f);
  }
  T* o = (T*)a.o + r * a.o_r + h * a.o_h;
  for (int e = 0; e < 4; ++e) if (lane + 64 * e < a.d) Elem<T>::st(o + lane + 64 * e, m == -INFINITY ? 0.f : acc[e] / l);
  if (a.lse && lane == 0) a.lse[r * a.heads_q + h] = m == -INFINITY ? -INFINITY : m + logf(l);
}

size_t paged_attention_workspace(int, int, int, int, int, int, int) { return 256; }
int launch_paged_attention(const PagedAttnArgs& a, int dtype, void* stream, int* launches) {
  const dim3 grid(a.heads_q, a.n_req);
  if (dtype == 0) paged_attn_kernel<float><<<grid, dim3(64), 0, (hipStream_t)stream>>>(a);
  else paged_attn_kernel<bf16_t><<<grid, dim3(64), 0, (hipStream_t)stream>>>(a);
  *launches = 1;
  return (int)hipGetLastError();
}

}  // namespace sm
