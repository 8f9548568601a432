// Linear with 4-bit weights, group scales and zero points, on few rows.
#include "device_common.h"
#include "paged.h"

namespace sm {

// packed: the weights as they came [N, K / 2], the scales [N, K / group] bf16, the zero points [N, K / group] bytes
static size_t w4_part(size_t n) { return (n + 255) & ~(size_t)255; }
size_t w4_packed_bytes(int N, int K, int group) {
  return w4_part((size_t)N * K / 2) + w4_part((size_t)N * (K / group) * 2) + w4_part((size_t)N * (K / group));
}

__global__ __launch_bounds__(256) void w4_pack_kernel(const unsigned char* w, const bf16_t* s, const unsigned char* z, int64_t nw, int64_t ng,
                                                      unsigned char* pw, bf16_t* ps, unsigned char* pz) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < nw; i += (int64_t)gridDim.x * 256) {
    pw[i] = w[i];
    if (i < ng) { ps[i] = s[i]; pz[i] = z ? z[i] : 8; }
  }
}
int launch_w4_pack(const void* w, const void* scales, const void* zeros, int N, int K, int group, void* packed, void* stream) {
  const int64_t nw = (int64_t)N * K / 2, ng = (int64_t)N * (K / group);
  unsigned char* p = (unsigned char*)packed;
  w4_pack_kernel<<<dim3(1024), dim3(256), 0, (hipStream_t)stream>>>((const unsigned char*)w, (const bf16_t*)scales, (const unsigned char*)zeros, nw, ng, p,
      (bf16_t*)(p + w4_part(nw)), p + w4_part(nw) + w4_part(2 * ng));
  return (int)hipGetLastError();
}

// one wave per output
__global__ __launch_bounds__(64) void w4_kernel(LinearW4Args a) {
  const int n = blockIdx.x, m = blockIdx.y, lane = threadIdx.x;
  const unsigned char* w = (const unsigned char*)a.packed;
  const bf16_t* s = (const bf16_t*)(w + (((size_t)a.N * a.K / 2 + 255) & ~(size_t)255));
  const unsigned char* z = (const unsigned char*)s + (((size_t)a.N * (a.K / a.group) * 2 + 255) & ~(size_t)255);
  const bf16_t* x = (const bf16_t*)a.x + (int64_t)m * a.K;
  float acc = 0.f;
  for (int k = lane; k < a.K; k += 64) {
    const int64_t g = (int64_t)n * (a.K / a.group) + k / a.group;
    const int b = w[((int64_t)n * a.K + k) / 2], q = (k & 1) ? b >> 4 : b & 15;
    acc = fmaf((float)(q - z[g]) * bf2f(s[g]), bf2f(x[k]), acc);
  }
  acc = wave_sum(acc);
  if (lane == 0) {
    const int64_t at = (int64_t)m * a.N + n;
    if (a.bias) acc += bf2f(((const bf16_t*)a.bias)[n]);
    if (a.act) acc = gelu_erf(acc);
    if (a.residual) acc += bf2f(((const bf16_t*)a.residual)[at]);
    ((bf16_t*)a.y)[at] = f2bf(acc);
  }
}
int launch_w4(const LinearW4Args& a, void* stream) {
  w4_kernel<<<dim3(a.N, a.M), dim3(64), 0, (hipStream_t)stream>>>(a);
  return (int)hipGetLastError();
}

}  // namespace sm
