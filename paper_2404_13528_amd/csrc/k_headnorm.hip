// Norm of every query / key head, rotary embedding, and the store of queries, keys and values where the attention reads
// them (a page pool or plain rows), one pass over the fused projection's result.
//
// A head of d features lies over G lanes of 16 bytes; a wave takes 64 / G heads of one token at a time, and the workgroup's
// waves share the heads of a token.  An element's rotation partner is in the same wave, rot / 2 features away.
// Angles: position times theta_i / 2 pi as a fraction of 2^64, modulo one revolution, is an integer product, exact at any
// position; its upper 32 bits go to the sine and cosine (bf16: the hardware's, whose 1e-6 is far below the rounding of the
// store; fp32: the library's, in units of pi).
#include "device_common.h"
#include "paged.h"

namespace sm {

namespace {
typedef unsigned int hn_u32x4 __attribute__((ext_vector_type(4)));

template <typename T> __device__ __forceinline__ void hn_unpack(hn_u32x4 v, float* f);
template <> __device__ __forceinline__ void hn_unpack<float>(hn_u32x4 v, float* f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(v[e]);
}
template <> __device__ __forceinline__ void hn_unpack<bf16_t>(hn_u32x4 v, float* f) { unpack8(v, f); }
template <typename T> __device__ __forceinline__ hn_u32x4 hn_pack(const float* f);
template <> __device__ __forceinline__ hn_u32x4 hn_pack<float>(const float* f) {
  hn_u32x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(f[e]);
  return o;
}
template <> __device__ __forceinline__ hn_u32x4 hn_pack<bf16_t>(const float* f) { return pack8(f); }

template <typename T>
__device__ __forceinline__ void hn_sincos(uint64_t turn, unsigned pos, float* sn, float* cs) {
  const int rev = (int)(pos * (unsigned)(turn >> 32) + __umulhi(pos, (unsigned)turn));      // 2^32 to a revolution, -half .. half
  if constexpr (sizeof(T) == 4) sincospif((float)rev * 0x1p-31f, sn, cs);
  else { const float f = (float)rev * 0x1p-32f; *sn = __builtin_amdgcn_sinf(f); *cs = __builtin_amdgcn_cosf(f); }
}
}  // namespace

template <typename T, int G>
__global__ __launch_bounds__(256) void head_norm_rope_kernel(HeadNormArgs a_) {
  const SM_KARG HeadNormArgs* a = kernarg_ptr<HeadNormArgs>();
  constexpr int V = Elem<T>::VEC, HPW = 64 / G;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, t = blockIdx.x;
  const int pos = a->positions[t];
  if (pos < 0) return;
  const int e0 = (lane & (G - 1)) * V, sub = lane / G, half = a->rot / 2, d = a->d;
  const bool in = e0 < d, turns = e0 < a->rot, low = e0 < half;
  const int partner = low ? lane + half / V : lane - half / V;
  float sn[V], cs[V];
  if (turns) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      hn_sincos<T>(a->turn[(low ? e0 : e0 - half) + e], (unsigned)pos, &sn[e], &cs[e]);
      if (low) sn[e] = -sn[e];
    }
  }
  int64_t slot = t, page = 0;
  bool store = true;
  if (a->slots) {
    slot = a->slots[t];
    store = slot >= 0 && slot < a->n_slots;
    page = store ? (int)slot / a->page : 0;
    slot -= page * a->page;
  }
  int u = w;
  for (int p = 0; p < 3; ++p) {
    const SM_KARG HeadNormPart* q = &a->part[p];
    for (; u < q->units; u += 4) {
      const int h = u * HPW + sub;
      const bool on = in && h < q->heads;
      hn_u32x4 x = {0, 0, 0, 0};
      if (on) x = *(const hn_u32x4*)((const T*)q->x + t * q->x_t + h * q->x_h + e0);
      if (q->rotate) {
        float f[V];
        hn_unpack<T>(x, f);
        if (a->norm) {
          float mean = 0.f, sq = 0.f;
          if (a->norm == 1) {
#pragma unroll
            for (int e = 0; e < V; ++e) mean += f[e];
#pragma unroll
            for (int o = 1; o < G; o <<= 1) mean += __shfl_xor(mean, o, 64);
            mean /= d;
          }
#pragma unroll
          for (int e = 0; e < V; ++e) { f[e] = in ? f[e] - mean : 0.f; sq = fmaf(f[e], f[e], sq); }
#pragma unroll
          for (int o = 1; o < G; o <<= 1) sq += __shfl_xor(sq, o, 64);
          const float r = 1.f / sqrtf(sq / d + a->eps);
          float g[V], b[V];
          hn_u32x4 gv = {0, 0, 0, 0}, bv = {0, 0, 0, 0};
          if (in) gv = *(const hn_u32x4*)((const T*)q->gamma + e0);
          if (in && a->norm == 1) bv = *(const hn_u32x4*)((const T*)q->beta + e0);
          hn_unpack<T>(gv, g);
          hn_unpack<T>(bv, b);
#pragma unroll
          for (int e = 0; e < V; ++e) f[e] = fmaf(f[e] * r, g[e], b[e]);
        }
        if (half) {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float o = __shfl(f[e], partner & 63, 64);
            if (turns) f[e] = fmaf(o, sn[e], f[e] * cs[e]);
          }
        }
        x = hn_pack<T>(f);
      }
      const int64_t off = q->paged ? page * q->y_page + slot * q->y_t : t * q->y_t;
      if (on && (store || !q->paged)) *(hn_u32x4*)((T*)q->y + off + h * q->y_h + e0) = x;
    }
    u -= q->units;
  }
}

template <typename T>
static int launch_head_norm_t(HeadNormArgs& a, hipStream_t stream) {
  const int lanes = a.d / Elem<T>::VEC;
#define SM_HN(G) { for (auto& p : a.part) p.units = (p.heads + 64 / G - 1) / (64 / G); \
    head_norm_rope_kernel<T, G><<<dim3(a.tokens), dim3(256), 0, stream>>>(a); }
  if (lanes <= 8) SM_HN(8) else if (lanes <= 16) SM_HN(16) else if (lanes <= 32) SM_HN(32) else SM_HN(64)
#undef SM_HN
  return (int)hipGetLastError();
}
int launch_head_norm_rope(HeadNormArgs& a, int dtype, void* stream) {
  return dtype == 0 ? launch_head_norm_t<float>(a, (hipStream_t)stream) : launch_head_norm_t<bf16_t>(a, (hipStream_t)stream);
}

}  // namespace sm
