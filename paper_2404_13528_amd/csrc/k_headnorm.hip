// Norm of every query / key head, rotary embedding, and the store of queries, keys and values where the attention reads
// them (a page pool or plain rows), one pass over the fused projection's result.
//
// A lane has two 16-byte pieces of a head: below `rot` the two halves of its pairs, so that the rotation stays in the lane and an angle
// serves both, behind it two adjacent pieces.  G lanes make a head, a wave takes 64 / G heads of one token at a time.
// Angles: position times theta_i / 2 pi as a fraction of 2^64, modulo one revolution, is an integer product, which loses
// nothing at far positions; its upper 32 bits go to the sine and cosine as a float, off by at most 2^-26 of a revolution (bf16: the hardware's, whose 1e-6 is far below the rounding of the
// store; fp32: the library's, in units of pi).
// Bound by the bytes read and written.
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

// sum over groups of G adjacent lanes, in all of them
template <int G>
__device__ __forceinline__ float hn_sum(float v) {
#define HN_DPP(c) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), c, 0xf, 0xf, true))
  HN_DPP(0xb1);                                        // quad_perm 1 0 3 2
  HN_DPP(0x4e);                                        // quad_perm 2 3 0 1
  if (G >= 8) HN_DPP(0x141);                           // row_half_mirror: the other four of eight
  if (G >= 16) HN_DPP(0x128);                          // row_ror 8: the other eight of sixteen
#undef HN_DPP
  if (G >= 32) v += __shfl_xor(v, 16, 64);
  return v;
}

// WPT waves share a token.  A wave's heads (of q, then k, then v: `units` of 64 / G) are requested one unit ahead of the work; position,
// slot, gains and the first heads are all on their way at the same time.
template <typename T, int G, int WPT>
__global__ __launch_bounds__(256) void head_norm_rope_kernel(HeadNormArgs a_) {
  const SM_KARG HeadNormArgs* a = kernarg_ptr<HeadNormArgs>();
  constexpr int V = Elem<T>::VEC, HPW = 64 / G;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = WPT == 1 ? (int64_t)blockIdx.x * 4 + w : blockIdx.x;
  if (t >= a->tokens) return;
  const int l = lane & (G - 1), sub = lane / G, hv = a->rot / (2 * V), dv = a->d / V, norm = a->norm;
  const bool turns = l < hv;
  const int i0 = turns ? l : 2 * l, i1 = turns ? l + hv : i0 + 1;      // (behind rot: piece rot / V + 2 (l - hv) and the next)
  const bool on0 = i0 < dv, on1 = i1 < dv;
  const int n0 = a->part[0].units, n1 = n0 + a->part[1].units, n2 = n1 + a->part[2].units;
  auto load = [&](int u, hn_u32x4& x0, hn_u32x4& x1) {
    const int p = u < n0 ? 0 : u < n1 ? 1 : 2;
    const T* x = (const T*)(p == 0 ? a->part[0].x : p == 1 ? a->part[1].x : a->part[2].x);
    const int64_t xt = p == 0 ? a->part[0].x_t : p == 1 ? a->part[1].x_t : a->part[2].x_t, xh = p == 0 ? a->part[0].x_h : p == 1 ? a->part[1].x_h : a->part[2].x_h;
    const int heads = p == 0 ? a->part[0].heads : a->part[p].heads, h = (u - (p == 0 ? 0 : p == 1 ? n0 : n1)) * HPW + sub;
    x0 = x1 = hn_u32x4{0, 0, 0, 0};
    if (u < n2 && h < heads) {
      x += t * xt + h * xh;
      if (on0) x0 = *(const hn_u32x4*)(x + i0 * V);
      if (on1) x1 = *(const hn_u32x4*)(x + i1 * V);
    }
  };
  int u = WPT == 1 ? 0 : w;
  if (u >= n2) return;
  hn_u32x4 x0, x1, gain[2][2], shift[2][2];
  load(u, x0, x1);
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const T *g = (const T*)a->part[p].gamma, *b = (const T*)a->part[p].beta;
    gain[p][0] = gain[p][1] = shift[p][0] = shift[p][1] = hn_u32x4{0, 0, 0, 0};
    if (norm && a->part[p].units) {
      if (on0) gain[p][0] = *(const hn_u32x4*)(g + i0 * V);
      if (on1) gain[p][1] = *(const hn_u32x4*)(g + i1 * V);
      if (norm == 1 && on0) shift[p][0] = *(const hn_u32x4*)(b + i0 * V);
      if (norm == 1 && on1) shift[p][1] = *(const hn_u32x4*)(b + i1 * V);
    }
  }
  const int pos = a->positions[t];
  const int slot = a->slots ? a->slots[t] : 0;
  if (pos < 0) return;
  const bool store = !a->slots || (slot >= 0 && slot < a->n_slots);
  const int page = a->slots && store ? slot / a->page : 0;
  const int64_t row = a->slots ? slot - page * a->page : t;
  float sn[V], cs[V];
#pragma unroll
  for (int e = 0; e < V; ++e) { sn[e] = 0.f; cs[e] = 1.f; }
  if (turns) {
#pragma unroll
    for (int e = 0; e < V; ++e) hn_sincos<T>(a->turn[l * V + e], (unsigned)pos, &sn[e], &cs[e]);
  }
  const float inv_d = 1.f / a->d, eps = a->eps;
  auto work = [&](const hn_u32x4 (&gv)[2], const hn_u32x4 (&bv)[2]) {
    float f0[V], f1[V];
    hn_unpack<T>(x0, f0);
    hn_unpack<T>(x1, f1);
    if (norm) {
      float sq = 0.f, g0[V], g1[V], b0[V], b1[V];
      if (norm == 1) {
        float mean = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) mean += f0[e] + f1[e];
        mean = hn_sum<G>(mean) * inv_d;
#pragma unroll
        for (int e = 0; e < V; ++e) { f0[e] = on0 ? f0[e] - mean : 0.f; f1[e] = on1 ? f1[e] - mean : 0.f; }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) { sq = fmaf(f0[e], f0[e], sq); sq = fmaf(f1[e], f1[e], sq); }
      const float r = rsqrtf(fmaf(hn_sum<G>(sq), inv_d, eps));
      hn_unpack<T>(gv[0], g0);
      hn_unpack<T>(gv[1], g1);
      hn_unpack<T>(bv[0], b0);
      hn_unpack<T>(bv[1], b1);
#pragma unroll
      for (int e = 0; e < V; ++e) { f0[e] = fmaf(f0[e] * r, g0[e], b0[e]); f1[e] = fmaf(f1[e] * r, g1[e], b1[e]); }
    }
    if (turns) {                               // (the others' two pieces are no pair: an infinity in one would be a NaN in the other)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float lo = f0[e], hi = f1[e];
        f0[e] = fmaf(-hi, sn[e], lo * cs[e]);
        f1[e] = fmaf(lo, sn[e], hi * cs[e]);
      }
    }
    x0 = hn_pack<T>(f0);
    x1 = hn_pack<T>(f1);
  };
  for (; u < n2; u += WPT) {
    hn_u32x4 y0, y1;
    load(u + WPT, y0, y1);
    const int p = u < n0 ? 0 : u < n1 ? 1 : 2, h = (u - (p == 0 ? 0 : p == 1 ? n0 : n1)) * HPW + sub;
    if (p == 0) work(gain[0], shift[0]);
    else if (p == 1) work(gain[1], shift[1]);
    const SM_KARG HeadNormPart* q = &a->part[p];
    if (h < q->heads && (store || !q->paged)) {
      T* y = (T*)q->y + h * q->y_h + (q->paged ? page * q->y_page + row * q->y_t : t * q->y_t);
      // (a long prompt's result is larger than the L2 when its reader starts)
      auto put = [](T* at, hn_u32x4 v) { if (WPT == 1) __builtin_nontemporal_store(v, (hn_u32x4*)at); else *(hn_u32x4*)at = v; };
      if (on0) put(y + i0 * V, x0);
      if (on1) put(y + i1 * V, x1);
    }
    x0 = y0;
    x1 = y1;
  }
}

// Few tokens: four waves share one (8 tokens of 32 + 8 + 8 heads of 128: 4.7 us instead of 7.9; 512 tokens: 7.3 instead of 9.5).  Once there is
// a token for most of the 1024 SIMDs, one wave has all heads of a token and the angles are computed once (768 tokens: 9.6 us instead of 8.3;
// 1024: 9.8 instead of 11.2; 16411: 81 instead of 122, 5.0 TB/s read and written).  Calls in a replayed graph.
template <typename T, int G>
static void launch_head_norm_g(HeadNormArgs& a, hipStream_t stream) {
  for (auto& p : a.part) p.units = (p.heads + 64 / G - 1) / (64 / G);
  if (a.tokens < 768) head_norm_rope_kernel<T, G, 4><<<dim3(a.tokens), dim3(256), 0, stream>>>(a);
  else head_norm_rope_kernel<T, G, 1><<<dim3((a.tokens + 3) / 4), dim3(256), 0, stream>>>(a);
}
template <typename T>
static int launch_head_norm_t(HeadNormArgs& a, hipStream_t stream) {
  const int lanes = (a.d / Elem<T>::VEC + 1) / 2;
  if (lanes <= 4) launch_head_norm_g<T, 4>(a, stream);
  else if (lanes <= 8) launch_head_norm_g<T, 8>(a, stream);
  else if (lanes <= 16) launch_head_norm_g<T, 16>(a, stream);
  else launch_head_norm_g<T, 32>(a, stream);
  return (int)hipGetLastError();
}
int launch_head_norm_rope(HeadNormArgs& a, int dtype, void* stream) {
  return dtype == 0 ? launch_head_norm_t<float>(a, (hipStream_t)stream) : launch_head_norm_t<bf16_t>(a, (hipStream_t)stream);
}

}  // namespace sm
