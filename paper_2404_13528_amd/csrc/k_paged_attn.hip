// Attention of one new token per request over a paged key / value cache: softmax(scale * q . K^T) V.
//
// Bound by the stream of K and V from HBM (4 d bytes and, with g query heads to a key head, 4 g d operations per token and key
// head in bf16).  Work is cut by the lengths that the device finds: all requests' tokens are divided into chunks of one
// length, such that about PA_ITEMS workgroups have one each, whatever the mix of short and long requests; every wave finds
// its workgroup's chunk with one scan over the lengths.  Chunks of a request are joined by a second, small kernel.
//
//  * A wave takes tiles of 32 (bf16) or 16 (fp32) keys straight from memory into registers, the next keys and values requested
//    as soon as the present ones are used up; there is no LDS on the way and no barrier in the loop.
//  * S^T = K Q^T on the matrix pipe: K is the first operand as it lies in memory, the up to 16 query heads of a key head are
//    the columns.  The result has four keys per lane, column = query: softmax statistics are sums over a lane's values and
//    two steps between lanes.
//  * O^T += V^T P^T: the lanes of P^T's columns hold just the keys that the product wants from them, if the same keys are
//    taken in the order 4 (lane / 16) + i; V^T's rows may be any features, and a lane's are the adjacent ones that a 16-byte
//    load brings.  bf16 pairs of two keys are put together with byte permutes in registers.
//  * P enters the bf16 product as two terms (its upper 8 bits and the rest, rounded): the matrix pipe is idle most of the
//    time, and the weights then carry 16 bits.  Running maximum, sums and O are fp32.
//  * Keys behind the length and pages outside the pool: their loads go to the pool's first place, their logits become -inf
//    and their values zero (a NaN there would survive a weight of zero).
#include <algorithm>
#include "device_common.h"
#include "paged.h"

namespace sm {

namespace {
typedef unsigned int pa_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int pa_u32x2 __attribute__((ext_vector_type(2)));
typedef float pa_f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 pa_bf16x8;

constexpr int PA_WAVES = 4;
constexpr int PA_ITEMS = 1024;            // workgroups that the work is cut for
constexpr int PA_CHUNK = 256;             // no chunk shorter than this
constexpr int PA_ROWS = 16;               // query heads a workgroup serves at once

struct PaShape { int rows, tiles, groups, items; };      // query heads per tile, tiles per key head, workgroups per chunk, chunks at most
PaShape pa_shape(int n_req, int heads_q, int heads_kv, int64_t max_keys) {
  PaShape s;
  const int g = heads_q / heads_kv;
  s.rows = std::min(g, PA_ROWS);
  s.tiles = (g + PA_ROWS - 1) / PA_ROWS;
  s.groups = heads_kv * s.tiles;
  const int64_t most = (int64_t)n_req * ((max_keys + PA_CHUNK - 1) / PA_CHUNK);
  s.items = (int)std::min<int64_t>(std::max(1, PA_ITEMS / s.groups) + n_req, most);
  return s;
}
// floats of a workgroup's partial result: [rows][d] sums, [rows][2] maximum and sum of the weights
__host__ __device__ constexpr int pa_record(int rows, int d) { return (rows * (d + 2) + 3) & ~3; }
constexpr size_t pa_align(size_t n) { return (n + 255) & ~(size_t)255; }

struct PaArgs { PagedAttnArgs a; int rows, tiles, groups, items; float scale_log2e; int2* plan; };

// The chunk of workgroup `item`: request, first key, one behind the last key, number of the request's chunks.
struct PaItem { int r, k0, k1, n; };
__device__ __forceinline__ int pa_len(const PagedAttnArgs& a, int r) { return min(max(a.lens[r], 0), a.max_pages * a.page); }
__device__ __forceinline__ PaItem pa_item(const PaArgs& p, const int item) {
  const int lane = threadIdx.x & 63, R = p.a.n_req, per = (R + 63) / 64;
  const int r0 = min(R, lane * per), r1 = min(R, r0 + per);
  int64_t total = 0;
  for (int r = r0; r < r1; ++r) total += pa_len(p.a, r);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
  const int64_t share = (total * p.groups + PA_ITEMS - 1) / PA_ITEMS;
  const int chunk = max(PA_CHUNK, (int)min((share + 127) & ~(int64_t)127, (int64_t)1 << 30));
  int mine = 0;
  for (int r = r0; r < r1; ++r) mine += max(1, (pa_len(p.a, r) + chunk - 1) / chunk);
  int end = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) { const int u = __shfl_up(end, o, 64); if (lane >= o) end += u; }
  PaItem it = {-1, 0, 0, 0};
  const uint64_t holds = __ballot(item < end);
  if (!holds) return it;
  const int src = __builtin_ctzll(holds);
  int first = __shfl(end - mine, src, 64), r = src * per;
  for (;; ++r) {                                       // (ends: the lane's requests have the item)
    const int len = pa_len(p.a, r), n = max(1, (len + chunk - 1) / chunk);
    if (item < first + n) {
      const int64_t k0 = (int64_t)(item - first) * chunk;
      it = {r, (int)k0, (int)min(k0 + chunk, (int64_t)len), n};
      break;
    }
    first += n;
  }
  it.r = __builtin_amdgcn_readfirstlane(it.r); it.k0 = __builtin_amdgcn_readfirstlane(it.k0);
  it.k1 = __builtin_amdgcn_readfirstlane(it.k1); it.n = __builtin_amdgcn_readfirstlane(it.n);
  return it;
}

template <typename T, int DP> struct PaTile {
  static constexpr int TK = sizeof(T) == 2 ? 32 : 16;      // keys
  static constexpr int NK = DP / 16;                        // 16-byte pieces of K a lane holds
  static constexpr int NV = TK / 4, EV = DP / 16;           // V: keys and adjacent features a lane holds
  static constexpr int VW = EV * (int)sizeof(T) / 4;        // words of V per key
  pa_u32x4 k[NK];
  unsigned v[NV][VW];
};
struct PaWhere { unsigned k, v; bool on; };                 // place of this lane's key of a tile in units of 16 bytes, and whether it is there
struct PaUnits { unsigned k_page, k_t, v_page, v_t; };      // strides of the pools in units of 16 bytes

// the place of a key whose page table entry is `id`; keys that are not there get the pool's first place
__device__ __forceinline__ PaWhere pa_where(const PagedAttnArgs& a, const PaUnits& u, int id, int key, int k1) {
  const unsigned in = (unsigned)key % (unsigned)a.page;
  PaWhere w;
  w.on = key < k1 && id >= 0 && id < a.n_pages;
  w.k = w.on ? (unsigned)id * u.k_page + in * u.k_t : 0;
  w.v = w.on ? (unsigned)id * u.v_page + in * u.v_t : 0;
  return w;
}

template <typename T, int DP, bool FULL>
__device__ __forceinline__ void pa_load_k(PaTile<T, DP>& t, const unsigned where, const char* kb, const int d) {
  typedef PaTile<T, DP> Tile;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  constexpr int SUB = Tile::TK / 16, STEPS = Tile::NK / SUB, E = 16 / (int)sizeof(T);
#pragma unroll
  for (int j = 0; j < SUB; ++j) {
    const char* p = kb + (uint64_t)__shfl(where, 16 * j + c, 64) * 16 + g * 16;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if (FULL || (s * 4 + g) * E < d) t.k[j * STEPS + s] = *(const pa_u32x4*)(p + s * 64);
      else t.k[j * STEPS + s] = pa_u32x4{0, 0, 0, 0};
    }
  }
}
template <typename T, int DP, bool FULL>
__device__ __forceinline__ void pa_load_v(PaTile<T, DP>& t, const unsigned where, const char* vb, const int d) {
  typedef PaTile<T, DP> Tile;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < Tile::NV; ++i) {
    const char* p = vb + (uint64_t)__shfl(where, 16 * (i / 4) + 4 * g + (i & 3), 64) * 16 + c * Tile::VW * 4;
    if constexpr (Tile::VW == 2) {
      pa_u32x2 x = {0, 0};
      if (FULL || c * Tile::EV < d) x = *(const pa_u32x2*)p;
      t.v[i][0] = x[0]; t.v[i][1] = x[1];
    } else {
#pragma unroll
      for (int u = 0; u < Tile::VW / 4; ++u) {
        pa_u32x4 x = {0, 0, 0, 0};
        if (FULL || c * Tile::EV + u * E < d) x = *(const pa_u32x4*)(p + u * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) t.v[i][4 * u + e] = x[e];
      }
    }
  }
}

__device__ __forceinline__ pa_f32x4 pa_mfma(pa_u32x4 a, pa_u32x4 b, pa_f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pa_bf16x8, a), __builtin_bit_cast(pa_bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ pa_f32x4 pa_mfma1(unsigned a, unsigned b, pa_f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a), __uint_as_float(b), c, 0, 0, 0);
}

// features e .. of query lane % 16
template <typename T>
__device__ __forceinline__ pa_u32x4 pa_query(const PagedAttnArgs& a, int r, int h0, int rows, int e) {
  const int c = threadIdx.x & 15;
  if (c >= rows || e >= a.d) return pa_u32x4{0, 0, 0, 0};
  return *(const pa_u32x4*)((const T*)a.q + (int64_t)r * a.q_r + (int64_t)(h0 + c) * a.q_h + e);
}
// logits of a tile, times log2 e: q(step) is the query operand; a lane gets keys 4 (lane / 16) + i (+ 16) of query lane % 16
template <typename T, int DP, typename Q>
__device__ __forceinline__ void pa_logits(const PaTile<T, DP>& t, const Q& q, const float scale, float* s) {
  typedef PaTile<T, DP> Tile;
  constexpr int SUB = Tile::TK / 16, STEPS = Tile::NK / SUB;
#pragma unroll
  for (int j = 0; j < SUB; ++j) {
    pa_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      if constexpr (sizeof(T) == 2) acc = pa_mfma(t.k[j * STEPS + i], q(i), acc);
      else {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = pa_mfma1(t.k[i][e], q(i)[e], acc);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[4 * j + i] = acc[i] * scale;
  }
}
// weights and values of a tile into the running maximum, sum and result; mask: the keys that are there (bit = key)
template <typename T, int DP>
__device__ __forceinline__ void pa_values(PaTile<T, DP>& t, float* s, const unsigned mask, float& m, float& l, pa_f32x4* o) {
  typedef PaTile<T, DP> Tile;
  constexpr int NV = Tile::NV;
  const int g = (threadIdx.x & 63) >> 4;
  constexpr unsigned ALL = Tile::TK == 32 ? 0xffffffffu : 0xffffu;
  if (mask != ALL) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (!((mask >> (16 * (i / 4) + 4 * g + (i & 3))) & 1)) {
        s[i] = -INFINITY;
#pragma unroll
        for (int e = 0; e < Tile::VW; ++e) t.v[i][e] = 0;
      }
    }
  }
  float mt = s[0];
#pragma unroll
  for (int i = 1; i < NV; ++i) mt = fmaxf(mt, s[i]);
  mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
  mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
  const float mn = fmaxf(m, mt), ref = mn == -INFINITY ? 0.f : mn;
  if (__any(mn > m)) {
    const float f = __builtin_amdgcn_exp2f(m - ref);                      // 0 where there was nothing
    l *= f;
#pragma unroll
    for (int n = 0; n < Tile::EV; ++n) o[n] *= f;
    m = mn;
  }
  float p[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) { p[i] = __builtin_amdgcn_exp2f(s[i] - ref); l += p[i]; }
  if constexpr (sizeof(T) == 2) {
    // the rest is never negative, and kept above zero, so that an infinite value keeps its sign: 0 x inf is no number
    pa_u32x4 hi;
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = fmaxf(p[i] - __uint_as_float(__float_as_uint(p[i]) & 0xffff0000u), 1e-37f);
#pragma unroll
    for (int e = 0; e < 4; ++e) hi[e] = __builtin_amdgcn_perm(__float_as_uint(p[2 * e + 1]), __float_as_uint(p[2 * e]), 0x07060302u);
    const pa_u32x4 lo = pack8(rest);
#pragma unroll
    for (int n = 0; n < Tile::EV; ++n) {
      pa_u32x4 vt;
#pragma unroll
      for (int e = 0; e < 4; ++e) vt[e] = __builtin_amdgcn_perm(t.v[2 * e + 1][n / 2], t.v[2 * e][n / 2], (n & 1) ? 0x07060302u : 0x05040100u);
      o[n] = pa_mfma(vt, hi, o[n]);
      o[n] = pa_mfma(vt, lo, o[n]);
    }
  } else {
#pragma unroll
    for (int n = 0; n < Tile::EV; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n] = pa_mfma1(t.v[i][n], __float_as_uint(p[i]), o[n]);
  }
}
}  // namespace

template <typename T, int DP, bool FULL>
__global__ __launch_bounds__(64 * PA_WAVES, DP == 64 ? 4 : DP == 128 ? 3 : 2) void paged_attn_kernel(PaArgs p) {
  typedef PaTile<T, DP> Tile;
  constexpr int TK = Tile::TK, STEPS = Tile::NK / (TK / 16), E = 16 / (int)sizeof(T);
  constexpr bool Q_LDS = DP == 256;                 // the widest head's query operand takes its registers' place in LDS, under the results
  __shared__ alignas(16) float s_o[PA_WAVES][PA_ROWS][DP];
  __shared__ float s_m[PA_WAVES][PA_ROWS], s_l[PA_WAVES][PA_ROWS];
  pa_u32x4* s_q = (pa_u32x4*)s_o;
  const PagedAttnArgs& a = p.a;
  const int grp = blockIdx.x % p.groups, item = blockIdx.x / p.groups;
  const PaItem it = pa_item(p, item);
  if (it.r < 0) return;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const int hk = grp / p.tiles, qt = grp - hk * p.tiles, per_kv = a.heads_q / a.heads_kv;
  const int h0 = hk * per_kv + qt * PA_ROWS, rows = min(PA_ROWS, per_kv - qt * PA_ROWS);
  const int* row = a.table + (int64_t)it.r * a.pitch;
  const PaUnits units = {(unsigned)(a.k_page / E), (unsigned)(a.k_t / E), (unsigned)(a.v_page / E), (unsigned)(a.v_t / E)};
  const char* kb = (const char*)((const T*)a.k + (int64_t)hk * a.k_h);
  const char* vb = (const char*)((const T*)a.v + (int64_t)hk * a.v_h);

  pa_u32x4 q[Q_LDS ? 1 : STEPS];
  if constexpr (Q_LDS) {
    for (int s = w; s < STEPS; s += PA_WAVES) s_q[s * 64 + lane] = pa_query<T>(a, it.r, h0, rows, (s * 4 + g) * E);
    __syncthreads();
  } else {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) q[s] = pa_query<T>(a, it.r, h0, rows, (s * 4 + g) * E);
  }
  pa_f32x4 o[Tile::EV];
#pragma unroll
  for (int n = 0; n < Tile::EV; ++n) o[n] = pa_f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  // The wave's tiles: w, w + PA_WAVES, ... of the chunk.  The next tile's keys are requested when the logits are done, its values when
  // the present ones are used up: one set of registers, and something is always on its way.  Loads return in the order of their
  // issue, so the page table entries are asked for a tile ahead of the loads that need them: waiting for them waits for nothing else.
  constexpr int STEP = TK * PA_WAVES;
  const int tiles = max(0, (it.k1 - it.k0 - w * TK + STEP - 1) / STEP);
  if (tiles > 0) {
    int key = it.k0 + w * TK + (lane & (TK - 1));
    Tile t;
    PaWhere at = pa_where(a, units, row[(unsigned)min(key, it.k1 - 1) / (unsigned)a.page], key, it.k1);
    int id = row[(unsigned)min(key + STEP, it.k1 - 1) / (unsigned)a.page];
    pa_load_k<T, DP, FULL>(t, at.k, kb, a.d);
    __builtin_amdgcn_sched_barrier(0);
    pa_load_v<T, DP, FULL>(t, at.v, vb, a.d);
#pragma unroll 1
    for (int i = 0; i < tiles; ++i) {
      const unsigned mask = (unsigned)__ballot(at.on) & (TK == 32 ? 0xffffffffu : 0xffffu);
      float s[Tile::NV];
      __builtin_amdgcn_sched_barrier(0);
      pa_logits<T, DP>(t, [&](int i) { return Q_LDS ? s_q[i * 64 + lane] : q[Q_LDS ? 0 : i]; }, p.scale_log2e, s);
      key += STEP;
      at = pa_where(a, units, id, key, it.k1);
      id = row[(unsigned)min(key + STEP, it.k1 - 1) / (unsigned)a.page];
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 < tiles) pa_load_k<T, DP, FULL>(t, at.k, kb, a.d);
      __builtin_amdgcn_sched_barrier(0);
      pa_values<T, DP>(t, s, mask, m, l, o);
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 < tiles) pa_load_v<T, DP, FULL>(t, at.v, vb, a.d);
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if constexpr (Q_LDS) __syncthreads();
  if (g == 0) { s_m[w][c] = m; s_l[w][c] = l; }
#pragma unroll
  for (int n = 0; n < Tile::EV; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s_o[w][c][(4 * g + i) * Tile::EV + n] = o[n][i];
  __syncthreads();
  float* part = a.part + ((int64_t)item * p.groups + grp) * pa_record(p.rows, a.d);
  if (grp == 0 && it.k0 == 0 && threadIdx.x == 0) p.plan[it.r] = make_int2(item, it.n);
  for (int x = threadIdx.x; x < rows * a.d; x += 64 * PA_WAVES) {
    const int r = x / a.d, e = x - r * a.d;
    float M = s_m[0][r];
#pragma unroll
    for (int i = 1; i < PA_WAVES; ++i) M = fmaxf(M, s_m[i][r]);
    const float ref = M == -INFINITY ? 0.f : M;
    float os = 0.f, ls = 0.f;
#pragma unroll
    for (int i = 0; i < PA_WAVES; ++i) {
      const float f = __builtin_amdgcn_exp2f(s_m[i][r] - ref);
      os = fmaf(f, s_o[i][r][e], os);
      ls = fmaf(f, s_l[i][r], ls);
    }
    if (it.n == 1) {
      Elem<T>::st((T*)a.o + (int64_t)it.r * a.o_r + (int64_t)(h0 + r) * a.o_h + e, M == -INFINITY ? 0.f : os / ls);
      if (a.lse && e == 0) a.lse[(int64_t)it.r * a.heads_q + h0 + r] = M == -INFINITY ? -INFINITY : (M + __builtin_amdgcn_logf(ls)) * 0.69314718055994531f;
    } else {
      part[r * a.d + e] = os;
      if (e == 0) { part[p.rows * a.d + 2 * r] = M; part[p.rows * a.d + 2 * r + 1] = ls; }
    }
  }
}

// Joins the chunks of a request's query head: a workgroup's threads are groups of d / 4 lanes, which take the chunks in turn.
template <typename T>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(PaArgs p) {
  __shared__ float s_o[256][4], s_m[256], s_l[256];
  const PagedAttnArgs& a = p.a;
  const int r = blockIdx.y, h = blockIdx.x;
  const int2 pl = p.plan[r];
  if (pl.y <= 1) return;
  const int per_kv = a.heads_q / a.heads_kv, hk = h / per_kv, hr = h - hk * per_kv, qt = hr / PA_ROWS, row = hr - qt * PA_ROWS;
  const int d4 = a.d / 4, lg = d4 <= 16 ? 16 : (d4 <= 32 ? 32 : 64), ng = 256 / lg, e = threadIdx.x & (lg - 1), grp = threadIdx.x / lg;
  const int64_t rec = (int64_t)p.groups * pa_record(p.rows, a.d);
  const float* base = a.part + ((int64_t)pl.x * p.groups + hk * p.tiles + qt) * pa_record(p.rows, a.d);
  float m = -INFINITY, l = 0.f;
  pa_f32x4 o = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 8;
  for (int i0 = grp; i0 < pl.y; i0 += ng * U) {
    float mi[U], li[U];
    pa_f32x4 oi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* q = base + (int64_t)min(i0 + u * ng, pl.y - 1) * rec;
      const float2 ml = *(const float2*)(q + p.rows * a.d + 2 * row);
      mi[u] = i0 + u * ng < pl.y ? ml.x : -INFINITY; li[u] = ml.y;
      oi[u] = e < d4 ? *(const pa_f32x4*)(q + row * a.d + 4 * e) : pa_f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < U; ++u) mn = fmaxf(mn, mi[u]);
    const float ref = mn == -INFINITY ? 0.f : mn, f = __builtin_amdgcn_exp2f(m - ref);
    o *= f; l *= f; m = mn;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * ng >= pl.y) continue;
      const float fu = __builtin_amdgcn_exp2f(mi[u] - ref);
      l = fmaf(fu, li[u], l);
#pragma unroll
      for (int x = 0; x < 4; ++x) o[x] = fmaf(fu, oi[u][x], o[x]);
    }
  }
  s_m[threadIdx.x] = m; s_l[threadIdx.x] = l;
#pragma unroll
  for (int x = 0; x < 4; ++x) s_o[threadIdx.x][x] = o[x];
  __syncthreads();
  if (grp || e >= d4) return;
  float M = -INFINITY, L = 0.f, O[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < ng; ++i) M = fmaxf(M, s_m[i * lg + e]);
  const float ref = M == -INFINITY ? 0.f : M;
  for (int i = 0; i < ng; ++i) {
    const float f = __builtin_amdgcn_exp2f(s_m[i * lg + e] - ref);
    L = fmaf(f, s_l[i * lg + e], L);
    for (int x = 0; x < 4; ++x) O[x] = fmaf(f, s_o[i * lg + e][x], O[x]);
  }
  T* out = (T*)a.o + (int64_t)r * a.o_r + (int64_t)h * a.o_h + 4 * e;
  for (int x = 0; x < 4; ++x) Elem<T>::st(out + x, M == -INFINITY ? 0.f : O[x] / L);
  if (a.lse && e == 0) a.lse[(int64_t)r * a.heads_q + h] = M == -INFINITY ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.69314718055994531f;
}

bool paged_attention_fits(int n_req, int heads_q, int heads_kv, int64_t max_keys) {
  const PaShape s = pa_shape(n_req, heads_q, heads_kv, max_keys);
  return (int64_t)s.items * s.groups < (1 << 24);      // a launch has less than 2^32 threads
}
size_t paged_attention_workspace(int, int n_req, int heads_q, int heads_kv, int d, int page, int max_pages) {
  const PaShape s = pa_shape(n_req, heads_q, heads_kv, (int64_t)page * max_pages);
  return pa_align((size_t)std::max(1, n_req) * sizeof(int2)) + pa_align((size_t)s.items * s.groups * pa_record(s.rows, d) * sizeof(float));
}

template <typename T, int DP, bool FULL>
static int pa_launch(const PaArgs& p, bool join, hipStream_t stream) {
  paged_attn_kernel<T, DP, FULL><<<dim3(p.items * p.groups), dim3(64 * PA_WAVES), 0, stream>>>(p);
  if (const int e = (int)hipGetLastError()) return e;
  if (join) paged_attn_join_kernel<T><<<dim3(p.a.heads_q, p.a.n_req), dim3(256), 0, stream>>>(p);
  return (int)hipGetLastError();
}
template <typename T>
static int pa_launch_d(const PaArgs& p, bool join, hipStream_t stream) {
  const int d = p.a.d;
  if (d == 64) return pa_launch<T, 64, true>(p, join, stream);
  if (d < 64) return pa_launch<T, 64, false>(p, join, stream);
  if (d == 128) return pa_launch<T, 128, true>(p, join, stream);
  if (d < 128) return pa_launch<T, 128, false>(p, join, stream);
  if (d == 256) return pa_launch<T, 256, true>(p, join, stream);
  return pa_launch<T, 256, false>(p, join, stream);
}

int launch_paged_attention(const PagedAttnArgs& a, int dtype, void* stream, int* launches) {
  const int64_t max_keys = (int64_t)a.page * a.max_pages;
  const PaShape s = pa_shape(a.n_req, a.heads_q, a.heads_kv, max_keys);
  PaArgs p{a, s.rows, s.tiles, s.groups, s.items, a.scale * 1.4426950408889634f, (int2*)a.part};
  p.a.part = (float*)((char*)a.part + pa_align((size_t)a.n_req * sizeof(int2)));
  const bool join = max_keys > PA_CHUNK;               // else no request has two chunks
  *launches = join ? 2 : 1;
  return dtype == 0 ? pa_launch_d<float>(p, join, (hipStream_t)stream) : pa_launch_d<bf16_t>(p, join, (hipStream_t)stream);
}

}  // namespace sm
