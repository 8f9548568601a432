// Attention of one new token per request over a paged key / value cache: softmax(scale * q . K^T) V.
//
// Bound by the stream of K and V from HBM (4 d bytes and, with g query heads to a key head, 4 g d operations per token and key
// head in bf16).  Work is cut by the lengths that the device finds: all requests' tokens are divided into chunks of one
// length, such that a workgroup has one, whatever the mix of short and long requests; every wave finds its workgroup's chunk
// with two scans over the lengths.  Chunks of a request are joined by a second, small kernel.
//
//  * A wave takes tiles of 32 (bf16) or 16 (fp32) keys straight from memory into registers, the next keys and values requested
//    as soon as the present ones are used up; there is no LDS on the way and no barrier in the loop.
//  * S^T = K Q^T on the matrix pipe: K is the first operand as it lies in memory, the up to 16 query heads of a key head are
//    the columns.  The result has four keys per lane, column = query: softmax statistics are sums over a lane's values and
//    two steps between lanes.
//  * O^T += V^T P^T: the lanes of P^T's columns hold just the keys that the product wants from them, if the same keys are
//    taken in the order 4 (lane / 16) + i; V^T's rows may be any features, and a lane's are the adjacent ones that a 16-byte
//    load brings.  bf16 pairs of two keys are put together with byte permutes in registers.
//  * P enters the bf16 product as three terms of 8 bits each, so that the weights stay fp32: the matrix pipe is idle most of the
//    time, and two terms (16 bits) are no faster.  Running maximum, sums and O are fp32.
//  * Keys behind the length and pages outside the pool: their loads go to the pool's first place, their logits become -inf
//    and their values zero (a NaN there would survive a weight of zero).
//  * No key with a weight: the sum of the weights is zero (with one it is at least 1), not only the maximum -inf, which it also is if every
//    logit is NaN, as fmax passes over them; then the sum is NaN, and so is the result.
#include <algorithm>
#include "device_common.h"
#include "paged.h"

namespace sm {

namespace {
typedef unsigned int pa_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int pa_u32x2 __attribute__((ext_vector_type(2)));
typedef float pa_f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 pa_bf16x8;

constexpr int PA_ROWS = 16;               // query heads a workgroup serves at once
constexpr int PA_UNIT = 128;              // keys: chunks are whole units
// The weights go to their product with the values as multiples of this, so that a sum of 2^20 values of any finite size is finite.  Every wave and
// chunk sums by its own maximum: without it large values of keys that weigh nothing beside another chunk's would be infinite there.  The
// smallest number a sum can hold becomes 2^-129, an eighth of the smallest normal one.
constexpr float PA_LOW = 0x1p-20f;

// How the work is cut.  A chunk's start costs some 4 us (lengths, page table, first keys: three trips to memory), so at first there are as
// many chunks as two workgroups a CU (heads over 128: one): 64 requests of 1000 keys take 53 us, with twice as many chunks 59.  But where
// that makes a chunk longer than 512 KB of keys and values, up to 4096 shorter ones balance the load better than they cost (64 requests of
// 100 to 30000 keys, attention and join: 270 us instead of 313).  A table wider than its requests has more workgroups that end at once: one request
// of 150 keys takes 7.4 us under a table of 160 tokens, 9.6 under one of 8192 and 10.2 under one of 131072.
constexpr int PA_MANY_LOG2 = 12;
struct PaShape {
  int rows, tiles, groups;                // query heads per tile, tiles per key head, workgroups per chunk
  int fill_log2, cap, least;              // workgroups at first, units of a long and of the shortest chunk
  int items;                              // chunks at most
};
PaShape pa_shape(int dtype, int n_req, int heads_q, int heads_kv, int d, int64_t max_keys) {
  PaShape s;
  const int g = heads_q / heads_kv;
  s.rows = std::min(g, PA_ROWS);
  s.tiles = (g + PA_ROWS - 1) / PA_ROWS;
  s.groups = heads_kv * s.tiles;
  s.fill_log2 = d > 128 ? 8 : 9;
  s.cap = std::max(1, (512 << 10) / (2 * d * (dtype == 0 ? 4 : 2) * PA_UNIT));
  s.least = max_keys <= 2 * PA_UNIT ? 2 : 1;          // (256 keys are one workgroup's, without a join)
  const int64_t units = (max_keys + PA_UNIT - 1) / PA_UNIT, share = (n_req * units * s.groups + (1 << s.fill_log2) - 1) >> s.fill_log2;
  const int64_t most = n_req * ((units + s.least - 1) / s.least);
  s.items = (int)std::min<int64_t>(((1 << (share <= s.cap ? s.fill_log2 : PA_MANY_LOG2)) / s.groups) + n_req, most);
  return s;
}
// floats of a workgroup's partial result: [rows][d] sums, [rows][2] maximum and sum of the weights
__host__ __device__ constexpr int pa_record(int rows, int d) { return (rows * (d + 2) + 3) & ~3; }
constexpr size_t pa_align(size_t n) { return (n + 255) & ~(size_t)255; }

struct PaArgs { PagedAttnArgs a; PaShape s; float scale_log2e; int2* plan; };

// sum over the lanes up to and including this one
__device__ __forceinline__ unsigned pa_scan(unsigned x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8: within rows of 16 lanes
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // row_bcast 15, 31: the rows before
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// The chunk of workgroup `item`: request (-1: none), first key, one behind the last key, number of the request's chunks.
// A lane has `per` requests.  Every workgroup reads all lengths, those past the fourth of a lane twice more: from some 500 requests on that takes longer
// than the keys of short ones (requests of 100 keys with 32 heads over 8: 34 us for 256, 240 for 1024, 2300 for 4096).
//  With U units in all, `share` = U groups / 2^fill units would make 2^fill workgroups; every request has at least one
// chunk, so chunks of at least that length are at most 2^fill / groups + n_req.
struct PaItem { int r, k0, k1, n; };
__device__ __forceinline__ int pa_len(const PagedAttnArgs& a, int r) { return min(max(a.lens[r], 0), a.max_pages * a.page); }
__device__ __forceinline__ unsigned pa_chunks(int len, unsigned chunk) { return max(1u, ((unsigned)(len + PA_UNIT - 1) / PA_UNIT + chunk - 1) / chunk); }
__device__ __forceinline__ PaItem pa_item(const PaArgs& p, const unsigned item) {
  const int lane = threadIdx.x & 63, R = p.a.n_req, per = (R + 63) / 64;
  const int r0 = min(R, lane * per), r1 = min(R, r0 + per);
  constexpr int KEEP = 4;                              // lengths of a lane that stay in registers: all, up to 256 requests
  int len[KEEP];
  unsigned mine = 0;
#pragma unroll
  for (int j = 0; j < KEEP; ++j) len[j] = pa_len(p.a, min(r0 + j, R - 1));      // (no branch: the loads go out together)
#pragma unroll
  for (int j = 0; j < KEEP; ++j) len[j] = r0 + j < r1 ? len[j] : 0;
#pragma unroll
  for (int j = 0; j < KEEP; ++j) mine += (unsigned)(len[j] + PA_UNIT - 1) / PA_UNIT;
  for (int r = r0 + KEEP; r < r1; ++r) mine += (unsigned)(pa_len(p.a, r) + PA_UNIT - 1) / PA_UNIT;
  // (a lane's units fit 32 bits, their sum over the lanes is taken in two halves)
  const uint64_t units = (uint64_t)__builtin_amdgcn_readlane(pa_scan(mine & 0xffffu), 63) + ((uint64_t)__builtin_amdgcn_readlane(pa_scan(mine >> 16), 63) << 16);
  const uint64_t total = units * (unsigned)p.s.groups;
  const uint64_t share = (total + (1u << p.s.fill_log2) - 1) >> p.s.fill_log2, many = (total + (1u << PA_MANY_LOG2) - 1) >> PA_MANY_LOG2;
  const uint64_t want = share <= (uint64_t)p.s.cap ? share : max((uint64_t)p.s.cap, many);
  const unsigned chunk = max((unsigned)p.s.least, (unsigned)min(want, (uint64_t)1 << 23));
  mine = 0;
#pragma unroll
  for (int j = 0; j < KEEP; ++j) mine += r0 + j < r1 ? pa_chunks(len[j], chunk) : 0;
  for (int r = r0 + KEEP; r < r1; ++r) mine += pa_chunks(pa_len(p.a, r), chunk);
  const unsigned end = pa_scan(mine);
  PaItem it = {-1, 0, 0, 0};
  const uint64_t holds = __ballot(item < end);
  if (!holds) return it;
  const int src = __builtin_ctzll(holds);
  unsigned first = __builtin_amdgcn_readlane(end, src) - __builtin_amdgcn_readlane(mine, src);
  int r = src * per, l = 0;
  unsigned n = 0;
  for (int j = 0;; ++j) {                              // (ends: the lane's requests have the item)
    l = j == 0 ? __builtin_amdgcn_readlane(len[0], src) : j == 1 ? __builtin_amdgcn_readlane(len[1], src) : j == 2 ? __builtin_amdgcn_readlane(len[2], src) :
        j == 3 ? __builtin_amdgcn_readlane(len[3], src) : pa_len(p.a, r + j);
    n = pa_chunks(l, chunk);
    if (item < first + n) { r += j; break; }
    first += n;
  }
  const int64_t k0 = (int64_t)(item - first) * chunk * PA_UNIT;
  it = {r, (int)k0, (int)min(k0 + (int64_t)chunk * PA_UNIT, (int64_t)l), (int)n};
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

// A load of K takes 128 bytes of 8 keys, whole lines of memory (64 bytes of 16 keys, as the product wants them, would ask for every line
// twice); two of them become two operands when lanes 8 .. 15 of a row of lanes change places with lanes 0 .. 7 of the other (pa_order_k).
template <typename T, int DP, bool FULL>
__device__ __forceinline__ void pa_load_k(PaTile<T, DP>& t, const unsigned where, const char* kb, const int d) {
  typedef PaTile<T, DP> Tile;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, piece = (c >> 3) * 4 + g;
  constexpr int SUB = Tile::TK / 16, STEPS = Tile::NK / SUB, E = 16 / (int)sizeof(T);
#pragma unroll
  for (int j = 0; j < SUB; ++j) {
    const char* pa = kb + (uint64_t)__shfl(where, 16 * j + (c & 7), 64) * 16 + piece * 16;
    const char* pb = kb + (uint64_t)__shfl(where, 16 * j + (c & 7) + 8, 64) * 16 + piece * 16;
#pragma unroll
    for (int s = 0; s < STEPS; s += 2) {
      t.k[j * STEPS + s] = t.k[j * STEPS + s + 1] = pa_u32x4{0, 0, 0, 0};
      if (FULL || (s * 4 + piece) * E < d) {
        t.k[j * STEPS + s] = *(const pa_u32x4*)(pa + s * 64);
        t.k[j * STEPS + s + 1] = *(const pa_u32x4*)(pb + s * 64);
      }
    }
  }
}
template <typename T, int DP>
__device__ __forceinline__ void pa_order_k(PaTile<T, DP>& t) {
#pragma unroll
  for (int i = 0; i < PaTile<T, DP>::NK; i += 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int a = t.k[i][e], b = t.k[i + 1][e];
      t.k[i][e] = __builtin_amdgcn_update_dpp(a, b, 0x128, 0xf, 0xc, false);          // row_ror 8
      t.k[i + 1][e] = __builtin_amdgcn_update_dpp(b, a, 0x128, 0xf, 0x3, false);
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
    // A term is the upper 8 bits of what is left of the weight.  All three are above zero wherever the weight is (down to 2^-67), so that an infinite
    // value keeps its sign: 0 x inf is no number.  That takes a factor of 1 + 2^-23 on all weights alike and one of 1 + 2^-16 on the part below
    // 2^-7 of one, so a weight is off by at most 2^-22.  (With a step more per term two registers spill: 64 requests of 100 to 30000 keys take
    // 282 us instead of 270, as with two terms.)
    pa_u32x4 term[3];
    float left[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] *= PA_LOW;
      left[i] = fmaf(p[i], 1.f + 0x1p-23f, -__uint_as_float(__float_as_uint(p[i]) & 0xffff0000u));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) term[0][e] = __builtin_amdgcn_perm(__float_as_uint(p[2 * e + 1]), __float_as_uint(p[2 * e]), 0x07060302u);
#pragma unroll
    for (int e = 0; e < 4; ++e) term[1][e] = __builtin_amdgcn_perm(__float_as_uint(left[2 * e + 1]), __float_as_uint(left[2 * e]), 0x07060302u);
#pragma unroll
    for (int i = 0; i < 8; ++i) left[i] = fmaf(left[i], 1.f + 0x1p-16f, -__uint_as_float(__float_as_uint(left[i]) & 0xffff0000u));
    term[2] = pack8(left);
#pragma unroll
    for (int n = 0; n < Tile::EV; ++n) {
      pa_u32x4 vt;
#pragma unroll
      for (int e = 0; e < 4; ++e) vt[e] = __builtin_amdgcn_perm(t.v[2 * e + 1][n / 2], t.v[2 * e][n / 2], (n & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int u = 0; u < 3; ++u) o[n] = pa_mfma(vt, term[u], o[n]);
    }
  } else {
#pragma unroll
    for (int n = 0; n < Tile::EV; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n] = pa_mfma1(t.v[i][n], __float_as_uint(p[i] * PA_LOW), o[n]);
  }
}
}  // namespace

template <typename T, int DP, bool FULL, int PA_WAVES>
__global__ __launch_bounds__(64 * PA_WAVES, DP == 64 ? 4 : DP == 128 && PA_WAVES == 4 ? 3 : 2) void paged_attn_kernel(PaArgs p) {
  typedef PaTile<T, DP> Tile;
  constexpr int TK = Tile::TK, STEPS = Tile::NK / (TK / 16), E = 16 / (int)sizeof(T);
  constexpr bool Q_LDS = DP == 256;                 // the widest head's query operand takes its registers' place in LDS, under the results
  __shared__ alignas(16) float s_o[PA_WAVES][PA_ROWS][DP + 4];      // (rows four banks apart)
  __shared__ float s_m[PA_WAVES][PA_ROWS], s_l[PA_WAVES][PA_ROWS];
  pa_u32x4* s_q = (pa_u32x4*)s_o;
  const PagedAttnArgs& a = p.a;
  const int grp = blockIdx.x % p.s.groups, item = blockIdx.x / p.s.groups;
  const PaItem it = pa_item(p, item);
  if (it.r < 0) return;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const int hk = grp / p.s.tiles, qt = grp - hk * p.s.tiles, per_kv = a.heads_q / a.heads_kv;
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
      pa_order_k<T, DP>(t);
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
  if (c < rows) {
#pragma unroll
    for (int n = 0; n < Tile::EV; n += 4)
#pragma unroll
      for (int i = 0; i < 4; ++i) *(pa_f32x4*)&s_o[w][c][(4 * g + i) * Tile::EV + n] = pa_f32x4{o[n][i], o[n + 1][i], o[n + 2][i], o[n + 3][i]};
  }
  __syncthreads();
  float* part = a.part + ((int64_t)item * p.s.groups + grp) * pa_record(p.s.rows, a.d);
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
      Elem<T>::st((T*)a.o + (int64_t)it.r * a.o_r + (int64_t)(h0 + r) * a.o_h + e, ls == 0.f ? 0.f : os / ls * (1.f / PA_LOW));
      if (a.lse && e == 0) a.lse[(int64_t)it.r * a.heads_q + h0 + r] = ls == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(ls)) * 0.69314718055994531f;
    } else {
      part[r * a.d + e] = os;
      if (e == 0) { part[p.s.rows * a.d + 2 * r] = M; part[p.s.rows * a.d + 2 * r + 1] = ls; }
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
  const int64_t rec = (int64_t)p.s.groups * pa_record(p.s.rows, a.d);
  const float* base = a.part + ((int64_t)pl.x * p.s.groups + hk * p.s.tiles + qt) * pa_record(p.s.rows, a.d);
  float m = -INFINITY, l = 0.f;
  pa_f32x4 o = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 4;
  for (int i0 = grp; i0 < pl.y; i0 += ng * U) {
    float mi[U], li[U];
    pa_f32x4 oi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // (no branch around a load: the loads go out together; the last chunk again where there is none)
      const float* q = base + (int64_t)min(i0 + u * ng, pl.y - 1) * rec;
      const float2 ml = *(const float2*)(q + p.s.rows * a.d + 2 * row);
      mi[u] = i0 + u * ng < pl.y ? ml.x : -INFINITY; li[u] = ml.y;
      oi[u] = *(const pa_f32x4*)(q + row * a.d + 4 * min(e, d4 - 1));
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
  for (int x = 0; x < 4; ++x) Elem<T>::st(out + x, L == 0.f ? 0.f : O[x] / L * (1.f / PA_LOW));
  if (a.lse && e == 0) a.lse[(int64_t)r * a.heads_q + h] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.69314718055994531f;
}

bool paged_attention_fits(int dtype, int n_req, int heads_q, int heads_kv, int d, int64_t max_keys) {
  const PaShape s = pa_shape(dtype, n_req, heads_q, heads_kv, d, max_keys);
  // a launch has less than 2^32 threads, and a lane's share of the requests less than 2^32 units
  return (int64_t)s.items * s.groups < (1 << 23) && (int64_t)((n_req + 63) / 64) * ((max_keys + PA_UNIT - 1) / PA_UNIT) < ((int64_t)1 << 32);
}
size_t paged_attention_workspace(int dtype, int n_req, int heads_q, int heads_kv, int d, int64_t max_keys) {
  const PaShape s = pa_shape(dtype, n_req, heads_q, heads_kv, d, max_keys);
  return pa_align((size_t)std::max(1, n_req) * sizeof(int2)) + pa_align((size_t)s.items * s.groups * pa_record(s.rows, d) * sizeof(float));
}

// Requests of at most 256 keys have one workgroup each: eight waves finish its eight tiles at once, and nothing is joined.
template <typename T, int DP, bool FULL>
static int pa_launch(const PaArgs& p, bool join, hipStream_t stream) {
  if (!join) {
    paged_attn_kernel<T, DP, FULL, 8><<<dim3(p.s.items * p.s.groups), dim3(512), 0, stream>>>(p);
    return (int)hipGetLastError();
  }
  paged_attn_kernel<T, DP, FULL, 4><<<dim3(p.s.items * p.s.groups), dim3(256), 0, stream>>>(p);
  if (const int e = (int)hipGetLastError()) return e;
  paged_attn_join_kernel<T><<<dim3(p.a.heads_q, p.a.n_req), dim3(256), 0, stream>>>(p);
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
  PaArgs p{a, pa_shape(dtype, a.n_req, a.heads_q, a.heads_kv, a.d, max_keys), a.scale * 1.4426950408889634f, (int2*)a.part};
  p.a.part = (float*)((char*)a.part + pa_align((size_t)a.n_req * sizeof(int2)));
  const bool join = max_keys > p.s.least * PA_UNIT;    // else no request has two chunks
  *launches = join ? 2 : 1;
  return dtype == 0 ? pa_launch_d<float>(p, join, (hipStream_t)stream) : pa_launch_d<bf16_t>(p, join, (hipStream_t)stream);
}

}  // namespace sm
