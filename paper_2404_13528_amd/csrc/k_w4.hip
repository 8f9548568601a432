// Linear with 4-bit weights, group scales and zero points, on few rows: y = act(x W^T + bias) + residual.
//
// Bound by the stream of the packed weights (half a byte each, and 4 bytes a group for scale and zero point).  A workgroup
// takes 16 or 32 output features, its waves take turns over blocks of 128 k and meet in LDS at the end; every weight load of a wave
// is one contiguous KiB, requested blocks ahead.
//
//  * The matrix pipe's first operand is 16 features x 32 k: a lane's 8 k of a feature are one 32-bit word, and its four words
//    of a block one 16-byte load.  Nibble j and j + 4 of a word are the k of a pair: (word >> 4 j) & 0x000f000f with
//    0x4300 in both halves is the pair of bf16 numbers 128 + w, exactly, in at most two instructions.
//  * The products are integers times bf16 and the sums fp32.  What the offsets 128 + z add, (128 + z) sum of x, is taken off per
//    group; the sum of x comes from the same instruction with ones as the first operand, so it has the layout of the result.
//    Then the group's scale is applied, in fp32.
#include <algorithm>
#include "device_common.h"
#include "paged.h"

namespace sm {

namespace {
typedef unsigned int w4_u32x4 __attribute__((ext_vector_type(4)));
typedef float w4_f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 w4_bf16x8;

constexpr int W4_BLOCK = 128;            // k of a block
constexpr int W4_WAVES = 8;

struct W4Shape { int tiles, blocks; size_t weights, scales; };       // tiles of 16 features, blocks of k; bytes of either part
W4Shape w4_shape(int N, int K, int group) {
  W4Shape s;
  s.tiles = (N + 15) / 16; s.blocks = (K + W4_BLOCK - 1) / W4_BLOCK;
  s.weights = (size_t)s.tiles * s.blocks * 1024;
  s.scales = (size_t)s.tiles * s.blocks * (W4_BLOCK / group) * 64;
  return s;
}

__device__ __forceinline__ w4_f32x4 w4_mfma(w4_u32x4 a, w4_u32x4 b, w4_f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(w4_bf16x8, a), __builtin_bit_cast(w4_bf16x8, b), c, 0, 0, 0);
}
// the eight weights of a word as bf16 128 + w
__device__ __forceinline__ w4_u32x4 w4_widen(unsigned u) {
  w4_u32x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = ((u >> (4 * j)) & 0x000f000fu) | 0x43004300u;
  return v;
}
}  // namespace

size_t w4_packed_bytes(int N, int K, int group) { const W4Shape s = w4_shape(N, K, group); return s.weights + s.scales; }

// weights: word (tile, block, lane, step) holds k = 128 block + 32 step + 8 (lane / 16) + 0..7 of feature 16 tile + lane % 16, k = 2 j
// in nibble j and 2 j + 1 in nibble j + 4; scales: word (tile, group, feature) = scale (bf16, upper half) and 128 + zero point (bf16)
__global__ __launch_bounds__(256) void w4_pack_kernel(const unsigned* w, const bf16_t* s, const unsigned char* z, int N, int K, int group, int blocks,
                                                      int64_t n_words, int64_t n_scales, unsigned* pw, unsigned* ps) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n_words; i += (int64_t)gridDim.x * 256) {
    const int step = (int)(i & 3), lane = (int)(i >> 2) & 63;
    const int64_t tb = i >> 8;
    const int tile = (int)(tb / blocks), block = (int)(tb - (int64_t)tile * blocks);
    const int n = tile * 16 + (lane & 15), k = block * W4_BLOCK + step * 32 + (lane >> 4) * 8;
    unsigned u = 0;
    if (n < N && k < K) {
      const unsigned src = w[((int64_t)n * K + k) / 8];          // nibble e is k + e
#pragma unroll
      for (int j = 0; j < 4; ++j) u |= ((src >> (8 * j)) & 15) << (4 * j) | ((src >> (8 * j + 4)) & 15) << (4 * j + 16);
    }
    pw[i] = u;
  }
  const int groups = blocks * (W4_BLOCK / group), real = K / group;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n_scales; i += (int64_t)gridDim.x * 256) {
    const int64_t tg = i >> 4;
    const int tile = (int)(tg / groups), g = (int)(tg - (int64_t)tile * groups), n = tile * 16 + (int)(i & 15);
    unsigned u = 0;
    if (n < N && g < real) {
      const int64_t at = (int64_t)n * real + g;
      u = (unsigned)s[at] << 16 | f2bf(128.f + (z ? (float)(z[at] & 15) : 8.f));
    }
    ps[i] = u;
  }
}
int launch_w4_pack(const void* w, const void* scales, const void* zeros, int N, int K, int group, void* packed, void* stream) {
  const W4Shape s = w4_shape(N, K, group);
  const int64_t words = (int64_t)(s.weights / 4);
  w4_pack_kernel<<<dim3((unsigned)std::min<int64_t>((words + 255) / 256, 4096)), dim3(256), 0, (hipStream_t)stream>>>(
      (const unsigned*)w, (const bf16_t*)scales, (const unsigned char*)zeros, N, K, group, s.blocks, words, (int64_t)(s.scales / 4), (unsigned*)packed,
      (unsigned*)((char*)packed + s.weights));
  return (int)hipGetLastError();
}

namespace {
struct W4Args { LinearW4Args a; int blocks, tiles; const w4_u32x4* scales; };

// what a wave holds of one block of k
template <int MT, int NT, int GPB> struct W4Block { w4_u32x4 w[NT], s[NT][GPB], x[MT][4]; };

template <int MT, int NT, int GPB>
__device__ __forceinline__ void w4_load(W4Block<MT, NT, GPB>& b, const W4Args& p, int block, int tile0, const bf16_t* x, int rows) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  if (block >= p.blocks) return;                       // (wave-uniform)
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t tb = (int64_t)min(tile0 + n, p.tiles - 1) * p.blocks + block;
    b.w[n] = ((const w4_u32x4*)p.a.packed)[tb * 64 + lane];
#pragma unroll
    for (int i = 0; i < GPB; ++i) b.s[n][i] = p.scales[(tb * GPB + i) * 4 + g];
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int k = block * W4_BLOCK + s * 32 + g * 8;
      b.x[m][s] = w4_u32x4{0, 0, 0, 0};
      if (16 * m + c < rows && k < p.a.K) b.x[m][s] = *(const w4_u32x4*)(x + (int64_t)(16 * m + c) * p.a.K + k);
    }
}
template <int MT, int NT, int GPB>
__device__ __forceinline__ void w4_block(const W4Block<MT, NT, GPB>& b, w4_f32x4 (&tot)[NT][MT]) {
  constexpr int STEPS = 4 / GPB;
  const w4_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const w4_u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
  for (int i = 0; i < GPB; ++i) {
    w4_f32x4 sum[MT], acc[NT][MT];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
#pragma unroll
      for (int m = 0; m < MT; ++m) sum[m] = w4_mfma(ones, b.x[m][i * STEPS + s], s ? sum[m] : zero);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const w4_u32x4 w = w4_widen(b.w[n][i * STEPS + s]);
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = w4_mfma(w, b.x[m][i * STEPS + s], s ? acc[n][m] : zero);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float scale = __uint_as_float(b.s[n][i][r] & 0xffff0000u), off = __uint_as_float(b.s[n][i][r] << 16);
#pragma unroll
        for (int m = 0; m < MT; ++m) tot[n][m][r] = fmaf(scale, fmaf(-off, sum[m][r], acc[n][m][r]), tot[n][m][r]);
      }
  }
}
}  // namespace

template <int MT, int NT, int GPB, int PF>
__global__ __launch_bounds__(64 * W4_WAVES) void w4_kernel(W4Args p) {
  __shared__ float red[W4_WAVES][NT][MT][16][17];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const int tile0 = blockIdx.x * NT, m0 = blockIdx.y * 16 * MT, rows = min(16 * MT, p.a.M - m0);
  const bf16_t* x = (const bf16_t*)p.a.x + (int64_t)m0 * p.a.K;
  w4_f32x4 tot[NT][MT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) tot[n][m] = w4_f32x4{0.f, 0.f, 0.f, 0.f};
  if (w < p.blocks) {
    W4Block<MT, NT, GPB> b[PF];
#pragma unroll
    for (int i = 0; i < PF; ++i) w4_load<MT, NT, GPB>(b[i], p, w + i * W4_WAVES, tile0, x, rows);
    for (int k = w; k < p.blocks; k += PF * W4_WAVES) {
#pragma unroll
      for (int i = 0; i < PF; ++i) {
        if (k + i * W4_WAVES < p.blocks) w4_block<MT, NT, GPB>(b[i], tot);
        w4_load<MT, NT, GPB>(b[i], p, k + (i + PF) * W4_WAVES, tile0, x, rows);
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[w][n][m][c][4 * g + r] = tot[n][m][r];
  __syncthreads();
  for (int i = threadIdx.x; i < NT * MT * 256; i += 64 * W4_WAVES) {
    const int f = i & (16 * NT - 1), row = i / (16 * NT), n = tile0 * 16 + f;
    if (row >= rows || n >= p.a.N) continue;
    float v = 0.f;
#pragma unroll
    for (int u = 0; u < W4_WAVES; ++u) v += red[u][f >> 4][row >> 4][row & 15][f & 15];
    const int64_t at = (int64_t)(m0 + row) * p.a.N + n;
    if (p.a.bias) v += bf2f(((const bf16_t*)p.a.bias)[n]);
    if (p.a.act) v = gelu_erf(v);
    if (p.a.residual) v += bf2f(((const bf16_t*)p.a.residual)[at]);
    ((bf16_t*)p.a.y)[at] = f2bf(v);
  }
}

template <int GPB>
static void w4_launch(const W4Args& p, hipStream_t stream) {
  if (p.a.M <= 16) w4_kernel<1, 1, GPB, 4><<<dim3(p.tiles), dim3(64 * W4_WAVES), 0, stream>>>(p);
  else w4_kernel<2, 2, GPB, 2><<<dim3((p.tiles + 1) / 2, (p.a.M + 31) / 32), dim3(64 * W4_WAVES), 0, stream>>>(p);
}
int launch_w4(const LinearW4Args& a, void* stream) {
  const W4Shape s = w4_shape(a.N, a.K, a.group);
  const W4Args p{a, s.blocks, s.tiles, (const w4_u32x4*)((const char*)a.packed + s.weights)};
  if (a.group == 128) w4_launch<1>(p, (hipStream_t)stream);
  else if (a.group == 64) w4_launch<2>(p, (hipStream_t)stream);
  else w4_launch<4>(p, (hipStream_t)stream);
  return (int)hipGetLastError();
}

}  // namespace sm
