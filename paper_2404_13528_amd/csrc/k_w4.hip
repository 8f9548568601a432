// Linear with 4-bit weights, group scales and zero points, on few rows: y = act(x W^T + bias) + residual.
//
// Bound by the stream of the packed weights (half a byte each, and 4 bytes a group for scale and zero point), with many rows also by the
// x that every workgroup loads.  A workgroup has all of K for its 16 to 96 features: its waves take turns over blocks of 128 k and meet in
// LDS at the end.
//
//  * The matrix pipe's second operand is 16 features x 32 k: a lane's 8 k of a feature are one 32-bit word, and its four words
//    of a block one 16-byte load.  Nibble j and j + 4 of a word are the k of a pair: (word >> 4 j) & 0x000f000f with
//    0x4300 in both halves is the pair of bf16 numbers 128 + w, exactly, in at most two instructions.
//  * The products are integers times bf16 and the sums fp32.  What the offsets 128 + z add, (128 + z) sum of x, is taken off per
//    group; the sum of x comes from the same instruction with ones as the second operand, so it has the layout of the result.
//    The sums round relative to up to 143 |x| instead of |w - z| |x|, still far below the store's rounding (17 x 22016 x 4096: 432 of the
//    374272 results are not the bf16 number nearest to the exact one, 215 of a plain fp32 computation).  From |x| = 2^113 on they overflow.
//    Then the group's scale is applied, in fp32.  The rows of the result are the rows of x, a lane's column is one feature:
//    it needs one word of scale and zero point per group.
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

constexpr int w4_record(int groups) { return 1024 + 64 * groups; }      // bytes of a tile's block: weights, then the words of its groups

__device__ __forceinline__ w4_f32x4 w4_mfma(w4_u32x4 a, w4_u32x4 b, w4_f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(w4_bf16x8, a), __builtin_bit_cast(w4_bf16x8, b), c, 0, 0, 0);
}
// the eight weights of a word as bf16 128 + w; mask 0x000f000f and offset 0x43004300 are kernel arguments, which the compiler keeps
// in registers (literals would make two instructions of the and-or)
__device__ __forceinline__ w4_u32x4 w4_widen(unsigned u, unsigned mask, unsigned offset) {
  w4_u32x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = ((u >> (4 * j)) & mask) | offset;
  return v;
}
}  // namespace

size_t w4_packed_bytes(int N, int K, int group) {
  return (size_t)((N + 15) / 16) * ((K + W4_BLOCK - 1) / W4_BLOCK) * w4_record(W4_BLOCK / group);
}

// A record per tile of 16 features and block of 128 k, blocks of a tile one behind the other.  Weights: word (lane, step) holds
// k = 128 block + 32 step + 8 (lane / 16) + 0..7 of feature 16 tile + lane % 16, k = 2 j in nibble j and 2 j + 1 in nibble j + 4;
// then word (group, feature) = scale (bf16, upper half) and 128 + zero point (bf16).
__global__ __launch_bounds__(256) void w4_pack_kernel(const unsigned* w, const bf16_t* s, const unsigned char* z, int N, int K, int group, int blocks,
                                                      int64_t n_words, unsigned* packed) {
  const int words = w4_record(W4_BLOCK / group) / 4, real = K / group;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n_words; i += (int64_t)gridDim.x * 256) {
    const int64_t tb = i / words, tile = tb / blocks;
    const int at = (int)(i - tb * words), block = (int)(tb - tile * blocks);
    unsigned u = 0;
    if (at < 256) {
      const int step = at & 3, lane = at >> 2, k = block * W4_BLOCK + step * 32 + (lane >> 4) * 8;
      const int64_t n = tile * 16 + (lane & 15);
      if (n < N && k < K) {
        const unsigned src = w[(n * K + k) / 8];                 // nibble e is k + e
#pragma unroll
        for (int j = 0; j < 4; ++j) u |= ((src >> (8 * j)) & 15) << (4 * j) | ((src >> (8 * j + 4)) & 15) << (4 * j + 16);
      }
    } else {
      const int g = block * (W4_BLOCK / group) + (at - 256) / 16;
      const int64_t n = tile * 16 + (at & 15);
      if (n < N && g < real) u = (unsigned)s[n * real + g] << 16 | f2bf(128.f + (z ? (float)(z[n * real + g] & 15) : 8.f));
    }
    packed[i] = u;
  }
}
int launch_w4_pack(const void* w, const void* scales, const void* zeros, int N, int K, int group, void* packed, void* stream) {
  const int64_t words = (int64_t)(w4_packed_bytes(N, K, group) / 4);
  w4_pack_kernel<<<dim3((unsigned)std::min<int64_t>((words + 255) / 256, 8192)), dim3(256), 0, (hipStream_t)stream>>>(
      (const unsigned*)w, (const bf16_t*)scales, (const unsigned char*)zeros, N, K, group, (K + W4_BLOCK - 1) / W4_BLOCK, words, (unsigned*)packed);
  return (int)hipGetLastError();
}

namespace {
struct W4Args { LinearW4Args a; int blocks, tiles; unsigned mask, offset; };

// sums of x over the groups of a block, in the layout of the products
template <int MT, int GPB>
__device__ __forceinline__ void w4_sums(const w4_u32x4 (&x)[MT][4], w4_f32x4 (&sum)[GPB][MT]) {
  constexpr int STEPS = 4 / GPB;
  const w4_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const w4_u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
  for (int i = 0; i < GPB; ++i)
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int m = 0; m < MT; ++m) sum[i][m] = w4_mfma(x[m][i * STEPS + s], ones, s ? sum[i][m] : zero);
}
// One block of one tile: tot += scale (sum over the group of (128 + w) x - (128 + z) sum of x).  keep: 0 takes the block's scales away.
template <int MT, int GPB>
__device__ __forceinline__ void w4_block(const w4_u32x4 wv, const unsigned (&sv)[GPB], const w4_u32x4 (&x)[MT][4], const w4_f32x4 (&sum)[GPB][MT], w4_f32x4 (&tot)[MT],
                                         unsigned mask, unsigned offset, unsigned keep) {
  constexpr int STEPS = 4 / GPB;
  const w4_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < GPB; ++i) {
    w4_f32x4 acc[MT];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const w4_u32x4 w = w4_widen(wv[i * STEPS + s], mask, offset);
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m] = w4_mfma(x[m][i * STEPS + s], w, s ? acc[m] : zero);
    }
    const float scale = __uint_as_float(sv[i] & keep), off = __uint_as_float(sv[i] << 16);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) tot[m][r] = fmaf(scale, fmaf(-off, sum[i][m][r], acc[m][r]), tot[m][r]);
  }
}

}  // namespace

// A workgroup has NT tiles of 16 features and MT tiles of 16 rows (HALF: up to 8 rows).  Its waves have PB blocks of k each at a time:
// a wave's x of these blocks stays in registers while the tiles' weights of the same blocks go by, all of them requested at once (a cold
// load takes 2 us, so the kernel's time is that of its longest chain of them), the next turn's as the present ones are used up.  The
// waves' sums of a tile meet in LDS.
// Loads return in the order of their issue, and the compiler's counting of them survives no branch: all loads are unconditional, and their
// order is pinned.
// Calls in a replayed graph, groups of 128: 1 x 4096 x 4096 4.0 us, 1 x 22016 x 4096 11.7 us (4.1 TB/s), 32 x 22016 x 4096 18 us, 32 x 4096 x 11008
// 15 us.  Of the 16 us of 17 x 22016 x 4096 in groups of 64 the stream of the weights alone takes 11; the rest is x, the products and the end.
template <int MT, bool HALF, int NT, int GPB, int PB>
__global__ __launch_bounds__(64 * W4_WAVES, 2) void w4_kernel(W4Args p) {
  __shared__ float red[W4_WAVES][NT][MT][16][17];
  __shared__ float s_bias[NT * 16];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  constexpr int ROWS = HALF ? 8 : 16 * MT;
  const int tile0 = blockIdx.x * NT, m0 = blockIdx.y * ROWS, rows = min(ROWS, p.a.M - m0), K = p.a.K;
  const unsigned mask = p.mask;
  unsigned offset;
  asm("v_mov_b32 %0, %1" : "=v"(offset) : "s"(p.offset));      // (an instruction takes one scalar register: the other constant goes to a vector one)
  const char* xp = (const char*)p.a.x + (int64_t)m0 * K * 2;
  // rows behind the end read the last one and are not stored
  unsigned xa[MT], xb[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    xa[m] = (unsigned)min(16 * m + (c & 7), rows - 1) * (unsigned)K;
    xb[m] = (unsigned)min(16 * m + (c & 7) + 8, rows - 1) * (unsigned)K;
  }
  const int k_lane = (c >> 3) * 32 + g * 8;
  w4_f32x4 tot[NT][MT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) tot[n][m] = w4_f32x4{0.f, 0.f, 0.f, 0.f};

  w4_u32x4 x[PB][MT][4], wv[PB][NT];
  unsigned sv[PB][NT][GPB];
  w4_f32x4 sum[GPB][MT];
  // blocks behind the end read the last one there is, and lose its scales; so do k behind the end, whose scales are zero.
  // A load of x takes 64 k of 8 rows, whole lines of memory.  Two such loads become two operands of 32 k of 16 rows when lanes 8 .. 15 of a row of
  // lanes change places with lanes 0 .. 7 of the other; up to 8 rows one load is both operands (half the loads and registers).
  auto load_x = [&](int i, int block) {
    block = min(block, p.blocks - 1);
#pragma unroll
    for (int s = 0; s < 4; s += 2) {
      const unsigned k = min(block * W4_BLOCK + s * 32 + k_lane, K - 8);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        x[i][m][s] = *(const w4_u32x4*)(xp + 2 * (xa[m] + k));
        if (!HALF) x[i][m][s + 1] = *(const w4_u32x4*)(xp + 2 * (xb[m] + k));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto order_x = [&](int i) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int s = 0; s < 4; s += 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int a = x[i][m][s][e], b = HALF ? a : x[i][m][s + 1][e];      // (up to 8 rows: the others are anything)
          if (!HALF) x[i][m][s][e] = __builtin_amdgcn_update_dpp(a, b, 0x128, 0xf, 0xc, false);
          x[i][m][s + 1][e] = __builtin_amdgcn_update_dpp(b, a, 0x128, 0xf, 0x3, false);
        }
  };
  auto load_w = [&](int i, int n, int block) {
    block = min(block, p.blocks - 1);
    const char* r = (const char*)p.a.packed + ((int64_t)min(tile0 + n, p.tiles - 1) * p.blocks + block) * w4_record(GPB);
    wv[i][n] = *(const w4_u32x4*)(r + lane * 16);
#pragma unroll
    for (int j = 0; j < GPB; ++j) sv[i][n][j] = *(const unsigned*)(r + 1024 + j * 64 + c * 4);
    __builtin_amdgcn_sched_barrier(0);
  };
  if (threadIdx.x < NT * 16) {
    const int n = tile0 * 16 + threadIdx.x;
    s_bias[threadIdx.x] = p.a.bias && n < p.a.N ? bf2f(((const bf16_t*)p.a.bias)[n]) : 0.f;
  }
  constexpr int TURN = W4_WAVES * PB;                  // blocks of a turn: wave w has w * PB ..
  int block = w * PB;
  if (block < p.blocks) {
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      load_x(i, block + i);
#pragma unroll
      for (int n = 0; n < NT; ++n) load_w(i, n, block + i);
    }
#pragma unroll 1
    for (; block + TURN < p.blocks; block += TURN) {
#pragma unroll
      for (int i = 0; i < PB; ++i) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (n == 0) {
            order_x(i);
            w4_sums<MT, GPB>(x[i], sum);
          }
          w4_block<MT, GPB>(wv[i][n], sv[i][n], x[i], sum, tot[n], mask, offset, 0xffff0000u);
          __builtin_amdgcn_sched_barrier(0);
          if (n + 1 == NT) load_x(i, block + TURN + i);
          load_w(i, n, block + TURN + i);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      order_x(i);
      w4_sums<MT, GPB>(x[i], sum);
#pragma unroll
      for (int n = 0; n < NT; ++n) w4_block<MT, GPB>(wv[i][n], sv[i][n], x[i], sum, tot[n], mask, offset, block + i < p.blocks ? 0xffff0000u : 0u);
    }
  }
  // the tiles' sums meet: output i is row i / (16 NT), feature i % (16 NT); a thread's residuals are asked for before the waves meet
  constexpr int OUT = NT * MT * 256, PER = (OUT + 64 * W4_WAVES - 1) / (64 * W4_WAVES);
  float res[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = threadIdx.x + j * 64 * W4_WAVES, row = i / (16 * NT), n = tile0 * 16 + i % (16 * NT);
    res[j] = 0.f;
    if (p.a.residual && row < rows && n < p.a.N) res[j] = bf2f(((const bf16_t*)p.a.residual)[(int64_t)(m0 + row) * p.a.N + n]);
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[w][n][m][4 * g + r][c] = tot[n][m][r];
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = threadIdx.x + j * 64 * W4_WAVES, row = i / (16 * NT), f = i % (16 * NT), n = tile0 * 16 + f;
    if (row >= rows || n >= p.a.N) continue;           // (rows <= ROWS: no output behind the last one)
    float v = 0.f;
#pragma unroll
    for (int u = 0; u < W4_WAVES; ++u) v += red[u][f >> 4][row >> 4][row & 15][f & 15];
    v += s_bias[f];
    if (p.a.act) v = gelu_erf(v);
    ((bf16_t*)p.a.y)[(int64_t)(m0 + row) * p.a.N + n] = f2bf(v + res[j]);
  }
}

// Rows and tiles of a workgroup.  The time goes by the bytes that a CU takes in: a workgroup's rows of x (2 a k) and tiles of weights (8 and a
// half a k, scales included), times the workgroups that a CU has; a tile's sums that meet at the end count like 6 more.  Measured against all
// 15 choices at twelve sizes the one taken was within 0.6 us of the best: 32 x 4096 x 4096 takes 7.1 us with 16 rows and two tiles, 10.3 with
// 32 and one; 32 x 11008 x 4096 12.8 us with 32 and three, 25 with 16 and one; 1 x 22016 x 4096 11.5 to 13.3 us.
struct W4Choice { int rows, nt; };
static W4Choice w4_choose(int M, int tiles) {
  static const int NTS[5] = {1, 2, 3, 4, 6};
  W4Choice best = {0, 0};
  double least = 0;
  for (int rows = 8; rows <= 32; rows *= 2) {
    if (rows > 8 && rows / 2 >= M) break;
    if ((M + rows - 1) / rows > 65535) continue;       // (a launch's second extent)
    for (int nt : NTS) {
      const int64_t groups = (int64_t)((tiles + nt - 1) / nt) * ((M + rows - 1) / rows);
      const double cost = (double)((groups + 255) / 256) * (2.0 * std::min(rows, M) + 8.5 * nt) + 6.0 * nt;
      if (!best.rows || cost <= least) { best = W4Choice{rows, nt}; least = cost; }
    }
  }
  return best;
}
template <int GPB, int MT, bool HALF, int NT>
static void w4_go(const W4Args& p, hipStream_t stream) {
  constexpr int PB = MT == 1 ? 2 : 1, ROWS = HALF ? 8 : 16 * MT;
  w4_kernel<MT, HALF, NT, GPB, PB><<<dim3((p.tiles + NT - 1) / NT, (p.a.M + ROWS - 1) / ROWS), dim3(64 * W4_WAVES), 0, stream>>>(p);
}
template <int GPB, int MT, bool HALF>
static void w4_tiles(const W4Args& p, int nt, hipStream_t stream) {
  if (nt == 1) w4_go<GPB, MT, HALF, 1>(p, stream);
  else if (nt == 2) w4_go<GPB, MT, HALF, 2>(p, stream);
  else if (nt == 3) w4_go<GPB, MT, HALF, 3>(p, stream);
  else if (nt == 4) w4_go<GPB, MT, HALF, 4>(p, stream);
  else w4_go<GPB, MT, HALF, 6>(p, stream);
}
template <int GPB>
static void w4_launch(const W4Args& p, hipStream_t stream) {
  const W4Choice c = w4_choose(p.a.M, p.tiles);
  if (c.rows == 8) w4_tiles<GPB, 1, true>(p, c.nt, stream);
  else if (c.rows == 16) w4_tiles<GPB, 1, false>(p, c.nt, stream);
  else w4_tiles<GPB, 2, false>(p, c.nt, stream);
}
int launch_w4(const LinearW4Args& a, void* stream) {
  const W4Args p{a, (a.K + W4_BLOCK - 1) / W4_BLOCK, (a.N + 15) / 16, 0x000f000fu, 0x43004300u};
  if (a.group == 128) w4_launch<1>(p, (hipStream_t)stream);
  else if (a.group == 64) w4_launch<2>(p, (hipStream_t)stream);
  else w4_launch<4>(p, (hipStream_t)stream);
  return (int)hipGetLastError();
}

}  // namespace sm
