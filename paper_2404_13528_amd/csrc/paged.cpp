// C ABI of the operators over a paged key / value cache and of the 4-bit Linear: validation, then the launches.
#include <algorithm>
#include <cmath>
#include <cstring>
#include "common.h"
#include "paged.h"

using namespace sm;

namespace {
constexpr int64_t CAP = (int64_t)1 << 30;
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
// the last place of a page pool in units of 16 bytes, -1 if it does not fit 32 bits or a stride is negative
int64_t pool_units(const int64_t (&s)[3], int n_pages, int page, int vec) {
  const int64_t top = (int64_t)1 << 32;
  if (s[0] < 0 || s[1] < 0 || s[0] / vec >= top || s[1] / vec >= top) return -1;
  const int64_t u = (int64_t)(n_pages - 1) * (s[0] / vec);          // (both factors below 2^30 resp. 2^32)
  const int64_t v = (int64_t)(page - 1) * (s[1] / vec);
  return u < top && v < top && u + v < top ? u + v : -1;
}
// An array of `rows` rows of `width` bytes, `pitch` >= width apart; a plain array is one row.
struct Span { const void* p; uint64_t width, rows, pitch; };
// whether a plain array and another have a byte in common
bool meet(const Span& plain, const Span& s) {
  const uint64_t lo = reinterpret_cast<uintptr_t>(plain.p), hi = lo + plain.width, at = reinterpret_cast<uintptr_t>(s.p);
  if (!plain.width || !s.width) return false;
  const uint64_t k = lo <= at || s.rows == 1 ? 0 : std::min((lo - at) / s.pitch, s.rows - 1);      // the last row that starts at or before lo, or the first
  return (lo < at + k * s.pitch + s.width && hi > at + k * s.pitch) || (k + 1 < s.rows && hi > at + (k + 1) * s.pitch);
}
Span flat(const void* p, uint64_t bytes) { return Span{p, p ? bytes : 0, 1, 0}; }
template <int N> bool multiples(const int64_t (&s)[N], int vec) {
  for (int64_t v : s) if (v % vec) return false;
  return true;
}
}  // namespace

extern "C" int sm_page_table(const sm_page_cfg* c, const int32_t* cached, const int32_t* fresh, const int32_t* free_pages, const int32_t* n_free,
                             int32_t* table, int32_t* starts, int32_t* lens, int32_t* positions, int32_t* slots, int32_t* need, void* stream) {
  const char* who = "sm_page_table";
  if (!c) return fail(SM_ERR_INVALID_ARG, "%s: null configuration", who);
  if (c->n_req < 1 || c->n_req > 65536) return fail(SM_ERR_SHAPE, "%s: 1 to 65536 requests", who);
  if (c->page < 1 || c->max_pages < 1 || c->n_pages < 1 || c->free_cap < 0 || c->max_tokens < 0) return fail(SM_ERR_SHAPE, "%s: bad size", who);
  if (c->table_pitch < c->max_pages) return fail(SM_ERR_SHAPE, "%s: a table row of %d pages does not fit a pitch of %lld", who, c->max_pages, (long long)c->table_pitch);
  if (c->max_tokens > CAP || (int64_t)c->n_req * c->max_pages > CAP || (int64_t)c->n_pages * c->page > CAP || (int64_t)c->max_pages * c->page > CAP)
    return fail(SM_ERR_SHAPE, "%s: tokens, table entries, slots and the tokens of a table row are limited to 2^30", who);
  if (!cached || !fresh || !n_free || !table || !starts || !lens || !need || (c->free_cap && !free_pages) || (c->max_tokens && (!positions || !slots)))
    return fail(SM_ERR_INVALID_ARG, "%s: null pointer", who);
  const void* all[11] = {cached, fresh, free_pages, n_free, table, starts, lens, positions, slots, need, nullptr};
  for (const void* p : all) if (!aligned4(p)) return fail(SM_ERR_INVALID_ARG, "%s: arrays must be 4-byte aligned", who);
  const uint64_t R = (uint64_t)c->n_req, T = (uint64_t)c->max_tokens;
  const Span spans[10] = {flat(starts, 4 * (R + 1)), flat(lens, 4 * R), flat(positions, 4 * T), flat(slots, 4 * T), flat(need, 4),      // written
                          flat(cached, 4 * R), flat(fresh, 4 * R), flat(free_pages, 4 * (uint64_t)c->free_cap), flat(n_free, 4),
                          Span{table, 4 * (uint64_t)c->max_pages, R, 4 * (uint64_t)c->table_pitch}};
  for (int i = 0; i < 9; ++i)
    for (int j = i + 1; j < 10; ++j)
      if ((i < 5 || j == 9) && meet(spans[i], spans[j])) return fail(SM_ERR_INVALID_ARG, "%s: an output overlaps an input or another output", who);
  PageTableArgs a{cached, fresh, free_pages, n_free, table, starts, lens, positions, slots, need,
                  c->n_req, c->page, c->max_pages, c->n_pages, c->free_cap, c->max_tokens, c->table_pitch};
  char label[96] = "";
  if (timing_on()) snprintf(label, sizeof(label), "page_table[%d,%d]", c->n_req, c->max_tokens);
  Timed tm(label, stream);
  if (int e = launch_page_table(a, stream)) return fail(SM_ERR_DEVICE, "%s: launch failed (hip error %d)", who, e);
  count_compute();
  return SM_OK;
}

extern "C" int sm_head_norm_rope(const sm_head_norm_rope_desc* c, const void* q, const void* k, const void* v, const int32_t* positions,
                                 const int32_t* slots, void* q_out, void* k_out, void* v_out, void* stream) {
  const char* who = "sm_head_norm_rope";
  if (!c) return fail(SM_ERR_INVALID_ARG, "%s: null descriptor", who);
  if (!dtype_ok(c->dtype)) return fail(SM_ERR_INVALID_ARG, "%s: unknown dtype", who);
  const int vec = c->dtype == SM_F32 ? 4 : 8;
  if (c->tokens < 0 || c->tokens > (1 << 25)) return fail(SM_ERR_SHAPE, "%s: 0 to 2^25 tokens", who);      // (a launch has less than 2^32 threads)
  if ((q && (c->heads_q < 1 || c->heads_q > 65536)) || ((k || v) && (c->heads_kv < 1 || c->heads_kv > 65536))) return fail(SM_ERR_SHAPE, "%s: bad number of heads", who);
  if (c->d < vec || c->d > 256 || c->d % vec) return fail(SM_ERR_SHAPE, "%s: head size must be a multiple of %d, at most 256", who, vec);
  if (c->rot < 0 || c->rot > c->d || c->rot % (2 * vec)) return fail(SM_ERR_SHAPE, "%s: rotated features must be a multiple of %d, at most the head size", who, 2 * vec);
  if (c->norm < 0 || c->norm > 2) return fail(SM_ERR_INVALID_ARG, "%s: unknown norm %d", who, c->norm);
  if (c->rot && !(c->rope_base >= 1.f && std::isfinite(c->rope_base))) return fail(SM_ERR_INVALID_ARG, "%s: the rotation's base must be at least 1", who);
  if (!k && !v) slots = nullptr;                     // (places of keys and values only)
  if (slots && (c->page < 1 || c->n_pages < 1 || (int64_t)c->page * c->n_pages > CAP)) return fail(SM_ERR_SHAPE, "%s: bad page pool", who);
  if (c->tokens == 0) return SM_OK;                  // no tokens: no pointer is looked at, nothing is launched
  if (!q && !k && !v) return fail(SM_ERR_INVALID_ARG, "%s: nothing to do: q, k and v are null", who);
  if (!positions) return fail(SM_ERR_INVALID_ARG, "%s: null positions", who);
  if (!aligned4(positions) || !aligned4(slots)) return fail(SM_ERR_INVALID_ARG, "%s: positions and slots must be 4-byte aligned", who);
  if ((q && !q_out) || (k && !k_out) || (v && !v_out)) return fail(SM_ERR_INVALID_ARG, "%s: null output", who);
  if (c->norm && ((q && !c->q_gamma) || (k && !c->k_gamma))) return fail(SM_ERR_INVALID_ARG, "%s: the norm needs its gain", who);
  if (c->norm == 1 && ((q && !c->q_beta) || (k && !c->k_beta))) return fail(SM_ERR_INVALID_ARG, "%s: LayerNorm needs its shift", who);
  const void* all[] = {q, k, v, q ? q_out : nullptr, k ? k_out : nullptr, v ? v_out : nullptr, c->norm && q ? c->q_gamma : nullptr, c->norm && k ? c->k_gamma : nullptr,
                       c->norm == 1 && q ? c->q_beta : nullptr, c->norm == 1 && k ? c->k_beta : nullptr};
  for (const void* p : all) if (!aligned16(p)) return fail(SM_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", who);
  if ((q && (!multiples(c->q_stride, vec) || !multiples(c->q_out_stride, vec))) || (k && (!multiples(c->k_stride, vec) || !multiples(c->k_out_stride, vec))) ||
      (v && (!multiples(c->v_stride, vec) || !multiples(c->v_out_stride, vec))))
    return fail(SM_ERR_SHAPE, "%s: strides must keep 16-byte alignment", who);
  HeadNormArgs a; std::memset(&a, 0, sizeof(a));
  if (q) a.part[0] = HeadNormPart{q, c->q_gamma, c->q_beta, q_out, c->q_stride[0], c->q_stride[1], 0, c->q_out_stride[0], c->q_out_stride[1], c->heads_q, 0, 0};
  const int paged = slots != nullptr;
  if (k) a.part[1] = HeadNormPart{k, c->k_gamma, c->k_beta, k_out, c->k_stride[0], c->k_stride[1], c->k_out_stride[0], c->k_out_stride[1], c->k_out_stride[2], c->heads_kv, 0, paged};
  if (v) a.part[2] = HeadNormPart{v, nullptr, nullptr, v_out, c->v_stride[0], c->v_stride[1], c->v_out_stride[0], c->v_out_stride[1], c->v_out_stride[2], c->heads_kv, 0, paged};
  if (c->rot) {
    // theta_i / 2 pi in 64 bits behind the point.  The repeated product in 64-bit mantissas is off by at most 2 i 2^-64 of theta_i / 2 pi
    // <= 0.16, with at most 127 factors 2^-58: at positions below 2^31 less than 2^-27 of a revolution
    const long double step = powl((long double)c->rope_base, -2.0L / c->rot);
    long double f = 0.15915494309189533576888376337251436L;
    for (int i = 0; i < c->rot / 2; ++i, f *= step) a.turn[i] = (uint64_t)(f * 18446744073709551616.0L);
  }
  a.positions = positions; a.slots = slots; a.tokens = c->tokens; a.d = c->d; a.rot = c->rot; a.norm = c->norm;
  a.page = slots ? c->page : 1; a.n_slots = slots ? c->page * c->n_pages : 0; a.eps = c->eps;
  char label[128] = "";
  if (timing_on()) snprintf(label, sizeof(label), "head_norm_rope_%s[%d,%d+%d+%d,%d]%s", c->dtype == SM_F32 ? "f32" : "bf16", c->tokens, q ? c->heads_q : 0, k ? c->heads_kv : 0,
           v ? c->heads_kv : 0, c->d, slots ? "+pages" : "");
  Timed tm(label, stream);
  if (int e = launch_head_norm_rope(a, c->dtype, stream)) return fail(SM_ERR_DEVICE, "%s: launch failed (hip error %d)", who, e);
  count_compute();
  return SM_OK;
}

namespace {
int check_paged_attention(const sm_paged_attention_desc* c, const char* who) {
  if (!c) return fail(SM_ERR_INVALID_ARG, "%s: null descriptor", who);
  if (!dtype_ok(c->dtype)) return fail(SM_ERR_INVALID_ARG, "%s: unknown dtype", who);
  const int vec = c->dtype == SM_F32 ? 4 : 8;
  if (c->n_req < 0 || c->n_req > 65535) return fail(SM_ERR_SHAPE, "%s: at most 65535 requests", who);
  if (c->heads_q < 1 || c->heads_kv < 1 || c->heads_q % c->heads_kv || c->heads_q > 65535) return fail(SM_ERR_SHAPE, "%s: the query heads must be a multiple of the key heads, at most 65535", who);
  if (c->d < vec || c->d > 256 || c->d % vec) return fail(SM_ERR_SHAPE, "%s: head size must be a multiple of %d, at most 256", who, vec);
  if (c->page < 1 || c->max_pages < 1 || c->n_pages < 1 || c->table_pitch < c->max_pages) return fail(SM_ERR_SHAPE, "%s: bad page size, table or pool", who);
  if ((int64_t)c->page * c->max_pages > CAP || (int64_t)c->page * c->n_pages > CAP) return fail(SM_ERR_SHAPE, "%s: a request's tokens and the pool's are limited to 2^30", who);
  if (!std::isfinite(c->scale)) return fail(SM_ERR_INVALID_ARG, "%s: the scale must be finite", who);
  if (!multiples(c->q_stride, vec) || !multiples(c->o_stride, vec) || !multiples(c->k_stride, vec) || !multiples(c->v_stride, vec))
    return fail(SM_ERR_SHAPE, "%s: strides must keep 16-byte alignment", who);
  const int64_t last[2] = {pool_units(c->k_stride, c->n_pages, c->page, vec), pool_units(c->v_stride, c->n_pages, c->page, vec)};
  if (last[0] < 0 || last[1] < 0) return fail(SM_ERR_SHAPE, "%s: a pool has strides of at least zero and spans at most 64 GiB", who);
  if (!paged_attention_fits(c->dtype, c->n_req, c->heads_q, c->heads_kv, c->d, (int64_t)c->page * c->max_pages)) return fail(SM_ERR_SHAPE, "%s: too many requests, heads and keys for one launch", who);
  return SM_OK;
}
}  // namespace

extern "C" size_t sm_paged_attention_workspace_bytes(const sm_paged_attention_desc* c) {
  if (check_paged_attention(c, "sm_paged_attention_workspace_bytes") != SM_OK) return 0;
  return paged_attention_workspace(c->dtype, c->n_req, c->heads_q, c->heads_kv, c->d, (int64_t)c->page * c->max_pages);
}

extern "C" int sm_paged_attention(const sm_paged_attention_desc* c, const void* q, const void* k_pages, const void* v_pages, const int32_t* table,
                                  const int32_t* lens, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "sm_paged_attention";
  if (int rc = check_paged_attention(c, who)) return rc;
  if (c->n_req == 0) return SM_OK;                   // no requests: no pointer is looked at, nothing is launched
  if (!q || !k_pages || !v_pages || !table || !lens || !o || !ws) return fail(SM_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(o) || !aligned16(ws)) return fail(SM_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", who);
  if (!aligned4(table) || !aligned4(lens) || !aligned4(lse)) return fail(SM_ERR_INVALID_ARG, "%s: table, lens and lse must be 4-byte aligned", who);
  const size_t want = paged_attention_workspace(c->dtype, c->n_req, c->heads_q, c->heads_kv, c->d, (int64_t)c->page * c->max_pages);
  if (ws_bytes < want) return fail(SM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, want);
  PagedAttnArgs a{q, k_pages, v_pages, table, lens, o, lse, (float*)ws, c->n_req, c->heads_q, c->heads_kv, c->d, c->page, c->max_pages, c->n_pages, c->scale,
                  c->table_pitch, c->q_stride[0], c->q_stride[1], c->o_stride[0], c->o_stride[1], c->k_stride[0], c->k_stride[1], c->k_stride[2],
                  c->v_stride[0], c->v_stride[1], c->v_stride[2]};
  char label[128] = "";
  if (timing_on()) snprintf(label, sizeof(label), "paged_attention_%s[%d,%d/%d,%d,%d]", c->dtype == SM_F32 ? "f32" : "bf16", c->n_req, c->heads_q, c->heads_kv, c->max_pages * c->page, c->d);
  Timed tm(label, stream);
  int launches = 0;
  if (int e = launch_paged_attention(a, c->dtype, stream, &launches)) return fail(SM_ERR_DEVICE, "%s: launch failed (hip error %d)", who, e);
  count_compute(launches);
  return SM_OK;
}

namespace {
int check_w4(int N, int K, int group, const char* who) {
  if (group != 32 && group != 64 && group != 128) return fail(SM_ERR_UNSUPPORTED, "%s: groups of 32, 64 or 128 weights", who);
  if (N < 1 || K < group || K % group) return fail(SM_ERR_SHAPE, "%s: K must be a multiple of the group (N = %d, K = %d, group %d)", who, N, K, group);
  if (N > (1 << 24) || K > (1 << 24)) return fail(SM_ERR_SHAPE, "%s: N and K are limited to 2^24", who);
  return SM_OK;
}
}  // namespace

extern "C" size_t sm_linear_w4_packed_bytes(int N, int K, int group) {
  return check_w4(N, K, group, "sm_linear_w4_packed_bytes") == SM_OK ? w4_packed_bytes(N, K, group) : 0;
}

extern "C" int sm_linear_w4_pack(const void* w, const void* scales, const void* zeros, int N, int K, int group, void* packed, void* stream) {
  const char* who = "sm_linear_w4_pack";
  if (int rc = check_w4(N, K, group, who)) return rc;
  if (!w || !scales || !packed) return fail(SM_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned16(w) || !aligned16(scales) || !aligned16(packed)) return fail(SM_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", who);
  const Span out = flat(packed, w4_packed_bytes(N, K, group));
  const uint64_t groups = (uint64_t)N * (K / group);
  for (const Span& in : {flat(w, (uint64_t)N * K / 2), flat(scales, 2 * groups), flat(zeros, groups)})
    if (meet(out, in)) return fail(SM_ERR_INVALID_ARG, "%s: the packed weights overlap their sources", who);
  Timed tm("linear_w4_pack", stream);
  if (int e = launch_w4_pack(w, scales, zeros, N, K, group, packed, stream)) return fail(SM_ERR_DEVICE, "%s: launch failed (hip error %d)", who, e);
  return SM_OK;
}

extern "C" int sm_linear_w4(const sm_linear_w4_desc* c, const void* x, const void* packed, const void* bias, const void* residual, void* y, void* stream) {
  const char* who = "sm_linear_w4";
  if (!c) return fail(SM_ERR_INVALID_ARG, "%s: null descriptor", who);
  if (int rc = check_w4(c->N, c->K, c->group, who)) return rc;
  if (c->M < 0 || c->M > (1 << 20)) return fail(SM_ERR_SHAPE, "%s: at most 2^20 rows", who);
  if (c->act != SM_ACT_NONE && c->act != SM_ACT_GELU) return fail(SM_ERR_UNSUPPORTED, "%s: activation none or GELU", who);
  if (c->M == 0) return SM_OK;                       // no rows: nothing is launched
  if (!x || !packed || !y) return fail(SM_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned16(x) || !aligned16(packed) || !aligned16(y) || !aligned16(bias) || !aligned16(residual)) return fail(SM_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", who);
  const Span out = flat(y, 2 * (uint64_t)c->M * c->N);
  for (const Span& in : {flat(x, 2 * (uint64_t)c->M * c->K), flat(packed, w4_packed_bytes(c->N, c->K, c->group)), flat(bias, 2 * (uint64_t)c->N),
                         flat(y == residual ? nullptr : residual, out.width)})
    if (meet(out, in)) return fail(SM_ERR_INVALID_ARG, "%s: y overlaps an operand (it may be the residual)", who);
  LinearW4Args a{x, packed, bias, residual, y, c->M, c->N, c->K, c->group, c->act};
  char label[96] = "";
  if (timing_on()) snprintf(label, sizeof(label), "linear_w4g%d[%d,%d,%d]%s%s", c->group, c->M, c->N, c->K, c->act ? "+gelu" : "", residual ? "+res" : "");
  Timed tm(label, stream);
  if (int e = launch_w4(a, stream)) return fail(SM_ERR_DEVICE, "%s: launch failed (hip error %d)", who, e);
  count_compute();
  return SM_OK;
}
