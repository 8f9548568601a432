// Kernel arguments and launchers of the operators over a paged key / value cache and of the 4-bit Linear.  The launchers
// check nothing (the C-ABI layer does, before anything is enqueued) and return the hipError_t of the launch as an int.
#pragma once
#include <cstddef>
#include <cstdint>

namespace sm {

struct PageTableArgs {
  const int *cached, *fresh, *free_pages, *n_free;
  int *table, *starts, *lens, *positions, *slots, *need;
  int n_req, page, max_pages, n_pages, free_cap, max_tokens;
  int64_t pitch;
};
int launch_page_table(const PageTableArgs& a, void* stream);

constexpr int HN_MAX_PAIRS = 128;
struct HeadNormPart {               // q, k or v: one input and where its rows go
  const void *x, *gamma, *beta; void* y;
  int64_t x_t, x_h, y_page, y_t, y_h;
  int heads, units, paged;          // units: groups of heads that a wave takes at once
};
struct HeadNormArgs {
  uint64_t turn[HN_MAX_PAIRS];      // theta_i / 2 pi as a fraction of 2^64
  HeadNormPart part[3];
  const int *positions, *slots;
  int tokens, d, rot, norm, page, n_slots;
  float eps;
};
int launch_head_norm_rope(HeadNormArgs& a, int dtype, void* stream);

struct PagedAttnArgs {
  const void *q, *k, *v; const int *table, *lens; void* o; float* lse; float* part;
  int n_req, heads_q, heads_kv, d, page, max_pages, n_pages;
  float scale;
  int64_t pitch, q_r, q_h, o_r, o_h, k_page, k_t, k_h, v_page, v_t, v_h;
};
bool paged_attention_fits(int dtype, int n_req, int heads_q, int heads_kv, int d, int64_t max_keys);      // whether one launch can hold the call
size_t paged_attention_workspace(int dtype, int n_req, int heads_q, int heads_kv, int d, int64_t max_keys);
int launch_paged_attention(const PagedAttnArgs& a, int dtype, void* stream, int* launches);

struct LinearW4Args {
  const void *x, *packed, *bias, *residual; void* y;
  int M, N, K, group, act;
};
size_t w4_packed_bytes(int N, int K, int group);
int launch_w4_pack(const void* w, const void* scales, const void* zeros, int N, int K, int group, void* packed, void* stream);
int launch_w4(const LinearW4Args& a, void* stream);

}  // namespace sm
