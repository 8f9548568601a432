// Page table and slot map of a serving iteration from the lengths of its requests (device arrays), one launch.
//
// Two exclusive sums over the requests decide everything: of the new tokens (the first row of a request) and of the pages
// that these open (where the request's share of the free list begins).  Every workgroup computes both by itself, 256
// segments of requests at a time in LDS (reading 8 bytes a request from the L2 is cheaper than a second launch, and no
// workgroup waits for another), then finds the request of each of its token rows by bisection.  A page that opens does so
// at exactly one new token, the one at a multiple of the page size: that token's thread writes the table entry.
#include <algorithm>
#include "device_common.h"
#include "paged.h"

namespace sm {

namespace {
struct PtRequest { int c, f, old, n; };      // cached tokens, new tokens with a row, pages there are, pages that open
__device__ __forceinline__ PtRequest pt_request(const PageTableArgs& a, int r, int start) {
  PtRequest q;
  const int row = a.max_pages * a.page;
  q.c = min(max(a.cached[r], 0), row);
  q.f = min(max(a.fresh[r], 0), a.max_tokens - start);
  const int end = (int)min((unsigned)q.c + q.f, (unsigned)row);      // (two numbers up to 2^30)
  q.old = (q.c + a.page - 1) / a.page;
  q.n = (end + a.page - 1) / a.page - q.old;
  return q;
}

// exclusive sum of v over the workgroup's threads into out[0 .. PT_THREADS], every partial sum cut at cap (v and cap at most 2^30)
template <int PT_THREADS>
__device__ __forceinline__ void pt_scan(int v, int cap, int* out) {
  __shared__ unsigned waves[PT_THREADS / 64];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  unsigned s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned u = __shfl_up(s, o, 64);
    if (lane >= o) s = min(s + u, (unsigned)cap);
  }
  if (lane == 63) waves[w] = s;
  __syncthreads();
  unsigned before = 0;
  for (int i = 0; i < w; ++i) before = min(before + waves[i], (unsigned)cap);
  if (tid == 0) out[0] = 0;
  out[tid + 1] = (int)min(before + s, (unsigned)cap);
  __syncthreads();
}
}  // namespace

template <int PT_THREADS>
__global__ __launch_bounds__(PT_THREADS) void page_table_kernel(PageTableArgs a) {
  __shared__ int s_start[PT_THREADS + 1], s_base[PT_THREADS + 1];
  const int tid = threadIdx.x, per = (a.n_req + PT_THREADS - 1) / PT_THREADS;
  const int r0 = min(a.n_req, tid * per), r1 = min(a.n_req, r0 + per);
  unsigned sum = 0;
  for (int r = r0; r < r1; ++r) sum = min(sum + min(max(a.fresh[r], 0), a.max_tokens), (unsigned)a.max_tokens);
  pt_scan<PT_THREADS>((int)sum, a.max_tokens, s_start);
  int start = s_start[tid], pages = 0;
  for (int r = r0; r < r1; ++r) {
    const PtRequest q = pt_request(a, r, start);
    start += q.f; pages += q.n;
  }
  pt_scan<PT_THREADS>(pages, 1 << 30, s_base);
  const int total = s_start[PT_THREADS], free = min(max(*a.n_free, 0), a.free_cap);
  if (blockIdx.x == 0) {
    int base = s_base[tid];
    start = s_start[tid];
    for (int r = r0; r < r1; ++r) {
      const PtRequest q = pt_request(a, r, start);
      const int got = min(max(free - base, 0), q.n);
      const int end = (int)min((unsigned)q.c + q.f, (unsigned)(a.max_pages * a.page));
      a.starts[r] = start;
      a.lens[r] = got == q.n ? end : min(end, (q.old + got) * a.page);
      start += q.f; base += q.n;
    }
    if (tid == 0) { a.starts[a.n_req] = total; *a.need = s_base[PT_THREADS]; }
  }
  const int64_t t = (int64_t)blockIdx.x * PT_THREADS + tid;
  if (t >= a.max_tokens) return;
  int pos = -1, slot = -1;
  if (t < total) {
    int lo = 0;                                // the last segment that starts at or before t: it has the row, the ones behind do not
#pragma unroll
    for (int h = PT_THREADS / 2; h > 0; h >>= 1) if (s_start[lo + h] <= t) lo += h;
    int first = s_start[lo], base = s_base[lo], r = lo * per;
    PtRequest q = pt_request(a, r, first);
    while (t >= first + q.f) { first += q.f; base += q.n; q = pt_request(a, ++r, first); }
    pos = q.c + ((int)t - first);
    const int pg = pos / a.page, in = pos - pg * a.page;
    int id = -1;
    if (pg < q.old) id = a.table[r * a.pitch + pg];
    else if (pg < a.max_pages && base + pg - q.old < free) {
      id = a.free_pages[base + pg - q.old];
      if (in == 0) a.table[r * a.pitch + pg] = id;
    }
    if (id >= 0 && id < a.n_pages) slot = id * a.page + in;
  }
  a.positions[t] = pos;
  a.slots[t] = slot;
}

int launch_page_table(const PageTableArgs& a, void* stream) {
  // large workgroups from three requests a thread on (2000 requests with a token each: 7.6 us instead of 10.1; 600: 5.6 instead of 5.3)
  const int threads = a.n_req <= 768 ? 256 : 1024, blocks = std::max(1, (a.max_tokens + threads - 1) / threads);
  if (threads == 256) page_table_kernel<256><<<dim3(blocks), dim3(256), 0, (hipStream_t)stream>>>(a);
  else page_table_kernel<1024><<<dim3(blocks), dim3(1024), 0, (hipStream_t)stream>>>(a);
  return (int)hipGetLastError();
}

}  // namespace sm
