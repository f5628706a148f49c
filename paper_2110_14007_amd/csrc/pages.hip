// Paged key / value cache: the map from request lengths to pages and slots,
// and the write of new keys and values into their slots.
#include "seq.h"

namespace tod {
namespace {

constexpr int kMapThreads = 256;
constexpr int kMapTokens = 1024;  // tokens of one workgroup

// Exclusive prefix sum of one value per thread, and the workgroup's total.
__device__ __forceinline__ int64_t block_prefix(int64_t v, int64_t* total, int64_t* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kMapThreads / 64; ++w) {
    if (w < wave) before += lds[w];
    all += lds[w];
  }
  *total = all;
  return before + x - v;
}

// One request's pages.  With c cached and f fresh tokens (cut to the room for
// tokens), P rows a page and C table columns:
//   have = min(ceil(c / P), C),  need = min(ceil((c + f) / P), C) - have.
struct Pages {
  int64_t c, f, have, need;
};

// ceil(n / P) for 0 <= n < 2^31.
__device__ __forceinline__ int64_t pages_up(int64_t n, const FastDiv& page) {
  return n == 0 ? 0 : (int64_t)div_by((uint32_t)n - 1u, page) + 1;
}

__device__ __forceinline__ Pages pages_of(const PageMapArgs& a, int32_t cached, int32_t fresh,
                                          int64_t start) {
  Pages p;
  p.c = cached;
  p.f = min((int64_t)fresh, max(a.tokens - start, (int64_t)0));
  // Positions past the table need no more pages than it has columns; cols * P < 2^31.
  const int64_t end = a.cols * a.page.d;
  p.have = pages_up(min(p.c, end), a.page);
  p.need = pages_up(min(p.c + p.f, end), a.page) - p.have;
  return p;
}

// Each workgroup maps kMapTokens tokens.  All of them form the prefix sums of
// the fresh tokens and of the needed pages over all requests for themselves
// (8 bytes a request from L2), which costs less than a second launch or a wait
// between workgroups.  A request's first token in the workgroup's range leaves
// a marker at its place; a running maximum over the places then gives every
// token its request.  A token that opens a page writes the table's entry, so
// long requests are spread over many threads.
// 2,000 requests and 54,900 tokens, 55 workgroups: see the measurements with the operators.
__global__ void __launch_bounds__(kMapThreads) page_map_kernel(PageMapArgs a) {
  __shared__ int64_t sums[kMapThreads / 64];
  __shared__ int32_t mark[kMapTokens];   // place of the token's request's first token here
  __shared__ int32_t who[kMapTokens];    // at such a place: the request,
  __shared__ int64_t start_of[kMapTokens], page_of[kMapTokens];  // its first token and page
  const int tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * kMapTokens;
  const int64_t t1 = min(t0 + kMapTokens, a.tokens);
  const bool first = blockIdx.x == 0;
  for (int i = tid; i < kMapTokens; i += kMapThreads) mark[i] = -1;

  // The sequences in rounds of kMapThreads * kEach, kEach neighbours a thread, with the sums so
  // far in front.  Workgroups but the first leave when a round ends past their tokens.
  constexpr int kEach = 8;
  int64_t sum_fresh = 0, sum_need = 0, lost = 0;
  for (int64_t q0 = 0; q0 < a.n_seq; q0 += kMapThreads * kEach) {
    const int64_t r0 = q0 + tid * kEach;
    int32_t c[kEach], f[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const bool in = r0 + i < a.n_seq;
      c[i] = in ? max(a.cached[r0 + i], 0) : 0;
      f[i] = in ? max(a.fresh[r0 + i], 0) : 0;
    }
    int64_t mine = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) mine += f[i];
    int64_t start = sum_fresh + block_prefix(mine, &all, sums);
    sum_fresh += all;
    const int64_t start0 = start;
    mine = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      mine += pages_of(a, c[i], f[i], start).need;
      start += f[i];
    }
    int64_t base = sum_need + block_prefix(mine, &all, sums);
    sum_need += all;
    start = start0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int64_t r = r0 + i;
      const Pages p = pages_of(a, c[i], f[i], start);
      if (p.f > 0 && start < t1 && start + p.f > t0) {
        const int at = (int)(max(start, t0) - t0);
        mark[at] = at;
        who[at] = (int32_t)r;
        start_of[at] = start;
        page_of[at] = base - p.have;  // free page of column c: page_of + c
      }
      if (first && r < a.n_seq) {
        a.row_start[r] = (int32_t)min(start, a.tokens);
        // Tokens without a slot: cut off, past the pages, or in a page that the table lacks.
        const int64_t got = p.have + min(max(a.n_free - base, (int64_t)0), p.need);
        lost += f[i] - p.f + max(p.c + p.f - max(p.c, got * a.page.d), (int64_t)0);
        // The column of the first new token, if its page was begun before.
        const int64_t open = p.have - 1;
        if (p.f > 0 && p.c < p.have * a.page.d && a.table[r * a.cols + open] < 0)
          lost += min(p.f, p.have * a.page.d - p.c);
      }
      base += p.need;
      start += f[i];
    }
    if (!first && sum_fresh >= t1) break;
  }
  if (first) {
    int64_t lost_all;
    block_prefix(lost, &lost_all, sums);
    if (tid == 0) {
      a.row_start[a.n_seq] = (int32_t)min(sum_fresh, a.tokens);
      if (a.used) {
        a.used[0] = sum_need;
        a.used[1] = lost_all;
      }
    }
  }
  __syncthreads();

  // Running maximum of the markers: four places a thread, then over the threads.
  constexpr int kPlaces = kMapTokens / kMapThreads;
  int m[kPlaces], top = -1;
#pragma unroll
  for (int i = 0; i < kPlaces; ++i) m[i] = top = max(top, mark[tid * kPlaces + i]);
  const int lane = tid & 63, wave = tid >> 6;
  int x = top;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x = max(x, y);
  }
  int prev = __shfl_up(x, 1, 64);
  if (lane == 0) prev = -1;
  __syncthreads();
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  for (int w = 0; w < wave; ++w) prev = max(prev, (int)sums[w]);
#pragma unroll
  for (int i = 0; i < kPlaces; ++i) mark[tid * kPlaces + i] = max(prev, m[i]);
  __syncthreads();

  for (int i = tid; i < (int)(t1 - t0); i += kMapThreads) {
    const int64_t t = t0 + i;
    const int at = mark[i];
    int64_t slot = -1, pos = -1;
    if (at >= 0 && t < sum_fresh) {
      const int64_t r = who[at];
      const int64_t c = max(a.cached[r], 0);
      pos = c + (t - start_of[at]);
      if (pos < a.cols * a.page.d) {
        const int64_t col = div_by((uint32_t)pos, a.page), in = pos - col * a.page.d;
        int32_t* const entry = a.table + r * a.cols + col;
        int32_t page;
        if (col * a.page.d < c) {
          page = *entry;  // begun before this step
        } else {
          const int64_t g = page_of[at] + col;
          page = g < a.n_free ? a.free_pages[g] : -1;
          if (in == 0) *entry = page;
        }
        if (page >= 0) slot = (int64_t)page * a.page.d + in;
      }
    }
    a.slot[t] = slot;
    if (a.pos) a.pos[t] = (int32_t)min(pos, (int64_t)0x7fffffff);
  }
}

// One thread moves 16 bytes of a key row and of its value row.  Bound by the
// bytes: 4 d a token and head in each direction.
__global__ void __launch_bounds__(256) page_write_kernel(PageWriteArgs a) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  const uint32_t t = div_by(i, a.per_token);
  if (t >= (uint32_t)a.tokens) return;
  const int64_t slot = a.slot[t];
  if (slot < 0 || slot >= a.slots) return;
  const uint32_t in = i - t * a.per_token.d;
  const uint32_t h = div_by(in, a.per_row), c = in - h * a.per_row.d;
  const uint32_t page = div_by((uint32_t)slot, a.page), row = (uint32_t)slot - page * a.page.d;
  const int64_t to = (((int64_t)page * a.kv_heads + h) * a.page.d + row) * a.per_row.d + c;
  const uint4 kv = *(const uint4*)((const uint16_t*)a.k + t * a.k_row + h * a.k_head + 8 * c);
  const uint4 vv = *(const uint4*)((const uint16_t*)a.v + t * a.v_row + h * a.v_head + 8 * c);
  ((uint4*)a.k_pages)[to] = kv;
  ((uint4*)a.v_pages)[to] = vv;
}

}  // namespace

hipError_t launch_page_map(const PageMapArgs& a, hipStream_t s) {
  const int64_t blocks = (a.tokens + kMapTokens - 1) / kMapTokens;
  hipLaunchKernelGGL(page_map_kernel, dim3((unsigned)blocks), dim3(kMapThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_page_write(const PageWriteArgs& a, hipStream_t s) {
  const int64_t pieces = a.tokens * a.per_token.d;
  hipLaunchKernelGGL(page_write_kernel, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, s,
                     a);
  return hipGetLastError();
}

}  // namespace tod
