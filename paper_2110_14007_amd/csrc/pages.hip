// Paged key / value cache: the map from request lengths to pages and slots,
// and the write of new keys and values into their slots.
#include "seq.h"

namespace tod {
namespace {

constexpr int kMapThreads = 256;
constexpr int kMapTokens = 1024;  // tokens of one workgroup

// ceil(n / P) for 0 <= n < 2^31.
__device__ __forceinline__ int32_t pages_up(int32_t n, const FastDiv& page) {
  return n == 0 ? 0 : (int32_t)div_by((uint32_t)n - 1u, page) + 1;
}

// Exclusive prefix sum of one value per thread, and the workgroup's total.
template <typename T>
__device__ __forceinline__ T block_prefix(T v, T* total, int64_t* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kMapThreads / 64; ++w) {
    if (w < wave) before += (T)lds[w];
    all += (T)lds[w];
  }
  *total = all;
  return before + x - v;
}

// Each workgroup maps kMapTokens tokens.  All of them form the prefix sums of
// the fresh tokens and of the needed pages over all requests for themselves
// (8 bytes a request from L2), which costs less than a second launch or a wait
// between workgroups.  A request's first token in the workgroup's range leaves
// a marker at its place; a running maximum over the places then gives every
// token its request.  A token that opens a page writes the table's entry, so
// long requests are spread over many threads.  A thread takes EACH neighbouring
// requests of a round.  Bound by latency: launch, the lengths, two prefix sums.
// 4.3 us for 48 requests of one token, 10.8 us for 2,000 with 54,900.
template <int EACH>
__global__ void __launch_bounds__(kMapThreads) page_map_kernel(PageMapArgs a) {
  __shared__ int64_t sums[kMapThreads / 64];
  __shared__ int32_t mark[kMapTokens];   // place of the token's request's first token here
  __shared__ int32_t who[kMapTokens];    // at such a place: the request,
  __shared__ int32_t start_of[kMapTokens], page_of[kMapTokens];  // its first token and page
  const int tid = threadIdx.x;
  const int32_t tokens = (int32_t)a.tokens;
  const int32_t t0 = (int32_t)blockIdx.x * kMapTokens;
  const int32_t count = min(kMapTokens, tokens - t0);  // (t0 + kMapTokens may be 2^31)
  const int32_t t1 = t0 + count;
  const int32_t room = (int32_t)(a.cols * a.page.d);  // positions that the table holds
  const bool first = blockIdx.x == 0;
  for (int i = tid; i < kMapTokens; i += kMapThreads) mark[i] = -1;

  // The requests in rounds of kMapThreads * EACH, with the sums so far in front.  Workgroups but
  // the first leave when a round ends past their tokens.  The fresh tokens are summed in 64 bits;
  // from there on all is cut to `tokens` and to the table, below 2^31.
  int64_t sum_fresh = 0, sum_need = 0, lost = 0;
  for (int64_t q0 = 0; q0 < a.n_seq; q0 += kMapThreads * EACH) {
    const int64_t r0 = q0 + tid * EACH;
    int32_t c[EACH], f[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const bool in = r0 + i < a.n_seq;
      c[i] = in ? max(a.cached[r0 + i], 0) : 0;
      f[i] = in ? max(a.fresh[r0 + i], 0) : 0;
    }
    int64_t mine = 0, all;
#pragma unroll
    for (int i = 0; i < EACH; ++i) mine += f[i];
    int64_t at = sum_fresh + block_prefix(mine, &all, sums);
    sum_fresh += all;
    // With c cached and g new tokens (cut to the room for tokens), P rows a page, C columns:
    //   have = min(ceil(c / P), C),  need = min(ceil((c + g) / P), C) - have.
    int32_t start[EACH], g[EACH], have[EACH], need[EACH], sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      start[i] = (int32_t)min(at, (int64_t)tokens);
      g[i] = min(f[i], tokens - start[i]);
      at += f[i];
      have[i] = pages_up(min(c[i], room), a.page);
      need[i] = pages_up((int32_t)min((uint32_t)c[i] + (uint32_t)g[i], (uint32_t)room), a.page) -
                have[i];
      sum += need[i];
    }
    int32_t last[EACH];  // the table's entry of the page that the cached tokens end in
    if (first) {
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        last[i] = a.table[min(r0 + i, a.n_seq - 1) * a.cols + max(have[i] - 1, 0)];
    }
    int32_t pages;  // (at most one a token)
    int64_t base = sum_need + block_prefix(sum, &pages, sums);
    sum_need += pages;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int64_t r = r0 + i;
      if (g[i] > 0 && start[i] < t1 && start[i] + g[i] > t0) {
        const int place = max(start[i], t0) - t0;
        mark[place] = place;
        who[place] = (int32_t)r;
        start_of[place] = start[i];
        page_of[place] = (int32_t)base - have[i];  // free page of column c: page_of + c
      }
      if (first && r < a.n_seq) {
        a.row_start[r] = start[i];
        // Tokens without a slot: cut off, past the pages, or in a page that the table lacks.
        const int64_t end = (int64_t)c[i] + g[i];
        const int64_t got = have[i] + min(max(a.n_free - base, (int64_t)0), (int64_t)need[i]);
        lost += f[i] - g[i] + max(end - max((int64_t)c[i], got * a.page.d), (int64_t)0);
        const int64_t begun = (int64_t)have[i] * a.page.d;
        if (g[i] > 0 && c[i] < begun && last[i] < 0) lost += min((int64_t)g[i], begun - c[i]);
      }
      base += need[i];
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

  // Four tokens a thread, their loads side by side.
  int32_t pos[kPlaces], page[kPlaces], in[kPlaces];
  int32_t* entry[kPlaces];
#pragma unroll
  for (int k = 0; k < kPlaces; ++k) {
    const int i = tid + k * kMapThreads;
    const int place = mark[i];
    const bool live = place >= 0 && i < count && t0 + i < sum_fresh;
    const int64_t r = live ? who[place] : 0;
    const int32_t c = max(a.cached[r], 0);
    const int64_t at = (int64_t)c + (live ? t0 + i - start_of[place] : 0);
    pos[k] = live ? (int32_t)min(at, (int64_t)0x7fffffff) : -1;
    page[k] = -1;
    entry[k] = nullptr;
    in[k] = 0;
    if (live && at < room) {
      const int32_t col = (int32_t)div_by((uint32_t)at, a.page), opens = col * (int32_t)a.page.d;
      in[k] = (int32_t)at - opens;
      if (opens < c) {
        page[k] = a.table[r * a.cols + col];  // begun before this step
      } else {
        const int32_t g = page_of[place] + col;
        if (g < a.n_free) page[k] = a.free_pages[g];
        if (in[k] == 0) entry[k] = a.table + r * a.cols + col;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kPlaces; ++k) {
    const int32_t i = tid + k * kMapThreads, t = t0 + i;
    if (i >= count) break;
    if (entry[k]) *entry[k] = page[k];
    a.slot[t] = page[k] >= 0 ? (int64_t)page[k] * a.page.d + in[k] : -1;
    if (a.pos) a.pos[t] = pos[k];
  }
}

// One thread moves 16 bytes of a key row and of its value row.  Bound by the
// bytes: 4 d a token and head in each direction.  48 tokens of 8 heads of 128
// take 2.6 us (a launch), 20,011 of them 25 us (6.6 TB/s of both directions).
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
  // One request a thread while one round takes them all: its chain is the shortest (48 requests
  // 4.2 us, eight a thread 7.0).  Beyond that eight, for fewer rounds (2,000 requests 10.7 us, one
  // a thread 14.3).
  const auto kern = a.n_seq <= kMapThreads ? page_map_kernel<1> : page_map_kernel<8>;
  hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(kMapThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_page_write(const PageWriteArgs& a, hipStream_t s) {
  const int64_t pieces = a.tokens * a.per_token.d;
  hipLaunchKernelGGL(page_write_kernel, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, s,
                     a);
  return hipGetLastError();
}

}  // namespace tod
