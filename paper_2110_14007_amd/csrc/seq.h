// Device-side arguments of the sequence operators (page map, page write,
// attention) and the launch functions of their kernels.  Not part of the
// public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tod.h"

namespace tod {

// Division of a 32-bit unsigned number below 2^31 by a constant d >= 1 that is
// known at run time only: n / d = (n * mul) >> 32 >> shift with
// mul = floor(2^(32 + shift) / d) + 1 and 2^shift <= d < 2^(shift + 1).  The
// error term n / 2^(32 + shift) stays below 1 / d for n < 2^31 < 2^32.
struct FastDiv {
  uint32_t d, mul, shift;
};

inline FastDiv fast_div(uint32_t d) {
  FastDiv f{d, 0, 0};
  while ((2ull << f.shift) <= d) ++f.shift;
  const uint64_t m = (1ull << (32 + f.shift)) / d + 1;
  f.mul = m > 0xffffffffull ? 0 : (uint32_t)m;  // d = 2^shift: mul would be 2^32 + 1
  return f;
}

__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f) {
  return (f.mul ? __umulhi(n, f.mul) : n) >> f.shift;
}

struct PageMapArgs {
  const int32_t *cached, *fresh, *free_pages;
  int64_t n_seq, n_free, cols, tokens;
  FastDiv page;
  int32_t *table, *row_start, *pos;
  int64_t *slot, *used;
};

struct PageWriteArgs {
  const void *k, *v;
  int64_t k_row, k_head, v_row, v_head;  // strides in elements
  const int64_t* slot;
  void *k_pages, *v_pages;
  int64_t tokens, slots;  // slots: n_pages * page
  FastDiv page, per_token, per_row;  // 16-byte pieces of a token and of one head's row
  int32_t kv_heads;
};

struct AttnArgs {
  const void *q, *k, *v;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head;  // strides in elements
  const int32_t *row_start, *cached, *table;            // cached, table: paged only
  int64_t cols;
  int32_t n_seq, tokens, n_pages;
  FastDiv page, group;  // rows of a page; query heads per key / value head
  int32_t heads, kv_heads, dim;
  int32_t causal;
  float scale, unscale;  // of q k^T, times log2(e), and its inverse
  void* out;
  float* lse;
  // Sequences of at most skip_rows packed rows are the token kernel's (0: none).
  int32_t skip_rows, token_tail;
  int64_t* token_line;  // [n_seq + 1]
  float2* token_stat;   // [2 workers, skip_rows]
  float* token_o;       // [2 workers, skip_rows, padded dim]
  // Splits of a tile's keys.
  int32_t tile_slots;   // of a key / value head
  int32_t tile_parts;   // most splits of a tile
  uint32_t tile_groups;  // workgroups: slots, heads, splits
  FastDiv parts_div, heads_div;  // by tile_parts and kv_heads
  int32_t part_keys;    // fewest keys of a split
  float2* tile_stat;    // [tiles of all heads, parts, rows]
  float* tile_o;        // [tiles of all heads, parts, rows, padded dim]
};

// Packed rows that the token kernel takes: a product's 32 columns.  (96 tokens over caches of 100
// to 6,000, 8 heads of 128: 228 us, with the tile kernel for them 277; one over 900: 16.6 and 30.)
constexpr int kTokenMaxRows = 32;
// Its workers, a power of two: four waves on each of 256 compute units with 32 KiB of LDS buffers
// each, two with 64 KiB for more than 128 elements.  (Reads of 1.5 GiB by such waves alone: 6.1
// TB/s with four a unit, 5.3 with five, which do not all stay resident, 6.0 with eight of 16 KiB.)
constexpr int64_t token_workers(int32_t dim) { return dim > 128 ? 512 : 1024; }

hipError_t launch_page_map(const PageMapArgs& a, hipStream_t s);
hipError_t launch_page_write(const PageWriteArgs& a, hipStream_t s);
hipError_t launch_attn_tile_f16(const AttnArgs& a, bool paged, hipStream_t s);
hipError_t launch_attn_tile_bf16(const AttnArgs& a, bool paged, hipStream_t s);
hipError_t launch_attn_token_f16(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_token_bf16(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_token_join_f16(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_token_join_bf16(const AttnArgs& a, hipStream_t s);

// Records a call's error for tod_last_error (never throws) and returns it.
tod_status set_error(tod_status s, const char* msg) noexcept;

}  // namespace tod
