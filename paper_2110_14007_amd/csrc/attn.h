// Attention of packed sequences: softmax(scale q k^T) v, one pass over the
// keys with the running maximum and sum of the softmax.
//
// Rows.  The G query heads that share one key / value head are packed into
// the rows of one product: row m of a sequence is token m / G, head m % G of
// the group, so that a sequence of n new tokens has n G rows per key / value
// head and each staged key serves all of them.
//
// Tile.  A workgroup of 4 waves owns kRows = 128 rows, 32 a wave, and walks the
// keys in stages of 64.  v_mfma_f32_32x32x16 takes the keys as A and the
// queries as B, so that lane l holds, for query l % 32, the scores of keys
// 8 (r / 4) + 4 (l / 32) + r % 4 in accumulators r = 0..15: the maximum and
// the sum over the keys are then in-lane but for one exchange between lanes l
// and l + 32.  The second product, O^T = V^T P^T, takes P as its B operand
// right from those registers: the contraction runs over the keys in any
// order, and the one that the accumulators hold is used, 16 of them a product
// (elements 0..3 of lane half h are keys 4h.., elements 4..7 keys 8 + 4h..).
// V^T is read from the row-major stage by the LDS's transposing read (16
// lanes read four rows of 16 columns, and lane i of them gets column i).
//
// Softmax.  In base 2: t = s scale log2(e), p = 2^(t - m).  m follows the
// running maximum only when that has grown by more than 8, so that most
// stages rescale nothing; p is then at most 2^8, far inside fp16's range.  m,
// the sum and O are fp32; p is rounded to the input type for the second
// product (half an ulp each, unbiased, like the inputs' own rounding), while
// the sum takes the unrounded p.
#pragma once

#include "mtile.h"
#include "seq.h"

namespace tod {
namespace attn {

using mt::f32x16;
using mt::Frag;
using mt::mfma;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;
constexpr int kRows = 32 * kWaves;  // rows of a workgroup
constexpr int kKeys = 64;           // keys of a stage
// Before the first visible key: every finite score replaces it.
constexpr float kNoMax = -3.0e38f;
constexpr float kSlack = 8.0f;  // growth of the maximum (log2) that m may lag behind

// What a workgroup works on.
struct Tile {
  int32_t start, n;    // the sequence's first token and its number of tokens
  int32_t row0, rows;  // first packed row of the tile; packed rows of the sequence (n G)
  int32_t keys;        // keys that exist
  int32_t shift;       // token i of the sequence stands at position shift + i
};

// Tile slot b of a key / value head.  Sequence s, whose packed rows begin at
// R_s = row_start[s] G, owns the slots from floor(R_s / kRows) + s on: at
// least as many as it has tiles, whatever the lengths, and the last slot is
// known on the host without them.  After the last sequence comes one without
// keys that holds the rows past row_start[n_seq].  The search takes 64
// candidates a step (one a lane).
__device__ __forceinline__ bool find_tile(const AttnArgs& a, int64_t b, bool paged, Tile* t,
                                          int32_t* seq) {
  const int lane = threadIdx.x & 63;
  auto start_of = [&](int32_t s) {
    return s <= 0 ? 0 : min(max(a.row_start[s], 0), a.tokens);
  };
  auto slot_of = [&](int32_t s) {
    return (int64_t)start_of(s) * (int64_t)a.group.d / kRows + s;
  };
  int32_t lo = 0, span = a.n_seq + 1;  // the answer lies in [lo, lo + span)
  while (span > 1) {
    const int32_t step = (span + 63) / 64;
    const int32_t s = lo + lane * step;
    const bool under = s < lo + span && slot_of(s) <= b;
    const int hit = max(__popcll(__ballot(under)), 1);
    const int32_t end = lo + span;
    lo += (hit - 1) * step;
    span = min(step, end - lo);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const int32_t start = start_of(lo);
  const int32_t end = lo < a.n_seq ? max(start_of(lo + 1), start) : a.tokens;
  const int32_t n = end - start;
  const int64_t row0 = (b - slot_of(lo)) * kRows;
  t->start = start;
  t->n = n;
  t->rows = n * (int32_t)a.group.d;
  if (row0 >= t->rows) return false;
  t->row0 = (int32_t)row0;
  *seq = lo;
  t->shift = 0;
  t->keys = 0;
  if (lo < a.n_seq) {
    if (paged) {
      const int32_t room = (int32_t)(a.cols * a.page.d);
      t->shift = min(max(a.cached[lo], 0), room);
      t->keys = min(t->shift + n, room);
    } else {
      t->keys = n;
    }
  }
  return true;
}

// 16 zero bytes: what a lane stages for a key, or a piece of one, that does not exist.
static __device__ const uint4 kZeros = {0, 0, 0, 0};

template <typename ET>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  typedef ET e2 __attribute__((ext_vector_type(2)));
  e2 v;
  v[0] = (ET)x;
  v[1] = (ET)y;
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ float other_half(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 32) ? p[0] : p[1]);
}

// Stage layout: row-major, DP elements a row, with its 16-byte pieces c at
// c ^ swizzle(row).  K is read by 32 rows at one piece: over any 16 rows that
// differ modulo 16 the pieces fall on different banks.  V is read by the
// transposing read, four rows of 32 bytes at a time.  (Reads measured at
// 320-345 bytes / ns a compute unit for K and 195 for V; with no swizzle 38 and 151.)
template <int DP>
__device__ __forceinline__ int swizzle_k(int row) {
  return DP == 64 ? (row >> 1) & 7 : row & 15;
}
template <int DP>
__device__ __forceinline__ int swizzle_v(int row) {
  return DP == 64 ? 0 : (row & 3) << 1;
}

template <typename ET, int DP, bool PAGED>
__global__ void __launch_bounds__(64 * kWaves) tile_kernel(AttnArgs a) {
  using V8 = typename Frag<ET>::V;
  constexpr int kPieces = DP / 8;             // 16-byte pieces of a row
  constexpr int kStage = kKeys * DP;          // elements of a stage
  constexpr int kLoads = kPieces / kWaves;    // staging loads of a lane, each for K and V
  constexpr int kRowsLoad = 64 / kPieces;     // rows of one staging load
  constexpr int KC = DP / 16;                 // steps of the first product
  constexpr int DB = DP / 32;                 // 32-column blocks of O
  extern __shared__ __align__(16) uint16_t lds[];  // two buffers of a K and a V stage

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, h = lane >> 5;
  const uint32_t head = blockIdx.x % (uint32_t)a.kv_heads;
  // Late rows see the most keys: they are taken first.
  const int64_t slot =
      (int64_t)(gridDim.x / (uint32_t)a.kv_heads) - 1 - blockIdx.x / (uint32_t)a.kv_heads;
  Tile t;
  int32_t seq;
  if (!find_tile(a, slot, PAGED, &t, &seq)) return;

  // This lane's query row, and the last key that it sees.
  const int32_t m = min(t.row0 + 32 * wave + col, t.rows - 1);
  const int32_t tok = (int32_t)div_by((uint32_t)m, a.group);
  const int32_t qh = (int32_t)head * (int32_t)a.group.d + m - tok * (int32_t)a.group.d;
  const bool bounded = PAGED || a.causal;
  const int32_t limit = bounded ? min(t.shift + tok, t.keys - 1) : t.keys - 1;
  // Over the wave, and the number of keys that some row of the workgroup sees.
  const int32_t wlo = __builtin_amdgcn_readfirstlane(limit);
  const int32_t whi = __builtin_amdgcn_readlane(limit, 31);
  const int32_t last = (int32_t)div_by((uint32_t)min(t.row0 + kRows - 1, t.rows - 1), a.group);
  const int32_t seen = bounded ? min(t.shift + last + 1, t.keys) : t.keys;

  V8 q[KC];
  {
    const ET* const p = (const ET*)a.q + (int64_t)(t.start + tok) * a.q_row +
                        (int64_t)qh * a.q_head;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const int e = 16 * c + 8 * h;
      q[c] = e < a.dim ? *(const V8*)(p + e) : V8{};
    }
  }

  // Staging.  Lane l of a wave finds where the stage's key l lies; a load moves
  // 16 bytes a lane, kRowsLoad rows a wave.
  auto place = [&](int32_t j0) -> uint32_t {  // row of the cache, ~0: none
    const int32_t j = j0 + lane;
    if (j >= seen) return ~0u;
    if constexpr (PAGED) {
      const uint32_t pg = div_by((uint32_t)j, a.page);
      const int32_t id = a.table[(int64_t)seq * a.cols + pg];
      if (id < 0 || id >= a.n_pages) return ~0u;
      return ((uint32_t)id * (uint32_t)a.kv_heads + head) * a.page.d + ((uint32_t)j - pg * a.page.d);
    } else {
      return (uint32_t)(t.start + j);
    }
  };
  auto stage = [&](int buf, uint32_t at) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r0 = (wave * kLoads + i) * kRowsLoad;
      const int r = r0 + lane / kPieces;
      const uint32_t row = (uint32_t)__shfl((int)at, r, 64);
      const int pc = lane % kPieces;
      const int ck = pc ^ swizzle_k<DP>(r), cv = pc ^ swizzle_v<DP>(r);
      const ET *kp, *vp;
      if constexpr (PAGED) {
        kp = (const ET*)a.k + (int64_t)row * a.dim;
        vp = (const ET*)a.v + (int64_t)row * a.dim;
      } else {
        kp = (const ET*)a.k + (int64_t)row * a.k_row + (int64_t)head * a.k_head;
        vp = (const ET*)a.v + (int64_t)row * a.v_row + (int64_t)head * a.v_head;
      }
      const bool ok = row != ~0u;
      const void* const ks = ok && 8 * ck < a.dim ? (const void*)(kp + 8 * ck) : &kZeros;
      const void* const vs = ok && 8 * cv < a.dim ? (const void*)(vp + 8 * cv) : &kZeros;
      const uint32_t to = mt::lds_off(lds) + 2u * (uint32_t)(2 * buf * kStage + r0 * DP);
      mt::dma16(ks, to);
      mt::dma16(vs, to + 2u * kStage);
    }
  };

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
  float mref = kNoMax, sum = 0.0f;

  const int32_t stages = (seen + kKeys - 1) / kKeys;
  if (stages > 0) stage(0, place(0));
  for (int32_t j = 0; j < stages; ++j) {
    const int buf = j & 1;
    mt::dl_barrier<0>();
    if (j + 1 < stages) stage(buf ^ 1, place((j + 1) * kKeys));
    const int32_t j0 = j * kKeys;
    if (j0 > whi) continue;  // nothing that this wave's rows see
    const uint16_t* const ks = lds + 2 * buf * kStage;
    const uint16_t* const vs = ks + kStage;

    f32x16 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kt][r] = 0.0f;
      const int row = 32 * kt + col;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const V8 k = *(const V8*)(ks + row * DP + 8 * ((2 * c + h) ^ swizzle_k<DP>(row)));
        s[kt] = mfma<ET>(k, q[c], s[kt]);
      }
    }
    if (j0 + kKeys - 1 > wlo) {  // some row of the wave does not see some key
      int32_t left = limit - j0 - 4 * h;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kt + mt::out_row_c(r) > left) s[kt][r] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kt][r]);
    top = fmaxf(top, other_half(top)) * a.scale;
    const bool grow = top > mref + kSlack;
    if (__ballot(grow)) {
      const float next = grow ? top : mref;
      const float f = __builtin_amdgcn_exp2f(mref - next);
      mref = next;
      sum *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= f;
    }
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][r], a.scale, -mref));
        sum += p;
        s[kt][r] = p;
      }
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        u32x4 pw;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          pw[e] = pack2<ET>(s[kt][8 * c + 2 * e], s[kt][8 * c + 2 * e + 1]);
        const V8 p = __builtin_bit_cast(V8, pw);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          // Lane i of 16 reads row i / 4, columns 4 (i % 4).. of its four rows.
          const int row = 32 * kt + 16 * c + 4 * h + (lane & 15) / 4;
          const int piece = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
          const int within = 4 * (lane & 1);
          typedef __attribute__((address_space(3))) s16x4* lds4;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds4)(vs + row * DP + 8 * (piece ^ swizzle_v<DP>(row)) + within));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds4)(vs + (row + 8) * DP + 8 * (piece ^ swizzle_v<DP>(row + 8)) + within));
          const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          o[d] = mfma<ET>(__builtin_bit_cast(V8, v), p, o[d]);
        }
      }
  }

  sum += other_half(sum);
  const bool mine = t.row0 + 32 * wave + col < t.rows;
  if (!mine) return;
  const float inv = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);
  const int64_t orow = (int64_t)(t.start + tok) * a.heads + qh;
  ET* const op = (ET*)a.out + orow * a.dim;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int e = 32 * d + 8 * g + 4 * h;
      if (e < a.dim) {
        uint2 w;
        w.x = pack2<ET>(o[d][4 * g] * inv, o[d][4 * g + 1] * inv);
        w.y = pack2<ET>(o[d][4 * g + 2] * inv, o[d][4 * g + 3] * inv);
        *(uint2*)(op + e) = w;
      }
    }
  if (a.lse && h == 0)
    a.lse[orow] = sum == 0.0f ? -INFINITY
                              : (mref + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
}

template <typename ET, int DP, bool PAGED>
hipError_t launch_tile(const AttnArgs& a, hipStream_t s) {
  const int64_t slots = (int64_t)a.tokens * a.group.d / kRows + a.n_seq + 1;
  constexpr unsigned bytes = 2 * 2 * kKeys * DP * 2;  // two buffers, K and V, 16 bits
  const auto kern = tile_kernel<ET, DP, PAGED>;
  if constexpr (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(
        (const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)(slots * a.kv_heads)), dim3(64 * kWaves), bytes, s, a);
  return hipGetLastError();
}

template <typename ET>
hipError_t launch_any(const AttnArgs& a, bool paged, hipStream_t s) {
  if (a.dim <= 64)
    return paged ? launch_tile<ET, 64, true>(a, s) : launch_tile<ET, 64, false>(a, s);
  if (a.dim <= 128)
    return paged ? launch_tile<ET, 128, true>(a, s) : launch_tile<ET, 128, false>(a, s);
  return paged ? launch_tile<ET, 256, true>(a, s) : launch_tile<ET, 256, false>(a, s);
}

}  // namespace attn
}  // namespace tod
