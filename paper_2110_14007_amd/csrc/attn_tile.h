// Attention tile: whole prompts, and chunks of new tokens over pages.
//
// A workgroup of 4 waves owns kRows = 128 packed rows of one key / value head,
// 32 a wave, and walks the keys in stages of 64, double-buffered: the next
// stage's loads are in flight while the current one is consumed, one barrier
// a stage.  Where a call has too few tiles for the GPU, each tile's keys are
// split over several workgroups and a second kernel joins their results.
#pragma once

#include "attn.h"

namespace tod {
namespace attn {

constexpr int kWaves = 4;
constexpr int kRows = 32 * kWaves;  // rows of a workgroup
constexpr int kKeys = 64;           // keys of a stage
constexpr float kSlack = 8.0f;  // growth of the maximum (log2) that m may lag behind
constexpr int kMinStages = 8;   // of a split

// What a workgroup works on.
struct Tile : Seq {
  int32_t seq, row0, rows;  // first packed row of the tile; packed rows of the sequence (n G)
  int32_t seen;             // keys that some row of the tile sees
  int32_t stages, parts;    // stages of those keys, and the splits that share them
};

// Tile slot b of a key / value head.  Sequence s, whose packed rows begin at
// R_s = row_start[s] G, owns the slots from floor(R_s / kRows) + s on: at
// least as many as it has tiles, whatever the lengths, and the last slot is
// known on the host without them.  The search takes 64 candidates a step (one
// a lane).  Sequences of at most skip_rows rows are the token kernel's.
template <bool PAGED>
__device__ __forceinline__ bool find_tile(const AttnArgs& a, int64_t b, Tile* t) {
  const int lane = threadIdx.x & 63;
  auto slot_of = [&](int32_t s) {
    return (int64_t)start_of(a, s) * (int64_t)a.group.d / kRows + s;
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
  *(Seq*)t = seq_of<PAGED>(a, lo);
  const int64_t row0 = (b - slot_of(lo)) * kRows;
  t->seq = lo;
  t->rows = t->n * (int32_t)a.group.d;
  if (row0 >= t->rows || (lo < a.n_seq && t->rows <= a.skip_rows)) return false;
  t->row0 = (int32_t)row0;
  const int32_t last = (int32_t)div_by((uint32_t)min(t->row0 + kRows - 1, t->rows - 1), a.group);
  t->seen = PAGED || a.causal ? min(t->shift + last + 1, t->keys) : t->keys;
  t->stages = (t->seen + kKeys - 1) / kKeys;
  t->parts = max(min(a.tile_parts, t->stages / kMinStages), 1);
  return true;
}

template <typename ET, int DP, bool PAGED>
__global__ void __launch_bounds__(64 * kWaves) tile_kernel(AttnArgs a) {
  using V8 = typename Frag<ET>::V;
  using St = Stager<ET, DP, PAGED>;
  constexpr int kStage = kKeys * DP;        // elements of a stage
  constexpr int kRowsWave = kKeys / kWaves;  // rows of a stage that a wave loads
  constexpr int DB = DP / 32;               // 32-column blocks of O
  extern __shared__ __align__(16) uint16_t lds[];  // two buffers of a K and a V stage

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, h = lane >> 5;
  uint32_t b = blockIdx.x;
  const uint32_t part = b % (uint32_t)a.tile_parts;
  b /= (uint32_t)a.tile_parts;
  const uint32_t head = b % (uint32_t)a.kv_heads;
  const int64_t slots = gridDim.x / ((uint32_t)a.kv_heads * (uint32_t)a.tile_parts);
  // Late rows see the most keys: they are taken first.
  const int64_t slot = slots - 1 - b / (uint32_t)a.kv_heads;
  Tile t;
  if (!find_tile<PAGED>(a, slot, &t) || (int)part >= t.parts) return;
  const int32_t jb = (int32_t)((int64_t)t.stages * part / t.parts);
  const int32_t je = (int32_t)((int64_t)t.stages * (part + 1) / t.parts);

  // This lane's query row, and the last key that it sees.
  const int32_t m = min(t.row0 + 32 * wave + col, t.rows - 1);
  const int32_t tok = (int32_t)div_by((uint32_t)m, a.group);
  const int32_t qh = (int32_t)head * (int32_t)a.group.d + m - tok * (int32_t)a.group.d;
  const int32_t limit = PAGED || a.causal ? min(t.shift + tok, t.keys - 1) : t.keys - 1;
  const int32_t wlo = __builtin_amdgcn_readfirstlane(limit);  // over the wave
  const int32_t whi = __builtin_amdgcn_readlane(limit, 31);

  V8 q[DP / 16];
  load_query<ET, DP>(q, (const ET*)a.q + (int64_t)(t.start + tok) * a.q_row + (int64_t)qh * a.q_head,
                     a.dim, h);

  St st(a, head);
  st.seq = t.seq;
  st.start = t.start;
  st.seen = t.seen;
  const uint32_t base = mt::lds_off(lds);
  auto stage = [&](int32_t j) {
    const uint32_t at = st.place(j * kKeys, kKeys);
    const uint32_t k = base + 4u * kStage * (uint32_t)(j & 1);
#pragma unroll
    for (int i = 0; i < kRowsWave / St::kRowsLoad; ++i)
      st.load(at, wave * kRowsWave + i * St::kRowsLoad, k, k + 2u * kStage);
  };

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
  float mref = kNoMax, sum = 0.0f;

  if (jb < je) stage(jb);
  for (int32_t j = jb; j < je; ++j) {
    mt::dl_barrier<0>();
    if (j + 1 < je) stage(j + 1);
    const int32_t j0 = j * kKeys;
    if (j0 > whi) continue;  // nothing that this wave's rows see
    const uint16_t* const ks = lds + 2 * (j & 1) * kStage;
    const uint16_t* const vs = ks + kStage;

    f32x16 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) s[kt] = scores<ET, DP>(ks, 32 * kt, q);
    if (j0 + kKeys - 1 > wlo) {  // some row of the wave does not see some key
      const int32_t left = limit - j0 - 4 * h;
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
    // m follows the maximum only when that has grown by more than kSlack, so
    // that most stages rescale nothing; p is then at most 2^8, far inside
    // fp16's range.
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
    // p is rounded to the input type for the second product (half an ulp each,
    // unbiased, like the inputs' own rounding): two products of its halves
    // would cost half again as many MFMAs as the tile has.
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        u32x4 pw;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          pw[e] = pack2<ET>(s[kt][8 * c + 2 * e], s[kt][8 * c + 2 * e + 1]);
        const V8 p = __builtin_bit_cast(V8, pw);
#pragma unroll
        for (int d = 0; d < DB; ++d)
          o[d] = mfma<ET>(values<ET, DP>(vs, 32 * kt + 16 * c, d), p, o[d]);
      }
  }

  sum += other_half(sum);
  if (t.row0 + 32 * wave + col >= t.rows) return;
  if (t.parts > 1) {
    const int64_t row = (((slots - 1 - slot) * a.kv_heads + head) * a.tile_parts + part) * kRows +
                        32 * wave + col;
    store_part<DP>(o, a.tile_o + row * DP, h);
    if (h == 0) a.tile_stat[row] = {mref, sum};
    return;
  }
  const int64_t orow = (int64_t)(t.start + tok) * a.heads + qh;
  store_row<ET, DP>(o, inverse(sum), (ET*)a.out + orow * a.dim, a.dim, h);
  if (a.lse && h == 0) a.lse[orow] = log_sum(mref, sum);
}

// Joins the splits of a tile, one wave a row.
template <typename ET, int DP, bool PAGED>
__global__ void __launch_bounds__(256) tile_join_kernel(AttnArgs a) {
  constexpr int kRowsGroup = 16;
  uint32_t b = blockIdx.x;
  const int first = (int)(b % (kRows / kRowsGroup)) * kRowsGroup;
  b /= kRows / kRowsGroup;
  const uint32_t head = b % (uint32_t)a.kv_heads;
  const int64_t slots = gridDim.x / ((uint32_t)a.kv_heads * (kRows / kRowsGroup));
  Tile t;
  if (!find_tile<PAGED>(a, slots - 1 - b / (uint32_t)a.kv_heads, &t) || t.parts == 1) return;
  for (int r = first + (threadIdx.x >> 6); r < first + kRowsGroup; r += 4) {
    const int32_t m = t.row0 + r;
    if (m >= t.rows) break;
    const int32_t tok = (int32_t)div_by((uint32_t)m, a.group);
    const int32_t qh = (int32_t)head * (int32_t)a.group.d + m - tok * (int32_t)a.group.d;
    const int64_t orow = (int64_t)(t.start + tok) * a.heads + qh;
    const int64_t row = (int64_t)b * a.tile_parts * kRows + r;
    join_row<ET, DP>(a.tile_stat, a.tile_o, row, row + kRows, kRows, t.parts,
                     (ET*)a.out + orow * a.dim, a.lse ? a.lse + orow : nullptr, a.dim);
  }
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
  hipLaunchKernelGGL(kern, dim3((unsigned)(slots * a.kv_heads * a.tile_parts)), dim3(64 * kWaves),
                     bytes, s, a);
  if (a.tile_parts > 1)
    hipLaunchKernelGGL((tile_join_kernel<ET, DP, PAGED>),
                       dim3((unsigned)(slots * a.kv_heads * (kRows / 16))), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace attn
}  // namespace tod
