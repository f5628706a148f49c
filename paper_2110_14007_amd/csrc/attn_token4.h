// Attention of few new tokens a sequence over a 4-bit cache: bound by the bytes
// of codes and scales, each read once.
//
// The line of stages is that of attn_token.h, its workers three waves on every
// SIMD (two for more than 128 elements, whose registers allow no more) with
// stages of 32 keys (64 for up to 64 elements).  A quarter of the bytes of
// 16-bit rows leaves a wave a quarter of the time for a key, so that its
// arithmetic is laid out for few instructions:
//
// * v_mfma_f32_16x16x32: 16 keys by 16 packed rows, half the columns of the
//   larger product, which few rows leave empty anyway.  In both operands lane l
//   holds row l % 16 and eight elements of the contraction, in any order that is the
//   same on both sides; of the result it holds column l % 16, rows
//   4 (l / 16) + r.
// * Keys go from memory to registers: lane l loads 16 bytes of key l % 16, the
//   block l / 16 of its row, which is one scale and the operand of four products
//   after 16 conversions.  (A row of 64 elements: eight bytes, half a block.)
//   A block's registers take the next stage's as soon as they are converted.
// * Values are loaded the same way, converted with their block's scale, written to
//   the wave's own LDS as 32 rows of 16-bit elements and read by the transposing
//   read as the second product's operand.
// * The scores of two blocks of keys are its other operand right from the
//   accumulators: lane l holds keys 4 (l / 16) + r of each, and the values are read
//   in that order.
//
// Softmax, halves of the weights and values that are not finite: as in attn.h and
// attn_token.h.
//
// Measured, 8 heads of 128, with the join: 162 us for 128 caches of 100 to 12,000
// tokens (840 MB, 5.2 TB/s), 126 us for 5 of 120,000 to 131,071 (685 MB, 5.4 TB/s), 28
// us for one of 60,000.  Two waves a SIMD with stages of 64 keys: 171 and 127 us.
// Pages of 8 rows, whose addresses each lane finds for itself: 97 us for 96 caches
// of 100 to 8,000, pages of 16 or 64 91.  32 packed rows instead of 4 (a group of 8
// and 4 new tokens each) over the same caches: 157, where the bytes alone would take
// 85: two blocks of rows leave two waves a SIMD, and the second product takes both
// halves of the weights for each (16 packed rows: 115).
#pragma once

#include "attn_token.h"

namespace tod {
namespace attn {

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename ET>
__device__ __forceinline__ f32x4 mfma16(typename Frag<ET>::V a, typename Frag<ET>::V b, f32x4 c) {
  if constexpr (std::is_same<ET, _Float16>::value)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
template <typename F>
__device__ __forceinline__ float over_quarters(float v, F&& f) {
  const uint32_t u = __float_as_uint(v);
  const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t w = __float_as_uint(f(__uint_as_float(p[0]), __uint_as_float(p[1])));
  const auto q = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return f(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// The elements of a packed pair in 32 bits.
template <typename ET>
__device__ __forceinline__ float low_half(uint32_t w) {
  if constexpr (std::is_same<ET, _Float16>::value)
    return (float)__builtin_bit_cast(_Float16, (uint16_t)w);
  else
    return __uint_as_float(w << 16);
}
template <typename ET>
__device__ __forceinline__ float high_half(uint32_t w) {
  if constexpr (std::is_same<ET, _Float16>::value)
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16));
  else
    return __uint_as_float(w & 0xffff0000u);
}

template <int DP>
constexpr int token4_tiles() { return DP == 64 ? 4 : 2; }  // blocks of 16 keys of a stage
template <int DP>
constexpr int token4_keys() { return 16 * token4_tiles<DP>(); }

// Stage of 32 rows of values: piece c of row r at c ^ swizzle.  A wave writes 16 rows at one piece and
// reads, with each 16 lanes, two pieces of four rows.
template <int DP>
__device__ __forceinline__ int swizzle4(int row) {
  if constexpr (DP == 64)
    return (row >> 1 & 3) << 1 | (row >> 3 & 1);
  else
    return (row & 3) << 1 | (row >> 2 & 1) | (row & 8);
}

// A lane's codes of a stage's keys or values: words of a row of each block of keys, and a scale for
// four of them.
template <int DP>
struct Lane4 {
  static constexpr int kWords = DP / 32, kScales = DP == 256 ? 2 : 1, kTiles = token4_tiles<DP>();
  uint32_t w[kTiles][kWords];
  uint32_t scale[kTiles][kScales];
};

// First element of word i of lane group g's codes of a row.
template <int DP>
__device__ __forceinline__ int element4(int i, int g) {
  if constexpr (DP == 64)
    return 16 * g + 8 * i;
  else
    return 32 * (g + 4 * (i / 4)) + 8 * (i % 4);
}

// A worker: a wave, with LDS for 32 rows of values.  NB: blocks of 16 packed rows that it keeps.
// EVEN: pages hold whole blocks of 16 keys, so that the wave finds a block by one address.
template <typename ET, int DP, int NB, bool EVEN>
__device__ __forceinline__ void token4_work(const AttnArgs& a, const uint32_t worker,
                                            const uint32_t grid, uint16_t* const lds,
                                            const int lane = threadIdx.x & 63) {
  constexpr int KT = token4_tiles<DP>(), KEYS = token4_keys<DP>(), C = DP / 32, DB = DP / 16;
  using V8 = typename Frag<ET>::V;
  using L4 = Lane4<DP>;
  const int n = lane & 15, g = lane >> 4;

  const Share mine = deal<KEYS>(a, worker, grid);
  int64_t at = mine.at, off = mine.off;
  const int64_t end = mine.end;
  int32_t s = mine.s;

  for (bool opening = true; at < end; opening = false) {
    Seq sq = dealt(a, mine, s);
    sq = {uniform(sq.start), uniform(sq.n), uniform(sq.keys), uniform(sq.shift)};
    const int32_t stages = token_stages<KEYS>(a, sq);
    if (stages == 0) {  // another kernel's, or idle
      ++s;
      off = 0;
      continue;
    }
    const uint32_t head = (uint32_t)uniform((int32_t)quotient(off, stages));
    const int32_t jb = uniform((int32_t)(off - (int64_t)head * stages));
    const int32_t je = uniform((int32_t)min((int64_t)stages, jb + (end - at)));

    const int32_t rows = sq.n * (int32_t)a.group.d;
    int32_t tok[NB], qh[NB], limit[NB];
    V8 q[NB][C];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int32_t m = min(16 * b + n, rows - 1);
      tok[b] = (int32_t)div_by((uint32_t)m, a.group);
      qh[b] = (int32_t)head * (int32_t)a.group.d + m - tok[b] * (int32_t)a.group.d;
      limit[b] = min(sq.shift + tok[b], sq.keys - 1);
      const ET* const p =
          (const ET*)a.q + (int64_t)(sq.start + tok[b]) * a.q_row + (int64_t)qh[b] * a.q_head;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int e = element4<DP>(c, g);
        u32x4 w = *(const u32x4*)(p + (e < a.dim ? e : 0));
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = e < a.dim ? w[i] : 0u;
        q[b][c] = __builtin_bit_cast(V8, w);
      }
    }
    const int32_t wlo = uniform(limit[0]);

    Stager<ET, DP, true> st(a, head, lane);
    st.seq = s;
    st.start = sq.start;
    st.seen = sq.keys;
    // Rows of the cache of a stage's keys: of each block's first key (EVEN), or of key `lane`.  gone:
    // blocks without a page.
    uint32_t block[KT], each = 0, gone = 0;
    auto find = [&](int32_t j) __attribute__((always_inline)) {
      if constexpr (EVEN) {
        gone = 0;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          const uint32_t row = (uint32_t)uniform((int32_t)st.row_of(j * KEYS + 16 * t));
          gone |= row == ~0u ? 1u << t : 0u;
          block[t] = row == ~0u ? 0u : row;
        }
      } else {
        each = st.place(j * KEYS, KEYS);
      }
    };
    // Loads of block t.  There is no branch around them: they are waited for by their number.  What is
    // loaded for a block without a page (the cache's first rows) is cleared in its turn.
    const uint32_t row_bytes = (uint32_t)a.dim / 2, row_scales = (uint32_t)a.dim / 32;
    auto load = [&](const void* codes, const uint8_t* scales, L4& to, int t)
        __attribute__((always_inline)) {
      constexpr int kBytes = DP == 64 ? 8 : 16;
      typedef uint32_t words __attribute__((ext_vector_type(kBytes / 4)));
      const uint32_t row = EVEN ? 0u : (uint32_t)__shfl((int)each, 16 * t + n, 64);
#pragma unroll
      for (int i = 0; i < L4::kScales; ++i) {
        const int e = element4<DP>(4 * i, g);
        const uint8_t *c, *b;
        if constexpr (EVEN) {
          const uint32_t in = e < a.dim ? (uint32_t)e : 0u;
          c = (const uint8_t*)codes + (uint64_t)block[t] * row_bytes + (n * row_bytes + in / 2);
          b = scales + (uint64_t)block[t] * row_scales + ((n * row_scales + in / 32) & ~3u);
        } else {
          const bool ok = row != ~0u && e < a.dim;
          const uint8_t* const zeros = (const uint8_t*)&kZeros;
          c = ok ? (const uint8_t*)codes + (uint64_t)row * row_bytes + (uint32_t)e / 2 : zeros;
          b = ok ? scales + (uint64_t)row * row_scales + (uint32_t)e / 32 : zeros;
        }
        const words w = load_once<words>(c);
#pragma unroll
        for (int x = 0; x < kBytes / 4; ++x) to.w[t][4 * i + x] = w[x];
        to.scale[t][i] = EVEN ? load_global<uint32_t>(b) : load_global<uint8_t>(b);
      }
    };
    // The scales of a block's 16 rows come as whole words: a byte loaded for the next turn would be
    // extended, and so waited for, at the end of this one.
    auto scale_in = [&](const L4& x, int t, int i) __attribute__((always_inline)) {
      const int e = element4<DP>(4 * i, g);
      const uint32_t in = e < a.dim ? (uint32_t)e : 0u;
      return scale_of(EVEN ? x.scale[t][i] >> (8 * ((n * row_scales + in / 32) & 3)) & 0xff
                           : x.scale[t][i]);
    };
    // Clears what is no code: of a key that is out, or of a lane past a row's last element.
    auto clear = [&](L4& x, int t, bool out) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < L4::kWords; ++i)
        x.w[t][i] = out || element4<DP>(i, g) >= a.dim ? 0u : x.w[t][i];
#pragma unroll
      for (int i = 0; i < L4::kScales; ++i)
        x.scale[t][i] = out || element4<DP>(4 * i, g) >= a.dim ? 0u : x.scale[t][i];
    };

    f32x4 o[DB][NB];
    float mref[NB], limit_raw[NB];  // a score above limit_raw makes mref follow
    Sum acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d][b] = f32x4{0, 0, 0, 0};
      mref[b] = kNoMax;
      limit_raw[b] = -INFINITY;
    }
    bool cleared = false;  // values that are not finite were taken for 0

    L4 k, v;
    auto turn = [&](int32_t j, auto MORE) __attribute__((always_inline)) {
      constexpr bool more = decltype(MORE)::value;  // a stage follows: its loads are issued
      const int32_t j0 = j * KEYS;
      const uint32_t none = gone;  // of this stage
      f32x4 x[KT][NB];
      const bool narrow = a.dim < DP;  // some lanes have no element
      if (none || narrow) {
#pragma unroll
        for (int t = 0; t < KT; ++t) clear(k, t, none >> t & 1);
      }
      float scale[KT][L4::kScales];
#pragma unroll
      for (int t = 0; t < KT; ++t) {
#pragma unroll
        for (int i = 0; i < L4::kScales; ++i) scale[t][i] = scale_in(k, t, i);
#pragma unroll
        for (int b = 0; b < NB; ++b) x[t][b] = f32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          const V8 f = __builtin_bit_cast(V8, eight_values<ET>(k.w[t][c], scale[t][c / 4]));
#pragma unroll
          for (int b = 0; b < NB; ++b) x[t][b] = mfma16<ET>(f, q[b][c], x[t][b]);
        }
      if constexpr (more) {
        find(j + 1);
        __builtin_amdgcn_sched_barrier(0);  // into the registers that the conversions left
#pragma unroll
        for (int t = 0; t < KT; ++t) load(a.k, a.k_scales, k, t);
        __builtin_amdgcn_sched_barrier(0);
      }
      const bool edge = j0 + KEYS - 1 > wlo;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if (edge) {
          const int32_t left = limit[b] - j0 - 4 * g;
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (16 * t + r > left) x[t][b][r] = -INFINITY;
        }
        float top = x[0][b][0];
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) top = fmaxf(top, x[t][b][r]);
        if (__ballot(top > limit_raw[b])) {
          // m follows the maximum only when that has grown by more than kSlack.
          constexpr float kRoom = kSlack<ET> + kBias<ET>;
          const float raw = over_quarters(top, [](float p, float r) { return fmaxf(p, r); });
          const float t2 = raw * a.scale;
          const bool far = fabsf(fmaxf(t2, mref[b])) > kFar;  // m follows every growth
          const float next =
              t2 > mref[b] + (far ? 0.0f : kRoom) ? t2 - (far ? 0.0f : kBias<ET>) : mref[b];
          const float f = __builtin_amdgcn_exp2f(mref[b] - next);
          mref[b] = next;
          limit_raw[b] = far ? fmaxf(raw, limit_raw[b]) : (next + kRoom) * a.unscale;
          acc[b].scale(f);
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[d][b][r] *= f;
        }
        float part = 0.0f;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            x[t][b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][b][r], a.scale, -mref[b]));
            part += x[t][b][r];
          }
        acc[b].add(part);
      }
      if (edge || none || narrow) {
        // No value that does not exist may meet a weight, not even one of 0.
#pragma unroll
        for (int t = 0; t < KT; ++t) clear(v, t, (none >> t & 1) || j0 + 16 * t + n >= sq.keys);
      }
#pragma unroll
      for (int u = 0; u < KT / 2; ++u) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int row = 16 * t + n;
          float scale[L4::kScales];
#pragma unroll
          for (int i = 0; i < L4::kScales; ++i) scale[i] = scale_in(v, 2 * u + t, i);
#pragma unroll
          for (int i = 0; i < L4::kWords; ++i)
            *(u32x4*)(lds + row * DP + 8 * ((element4<DP>(i, g) / 8) ^ swizzle4<DP>(row))) =
                eight_values<ET>(v.w[2 * u + t][i], scale[i / 4]);
        }
        if constexpr (more) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int t = 0; t < 2; ++t) load(a.v, a.v_scales, v, 2 * u + t);
          __builtin_amdgcn_sched_barrier(0);
        }
        // (One wave's LDS accesses are done in order.)
        asm volatile("" ::: "memory");
        // A value that is not finite must not meet the zero weight of a row that does not see it.
        if (edge && rows > (int32_t)a.group.d) {
          asm volatile("" ::: "memory");  // (the stage is not read where it need not be)
          if (holds_nonfinite<ET, DP>(lds, lane)) {
#pragma unroll 1
            for (int i = 0; i < 32 * DP; i += 512) clear_nonfinite<ET, 16>(lds + i, 0, 64, lane);
            cleared = true;
          }
        }
        u32x4 hi[NB], lo[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p0 = x[2 * u + e / 2][b][e % 2 * 2], p1 = x[2 * u + e / 2][b][e % 2 * 2 + 1];
            hi[b][e] = pack2<ET>(p0, p1);
            lo[b][e] = pack2<ET>(p0 - low_half<ET>(hi[b][e]), p1 - high_half<ET>(hi[b][e]));
          }
        // Reads of four blocks of columns, then their products: each half of the weights in turn, so
        // that no product waits for the one before.
        constexpr int kColumns = 4;
#pragma unroll
        for (int d0 = 0; d0 < DB; d0 += kColumns) {
          V8 f[kColumns];
#pragma unroll
          for (int d = 0; d < kColumns; ++d) {
            const int row = 4 * g + n / 4;
            const int piece = 2 * (d0 + d) + ((n & 3) >> 1), within = 4 * (n & 1);
            typedef __attribute__((address_space(3))) s16x4* lds4;
            const s16x4 first = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds4)(lds + row * DP + 8 * (piece ^ swizzle4<DP>(row)) + within));
            const s16x4 second = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds4)(lds + (row + 16) * DP + 8 * (piece ^ swizzle4<DP>(row + 16)) + within));
            f[d] = __builtin_bit_cast(
                V8, __builtin_shufflevector(first, second, 0, 1, 2, 3, 4, 5, 6, 7));
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int d = 0; d < kColumns; ++d)
              o[d0 + d][b] = mfma16<ET>(f[d], __builtin_bit_cast(V8, hi[b]), o[d0 + d][b]);
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int d = 0; d < kColumns; ++d)
              o[d0 + d][b] = mfma16<ET>(f[d], __builtin_bit_cast(V8, lo[b]), o[d0 + d][b]);
        }
        asm volatile("" ::: "memory");
      }
    };

    // Each block's registers take the next stage's codes as soon as they are converted.
    find(jb);
#pragma unroll
    for (int t = 0; t < KT; ++t) load(a.k, a.k_scales, k, t);
#pragma unroll
    for (int t = 0; t < KT; ++t) load(a.v, a.v_scales, v, t);
    for (int32_t j = jb; j < je - 1; ++j) turn(j, std::true_type{});
    turn(je - 1, std::false_type{});

    float sum[NB];
    bool restore = cleared;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      sum[b] = over_quarters(acc[b].v, [](float p, float r) { return p + r; });
      float all = 0.0f;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) all += fabsf(o[d][b][r]);
      restore |= __ballot(!finite(all) && finite(sum[b])) != 0;
    }
    const float own_sum = NB == 2 && (lane & 16) ? sum[NB - 1] : sum[0];  // of row lane % 32

    const bool whole = jb == 0 && je == stages;
    // At most two of a worker's pieces are not whole: its first and its last.
    const int64_t row0 = (2 * (int64_t)worker + !opening) * a.skip_rows;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int32_t m = 16 * b + n;
      if (m >= rows) continue;
      const int64_t orow = (int64_t)(sq.start + tok[b]) * a.heads + qh[b];
      if (whole) {
        if (a.lse && g == 0) a.lse[orow] = log_sum(mref[b], sum[b]);
        const float f = inverse(sum[b]);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const int e = 16 * d + 4 * g;
          if (e >= a.dim) break;
          uint2 w;
          w.x = pack2<ET>(o[d][b][0] * f, o[d][b][1] * f);
          w.y = pack2<ET>(o[d][b][2] * f, o[d][b][3] * f);
          *(uint2*)((ET*)a.out + orow * a.dim + e) = w;
        }
      } else {
        if (g == 0) a.token_stat[row0 + m] = {mref[b], sum[b]};
#pragma unroll
        for (int d = 0; d < DB; ++d)
          *(f32x4*)(a.token_o + (row0 + m) * DP + 16 * d + 4 * g) = o[d][b];
      }
    }
    if (restore) {
      if (whole)
        restore_nonfinite<ET, DP, true, true>(st, (ET*)a.out, 0, sq, 0, 0, sq.keys, own_sum);
      else
        restore_nonfinite<ET, DP, true, true>(st, a.token_o + row0 * DP, DP, sq, 0, jb * KEYS,
                                              je * KEYS, own_sum);
    }
    at += je - jb;
    off += je - jb;
    if (off == (int64_t)stages * a.kv_heads) {
      ++s;
      off = 0;
    }
  }
  clear_tail(a, worker, grid);
}

// Waves on a SIMD, by the registers that they need.
template <int DP, int NB>
constexpr int token4_waves() { return DP == 256 ? NB == 1 ? 2 : 1 : NB == 1 ? 3 : 2; }

template <typename ET, int DP, int NB, bool EVEN>
__global__ void __launch_bounds__(64, (token4_waves<DP, NB>())) token4_kernel(AttnArgs a) {
  __shared__ __align__(16) uint16_t lds[32 * DP];
  token4_work<ET, DP, NB, EVEN>(a, blockIdx.x, (uint32_t)token4_workers(DP), lds);
}

template <typename ET, int DP>
hipError_t launch_token4(const AttnArgs& a, hipStream_t s) {
  const bool even = a.page.d % 16 == 0;
  const auto kern = a.skip_rows <= 16
                        ? even ? token4_kernel<ET, DP, 1, true> : token4_kernel<ET, DP, 1, false>
                        : even ? token4_kernel<ET, DP, 2, true> : token4_kernel<ET, DP, 2, false>;
  hipLaunchKernelGGL(kern, dim3((unsigned)token4_workers(DP)), dim3(64), 0, s, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_token_join<ET, DP, (uint32_t)token4_workers(DP)>(a, s);
}

template <typename ET>
hipError_t launch_token4(const AttnArgs& a, hipStream_t s) {
  if (a.dim <= 64) return launch_token4<ET, 64>(a, s);
  if (a.dim <= 128) return launch_token4<ET, 128>(a, s);
  return launch_token4<ET, 256>(a, s);
}

}  // namespace attn
}  // namespace tod
