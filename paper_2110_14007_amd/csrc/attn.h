// Common parts of the attention kernels: attn_tile.h (whole prompts and
// chunks, 128 rows a workgroup) and attn_token.h (few new tokens over a long
// cache, one wave a share of the keys).
//
// Attention of packed sequences: softmax(scale q k^T) v, one pass over the
// keys with the running maximum and sum of the softmax.
//
// Rows.  The G query heads that share one key / value head are packed into
// the rows of one product: row m of a sequence is token m / G, head m % G of
// the group, so that a sequence of n new tokens has n G rows per key / value
// head and each staged key serves all of them.
//
// Products.  v_mfma_f32_32x32x16 takes 32 keys as A and 32 rows of queries as
// B, so that lane l holds, for query l % 32, the scores of keys
// 8 (r / 4) + 4 (l / 32) + r % 4 in accumulators r = 0..15: the maximum and
// the sum over the keys are then in-lane but for one exchange between lanes l
// and l + 32.  The second product, O^T = V^T P^T, takes P as its B operand
// right from those registers: the contraction runs over the keys in any
// order, and the one that the accumulators hold is used, 16 of them a product
// (elements 0..3 of lane half h are keys 4h.., elements 4..7 keys 8 + 4h..).
// V^T is read from the row-major stage by the LDS's transposing read (16
// lanes read four rows of 16 columns, and lane i of them gets column i).
//
// Softmax.  In base 2: t = s scale log2(e), p = 2^(t - m) with m the running
// maximum.  m, the sum and O are fp32, and the sum takes the unrounded p, those of
// a stage or of a few together.
// The second product takes p in the input type.  fp16 ends at 2^-24, where a long cache may have
// most of its weight (100,000 keys of p = 2^-24 beside one of 1 are 0.6% of the output), so that
// for fp16 m is the running maximum less kBias: weights reach 2^kBias, and what is rounded away
// of each is 2^-35 of the largest at most.
// Splits of the keys leave (m, sum, O) in the workspace, joined by 2^(m - max).
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
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Before the first visible key: every finite score replaces it.
constexpr float kNoMax = -3.0e38f;
constexpr float kLn2 = 0.69314718055994531f;
// How far below the running maximum m is taken (log2).  For bf16, whose values reach fp32's largest,
// it lies above by what m may lag behind in the tiles: weights are 1 at most, and O overflows no
// sooner than the formula's sum does.
template <typename ET>
constexpr float kBias = std::is_same<ET, _Float16>::value ? 10.0f : -8.0f;
// Where |t| is larger, the rounding of t itself takes up the room that is left to fp16's 2^16: there
// m is the maximum as it is.
constexpr float kFar = 1048576.0f;

// A sequence of the call.  After the last one comes one without keys that
// holds the rows past row_start[n_seq].
struct Seq {
  int32_t start, n;  // its first token and its number of tokens
  int32_t keys;      // keys that exist
  int32_t shift;     // token i of it stands at position shift + i
};

__device__ __forceinline__ int32_t start_of(const AttnArgs& a, int32_t s) {
  return s <= 0 ? 0 : min(max(a.row_start[s], 0), a.tokens);
}

// From the sequence's row_start, the next one's and its cached tokens.
template <bool PAGED>
__device__ __forceinline__ Seq make_seq(const AttnArgs& a, int32_t s, int32_t start, int32_t next,
                                        int32_t cached) {
  Seq q;
  q.start = start;
  q.n = (s < a.n_seq ? max(next, start) : a.tokens) - start;
  q.shift = 0;
  q.keys = 0;
  if (s < a.n_seq) {
    if constexpr (PAGED) {
      const int32_t room = (int32_t)a.cols * (int32_t)a.page.d;
      q.shift = min(max(cached, 0), room);
      q.keys = min(q.shift + q.n, room);
    } else {
      q.keys = q.n;
    }
  }
  return q;
}

template <bool PAGED>
__device__ __forceinline__ Seq seq_of(const AttnArgs& a, int32_t s) {
  const bool real = s < a.n_seq;
  return make_seq<PAGED>(a, s, start_of(a, s), real ? start_of(a, s + 1) : 0,
                         PAGED && real ? a.cached[s] : 0);
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
// transposing read, four rows of 32 bytes at a time.  (Reads measured at 343
// bytes / ns a compute unit for K and 244 for V, whose reads reach 248 at best;
// with no swizzle 38 and 151.)
template <int DP>
__device__ __forceinline__ int swizzle_k(int row) {
  return DP == 64 ? (row >> 1) & 7 : row & 15;
}
template <int DP>
__device__ __forceinline__ int swizzle_v(int row) {
  return DP == 64 ? 0 : (row & 3) << 1;
}

// mt::dma16 for data that no other wave reads: marked as streaming, so that it does not push
// others' data out of the caches.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16_once(const void* g, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(g),
               "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory", "m0");
}
#pragma clang diagnostic pop

// Staging of keys and values for one wave, straight from global memory to LDS.
// Over pages, lane l holds entry `first` + l of the sequence's table, so that
// a stage (64 keys at most) finds its rows without a load from memory unless
// it leaves those 64 pages.
template <typename ET, int DP, bool PAGED>
struct Stager {
  static constexpr int kPieces = DP / 8;       // 16-byte pieces of a row
  static constexpr int kRowsLoad = 64 / kPieces;  // rows that one load of the wave moves
  const AttnArgs& a;
  uint32_t head;
  int32_t seq, start, seen;  // keys from `seen` on are not loaded
  int32_t first = INT32_MIN / 2, entry = 0;

  __device__ Stager(const AttnArgs& args, uint32_t hd) : a(args), head(hd) {}

  // Row of the cache (or of k) of key j0 + lane; ~0: none.
  __device__ __forceinline__ uint32_t place(int32_t j0, int32_t keys) {
    const int lane = threadIdx.x & 63;
    const int32_t j = j0 + lane;
    if constexpr (PAGED) {
      const int32_t lo = (int32_t)div_by((uint32_t)j0, a.page);
      const int32_t hi = (int32_t)div_by((uint32_t)(j0 + keys - 1), a.page);
      if (lo < first || hi - first >= 64) {
        first = lo;
        entry = lo + lane < a.cols ? a.table[(int64_t)seq * a.cols + lo + lane] : -1;
        asm volatile("" : "+v"(entry));  // waited for here, not by every stage's first use
      }
      const uint32_t pg = div_by((uint32_t)j, a.page);
      const int32_t id = __shfl(entry, (int)(pg - (uint32_t)first) & 63, 64);
      if (j >= seen || id < 0 || id >= a.n_pages) return ~0u;
      return ((uint32_t)id * (uint32_t)a.kv_heads + head) * a.page.d +
             ((uint32_t)j - pg * a.page.d);
    } else {
      return j < seen ? (uint32_t)(start + j) : ~0u;
    }
  }

  // Row of the cache of key j, the same for the whole wave; ~0: none.  The window of entries
  // begins a little before it, for the values that are staged after their keys.
  __device__ __forceinline__ uint32_t row_of(int32_t j) {
    const int32_t pg = (int32_t)div_by((uint32_t)j, a.page);
    if (pg < first || pg - first >= 64) {
      first = max(pg - 16, 0);
      const int32_t e = first + (int32_t)(threadIdx.x & 63);
      entry = e < a.cols ? a.table[(int64_t)seq * a.cols + e] : -1;
      asm volatile("" : "+v"(entry));  // waited for here, not by every stage's first use
    }
    const int32_t id = __builtin_amdgcn_readlane(entry, pg - first);
    if (id < 0 || id >= a.n_pages) return ~0u;
    return ((uint32_t)id * (uint32_t)a.kv_heads + head) * a.page.d +
           ((uint32_t)j - (uint32_t)pg * a.page.d);
  }

  // Rows r0 .. r0 + kRowsLoad - 1 of a K (or V) stage that begins at LDS address `to`.
  __device__ __forceinline__ void load_one(bool isk, uint32_t at, int r0, uint32_t to) const {
    const int lane = threadIdx.x & 63;
    const int r = r0 + lane / kPieces, pc = lane % kPieces;
    const uint32_t row = (uint32_t)__shfl((int)at, r, 64);
    const int c = 8 * (pc ^ (isk ? swizzle_k<DP>(r) : swizzle_v<DP>(r)));
    const ET* p = (const ET*)(isk ? a.k : a.v);
    if constexpr (PAGED)
      p += (int64_t)row * a.dim;
    else
      p += (int64_t)row * (isk ? a.k_row : a.v_row) + (int64_t)head * (isk ? a.k_head : a.v_head);
    const void* const src = row != ~0u && c < a.dim ? (const void*)(p + c) : &kZeros;
    mt::dma16(src, to + 2u * (uint32_t)(r0 * DP));
  }

  // Rows r0 .. r0 + kRowsLoad - 1 of a stage over pages whose K begins at LDS address k and V at v,
  // read by no other wave; at: place().
  __device__ __forceinline__ void load(uint32_t at, int r0, uint32_t k, uint32_t v) const {
    const int lane = threadIdx.x & 63;
    const int r = r0 + lane / kPieces, pc = lane % kPieces;
    const uint32_t row = (uint32_t)__shfl((int)at, r, 64);
    const int ck = 8 * (pc ^ swizzle_k<DP>(r)), cv = 8 * (pc ^ swizzle_v<DP>(r));
    static_assert(PAGED, "rows of a cache");
    const ET* const kp = (const ET*)a.k + (int64_t)row * a.dim;
    const ET* const vp = (const ET*)a.v + (int64_t)row * a.dim;
    const bool ok = row != ~0u;
    const void* const ks = ok && ck < a.dim ? (const void*)(kp + ck) : &kZeros;
    const void* const vs = ok && cv < a.dim ? (const void*)(vp + cv) : &kZeros;
    dma16_once(ks, k + 2u * (uint32_t)(r0 * DP));
    dma16_once(vs, v + 2u * (uint32_t)(r0 * DP));
  }
};

// Query operand: elements 16 c + 8 h .. + 7 of row p, zero from dim on.  Every lane loads (from the
// row's start where there is nothing): with a branch around each, the loads would run one by one.
template <typename ET, int W>
__device__ __forceinline__ void load_query(typename Frag<ET>::V (&q)[W / 16], const ET* p,
                                           int32_t dim, int h) {
  u32x4 w[W / 16];
#pragma unroll
  for (int c = 0; c < W / 16; ++c) {
    const int e = 16 * c + 8 * h;
    w[c] = *(const u32x4*)(p + (e < dim ? e : 0));
  }
#pragma unroll
  for (int c = 0; c < W / 16; ++c) {
    const bool in = 16 * c + 8 * h < dim;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[c][i] = in ? w[c][i] : 0u;
    q[c] = __builtin_bit_cast(typename Frag<ET>::V, w[c]);
  }
}

// Scores of the 32 keys at rows `row0`.. of the K stage ks.
template <typename ET, int DP>
__device__ __forceinline__ f32x16 scores(const uint16_t* ks, int row0,
                                         const typename Frag<ET>::V (&q)[DP / 16]) {
  const int col = threadIdx.x & 31, h = (threadIdx.x >> 5) & 1;
  f32x16 s;
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 0.0f;
  const int row = row0 + col;
#pragma unroll
  for (int c = 0; c < DP / 16; ++c)
    s = mfma<ET>(*(const typename Frag<ET>::V*)(ks + row * DP + 8 * ((2 * c + h) ^ swizzle_k<DP>(row))),
                 q[c], s);
  return s;
}

// A operand of the second product: columns 32 d .. + 31 of the 16 keys at rows row0.. of the
// V stage vs.  Lane i of 16 reads row i / 4, columns 4 (i % 4).. of its four rows.
template <typename ET, int DP>
__device__ __forceinline__ typename Frag<ET>::V values(const uint16_t* vs, int row0, int d) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int row = row0 + 4 * h + (lane & 15) / 4;
  const int piece = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const int within = 4 * (lane & 1);
  typedef __attribute__((address_space(3))) s16x4* lds4;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds4)(vs + row * DP + 8 * (piece ^ swizzle_v<DP>(row)) + within));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds4)(vs + (row + 8) * DP + 8 * (piece ^ swizzle_v<DP>(row + 8)) + within));
  return __builtin_bit_cast(typename Frag<ET>::V,
                            __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Whether a V stage of 32 keys holds an infinity or a NaN, the same for the whole wave.
template <typename ET, int DP>
__device__ __forceinline__ bool holds_nonfinite(const uint16_t* vs) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  constexpr uint16_t kInf = std::is_same<ET, _Float16>::value ? 0x7c00 : 0x7f80;
  u16x2 top = {0, 0};
#pragma unroll
  for (int i = 0; i < 32 * DP / 512; ++i) {
    const u32x4 v = *(const u32x4*)(vs + 8 * (64 * i + (threadIdx.x & 63)));
#pragma unroll
    for (int e = 0; e < 4; ++e)
      top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, v[e] & 0x7fff7fffu));
  }
  return __ballot(top[0] >= kInf || top[1] >= kInf) != 0;
}

// Clears those of the stage's values, the thread's share of it (from first, every step threads).
template <typename ET, int DP>
__device__ __forceinline__ void clear_nonfinite(uint16_t* vs, int first, int step) {
  constexpr uint16_t kInf = std::is_same<ET, _Float16>::value ? 0x7c00 : 0x7f80;
  for (int i = first + (threadIdx.x & 63); i < 32 * DP; i += step)
    if ((vs[i] & 0x7fff) >= kInf) vs[i] = 0;
}

// Adds the weights of a stage or of a few to a running sum, with what the additions before lost: a
// long tail of keys whose weights are near 2^-24 of the sum would not move it otherwise.
struct Sum {
  float v = 0.0f, lost = 0.0f;
  __device__ __forceinline__ void add(float part) {
    const float x = part - lost, next = v + x;
    lost = (next - v) - x;
    v = next;
  }
  __device__ __forceinline__ void scale(float f) {
    v *= f;
    lost *= f;
  }
};

// Whether v is neither an infinity nor a NaN.  (These files are compiled as if none met a NaN: the
// compiler must not know that the bits are a float's, or it leaves the NaN out of the test.)
__device__ __forceinline__ bool finite(float v) {
  uint32_t u = __float_as_uint(v);
  asm("" : "+v"(u));
  return (u & 0x7f800000u) != 0x7f800000u;
}

// Whether O of some of the wave's 32 rows, whose sums of weights are `sum`, met values that are not
// finite: the sum of magnitudes shows one, at an addition an element.
template <int N>
__device__ __forceinline__ bool met_nonfinite(const f32x16 (&o)[N], float sum) {
  float all = 0.0f;
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) all += fabsf(o[d][r]);
  return __ballot(!finite(all) && finite(sum)) != 0;
}

// After the stores of a wave's 32 packed rows from m0 on: where a row sees values that are not
// finite among the keys j0 .. j1 - 1, its output is their sum, since all weights are positive.
// (The products do not say so: a value may have been cleared, or met a weight or a half of one that
// was rounded to 0.)  Rows whose weights are NaN, so that `sum` is, stay NaN.  step 0: rows of the
// output; else partial results of the rows one after the other, step elements each.
template <typename ET, int DP, bool PAGED, typename OT, typename ST>
__device__ __forceinline__ void restore_nonfinite(ST& st, OT* out, int32_t step, const Seq& s,
                                                  int32_t m0, int32_t j0, int32_t j1, float sum) {
  const AttnArgs& a = st.a;
  const int lane = threadIdx.x & 63;
  constexpr uint16_t kInf = std::is_same<ET, _Float16>::value ? 0x7c00 : 0x7f80;
  const uint64_t sound = __ballot(finite(sum));
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the stores that this one follows
#pragma unroll 1
  for (int32_t e = lane; e < a.dim; e += 64) {
    float total = 0.0f;
    bool any = false;
    int32_t j = j0;  // (each row sees at least the keys of the one before)
#pragma unroll 1
    for (int32_t r = 0; r < 32; ++r) {
      const int32_t m = m0 + r;
      if (m >= s.n * (int32_t)a.group.d) break;
      const int32_t tok = (int32_t)div_by((uint32_t)m, a.group);
      const int32_t end = min(PAGED || a.causal ? min(s.shift + tok + 1, s.keys) : s.keys, j1);
      constexpr int kAhead = 8;  // values in flight; the last again where there are fewer
#pragma unroll 1
      for (; j < end; j += min(end - j, kAhead)) {
        uint16_t u[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int32_t key = min(j + k, end - 1);
          const ET* p = (const ET*)a.v;
          if constexpr (PAGED) {
            const uint32_t pg = div_by((uint32_t)key, a.page);
            const int32_t id = a.table[(int64_t)st.seq * a.cols + pg];
            const bool none = id < 0 || id >= a.n_pages;  // zeros
            p += (((int64_t)id * a.kv_heads + st.head) * a.page.d +
                  (key - (int32_t)(pg * a.page.d))) * a.dim;
            const uint16_t* const from = (const uint16_t*)p + e;
            u[k] = *(none ? (const uint16_t*)&kZeros : from);
          } else {
            p += (int64_t)(s.start + key) * a.v_row + (int64_t)st.head * a.v_head;
            u[k] = ((const uint16_t*)p)[e];
          }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          if ((u[k] & 0x7fff) >= kInf) {
            any = true;
            total += (float)__builtin_bit_cast(ET, u[k]);
          }
        }
      }
      if (any && (sound >> r & 1)) {
        const int64_t row = (int64_t)(s.start + tok) * a.heads +
                            (int64_t)st.head * (int32_t)a.group.d + m - tok * (int32_t)a.group.d;
        (step ? out + (int64_t)r * step : out + row * a.dim)[e] = (OT)total;
      }
    }
  }
}

// What a row's O is multiplied by, and its log sum.  A row without keys has the sum 0 and O = 0:
// its output is 0 and its log sum -inf without a test for it (a comparison would not do: these
// files are compiled as if none met a NaN, and where a score is NaN the sum and O are).
__device__ __forceinline__ float inverse(float sum) { return 1.0f / fmaxf(sum, 1.17549435e-38f); }

__device__ __forceinline__ float log_sum(float m, float sum) {
  return (m + __builtin_amdgcn_logf(sum)) * kLn2;
}

// O^T accumulators of a wave's 32 rows, row l % 32 times f, as the output type into the rows at
// out: rows that lie at the lanes' element offsets `at` (below 0: no such row).  They pass through
// the wave's own 32 x DP elements of LDS at `lds`, so that each store writes whole rows: from
// the accumulators a lane could write 8 bytes at a time only.
template <typename ET, int DP, int W>
__device__ __forceinline__ void store_rows(const f32x16 (&o)[W / 32], float f, ET* out, int64_t at,
                                           int32_t dim, uint16_t* lds) {
  constexpr int kPieces = DP / 8, kRowsStore = 64 / kPieces;  // 16-byte pieces; rows of a store
  const int lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5;
#pragma unroll
  for (int d = 0; d < W / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      uint2 w;
      w.x = pack2<ET>(o[d][4 * g] * f, o[d][4 * g + 1] * f);
      w.y = pack2<ET>(o[d][4 * g + 2] * f, o[d][4 * g + 3] * f);
      const int piece = (4 * d + g) ^ swizzle_k<DP>(col);
      *(uint2*)(lds + col * DP + 8 * piece + 4 * h) = w;
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32 / kRowsStore; ++i) {
    const int row = i * kRowsStore + lane / kPieces, piece = lane % kPieces;
    const u32x4 w = *(const u32x4*)(lds + row * DP + 8 * (piece ^ swizzle_k<DP>(row)));
    const int64_t to = __shfl(at, row, 64);
    if (to >= 0 && 8 * piece < dim) *(u32x4*)(out + to + 8 * piece) = w;
  }
}

// The same, unscaled fp32, into a row of a split's partial result.
template <int W>
__device__ __forceinline__ void store_part(const f32x16 (&o)[W / 32], float* p, int h) {
#pragma unroll
  for (int d = 0; d < W / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 w = {o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
      *(float4*)(p + 32 * d + 8 * g + 4 * h) = w;
    }
}

// A part of O by its weight.  An infinity stays one, also where the weight is 0.
__device__ __forceinline__ float weighted(float v, float w) {
  return fabsf(v) == INFINITY ? v : v * w;
}

// A row's running maximum, sum and O: lane l holds columns DP / 64 l on.
template <int DP>
struct Joined {
  float m, sum, acc[DP / 64];
};

// One wave joins the partial results i .. end - 1 of a row: (m, sum) at stat[row], the DP columns
// of O at o[row * DP], where row is row0 for the first, then row1, row1 + step, ...
template <int DP>
__device__ __forceinline__ Joined<DP> join_parts(const float2* stat, const float* o, int64_t row0,
                                                 int64_t row1, int64_t step, int32_t i,
                                                 int32_t end) {
  constexpr int C = DP / 64;
  const int lane = threadIdx.x & 63;
  auto row_of = [&](int32_t k) { return k == 0 ? row0 : row1 + (k - 1) * step; };
  Joined<DP> j = {kNoMax, 0.0f, {}};
  auto& [m, sum, acc] = j;
  for (int32_t i0 = i; i0 < end; i0 += 64) {  // 64 parts a turn, the statistics one a lane
    const int32_t n = min(end - i0, 64);
    const float2 st = lane < n ? stat[row_of(i0 + lane)] : float2{kNoMax, 0.0f};
    float top = fmaxf(m, st.x);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float keep = __builtin_amdgcn_exp2f(m - top), f = __builtin_amdgcn_exp2f(st.x - top);
    m = top;
    float part = st.y * f;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) part += __shfl_xor(part, d, 64);
    sum = sum * keep + part;
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = weighted(acc[c], keep);
    constexpr int kAhead = 8;  // parts in flight
    for (int32_t i = 0; i < n; i += kAhead) {
      float v[kAhead][C];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float* const p = o + row_of(i0 + min(i + k, n - 1)) * DP + C * lane;
#pragma unroll
        for (int c = 0; c < C; ++c) v[k][c] = p[c];
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {  // a part past the last has weight 0 (i + k < 64)
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i + k));
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] += i + k < n ? weighted(v[k][c], w) : 0.0f;
      }
    }
  }
  return j;
}

template <typename ET, int DP>
__device__ __forceinline__ void store_joined(const Joined<DP>& j, ET* out, float* lse,
                                             int32_t dim) {
  constexpr int C = DP / 64;
  const int lane = threadIdx.x & 63;
  const float inv = inverse(j.sum);
#pragma unroll
  for (int c = 0; c < C; ++c)
    if (C * lane + c < dim) out[C * lane + c] = (ET)(j.acc[c] * inv);
  if (lse && lane == 0) *lse = log_sum(j.m, j.sum);
}

}  // namespace attn
}  // namespace tod
