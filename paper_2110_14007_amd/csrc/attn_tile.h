// Attention tile: whole prompts, and chunks of new tokens over pages.
//
// A workgroup of 4 waves owns kRows = 128 packed rows of one key / value head,
// 32 a wave, and walks the keys in stages of 32 with one barrier a stage.  Rings
// of four stages of K and of V lie in LDS: a turn consumes stage j of the
// softmax, j + 1 of the first product and j - 1 of the second, which do not
// depend on each other, while the loads of K j + 3 and V j + 1 are in flight.
// Where a call has too few tiles for the GPU, each tile's keys are split over
// several workgroups and a second kernel joins their results.
//
// Bound by the matrix and vector instructions that a SIMD's two waves issue: a
// stage is 16 MFMAs (14.3 ns each from one SIMD), 16 exponentials a lane (4.6)
// and some 60 other vector instructions (2.1), and the clock falls to 1.75 GHz
// under them.  One prompt of 16,001 tokens, 32 heads of 128, takes 1.87 to 2.03 ms on
// four cards: 1,120 to 1,035 TFLOP/s of bf16, where an 8192^3 matrix product
// reaches 1,182.  32 rows a wave
// leave room for two workgroups a compute unit, whose waves fill each other's
// gaps; 64 rows a wave halve the LDS reads, but need all 512 registers and were
// slower.  24 packed prompts of up to 2,500 tokens take 0.49 to 0.60 ms, 850 to 700
// TFLOP/s: a third of a workgroup's time is its start and its stores there.
#pragma once

#include "attn_token.h"

namespace tod {
namespace attn {

constexpr int kWaves = 4;
constexpr int kRows = 32 * kWaves;  // rows of a workgroup
constexpr int kKeys = 32;           // keys of a stage
constexpr int kRing = 4;            // stages of K, and of V, in LDS
constexpr uint32_t kNoLoad = ~0u;   // offset of a lane that loads nothing

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
// a lane).  Starts that do not ascend can make it end at a sequence whose slots
// begin past b: that slot is left empty, as its rows would lie outside the call.
// Sequences of at most skip_rows rows are the token kernel's.
template <bool PAGED>
__device__ __forceinline__ bool find_tile(const AttnArgs& a, int32_t b, Tile* t) {
  const int lane = threadIdx.x & 63;
  auto slot_of = [&](int32_t s, int32_t start) {
    return (int32_t)(((int64_t)start * (int64_t)a.group.d) / kRows) + s;
  };
  // The answer lies in [lo, lo + span); each lane holds its candidate's row_start and cached
  // tokens, and one lane more the end of the last candidate.
  int32_t lo = 0, span = a.n_seq + 1, hit, begin, cached;
  for (;;) {
    const int32_t step = (span + 62) / 63;
    const int32_t s = min(lo + lane * step, a.n_seq);
    begin = start_of(a, s);
    cached = PAGED && s < a.n_seq ? a.cached[s] : 0;
    const bool under = lane * step < span && slot_of(s, begin) <= b;
    hit = max(__popcll(__ballot(under)), 1);
    if (step == 1) break;
    lo += (hit - 1) * step;
    span = min(step, span - (hit - 1) * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo + hit - 1);
  const int32_t first = __builtin_amdgcn_readlane(begin, hit - 1);
  *(Seq*)t = make_seq<PAGED>(a, lo, first, __builtin_amdgcn_readlane(begin, hit),
                             __builtin_amdgcn_readlane(cached, hit - 1));
  const int32_t row0 = (b - slot_of(lo, first)) * kRows;
  t->seq = lo;
  t->rows = t->n * (int32_t)a.group.d;
  if (row0 < 0 || row0 >= t->rows || (lo < a.n_seq && t->rows <= a.skip_rows)) return false;
  t->row0 = row0;
  const int32_t last = (int32_t)div_by((uint32_t)min(t->row0 + kRows - 1, t->rows - 1), a.group);
  t->seen = PAGED || a.causal ? min(t->shift + last + 1, t->keys) : t->keys;
  t->stages = (t->seen + kKeys - 1) / kKeys;
  t->parts = max(min(a.tile_parts, t->stages * kKeys / a.part_keys), 1);
  return true;
}

// LDS-DMA of 16 bytes a lane from base (of the wave) + off (see mt::dma16).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16_at(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off),
               "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ const void* uniform(const void* p) {
  const uint64_t u = (uint64_t)(uintptr_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return (const void*)(uintptr_t)(((uint64_t)hi << 32) | lo);
}

// Token workers that share a workgroup's LDS in a tile kernel's launch.
template <int DP>
constexpr int tile_workers() { return 2 * kRing * kKeys * DP * 2 / token_lds<DP>(); }

// The kernel's arguments, read anew: a branch that takes them this way leaves the scalar registers
// of the other one alone.
__device__ __forceinline__ AttnArgs own_args() {
  typedef const __attribute__((address_space(4))) uint64_t* words;
  words p = (words)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  struct { uint64_t w[sizeof(AttnArgs) / 8]; } v;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(AttnArgs) / 8); ++i) v.w[i] = p[i];
  return __builtin_bit_cast(AttnArgs, v);
}

// W: the elements of a row that the products take, of the DP that its stages have room for.  FULL:
// the rows have DP elements.
template <typename ET, int DP, int W, bool FULL, bool PAGED>
__global__ void __launch_bounds__(64 * kWaves, DP > 128 ? 1 : DP > 64 ? 2 : 3)
    tile_kernel(AttnArgs a) {
  using V8 = typename Frag<ET>::V;
  using St = Stager<ET, DP, PAGED>;
  constexpr int kStage = kKeys * DP;         // elements of a stage
  constexpr int kRowsWave = kKeys / kWaves;  // rows of a stage that a wave loads
  constexpr int kLoads = kRowsWave / St::kRowsLoad;
  constexpr int DB = W / 32, KC = W / 16;
  extern __shared__ __align__(16) uint16_t lds[];  // kRing K stages, then as many V stages

  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // The last workgroups, if any, are the token workers': they read the memory while the tiles
  // that are left compute.
  if constexpr (PAGED) {
    if (blockIdx.x >= a.tile_groups) {
      if (wave < tile_workers<DP>())
        token_work<ET, DP>(own_args(), (blockIdx.x - a.tile_groups) * tile_workers<DP>() + wave,
                           lds + wave * (token_lds<DP>() / 2));
      return;
    }
  }
  const uint32_t b = div_by(blockIdx.x, a.parts_div), part = blockIdx.x - b * a.parts_div.d;
  const uint32_t at = div_by(b, a.heads_div), head = b - at * a.heads_div.d;
  Tile t;
  // Late rows see the most keys: they are taken first.
  if (!find_tile<PAGED>(a, a.tile_slots - 1 - (int32_t)at, &t) || (int)part >= t.parts) return;
  const int32_t jb = (int32_t)((uint32_t)t.stages * part / (uint32_t)t.parts);
  const int32_t count = (int32_t)((uint32_t)t.stages * (part + 1) / (uint32_t)t.parts) - jb;

  // This lane's query row, and the last key that it sees.
  const int32_t m = min(t.row0 + 32 * wave + col, t.rows - 1);
  const int32_t tok = (int32_t)div_by((uint32_t)m, a.group);
  const int32_t qh = (int32_t)head * (int32_t)a.group.d + m - tok * (int32_t)a.group.d;
  const int32_t limit = PAGED || a.causal ? min(t.shift + tok, t.keys - 1) : t.keys - 1;
  // Stages (of this split's) whose keys every row of the tile sees.
  const int32_t tok0 = (int32_t)div_by((uint32_t)t.row0, a.group);
  const int32_t least = PAGED || a.causal ? min(t.shift + tok0, t.keys - 1) : t.keys - 1;
  const int32_t open = min(max((least + 1) / kKeys - jb, 0), count);
  V8 q[KC];
  load_query<ET, W>(q, (const ET*)a.q + (int64_t)(t.start + tok) * a.q_row + (int64_t)qh * a.q_head,
                     a.dim, h);

  // Staging.
  St st(a, head);
  st.seq = t.seq;
  st.start = t.start;
  st.seen = t.seen;
  const uint32_t base = mt::lds_off(lds);
  constexpr int kTurns = St::kRowsLoad < 4 ? 4 / St::kRowsLoad : 1;  // loads until V's swizzle repeats
  uint32_t ko[kLoads], vo[kTurns];
  {
    const int r = lane / St::kPieces, pc = lane % St::kPieces;
    const int64_t kr = PAGED ? a.dim : a.k_row, vr = PAGED ? a.dim : a.v_row;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = wave * kRowsWave + i * St::kRowsLoad + r;
      const int c = 8 * (pc ^ swizzle_k<DP>(row));
      ko[i] = c < a.dim ? (uint32_t)(2 * (kr * r + c)) : kNoLoad;
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int c = 8 * (pc ^ swizzle_v<DP>(i * St::kRowsLoad + r));
      vo[i] = c < a.dim ? (uint32_t)(2 * (vr * r + c)) : kNoLoad;
    }
  }
  // Whole stages whose rows of a wave lie together move by a base of the wave and an offset of
  // the lane that stays; the others (the last stage, small or odd pages, strides for which those
  // offsets would pass 32 bits) one by one.  Pieces from dim on are not loaded: the stages are
  // cleared once.  (Of every load some lane has a piece, so that the loads in flight count the same.)
  const bool plain = PAGED ? a.page.d % kRowsWave == 0 : max(a.k_row, a.v_row) < (1 << 27);
  const int32_t fast = plain ? __builtin_amdgcn_readfirstlane(t.seen / kKeys - jb) : 0;
  const int32_t first = __builtin_amdgcn_readfirstlane(jb * kKeys + wave * kRowsWave);
  const ET *kb, *vb;
  if constexpr (!PAGED) {
    kb = (const ET*)uniform((const ET*)a.k + (int64_t)(t.start + first) * a.k_row +
                            (int64_t)head * a.k_head);
    vb = (const ET*)uniform((const ET*)a.v + (int64_t)(t.start + first) * a.v_row +
                            (int64_t)head * a.v_head);
  }
  // Stage i of this split's into buffer `ring`; each of K and V in turn from 0 on.
  auto stage = [&](auto ISK, int32_t i, int ring) __attribute__((always_inline)) {
    constexpr bool isk = decltype(ISK)::value;
    if (i >= count) return;
    const uint32_t buf = 2u * kStage * (uint32_t)(ring + (isk ? 0 : kRing));
    uint32_t row = 0;
    if constexpr (PAGED) row = i < fast ? st.row_of(first + i * kKeys) : ~0u;
    if (PAGED ? row != ~0u : i < fast) {
      const ET* p;
      int64_t stride = FULL ? DP : a.dim;
      if constexpr (PAGED) {
        p = (const ET*)(isk ? a.k : a.v) + (int64_t)row * stride;
      } else {
        stride = isk ? a.k_row : a.v_row;
        p = isk ? kb : vb;
        (isk ? kb : vb) += kKeys * stride;
      }
#pragma unroll
      for (int l = 0; l < kLoads; ++l) {
        const uint32_t off = isk ? ko[l] : vo[l % kTurns];
        if (FULL || off != kNoLoad)
          dma16_at(p + l * St::kRowsLoad * stride, off,
                   base + buf + 2u * (uint32_t)(wave * kRowsWave * DP + l * St::kRowsLoad * DP));
      }
      return;
    }
    const uint32_t at = st.place((jb + i) * kKeys, kKeys);
#pragma unroll
    for (int l = 0; l < kLoads; ++l)
      st.load_one(isk, at, wave * kRowsWave + l * St::kRowsLoad, base + buf);
  };
  constexpr std::true_type kIsK{};
  constexpr std::false_type kIsV{};

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
  float mref = kNoMax, few = 0.0f;  // few: weights of up to four stages, on their way to acc
  Sum acc;
  float limit_raw = -INFINITY;  // a score above it makes m follow
  // P of the stage before the first is zero, and so must its values be.
  for (int i = (FULL ? 2 * kRing - 1 : 0) * kStage / 8 + tid; i < 2 * kRing * kStage / 8;
       i += 64 * kWaves)
    ((uint4*)lds)[i] = uint4{0, 0, 0, 0};
  if constexpr (!FULL) mt::stage_barrier();

  // LDS addresses of this lane's fragments in buffer 0; the rest is a constant offset.
  typedef __attribute__((address_space(3))) const char* ldsp;
  const ldsp lbase = (ldsp)(__attribute__((address_space(3))) uint16_t*)lds;
  ldsp ka[KC], va[2];
#pragma unroll
  for (int c = 0; c < KC; ++c)
    ka[c] = lbase + 2 * (col * DP + 8 * ((2 * c + h) ^ swizzle_k<DP>(col)));
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    const int row = 4 * h + (lane & 15) / 4;
    const int piece = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    va[d] = lbase + 2 * (kRing * kStage + row * DP + 8 * (piece ^ swizzle_v<DP>(row)) + 4 * (lane & 1));
  }
  // at: byte offset of the 32 (K) or 16 (V) rows in the ring.
  auto kfrag = [&](int at, int c) {
    return *(const __attribute__((address_space(3))) V8*)(ka[c] + at);
  };
  auto vfrag = [&](int at, int d) {
    typedef __attribute__((address_space(3))) s16x4* lds4;
    const ldsp q0 = va[d & 1] + at + (d >> 1) * 128;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)q0);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(q0 + 8 * DP * 2));
    return __builtin_bit_cast(V8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };

  // One step: softmax of the 32 keys from j0 on (scores s -> weights pn), the scores of the next
  // 32 (n; at kat in the K ring) and the product of the 32 before (weights p; at vat in the V
  // ring).  The three do not depend on each other.  They are laid out in slots of one MFMA, the
  // LDS reads of the MFMA kAhead slots on, and a share of the exponentials.
  constexpr int kSlots = KC + 2 * DB, kAhead = 4, kCheck = 2;
  auto step = [&](int32_t j0, int kat, int vat, f32x16& s, f32x16& n,
                  const u32x4 (&p0)[2], u32x4 (&pn)[2]) __attribute__((always_inline)) {
    u32x4 p[2] = {p0[0], p0[1]};
    V8 fr[kSlots];
    auto read = [&](auto I) __attribute__((always_inline)) {
      constexpr int i = decltype(I)::value;
      if constexpr (i < KC)
        fr[i] = kfrag(kat, i);
      else if constexpr (i < kSlots)
        fr[i] = vfrag(vat + 16 * ((i - KC) / DB) * DP * 2, (i - KC) % DB);
    };
    mt::static_for<0, kAhead>([&](auto I) __attribute__((always_inline)) { read(I); });
    if (j0 + kKeys - 1 > least) {
      const int32_t left = limit - j0 - 4 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (mt::out_row_c(r) > left) s[r] = -INFINITY;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) n[r] = 0.0f;
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    mt::static_for<0, kSlots>([&](auto I) __attribute__((always_inline)) {
      constexpr int i = decltype(I)::value;
      if constexpr (i < KC)
        n = mfma<ET>(fr[i], q[i], n);
      else
        o[(i - KC) % DB] = mfma<ET>(fr[i], __builtin_bit_cast(V8, p[(i - KC) / DB]), o[(i - KC) % DB]);
      read(std::integral_constant<int, i + kAhead>{});
      if constexpr (i == kCheck - 1) {
        if (__builtin_expect(__ballot(top > limit_raw) != 0, 0)) {
          // m follows the maximum only when that has grown by more than kSlack, so that most
          // steps rescale nothing.  The product of the 32 keys before is still to come: its weights
          // follow m too.
          constexpr float kRoom = kSlack<ET> + kBias<ET>;
          const float raw = fmaxf(top, other_half(top)), t2 = raw * a.scale;
          const bool far = fabsf(fmaxf(t2, mref)) > kFar;  // m follows every growth
          const float next = t2 > mref + (far ? 0.0f : kRoom) ? t2 - (far ? 0.0f : kBias<ET>) : mref;
          const float f = __builtin_amdgcn_exp2f(mref - next);
          mref = next;
          limit_raw = far ? fmaxf(raw, limit_raw) : (next + kRoom) * a.unscale;
          acc.scale(f);
          few *= f;
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] *= f;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const V8 w = __builtin_bit_cast(V8, p[c]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              p[c][e] = pack2<ET>((float)w[2 * e] * f, (float)w[2 * e + 1] * f);
          }
        }
      }
      if constexpr (i >= kCheck) {
        constexpr int k = i - kCheck, of = kSlots - kCheck;
        constexpr int e0 = (8 * k + of - 1) / of, e1 = (8 * (k + 1) + of - 1) / of;  // pairs
#pragma unroll
        for (int e = e0; e < e1; ++e) {
          // The weights are rounded to the input type for the second product (half an ulp each,
          // unbiased, like the inputs' own rounding): two products of their halves would cost
          // half again as many MFMAs as the tile has.
          const float x0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * e], a.scale, -mref));
          const float x1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * e + 1], a.scale, -mref));
          few += x0;
          few += x1;
          pn[e / 4][e % 4] = pack2<ET>(x0, x1);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    });
  };

  constexpr int kS = 2 * kStage;  // bytes of a stage
  // Values that some rows of the tile do not see meet their zero weights in the second product,
  // which is no zero where a value is not finite.  Those values are cleared in their stage (of
  // index i), and what they make of the rows that do see them is restored at the end, as it is for
  // values that all rows see.
  bool cleared = false;
  auto clear = [&](int32_t i) __attribute__((always_inline)) {
    if (!(PAGED || a.causal)) return;
    uint16_t* const vs = lds + (kRing + i % kRing) * kStage;
    if (!holds_nonfinite<ET, DP>(vs)) return;
    cleared = true;
    mt::stage_barrier();
    clear_nonfinite<ET, DP>(vs, wave * 64, kWaves * 64);
    mt::stage_barrier();
  };
  f32x16 sa, sb;
  u32x4 pa[2], pb[2];
  pb[0] = pb[1] = u32x4{0, 0, 0, 0};
  stage(kIsK, 0, 0);
  stage(kIsK, 1, 1);
  stage(kIsV, 0, 0);
  stage(kIsK, 2, 2);
  mt::dl_barrier<0>();
#pragma unroll
  for (int r = 0; r < 16; ++r) sa[r] = 0.0f;
#pragma unroll
  for (int c = 0; c < KC; ++c) sa = mfma<ET>(kfrag(0, c), q[c], sa);
  auto turn = [&](int32_t j, int r, f32x16& s, f32x16& n, const u32x4 (&p)[2],
                  u32x4 (&pn)[2]) __attribute__((always_inline)) {  // r: j % kRing
    // The loads of the turn before stay in flight while there are as many as a turn issues.
    if (j + 2 < count)
      mt::dl_barrier<2 * kLoads>();
    else
      mt::dl_barrier<0>();
    stage(kIsK, j + 3, (r + 3) % kRing);
    stage(kIsV, j + 1, (r + 1) % kRing);
    if (j > open) clear(j - 1);
    step((jb + j) * kKeys, (r + 1) % kRing * kS, (r + kRing - 1) % kRing * kS, s, n, p, pn);
  };
  // Scores and weights change places every turn: a pass of the loop takes an even number.
  for (int32_t j = 0; j < count; j += 4) {
    turn(j, 0, sa, sb, pb, pa);
    if (j + 1 >= count) break;
    turn(j + 1, 1, sb, sa, pa, pb);
    if (j + 2 >= count) break;
    turn(j + 2, 2, sa, sb, pb, pa);
    if (j + 3 >= count) break;
    turn(j + 3, 3, sb, sa, pa, pb);
    acc.add(few);
    few = 0.0f;
  }
  acc.add(few);
  if (count > 0) {
    if (count > open) clear(count - 1);
    const int at = (count - 1) % kRing * kS;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int d = 0; d < DB; ++d)
        o[d] = mfma<ET>(vfrag(at + 16 * c * DP * 2, d),
                        __builtin_bit_cast(V8, count % 2 ? pa[c] : pb[c]), o[d]);
  }
  const float sum = acc.v + other_half(acc.v);
  const bool restore = cleared || met_nonfinite(o, sum);
  const bool mine = t.row0 + 32 * wave + col < t.rows;
  if (t.parts > 1) {
    const int64_t row = ((int64_t)b * a.tile_parts + part) * kRows + 32 * wave + col;
    if (mine) store_part<W>(o, a.tile_o + row * DP, h);
    if (mine && h == 0) a.tile_stat[row] = {mref, sum};
    if (restore)
      restore_nonfinite<ET, DP, PAGED>(st, a.tile_o + (row - col) * DP, DP, t, t.row0 + 32 * wave,
                                       jb * kKeys, (jb + count) * kKeys, sum);
    return;
  }
  const int64_t orow = (int64_t)(t.start + tok) * a.heads + qh;
  if (mine && a.lse && h == 0) a.lse[orow] = log_sum(mref, sum);
  mt::stage_barrier();  // the other waves' reads of the stages are done
  store_rows<ET, DP, W>(o, inverse(sum), (ET*)a.out, mine ? orow * a.dim : -1, a.dim,
                     lds + wave * 32 * DP);
  if (restore)
    restore_nonfinite<ET, DP, PAGED>(st, (ET*)a.out, 0, t, t.row0 + 32 * wave, jb * kKeys,
                                     (jb + count) * kKeys, sum);
}

// Joins the splits of a tile, one wave a row.
template <typename ET, int DP, bool PAGED>
__global__ void __launch_bounds__(256) tile_join_kernel(AttnArgs a) {
  constexpr int kRowsGroup = 16;
  const int first = (int)(blockIdx.x % (kRows / kRowsGroup)) * kRowsGroup;
  const uint32_t b = blockIdx.x / (kRows / kRowsGroup);
  const uint32_t at = div_by(b, a.heads_div), head = b - at * a.heads_div.d;
  Tile t;
  if (!find_tile<PAGED>(a, a.tile_slots - 1 - (int32_t)at, &t) || t.parts == 1) return;
  for (int r = first + (threadIdx.x >> 6); r < first + kRowsGroup; r += 4) {
    const int32_t m = t.row0 + r;
    if (m >= t.rows) break;
    const int32_t tok = (int32_t)div_by((uint32_t)m, a.group);
    const int32_t qh = (int32_t)head * (int32_t)a.group.d + m - tok * (int32_t)a.group.d;
    const int64_t orow = (int64_t)(t.start + tok) * a.heads + qh;
    const int64_t row = (int64_t)b * a.tile_parts * kRows + r;
    store_joined<ET, DP>(
        join_parts<DP>(a.tile_stat, a.tile_o, row, row + kRows, kRows, 0, t.parts),
        (ET*)a.out + orow * a.dim, a.lse ? a.lse + orow : nullptr, a.dim);
  }
}

template <typename ET, int DP, int W, bool FULL, bool PAGED>
hipError_t launch_tile(const AttnArgs& a, hipStream_t s) {
  const int64_t slots = a.tile_slots;
  constexpr unsigned bytes = 2 * kRing * kKeys * DP * 2;  // K and V, 16 bits
  const auto kern = tile_kernel<ET, DP, W, FULL, PAGED>;
  if constexpr (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(
        (const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
  }
  const int64_t tokens = PAGED && a.skip_rows ? token_workers(DP) / tile_workers<DP>() : 0;
  hipLaunchKernelGGL(kern, dim3((unsigned)(a.tile_groups + tokens)), dim3(64 * kWaves), bytes, s, a);
  if (a.tile_parts > 1)
    hipLaunchKernelGGL((tile_join_kernel<ET, DP, PAGED>),
                       dim3((unsigned)(slots * a.kv_heads * (kRows / 16))), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename ET, bool PAGED>
hipError_t launch_tile(const AttnArgs& a, hipStream_t s) {
  if (a.dim < 64) return launch_tile<ET, 64, 64, false, PAGED>(a, s);
  if (a.dim == 64) return launch_tile<ET, 64, 64, true, PAGED>(a, s);
  if (a.dim <= 96) return launch_tile<ET, 128, 96, false, PAGED>(a, s);
  if (a.dim < 128) return launch_tile<ET, 128, 128, false, PAGED>(a, s);
  if (a.dim == 128) return launch_tile<ET, 128, 128, true, PAGED>(a, s);
  if (a.dim < 256) return launch_tile<ET, 256, 256, false, PAGED>(a, s);
  return launch_tile<ET, 256, 256, true, PAGED>(a, s);
}

}  // namespace attn
}  // namespace tod
