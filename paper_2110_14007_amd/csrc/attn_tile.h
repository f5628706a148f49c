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
constexpr int kWideWaves = 8, kWideRows = 32 * kWideWaves;  // of the wide kernel
constexpr int kKeys = 64;           // keys of a stage
constexpr float kSlack = 8.0f;  // growth of the maximum (log2) that m may lag behind

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
template <bool PAGED, int kRows>
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
  t->parts = max(min(a.tile_parts, t->stages / a.part_stages), 1);
  return true;
}

template <typename ET, int DP, bool PAGED>
__global__ void __launch_bounds__(64 * kWaves, DP > 128 ? 1 : 2) tile_kernel(AttnArgs a) {
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
  if (!find_tile<PAGED, kRows>(a, slot, &t) || (int)part >= t.parts) return;
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
    const int64_t row = ((int64_t)b * a.tile_parts + part) * kRows + 32 * wave + col;
    store_part<DP>(o, a.tile_o + row * DP, h);
    if (h == 0) a.tile_stat[row] = {mref, sum};
    return;
  }
  const int64_t orow = (int64_t)(t.start + tok) * a.heads + qh;
  store_row<ET, DP>(o, inverse(sum), (ET*)a.out + orow * a.dim, a.dim, h);
  if (a.lse && h == 0) a.lse[orow] = log_sum(mref, sum);
}


// LDS-DMA of 16 bytes a lane from base + off (see mt::dma16).
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

template <typename ET, int DP, bool PAGED>
__global__ void __launch_bounds__(64 * kWideWaves, 2) wide_kernel(AttnArgs a) {
  using V8 = typename Frag<ET>::V;
  using St = Stager<ET, DP, PAGED>;
  constexpr int kRows = kWideRows;
  constexpr int kStage = kKeys * DP;         // elements of a stage
  constexpr int kRowsWave = kKeys / kWideWaves;  // rows of a stage that a wave loads
  constexpr int kLoads = kRowsWave / St::kRowsLoad;
  constexpr int DB = DP / 32, KC = DP / 16;
  constexpr int kRing = 3;
  constexpr int kBeside = KC / 2 + 2 * DB;
  constexpr int kValuBeside = (56 + kBeside - 1) / kBeside;
  extern __shared__ __align__(16) uint16_t lds[];  // three K stages, then three V stages

  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint32_t b = blockIdx.x;
  const uint32_t part = b % (uint32_t)a.tile_parts;
  b /= (uint32_t)a.tile_parts;
  const uint32_t head = b % (uint32_t)a.kv_heads;
  const int64_t slots = gridDim.x / ((uint32_t)a.kv_heads * (uint32_t)a.tile_parts);
  const int64_t slot = slots - 1 - b / (uint32_t)a.kv_heads;
  Tile t;
  if (!find_tile<PAGED, kRows>(a, slot, &t) || (int)part >= t.parts) return;
  const int32_t jb = (int32_t)((int64_t)t.stages * part / t.parts);
  const int32_t count = (int32_t)((int64_t)t.stages * (part + 1) / t.parts) - jb;

  // This lane's query row, and the last key that it sees.
  const int32_t m = min(t.row0 + 32 * wave + col, t.rows - 1);
  const int32_t tok = (int32_t)div_by((uint32_t)m, a.group);
  const int32_t qh = (int32_t)head * (int32_t)a.group.d + m - tok * (int32_t)a.group.d;
  const int32_t limit = PAGED || a.causal ? min(t.shift + tok, t.keys - 1) : t.keys - 1;
  const int32_t wlo = __builtin_amdgcn_readfirstlane(limit);
  V8 q[KC];
  load_query<ET, DP>(q, (const ET*)a.q + (int64_t)(t.start + tok) * a.q_row + (int64_t)qh * a.q_head,
                     a.dim, h);

  // Staging.
  St st(a, head);
  st.seq = t.seq;
  st.start = t.start;
  st.seen = t.seen;
  const uint32_t base = mt::lds_off(lds);
  auto kbuf = [&](int32_t j) { return (uint32_t)((j + kRing) % kRing) * kStage; };
  auto vbuf = [&](int32_t j) { return (uint32_t)(kRing + (j + kRing) % kRing) * kStage; };
  uint32_t ko[kLoads], vo;
  {
    const int r = lane / St::kPieces, pc = lane % St::kPieces;
    const int64_t kr = PAGED ? a.dim : a.k_row, vr = PAGED ? a.dim : a.v_row;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = wave * kRowsWave + i * St::kRowsLoad + r;
      ko[i] = (uint32_t)(2 * (kr * r + 8 * (pc ^ swizzle_k<DP>(row))));
    }
    vo = (uint32_t)(2 * (vr * r + 8 * (pc ^ swizzle_v<DP>(r))));
  }
  // Whole stages whose rows of a wave lie together move by a base of the wave and an offset of
  // the lane that stays; the others (the last stage, small or odd pages, padded rows) one by one.
  const bool plain = a.dim == DP && (!PAGED || a.page.d % kRowsWave == 0);
  auto stage = [&](bool isk, int32_t i0) {  // stage i0 of this split's
    if (i0 >= count) return;
    const int32_t j = jb + i0;
    const uint32_t to = base + 2u * ((isk ? kbuf(i0) : vbuf(i0)) + (uint32_t)(wave * kRowsWave * DP));
    const int32_t j0 = j * kKeys + wave * kRowsWave;
    if (plain && (j + 1) * kKeys <= t.seen) {
      const ET* p;
      int64_t stride;
      if constexpr (PAGED) {
        const uint32_t at = st.place(j * kKeys, kKeys);
        const uint32_t row = __builtin_amdgcn_readlane(at, wave * kRowsWave);
        p = (const ET*)(isk ? a.k : a.v) + (int64_t)row * DP;
        stride = DP;
        if (row == ~0u) goto slow;
      } else {
        p = (isk ? (const ET*)a.k + (int64_t)(t.start + j0) * a.k_row + (int64_t)head * a.k_head
                 : (const ET*)a.v + (int64_t)(t.start + j0) * a.v_row + (int64_t)head * a.v_head);
        stride = isk ? a.k_row : a.v_row;
      }
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        dma16_at(uniform(p + i * St::kRowsLoad * stride), isk ? ko[i] : vo,
                 to + 2u * (uint32_t)(i * St::kRowsLoad * DP));
      return;
    }
  slow:
    const uint32_t at = st.place(j * kKeys, kKeys);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      st.load_one(isk, at, wave * kRowsWave + i * St::kRowsLoad, base + 2u * (isk ? kbuf(i0) : vbuf(i0)));
  };

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
  float mref = kNoMax, sum = 0.0f;
  // P of the stage before the first is zero, and so must its values be.
  for (int i = tid; i < kStage / 8; i += 64 * kWideWaves)
    ((uint4*)(lds + vbuf(-1)))[i] = uint4{0, 0, 0, 0};
  u32x4 p[2];  // [16 keys]
  p[0] = p[1] = u32x4{0, 0, 0, 0};

  // LDS addresses of this lane's fragments in buffer 0; the rest is an offset of the wave.
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

  f32x16 s;
  // One step: softmax of the 32 keys from j0 on (scores s), the scores of the next 32 (at kat in
  // the K ring) and the product of the 32 before (at vat in the V ring).  The three do not depend
  // on each other, so the wave's MFMAs run under its exponentials.
  auto step = [&](int32_t j0, auto KAT, auto VAT) __attribute__((always_inline)) {
    constexpr int kat = decltype(KAT)::value, vat = decltype(VAT)::value;
    f32x16 x = s;
    if (j0 + 31 > wlo) {
      const int32_t left = limit - j0 - 4 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (mt::out_row_c(r) > left) x[r] = -INFINITY;
    }
    f32x16 n;
#pragma unroll
    for (int r = 0; r < 16; ++r) n[r] = 0.0f;
#pragma unroll
    for (int c = 0; c < KC / 2; ++c) n = mfma<ET>(kfrag(kat, c), q[c], n);
    float top = x[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, x[r]);
    top = fmaxf(top, other_half(top)) * a.scale;
    const bool grow = top > mref + kSlack;
    if (__builtin_expect(__ballot(grow) != 0, 0)) {
      // The product of the 32 keys before is still to come: its P follows m too.
      const float next = grow ? top : mref;
      const float f = __builtin_amdgcn_exp2f(mref - next);
      mref = next;
      sum *= f;
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
      asm volatile("" ::: "memory");
    }
#pragma unroll
    for (int c = KC / 2; c < KC; ++c) n = mfma<ET>(kfrag(kat, c), q[c], n);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int d = 0; d < DB; ++d)
        o[d] = mfma<ET>(vfrag(vat + 16 * c * DP * 2, d), __builtin_bit_cast(V8, p[c]), o[d]);
    u32x4 pn[2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 8 * c + 2 * e;
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.scale, -mref));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r + 1], a.scale, -mref));
        sum += p0;
        sum += p1;
        pn[c][e] = pack2<ET>(p0, p1);
      }
    // One MFMA, then what fits beside it.
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < kBeside; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, kValuBeside, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    s = n;
    asm volatile("" : "+v"(pn[0]), "+v"(pn[1]), "+v"(sum));  // computed here, not where used
    p[0] = pn[0];
    p[1] = pn[1];
  };

  constexpr int kS = 2 * kStage, kH = 32 * DP * 2;  // bytes of a stage and of half of it
  stage(true, 0);
  stage(true, 1);
  stage(false, 0);
  mt::dl_barrier<0>();
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll
  for (int c = 0; c < KC; ++c) s = mfma<ET>(kfrag(0, c), q[c], s);
  auto turn = [&](int32_t j, auto R) __attribute__((always_inline)) {
    constexpr int r = decltype(R)::value;  // j % kRing
    mt::dl_barrier<0>();
    stage(true, j + 2);
    stage(false, j + 1);
    step((jb + j) * kKeys, std::integral_constant<int, r * kS + kH>{},
         std::integral_constant<int, (r + 2) % 3 * kS + kH>{});
    step((jb + j) * kKeys + 32, std::integral_constant<int, (r + 1) % 3 * kS>{},
         std::integral_constant<int, r * kS>{});
  };
  for (int32_t j = 0; j < count; j += 3) {
    turn(j, std::integral_constant<int, 0>{});
    if (j + 1 < count) turn(j + 1, std::integral_constant<int, 1>{});
    if (j + 2 < count) turn(j + 2, std::integral_constant<int, 2>{});
  }
  if (count > 0) {
    const int at = (count - 1) % kRing * kS + kH;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int d = 0; d < DB; ++d)
        o[d] = mfma<ET>(vfrag(at + 16 * c * DP * 2, d), __builtin_bit_cast(V8, p[c]), o[d]);
  }
  sum += other_half(sum);
  if (t.row0 + 32 * wave + col >= t.rows) return;
  if (t.parts > 1) {
    const int64_t row = ((int64_t)b * a.tile_parts + part) * kRows + 32 * wave + col;
    store_part<DP>(o, a.tile_o + row * DP, h);
    if (h == 0) a.tile_stat[row] = {mref, sum};
    return;
  }
  const int64_t orow = (int64_t)(t.start + tok) * a.heads + qh;
  store_row<ET, DP>(o, inverse(sum), (ET*)a.out + orow * a.dim, a.dim, h);
  if (a.lse && h == 0) a.lse[orow] = log_sum(mref, sum);
}

// Joins the splits of a tile, one wave a row.
template <typename ET, int DP, bool PAGED, int kRows>
__global__ void __launch_bounds__(256) tile_join_kernel(AttnArgs a) {
  constexpr int kRowsGroup = 16;
  uint32_t b = blockIdx.x;
  const int first = (int)(b % (kRows / kRowsGroup)) * kRowsGroup;
  b /= kRows / kRowsGroup;
  const uint32_t head = b % (uint32_t)a.kv_heads;
  const int64_t slots = gridDim.x / ((uint32_t)a.kv_heads * (kRows / kRowsGroup));
  Tile t;
  if (!find_tile<PAGED, kRows>(a, slots - 1 - b / (uint32_t)a.kv_heads, &t) || t.parts == 1) return;
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

template <typename ET, int DP, bool PAGED, int kRows>
hipError_t launch_rows(const AttnArgs& a, hipStream_t s) {
  constexpr bool wide = kRows == kWideRows;
  const int64_t slots = (int64_t)a.tokens * a.group.d / kRows + a.n_seq + 1;
  constexpr unsigned bytes = 2 * (wide ? 3 : 2) * kKeys * DP * 2;  // K and V stages, 16 bits
  constexpr unsigned threads = 64 * (wide ? kWideWaves : kWaves);
  void (*kern)(AttnArgs);
  if constexpr (wide)
    kern = wide_kernel<ET, DP, PAGED>;
  else
    kern = tile_kernel<ET, DP, PAGED>;
  if constexpr (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(
        (const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)(slots * a.kv_heads * a.tile_parts)), dim3(threads),
                     bytes, s, a);
  if (a.tile_parts > 1)
    hipLaunchKernelGGL((tile_join_kernel<ET, DP, PAGED, kRows>),
                       dim3((unsigned)(slots * a.kv_heads * (kRows / 16))), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename ET, int DP, bool PAGED>
hipError_t launch_tile(const AttnArgs& a, hipStream_t s) {
  if constexpr (DP <= 128)
    if (a.tile_rows == kWideRows) return launch_rows<ET, DP, PAGED, kWideRows>(a, s);
  return launch_rows<ET, DP, PAGED, kRows>(a, s);
}

}  // namespace attn
}  // namespace tod
