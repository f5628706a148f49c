// Attention tiles over a 4-bit cache: the steps of attn_tile.h (S^T = K Q^T, the
// softmax in a lane, P from the accumulators, three products' work in slots of
// one MFMA), with stages that are converted on the way.  A wave loads its eight
// rows of a stage's codes into registers a turn ahead and writes their values to
// LDS between the products, word by word: conversions and LDS writes then fill
// slots that the matrix pipe leaves.  Bound by the products and what is issued
// beside them, as over 16-bit pages: fewer vector instructions or other orders changed
// the time by 1% at most, and cards differ by 10% by their clocks.
//
// The tiles of all sequences and key / value heads form one line, each as long
// as the keys that it sees and a constant for its start and its stores, and as
// many workgroups as fit on the GPU at once take shares of it, wherever those
// begin and end: chunks of prompts over caches of any lengths beside each
// other leave no worker waiting for the longest, and a single chunk is shared by
// all.  At most the first and the last tile of a share are cut; of those a
// worker leaves (m, sum, O) and a second kernel joins the pieces.
//
// The lengths are known on the device only.  Tile i of a sequence weighs
// base + step (i + 1), so that the line's sums have a closed form: the worker
// finds its place in it by the sequences' sums, one segment a lane, and a root.
//
// Sequences of few rows are the token workers' of attn_token4.h, which here are
// the tiles' waves: half of the workgroups begin with them, half end with them, so
// that the memory is read while products are formed.
//
// Measured, rows of 128, whole calls: a chunk of 512 after 60,007, 16 / 2 heads, fp16
// 284 us (910 TFLOP/s); 12 prompts of 90 to 2,500, 32 / 8 heads 310 us; a prompt of
// 8,000 558 us (940 TFLOP/s); 4 chunks and 40 tokens 203 us.  Steps on the way: tiles in
// a grid with the keys of all split alike, as over 16-bit pages, 308 us for those 4
// chunks and 40 tokens, dealt 255; tokens in a launch of their own 235, in this one 223.
// Conversions in front of the products instead of between them: 338 us for the chunk, where
// this took 316; pages found between the products, whose branches moved the exponentials
// behind them, 297 and 284.  8 chunks of 300 to 600, rows of 64: 230 us with three
// workgroups a unit, 256 with two.
#pragma once

#include "attn_tile.h"
#include "attn_token4.h"

namespace tod {
namespace attn {

// Of a tile's start and stores, in keys.  (12 prompts of 90 to 2,500: 343 us with 256, 388 with 128,
// 353 with 384, 378 with 640.)
constexpr int32_t kTileWeight = 256;
// Least weight of a worker's share, where there are few tiles.  (60 tokens after 500, 32 / 8 heads:
// 27 us with 128, 28 with 64, 33 with 32, 37 with 512; a prompt of 300: 30, 35, 35 and 36.)
constexpr int32_t kShareKeys = 128;
// Stages that a cut leaves on either side, else it moves to the tile's end: a piece has its partial
// results to store and to join.  (A prompt of 300 25 us with 6, 30 with 4; 100 prompts of 100 to 200
// 124 us with 4 to 16, 141 with 1; 6 chunks and 54 tokens 140 us, 147 with 12.)
constexpr int32_t kLeastPiece = 6;
constexpr int32_t kUnits = 32;  // compute units of an XCD
// By which the share of a unit's first workgroup is larger.  (12 prompts 325 us with 0.15, 339 with 0,
// 330 with 0.2; a chunk of 512 after 60,007 298, 309 and 301; one of 64 after 30,000, whose shares are
// short, 72 and 68 with 0.)
constexpr double kOlder = 0.15;

// The tiles of a sequence (of one key / value head).
struct Tiles {
  int32_t count;
  int64_t base, step;
  __device__ __forceinline__ int64_t before(int64_t i) const {  // weight of the first i
    return i * base + step * (i * (i + 1) / 2);
  }
  __device__ __forceinline__ int64_t all() const { return before(count); }
  // The tile that holds weight y, 0 <= y < all().
  __device__ __forceinline__ int32_t at(int64_t y) const {
    const double b = (double)base + 0.5 * (double)step;
    int64_t i = (int64_t)(2.0 * (double)y / (b + sqrt(b * b + 2.0 * (double)step * (double)y)));
    i = min(max(i, (int64_t)0), (int64_t)count - 1);
    while (i > 0 && before(i) > y) --i;
    while (i + 1 < count && before(i + 1) <= y) ++i;
    return (int32_t)i;
  }
};

// Sequence s; after the last one come the rows past row_start[n_seq], which have no keys.
__device__ __forceinline__ Tiles tiles_of(const AttnArgs& a, int32_t s, const Seq& q) {
  const int32_t rows = q.n * (int32_t)a.group.d;
  if (s > a.n_seq || rows <= 0 || (s < a.n_seq && rows <= a.skip_rows)) return {0, kTileWeight, 0};
  const bool keys = q.keys > 0;
  return {(rows + kRows - 1) / kRows, kTileWeight + (keys ? q.shift : 0),
          keys ? max(kRows / (int32_t)a.group.d, 1) : 0};
}
__device__ __forceinline__ int64_t uniform64(int64_t v) {
  const uint32_t lo = (uint32_t)uniform((int32_t)v), hi = (uint32_t)uniform((int32_t)(v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// floor(n / d) for 0 <= n, 0 < d and a quotient below 2^31, by an estimate that is off by one at most.
__device__ __forceinline__ int32_t ratio(int64_t n, int64_t d) {
  int64_t q = (int64_t)((double)n / (double)d);
  q -= q * d > n ? 1 : 0;
  q += (q + 1) * d <= n ? 1 : 0;
  return (int32_t)q;
}

__device__ __forceinline__ Tile tile_at(const AttnArgs& a, int32_t s, const Seq& q, int32_t i) {
  Tile t;
  *(Seq*)&t = q;
  t.seq = s;
  t.rows = t.n * (int32_t)a.group.d;
  t.row0 = i * kRows;
  const int32_t last = (int32_t)div_by((uint32_t)min(t.row0 + kRows - 1, t.rows - 1), a.group);
  t.seen = min(t.shift + last + 1, t.keys);
  t.stages = (t.seen + kKeys - 1) / kKeys;
  t.parts = 1;
  return t;
}

// The line, lane l's segment of the sequences, the same in every wave.
struct TileLine {
  int32_t seg;
  Seq own;             // the lane's sequence, where a segment is one
  int64_t incl, mine;  // weights of a key / value head: up to and with the segment, and of it
  int64_t all;         // of all heads
  int32_t workers;     // that have a share

  __device__ __forceinline__ TileLine(const AttnArgs& a) {
    const int lane = threadIdx.x & 63;
    seg = (a.n_seq + 1 + 63) / 64;
    int64_t tiles = 0, tokens = 0;
    mine = 0;
    own = Seq{0, 0, 0, 0};
    for (int32_t i = 0; i < seg; ++i) {
      const int32_t s = lane * seg + i;
      if (s > a.n_seq) break;
      own = seq_of<true>(a, s);
      const Tiles t = tiles_of(a, s, own);
      mine += t.all();
      tiles += t.count;
      tokens += own.n;
    }
    incl = lane_prefix(mine);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      tiles += __shfl_xor(tiles, d, 64);
      tokens += __shfl_xor(tokens, d, 64);
    }
    all = uniform64(__shfl(incl, 63, 64)) * a.kv_heads;
    const int64_t most = (int64_t)a.tile_groups;
    workers = uniform((int32_t)min(most, max(tiles * a.kv_heads, all / kShareKeys)));
    if (tokens > a.tokens) workers = 0;  // starts that do not ascend: rows would be worked on often
  }

  __device__ __forceinline__ Seq seq(const AttnArgs& a, int32_t s) const {
    Seq q;
    if (seg == 1) {
      q = {__builtin_amdgcn_readlane(own.start, s), __builtin_amdgcn_readlane(own.n, s),
           __builtin_amdgcn_readlane(own.keys, s), __builtin_amdgcn_readlane(own.shift, s)};
    } else {
      q = seq_of<true>(a, s);
      q = {uniform(q.start), uniform(q.n), uniform(q.keys), uniform(q.shift)};
    }
    return q;
  }

  // The shares before worker w's, in mean ones.  A compute unit issues its oldest waves first: of the
  // workgroups on it the first placed gets a larger share, where all have one.
  __device__ __forceinline__ double ahead(const AttnArgs& a, int32_t w) const {
    const int32_t each = (int32_t)a.tile_groups / 8, on = (int32_t)a.tile_groups / (8 * kUnits);
    if (workers != (int32_t)a.tile_groups || on < 2) return w;
    const int32_t p = w % each, k = p / kUnits, r = p % kUnits;  // k have been placed on its unit before
    const double step = 2 * kOlder / (on - 1);
    return w - p + kUnits * (k * (1 + kOlder) - step * (k * (k - 1) / 2)) + r * (1 + kOlder - step * k);
  }

  // Where worker w's share begins (the others' and w = workers: nowhere).
  __device__ __forceinline__ TileCut cut(const AttnArgs& a, int32_t w) const {
    const TileCut none = {-1, a.n_seq + 1, 0, 0, 0, 0, 0, 0, 0};
    if (w >= workers) return none;
    // (Formed by the worker that begins here and by the one that ends here, in the same way.)
    const int64_t x = (int64_t)((double)all * (ahead(a, w) / (double)workers));
    // Its segment, then its sequence: a sequence's tiles of all heads follow each other.
    const int L = __popcll(__ballot((incl - mine) * a.kv_heads <= x)) - 1;
    int64_t before = uniform64(__shfl(incl - mine, L, 64));
    int32_t s = uniform(L * seg);
    const int32_t past = min(s + seg, a.n_seq + 1);
    while (seg > 1) {  // 64 sequences a step
      const int32_t i = s + (int32_t)(threadIdx.x & 63);
      const int64_t c = i < past ? tiles_of(a, i, seq_of<true>(a, i)).all() : 0;
      const int64_t in = lane_prefix(c);
      const int64_t sum = uniform64(__shfl(in, 63, 64));
      if (x < (before + sum) * a.kv_heads || s + 64 >= past) {
        const int k = __popcll(__ballot((before + in - c) * a.kv_heads <= x)) - 1;
        before += uniform64(__shfl(in - c, k, 64));
        s += k;
        break;
      }
      before += sum;
      s += 64;
    }
    if (s >= past) return none;
    const Seq q = seq(a, s);
    const Tiles t = tiles_of(a, s, q);
    const int64_t sum = uniform64(t.all());
    if (sum == 0) return none;
    const int64_t off = x - before * a.kv_heads;
    const int32_t head = uniform(min(ratio(off, sum), a.kv_heads - 1));
    const int64_t y = off - head * sum;
    const int32_t i = uniform(t.at(y));
    const int64_t first = uniform64(t.before(i)), weight = uniform64(t.base + t.step * (i + 1));
    const Tile tile = tile_at(a, s, q, i);
    int32_t stage = (int32_t)((double)tile.stages * (double)(y - first) / (double)weight);
    stage = min(max(stage, 0), tile.stages);
    if (stage < kLeastPiece)
      stage = 0;
    else if (tile.stages - stage < kLeastPiece)
      stage = tile.stages;
    return {before * a.kv_heads + head * sum + first, s, i, head, uniform(stage), tile.stages, q.start,
            q.n, 0};
  }
};

// A wave's share of a stage of keys or values, on its way from memory to LDS: eight rows of eight
// lanes, DP / 8 elements a lane.
template <int DP>
struct Codes {
  typedef uint32_t W __attribute__((ext_vector_type(DP / 64)));
  W words;
  uint32_t scale[DP > 128 ? 2 : 1];
};

constexpr int kRing4 = 2;  // stages of K, and of V, in LDS

// A wave's rows of a page that does not exist.
static __device__ const uint4 kZeroRows[64] = {};

// Pieces of V rows: as swizzle_v for the transposing read; that neighbouring rows differ in the lowest
// bit too puts a wave's writes, every other piece of two rows at a time, on different banks.
template <int DP>
__device__ __forceinline__ int swizzle_v4(int row) {
  return DP == 64 ? 0 : (row & 3) << 1 | (row & 1);
}

// A workgroup's work on `count` stages, at least one, of a tile from jb on: the tile's output, or
// partial results into the rows from part_row on where that is not below 0.  W: the elements of a row
// that the products take, of the DP that its stages have room for.  FULL: the rows have DP elements.
// EVEN: pages hold whole groups of eight rows.
template <typename ET, int DP, int W, bool FULL, bool EVEN>
__device__ __forceinline__ void tile4_work(const AttnArgs& a, const Tile& given, uint32_t head,
                                           int32_t jb, int32_t count, const int64_t part_row,
                                           uint16_t* const lds) {
  using V8 = typename Frag<ET>::V;
  constexpr int kStage = kKeys * DP;         // elements of a stage
  constexpr int kRowsWave = kKeys / kWaves;  // rows of a stage that a wave loads
  constexpr int DB = W / 32, KC = W / 16;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // what follows from it is formed for each tile, and not kept
  const int lane = tid & 63, col = lane & 31, h = lane >> 5;
  const int wave = uniform(tid >> 6);

  // (All of the workgroup's: kept in scalar registers.)
  Tile t = given;
  t.start = uniform(t.start);
  t.n = uniform(t.n);
  t.keys = uniform(t.keys);
  t.shift = uniform(t.shift);
  t.seq = uniform(t.seq);
  t.row0 = uniform(t.row0);
  t.rows = uniform(t.rows);
  t.seen = uniform(t.seen);
  head = (uint32_t)uniform((int32_t)head);
  jb = uniform(jb);
  count = uniform(count);

  // This lane's query row, and the last key that it sees.
  const int32_t m = min(t.row0 + 32 * wave + col, t.rows - 1);
  const int32_t tok = (int32_t)div_by((uint32_t)m, a.group);
  const int32_t qh = (int32_t)head * (int32_t)a.group.d + m - tok * (int32_t)a.group.d;
  const int32_t limit = min(t.shift + tok, t.keys - 1);
  // Stages (of this piece's) whose keys every row of the tile sees.
  const int32_t tok0 = (int32_t)div_by((uint32_t)t.row0, a.group);
  const int32_t least = min(t.shift + tok0, t.keys - 1);
  const int32_t open = min(max((least + 1) / kKeys - jb, 0), count);
  V8 q[KC];
  load_query<ET, W>(q, (const ET*)a.q + (int64_t)(t.start + tok) * a.q_row + (int64_t)qh * a.q_head,
                     a.dim, h);

  // Staging: a stage's codes into registers, and those as 16-bit elements into buffer `ring`.  Stages
  // past the last stand for it: there is no branch around the loads, which are waited for by their
  // number.  EVEN: a wave's eight rows lie together, and the scales of their elements in whole words (a
  // byte loaded for the next turn would be extended, and so waited for, at the end of this one).
  Stager<ET, DP, true> st(a, head, lane);
  st.seq = t.seq;
  st.start = t.start;
  st.seen = t.seen;
  const int32_t first = uniform(jb * kKeys + wave * kRowsWave);
  // SPREAD: word x of a lane is piece lane % 8 + 8 x of its row, so that the eight lanes of a row write to
  // different banks; the row's scales are whole words.  Else a lane's words are all of one block.  (4
  // chunks of 300 to 600, rows of 256: 219 us, 237 without; of 128: the same time, half the conflicts.)
  constexpr bool SPREAD = EVEN && FULL && DP >= 128;
  const int row4 = wave * kRowsWave + lane / 8, e4 = (SPREAD ? 8 : DP / 8) * (lane % 8);
  const uint32_t row_bytes = FULL ? DP / 2 : (uint32_t)a.dim / 2;
  const uint32_t row_scales = FULL ? DP / 32 : (uint32_t)a.dim / 32;
  const uint32_t in4 = FULL || e4 < a.dim ? e4 : 0;
  const uint32_t code_at = lane / 8 * row_bytes + in4 / 2, scale_at = lane / 8 * row_scales + in4 / 32;
  const uint32_t scale_turn = 9 + 8 * (scale_at & 3);  // of a word's bytes, to a float's exponent
  // EVEN: the wave's first row of the stage, else this lane's row.
  auto find = [&](int32_t i) __attribute__((always_inline)) {
    i = min(i, count - 1);
    if constexpr (EVEN)
      return (uint32_t)uniform((int32_t)st.row_of(first + i * kKeys));
    else
      return (uint32_t)__shfl((int)st.place((jb + i) * kKeys, kKeys), row4, 64);
  };
  auto fetch = [&](auto ISK, uint32_t row, Codes<DP>& to) __attribute__((always_inline)) {
    constexpr bool isk = decltype(ISK)::value;
    const uint8_t* c = (const uint8_t*)(isk ? a.k : a.v);
    const uint8_t* b = isk ? a.k_scales : a.v_scales;
    if constexpr (EVEN) {
      const uint64_t r = row;
      const uint8_t* const zeros = (const uint8_t*)kZeroRows;
      c = row == ~0u ? zeros : c + r * row_bytes;
      b = row == ~0u ? zeros : b + r * row_scales;
      if constexpr (SPREAD) {
#pragma unroll
        for (int x = 0; x < DP / 64; ++x) to.words[x] = load_global<uint32_t>(c + code_at + 32 * x);
#pragma unroll
        for (int x = 0; x < DP / 128; ++x)
          to.scale[x] = load_global<uint32_t>(b + (scale_at & ~3u) + 4 * x);
      } else {
        to.words = load_global<typename Codes<DP>::W>(c + code_at);
        to.scale[0] = load_global<uint32_t>(b + (scale_at & ~3u));
      }
    } else {
      const bool ok = row != ~0u;
      const uint8_t* const zeros = (const uint8_t*)&kZeros;
      to.words = load_global<typename Codes<DP>::W>(ok ? c + (uint64_t)row * row_bytes + in4 / 2 : zeros);
      to.scale[0] = load_global<uint8_t>(ok ? b + (uint64_t)row * row_scales + in4 / 32 : zeros);
    }
  };
  // Word x of stage i's codes.  A row that does not exist may hold values that are not finite, which
  // may not meet a weight, not even one of 0: it gets the least scale.
  auto put = [&](auto ISK, int x, int32_t i, int ring, const Codes<DP>& from)
      __attribute__((always_inline)) {
    constexpr bool isk = decltype(ISK)::value;
    if (!FULL && e4 >= a.dim) return;
    uint16_t* const to = lds + kStage * (ring + (isk ? 0 : kRing4)) + row4 * DP;
    const int swizzle = isk ? swizzle_k<DP>(row4) : swizzle_v4<DP>(row4);
    const uint32_t all = from.scale[SPREAD ? x / 2 : 0];
    uint32_t s = EVEN ? __builtin_amdgcn_alignbit(all, all, scale_turn + (SPREAD ? x % 2 * 16 : 0))
                      : all << 23;
    if (EVEN && !isk) s = (jb + i) * kKeys + row4 < t.seen ? s : 0;
    *(u32x4*)(to + 8 * ((e4 / 8 + (SPREAD ? 8 * x : x)) ^ swizzle)) =
        eight_values<ET>(from.words[x], __uint_as_float(s));
  };
  constexpr std::true_type kIsK{};
  constexpr std::false_type kIsV{};

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
  float mref = kNoMax, few = 0.0f;  // few: weights of up to two stages, on their way to acc
  Sum acc;
  float limit_raw = -INFINITY;  // a score above it makes m follow
  // P of the stage before the first is zero, and so must its values be.
  for (int i = (FULL ? 2 * kRing4 - 1 : 0) * kStage / 8 + tid; i < 2 * kRing4 * kStage / 8;
       i += 64 * kWaves)
    ((uint4*)lds)[i] = uint4{0, 0, 0, 0};
  if constexpr (!FULL) mt::stage_barrier();

  // LDS addresses of this lane's fragments in buffer 0; the rest is a constant offset.
  typedef __attribute__((address_space(3))) const char* ldsp;
  const ldsp lbase = (ldsp)(__attribute__((address_space(3))) uint16_t*)lds;
  constexpr int KA = KC < 8 ? KC : 8;  // the pieces repeat from the sixteenth on
  ldsp ka[KA], va[2];
#pragma unroll
  for (int c = 0; c < KA; ++c)
    ka[c] = lbase + 2 * (col * DP + 8 * ((2 * c + h) ^ swizzle_k<DP>(col)));
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    const int row = 4 * h + (lane & 15) / 4;
    const int piece = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    va[d] = lbase + 2 * (kRing4 * kStage + row * DP + 8 * (piece ^ swizzle_v4<DP>(row)) + 4 * (lane & 1));
  }
  // at: byte offset of the 32 (K) or 16 (V) rows in the ring.
  auto kfrag = [&](int at, int c) {
    return *(const __attribute__((address_space(3))) V8*)(ka[c % 8] + at + c / 8 * 256);
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
  // LDS reads of the MFMA kAhead slots on, a share of the exponentials, and of the staging.
  constexpr int kSlots = KC + 2 * DB, kAhead = DP > 128 ? 2 : 3, kCheck = 2;
  auto step = [&](int32_t j0, int kat, int vat, f32x16& s, f32x16& n, const u32x4 (&p0)[2],
                  u32x4 (&pn)[2], auto&& staging) __attribute__((always_inline)) {
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
        staging(I);
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
    uint16_t* const vs = lds + (kRing4 + i % kRing4) * kStage;
    if (!holds_nonfinite<ET, DP>(vs, lane)) return;
    cleared = true;
    mt::stage_barrier();
#pragma unroll 1
    for (int r = 0; r < 32 * DP; r += 512) clear_nonfinite<ET, 16>(vs + r, wave * 64, kWaves * 64, lane);
    mt::stage_barrier();
  };
  f32x16 sa, sb;
  u32x4 pa[2], pb[2];
  pb[0] = pb[1] = u32x4{0, 0, 0, 0};
  Codes<DP> kcodes, vcodes;  // of K j + 2 and V j, from the turn before
  uint32_t r1 = find(1), r2 = find(2);  // rows of stages j + 1 and j + 2
  {
    const uint32_t r0 = find(0);
    Codes<DP> k0, k1;
    fetch(kIsK, r0, k0);
    fetch(kIsK, r1, k1);
    fetch(kIsK, r2, kcodes);
    fetch(kIsV, r0, vcodes);
#pragma unroll
    for (int x = 0; x < DP / 64; ++x) {
      put(kIsK, x, 0, 0, k0);
      put(kIsK, x, 1, 1, k1);
    }
    mt::stage_barrier();
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) sa[r] = 0.0f;
#pragma unroll
  for (int c = 0; c < KC; ++c) sa = mfma<ET>(kfrag(0, c), q[c], sa);
  auto turn = [&](int32_t j, int r, f32x16& s, f32x16& n, const u32x4 (&p)[2],
                  u32x4 (&pn)[2]) __attribute__((always_inline)) {  // r: j % 2
    mt::stage_barrier();
    if (j > open) clear(j - 1);
    // K j + 2 and V j go to LDS word by word; the loads of those after them begin as soon as their
    // registers are free.
    constexpr int kWords = DP / 64, kFirst = kCheck + 1, kLast = kSlots - 2;
    const uint32_t next = find(j + 3);  // (here, for it branches)
    step((jb + j) * kKeys, (1 - r) * kS, (1 - r) * kS, s, n, p, pn,
         [&](auto I) __attribute__((always_inline)) {
           constexpr int i = decltype(I)::value;
           mt::static_for<0, 2 * kWords>([&](auto X) __attribute__((always_inline)) {
             constexpr int x = decltype(X)::value;
             if constexpr (i == kFirst + (DP > 128 ? 0 : x * (kLast - kFirst) / (2 * kWords))) {
               if constexpr (x < kWords)
                 put(kIsK, x, j + 2, r, kcodes);
               else
                 put(kIsV, x - kWords, j, r, vcodes);
               if constexpr (x == kWords - 1) fetch(kIsK, next, kcodes);
               if constexpr (x == 2 * kWords - 1) fetch(kIsV, r1, vcodes);
             }
           });
         });
    r1 = r2;
    r2 = next;
  };
  // Scores and weights change places every turn: a pass of the loop takes an even number.
  for (int32_t j = 0; j < count; j += 2) {
    turn(j, 0, sa, sb, pb, pa);
    if (j + 1 >= count) break;
    turn(j + 1, 1, sb, sa, pa, pb);
    acc.add(few);
    few = 0.0f;
  }
  acc.add(few);
  {
    mt::stage_barrier();  // the last values are there
    if (count > open) clear(count - 1);
    const int at = (count - 1) % kRing4 * kS;
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
  if (part_row >= 0) {
    const int64_t row = part_row + 32 * wave + col;
    if (mine) store_part<W>(o, a.tile_o + row * DP, h);
    if (mine && h == 0) a.tile_stat[row] = {mref, sum};
    if (restore)
      restore_nonfinite<ET, DP, true, true>(st, a.tile_o + (row - col) * DP, DP, t,
                                            t.row0 + 32 * wave, jb * kKeys, (jb + count) * kKeys,
                                            sum);
    return;
  }
  const int64_t orow = (int64_t)(t.start + tok) * a.heads + qh;
  if (mine && a.lse && h == 0) a.lse[orow] = log_sum(mref, sum);
  mt::stage_barrier();  // the other waves' reads of the stages are done
  store_rows<ET, DP, W>(o, inverse(sum), (ET*)a.out, mine ? orow * a.dim : -1, a.dim,
                         lds + wave * 32 * DP, lane);
  if (restore)
    restore_nonfinite<ET, DP, true, true>(st, (ET*)a.out, 0, t, t.row0 + 32 * wave, jb * kKeys,
                                          (jb + count) * kKeys, sum);
}

// Where a worker is in its share: the tile and its first stage, and the share's end.
struct TilePlace {
  Seq q;
  int32_t seq, tile, head, stage, end_seq, end_tile, end_head, end_stage;
  int32_t first;  // 1: the share's first tile
};

// The next sequence after s that has tiles, 64 of them a step.
__device__ __forceinline__ int32_t next_of(const AttnArgs& a, int32_t s) {
  for (++s; s <= a.n_seq; s += 64) {
    const int32_t i = s + (int32_t)(threadIdx.x & 63);
    const uint64_t has = __ballot(i <= a.n_seq && tiles_of(a, i, seq_of<true>(a, i)).count > 0);
    if (has) return s + __builtin_ctzll(has);
  }
  return s;
}

// A piece without stages, where others of its tile follow: rows of weight 0.
template <int DP>
__device__ __forceinline__ void clear_piece(const AttnArgs& a, int64_t row) {
  for (int i = threadIdx.x; i < kRows * DP; i += 64 * kWaves) a.tile_o[row * DP + i] = 0.0f;
  for (int i = threadIdx.x; i < kRows; i += 64 * kWaves) a.tile_stat[row + i] = {kNoMax, 0.0f};
}

// Rows of a tile that sees no key: zeros, and -inf.
template <typename ET>
__device__ __forceinline__ void clear_rows(const AttnArgs& a, const Tile& t, int32_t head) {
  const int32_t words = a.dim / 8;
  for (int32_t m = t.row0 + (int32_t)(threadIdx.x >> 6); m < min(t.row0 + kRows, t.rows); m += kWaves) {
    const int32_t tok = (int32_t)div_by((uint32_t)m, a.group);
    const int32_t qh = head * (int32_t)a.group.d + m - tok * (int32_t)a.group.d;
    const int64_t orow = (int64_t)(t.start + tok) * a.heads + qh;
    for (int32_t i = threadIdx.x & 63; i < words; i += 64)
      ((uint4*)((ET*)a.out + orow * a.dim))[i] = uint4{0, 0, 0, 0};
    if (a.lse && (threadIdx.x & 63) == 0) a.lse[orow] = -INFINITY;
  }
}

// A worker's share of the tiles.
template <typename ET, int DP, int W, bool FULL, bool EVEN>
__device__ __forceinline__ void tile4_share(const AttnArgs& a, uint16_t* const lds) {
  // Neighbours in the line, which read the same keys, run on the same XCD (its workgroups are those
  // of every eighth number); the workers are the first of every XCD's.
  const TileLine line(a);
  const int32_t xcd = blockIdx.x % 8, p = blockIdx.x / 8, each = (line.workers + 7) / 8;
  const int32_t w = p < each ? xcd * each + p
                             : 8 * each + xcd * ((int32_t)a.tile_groups / 8 - each) + p - each;
  const TileCut from = line.cut(a, w), end = line.cut(a, w + 1);
  if (threadIdx.x == 0) a.tile_cut[w] = from;
  if (from.x < 0) return;
  // Where the worker is in its share lies in LDS meanwhile: a tile's work needs all registers.
  typedef __attribute__((address_space(3))) TilePlace* place;
  const place at = (place)(__attribute__((address_space(3))) uint16_t*)(lds + 2 * kRing4 * kKeys * DP);
  TilePlace now = {line.seq(a, from.seq), from.seq, from.tile, from.head, from.stage,
                   end.seq, end.tile, end.head, end.stage, 1};
  for (;;) {
    const Tile t = tile_at(a, now.seq, now.q, now.tile);
    const bool last = now.seq == now.end_seq && now.head == now.end_head && now.tile == now.end_tile;
    const int32_t j0 = now.stage, j1 = last ? now.end_stage : t.stages;
    const bool whole = j0 == 0 && j1 == t.stages;
    const int64_t row = (2 * (int64_t)w + !now.first) * kRows;
    if (t.stages == 0) {
      if (!last) clear_rows<ET>(a, t, now.head);
    } else if (j0 < j1) {
      if (threadIdx.x == 0) *(TilePlace*)at = now;
      tile4_work<ET, DP, W, FULL, EVEN>(own_args(), t, (uint32_t)now.head, j0, j1 - j0,
                                        whole ? -1 : row, lds);
      mt::stage_barrier();  // the stages are free for the next tile's
      now = *(const TilePlace*)at;
      mt::stage_barrier();  // read before it is written again
    } else if (last && j0 > 0 && j0 < t.stages) {
      clear_piece<DP>(a, row);
    }
    if (last) return;
    // The next tile: of this head, of the next, of the next sequence that has any.
    now.first = 0;
    now.stage = 0;
    if (++now.tile * kRows >= now.q.n * (int32_t)a.group.d) {
      now.tile = 0;
      if (++now.head == a.kv_heads) {
        now.head = 0;
        now.seq = next_of(a, now.seq);
        if (now.seq > a.n_seq) return;
        now.q = seq_of<true>(a, now.seq);
      }
    }
  }
}

// The waves are the token workers too, where a call has both.  Of the workgroups that share a compute
// unit some begin with the tokens and some with the tiles, so that the memory is read while products
// are formed.
template <typename ET, int DP, int W, bool FULL, bool EVEN>
__global__ void __launch_bounds__(64 * kWaves, DP > 128 ? 1 : DP > 64 ? 2 : 3)
    tile4_kernel(AttnArgs a) {
  extern __shared__ __align__(16) uint16_t lds[];  // stages of K, as many of V, the place
  const bool late = blockIdx.x >= a.tile_groups / 2;
  for (int turn = 0; turn < 2; ++turn) {
    if (turn) mt::stage_barrier();  // the LDS is free
    if (late == (turn == 0)) {
      if (a.ride) {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));  // what follows from it is formed here, and not kept
        const int wave = uniform(tid >> 6);
        token4_work<ET, DP, 1, EVEN>(own_args(), blockIdx.x * kWaves + wave, a.tile_groups * kWaves,
                                     lds + wave * (32 * DP), tid & 63);
      }
    } else {
      tile4_share<ET, DP, W, FULL, EVEN>(own_args(), lds);
    }
  }
}

// One wave joins R rows of a tile's pieces side by side, from row r0 of the tile on: lanes 64 / R r
// and on hold row r's statistics, as many pieces a turn.  Rows from `rows` on are another's.  Row r0 of
// piece k is row_of(k).
template <typename ET, int DP, int R, typename F>
__device__ __forceinline__ void join_rows(const AttnArgs& a, const Tile& t, int32_t head, int32_t r0,
                                          int32_t pieces, int32_t rows, F&& row_of) {
  constexpr int C = DP / 64, L = 64 / R;
  const int lane = threadIdx.x & 63;
  float m = kNoMax, sum = 0.0f, acc[R][C];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < C; ++e) acc[r][e] = 0.0f;
  constexpr int kAhead = R == 1 ? 8 : 4;  // pieces in flight
  float v[kAhead][R][C];
  auto load = [&](int32_t k, int32_t end) __attribute__((always_inline)) {  // (the last again past it)
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float* const o = a.tile_o + row_of(min(k + i, end - 1)) * DP + C * lane;
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < C; ++e) v[i][r][e] = o[r * DP + e];
    }
  };
  for (int32_t k0 = 0; k0 < pieces; k0 += L) {
    const int32_t n = min(pieces - k0, L);
    float2 st = {kNoMax, 0.0f};
    if (lane % L < n) st = a.tile_stat[row_of(k0 + lane % L) + lane / L];
    load(k0, k0 + n);
    float top = fmaxf(m, st.x);
#pragma unroll
    for (int d = 1; d < L; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float keep = __builtin_amdgcn_exp2f(m - top), f = __builtin_amdgcn_exp2f(st.x - top);
    m = top;
    float part = st.y * f;
#pragma unroll
    for (int d = 1; d < L; d <<= 1) part += __shfl_xor(part, d, 64);
    sum = sum * keep + part;
    auto of_row = [&](float x, int r, int32_t k) {
      return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), L * r + k));
    };
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < C; ++e) acc[r][e] = weighted(acc[r][e], of_row(keep, r, 0));
    for (int32_t k = 0; k < n; k += kAhead) {
      if (k > 0) load(k0 + k, k0 + n);
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < C; ++e)
            acc[r][e] += k + i < n ? weighted(v[i][r][e], of_row(f, r, min(k + i, L - 1))) : 0.0f;
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int32_t row = t.row0 + r0 + r;
    if (row >= rows) break;
    const int32_t tok = (int32_t)div_by((uint32_t)row, a.group);
    const int32_t qh = head * (int32_t)a.group.d + row - tok * (int32_t)a.group.d;
    const int64_t orow = (int64_t)(t.start + tok) * a.heads + qh;
    Joined<DP> j;
    j.m = __shfl(m, L * r, 64);
    j.sum = __shfl(sum, L * r, 64);
#pragma unroll
    for (int e = 0; e < C; ++e) j.acc[e] = acc[r][e];
    store_joined<ET, DP>(j, (ET*)a.out + orow * a.dim, a.lse ? a.lse + orow : nullptr, a.dim);
  }
}

// Joins the pieces of the cut tiles.  A tile of n pieces is cut by n - 1 workers' beginnings; each of
// them stands for kJoinGroups workgroups, which share the tile's rows with the other beginnings'.
// (Bound by the chain of loads: 16 to 19 us for 512 workers in 1,022 workgroups, which are all there at
// once, 20 to 25 with four for every beginning.)
constexpr int kJoinGroups = 2, kJoinThreads = 64 * kJoinWaves, kJoinEach = 4;
template <typename ET, int DP>
__device__ __forceinline__ void tile4_join(const AttnArgs& a) {
  const int32_t w = (int32_t)(blockIdx.x / kJoinGroups) + 1, last = (int32_t)a.tile_groups - 1;
  const int lane = threadIdx.x & 63;
  const TileCut c = a.tile_cut[w];
  // The beginnings inside the tile: before this one, and with it and after, from the 64 around it.
  auto around = [&](int32_t from) {
    const int32_t k = from + lane;
    const TileCut n = a.tile_cut[min(max(k, 0), last)];
    return __ballot(k > 0 && k <= last && n.x == c.x && n.stage > 0 && n.stage < n.stages);
  };
  const uint64_t near = around(w - 32);
  if (c.x < 0 || c.stage == 0 || c.stage == c.stages) return;
  int32_t before = (uint32_t)near == ~0u ? 32 : __builtin_clz(~(uint32_t)near);
  if (before == 32)
    for (int32_t at = w - 32;; at -= 64) {
      const uint64_t in = around(at - 64);
      const int32_t run = in == ~0ull ? 64 : __builtin_clzll(~in);
      before += run;
      if (run < 64) break;
    }
  int32_t after = (uint32_t)(near >> 32) == ~0u ? 32 : __builtin_ctz(~(uint32_t)(near >> 32));
  if (after == 32)
    for (int32_t at = w + 32;; at += 64) {
      const uint64_t in = around(at);
      const int32_t run = in == ~0ull ? 64 : __builtin_ctzll(~in);
      after += run;
      if (run < 64) break;
    }
  const int32_t cuts = before + after, w0 = w - before;
  const Tile t = tile_at(a, c.seq, Seq{c.start, c.n, 0, 0}, c.tile);
  // The first piece is the last of worker w0 - 1's, or its only one.
  const int64_t begin = (2 * (int64_t)(w0 - 1) + (a.tile_cut[w0 - 1].x == c.x ? 0 : 1)) * kRows;
  const int64_t others = 2 * (int64_t)w0 * kRows;
  const int32_t wave = (int32_t)(blockIdx.x % kJoinGroups) * (kJoinThreads / 64) +
                       uniform(threadIdx.x >> 6);
  constexpr int32_t kAll = kJoinGroups * kJoinThreads / 64;
  const int32_t rows = min(t.rows - t.row0, kRows);
  const int32_t lo = rows * before / cuts, hi = rows * (before + 1) / cuts;
  // (A piece's rows are all there, also those that the tile does not have.)
  auto join = [&](auto EACH) {
    constexpr int R = decltype(EACH)::value;
    for (int32_t r = lo + wave * R; r < hi; r += kAll * R) {
      const int32_t r0 = min(r, kRows - R);
      join_rows<ET, DP, R>(a, t, c.head, r0, cuts + 1, t.row0 + hi, [&](int32_t k) {
        return r0 + (k == 0 ? begin : others + (int64_t)(k - 1) * 2 * kRows);
      });
    }
  };
  if (hi - lo <= kAll)
    join(std::integral_constant<int, 1>{});
  else
    join(std::integral_constant<int, kJoinEach>{});
}

// The joins of the tiles and, behind them, of the tokens that the same kernel worked on.
template <typename ET, int DP, bool ALL>
__global__ void __launch_bounds__(kJoinThreads) tile4_join_kernel(AttnArgs a) {
  const uint32_t tiles = (a.tile_groups - 1) * kJoinGroups;
  if (blockIdx.x < tiles) {
    tile4_join<ET, DP>(a);
  } else if constexpr (ALL) {
    __shared__ Joined<DP> left[kJoinWaves][64];
    token_join<ET, DP, true>(a, blockIdx.x - tiles, a.tile_groups * kWaves, left);
  } else {
    token_join<ET, DP, false>(a, blockIdx.x - tiles, a.tile_groups * kWaves, nullptr);
  }
}

template <typename ET, int DP, int W, bool FULL>
hipError_t launch_tile4(const AttnArgs& a, hipStream_t s) {
  constexpr unsigned bytes = 2 * kRing4 * kKeys * DP * 2 + 64;  // K and V, 16 bits; the place
  // Blocks of 16 rows, for the tokens; the tiles need eight.
  const auto kern = a.page.d % 16 == 0 ? tile4_kernel<ET, DP, W, FULL, true>
                                       : tile4_kernel<ET, DP, W, FULL, false>;
  if constexpr (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(
        (const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3(a.tile_groups), dim3(64 * kWaves), bytes, s, a);
  const unsigned tiles = (a.tile_groups - 1) * kJoinGroups;
  const int64_t pairs = a.ride ? (int64_t)a.n_seq * a.kv_heads : 0;
  // (As launch_token_join has it.)
  if (16 * pairs <= (int64_t)a.tile_groups * kWaves)
    hipLaunchKernelGGL((tile4_join_kernel<ET, DP, true>),
                       dim3(tiles + (unsigned)pairs * (unsigned)a.skip_rows), dim3(kJoinThreads), 0,
                       s, a);
  else
    hipLaunchKernelGGL((tile4_join_kernel<ET, DP, false>), dim3(tiles + (unsigned)pairs),
                       dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}

// (Rows of 160 to 224 take the products and stages of 256, and their scales and codes a block a lane: a
// chunk of 512 after 20,000, 16 / 2 heads, rows of 128 120 us, of 192 250, of 256 233.)
template <typename ET>
hipError_t launch_tile4(const AttnArgs& a, hipStream_t s) {
  if (a.dim < 64) return launch_tile4<ET, 64, 64, false>(a, s);
  if (a.dim == 64) return launch_tile4<ET, 64, 64, true>(a, s);
  if (a.dim <= 96) return launch_tile4<ET, 128, 96, false>(a, s);
  if (a.dim == 128) return launch_tile4<ET, 128, 128, true>(a, s);
  if (a.dim < 256) return launch_tile4<ET, 256, 256, false>(a, s);
  return launch_tile4<ET, 256, 256, true>(a, s);
}

}  // namespace attn
}  // namespace tod
