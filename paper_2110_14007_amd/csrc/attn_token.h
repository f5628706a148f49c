// Attention of few new tokens a sequence over a paged cache (the single-token
// form): bound by the bytes of the keys and values, each read once.
//
// The keys of all (sequence, key / value head) pairs, in stages of 32, form
// one line that is dealt to the workers, a wave each, in equal shares, so that
// neither one long sequence nor many of different lengths leave a part of the
// GPU idle.  A wave works alone: it stages its keys and values in its own ring
// of LDS buffers (the next stages are in flight while it computes), keeps up
// to 32 packed rows and waits for nobody.  A pair that one wave reads whole is
// finished by it; of the others each wave leaves (m, sum, O) and a second
// kernel joins them.
//
// MFMAs and exponentials run far below the matrix rate (a stage of 16 KiB
// takes one of 1024 waves about 2.8 us at the memory's rate, its arithmetic
// 0.6), so p goes through the second product as two halves, the rounded p and
// what the rounding lost: the weights then keep 16 bits, in fp16 down to 2^-19
// of the largest (each is off by 2^-35 of it at most).
//
// Measured, with 8 heads of 128: 243 us for 3 caches of 120,000 to 131,071
// tokens (6.3 TB/s, the rate of a plain read), 224 us for 96 of 100 to 6,000
// (5.4 TB/s), 7.3 us for one of 900, where a worker has one stage and its start
// counts; the join takes 5 to 8 us more.
#pragma once

#include "attn.h"

namespace tod {
namespace attn {

constexpr int kTokenKeys = 32;  // keys of a stage

// Buffers of a wave's ring, and loads of a stage.
template <int DP>
constexpr int token_ring() { return DP == 64 ? 4 : 2; }
template <int DP>
constexpr int token_loads() { return 2 * kTokenKeys * DP * 2 / 1024; }

// Bytes of the ring.
template <int DP>
constexpr int token_lds() { return token_ring<DP>() * 2 * kTokenKeys * DP * 2; }

// Stages of KEYS keys of a sequence that is the token kernel's, else 0.
template <int KEYS>
__device__ __forceinline__ int32_t token_stages(const AttnArgs& a, const Seq& q) {
  if (q.n <= 0 || (int64_t)q.n * a.group.d > a.skip_rows) return 0;
  return (q.keys + KEYS - 1) / KEYS;
}
template <int KEYS>
__device__ __forceinline__ int32_t token_stages(const AttnArgs& a, int32_t s) {
  return s < a.n_seq ? token_stages<KEYS>(a, seq_of<true>(a, s)) : 0;
}

// Of `all` stages worker w of `grid` has those from share(w) on (all w: below 2^63); where there are
// fewer stages than workers, one each.
__device__ __forceinline__ int64_t share(int64_t w, int64_t all, const uint32_t grid) {
  return all < grid ? w : (all * w) / grid;
}

// The worker that has stage x: from an estimate (below 2^53 exact to one) and its neighbours.
__device__ __forceinline__ int64_t worker_of(int64_t x, int64_t all, const uint32_t grid) {
  if (all < grid) return x;
  int64_t w = (int64_t)((double)x * grid / (double)all);
  while (w > 0 && share(w, all, grid) > x) --w;
  while (w + 1 < grid && share(w + 1, all, grid) <= x) ++w;
  return w;
}

// n / d for n >= 0, d > 0, in 32 bits where they fit.
__device__ __forceinline__ int64_t quotient(int64_t n, int64_t d) {
  return n <= 0xffffffffLL && d <= 0xffffffffLL ? (int64_t)((uint32_t)n / (uint32_t)d) : n / d;
}

// Inclusive prefix sum over the lanes.
__device__ __forceinline__ int64_t lane_prefix(int64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(v, d, 64);
    if (lane >= d) v += y;
  }
  return v;
}

template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// A worker's share of the line of stages, and where in it the share begins.
struct Share {
  int64_t at, end;  // its stages
  int32_t s;        // the sequence that holds stage `at`
  int64_t off;      // of `at` in the sequence's stages of all heads
  int32_t seg;      // sequences that a lane summed; of one, what it is:
  Seq own;
};

template <int KEYS>
__device__ __forceinline__ Share deal(const AttnArgs& a, const uint32_t worker,
                                      const uint32_t grid) {
  Share w;
  // The line of stages: lane l sums the sequences of its own segment (of one, where there are no
  // more than lanes: then it holds what that sequence is).
  const int lane = threadIdx.x & 63;
  const int32_t seg = w.seg = (a.n_seq + 63) / 64, s0 = lane * seg;
  w.own = s0 < a.n_seq ? seq_of<true>(a, s0) : Seq{0, 0, 0, 0};
  int64_t mine = token_stages<KEYS>(a, w.own);
  for (int32_t i = 1; i < seg; ++i) mine += token_stages<KEYS>(a, s0 + i);
  const int64_t incl = lane_prefix(mine);
  const int64_t all = __shfl(incl, 63, 64) * a.kv_heads;
  if (worker == 0) {  // for the join
    int64_t before = incl - mine;
    for (int32_t i = 0; i < seg && s0 + i < a.n_seq; ++i) {
      a.token_line[s0 + i] = before;
      before += i == 0 ? token_stages<KEYS>(a, w.own) : token_stages<KEYS>(a, s0 + i);
    }
    if (lane == 63) a.token_line[a.n_seq] = incl;
  }
  // This worker's share of it.
  w.at = share(worker, all, grid);
  w.end = share(worker + 1, all, grid);
  if (w.end > all) w.at = w.end = all;

  // The sequence that holds stage `at`: its segment, then 64 sequences a step.
  w.s = 0;
  w.off = 0;
  if (w.at < w.end) {
    const int64_t target = quotient(w.at, a.kv_heads);
    const int L = __popcll(__ballot(incl - mine <= target)) - 1;
    int64_t before = __shfl(incl - mine, L, 64);
    int32_t first = L * seg;
    int32_t s = first;
    while (seg > 1) {
      const int32_t c = first + lane < (L + 1) * seg ? token_stages<KEYS>(a, first + lane) : 0;
      const int64_t in = lane_prefix(c);
      const int64_t sum = __shfl(in, 63, 64);
      if (target < before + sum) {
        const int k = __popcll(__ballot(before + in - c <= target)) - 1;
        s = first + k;
        before += __shfl(in - c, k, 64);
        break;
      }
      before += sum;
      first += 64;
    }
    w.s = __builtin_amdgcn_readfirstlane(s);
    w.off = w.at - before * a.kv_heads;
  }
  return w;
}

// The sequence of number s: from the lane that summed it, or from memory.
__device__ __forceinline__ Seq dealt(const AttnArgs& a, const Share& w, int32_t s) {
  if (w.seg == 1)
    return {__builtin_amdgcn_readlane(w.own.start, s), __builtin_amdgcn_readlane(w.own.n, s),
            __builtin_amdgcn_readlane(w.own.keys, s), __builtin_amdgcn_readlane(w.own.shift, s)};
  return seq_of<true>(a, s);
}

// Rows past the last sequence, where no tile kernel takes them.
__device__ __forceinline__ void clear_tail(const AttnArgs& a, const uint32_t worker,
                                           const uint32_t grid) {
  if (!a.token_tail) return;
  const int lane = threadIdx.x & 63;
  const int32_t words = a.heads * a.dim / 8;
  for (int32_t t = start_of(a, a.n_seq) + (int32_t)worker; t < a.tokens; t += (int32_t)grid) {
    for (int32_t i = lane; i < words; i += 64)
      ((uint4*)a.out)[(int64_t)t * words + i] = uint4{0, 0, 0, 0};
    if (a.lse)
      for (int32_t i = lane; i < a.heads; i += 64) a.lse[(int64_t)t * a.heads + i] = -INFINITY;
  }
}

// A worker: a wave, with the LDS of its ring.
template <typename ET, int DP>
__device__ __forceinline__ void token_work(const AttnArgs& a, const uint32_t worker,
                                           uint16_t* const lds) {
  constexpr uint32_t grid = (uint32_t)token_workers(DP);
  using V8 = typename Frag<ET>::V;
  using St = Stager<ET, DP, true>;
  constexpr int kStage = kTokenKeys * DP;  // elements of a K or V stage
  constexpr int kRing = token_ring<DP>(), kLoads = token_loads<DP>(), DB = DP / 32;
  const int lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5;

  const Share mine = deal<kTokenKeys>(a, worker, grid);
  int64_t at = mine.at, off = mine.off;
  const int64_t end = mine.end;
  int32_t s = mine.s;

  const uint32_t base = mt::lds_off(lds);
  for (bool opening = true; at < end; opening = false) {
    const Seq sq = dealt(a, mine, s);
    const int32_t stages = token_stages<kTokenKeys>(a, sq);
    if (stages == 0) {  // another kernel's, or idle
      ++s;
      off = 0;
      continue;
    }
    const uint32_t head = (uint32_t)quotient(off, stages);
    const int32_t jb = (int32_t)(off - (int64_t)head * stages);
    const int32_t je = (int32_t)min((int64_t)stages, jb + (end - at));

    const int32_t rows = sq.n * (int32_t)a.group.d;
    const int32_t m = min(col, rows - 1);
    const int32_t tok = (int32_t)div_by((uint32_t)m, a.group);
    const int32_t qh = (int32_t)head * (int32_t)a.group.d + m - tok * (int32_t)a.group.d;
    const int32_t limit = min(sq.shift + tok, sq.keys - 1);
    const int32_t wlo = __builtin_amdgcn_readfirstlane(limit);

    St st(a, head);
    st.seq = s;
    st.start = sq.start;
    st.seen = sq.keys;
    auto stage = [&](int32_t j) {
      const uint32_t pl = st.place(j * kTokenKeys, kTokenKeys);
      const uint32_t k = base + 4u * kStage * (uint32_t)((j - jb) % kRing);
#pragma unroll
      for (int i = 0; i < kTokenKeys / St::kRowsLoad; ++i)
        st.load(pl, i * St::kRowsLoad, k, k + 2u * kStage);
    };
#pragma unroll
    for (int i = 0; i < kRing; ++i)
      if (jb + i < je) stage(jb + i);

    V8 q[DP / 16];
    load_query<ET, DP>(
        q, (const ET*)a.q + (int64_t)(sq.start + tok) * a.q_row + (int64_t)qh * a.q_head, a.dim, h);

    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
    float mref = kNoMax;
    Sum acc;
    bool cleared = false;  // values that are not finite were taken for 0

    for (int32_t j = jb; j < je; ++j) {
      if (j + kRing <= je)
        wait_loads<(kRing - 1) * kLoads>();
      else
        wait_loads<0>();
      const uint16_t* const ks = lds + 2 * kStage * ((j - jb) % kRing);
      const uint16_t* const vs = ks + kStage;
      const int32_t j0 = j * kTokenKeys;
      f32x16 x = scores<ET, DP>(ks, 0, q);
      if (j0 + kTokenKeys - 1 > wlo) {
        const int32_t left = limit - j0 - 4 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (mt::out_row_c(r) > left) x[r] = -INFINITY;
      }
      float top = x[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, x[r]);
      top = fmaxf(top, other_half(top)) * a.scale;
      const float next =
          fmaxf(mref, top - (fabsf(fmaxf(top, mref)) > kFar ? 0.0f : kBias<ET>));
      if (__ballot(next > mref)) {
        const float f = __builtin_amdgcn_exp2f(mref - next);
        mref = next;
        acc.scale(f);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= f;
      }
      float part = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.scale, -mref));
        part += x[r];
      }
      acc.add(part);
      // A value that is not finite must not meet the zero weight of a row that does not see it.
      if (j0 + kTokenKeys - 1 > wlo && rows > (int32_t)a.group.d && holds_nonfinite<ET, DP>(vs)) {
        clear_nonfinite<ET, DP>(lds + 2 * kStage * ((j - jb) % kRing) + kStage, 0, 64);
        cleared = true;
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        typedef ET e8 __attribute__((ext_vector_type(8)));
        e8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = x[8 * c + e];
          hi[e] = (ET)p;
          lo[e] = (ET)(p - (float)hi[e]);
        }
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const V8 v = values<ET, DP>(vs, 16 * c, d);
          o[d] = mfma<ET>(v, __builtin_bit_cast(V8, hi), o[d]);
          o[d] = mfma<ET>(v, __builtin_bit_cast(V8, lo), o[d]);
        }
      }
      if (j + kRing < je) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this buffer's reads are done
        stage(j + kRing);
      }
    }
    const float sum = acc.v + other_half(acc.v);
    const bool restore = cleared || met_nonfinite(o, sum);

    if (jb == 0 && je == stages) {
      const int64_t orow = (int64_t)(sq.start + tok) * a.heads + qh;
      if (a.lse && h == 0 && col < rows) a.lse[orow] = log_sum(mref, sum);
      store_rows<ET, DP, DP>(o, inverse(sum), (ET*)a.out, col < rows ? orow * a.dim : -1, a.dim, lds);
      if (restore) restore_nonfinite<ET, DP, true>(st, (ET*)a.out, 0, sq, 0, 0, sq.keys, sum);
    } else {
      // At most two of a worker's pieces are not whole: its first and its last.
      const int64_t row0 = (2 * (int64_t)worker + !opening) * a.skip_rows;
      if (col < rows) {
        store_part<DP>(o, a.token_o + (row0 + col) * DP, h);
        if (h == 0) a.token_stat[row0 + col] = {mref, sum};
      }
      if (restore)
        restore_nonfinite<ET, DP, true>(st, a.token_o + row0 * DP, DP, sq, 0, jb * kTokenKeys,
                                        je * kTokenKeys, sum);
    }
    // Its stores and LDS reads are done before the next pair's loads are counted.
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    at += je - jb;
    off += je - jb;
    if (off == (int64_t)stages * a.kv_heads) {
      ++s;
      off = 0;
    }
  }

  clear_tail(a, worker, grid);
}

template <typename ET, int DP>
__global__ void __launch_bounds__(64) token_kernel(AttnArgs a) {
  __shared__ __align__(16) uint16_t lds[token_lds<DP>() / 2];
  token_work<ET, DP>(a, blockIdx.x, lds);
}

// Joins the pieces of a (sequence, key / value head) pair.  ALL: a workgroup of kJoinWaves waves
// takes one of its packed rows, and each wave an equal part of the row's pieces.  Otherwise it
// takes all of the pair's rows, a wave a row at a time.
// left: LDS for a row of every wave (ALL).
constexpr int kJoinWaves = 8;
template <typename ET, int DP, bool ALL>
__device__ __forceinline__ void token_join(const AttnArgs& a, const uint32_t block,
                                           const uint32_t grid, Joined<DP> (*left)[64]) {
  const uint32_t row = ALL ? block % (uint32_t)a.skip_rows : 0;
  const uint32_t pair = ALL ? block / (uint32_t)a.skip_rows : block;
  const uint32_t s = div_by(pair, a.heads_div), head = pair - s * a.heads_div.d;
  const int64_t before = a.token_line[s], after = a.token_line[s + 1];
  const int64_t all = a.token_line[a.n_seq] * a.kv_heads, stages = after - before;
  const Seq sq = seq_of<true>(a, (int32_t)s);
  const int32_t rows = sq.n * (int32_t)a.group.d;
  if (stages == 0 || (int32_t)row >= rows) return;
  const int64_t lo = before * a.kv_heads + head * stages;
  const int64_t w0 = worker_of(lo, all, grid), w1 = worker_of(lo + stages - 1, all, grid);
  if (w0 == w1) return;
  // The first worker's piece is its last one if the pair begins within its share; the others
  // begin with theirs.
  const bool within = share(w0, all, grid) < lo;
  const int32_t pieces = (int32_t)(w1 - w0 + 1);
  auto join = [&](int32_t r, int32_t from, int32_t to) {
    return join_parts<DP>(a.token_stat, a.token_o, (2 * w0 + within) * a.skip_rows + r,
                          2 * (w0 + 1) * a.skip_rows + r, 2 * (int64_t)a.skip_rows, from, to);
  };
  auto store = [&](int32_t r, const Joined<DP>& j) {
    const int32_t tok = (int32_t)div_by((uint32_t)r, a.group);
    const int32_t qh = (int32_t)head * (int32_t)a.group.d + r - tok * (int32_t)a.group.d;
    const int64_t orow = (int64_t)(sq.start + tok) * a.heads + qh;
    store_joined<ET, DP>(j, (ET*)a.out + orow * a.dim, a.lse ? a.lse + orow : nullptr, a.dim);
  };
  const int wave = (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if constexpr (ALL) {
    Joined<DP> j = join((int32_t)row, pieces * wave / kJoinWaves, pieces * (wave + 1) / kJoinWaves);
    left[wave][lane] = j;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int i = 1; i < kJoinWaves; ++i) {
      const Joined<DP> k = left[i][lane];
      const float top = fmaxf(j.m, k.m);
      const float f = __builtin_amdgcn_exp2f(j.m - top), g = __builtin_amdgcn_exp2f(k.m - top);
      j.m = top;
      j.sum = j.sum * f + k.sum * g;
#pragma unroll
      for (int c = 0; c < DP / 64; ++c)
        j.acc[c] = weighted(j.acc[c], f) + weighted(k.acc[c], g);
    }
    store((int32_t)row, j);
  } else {
    for (int32_t r = wave; r < rows; r += kJoinWaves) store(r, join(r, 0, pieces));
  }
}

template <typename ET, int DP, bool ALL, uint32_t grid>
__global__ void __launch_bounds__(64 * kJoinWaves) token_join_kernel(AttnArgs a) {
  if constexpr (ALL) {
    __shared__ Joined<DP> left[kJoinWaves][64];
    token_join<ET, DP, true>(a, blockIdx.x, grid, left);
  } else {
    token_join<ET, DP, false>(a, blockIdx.x, grid, nullptr);
  }
}

template <typename ET, int DP>
hipError_t launch_token(const AttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((token_kernel<ET, DP>), dim3((unsigned)token_workers(DP)), dim3(64), 0, s, a);
  return hipGetLastError();
}

template <typename ET, int DP, uint32_t grid>
hipError_t launch_token_join(const AttnArgs& a, hipStream_t s) {
  // A pair has some workers / pairs pieces; from 16 on a workgroup a row joins them sooner (2
  // sequences of 20,000 to 32,000 tokens, 2 heads: the whole call 24 us, with a wave a row 50), and
  // below that a wave a row (16 of 3,000 to 9,000, 8 heads: 75.6 us, with a workgroup a row 77.4).
  const int64_t pairs = (int64_t)a.n_seq * a.kv_heads;
  const unsigned rows = (unsigned)a.skip_rows;
  if (16 * pairs <= (int64_t)grid)
    hipLaunchKernelGGL((token_join_kernel<ET, DP, true, grid>), dim3((unsigned)pairs * rows),
                       dim3(64 * kJoinWaves), 0, s, a);
  else
    hipLaunchKernelGGL((token_join_kernel<ET, DP, false, grid>), dim3((unsigned)pairs),
                       dim3(64 * (rows < kJoinWaves ? rows : kJoinWaves)), 0, s, a);
  return hipGetLastError();
}

}  // namespace attn
}  // namespace tod
