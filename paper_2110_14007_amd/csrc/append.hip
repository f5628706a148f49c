// Appends to a paged key / value cache with the position rotation applied on
// the way, as 16-bit rows or as 4-bit rows, and rows of a 4-bit cache read
// back.
//
// Rotation.  Elements (i, i + r / 2), or (2 i, 2 i + 1), of the first r of a
// head are a pair (x, y) that turns by the angle pos * rate_i:
//   x' = x cos - y sin,  y' = x sin + y cos.
// The angle of a far position has to be right to a small part of a turn, so
// that it is formed and reduced in 64 bits.  The product of a 32-bit position
// and a 24-bit rate has up to 55 of them: what it loses past the 53rd is kept
// beside it.
//
// 4-bit rows.  Of 32 elements with the largest magnitude a, the scale 2^e is
// the smallest with a <= 7 2^e: then the largest error is 2^e, at 7 and
// between 4 and 6 alike.  e stays in [-23, 13] (fp16) or [-125, 125] (bf16), so
// that every value that a code and a scale stand for is a number of the type.
// Keys are rotated in 64 bits and rounded to odd 32-bit numbers, which no border
// of scales and codes is: an element next to a border gets the code that the
// formula gives.
//
// All three are bound by their bytes, or by their start where there are few.
// Measured: 48 tokens of 32 + 8 heads of 128 4.8 us; 20,011 of them into 16-bit
// pages 95 us (492 MB, 5.2 TB/s), 16,001 into a 4-bit cache 72 us (345 MB, 4.8 TB/s:
// the 64-bit rotation of keys takes the rest), 90,001 rows of 8 heads read back
// 106 us (369 MB written, 98 read, in halves of 128-byte lines: 171 fetched).
#include "seq.h"

#include "seq4.h"

namespace tod {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kMostAngles = 128;  // of a head of 256 elements

template <typename ET>
struct Exponents;  // of a block's scale
template <>
struct Exponents<_Float16> {
  static constexpr int lo = -23, hi = 13;
};
template <>
struct Exponents<__bf16> {
  static constexpr int lo = -125, hi = 125;
};

template <typename ET, typename T>
__device__ __forceinline__ T number(uint16_t u) {
  return (T)(float)__builtin_bit_cast(ET, u);
}
template <typename ET, typename T>
__device__ __forceinline__ T element(const u32x4& w, int i) {
  return number<ET, T>((uint16_t)(w[i / 2] >> (16 * (i % 2))));
}

// How a head's pairs lie: neighbours, halves apart by a multiple of 8 elements (a piece's partners
// are a piece too), or halves apart otherwise.
enum class Pairs { kNeighbours, kPieces, kOdd };

// What the rotation of the eight elements from e0 on needs of the row at p.  What there is nothing to
// load for, is loaded from the row's start: there is no branch around the loads.
template <Pairs PAIRS>
struct Piece {
  u32x4 own, other;  // other: the partners, for kPieces
};

template <Pairs PAIRS>
__device__ __forceinline__ Piece<PAIRS> load_piece(const uint16_t* p, int e0, int rotary) {
  Piece<PAIRS> w;
  w.own = *(const u32x4*)(p + e0);
  if constexpr (PAIRS == Pairs::kPieces) {
    const int half = rotary / 2;
    w.other = *(const u32x4*)(p + (e0 >= rotary ? 0 : e0 < half ? e0 + half : e0 - half));
  }
  return w;
}

// Where the angle of pair m lies in LDS: the threads of a row read angles that are 8 (4) pairs apart.
template <Pairs PAIRS>
__device__ __forceinline__ int place_of(int m, int half) {
  if constexpr (PAIRS == Pairs::kNeighbours)
    return m % 4 * ((half + 3) / 4) + m / 4;
  else if constexpr (PAIRS == Pairs::kPieces)
    return m % 8 * (half / 8) + m / 8;
  else
    return m;
}

// The eight elements from e0 on, rotated, in the arithmetic of T.  `unit` is what the angles' cosines
// and sines are scaled by.
template <typename ET, typename T, Pairs PAIRS, typename Angle>
__device__ __forceinline__ void rotate(T (&x)[8], const Piece<PAIRS>& w, const uint16_t* p, int e0,
                                       int rotary, const Angle* turn, T unit) {
  const int half = rotary / 2;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = element<ET, T>(w.own, i);
  if (PAIRS == Pairs::kOdd || e0 >= rotary) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= unit;
    if (e0 >= rotary) return;
  }
  if constexpr (PAIRS == Pairs::kNeighbours) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      if (e0 + i < rotary) {
        const Angle t = turn[i / 2 * ((half + 3) / 4) + e0 / 8];
        const T a = x[i], b = x[i + 1];
        x[i] = a * t.x - b * t.y;
        x[i + 1] = a * t.y + b * t.x;
      } else {
        x[i] *= unit;
        x[i + 1] *= unit;
      }
    }
  } else if constexpr (PAIRS == Pairs::kPieces) {
    const bool first = e0 < half;
    const Angle* const at = turn + (first ? e0 : e0 - half) / 8;
    // The first of a pair takes its partner's sine with the other sign: the partner's is changed.
    const u32x4 other = w.other ^ (first ? 0x80008000u : 0u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Angle t = at[i * (half / 8)];
      x[i] = x[i] * t.x + element<ET, T>(other, i) * t.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = e0 + i;
      if (e >= rotary) break;
      const bool first = e < half;
      const Angle t = turn[first ? e : e - half];
      const T other = number<ET, T>(p[first ? e + half : e - half]);
      x[i] = element<ET, T>(w.own, i) * t.x + other * (first ? -t.y : t.y);
    }
  }
}

template <typename ET>
__device__ __forceinline__ u32x4 rounded(const float (&x)[8]) {
  typedef ET e2 __attribute__((ext_vector_type(2)));
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    e2 v;
    v[0] = (ET)x[2 * i];
    v[1] = (ET)x[2 * i + 1];
    w[i] = __builtin_bit_cast(uint32_t, v);
  }
  return w;
}

// y rounded to a float to odd: exact, or the one of its two neighbours whose last bit is set.  Floats
// whose last bit is clear, the borders of codes and of scales among them, then lie on the same side of
// the result as of y, and are met by no other y than themselves.
__device__ __forceinline__ float to_odd(double y) {
  const float f = (float)y;
  const uint32_t u = __float_as_uint(f);
  const double back = (double)f;
  return __uint_as_float((fabs(back) > fabs(y) ? u - 1 : u) | (back != y ? 1u : 0u));
}

// Exponent of the scale of a block whose largest magnitude is a (finite), from a's bits: from
// a = f 2^E with 1 <= f < 2, a <= 7 2^e = 1.75 2^(e + 2) holds from e = E - 2 on if f <= 1.75, else
// from E - 1.  (Below the normal numbers the least e is right.)
template <typename ET>
__device__ __forceinline__ int block_exponent(uint32_t a, int more) {
  const int e = (int)(a >> 23) - 129 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0) + more;
  return min(max(e, Exponents<ET>::lo), Exponents<ET>::hi);
}

// Maximum over the four lanes that hold a block.
__device__ __forceinline__ uint32_t over_block(uint32_t v) {
  v = max(v, (uint32_t)__shfl_xor((int)v, 1, 64));
  return max(v, (uint32_t)__shfl_xor((int)v, 2, 64));
}

// Codes of a lane's eight elements of a block, and the block's scale byte: 255 (and the codes 0)
// where an element is not finite.  Four lanes in a row hold a block.  The elements come halved: a
// rotated one may be larger than its type's numbers are.
template <typename ET>
__device__ __forceinline__ uint32_t encode(const double (&x)[8], uint32_t* scale) {
  float f[8];
  uint32_t top = 0;  // magnitudes compare as their bits
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f[i] = to_odd(x[i]);
    top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
  }
  top = over_block(top);
  if (top >= 0x7f800000u) {
    *scale = 255;
    return 0;
  }
  *scale = (uint32_t)(block_exponent<ET>(top, 1) + 127);
  const float by = scale_of(*scale - 1);
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0], f[1], by, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2], f[3], by, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4], f[5], by, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6], f[7], by, 3);
}

// The same for elements as they are.
template <typename ET>
__device__ __forceinline__ uint32_t encode16(const u32x4& w, uint32_t* scale) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  constexpr uint32_t kInf = std::is_same<ET, _Float16>::value ? 0x7c00 : 0x7f80;
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
  const uint32_t top = over_block(max((uint32_t)m[0], (uint32_t)m[1]));
  if (top >= kInf) {
    *scale = 255;
    return 0;
  }
  const float a = (float)__builtin_bit_cast(ET, (uint16_t)top);
  *scale = (uint32_t)(block_exponent<ET>(__float_as_uint(a), 0) + 127);
  const float by = scale_of(*scale);
  uint32_t codes = 0;
  codes = two_codes<ET, 0>(codes, w[0], by);
  codes = two_codes<ET, 1>(codes, w[1], by);
  codes = two_codes<ET, 2>(codes, w[2], by);
  return two_codes<ET, 3>(codes, w[3], by);
}

// Cosine and sine of pos * rate: the angle (of fewer than 2^31 radians) less the nearest multiple n of a
// quarter turn, in two parts (the first difference is exact, for its terms are multiples of 2^-53 and
// it is small), and what the product lost; then the Taylor series to the terms that a T holds, and the
// quarter's exchange.
template <typename T>
__device__ __forceinline__ void turn_by(int32_t pos, float rate, T* cosine, T* sine) {
  constexpr double kQuarter = 0x1.921fb54442d18p+0, kRest = 0x1.1a62633145c07p-54;  // pi / 2
  const double angle = (double)pos * (double)rate;
  const double lost = fma((double)pos, (double)rate, -angle);
  if (fabs(angle) >= 0x1p31) {  // (a NaN too, below)
    double s, c, s1, c1;
    sincos(angle, &s, &c);
    sincos(lost, &s1, &c1);
    *cosine = (T)(c * c1 - s * s1);
    *sine = (T)(s * c1 + c * s1);
    return;
  }
  const double n = rint(angle * 0.63661977236758134308);
  const T r = (T)(fma(-n, kRest, fma(-n, kQuarter, angle)) + lost);
  const T x = r * r;
  T s, c;
  if constexpr (sizeof(T) == 8) {
    s = 1.0 / 355687428096000.0;
    s = fma(s, x, -1.0 / 1307674368000.0);
    s = fma(s, x, 1.0 / 6227020800.0);
    s = fma(s, x, -1.0 / 39916800.0);
    s = fma(s, x, 1.0 / 362880.0);
    s = fma(s, x, -1.0 / 5040.0);
    s = fma(s, x, 1.0 / 120.0);
    s = fma(s, x, -1.0 / 6.0);
    c = -1.0 / 6402373705728000.0;
    c = fma(c, x, 1.0 / 20922789888000.0);
    c = fma(c, x, -1.0 / 87178291200.0);
    c = fma(c, x, 1.0 / 479001600.0);
    c = fma(c, x, -1.0 / 3628800.0);
    c = fma(c, x, 1.0 / 40320.0);
    c = fma(c, x, -1.0 / 720.0);
    c = fma(c, x, 1.0 / 24.0);
    c = fma(c, x, -0.5);
    s = fma(s * x, r, r);
    c = fma(c, x, 1.0);
  } else {
    s = 1.0f / 362880.0f;
    s = fmaf(s, x, -1.0f / 5040.0f);
    s = fmaf(s, x, 1.0f / 120.0f);
    s = fmaf(s, x, -1.0f / 6.0f);
    c = -1.0f / 3628800.0f;
    c = fmaf(c, x, 1.0f / 40320.0f);
    c = fmaf(c, x, -1.0f / 720.0f);
    c = fmaf(c, x, 1.0f / 24.0f);
    c = fmaf(c, x, -0.5f);
    s = fmaf(s * x, r, r);
    c = fmaf(c, x, 1.0f);
  }
  const int q = (int)n;
  const T p = q & 1 ? s : c, t = q & 1 ? c : s;
  *cosine = (q + 1) & 2 ? -p : p;
  *sine = q & 2 ? -t : t;
}

enum class Rows { kQueries, kKeys, kValues };

// A workgroup takes TOKENS tokens at a time: their angles' cosines and sines go to LDS, then each
// thread takes one 16-byte piece of every so many of their rows, several rows' loads at once.  For a
// 4-bit cache keys are rotated in 64 bits and halved (see encode).
template <typename ET, bool FOUR, Pairs PAIRS, int TOKENS>
__global__ void __launch_bounds__(kThreads) append_kernel(AppendArgs a) {
  __shared__ float2 turn[TOKENS][kMostAngles];
  __shared__ double2 turn4[FOUR ? TOKENS : 1][kMostAngles];
  const int tid = threadIdx.x;
  const int32_t per_row = (int32_t)a.per_row.d, half = a.rotary / 2;
  const int32_t step = (int32_t)a.step;  // rows of a pass; threads past them have none
  const int32_t r0 = (int32_t)div_by((uint32_t)tid, a.per_row), c = tid - r0 * per_row;

  for (int64_t t0 = (int64_t)blockIdx.x * TOKENS; t0 < a.tokens; t0 += (int64_t)gridDim.x * TOKENS) {
    const int32_t count = (int32_t)min((int64_t)TOKENS, a.tokens - t0);
    __syncthreads();  // the tokens before are done with the angles
    for (int i = tid; i < count * half; i += kThreads) {
      const int32_t k = (int32_t)div_by((uint32_t)i, a.angles), m = i - k * half;
      const int32_t pos = a.pos[t0 + k];
      const float rate = a.rates[m];
      const int at = place_of<PAIRS>(m, half);
      if constexpr (FOUR) {
        double x, y;
        turn_by<double>(pos, rate, &x, &y);
        turn[k][at] = {(float)x, (float)y};
        turn4[k][at] = {0.5 * x, 0.5 * y};
      } else {
        float x, y;
        turn_by<float>(pos, rate, &x, &y);
        turn[k][at] = {x, y};
      }
    }
    __syncthreads();

    auto pass = [&](auto KIND, const FastDiv& heads, const void* rows, int64_t token_stride,
                    int64_t head_stride) __attribute__((always_inline)) {
      constexpr Rows kind = decltype(KIND)::value;
      constexpr Pairs pairs = kind == Rows::kValues ? Pairs::kOdd : PAIRS;  // (values have no partners)
      constexpr int kAhead = FOUR && kind == Rows::kKeys ? 2 : 4;
      const int32_t n = r0 < step ? count * (int32_t)heads.d : 0;
      for (int32_t r = r0; r < n; r += kAhead * step) {
        const uint16_t* from[kAhead];
        Piece<pairs> w[kAhead];
        int64_t slot[kAhead];
        int32_t tok[kAhead], head[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int32_t at = min(r + i * step, n - 1);
          tok[i] = (int32_t)div_by((uint32_t)at, heads);
          head[i] = at - tok[i] * (int32_t)heads.d;
          from[i] = (const uint16_t*)rows + (t0 + tok[i]) * token_stride + head[i] * head_stride;
          if constexpr (kind != Rows::kQueries) slot[i] = a.slot[t0 + tok[i]];
          w[i] = load_piece<pairs>(from[i], 8 * c, a.rotary);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          if (r + i * step >= n) break;
          if constexpr (kind == Rows::kQueries) {
            float x[8];
            rotate<ET, float, pairs>(x, w[i], from[i], 8 * c, a.rotary, turn[tok[i]], 1.0f);
            ((u32x4*)a.q_out)[((t0 + tok[i]) * a.heads + head[i]) * per_row + c] = rounded<ET>(x);
          } else {
            if (slot[i] < 0 || slot[i] >= a.slots) continue;
            const uint32_t page = div_by((uint32_t)slot[i], a.page);
            const uint32_t row = (uint32_t)slot[i] - page * a.page.d;
            const int64_t to =
                (((int64_t)page * a.kv_heads + head[i]) * a.page.d + row) * per_row + c;
            void* const pages = kind == Rows::kKeys ? a.k_pages : a.v_pages;
            if constexpr (FOUR) {
              uint32_t scale;
              if constexpr (kind == Rows::kKeys) {
                double x[8];
                rotate<ET, double, pairs>(x, w[i], from[i], 8 * c, a.rotary, turn4[tok[i]], 0.5);
                ((uint32_t*)pages)[to] = encode<ET>(x, &scale);
              } else {
                ((uint32_t*)pages)[to] = encode16<ET>(w[i].own, &scale);
              }
              if (c % 4 == 0)
                (kind == Rows::kKeys ? a.k_scales : a.v_scales)[to / 4] = (uint8_t)scale;
            } else if constexpr (kind == Rows::kKeys) {
              float x[8];
              rotate<ET, float, pairs>(x, w[i], from[i], 8 * c, a.rotary, turn[tok[i]], 1.0f);
              ((u32x4*)pages)[to] = rounded<ET>(x);
            } else {
              ((u32x4*)pages)[to] = w[i].own;
            }
          }
        }
      }
    };
    pass(std::integral_constant<Rows, Rows::kQueries>{}, a.q_heads, a.q, a.q_row, a.q_head);
    pass(std::integral_constant<Rows, Rows::kKeys>{}, a.k_heads, a.k, a.k_row, a.k_head);
    pass(std::integral_constant<Rows, Rows::kValues>{}, a.k_heads, a.v, a.v_row, a.v_head);
  }
}

// One thread takes eight elements of a key row and of its value row.
template <typename ET>
__global__ void __launch_bounds__(kThreads) read4_kernel(Read4Args a) {
  const uint32_t i = blockIdx.x * (uint32_t)kThreads + threadIdx.x;
  const uint32_t t = div_by(i, a.per_token);
  if (t >= (uint32_t)a.tokens) return;
  const uint32_t in = i - t * a.per_token.d;
  const int64_t slot = a.slot[t];
  const bool kept = slot >= 0 && slot < a.slots;
  u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (kept) {
    const uint32_t h = div_by(in, a.per_row), c = in - h * a.per_row.d;
    const uint32_t page = div_by((uint32_t)slot, a.page), row = (uint32_t)slot - page * a.page.d;
    const int64_t at = (((int64_t)page * a.kv_heads + h) * a.page.d + row) * a.per_row.d + c;
    k = eight_values<ET>(((const uint32_t*)a.k_codes)[at], scale_of(a.k_scales[at / 4]));
    v = eight_values<ET>(((const uint32_t*)a.v_codes)[at], scale_of(a.v_scales[at / 4]));
  }
  const int64_t to = (int64_t)t * a.per_token.d + in;
  __builtin_nontemporal_store(k, (u32x4*)a.k_out + to);
  __builtin_nontemporal_store(v, (u32x4*)a.v_out + to);
}

template <typename ET, bool FOUR, Pairs PAIRS>
hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
  constexpr int kTokens = 4;
  const int64_t most = 1 << 20;
  // One token a workgroup while there are few of them: 100 tokens of 32 + 8 heads of 128, the call
  // alone, 23.4 us, by four tokens 25.3; 3,000, back to back, 16.5 and 14.4.
  const bool few = a.tokens <= 1024;
  const int64_t groups = few ? a.tokens : (a.tokens + kTokens - 1) / kTokens;
  hipLaunchKernelGGL((few ? append_kernel<ET, FOUR, PAIRS, 1> : append_kernel<ET, FOUR, PAIRS, kTokens>),
                     dim3((unsigned)(groups < most ? groups : most)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <typename ET, bool FOUR>
hipError_t launch_append(const AppendArgs& given, hipStream_t s) {
  AppendArgs a = given;
  a.step = kThreads / a.per_row.d;
  a.q_heads = fast_div((uint32_t)a.heads);
  a.k_heads = fast_div((uint32_t)a.kv_heads);
  a.angles = fast_div((uint32_t)(a.rotary > 2 ? a.rotary / 2 : 1));
  if (a.interleaved) return launch_append<ET, FOUR, Pairs::kNeighbours>(a, s);
  if (a.rotary % 16 == 0) return launch_append<ET, FOUR, Pairs::kPieces>(a, s);
  return launch_append<ET, FOUR, Pairs::kOdd>(a, s);
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, bool half, bool four, hipStream_t s) {
  if (four) return half ? launch_append<_Float16, true>(a, s) : launch_append<__bf16, true>(a, s);
  return half ? launch_append<_Float16, false>(a, s) : launch_append<__bf16, false>(a, s);
}

hipError_t launch_read4(const Read4Args& a, bool half, hipStream_t s) {
  const int64_t pieces = a.tokens * a.per_token.d;
  hipLaunchKernelGGL((half ? read4_kernel<_Float16> : read4_kernel<__bf16>),
                     dim3((unsigned)((pieces + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace tod
