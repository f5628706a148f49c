// Appends to a paged key / value cache with the position rotation applied on
// the way, as 16-bit rows or as 4-bit rows, and rows of a 4-bit cache read
// back.
//
// Rotation.  Elements (i, i + r / 2), or (2 i, 2 i + 1), of the first r of a
// head are a pair (x, y) that turns by the angle pos * rate_i:
//   x' = x cos - y sin,  y' = x sin + y cos.
// The angle of a far position has to be right to a small part of a turn, so
// that it is formed in 64 bits, where the product of a 32-bit position and a
// 24-bit rate is exact below 2^53, and so are its cosine and sine.
//
// 4-bit rows.  Of 32 elements with the largest magnitude a, the scale 2^e is
// the smallest with a <= 7 2^e: then the largest error is 2^e, at 7 and
// between 4 and 6 alike.  e stays in [-23, 13] (fp16) or [-125, 125] (bf16), so
// that every value that a code and a scale stand for is a number of the type.
// Rotated keys are scaled and rounded in 64 bits: an element next to the border
// of two codes gets the one that the formula gives.
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

template <typename ET>
__device__ __forceinline__ float element(const u32x4& w, int i) {
  return (float)__builtin_bit_cast(ET, (uint16_t)(w[i / 2] >> (16 * (i % 2))));
}

// Eight elements from e0 on of a head at p, rotated, in the arithmetic of T.  Pairs that are
// halves apart by a multiple of 8 elements lie in two loads of 16 bytes (WIDE), others are read one by
// one.
template <typename ET, typename T, bool PAIRS, bool WIDE, typename Angle>
__device__ __forceinline__ void rotate(T (&x)[8], const uint16_t* p, int e0, int rotary,
                                       const Angle* turn) {
  const u32x4 w = *(const u32x4*)(p + e0);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (T)element<ET>(w, i);
  if (e0 >= rotary) return;
  if constexpr (PAIRS) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      if (e0 + i >= rotary) break;
      const Angle t = turn[(e0 + i) / 2];
      const T a = x[i], b = x[i + 1];
      x[i] = a * (T)t.x - b * (T)t.y;
      x[i + 1] = a * (T)t.y + b * (T)t.x;
    }
  } else if constexpr (WIDE) {
    const int half = rotary / 2;
    const bool first = e0 < half;
    const u32x4 v = *(const u32x4*)(p + (first ? e0 + half : e0 - half));
    const Angle* const at = turn + (first ? e0 : e0 - half);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Angle t = at[i];
      const T other = (T)element<ET>(v, i), s = (T)t.y;
      x[i] = x[i] * (T)t.x + other * (first ? -s : s);
    }
  } else {
    const int half = rotary / 2;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = e0 + i;
      if (e >= rotary) break;
      const bool first = e < half;
      const Angle t = turn[first ? e : e - half];
      const T other = (T)(float)__builtin_bit_cast(ET, p[first ? e + half : e - half]);
      const T s = (T)t.y;
      x[i] = x[i] * (T)t.x + other * (first ? -s : s);
    }
  }
}

template <typename ET, typename T>
__device__ __forceinline__ u32x4 rounded(const T (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const ET a = (ET)(float)x[2 * i], b = (ET)(float)x[2 * i + 1];
    w[i] = (uint32_t)__builtin_bit_cast(uint16_t, a) |
           (uint32_t)__builtin_bit_cast(uint16_t, b) << 16;
  }
  return w;
}

// Exponent of the scale of a block whose largest magnitude is a (finite): from a = f 2^E with
// 1 <= f < 2, a <= 7 2^e = 1.75 2^(e + 2) holds from e = E - 2 on if f <= 1.75, else from E - 1.
template <typename ET>
__device__ __forceinline__ int block_exponent(double a) {
  const uint64_t u = (uint64_t)__double_as_longlong(a);
  const int e = (int)(u >> 52) - 1025 + ((u & 0xfffffffffffffull) > 0xc000000000000ull ? 1 : 0);
  return min(max(e, Exponents<ET>::lo), Exponents<ET>::hi);
}

__device__ __forceinline__ double power2(int e) {
  return __longlong_as_double((long long)(e + 1023) << 52);
}

// Code of x, in units of the scale: below 2 in steps of 1/2, below 4 of 1, from there of 2 up to 6,
// ties to the even code.
__device__ __forceinline__ uint32_t code_of(double x) {
  const double m = fabs(x);
  const double n = m < 2.0 ? rint(m + m) : m < 4.0 ? rint(m) + 2.0 : rint(0.5 * m) + 4.0;
  return (uint32_t)fmin(n, 7.0) | (x < 0.0 ? 8u : 0u);
}

// Maximum over the four lanes that hold a block.
template <typename T>
__device__ __forceinline__ T over_block(T v) {
  v = fmax(v, __shfl_xor(v, 1, 64));
  return fmax(v, __shfl_xor(v, 2, 64));
}

// Codes of a lane's eight elements of a block, and the block's scale byte: 255 (and the codes 0)
// where an element is not finite.  Four lanes in a row hold a block.
template <typename ET>
__device__ __forceinline__ uint32_t encode(const double (&x)[8], uint32_t* scale) {
  double top = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double m = fabs(x[i]);
    top = fmax(top, m <= 1.7e308 ? m : HUGE_VAL);  // (a NaN too)
  }
  top = over_block(top);
  if (!(top <= 1.7e308)) {
    *scale = 255;
    return 0;
  }
  const int e = block_exponent<ET>(top);
  *scale = (uint32_t)(e + 127);
  const double by = power2(-e);
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) codes |= code_of(x[i] * by) << (4 * i);
  return codes;
}

// A workgroup takes a token at a time: its angles' cosines and sines go to LDS, then each thread
// takes 16-byte pieces of the query heads, the keys and the values.
template <typename ET, bool FOUR, bool PAIRS, bool WIDE>
__global__ void __launch_bounds__(kThreads) append_kernel(AppendArgs a) {
  __shared__ double2 turn[kMostAngles];
  const int tid = threadIdx.x;
  const int32_t per_row = (int32_t)a.per_row.d, half = a.rotary / 2;
  const int32_t hq = a.heads, hk = a.kv_heads, pieces = (hq + 2 * hk) * per_row;
  for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    const int64_t slot = a.slot[t];
    const double pos = (double)a.pos[t];
    __syncthreads();  // the token before is done with the angles
    for (int i = tid; i < half; i += kThreads) {
      double2 w;
      sincos(pos * (double)a.rates[i], &w.y, &w.x);
      turn[i] = w;
    }
    __syncthreads();
    const bool kept = slot >= 0 && slot < a.slots;
    const uint32_t page = kept ? div_by((uint32_t)slot, a.page) : 0u;
    const uint32_t row = kept ? (uint32_t)slot - page * a.page.d : 0u;
    for (int32_t p = tid; p < pieces; p += kThreads) {
      const int32_t h = (int32_t)div_by((uint32_t)p, a.per_row), c = p - h * per_row;
      if (h < hq) {
        float x[8];
        rotate<ET, float, PAIRS, WIDE>(x, (const uint16_t*)a.q + t * a.q_row + h * a.q_head, 8 * c,
                                       a.rotary, turn);
        ((u32x4*)a.q_out)[(t * hq + h) * per_row + c] = rounded<ET>(x);
        continue;
      }
      if (!kept) continue;
      const bool isk = h < hq + hk;
      const int32_t kh = h - hq - (isk ? 0 : hk);
      const uint16_t* const from = isk ? (const uint16_t*)a.k + t * a.k_row + kh * a.k_head
                                       : (const uint16_t*)a.v + t * a.v_row + kh * a.v_head;
      const int64_t to = (((int64_t)page * hk + kh) * a.page.d + row) * per_row + c;
      if constexpr (FOUR) {
        double x[8];
        rotate<ET, double, PAIRS, WIDE>(x, from, 8 * c, isk ? a.rotary : 0, turn);
        uint32_t scale;
        const uint32_t codes = encode<ET>(x, &scale);
        ((uint32_t*)(isk ? a.k_pages : a.v_pages))[to] = codes;
        if (c % 4 == 0) (isk ? a.k_scales : a.v_scales)[to / 4] = (uint8_t)scale;
      } else {
        u32x4 w;
        if (isk) {
          float x[8];
          rotate<ET, float, PAIRS, WIDE>(x, from, 8 * c, a.rotary, turn);
          w = rounded<ET>(x);
        } else {
          w = *(const u32x4*)(from + 8 * c);
        }
        ((u32x4*)(isk ? a.k_pages : a.v_pages))[to] = w;
      }
    }
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
  ((u32x4*)a.k_out)[to] = k;
  ((u32x4*)a.v_out)[to] = v;
}

template <typename ET, bool FOUR>
hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
  const int64_t most = 1 << 20;
  const dim3 grid((unsigned)(a.tokens < most ? a.tokens : most));
  const auto kern = a.interleaved               ? append_kernel<ET, FOUR, true, true>
                    : a.rotary / 2 % 8 == 0 ? append_kernel<ET, FOUR, false, true>
                                                : append_kernel<ET, FOUR, false, false>;
  hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
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
