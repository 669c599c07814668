// paged_values.h — what the two attention kernels over pages share on the device: the two value types with their matrix
// instructions, exchanges between lanes, the transposing read of LDS.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qkv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __fp16 h16x2 __attribute__((ext_vector_type(2)));

__device__ inline float exp2f_(float x) { return __builtin_amdgcn_exp2f(x); }      // results below 2^-126 are 0

// Sum and maximum with the lane 16 or 32 further on (or back).  The instruction exchanges halves of two registers in place.
__device__ inline f32x2 pair16(float x) {
  const uint32_t a = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const uint32_t first = r[0], second = r[1];            // (a bit cast of the element itself takes the first one)
  return (f32x2){__builtin_bit_cast(float, first), __builtin_bit_cast(float, second)};
}
__device__ inline f32x2 pair32(float x) {
  const uint32_t a = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  const uint32_t first = r[0], second = r[1];            // (a bit cast of the element itself takes the first one)
  return (f32x2){__builtin_bit_cast(float, first), __builtin_bit_cast(float, second)};
}
__device__ inline float max16(float x) { const f32x2 p = pair16(x); return fmaxf(p.x, p.y); }
__device__ inline float max32(float x) { const f32x2 p = pair32(x); return fmaxf(p.x, p.y); }
__device__ inline float sum16(float x) { const f32x2 p = pair16(x); return p.x + p.y; }
__device__ inline float sum32(float x) { const f32x2 p = pair32(x); return p.x + p.y; }

// 16 lanes read four rows of 16 16-bit values, 8 bytes each (lane 4 r + c: piece c of row r), and get a column each: the four rows' values.
__device__ inline u32x2 read_turned(const uint8_t* at) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)at));
}

// Which 32-byte piece of a row of V stands where, by the row's token: pieces p ^ value_turn.  Rows of 128 bytes: two share the banks.
template <int D>
__device__ inline uint32_t value_turn(uint32_t token) {
  return D == 64 ? (token >> 1) & 3u : token & 7u;
}

// What is infinite or no number in the sums that parts of the keys have, of which `o` is the join by their weights: it stays that where a part weighs nothing.  0 times
// infinity is no number, and whether a value has no weight by itself or its part has none depends on how the keys were cut.  `part(i)`: the sums of part i < n.
template <typename Part>
__device__ inline void keep_odd(f32x4& o, uint32_t n, Part part) {
  const f32x4 zero = o * 0.0f;
  if (__builtin_expect(zero.x + zero.y + zero.z + zero.w == 0.0f, 1)) return;
  f32x4 odd = (f32x4)(0.0f);
  for (uint32_t i = 0; i < n; ++i) {
    const f32x4 x = part(i);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (!(__builtin_fabsf(x[k]) < INFINITY)) odd[k] += x[k];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (!(__builtin_fabsf(odd[k]) < INFINITY)) o[k] = odd[k];
}
// The same for a join's last factor, which is nothing where what it is joined with has all the weight.
__device__ inline f32x4 weighed(f32x4 o, float weight) {
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = __builtin_fabsf(o[k]) < INFINITY ? o[k] * weight : o[k];
  return o;
}

// Joins a result (lse, factor `scale` of its sums) with another one of log-sum `other_lse`: afterwards lse is that of both, and the
// result is the sums times `scale` plus the other one times `other`.
__device__ inline void join(float& lse, float other_lse, float& scale, float& other) {
  const float top = fmaxf(lse, other_lse);
  if (top == -INFINITY) {
    other = 0.0f;
    return;
  }
  const float a = exp2f_((lse - top) * 1.4426950408889634f), b = exp2f_((other_lse - top) * 1.4426950408889634f);
  const float both = a + b;
  scale *= a / both;
  other = b / both;
  lse = top + __builtin_amdgcn_logf(both) * 0.6931471805599453f;       // both: 1 to 2
}

struct Half {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  typedef _Float16 x4 __attribute__((ext_vector_type(4)));
  typedef _Float16 one;
  static constexpr uint32_t kExponent = 0x7C00u;
  static constexpr uint32_t kParts = 2;
  static __device__ inline f32x4 mfma16(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static __device__ inline f32x16 mfma32(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  // Weights are 2^kLift times what they are, the largest 2^15 (2^16 where a maximum's own steps are larger than that): a part's last bit is 2^-24 at the
  // smallest, 2^-39 of the largest weight.
  static constexpr float kLift = 15.0f;
  // e, at most 2^16, as a sum of parts: the first one cut off towards zero, which stops at 65504, the rest rounded.
  static __device__ inline void parts(const float (&e)[8], x8 (&w)[kParts]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const h16x2 high = __builtin_amdgcn_cvt_pkrtz(e[j], 0.0f);
      w[0][j] = (_Float16)high[0];
      w[1][j] = (_Float16)(e[j] - (float)w[0][j]);
    }
  }
};

struct BFloat {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 x4 __attribute__((ext_vector_type(4)));
  typedef __bf16 one;
  static constexpr uint32_t kExponent = 0x7F80u;
  static constexpr uint32_t kParts = 3;
  static __device__ inline f32x4 mfma16(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ inline f32x16 mfma32(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static constexpr float kLift = 0.0f;                   // parts reach as far down as e itself does
  static __device__ inline void parts(const float (&e)[8], x8 (&w)[kParts]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float high = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, e[j]) & 0xFFFF0000u), rest = e[j] - high;
      const float middle = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, rest) & 0xFFFF0000u), low = rest - middle;
      w[0][j] = (__bf16)high;
      w[1][j] = (__bf16)middle;
      w[2][j] = (__bf16)low;
    }
  }
};

}  // namespace qkv
