// paged_prompt.h — what the two kernels for many new tokens share: how a running maximum is kept, how rows stand in LDS.
#pragma once

#include "paged.h"
#include "paged_values.h"
#include "qkv_common.h"

namespace qkv {

constexpr float kLift = 7.0f, kSlack = 8.0f;
// From here on a maximum's rounding counts in an exponent that is not rounded: scores are multiplied with the scale by themselves, and m follows at once.
// A wave's pairs change over together.  Where one of them has a smaller maximum its scores were not rounded up to there and are afterwards, which may set
// equal ones apart by half a step: 2^-13 at most, a fraction of what rounding a weight to 16 bits does.
constexpr float kFar = 0x1p12f;
constexpr uint32_t kLost = 1u, kScaled = 2u;             // what a wave has met: an entry that names no page, a maximum beyond kFar
__device__ inline float uniform(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }

// Rows of K and V in LDS are longer than they need to be, by 16 and 64 bytes: 16 lanes that read a piece of 16 bytes of as many rows of K, and 32 that
// read 64 bytes of four rows of V through the transposing read, then meet every bank once.

constexpr uint32_t key_row(int D) { return D * 2u + 16u; }
constexpr uint32_t value_row(int D) { return D * 2u + 64u; }

}  // namespace qkv
