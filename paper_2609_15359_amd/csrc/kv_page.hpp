// The 4-bit KV cache's pages (layout and number format in include/maps.h) and
// the value types that meet them.
#pragma once

#include "maps_internal.hpp"

namespace maps {
namespace kv {

// Offsets in one page of S tokens and D channels: K codes, K scales, V codes, V scales.
__host__ __device__ constexpr int64_t codes_bytes(int S, int D) { return int64_t(S) * (D / 2); }
__host__ __device__ constexpr int64_t scales_bytes(int S, int D) { return int64_t(S) * (D / 32); }
__host__ __device__ constexpr int64_t page_bytes(int S, int D) { return 2 * (codes_bytes(S, D) + scales_bytes(S, D)); }

// In the V part, byte i of token t, channel group r (D / 16 channels) and the
// scale of token t, block c (32 channels).
__host__ __device__ constexpr int64_t v_code(int t, int r, int i, int D) {
    return (int64_t(t / 4 * 16 + r) * 4 + t % 4) * (D / 32) + i;
}
__host__ __device__ constexpr int64_t v_scale(int t, int c, int D) { return int64_t(t / 4 * (D / 32) + c) * 4 + t % 4; }

constexpr uint32_t kScaleNan = 255, kScaleMin = 2, kScaleOne = 127;

inline bool block_ok(int S) { return S >= 16 && S <= MAPS_MAX_CACHE_BLOCK && (S & (S - 1)) == 0; }
inline bool dim_ok(int D) { return D == 64 || D == 128 || D == 256; }
inline int type_bytes(int32_t dtype) { return dtype == MAPS_F32 ? 4 : 2; }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A scale byte as the float 2^(byte - 127); 255 gives the exponent field of a
// NaN, which the conversions below take for one.
__device__ inline float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace kv
}  // namespace maps
