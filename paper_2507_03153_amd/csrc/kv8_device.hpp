// Device code of the 8-bit tier: E4M3 values with one E8M0 scale (2^(code - 127)) per 32 columns.
#pragma once

#include "hgca_device.hpp"

namespace hgca {

typedef float FloatPair __attribute__((ext_vector_type(2)));

constexpr int kKv8LeastScale = 127 - 110;        // least scale code: the least E4M3 value times 2^-110 is a normal number
constexpr int kKv8TopScale = 127 + 120;          // largest: 448 * 2^119 is less than the largest fp32 number, which is less than 256 * 2^120

// the scales of a row's blocks as they lie in memory
template <int D> struct Kv8Scales;
template <> struct Kv8Scales<64> { typedef uint16_t Word; };
template <> struct Kv8Scales<128> { typedef uint32_t Word; };

// scale of block `blk` from a row's scales
__device__ __forceinline__ float kv8_scale(uint32_t scales, int blk) { return __uint_as_float((scales >> (8 * blk) & 0xffu) << 23); }

// Two adjacent codes of a word (the lower pair, or with HIGH the upper one), times the scale; exact.
template <bool HIGH> __device__ __forceinline__ FloatPair kv8_pair_f32(uint32_t codes, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, HIGH);
}
template <bool HIGH> __device__ __forceinline__ uint32_t kv8_pair_bf16(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HIGH));
}

}  // namespace hgca
