// What the kernels that attend with a few queries per sequence share (tree_kernels.hip: up to 32 rows per KV head and fp32,
// tree_rows_kernels.hip: more).
#pragma once

#include "append_device.hpp"
#include "kv8_device.hpp"

namespace hgca {

namespace {

constexpr float kLn2 = 0.6931471805599453f, kTreeLog2e = 1.4426950408889634f;
constexpr int kTreeWaves = 4, kTreeBlock = kTreeWaves * kWave;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{lo, hi}), bf16x2));
}

// A sequence's tokens of one tier that a workgroup goes through: a split, cut by the sequence's own length in whole steps of the
// workgroup.
struct Span {
    int len, begin, end;
    __device__ __forceinline__ Span(const TreeArgs &a, int b, int split, int unit) {
        len = tier_len(a.kv, b);
        const int64_t per = (((int64_t)len + a.n_splits - 1) / a.n_splits + unit - 1) / unit * unit;
        begin = (int)min(split * per, (int64_t)len);
        end = (int)min(begin + per, (int64_t)len);
    }
};

// Which of the 64 tokens from `base` on a row sees: below `tail` all, from there the bits of `mask`, nothing from `end` on.
__device__ __forceinline__ uint64_t seen_tokens(uint64_t mask, int base, int tail, int end) {
    const int j = base - tail, left = end - base;
    const uint64_t m = j >= 64 ? 0 : j >= 0 ? mask >> j : j > -64 ? mask << -j | ((1ull << -j) - 1) : ~0ull;
    return left <= 0 ? 0 : left >= 64 ? m : m & ((1ull << left) - 1);
}

// Infinities and NaN in bf16: the sum carries into the sign of a half whose exponent bits are all ones; those halves as a mask.
constexpr uint32_t kSigns = 0x80008000u;
__device__ __forceinline__ uint32_t odd_carry(uint32_t x) { return (x & 0x7fff7fffu) + 0x00800080u; }
__device__ __forceinline__ uint32_t odd_halves(uint32_t x) {
    const uint32_t bad = odd_carry(x) & kSigns;
    return bad | (bad - (bad >> 15));
}

// +inf, -inf and NaN are counted one after another, as products of ones: a half of `x` is of the kind iff (half & keep) - from <= more.
struct OddKind {
    uint32_t keep, from, more;
    float add;
    __device__ __forceinline__ explicit OddKind(int kind)
        : keep(kind == 2 ? 0x7fffu : 0xffffu), from(kind == 0 ? 0x7f80u : kind == 1 ? 0xff80u : 0x7f81u), more(kind == 2 ? 0x7eu : 0u),
          add(kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN) {}
    __device__ __forceinline__ uint32_t ones(uint32_t x) const {
        return ((x & keep) - from <= more ? 0x3f80u : 0u) | ((x >> 16 & keep) - from <= more ? 0x3f800000u : 0u);
    }
};

}  // namespace

}  // namespace hgca
