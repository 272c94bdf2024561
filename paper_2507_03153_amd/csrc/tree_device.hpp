// What the kernels that attend with a few queries per sequence share (tree_kernels.hip: few rows per KV head and fp32,
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

// The part of a sequence's tokens that a workgroup goes through.  With one split per sequence it is the whole; else the launch has
// batch * n_splits slots per KV head and block of rows.  Up to 64 sequences take as many of them as their own lengths ask for:
// slots of C whole steps, C about the least with which all sequences' slots are enough.  (With n_splits slots for every
// sequence the longest one sets the time: 16 queries x 4 over 61 to 122 K tokens 431 : 345 to 390 us.)  Every wave works the cut out for itself, a lane per sequence; a
// sequence without tokens takes a slot too.  More sequences fill the device with a few slots each: n_splits equal ones.
struct Span {
    int b, len, begin, end;
    int slot, first_slot, n_slots;               // first_slot, n_slots: the sequence's
    bool idle;                                   // no sequence needs the slot
    __device__ __forceinline__ Span(const TreeArgs &a, int slot_of_launch, int unit) {
        slot = slot_of_launch;
        idle = false;
        const int B = a.sh.batch;
        int64_t per;
        if (a.n_splits == 1 || B > kWave) {
            b = slot / a.n_splits;
            n_slots = a.n_splits;
            first_slot = b * n_slots;
            len = tier_len(a.kv, b);
            per = (((int64_t)len + n_slots - 1) / n_slots + unit - 1) / unit * unit;
        } else {
            const int lane = threadIdx.x % kWave, slots = B * a.n_splits;
            const int tokens = lane < B ? tier_len(a.kv, lane) : 0, steps = lane < B ? max((tokens + unit - 1) / unit, 1) : 0;
            auto counts = [&](int c) {           // ceil(steps / c): c is at least total / slots, so it is 1024 at most, and the
                int n = (int)((float)steps * __builtin_amdgcn_rcpf((float)c) * 0.999999f);       // quotient in fp32 off by one, downwards
                n += n * c < steps ? 1 : 0;
                return n + (n * c < steps ? 1 : 0);
            };
            auto enough = [&](int c) { return wave_sum((float)min(counts(c), slots + 1)) <= (float)slots; };     // whole numbers below 2^24
            // total / slots steps may do; total / (slots - B), rounded up generously, always does
            const float total = wave_sum((float)steps);
            int c = max((int)(total / (float)slots), 1), least = c;
            if (!enough(c)) {
                c = (int)(total / (float)(slots - B) * 1.0001f) + 2;
#pragma unroll 1
                while (c - least > max(least / 32, 1)) {
                    const int mid = least + (c - least) / 2;
                    if (enough(mid)) c = mid; else least = mid;
                }
            }
            const int n = counts(c), upto = (int)wave_inclusive_scan((uint32_t)n);
            const uint64_t behind = __ballot(upto > slot);
            b = 0;
            if (behind == 0) {
                idle = true;
                return;
            }
            b = __builtin_ctzll(behind);
            n_slots = __builtin_amdgcn_readlane(n, b);
            first_slot = __builtin_amdgcn_readlane(upto, b) - n_slots;
            len = __builtin_amdgcn_readlane(tokens, b);
            per = (int64_t)__builtin_amdgcn_readfirstlane(c) * unit;
        }
        const int64_t at = (slot - first_slot) * per;
        begin = (int)min(at, (int64_t)len);
        end = (int)min(at + per, (int64_t)len);
    }
    // what the fold has to know of the sequence
    __device__ __forceinline__ void tell(const TreeArgs &a) const {
        if (a.n_splits > 1 && slot == first_slot && threadIdx.x == 0) {
            a.seq_slots[2 * b] = first_slot;
            a.seq_slots[2 * b + 1] = n_slots;
        }
    }
};

// Where a row's partial of a slot lies: the rows of a KV head of a slot are consecutive.
__device__ __forceinline__ int64_t partial_row(const TreeArgs &a, int slot, int kvh, int row) {
    return ((int64_t)slot * a.sh.n_kv_heads + kvh) * (a.n_q * a.sh.group) + row;
}

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
