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

// What a row's weights are relative to, for a maximum m of its raw scores: 2^-shift_of, as rounded, so that a weight 2^fma(score, scale2,
// shift) has none of the rounding in it.  From 2^30 on the rounding is tens of powers of two and a weight would leave fp32: there scores
// have their maximum subtracted first, and a weight is 2^((score - m) scale2).  (Two such scores are 2^64 apart in weight or equal.)
constexpr float kFarShift = 1073741824.f, kLargest = 3.40282347e38f;
__device__ __forceinline__ float shift_of(float m, float scale2) {
    return m == -INFINITY ? 0.f : __builtin_amdgcn_fmed3f(-m * scale2, -kLargest, kLargest);
}
__device__ __forceinline__ bool is_far(float shift) { return fabsf(shift) >= kFarShift; }
// the factor that takes sums relative to one maximum to another, at least as large; 1 where they are equal
__device__ __forceinline__ float rescale_factor(float m, float m_new, float scale2) {
    const float from = shift_of(m, scale2), to = shift_of(m_new, scale2);
    return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(is_far(from) || is_far(to) ? (m - m_new) * scale2 : to - from);
}

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

// Infinities and NaN of the V rows that a row sees.  A weight enters a product in parts that may be negative or 0, and a weight or a
// factor between shares may be 0 in fp32, so such a value times them says nothing: where a sum is not finite, or an odd value of a
// drafted row has been taken out of an operand, the workgroup goes through its share of V once more and notes which kinds a column has
// among the tokens before the drafts, and in which drafted ones.  With an infinity in every share 64 drafts x 4 over 32 K tokens take
// 414 -> 731 us, 32 drafts x 8 over 4 K 51 -> 78.
template <int D> struct OddSeen {
    unsigned long long drafted[3][D];            // by kind (+inf, -inf, NaN) and column: bit j = draft j has one
    uint32_t before[D];                          // bit k = a token before the drafts has kind k
    // Tokens begin .. end - 1 of V; contains barriers.
    template <typename T, int BLOCK>
    __device__ void collect(uint32_t *s_row, const TreeArgs &a, int b, int kvh, int begin, int end, int tail) {
        constexpr int kPer = Elem<T>::kPerLoad, kPieces = D / kPer;              // elements of 16 bytes, such pieces of a row
        for (int i = threadIdx.x; i < D; i += BLOCK) {
            before[i] = 0;
            drafted[0][i] = drafted[1][i] = drafted[2][i] = 0;
        }
        const int total = end - begin, sub_len = pass_length(a.kv, total), piece = threadIdx.x % kPieces;
        for (int sub0 = 0; sub0 < total; sub0 += sub_len) {
            const int nsub = min(sub_len, total - sub0), first = begin + sub0;
            __syncthreads();                     // the table is no longer in use; the notes are cleared
            const BlockRows where = make_block_rows<BLOCK>(s_row, a.kv, a.sh.n_kv_heads, b, kvh, first, nsub);
#pragma unroll 4
            for (int tok = threadIdx.x / kPieces; tok < nsub; tok += BLOCK / kPieces) {
                const uint32_t row = where.table ? where.table[tok / kGranule] + tok % kGranule : where.base + tok;
                float x[kPer];
                Elem<T>::expand(load16(a.kv.v + (size_t)row * (D * sizeof(T)) + 16 * piece), x);
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    if (fabsf(x[i]) < INFINITY) continue;
                    const int kind = x[i] == INFINITY ? 0 : x[i] == -INFINITY ? 1 : 2, col = piece * kPer + i, j = first + tok - tail;
                    if (j < 0) atomicOr(&before[col], 1u << kind);
                    else atomicOr(&drafted[kind][col], 1ull << j);
                }
            }
        }
        __syncthreads();
    }
    // a column's sum of a row with this mask: what the values that it sees make of it
    __device__ __forceinline__ float result(int col, uint64_t mask, float x) const {
        uint32_t kinds = before[col];
#pragma unroll
        for (int k = 0; k < 3; ++k) kinds |= drafted[k][col] & mask ? 1u << k : 0u;
        return kinds == 0 ? x : kinds == 1 ? INFINITY : kinds == 2 ? -INFINITY : NAN;
    }
};

}  // namespace

}  // namespace hgca
