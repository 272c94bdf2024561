// What the kernels of packed chunks share (chunk_kernels.hip: bf16, chunk_f32_kernels.hip: fp32): how the work is cut, which
// tokens a row sees, how a score becomes what the softmax runs over.
#pragma once

#include "tree_device.hpp"

namespace hgca {

namespace {

constexpr int kChunkStep = kStepTokens;          // tokens of a step
constexpr int kChunkWaves = kTreeWaves, kChunkBlock = kTreeBlock;
static_assert(kChunkRows == 32 * kChunkWaves, "32 rows per wave");

// true where a lane has it, uniform over the wave
__device__ __forceinline__ bool any_lane(bool x) { return __builtin_amdgcn_ballot_w64(x) != 0; }

__device__ __forceinline__ int wave_min_int(int v) {
#pragma unroll
    for (int step = kWave / 2; step > 0; step /= 2) v = min(v, __shfl_xor(v, step));
    return v;
}
__device__ __forceinline__ int wave_max_int(int v) {
#pragma unroll
    for (int step = kWave / 2; step > 0; step /= 2) v = max(v, __shfl_xor(v, step));
    return v;
}

// a value that all lanes have, in a scalar register
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// ---- the cut ----
// A sequence of n tokens has u = ceil(n * group / kChunkRows) units, each over at most `steps` steps of its tokens.  Units are cut into shares
// of at most C steps: s = ceil(steps / C) each.  C is at least a.least, or all steps where they are no more than a.whole, and the least with which there are no more shares than the
// `target` that runs at once; where there are more units than that, the steps of all units over the target.  So there are at
// most target + (number of units) shares, and at most 2 target in units that have several.  One long sequence among many short ones, a
// prompt among single tokens: a share is as long as any other.  Up to 64 sequences every wave works it out for itself, a lane per
// sequence, from the lengths on the device; more are worked out by a launch before.

constexpr int kFewTile = 16;                     // rows that are worked on straight from memory (chunk_few.hpp)

struct SeqWork {
    int n0, nq, len, pre;                        // first row of q, rows, tokens, tokens that all rows see
    int units, steps;
    __device__ __forceinline__ SeqWork(const ChunkArgs &a, int b) {
        n0 = min(max(a.cu[b], 0), a.n_tokens);
        nq = min(max(a.cu[b + 1], n0), a.n_tokens) - n0;
        len = tier_len(a.kv, b);
        pre = a.prefix ? min(max(a.prefix[b], 0), len) : 0;
        units = (int)(((int64_t)nq * a.sh.group + kChunkRows - 1) / kChunkRows);
        int64_t tokens = len;                    // that a unit's rows may see
        if (a.causal) tokens = min(tokens, (int64_t)a.window + kChunkRows / a.sh.group + pre + 3 * kChunkStep);
        steps = max((int)((tokens + kChunkStep - 1) / kChunkStep), 1);
    }
    // Its shares come before those of sequences with a few rows: these take less time, and fill what the last ones of a round leave.
    __device__ __forceinline__ bool whole_units(const ChunkArgs &a) const { return (int64_t)nq * a.sh.group > kFewTile; }
    // all lanes have the same: the compiler is told so, and keeps them, and what follows from them, in scalar registers
    __device__ __forceinline__ void unify() {
        for (int *x : {&n0, &nq, &len, &pre, &units, &steps}) *x = __builtin_amdgcn_readfirstlane(*x);
    }
};

// C, for sums over the sequences of units and of units * steps, the longest steps, and shares(c), the number of shares of at most c steps (saturated, fp32)
template <typename Shares> __device__ __forceinline__ int share_steps(const ChunkArgs &a, float units, float work, int longest, Shares shares) {
    const float target = (float)a.target;
    if (longest <= a.whole) return max(longest, 1);
    // Half a round of units with most of their rows: in two shares each they would leave a whole round's partials, 33 MB in bf16, which takes as long as
    // eight steps do (a prompt of 1024 tokens 46.7 -> 39.0 us; 32 x 4 tokens over 1000, of 32 rows, 35.6 : 41.5).
    const float rows = (float)min(max(a.cu[a.sh.batch], 0), a.n_tokens) * (float)a.sh.group;
    if (longest <= 2 * a.whole && 2.f * units >= target && rows >= (float)(kChunkRows / 2) * units) return longest;
    int c = max((int)(work / target), a.least);
    if (units > target) return max((int)fminf(work / target * 1.0001f, (float)longest) + 1, a.least);
    if (c >= longest || shares(c) <= target) return c;
    // shares(c) <= work / c + units, and one share each is few enough
    int enough = units < target ? (int)min(work / (target - units) * 1.0001f + 1.f, (float)longest) : longest;
#pragma unroll 1
    while (enough - c > max(c / 32, 1)) {
        const int mid = c + (enough - c) / 2;
        if (shares(mid) <= target) enough = mid; else c = mid;
    }
    return max(enough, a.least);
}
// 0 for a sequence without new tokens
__device__ __forceinline__ int shares_of(const SeqWork &q, int c) { return q.units > 0 ? (q.steps + c - 1) / c : 0; }

// The entry of an ascending list at[0 .. n] with at[i] <= x < at[i + 1], by the lanes of a wave; -1: x >= at[n].
__device__ __forceinline__ int wave_search(const int32_t *at, int n, int x) {
    if (x >= at[n]) return -1;
    const int lane = threadIdx.x % kWave;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + kWave - 1) / kWave, i = lo + lane * step;
        const int up = __popcll(__ballot(i < hi && at[min(i, n)] <= x));         // lane 0 is one of them
        lo += (up - 1) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// A share of a unit, or (fold) a unit that has several.
struct Place {
    int b, unit, share, n_shares, part;          // part: where the unit's partials begin
    bool idle;
    // by slot of the launch, or, with FOLD, by number among the units with several shares
    template <bool FOLD> __device__ __forceinline__ void find(const ChunkArgs &a, int x) {
        const int B = a.sh.batch, lane = threadIdx.x % kWave;
        int inside, units;
        idle = true;
        if (B <= kWave) {
            units = n_shares = 0;
            int steps = 0;
            bool whole = false;
            if (lane < B) {
                const SeqWork q(a, lane);
                whole = q.whole_units(a);
                units = q.units;
                steps = units > 0 ? q.steps : 0;
            }
            const int c = share_steps(a, wave_sum((float)units), wave_sum((float)units * (float)steps), wave_max_int(steps),
                                      [&](int c) { return wave_sum((float)units * (float)((steps + c - 1) / c)); });
            const int shares = units > 0 ? (steps + c - 1) / c : 0, slots = units * shares, several = shares > 1 ? slots : 0;
            const int parts = (int)wave_inclusive_scan((uint32_t)several) - several;
            int mine = FOLD ? (shares > 1 ? units : 0) : whole ? slots : 0, upto = (int)wave_inclusive_scan((uint32_t)mine);
            const int before = __builtin_amdgcn_readlane(upto, kWave - 1);
            if (!FOLD && x >= before) {          // uniform over the wave
                mine = whole ? 0 : slots;
                upto = before + (int)wave_inclusive_scan((uint32_t)mine);
            }
            const uint64_t behind = __ballot(upto > x && mine > 0);
            if (behind == 0) return;
            b = __builtin_ctzll(behind);
            inside = x - (__builtin_amdgcn_readlane(upto, b) - __builtin_amdgcn_readlane(mine, b));
            units = __builtin_amdgcn_readlane(units, b);
            n_shares = __builtin_amdgcn_readlane(shares, b);
            part = __builtin_amdgcn_readlane(parts, b);
        } else {
            const int32_t *const slots = a.cut + 1, *const parts = slots + B + 1, *const several = parts + B + 1, *const later = several + B + 1;
            const int32_t *list = FOLD ? several : slots;
            if (!FOLD && x >= slots[B]) {
                x -= slots[B];
                list = later;
            }
            b = wave_search(list, B, x);
            if (b < 0) return;
            inside = x - list[b];
            const SeqWork q(a, b);
            units = q.units;
            n_shares = shares_of(q, a.cut[0]);
            part = parts[b];
        }
        b = __builtin_amdgcn_readfirstlane(b);
        inside = __builtin_amdgcn_readfirstlane(inside);
        units = __builtin_amdgcn_readfirstlane(units);
        n_shares = __builtin_amdgcn_readfirstlane(n_shares);
        part = __builtin_amdgcn_readfirstlane(part);
        // the units of a share run side by side (they read the same tokens), those that see most first
        share = FOLD ? 0 : inside / units;
        unit = FOLD ? inside : units - 1 - inside % units;
        part += unit * n_shares;
        // (a list of beginnings that does not ascend can ask for more than there is)
        idle = n_shares > 1 && (int64_t)part + n_shares > a.parts;
    }
};

// ---- what a row sees ----
struct RowSees {
    int lo, hi, pre;                             // tokens [0, pre) and [lo, hi)
    RowSees() = default;
    __device__ __forceinline__ RowSees(const ChunkArgs &a, const SeqWork &q, int query) {
        const int p = q.len - q.nq + query;
        pre = q.pre;
        hi = a.causal ? min(p + 1, q.len) : q.len;
        lo = a.window == INT32_MAX ? 0 : max(p - a.window + 1, 0);
        if (a.first) lo = max(lo, a.first[q.n0 + query]);
    }
    // of the 64 tokens from `base` on
    __device__ __forceinline__ uint64_t mask(int base) const {
        auto below = [&](int x) {
            const int n = x - base;
            return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1;
        };
        return below(pre) | (below(hi) & ~below(lo));
    }
};

// What the rows of a wave see together: everything in [0, pre) and [all_lo, all_hi), nothing outside [0, pre) and [any_lo, any_hi).
struct WaveSees {
    int pre, all_lo, all_hi, any_lo, any_hi;
    template <int N> __device__ __forceinline__ explicit WaveSees(const RowSees (&rows)[N]) {     // a lane's N rows
        pre = rows[0].pre;
        all_lo = 0, all_hi = INT32_MAX, any_lo = INT32_MAX, any_hi = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            all_lo = max(all_lo, rows[i].lo);
            all_hi = min(all_hi, rows[i].hi);
            if (rows[i].hi > rows[i].lo) {
                any_lo = min(any_lo, rows[i].lo);
                any_hi = max(any_hi, rows[i].hi);
            }
        }
        all_lo = __builtin_amdgcn_readfirstlane(wave_max_int(all_lo));
        all_hi = __builtin_amdgcn_readfirstlane(wave_min_int(all_hi));
        any_lo = __builtin_amdgcn_readfirstlane(wave_min_int(any_lo));
        any_hi = __builtin_amdgcn_readfirstlane(wave_max_int(any_hi));
    }
    __device__ __forceinline__ bool all(int t, int n) const { return t + n <= pre || (t >= all_lo && t + n <= all_hi); }
    __device__ __forceinline__ bool none(int t, int n) const { return t >= pre && (t >= any_hi || t + n <= any_lo); }
};

// The steps of a share: those of the prefix and those from the first token that a row of the unit sees to the last.
struct Steps {
    int begin0, end0, begin1, end1;
    __device__ __forceinline__ Steps(int pre, int lo, int hi, int share, int n_shares) {
        int head = (pre + kChunkStep - 1) / kChunkStep, from = 0, to = 0;
        if (hi > lo) {
            from = lo / kChunkStep;
            to = (hi + kChunkStep - 1) / kChunkStep;
        }
        if (from <= head) {                      // one run
            head = max(head, to);
            from = to = head;
        }
        const int total = head + (to - from), per = (total + n_shares - 1) / n_shares;
        const int i0 = min(share * per, total), i1 = min(i0 + per, total);
        begin0 = min(i0, head);
        end0 = min(i1, head);
        begin1 = from + max(i0 - head, 0);
        end1 = from + max(i1 - head, 0);
    }
    __device__ __forceinline__ int begin(int range) const { return range ? begin1 : begin0; }
    __device__ __forceinline__ int end(int range) const { return range ? end1 : end0; }
};

// ---- where the tokens lie ----
// A wave keeps the rows of 64 granules of 16 tokens in a register, a lane each, and requests the next 64 when it comes to them: a step's
// rows are then read off by number, with no round trip to LDS or memory before its loads.  (Blocks are whole granules.)
struct GranuleRows {
    const int32_t *blocks;                       // the sequence's table row, or null: contiguous
    uint32_t head;                               // first row of the KV head, of a block's heads if paged
    int bs, heads, last;                         // last: granule of the sequence's last token
    int base;
    uint32_t now, next;                          // of granules base + lane and base + 64 + lane
    __device__ __forceinline__ GranuleRows(const ChunkArgs &a, int b, int kvh, int len) {
        blocks = a.kv.block_table ? a.kv.block_table + (int64_t)b * a.kv.max_blocks + (a.kv.first_block ? a.kv.first_block[b] : 0) : nullptr;
        head = a.kv.block_table ? (uint32_t)kvh : (uint32_t)(((int64_t)b * a.sh.n_kv_heads + kvh) * a.kv.cap);
        bs = a.kv.block_size;
        heads = a.sh.n_kv_heads;
        last = max(len - 1, 0) / kGranule;
        base = 0;
        now = next = 0;
    }
    __device__ __forceinline__ uint32_t fetch(int first) const {
        const int g = min(first + (int)(threadIdx.x % kWave), last), tok = g * kGranule;
        if (!blocks) return head + (uint32_t)tok;
        const int blk = tok / bs;
        return ((uint32_t)blocks[blk] * (uint32_t)heads + head) * (uint32_t)bs + (uint32_t)(tok - blk * bs);
    }
    __device__ __forceinline__ void start(int granule) {
        base = granule;
        now = fetch(base);
        next = fetch(base + kWave);
    }
    // granules up to `granule` + 3 are to be had; called with ascending ones, by whole waves
    __device__ __forceinline__ void reach(int granule) {
        if (granule + 3 < base + kWave) return;
        base += kWave;
        now = next;
        next = fetch(base + kWave);
    }
    __device__ __forceinline__ uint32_t row(int granule) const { return __builtin_amdgcn_readlane(now, granule - base); }
};

// ---- scores ----
// kPlainScores: the softmax runs over the product, times sm_scale log2 e in the exponent of 2.  kCapped: cap tanh(product * sm_scale / cap), in
// units of ln 2.  kBiased: the product less slope / sm_scale * distance, kCapped + kBiased: the capped score less slope * distance.
enum { kPlainScores = 0, kCapped = 1, kBiased = 2 };

// tanh x.  Up to kTanhNear it is x P(x^2), P fitted to the least largest relative error (3.1e-7 of degree 4, 2.7e-8 of degree 5); beyond, 1 - 2 / (1 +
// e^2x), whose rounding is then small against the result.  The factors before and behind are in P's coefficients: six instructions a
// score.  (Four more for the other form, two of them slow; steps in which no score is beyond are the rule.)  The last coefficient has the tenth power
// of sm_scale / cap: where it would leave the range of ordinary numbers (heads of 128, scale 1 / sqrt(d): caps above 260 and below 2e-5) the factors
// stay outside.  The one behind P is then the score's own, in * out as one number, so that no cap is too large: P is 1 where the cap does nothing.
constexpr float kTanhNear = 0.7f;
template <bool FINE> struct TanhNear {
    static constexpr int kTerms = FINE ? 6 : 5;
    float a[kTerms];
    float before, behind;                        // 1 where they are in the coefficients
    __device__ __forceinline__ TanhNear() {}
    __device__ __forceinline__ TanhNear(float in, float in_out) {        // of in_out / in * tanh(in * x)
        constexpr float kFine[6] = {1.f, -0.33333131671f, 0.13328415155f, -0.05352601036f, 0.02002445795f, -0.00508833630f};
        constexpr float kCoarse[6] = {0.99999970198f, -0.33330214024f, 0.13281112909f, -0.05083623528f, 0.01377371047f, 0.f};
        float power = in_out;
#pragma unroll
        for (int i = 0; i < kTerms; ++i) {
            a[i] = (FINE ? kFine[i] : kCoarse[i]) * power;
            power *= in * in;
        }
        // they are a geometric series but for factors around 1: the first and the last say for all
        auto ordinary = [](float x) { return fabsf(x) >= 1.2e-38f && fabsf(x) <= 1e37f; };
        const bool folded = ordinary(a[0]) && ordinary(a[kTerms - 1]);
#pragma unroll
        for (int i = 0; i < kTerms; ++i) a[i] = uniform(folded ? a[i] : FINE ? kFine[i] : kCoarse[i]);
        before = uniform(folded ? 1.f : in);
        behind = uniform(folded ? 1.f : in_out);
    }
    __device__ __forceinline__ bool folded() const { return before == 1.f && behind == 1.f; }
    __device__ __forceinline__ float polynomial(float z) const {
        float p = a[kTerms - 1];
#pragma unroll
        for (int i = kTerms - 2; i >= 0; --i) p = fmaf(z, p, a[i]);
        return p;
    }
    // folded() only; the same number as operator()
    __device__ __forceinline__ float quick(float x) const { return x * polynomial(x * x); }
    __device__ __forceinline__ float operator()(float x) const {
        const float t = x * before;
        return x * behind * polynomial(t * t);
    }
};
__device__ __forceinline__ float tanh_far(float x) {
    return copysignf(fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(2.f * kTreeLog2e * fabsf(x))), 1.f), x);
}

template <int MODE, bool FINE> struct ScoreMap {
    static constexpr bool kCaps = (MODE & kCapped) != 0, kBiases = (MODE & kBiased) != 0;
    float k2;                                    // a weight is 2^(k2 * (what apply leaves) - its maximum's)
    float kx, scale2, cap2, slope2;
    TanhNear<FINE> near_zero;
    static __device__ __forceinline__ float slope_of(const ChunkArgs &a, int head) {
        return kBiases ? a.slopes[head] * (kCaps ? kTreeLog2e : 1.f / a.sh.sm_scale) : 0.f;
    }
    // (slope2 is the row's: set, where there are several)
    __device__ __forceinline__ ScoreMap(const ChunkArgs &a, int head) : ScoreMap(a) { slope2 = slope_of(a, head); }
    __device__ __forceinline__ explicit ScoreMap(const ChunkArgs &a) {
        slope2 = 0.f;
        scale2 = uniform(a.sh.sm_scale * kTreeLog2e);
        kx = kCaps ? uniform(a.sh.sm_scale / a.cap) : 0.f;
        cap2 = uniform(a.cap * kTreeLog2e);
        k2 = kCaps ? 1.f : scale2;
        if (kCaps) near_zero = TanhNear<FINE>(kx, scale2);
    }
    // The N values of a lane, get(i) and set(i, x): products with tokens first + off(i) of a row at position pos.
    template <int N, typename Get, typename Set, typename Off>
    __device__ __forceinline__ void each(Get get, Set set, Off off, int pos, int first) const {
        if constexpr (MODE == kPlainScores) return;
        const float d = (float)(pos - first);
        auto biased = [&](float x, int i) { return kBiases ? fmaf(-slope2, fabsf(d - (float)off(i)), x) : x; };
        if constexpr (!kCaps) {
#pragma unroll
            for (int i = 0; i < N; ++i) set(i, biased(get(i), i));
            return;
        } else {
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(get(i)));
            if (near_zero.folded() && !any_lane(!(most * kx <= kTanhNear))) {        // uniform over the wave
#pragma unroll
                for (int i = 0; i < N; ++i) set(i, biased(near_zero.quick(get(i)), i));
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float x = get(i) * kx;
                    set(i, biased(fabsf(x) <= kTanhNear ? near_zero(get(i)) : cap2 * tanh_far(x), i));
                }
            }
        }
    }
    // c[t][r]: token first + 32 t + 8 (r / 4) + r % 4
    template <int NT> __device__ __forceinline__ void apply(floatx16 (&c)[NT], int pos, int first) const {
        each<16 * NT>([&](int i) { return c[i / 16][i % 16]; }, [&](int i, float x) { c[i / 16][i % 16] = x; },
                      [](int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4; }, pos, first);
    }
};

// ---- infinities and NaN of V ----
// A weight of 0 does not keep such a value out of a matrix product, and a weight, or a factor between shares, may be 0 for a row that does
// see it.  Steps that some row of a wave does not see all of have them taken out of the operand; a workgroup that has taken some out, or whose
// sums are not finite, goes through its steps of V once more, 64 tokens at a time, and notes which columns of which tokens hold which kind.
template <int D> struct OddTokens {
    unsigned long long bits[3][D];               // by kind (+inf, -inf, NaN) and column: bit j = the step's token j holds one
    template <typename T>
    __device__ void note(const ChunkArgs &a, int b, int kvh, int first, int end) {
        constexpr int kPer = Elem<T>::kPerLoad, kPieces = D / kPer;
        __syncthreads();                         // the last step's notes have been read
        for (int i = threadIdx.x; i < 3 * D; i += kChunkBlock) (&bits[0][0])[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < kChunkStep * kPieces; i += kChunkBlock) {
            const int j = i / kPieces, piece = i % kPieces, tok = first + j;
            if (tok >= end) continue;
            int64_t row;
            if (a.kv.block_table) {
                const int32_t *const blocks = a.kv.block_table + (int64_t)b * a.kv.max_blocks + (a.kv.first_block ? a.kv.first_block[b] : 0);
                row = ((int64_t)blocks[tok / a.kv.block_size] * a.sh.n_kv_heads + kvh) * a.kv.block_size + tok % a.kv.block_size;
            } else {
                row = ((int64_t)b * a.sh.n_kv_heads + kvh) * a.kv.cap + tok;
            }
            float x[kPer];
            Elem<T>::expand(load16(a.kv.v + row * (int64_t)(D * sizeof(T)) + 16 * piece), x);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                if (fabsf(x[e]) < INFINITY) continue;
                const int kind = x[e] == INFINITY ? 0 : x[e] == -INFINITY ? 1 : 2;
                atomicOr(&bits[kind][piece * kPer + e], 1ull << j);
            }
        }
        __syncthreads();
    }
};

// A row's sums after the loop: acc[dt][r] is column 32 dt + 8 (r / 4) + 4 hw + r % 4 of the lane's row.  Brings in what the values that the row
// sees make of them, if any wave of the workgroup has met one.  All threads of the workgroup take part; s_odd and notes are LDS of its
// own.
template <typename T, int D>
__device__ void settle_odd(const ChunkArgs &a, int b, int kvh, const RowSees &sees, const Steps &steps, int len, bool met, int (&s_odd)[kChunkWaves],
                           OddTokens<D> &notes, floatx16 (&acc)[D / 32]) {
    constexpr int DT = D / 32;
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave, hw = lane / 32;
    float z[4] = {0.f, 0.f, 0.f, 0.f};           // NaN where a sum is not finite
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r % 4] = fmaf(acc[dt][r], 0.f, z[r % 4]);
    const float all = (z[0] + z[1]) + (z[2] + z[3]);
    met = any_lane(all != all) || met;
    if (lane == 0) s_odd[w] = met;
    __syncthreads();
    bool any = false;
#pragma unroll
    for (int i = 0; i < kChunkWaves; ++i) any = any || s_odd[i];
    if (!any) return;                            // uniform over the workgroup
    uint64_t kinds[3] = {0, 0, 0};               // a bit per element of acc
    for (int part = 0; part < 2; ++part)
        for (int s = steps.begin(part); s < steps.end(part); ++s) {
            const int first = s * kChunkStep;
            notes.template note<T>(a, b, kvh, first, len);
            const uint64_t seen = sees.mask(first);
#pragma unroll 1
            for (int k = 0; k < 3; ++k) {
                uint64_t got = 0;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (notes.bits[k][32 * dt + 8 * (r / 4) + 4 * hw + r % 4] & seen) got |= 1ull << (16 * dt + r);
                kinds[0] |= k == 0 ? got : 0;
                kinds[1] |= k == 1 ? got : 0;
                kinds[2] |= k == 2 ? got : 0;
            }
        }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int i = 16 * dt + r;
            const bool up = kinds[0] >> i & 1, down = kinds[1] >> i & 1, none = kinds[2] >> i & 1;
            acc[dt][r] = none || (up && down) ? NAN : up ? INFINITY : down ? -INFINITY : acc[dt][r];
        }
}

// Where a lane's row of a unit lies.
struct RowPlace {
    bool live;                                   // else the lane repeats the unit's last row and stores nothing
    int query, head, row;                        // query of the sequence, head of the tensors, row of the unit
    int64_t out;                                 // row of q, o and lse
    __device__ __forceinline__ RowPlace(const ChunkArgs &a, const SeqWork &q, int unit, int kvh, int r) {
        const int lg = __builtin_ctz(a.sh.group);
        const int64_t i = (int64_t)unit * kChunkRows + r, rows = (int64_t)q.nq << lg;
        live = i < rows;
        const int64_t mine = live ? i : rows - 1;
        row = r;
        query = (int)(mine >> lg);
        head = kvh * a.sh.group + (int)(mine & (a.sh.group - 1));
        out = (int64_t)(q.n0 + query) * a.sh.n_q_heads + head;
    }
};

// The unit's first and last seen token outside the prefix, over all its rows: s_range is LDS, cleared here.  lo and hi ascend with the row
// but for `first`.
__device__ __forceinline__ void unit_range(const WaveSees &w, int (&s_range)[2], int &lo, int &hi) {
    if (threadIdx.x == 0) {
        s_range[0] = INT32_MAX;
        s_range[1] = 0;
    }
    __syncthreads();
    if (threadIdx.x % kWave == 0) {
        atomicMin(&s_range[0], w.any_lo);
        atomicMax(&s_range[1], w.any_hi);
    }
    __syncthreads();
    lo = __builtin_amdgcn_readfirstlane(s_range[0]);
    hi = __builtin_amdgcn_readfirstlane(s_range[1]);
}

// A row's result, or its share's partial: l over all tokens of the share, sums relative to 2^-shift.
template <int D>
__device__ __forceinline__ void store_row(const ChunkArgs &a, const Place &at, int kvh, const RowPlace &rp, float l, float shift,
                                          const floatx16 (&acc)[D / 32]) {
    if (!rp.live) return;
    const int hw = threadIdx.x % kWave / 32;
    auto each = [&](auto store) {                // four adjacent columns at a time
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const floatx16 &x = acc[dt];
                store(32 * dt + 8 * q4 + 4 * hw, make_float4(x[4 * q4], x[4 * q4 + 1], x[4 * q4 + 2], x[4 * q4 + 3]));
            }
    };
    if (at.n_shares > 1) {                       // uniform over the workgroup
        const int64_t to = ((int64_t)(at.part + at.share) * a.sh.n_kv_heads + kvh) * kChunkRows + rp.row;
        float *const o = a.part_o + to * D;
        each([&](int col, const float4 &x) { *reinterpret_cast<float4 *>(o + col) = x; });
        if (hw == 0) {
            a.part_m[to] = l == 0.f ? -INFINITY : -shift;
            a.part_l[to] = l;
        }
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    auto result = [&](const float4 &x) {         // (sums of a row that sees nothing are 0)
        return make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    };
    if (a.o_bf16) {
        char *const o = static_cast<char *>(a.o) + 2 * rp.out * D;
        each([&](int col, const float4 &x) {
            const float4 y = result(x);
            *reinterpret_cast<uint2 *>(o + 2 * col) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
        });
    } else {
        float *const o = static_cast<float *>(a.o) + rp.out * D;
        each([&](int col, const float4 &x) { *reinterpret_cast<float4 *>(o + col) = result(x); });
    }
    if (hw == 0) a.lse[rp.out] = l == 0.f ? -INFINITY : (__builtin_amdgcn_logf(l) - shift) * kLn2;
}

// The running maximum, sum and rescaling of a row over a step's scores (as left by ScoreMap): returns the shift of a weight 2^(k2 c + shift).
template <int DT> struct Running {
    float m = -INFINITY, shift = 0.f, l = 0.f;   // shift: 0 for far rows (shift_of); l: over this lane's tokens
    bool far = false;                            // uniform over the wave: a row of it is
    template <int NT> __device__ __forceinline__ void update(floatx16 (&c)[NT], float k2, floatx16 (&acc)[DT]) {
        float mx = c[0][0];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, c[t][r]);
        if (any_lane(mx > m)) {                     // uniform over the wave
            const float m_new = fmaxf(m, halves_max(mx)), to = shift_of(m_new, k2), corr = rescale_factor(m, m_new, k2);
            m = m_new;
            shift = is_far(to) ? 0.f : to;
            far = any_lane(is_far(to));
            l *= corr;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) acc[dt] *= corr;
        }
        if (far) {
            const float less = is_far(shift_of(m, k2)) ? m : 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t) c[t] -= less;
        }
    }
};

}  // namespace

}  // namespace hgca
