// Drafted tokens accepted or refused by the target's probabilities p, the draft model's q and given random numbers, and the token that
// follows the accepted ones.
//
// At a node of the tree its children x are tried in order: x is accepted if u q(x) < p'(x), p' = p at first; if it is refused p'
// becomes max(p' - q, 0), divided by its sum.  Dividing the k-th of these out, p' is max(p - c q, 0) / S(c) with S(c) its sum: c = 0
// and S = 1 before the first refusal, c becomes c + S(c) with each.  So what a node's refusals have left of the target is one number, a
// test is two elements of the rows, u q(x) S < max(p(x) - c q(x), 0), and only a refusal asks for a pass over the rows.  Without q (the
// draft model was sure) q is 1 at x: p' is p without the refused tokens, S the sum over the rest.  Where the walk ends one more
// token is drawn from p': the first at which the running sum passes u_next times the whole.
//
// Sums are fp64: the order of additions is then in no result that a plain running sum would not give as well but once in some 10^10 draws, and
// the pass is bound by memory all the same.
//
// A pass reads two rows of the vocabulary for each sequence, and that and the latency of one dependent load after the other bound it: parents and
// tokens, elements of the rows, the rows.  So short rows are one workgroup's, two segments a wave, in one launch; for longer ones every workgroup
// of a launch over the chip finds for itself where the walk first stops (single elements), and leaves the sums of its segments; launches like it
// follow for trees with long rows, in which other refusals come next, and a last one, a workgroup per sequence, goes through what is
// left and draws, for which it reads one more segment.  Measured in a captured graph: 8 x 5 tokens, 32 000 elements,
// fp32, 10.9 us, 32 trees of 16 over 128 000 28.3 (33 MB a pass; 46.7 with one launch before the last), over 128 003, whose rows are of all
// alignments, 30.1.  Of a pass's arithmetic the conversions to fp64 take most, 56 cycles an element and wave in all.
#include <algorithm>

#include "hgca_launch.hpp"

namespace hgca {

namespace {

constexpr int kSumBlock = 256, kSumWaves = kSumBlock / kWave;
constexpr int kWalkBlock = 1024, kWalkWaves = kWalkBlock / kWave;

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int step = kWave / 2; step > 0; step /= 2) v += __shfl_xor(v, step);
    return v;
}

__device__ __forceinline__ double wave_scan64(double v) {
#pragma unroll
    for (int step = 1; step < kWave; step *= 2) {
        const double o = __shfl_up(v, step);
        if ((int)threadIdx.x % kWave >= step) v += o;
    }
    return v;
}

// A probability as it counts: what is negative, infinite or NaN is 0.
__device__ __forceinline__ float sane(float x) { return __float_as_uint(x) < 0x7f800000u ? x : 0.f; }

template <typename T> __device__ __forceinline__ float element(const char *row, int i);
template <> __device__ __forceinline__ float element<float>(const char *row, int i) { return sane(reinterpret_cast<const float *>(row)[i]); }
template <> __device__ __forceinline__ float element<bf16_t>(const char *row, int i) {
    return sane(__uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(row)[i] << 16));
}

// What is known of every drafted token before the walk, a lane each (there are at most 64).
struct Nodes {
    int parent, token;                           // parent -1: not in the tree
    float u, p, q;                               // p, q: of the token in its parent's rows
    template <typename T> __device__ __forceinline__ void load(const VerifyArgs &a, int b) {
        const int j = threadIdx.x % kWave;
        parent = -1;
        token = 0;
        u = p = q = 0.f;
        if (j < 1 || j >= a.n) return;
        const int64_t at = (int64_t)b * a.n + j;
        const int up = a.parents ? a.parents[at] : j - 1, x = a.tokens[at];
        if (up < 0 || up >= j || x < 0 || x >= a.vocab) return;
        parent = up;
        token = x;
        u = a.u[at];
        p = element<T>(target_row(a, b, up, sizeof(T)), x);
        q = a.draft ? element<T>(draft_row(a, b, up, sizeof(T)), x) : 1.f;
    }
    static __device__ __forceinline__ const char *target_row(const VerifyArgs &a, int b, int node, int e) {
        return a.target + (b * a.target_seq + node * a.target_row) * e;
    }
    static __device__ __forceinline__ const char *draft_row(const VerifyArgs &a, int b, int node, int e) {
        return a.draft + (b * a.draft_seq + node * a.draft_row) * e;
    }
    // children of `node` behind drafted token j, a bit each
    __device__ __forceinline__ uint64_t children(int node, int j) const {
        return __ballot(parent == node) & (j >= 63 ? 0ull : ~0ull << (j + 1));
    }
};

// Where a walk stands (kept between the launches): at `node`, the drafted tokens up to `tried` have been seen to, c and mass (S) of what is left of the
// target.  path: accepted tokens, a bit each; gone: without q, the refused children of the node.
using Walk = VerifyWalk;

__device__ __forceinline__ double lane_value(float x, int lane) {
    return (double)__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane));
}

// Goes on until a refusal (true: mass is to be formed anew, for c or without the tokens of `gone`) or the end of the walk (false).
// Uniform over the wave; every wave of a workgroup does the same.
__device__ __forceinline__ bool walk_on(Walk &w, const Nodes &nodes, bool with_q) {
    while (true) {
        const uint64_t next = nodes.children(w.node, w.tried);
        if (next == 0) return false;
        const int j = __builtin_ctzll(next);
        double left = lane_value(nodes.p, j);
        if (with_q) {
            const double less = w.c * lane_value(nodes.q, j);
            left = left > less ? left - less : 0.0;
        } else {
            const int x = __builtin_amdgcn_readlane(nodes.token, j);
            if (__ballot((w.gone >> (threadIdx.x % kWave) & 1) && nodes.token == x)) left = 0.0;         // refused before
        }
        w.tried = j;
        if (lane_value(nodes.u, j) * lane_value(nodes.q, j) * w.mass < left) {
            w.node = j;
            w.c = 0.0;
            w.mass = 1.0;
            w.path |= 1ull << j;
            w.gone = 0;
            continue;
        }
        w.c += w.mass;
        w.gone |= 1ull << j;
        return true;
    }
}

// Goes on from a refusal, for which `mass` is left of the target; true: sums have to be formed for where the walk stops now, another refusal or the end at a
// node of which there are none.
__device__ __forceinline__ bool go_on(Walk &w, const Nodes &nodes, bool with_q, double mass) {
    w.mass = mass;
    w.refused = walk_on(w, nodes, with_q);
    return w.refused || w.c == 0.0;
}

// 16 bytes of a row as elements.  Rows begin where they do: an odd vocabulary's are not aligned to 16 bytes, which the loads do not ask for.
typedef uint32_t AnyPiece __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> struct Piece {
    static constexpr int kPer = Elem<T>::kPerLoad;
    uint4 raw;
    __device__ __forceinline__ void load(const char *row, int i) {
        const AnyPiece x = *reinterpret_cast<const AnyPiece *>(row + (int64_t)i * (int)sizeof(T));
        raw = make_uint4(x[0], x[1], x[2], x[3]);
    }
    __device__ __forceinline__ void expand(float *x) const { Elem<T>::expand(raw, x); }
    // below kAllSane if every element counts as it is: neither negative nor infinite or NaN
    __device__ __forceinline__ uint32_t look(uint32_t so_far) const {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            so_far = max(so_far, w[k]);
            if (sizeof(T) == 2) so_far = max(so_far, w[k] << 16);
        }
        return so_far;
    }
};
constexpr uint32_t kAllSane = 0x7f800000u;       // the bits of infinity; those of negative numbers and NaN are above

// The walk's last segment is drawn from by a whole workgroup: this many elements a lane.
constexpr int kDrawPer = kVerifySegment / kWalkBlock;

// What is left of the target at a node, by element.
template <typename T>
struct Rest {
    const char *p, *q;                           // q null: without
    double c;
    uint64_t gone;
    int vocab;
    __device__ __forceinline__ Rest(const VerifyArgs &a, int b, const Walk &w) {
        p = Nodes::target_row(a, b, w.node, sizeof(T));
        q = a.draft && w.c > 0.0 ? Nodes::draft_row(a, b, w.node, sizeof(T)) : nullptr;
        c = w.c;
        gone = a.draft ? 0 : w.gone;
        vocab = a.vocab;
    }
    __device__ __forceinline__ double one(const Nodes &nodes, int i) const {
        if (i >= vocab) return 0.0;
        return gone ? left<true>(nodes, element<T>(p, i), 0.f, i) : left<false>(nodes, element<T>(p, i), q ? element<T>(q, i) : 0.f, i);
    }
    template <bool GONE> __device__ __forceinline__ double left(const Nodes &nodes, float v, float d, int i) const {
        if constexpr (!GONE) {
            double x = fma(-c, (double)d, (double)v);
            asm("v_max_f64 %0, %0, 0" : "+v"(x));                // (the compiler's has two more for signalling NaN)
            return x;
        }
        bool out = false;
        for (uint64_t m = gone; m; m &= m - 1) out = out || i == __builtin_amdgcn_readlane(nodes.token, __builtin_ctzll(m));
        return out ? 0.0 : (double)v;
    }
    // Sum of a segment, in every lane of the wave.  All of the lane's loads are under way before the first is waited for: one load
    // after the other would take so many times memory's latency.  (Segments of 2048: 64 registers of loads, which the walk's kernel does not have,
    // 30.9 : 28.7 us for 32 trees over 128 000.)
    __device__ __forceinline__ double segment(const Nodes &nodes, int seg) const {
        return gone ? segment_of<true>(nodes, seg) : segment_of<false>(nodes, seg);
    }
    template <bool GONE> __device__ __forceinline__ double segment_of(const Nodes &nodes, int seg) const {
        constexpr int kPer = Piece<T>::kPer, kRounds = kVerifySegment / (kPer * kWave);
        const int lane = threadIdx.x % kWave, i0 = seg * kVerifySegment + kPer * lane;
        double s[4] = {0.0, 0.0, 0.0, 0.0};
        if (vocab < kPer) return wave_sum64(one(nodes, lane));
        // The last pieces of a row begin where they end with it: `skip` of their elements belong to the piece before.
        const bool whole = (seg + 1) * kVerifySegment <= vocab;  // uniform over the wave
        auto at = [&](int r) { return whole ? i0 + r * kPer * kWave : min(i0 + r * kPer * kWave, vocab - kPer); };
        Piece<T> pv[kRounds], pd[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) pv[r].load(p, at(r));
        if (q) {
#pragma unroll
            for (int r = 0; r < kRounds; ++r) pd[r].load(q, at(r));
        } else {
#pragma unroll
            for (int r = 0; r < kRounds; ++r) pd[r].raw = make_uint4(0, 0, 0, 0);
        }
        uint32_t most = 0;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) most = pd[r].look(pv[r].look(most));
        const bool all_sane = __builtin_amdgcn_ballot_w64(most >= kAllSane) == 0;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            float v[kPer], d[kPer];
            pv[r].expand(v);
            pd[r].expand(d);
            if (!(all_sane && whole)) {          // uniform over the wave
                const int skip = i0 + r * kPer * kWave - at(r);
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    v[k] = k < skip ? 0.f : sane(v[k]);
                    d[k] = sane(d[k]);
                }
            }
#pragma unroll
            for (int k = 0; k < kPer; ++k) s[k % 4] += left<GONE>(nodes, v[k], d[k], at(r) + k);
        }
        return wave_sum64((s[0] + s[1]) + (s[2] + s[3]));
    }
};

__device__ __forceinline__ int segments_of(const VerifyArgs &a) { return (a.vocab + kVerifySegment - 1) / kVerifySegment; }

// The sum over all segments' sums, by a wave, in every lane.
__device__ __forceinline__ double sum_of(const double *sums, int segs) {
    double s = 0.0;
    for (int i = threadIdx.x % kWave; i < segs; i += kWave) s += sums[i];
    return wave_sum64(s);
}

__device__ __forceinline__ double *pass_sums(const VerifyArgs &a, int b, int pass, int segs) { return a.sums + ((int64_t)pass * a.batch + b) * segs; }

// One pass of a launch: where the walk stops for the PASS-th time (at a refusal or its end) the sums of all segments of the row, a wave per segment.
// Sequences whose walk has ended before have nothing to do but hand on where.
template <typename T, bool FIRST>
__global__ __launch_bounds__(kSumBlock) void verify_sums_kernel(VerifyArgs a, int pass)
{
    const int b = blockIdx.y, seg = blockIdx.x * kSumWaves + threadIdx.x / kWave, segs = segments_of(a);
    Nodes nodes;
    Walk w{0.0, 1.0, 1ull, 0, 0, 0, 0, 0};
    bool work = true;                            // uniform over the workgroup
    if (FIRST) {
        nodes.load<T>(a, b);
        w.refused = walk_on(w, nodes, a.draft != nullptr);
    } else {
        w = a.walks[(int64_t)(pass - 1) * a.batch + b];
        work = w.refused != 0;
        if (work) {
            nodes.load<T>(a, b);
            work = go_on(w, nodes, a.draft != nullptr, sum_of(pass_sums(a, b, w.pass, segs), segs));
            if (work) w.pass = pass;
        }
    }
    if (seg == 0 && threadIdx.x == 0) a.walks[(int64_t)pass * a.batch + b] = w;
    if (!work || seg >= segs) return;
    const Rest<T> rest(a, b, w);
    const double sum = rest.segment(nodes, seg);
    if (threadIdx.x % kWave == 0) pass_sums(a, b, pass, segs)[seg] = sum;
}

// The rest of the walk, a workgroup per sequence, and the draw.  ALONE: all of it, without launches before, for rows of kVerifyAlone segments at most.
template <typename T, bool ALONE>
__global__ __launch_bounds__(kWalkBlock) void verify_walk_kernel(VerifyArgs a)
{
    __shared__ double s_alone[ALONE ? kVerifyAlone : 1];
    __shared__ double s_sum[kWalkWaves];
    __shared__ int s_hit[kWalkWaves], s_last[kWalkWaves];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, segs = segments_of(a);
    Walk w{0.0, 1.0, 1ull, 0, 0, 0, 0, 0};
    Nodes nodes;
    double *sums = s_alone;
    if (ALONE) {
        nodes.load<T>(a, b);
        w.refused = walk_on(w, nodes, a.draft != nullptr);
    } else {
        w = a.walks[(int64_t)(a.passes - 1) * a.batch + b];
        sums = pass_sums(a, b, w.pass, segs);
        if (w.refused || w.gone) nodes.load<T>(a, b);            // uniform; else nobody asks
    }
    auto pass = [&] {
        const Rest<T> rest(a, b, w);
        __syncthreads();                         // nobody reads the old sums any more
        for (int seg = wave; seg < segs; seg += kWalkWaves) {
            const double sum = rest.segment(nodes, seg);
            if (lane == 0) sums[seg] = sum;
        }
        __syncthreads();
        return sum_of(sums, segs);
    };
    double total = ALONE ? pass() : sum_of(sums, segs);
    while (w.refused && go_on(w, nodes, a.draft != nullptr, total)) total = pass();         // (uniform: every wave has the same numbers)
    if (!(total > 0.0)) {                        // nothing is left: the target itself
        w.c = 0.0;
        w.gone = 0;
        total = pass();
    }
    // path and number of tokens
    if (wave == 0 && lane < a.n) {
        const int at = __popcll(w.path & ((1ull << lane) - 1)), cnt = __popcll(w.path);
        int32_t *const out = a.path + (int64_t)b * a.n;
        if (w.path >> lane & 1) out[at] = lane;
        if (lane >= cnt) out[lane] = -1;
        if (lane == 0) a.cnt[b] = cnt;
    }
    // The draw: the segment at which the running sum passes the threshold (every wave finds it), then the element, by the whole workgroup.
    // Where rounding leaves none, the last one that holds anything.
    if (!(total > 0.0)) {
        if (tid == 0) a.next[b] = -1;
        return;
    }
    const double t = (double)a.u_next[b] * total;
    double run = 0.0, before = 0.0;              // sum of what comes before the segment
    int seg = 0;
    for (int s0 = 0; s0 < segs; s0 += kWave) {
        const double mine = s0 + lane < segs ? sums[s0 + lane] : 0.0, upto = run + wave_scan64(mine);
        const uint64_t over = __ballot(upto > t && mine > 0.0), some = __ballot(mine > 0.0);
        const int l = over ? __builtin_ctzll(over) : some ? 63 - __builtin_clzll(some) : -1;
        if (l >= 0) {
            seg = s0 + l;
            before = __shfl(upto - mine, l);
        }
        if (over) break;
        run = __shfl(upto, kWave - 1);
    }
    const Rest<T> rest(a, b, w);
    const int first = seg * kVerifySegment + kDrawPer * tid;
    double x[kDrawPer], mine = 0.0;
#pragma unroll
    for (int k = 0; k < kDrawPer; ++k) mine += x[k] = rest.one(nodes, first + k);
    const double upto = wave_scan64(mine);
    __syncthreads();
    if (lane == kWave - 1) s_sum[wave] = upto;
    __syncthreads();
    for (int i = 0; i < wave; ++i) before += s_sum[i];
    before += upto - mine;
    int hit = INT32_MAX, last = -1;              // the first over the threshold, the last that holds anything
#pragma unroll
    for (int k = 0; k < kDrawPer; ++k) {
        before += x[k];
        if (x[k] > 0.0) {
            if (before > t) hit = min(hit, first + k);
            last = first + k;
        }
    }
#pragma unroll
    for (int step = kWave / 2; step > 0; step /= 2) {
        hit = min(hit, __shfl_xor(hit, step));
        last = max(last, __shfl_xor(last, step));
    }
    if (lane == 0) {
        s_hit[wave] = hit;
        s_last[wave] = last;
    }
    __syncthreads();
    if (tid == 0) {
        for (int i = 0; i < kWalkWaves; ++i) {
            hit = min(hit, s_hit[i]);
            last = max(last, s_last[i]);
        }
        a.next[b] = hit != INT32_MAX ? hit : last;
    }
}

}  // namespace

template <typename T> static hipError_t launch_verify(const VerifyArgs &a, hipStream_t s)
{
    const int segs = (a.vocab + kVerifySegment - 1) / kVerifySegment;
    if (a.passes == 0) {
        hipLaunchKernelGGL((verify_walk_kernel<T, true>), dim3(a.batch), dim3(kWalkBlock), 0, s, a);
        return hipGetLastError();
    }
    const dim3 grid((segs + kSumWaves - 1) / kSumWaves, a.batch);
    hipLaunchKernelGGL((verify_sums_kernel<T, true>), grid, dim3(kSumBlock), 0, s, a, 0);
    hipError_t rc = hipGetLastError();
    for (int pass = 1; pass < a.passes && rc == hipSuccess; ++pass) {
        hipLaunchKernelGGL((verify_sums_kernel<T, false>), grid, dim3(kSumBlock), 0, s, a, pass);
        rc = hipGetLastError();
    }
    if (rc != hipSuccess) return rc;
    hipLaunchKernelGGL((verify_walk_kernel<T, false>), dim3(a.batch), dim3(kWalkBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_verify_drafts(int dtype, const VerifyArgs &a, hipStream_t s)
{
    return dtype == 0 ? launch_verify<float>(a, s) : launch_verify<bf16_t>(a, s);
}

}  // namespace hgca
