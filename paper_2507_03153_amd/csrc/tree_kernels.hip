// Attention of a few queries per sequence over one tier (in bf16 with more than 32 rows, in part 16: tree_rows_kernels.hip): drafted tokens that
// are verified together, each of which sees the conversation and its own ancestors among the drafts (the tier's last n tokens, a
// bit per draft), and queries over an 8-bit tier.  A row is one query of one head of the group that shares a KV head; a launch
// reads K and V once per 16 or 32 rows.
//
// One wave is 16 rows (RT = 1) or 32 (RT = 2) against 32 tokens of its own at a time, straight from memory to the matrix operands:
//   S^T[token, row]  = K[token, :] . Q[row, :]             A = K rows as loaded, B = Q
//   O^T[col, row]   += V^T[col, token] . P^T[token, row]   A = V^T, transposed in registers, B = P
// In both results lane % 16 is the row, so maximum, sum and rescaling of a row stay in the lanes that hold its scores and its
// outputs.  A contraction may go through its index in any order as long as both operands do: the tokens of the second product come in
// the order in which a lane holds their scores (block_token), the columns of the first in the order in which 16-byte loads
// bring them.  V needs tokens side by side where rows have columns side by side: a lane loads E = D / 16 adjacent columns of the four
// tokens that it holds the scores of, and pairs of tokens are put together by one byte permutation each; output column m * E + e is row
// m of the e-th product.
//
// fp32 outputs ask for weights as exact as fp32: they enter the second product as three bf16 parts that add up to them (O is then 2e-7 to
// 1.1e-6 off 64 bits).  Outputs in bf16, whose own rounding is 2^-9, take two parts, 16 bits of a weight, 2e-6 of O: of 65536 outputs of 64 drafts
// over 32 K tokens 164 are not the nearest bf16 number, 73 with three parts and 134 of sums in fp32; three parts take 390 -> 478 us.
//
// What bounds it: the stream of K and V (16 rows meet a K row in one product, so a workgroup's arithmetic is short), and with few
// tokens a workgroup's chain of loads.  One token x 8 sequences over 28 K tokens of 8 heads of 128 in 8 bits, groups of 4: 79.5 us, 485 MB
// at 6.1 TB/s (streaming reads reach 6.9), and 4.6 us of fold; 5 fp32 queries x 2 over 4 K in 8 bits 14.9 + 4.1 us; 4 fp32 drafts
// over 260 tokens of 4 heads of 64 7.5 us, one launch.  (Rows two steps ahead in registers: level; three waves per SIMD: slower.)
#include <algorithm>
#include <type_traits>

#include "tree_device.hpp"

namespace hgca {

namespace {

constexpr uint32_t kLowHalves = 0x05040100u, kHighHalves = 0x07060302u;          // byte selectors: (b.lo, a.lo) and (b.hi, a.hi)

__device__ __forceinline__ floatx4 mfma16(const uint4 &a, const uint4 &b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// max / sum over the four rows of 16 lanes
__device__ __forceinline__ float rows_max(float x) {
    const LanePair r = rows_of(x);
    const LanePair h = halves_of(fmaxf(r.a, r.b));
    return fmaxf(h.a, h.b);
}
__device__ __forceinline__ float rows_sum(float x) { return strided_sum<16>(x); }

// x of lane I of every row of 16 lanes (row_newbcast)
template <int I> __device__ __forceinline__ uint32_t row_lane(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x150 + I, 0xf, 0xf, true);
}

// 16 tokens of K or of V: what a lane (n = lane % 16, g = lane / 16) holds of them.  `row` is the tile's first row, uniform over
// the wave, nv the number of tokens that exist (the others repeat the last one).
template <typename S, int D> struct KTile;
template <typename S, int D> struct VTile;

// STREAM: rows that pass once and are more than the last cache holds leave the caches alone
template <bool STREAM> __device__ __forceinline__ uint4 row16(const char *p) { return STREAM ? load16_stream(p) : load16(p); }
template <bool STREAM> __device__ __forceinline__ uint2 row8(const char *p) {
    const uint32_t *w = reinterpret_cast<const uint32_t *>(p);
    return STREAM ? make_uint2(__builtin_nontemporal_load(w), __builtin_nontemporal_load(w + 1)) : *reinterpret_cast<const uint2 *>(p);
}

template <int D> struct KTile<bf16_t, D> {
    uint4 k[D / 32];
    static __device__ __forceinline__ int column(int s, int g) { return 32 * s + 8 * g; }       // of slice s of the contraction
    template <bool STREAM> __device__ __forceinline__ void load(const TreeArgs &a, uint32_t row, int nv, int n, int g) {
        const char *p = a.kv.k + (size_t)row * (2 * D) + (uint32_t)(min(n, nv - 1) * (2 * D) + 16 * g);
#pragma unroll
        for (int s = 0; s < D / 32; ++s) k[s] = row16<STREAM>(p + 64 * s);
    }
    __device__ __forceinline__ void prepare(int) {}
    __device__ __forceinline__ uint4 operand(int s) const { return k[s]; }
};

template <int D> struct VTile<bf16_t, D> {
    static constexpr int E = D / 16;
    uint32_t v[4][E / 2];
    template <bool STREAM> __device__ __forceinline__ void load(const TreeArgs &a, uint32_t row, int nv, int n, int g) {
        const char *vp = a.kv.v + (size_t)row * (2 * D);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const char *p = vp + (uint32_t)(min(4 * g + j, nv - 1) * (2 * D) + n * 2 * E);
            if constexpr (D == 128) *reinterpret_cast<uint4 *>(v[j]) = row16<STREAM>(p);
            else *reinterpret_cast<uint2 *>(v[j]) = row8<STREAM>(p);
        }
    }
    __device__ __forceinline__ void words(uint32_t (&w)[4][E / 2], int) const {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < E / 2; ++i) w[j][i] = v[j][i];
    }
};

template <int D> struct KTile<kv8_t, D> {
    uint4 k[D / 64];
    uint32_t scales;
    float f[D / 64];
    static __device__ __forceinline__ int column(int s, int g) { return 64 * (s / 2) + 16 * g + 8 * (s % 2); }
    template <bool STREAM> __device__ __forceinline__ void load(const TreeArgs &a, uint32_t row, int nv, int n, int g) {
        const uint32_t r = min(n, nv - 1);
        const char *p = a.kv.k + (size_t)row * D + (r * D + 16 * g);
#pragma unroll
        for (int s = 0; s < D / 64; ++s) k[s] = row16<STREAM>(p + 64 * s);
        scales = (reinterpret_cast<const typename Kv8Scales<D>::Word *>(a.k_scale) + row)[r];
    }
    __device__ __forceinline__ void prepare(int lane) {          // a lane's 16 columns lie in one block of 32
#pragma unroll
        for (int s = 0; s < D / 64; ++s) f[s] = kv8_scale(scales, 2 * s + lane / 32);
    }
    __device__ __forceinline__ uint4 operand(int s) const {
        const uint32_t c0 = s % 2 ? k[s / 2].z : k[s / 2].x, c1 = s % 2 ? k[s / 2].w : k[s / 2].y;
        return make_uint4(kv8_pair_bf16<false>(c0, f[s / 2]), kv8_pair_bf16<true>(c0, f[s / 2]),
                          kv8_pair_bf16<false>(c1, f[s / 2]), kv8_pair_bf16<true>(c1, f[s / 2]));
    }
};

// (Scales are one word per row: a lane loads that of token 4 g + n % 4 and has the others from its row of 16 lanes.  With a load per token
// one token x 8 over 28 K, heads of 64: 73.9 against 69.3 us, of 128: level.)
template <int D> struct VTile<kv8_t, D> {
    static constexpr int E = D / 16;
    uint32_t v[4][E / 4], scales;
    template <bool STREAM> __device__ __forceinline__ void load(const TreeArgs &a, uint32_t row, int nv, int n, int g) {
        const char *vp = a.kv.v + (size_t)row * D;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const char *p = vp + (uint32_t)min(4 * g + j, nv - 1) * D + n * E;
            if constexpr (D == 128) *reinterpret_cast<uint2 *>(v[j]) = row8<STREAM>(p);
            else v[j][0] = *reinterpret_cast<const uint32_t *>(p);
        }
        scales = (reinterpret_cast<const typename Kv8Scales<D>::Word *>(a.v_scale) + row)[min(4 * g + n % 4, nv - 1)];
    }
    __device__ __forceinline__ void words(uint32_t (&w)[4][E / 2], int lane) const {     // a lane's E columns lie in one block
        const int blk = lane % 16 * E / 32;
        const float f[4] = {kv8_scale(row_lane<0>(scales), blk), kv8_scale(row_lane<1>(scales), blk), kv8_scale(row_lane<2>(scales), blk),
                            kv8_scale(row_lane<3>(scales), blk)};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int i = 0; i < E / 4; ++i) {
                w[j][2 * i] = kv8_pair_bf16<false>(v[j][i], f[j]);
                w[j][2 * i + 1] = kv8_pair_bf16<true>(v[j][i], f[j]);
            }
        }
    }
};

// Running softmax of RT row tiles over NT 16-token tiles per step.  The maximum is kept on raw scores (the scale is positive); a
// weight is 2^fma(score, scale2, shift) with the shift of the maximum (shift_of), which partial results are relative to.
template <int RT, int E> struct RowState {
    float m[RT], shift[RT], l[RT];               // shift: 0 for far rows; l: over the lane's own tokens
    bool far;                                    // a row of the wave is far (uniform over the wave)
    floatx4 o[RT][E];
    __device__ __forceinline__ void clear() {
        far = false;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            m[r] = -INFINITY;
            shift[r] = l[r] = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) o[r][e] = floatx4{};
        }
    }
    // scores become weights
    template <int NT> __device__ __forceinline__ void weigh(floatx4 (&s)[RT][NT], float scale2) {
        float mx[RT];
        bool more = false;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            mx[r] = s[r][0][0];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx[r] = fmaxf(mx[r], s[r][t][i]);
            more = more || mx[r] > m[r];
        }
        if (__any(more)) {                       // uniform over the wave
            bool any_far = false;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float m_new = fmaxf(m[r], rows_max(mx[r])), to = shift_of(m_new, scale2), corr = rescale_factor(m[r], m_new, scale2);
                m[r] = m_new;
                shift[r] = is_far(to) ? 0.f : to;
                any_far = any_far || is_far(to);
                l[r] *= corr;
#pragma unroll
                for (int e = 0; e < E; ++e) o[r][e] *= corr;
            }
            far = __any(any_far);
        }
        if (far) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float less = is_far(shift_of(m[r], scale2)) ? m[r] : 0.f;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[r][t][i] -= less;
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[r][t][i] = __builtin_amdgcn_exp2f(fmaf(s[r][t][i], scale2, shift[r]));             // masked scores give 0
                    l[r] += s[r][t][i];
                }
    }
};

// What the waves of a workgroup found for their own tokens becomes one result per row: the final one, or a split's partial.
struct NoOddSeen {};
template <typename S, int D, int RT> struct MergeShared {
    float m[kTreeWaves][16 * RT], l[kTreeWaves][16 * RT];
    float o[kTreeWaves][16][D + 4];
    uint32_t odd[kTreeWaves];                    // a wave met infinities or NaN, or sums that are not finite
    std::conditional_t<sizeof(S) == 1, NoOddSeen, OddSeen<D>> seen;      // (codes are finite or NaN, and a NaN stays one in every product)
};

template <int D, bool OUT_BF16> __device__ __forceinline__ void store_eight(void *o, int64_t at, const float *x) {
    constexpr int E = D / 16;
    if constexpr (OUT_BF16) {
        uint32_t w[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        char *p = static_cast<char *>(o) + 2 * at;
        if constexpr (E == 8) *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(w);
        else *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(w);
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 4)
            *reinterpret_cast<float4 *>(static_cast<float *>(o) + at + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    }
}

// odd: the lane has taken infinities or NaN out of V.
template <typename S, int D, int RT>
__device__ __forceinline__ void merge_waves(MergeShared<S, D, RT> &sh, uint32_t *s_row, const TreeArgs &a, RowState<RT, D / 16> &st,
                                            const Span &span, int tail, bool odd, int kvh, int row0)
{
    constexpr int E = D / 16;
    constexpr bool kOdd = sizeof(S) > 1;
    const int b = span.b, slot = span.slot;
    const int tid = threadIdx.x, w = tid / kWave, lane = tid % kWave, n = lane % 16, g = lane / 16;
    const int lg = __builtin_ctz(a.sh.group), group = a.sh.group, rows = a.n_q * group;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float l = rows_sum(st.l[r]);
        if (g == 0) {
            // nothing seen: l is 0 (with only NaN seen it is NaN)
            sh.m[w][16 * r + n] = l == 0.f ? -INFINITY : -shift_of(st.m[r], a.sh.sm_scale * kTreeLog2e);
            sh.l[w][16 * r + n] = l;
        }
    }
    if constexpr (kOdd) {
        float z[4] = {0.f, 0.f, 0.f, 0.f};       // NaN where a sum is not finite
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) z[i] = fmaf(st.o[r][e][i], 0.f, z[i]);
        const float all = (z[0] + z[1]) + (z[2] + z[3]);
        odd = __any(all != all || odd);
        if (lane == 0) sh.odd[w] = odd;
    }
    bool any_odd = false;                        // uniform over the workgroup
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (r > 0) __syncthreads();              // the tile before has been read
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = st.o[r][e][i];
#pragma unroll
            for (int e = 0; e < E; e += 4)
                *reinterpret_cast<float4 *>(&sh.o[w][n][(4 * g + i) * E + e]) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        }
        __syncthreads();
        if constexpr (kOdd) {
            if (r == 0) {
#pragma unroll
                for (int i = 0; i < kTreeWaves; ++i) any_odd = any_odd || sh.odd[i];
                if (any_odd)
                    sh.seen.template collect<S, kTreeBlock>(s_row, a, b, kvh, span.begin, span.end, tail);
            }
        }
        const int row = tid / 16, c = tid % 16, at_row = row0 + 16 * r + row;
        if (at_row >= rows) continue;            // (barriers are reached by all: the loop is unrolled and uniform)
        float M = -INFINITY, f[kTreeWaves], L = 0.f, x[E];
#pragma unroll
        for (int i = 0; i < kTreeWaves; ++i) M = fmaxf(M, sh.m[i][16 * r + row]);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = 0.f;
#pragma unroll
        for (int i = 0; i < kTreeWaves; ++i) {
            const float m = sh.m[i][16 * r + row];
            f[i] = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
            if (m == -INFINITY) continue;
            L = fmaf(sh.l[i][16 * r + row], f[i], L);
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const float4 o = *reinterpret_cast<const float4 *>(&sh.o[i][row][c * E + e]);
                x[e] = fmaf(o.x, f[i], x[e]);
                x[e + 1] = fmaf(o.y, f[i], x[e + 1]);
                x[e + 2] = fmaf(o.z, f[i], x[e + 2]);
                x[e + 3] = fmaf(o.w, f[i], x[e + 3]);
            }
        }
        const int64_t qr = (int64_t)b * a.n_q + (at_row >> lg), out_row = qr * a.sh.n_q_heads + kvh * group + (at_row & (group - 1));
        if constexpr (kOdd) {
            if (any_odd) {
                const uint64_t mask = a.mask ? a.mask[qr] : ~0ull;
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = sh.seen.result(c * E + e, mask, x[e]);
            }
        }
        if (a.n_splits > 1) {
            const int64_t at = partial_row(a, slot, kvh, at_row);
            store_eight<D, false>(a.part_o, at * D + c * E, x);
            if (c == 0) {
                a.part_m[at] = M;
                a.part_l[at] = L;
            }
        } else {
            const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = L == 0.f ? 0.f : x[e] * inv;
            if (a.o_bf16) store_eight<D, true>(a.o, out_row * D + c * E, x);
            else store_eight<D, false>(a.o, out_row * D + c * E, x);
            if (c == 0) a.lse[out_row] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
        }
    }
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// TQ: bf16_t, or float for fp32 queries over an 8-bit tier, which enter as three bf16 parts that add up to them.  PP: parts of a weight.
template <typename S, typename TQ, int D, int RT, int PP, bool STREAM>
__global__ __launch_bounds__(kTreeBlock, 2) void rows_attn_kernel(TreeArgs a)
{
    constexpr int KS = D / 32, E = D / 16, W = E / 2, QP = sizeof(TQ) == 4 ? 3 : 1, NW = kTreeWaves;
    constexpr bool kDrafts = sizeof(S) > 1;      // 8-bit tiers hold no drafted tokens
    __shared__ uint32_t s_row[kSub];
    __shared__ MergeShared<S, D, RT> s_merge;
    const int kvh = blockIdx.y, row0 = (int)(blockIdx.x % a.row_blocks) * 16 * RT;          // row blocks of a slot run side by side
    const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane % 16, g = lane / 16;
    const int lg = __builtin_ctz(a.sh.group), group = a.sh.group, rows = a.n_q * group;
    const Span span(a, blockIdx.x / a.row_blocks, 32 * NW);
    if (span.idle) return;                       // uniform over the workgroup
    if (kvh == 0 && row0 == 0) span.tell(a);

    uint4 q[RT][QP][KS];
    uint64_t mask[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = min(row0 + 16 * r + n, rows - 1);     // lanes without a row repeat the last one and store nothing
        const int64_t qr = (int64_t)span.b * a.n_q + (row >> lg);
        mask[r] = kDrafts && a.mask ? a.mask[qr] : ~0ull;
        const char *p = static_cast<const char *>(a.q) + (qr * a.sh.n_q_heads + kvh * group + (row & (group - 1))) * D * (int)sizeof(TQ);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const char *c = p + KTile<S, D>::column(s, g) * (int)sizeof(TQ);
            if constexpr (QP == 1) {
                q[r][0][s] = load16(c);
            } else {
                float x[8];
                Elem<float>::expand(load16(c), x);
                Elem<float>::expand(load16(c + 16), x + 4);
                uint32_t part[3][8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {                    // cut off, not rounded: the first part of no finite value overflows
                    const uint32_t u = __float_as_uint(x[i]);
                    const bool odd = not_finite(x[i]);           // infinities and NaN are their own first part
                    const float x1 = odd ? 0.f : x[i] - __uint_as_float(u & 0xffff0000u);
                    const float x2 = x1 - __uint_as_float(__float_as_uint(x1) & 0xffff0000u);
                    part[0][i] = odd && (u & 0x7fffffu) ? 0x7fffu : u >> 16;
                    part[1][i] = __float_as_uint(x1) >> 16;
                    part[2][i] = __float_as_uint(x2) >> 16;
                }
#pragma unroll
                for (int t = 0; t < 3; ++t)
                    q[r][t][s] = make_uint4(part[t][0] | part[t][1] << 16, part[t][2] | part[t][3] << 16,
                                            part[t][4] | part[t][5] << 16, part[t][6] | part[t][7] << 16);
            }
        }
    }

    RowState<RT, E> st;
    st.clear();
    const float scale2 = a.sh.sm_scale * kTreeLog2e;
    const int tail = kDrafts && a.mask ? span.len - a.n_q : span.len;      // first drafted token

    bool met_odd = false;                        // of the lane
    KTile<S, D> kt[2];
    VTile<S, D> vt[2];
    // One step: the scores of 32 tokens from kt, their weights, the outputs from vt.  next_k() and next_v() request the next step's
    // rows into the registers as soon as these have been read.
    auto consume = [&](int tok, auto next_k, auto next_v) {
        const bool masked = tok + 32 > min(tail, span.end);      // the step meets the end of the tokens or drafted ones; uniform
        kt[0].prepare(lane);
        kt[1].prepare(lane);
        floatx4 s[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r) s[r][0] = s[r][1] = floatx4{};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint4 op = kt[t].operand(k);
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int p = QP - 1; p >= 0; --p) s[r][t] = mfma16(op, q[r][p][k], s[r][t]);
            }
        next_k();
        uint32_t seen[RT];
        if (masked) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                seen[r] = (uint32_t)seen_tokens(mask[r], tok + 4 * g, tail, span.end);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(seen[r] >> (16 * t + i) & 1u)) s[r][t][i] = -INFINITY;
            }
        }
        st.weigh(s, scale2);
        uint4 p[RT][PP];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            uint32_t part[PP][4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float x0 = s[r][c / 2][2 * (c % 2)], x1 = s[r][c / 2][2 * (c % 2) + 1];
#pragma unroll
                for (int t = 0; t < PP; ++t) {
                    part[t][c] = pack_bf16(x0, x1);
                    x0 -= __uint_as_float(part[t][c] << 16);
                    x1 -= __uint_as_float(part[t][c] & 0xffff0000u);
                }
            }
#pragma unroll
            for (int t = 0; t < PP; ++t) p[r][t] = make_uint4(part[t][0], part[t][1], part[t][2], part[t][3]);
        }
        uint32_t v[2][4][W];
        vt[0].words(v[0], lane);
        vt[1].words(v[1], lane);
        auto pairs = [&](int e, auto word) {                     // eight tokens of column n * E + e
            const uint32_t sel = e % 2 ? kHighHalves : kLowHalves;
            return make_uint4(__builtin_amdgcn_perm(word(0, 1, e / 2), word(0, 0, e / 2), sel),
                              __builtin_amdgcn_perm(word(0, 3, e / 2), word(0, 2, e / 2), sel),
                              __builtin_amdgcn_perm(word(1, 1, e / 2), word(1, 0, e / 2), sel),
                              __builtin_amdgcn_perm(word(1, 3, e / 2), word(1, 2, e / 2), sel));
        };
        if (masked) {
            // a weight of 0 keeps a row out of the product only if the row is finite: rows behind the end become 0, and
            // infinities and NaN of drafted rows are taken out (OddSeen brings them to the queries that see them)
            uint32_t odd = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool gone = tok + 16 * t + 4 * g + j >= span.end;
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        uint32_t &x = v[t][j][i];
                        x = gone ? 0 : x;
                        odd |= odd_carry(x);
                    }
                }
            if (kDrafts && a.mask && (odd & kSigns)) {
                met_odd = true;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < W; ++i) v[t][j][i] &= ~odd_halves(v[t][j][i]);
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint4 op = pairs(e, [&](int t, int j, int i) { return v[t][j][i]; });
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int t = PP - 1; t >= 0; --t) st.o[r][e] = mfma16(op, p[r][t], st.o[r][e]);
        }
        next_v();
    };

    // the split in passes that the table of a paged tier covers; a wave takes every NW-th 32 tokens
    const int total = span.end - span.begin, sub_len = pass_length(a.kv, total);
    for (int sub0 = 0; sub0 < total; sub0 += sub_len) {
        const int nsub = min(sub_len, total - sub0), first = span.begin + sub0;
        __syncthreads();                         // the table of the pass before is no longer in use
        const BlockRows where = make_block_rows<kTreeBlock>(s_row, a.kv, a.sh.n_kv_heads, span.b, kvh, first, nsub);
        auto fetch = [&](auto &tile, int tok) {                  // tok: in the pass; nothing behind its end
            if (tok >= nsub) return;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int gr = min(tok / 16 + t, (nsub - 1) / 16);
                const uint32_t row = where.table ? where.table[gr] : where.base + 16 * gr;
                tile[t].template load<STREAM>(a, __builtin_amdgcn_readfirstlane(row), min(16, nsub - 16 * gr), n, g);
            }
        };
        constexpr int kStep = 32 * NW;
        int tok = 32 * w;
        fetch(kt, tok);
        fetch(vt, tok);
        for (; tok < nsub; tok += kStep)
            consume(first + tok, [&] { fetch(kt, tok + kStep); }, [&] { fetch(vt, tok + kStep); });
    }
    merge_waves<S, D, RT>(s_merge, s_row, a, st, span, tail, met_odd, kvh, row0);
}

// The same over fp32 rows, on the fp32 matrix instructions (products and sums in fp32, nothing rounded in between): 16 tokens at a time.  A
// lane's four tokens are the four slices of the second product.
template <int D, int RT>
__global__ __launch_bounds__(kTreeBlock, 2) void rows_attn_f32_kernel(TreeArgs a)
{
    constexpr int E = D / 16, U = D / 16, NW = kTreeWaves, RB = 4 * D;
    __shared__ uint32_t s_row[kSub];
    __shared__ MergeShared<float, D, RT> s_merge;
    const int kvh = blockIdx.y, row0 = (int)(blockIdx.x % a.row_blocks) * 16 * RT;          // row blocks of a slot run side by side
    const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane % 16, g = lane / 16;
    const int lg = __builtin_ctz(a.sh.group), group = a.sh.group, rows = a.n_q * group;
    const Span span(a, blockIdx.x / a.row_blocks, 32 * NW);
    if (span.idle) return;                       // uniform over the workgroup
    if (kvh == 0 && row0 == 0) span.tell(a);

    float q[RT][U][4];
    uint64_t mask[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = min(row0 + 16 * r + n, rows - 1);
        const int64_t qr = (int64_t)span.b * a.n_q + (row >> lg);
        mask[r] = a.mask ? a.mask[qr] : ~0ull;
        const char *p = static_cast<const char *>(a.q) + (qr * a.sh.n_q_heads + kvh * group + (row & (group - 1))) * RB + 16 * g;
#pragma unroll
        for (int u = 0; u < U; ++u) Elem<float>::expand(load16(p + 64 * u), q[r][u]);
    }
    RowState<RT, E> st;
    st.clear();
    const float scale2 = a.sh.sm_scale * kTreeLog2e;
    const int tail = a.mask ? span.len - a.n_q : span.len;

    bool met_odd = false;                        // of the lane
    float kr[U][4], vr[4][E];
    auto consume = [&](int tok, auto next_k, auto next_v) {
        const bool masked = tok + 16 > min(tail, span.end);
        floatx4 s[RT][1], s2[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) s[r][0] = s2[r] = floatx4{};
#pragma unroll
        for (int u = 0; u < U; u += 2)
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int r = 0; r < RT; ++r) {                   // two chains per row tile
                    s[r][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[u][c], q[r][u][c], s[r][0], 0, 0, 0);
                    s2[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[u + 1][c], q[r][u + 1][c], s2[r], 0, 0, 0);
                }
        next_k();
#pragma unroll
        for (int r = 0; r < RT; ++r) s[r][0] += s2[r];
        uint32_t seen[RT];
        if (masked) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                seen[r] = (uint32_t)seen_tokens(mask[r], tok + 4 * g, tail, span.end);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(seen[r] >> i & 1u)) s[r][0][i] = -INFINITY;
            }
        }
        st.weigh(s, scale2);
        if (masked) {                            // as above
            float odd[4] = {0.f, 0.f, 0.f, 0.f}; // NaN where a value is not finite
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool gone = tok + 4 * g + j >= span.end;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    vr[j][e] = gone ? 0.f : vr[j][e];
                    odd[j] = fmaf(vr[j][e], 0.f, odd[j]);
                }
            }
            if (a.mask && __builtin_isnan((odd[0] + odd[1]) + (odd[2] + odd[3]))) {
                met_odd = true;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < E; ++e) vr[j][e] = not_finite(vr[j][e]) ? 0.f : vr[j][e];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    st.o[r][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[j][e], s[r][0][j], st.o[r][e], 0, 0, 0);
        next_v();
    };

    const int total = span.end - span.begin, sub_len = pass_length(a.kv, total);
    for (int sub0 = 0; sub0 < total; sub0 += sub_len) {
        const int nsub = min(sub_len, total - sub0), first = span.begin + sub0;
        __syncthreads();
        const BlockRows where = make_block_rows<kTreeBlock>(s_row, a.kv, a.sh.n_kv_heads, span.b, kvh, first, nsub);
        auto first_row = [&](int tok) {
            return (uint32_t)__builtin_amdgcn_readfirstlane(where.table ? where.table[tok / 16] : where.base + tok);
        };
        auto fetch_k = [&](int tok) {
            if (tok >= nsub) return;
            const char *p = a.kv.k + (size_t)first_row(tok) * RB + (uint32_t)(min(n, min(16, nsub - tok) - 1) * RB + 16 * g);
#pragma unroll
            for (int u = 0; u < U; ++u) Elem<float>::expand(load16(p + 64 * u), kr[u]);
        };
        auto fetch_v = [&](int tok) {
            if (tok >= nsub) return;
            const char *vp = a.kv.v + (size_t)first_row(tok) * RB;
            const int last = min(16, nsub - tok) - 1;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < E; e += 4)
                    Elem<float>::expand(load16(vp + (uint32_t)(min(4 * g + j, last) * RB + n * 4 * E + 4 * e)), vr[j] + e);
        };
        constexpr int kStep = 16 * NW;
        int tok = 16 * w;
        fetch_k(tok);
        fetch_v(tok);
        for (; tok < nsub; tok += kStep)
            consume(first + tok, [&] { fetch_k(tok + kStep); }, [&] { fetch_v(tok + kStep); });
    }
    merge_waves<float, D, RT>(s_merge, s_row, a, st, span, tail, met_odd, kvh, row0);
}

// The splits of a row: M = max m_s, O = sum o_s 2^{m_s - M} / sum l_s 2^{m_s - M}.  A wave per row; 16 or 32 lanes across the columns,
// the others take further splits.  Bound by two round trips to memory and the partials: 8192 rows of 128 in 8 splits 8.6 us (34 MB, 3.9
// TB/s), 256 rows in 8 splits 4.6 us.  Few rows in many splits are loads one after another: they take a workgroup per row.  Wave :
// workgroup, whole calls, us: 4 rows in 128 splits 38.1 : 30.1 (120 K tokens in 8 bits), 32 in 64 31.9 : 27.8, 128 in 32 23.9 : 22.0, 40
// in 16 18.4 : 18.0; 2048 rows in 32 87.2 : 89.2.
template <int D, int WAVES> __global__ __launch_bounds__(kTreeBlock) void rows_fold_kernel(TreeArgs a, int64_t rows)
{
    constexpr int C4 = D / 4, SG = kWave / C4, PRE = 4;
    __shared__ float4 s_x[WAVES > 1 ? WAVES : 1][WAVES > 1 ? C4 : 1];
    __shared__ float s_l[WAVES];
    const int lane = threadIdx.x % kWave, sg = lane / C4, c4 = lane % C4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t row = WAVES > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kTreeWaves + wave;
    const int w = WAVES > 1 ? wave : 0;          // of the row's waves
    if (row >= rows) return;                     // (with several waves per row there are as many workgroups as rows)
    const int h = (int)(row % a.sh.n_q_heads), i = (int)(row / a.sh.n_q_heads % a.n_q), b = (int)(row / a.sh.n_q_heads / a.n_q);
    const int first = a.seq_slots[2 * b], S = a.seq_slots[2 * b + 1];
    const int64_t at = partial_row(a, first, h / a.sh.group, i * a.sh.group + h % a.sh.group);
    const int64_t stride = partial_row(a, 1, 0, 0);
    const float *m = a.part_m + at, *l = a.part_l + at, *o = a.part_o + at * D + 4 * c4;
    float M = -INFINITY;
    for (int s = lane; s < S; s += kWave) M = fmaxf(M, m[s * stride]);
    M = wave_max(M);
    float L = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = w * SG + sg; s0 < S; s0 += WAVES * SG * PRE) {
        float pm[PRE], pl[PRE];
        float4 po[PRE];
#pragma unroll
        for (int i = 0; i < PRE; ++i) {
            const int64_t s = min(s0 + i * WAVES * SG, S - 1) * stride;
            pm[i] = m[s];
            pl[i] = l[s];
            po[i] = *reinterpret_cast<const float4 *>(o + s * D);
        }
#pragma unroll
        for (int i = 0; i < PRE; ++i) {
            if (s0 + i * WAVES * SG >= S || pm[i] == -INFINITY) continue;
            const float f = __builtin_amdgcn_exp2f(pm[i] - M);
            L = fmaf(pl[i], f, L);
            x.x = fmaf(po[i].x, f, x.x);
            x.y = fmaf(po[i].y, f, x.y);
            x.z = fmaf(po[i].z, f, x.z);
            x.w = fmaf(po[i].w, f, x.w);
        }
    }
    L = strided_sum<C4>(L);
    x = make_float4(strided_sum<C4>(x.x), strided_sum<C4>(x.y), strided_sum<C4>(x.z), strided_sum<C4>(x.w));
    if constexpr (WAVES > 1) {
        if (sg == 0) s_x[w][c4] = x;
        if (lane == 0) s_l[w] = L;
        __syncthreads();
        if (w != 0) return;
#pragma unroll
        for (int i = 1; i < WAVES; ++i) {
            const float4 y = s_x[i][c4];
            x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
            L += s_l[i];
        }
    }
    if (sg != 0) return;
    if (not_finite(x.x) || not_finite(x.y) || not_finite(x.z) || not_finite(x.w)) {
        // a split's infinity is one whatever the split's factor, which may be 0
        float4 odd = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [](float &sum, float y) { sum += not_finite(y) ? y : 0.f; };
        for (int s = 0; s < S; ++s) {
            const float4 y = *reinterpret_cast<const float4 *>(o + s * stride * D);
            add(odd.x, y.x), add(odd.y, y.y), add(odd.z, y.z), add(odd.w, y.w);
        }
        x = make_float4(not_finite(odd.x) ? odd.x : x.x, not_finite(odd.y) ? odd.y : x.y, not_finite(odd.z) ? odd.z : x.z,
                        not_finite(odd.w) ? odd.w : x.w);
    }
    const float inv = 1.f / L;
    if (L == 0.f) x = make_float4(0.f, 0.f, 0.f, 0.f);
    else x = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    if (a.o_bf16)
        *reinterpret_cast<uint2 *>(static_cast<char *>(a.o) + 2 * (row * D + 4 * c4)) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
    else
        *reinterpret_cast<float4 *>(static_cast<float *>(a.o) + row * D + 4 * c4) = x;
    if (c4 == 0) a.lse[row] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
}

template <typename S, typename TQ, int D, int RT>
void launch_rows(const TreeArgs &a, dim3 grid, int batch, hipStream_t s)
{
    const dim3 block(kTreeBlock);
    if constexpr (sizeof(TQ) == 2 && !(sizeof(S) == 2 && D == 128 && RT == 2)) {       // (tree_block_rows takes that much elsewhere)
        // (fp32 queries take their rows in blocks of 16, which read K and V again)
        if (a.row_blocks == 1 && (int64_t)batch * a.sh.n_kv_heads * a.kv.cap * D * (int)sizeof(S) * 2 >= kLastCache) {
            if (a.o_bf16) hipLaunchKernelGGL((rows_attn_kernel<S, TQ, D, RT, 2, true>), grid, block, 0, s, a);
            else hipLaunchKernelGGL((rows_attn_kernel<S, TQ, D, RT, 3, true>), grid, block, 0, s, a);
            return;
        }
    }
    if (a.o_bf16) hipLaunchKernelGGL((rows_attn_kernel<S, TQ, D, RT, 2, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rows_attn_kernel<S, TQ, D, RT, 3, false>), grid, block, 0, s, a);
}

}  // namespace

int tree_block_rows(int dtype, bool kv8, int head_dim, int rows, int64_t tokens)
{
    if (rows <= 16 || (dtype == 0 && kv8)) return 16;
    if (dtype == 0) return 32;
    // 17 to 32 rows: with steps through LDS half of the waves have no rows, but those of this file spill registers over bf16 heads
    // of 128.  This file : LDS, 8 drafts in groups of 4, us: 8 x 16384 tokens of 8 heads 111 : 95.5, 8 x 4096 36.4 : 33.1, 64 x 300 25.1 :
    // 21.5, 1 x 60000 68.5 : 61.6; 2 x 4096 19.2 : 19.8, 1 x 1000 14.7 : 16.8.  Heads of 64: 20.2 : 21.4 at 8 x 4096; 8 bits 67.7 : 75.9 at 8 x 16384.
    const bool lds = rows > 32 || (!kv8 && head_dim == 128 && tokens >= int64_t(1) << 17);
    return lds ? kRowsPerBlock : 32;
}

hipError_t launch_tree_attn(int dtype, int head_dim, bool kv8, const TreeArgs &a, int batch, hipStream_t s)
{
    const int block_rows = tree_block_rows(dtype, kv8, head_dim, a.n_q * a.sh.group, (int64_t)batch * a.sh.n_kv_heads * a.kv.cap);
    const int rt = block_rows / 16;
    const dim3 grid((unsigned)((int64_t)batch * a.n_splits * a.row_blocks), (unsigned)a.sh.n_kv_heads);
#define HGCA_TREE_RT(S, D)                                               \
    do {                                                                 \
        if (rt == 1) launch_rows<S, bf16_t, D, 1>(a, grid, batch, s);    \
        else launch_rows<S, bf16_t, D, 2>(a, grid, batch, s);            \
    } while (0)
    if (block_rows == kRowsPerBlock) {
        const hipError_t rc = launch_tree_rows(head_dim, kv8, a, batch, s);
        if (rc != hipSuccess) return rc;
    } else if (kv8) {
        if (dtype == 1 && head_dim == 64) HGCA_TREE_RT(kv8_t, 64);
        else if (dtype == 1) HGCA_TREE_RT(kv8_t, 128);
        else if (head_dim == 64) launch_rows<kv8_t, float, 64, 1>(a, grid, batch, s);
        else launch_rows<kv8_t, float, 128, 1>(a, grid, batch, s);
    } else if (dtype == 1) {
        if (head_dim == 64) HGCA_TREE_RT(bf16_t, 64);
        else HGCA_TREE_RT(bf16_t, 128);
    } else if (head_dim == 64) {
        if (rt == 1) hipLaunchKernelGGL((rows_attn_f32_kernel<64, 1>), grid, dim3(kTreeBlock), 0, s, a);
        else hipLaunchKernelGGL((rows_attn_f32_kernel<64, 2>), grid, dim3(kTreeBlock), 0, s, a);
    } else {
        if (rt == 1) hipLaunchKernelGGL((rows_attn_f32_kernel<128, 1>), grid, dim3(kTreeBlock), 0, s, a);
        else hipLaunchKernelGGL((rows_attn_f32_kernel<128, 2>), grid, dim3(kTreeBlock), 0, s, a);
    }
#undef HGCA_TREE_RT
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess || a.n_splits == 1) return rc;
    const int64_t rows = (int64_t)batch * a.n_q * a.sh.n_q_heads;
    const bool several = a.n_splits >= 16 && rows <= 1024;
    const dim3 fold((unsigned)(several ? rows : (rows + kTreeWaves - 1) / kTreeWaves)), block(kTreeBlock);
    if (head_dim == 64 && several) hipLaunchKernelGGL((rows_fold_kernel<64, kTreeWaves>), fold, block, 0, s, a, rows);
    else if (head_dim == 64) hipLaunchKernelGGL((rows_fold_kernel<64, 1>), fold, block, 0, s, a, rows);
    else if (several) hipLaunchKernelGGL((rows_fold_kernel<128, kTreeWaves>), fold, block, 0, s, a, rows);
    else hipLaunchKernelGGL((rows_fold_kernel<128, 1>), fold, block, 0, s, a, rows);
    return hipGetLastError();
}

}  // namespace hgca
