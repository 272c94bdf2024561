// Attention of a few queries per sequence over one tier, 33 query rows and more per KV head, 17 and more over many tokens with heads of
// 128 (tree_block_rows; bf16 queries; a row is one query of one head of the group): drafted tokens with a mask over a bf16 tier, and queries over an 8-bit tier.
//
// Work unit: one workgroup = a split of the tokens of one (sequence, KV head) and up to 128 rows, 32 per wave.  K and V of a 64-token
// step go through a double-buffered LDS stage that all four waves read.  bf16 rows arrive by LDS-direct loads; 8-bit rows are loaded to
// registers during a step, become bf16 there (exact, two codes per conversion) and are stored to the other stage behind the step's
// products, a quarter of a row per thread.  Products as in the kernels for fewer rows, with 32 x 32 tiles:
//   S^T[token, row] = K . Q^T, O^T[col, row] += V^T . P^T, a lane's column is its row in both.
// fp32 results take the weights in three bf16 parts (4 units of matrix work per useful 2), bf16 results in two (3 per 2).
//
// What bounds it: matrix and vector instructions of a SIMD's two waves, which overlap in part, and the power they take.  64 drafts x 4 sequences
// over 32 K tokens, 64 / 8 heads of 128, bf16 result: 375 to 448 us, 275 GFLOP, 412 with the parts, matrix units busy 56 % of the cycles at 1.7
// GHz; with K and V of zeros 274 us.  16 queries x 4, 61 to 122 K tokens in 8 bits, fp32 result: 345 to 412 us for 204 (409)
// GFLOP.  32 drafts x 8 over 4 K tokens, 32 / 8 heads: 40 us, 102 MB read and 34 MB of partials written, about half of it a workgroup's start
// and end (eight steps each), and 8.6 us of fold.
#include <algorithm>
#include <type_traits>

#include "tree_device.hpp"

namespace hgca {

namespace {

constexpr int kNW = kAttnWaves;                  // waves of a workgroup
static_assert(kNW == kTreeWaves && kRowsPerBlock == 32 * kNW, "32 rows per wave");

// The rows of a step of an 8-bit tier on their way through registers: thread t has a quarter of row t / 4 of K and of V.
template <int D> struct CodesInFlight {
    static constexpr int kChunks = D / 64;       // of 16 codes, per thread and tensor: of K neighbours, of V every fourth, which
    uint4 k[kChunks], v[kChunks];                // halves the bank conflicts of its stores
    typename Kv8Scales<D>::Word ks, vs;
    __device__ __forceinline__ void load(const TreeArgs &a, const BlockRows &rows, int step, int nsub) {
        const int tok = min(step * kStepTokens + (int)threadIdx.x / 4, nsub - 1), part = threadIdx.x % 4;
        const size_t row = rows.table ? rows.table[tok / kGranule] + tok % kGranule : rows.base + tok;
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            k[i] = load16(a.kv.k + row * D + 16 * (part * kChunks + i));
            v[i] = load16(a.kv.v + row * D + 16 * (part + 4 * i));
        }
        ks = reinterpret_cast<const typename Kv8Scales<D>::Word *>(a.k_scale)[row];
        vs = reinterpret_cast<const typename Kv8Scales<D>::Word *>(a.v_scale)[row];
    }
    __device__ __forceinline__ void store(char *k_stage, char *v_stage) const {
        using S = DmaStage<D, kNW>;
        const int row = threadIdx.x / 4, part = threadIdx.x % 4;
        auto eight = [](uint32_t c0, uint32_t c1, float f) {
            return make_uint4(kv8_pair_bf16<false>(c0, f), kv8_pair_bf16<true>(c0, f), kv8_pair_bf16<false>(c1, f), kv8_pair_bf16<true>(c1, f));
        };
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {      // a chunk is two 16-byte pieces of bf16
            const int kc = part * kChunks + i, vc = part + 4 * i;
            const float kf = kv8_scale(ks, kc / 2), vf = kv8_scale(vs, vc / 2);
            *reinterpret_cast<uint4 *>(k_stage + S::k_offset(row, 2 * kc)) = eight(k[i].x, k[i].y, kf);
            *reinterpret_cast<uint4 *>(k_stage + S::k_offset(row, 2 * kc + 1)) = eight(k[i].z, k[i].w, kf);
            *reinterpret_cast<uint4 *>(v_stage + S::v_offset(row, vc)) = eight(v[i].x, v[i].y, vf);
            *reinterpret_cast<uint4 *>(v_stage + S::v_offset(row, vc) + 16) = eight(v[i].z, v[i].w, vf);
        }
    }
};

// HALVES: up to 64 rows per workgroup; two waves share 32 of them and take half of a step's tokens each, and add up at the end.
template <typename ST, int D, int PP, bool HALVES>
__global__ __launch_bounds__(kTreeBlock, 2) void many_rows_attn_kernel(TreeArgs a, int flat, int streamed)
{
    using S = DmaStage<D, kNW>;
    constexpr bool kCodes = sizeof(ST) == 1;
    constexpr int KK = D / 16, DT = D / 32, NT = HALVES ? 1 : kStepTokens / 32, kRows = HALVES ? kRowsPerBlock / 2 : kRowsPerBlock;
    __shared__ __attribute__((aligned(1024))) char s_k0[S::kBytes];
    __shared__ __attribute__((aligned(1024))) char s_k1[S::kBytes];
    __shared__ __attribute__((aligned(1024))) char s_v0[S::kBytes];
    __shared__ __attribute__((aligned(1024))) char s_v1[S::kBytes];
    __shared__ uint32_t s_row[kSub], s_odd[kNW];

    // Workgroups are dealt to the XCDs in turn: blocks of rows that read the same tokens take numbers that are equal modulo their number
    int slot = blockIdx.x, kvh = blockIdx.y, rb = 0;
    if (flat) {
        const int wg = (int)blockIdx.x, stream = wg % kXcds + kXcds * (wg / kXcds / a.row_blocks);
        if (stream >= a.n_splits * a.sh.batch * a.sh.n_kv_heads) return;         // uniform over the workgroup
        rb = wg / kXcds % a.row_blocks;
        kvh = stream % a.sh.n_kv_heads;
        slot = stream / a.sh.n_kv_heads;
    } else if (a.row_blocks > 1) {
        rb = slot % a.row_blocks;
        slot /= a.row_blocks;
    }
    const Span span(a, slot, kStepTokens);
    if (span.idle) return;                       // uniform over the workgroup
    if (kvh == 0 && rb == 0) span.tell(a);
    const int b = span.b;
    const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane % 32, hw = lane / 32;
    const int lg = __builtin_ctz(a.sh.group), group = a.sh.group, rows = a.n_q * group;
    const int row0 = rb * kRows + 32 * (HALVES ? w % 2 : w), half = HALVES ? w / 2 : 0;     // half: of every step's tokens
    const bool wave_live = row0 < rows, row_exists = row0 + n < rows;
    const int row = min(row0 + n, rows - 1);     // lanes without a row repeat the last one and store nothing
    const int64_t qr = (int64_t)b * a.n_q + (row >> lg), out_row = qr * a.sh.n_q_heads + kvh * group + (row & (group - 1));
    uint4 qop[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qop[kk] = load16(static_cast<const char *>(a.q) + out_row * S::kRowBytes + 16 * (2 * kk + hw));
    const uint64_t mask = !kCodes && a.mask ? a.mask[qr] : ~0ull;
    const float scale2 = a.sh.sm_scale * kTreeLog2e;
    int k_lane[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) k_lane[kk] = S::k_offset(n, 2 * kk + hw);
    const int v_lane = S::v_offset(4 * hw + lane % 16 / 4, lane / 16 % 2) + 8 * (lane % 4);

    const int tail = !kCodes && a.mask ? span.len - a.n_q : span.len;            // first drafted token
    bool met_odd = false, far = false;           // uniform over the wave; far: a row of it is (shift_of)
    float m = -INFINITY, shift = 0.f, l = 0.f;   // shift: 0 for far rows; l: over this lane's tokens
    floatx16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = floatx16{};

    // One step.  c[t][r] is the score of step token 32 t + 8 (r / 4) + 4 hw + r % 4; group g of the second product is 16 tokens, of
    // which the lane holds eight.
    auto body = [&](auto masked, const char *k_stage, const char *v_stage, int tok) {
        constexpr bool MASKED = decltype(masked)::value;
        if (HALVES) {                            // (half: tokens 32 half .. of the step)
            tok += 32 * half;
            k_stage += half * 32 * S::kRowBytes;
            v_stage += half * S::v_offset(32, 0);
        }
        floatx16 c[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) c[t] = floatx16{};
        uint4 kf[KK][NT];
        auto read_slice = [&](int kk) {
#pragma unroll
            for (int t = 0; t < NT; ++t) kf[kk][t] = *reinterpret_cast<const uint4 *>(k_stage + t * 32 * S::kRowBytes + k_lane[kk]);
        };
        read_slice(0);
        read_slice(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {        // operands are read two slices ahead
            if (kk + 2 < KK) read_slice(kk + 2);
#pragma unroll
            for (int t = 0; t < NT; ++t) c[t] = score_mfma(kf[kk][t], qop[kk], c[t]);
            __builtin_amdgcn_sched_barrier(0);
        }
        uint4 vop[2][DT];
        auto read_v = [&](int g, uint4 (&x)[DT]) {
            const char *v = v_stage + S::v_offset(16 * g, 0) + v_lane;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const short4v x0 = lds_read_tr16(v + 256 * dt), x1 = lds_read_tr16(v + S::v_offset(8, 0) + 256 * dt);
                const short8v both = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
                x[dt] = __builtin_bit_cast(uint4, both);
            }
        };
        read_v(0, vop[0]);
        __builtin_amdgcn_sched_barrier(0);
        uint64_t seen = 0;
        if constexpr (MASKED) {
            seen = seen_tokens(mask, tok + 4 * hw, tail, span.end);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(seen >> (32 * t + 8 * (r / 4) + r % 4) & 1)) c[t][r] = -INFINITY;
        }
        float mx = c[0][0];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, c[t][r]);
        if (__any(mx > m)) {                     // uniform over the wave
            const float m_new = fmaxf(m, halves_max(mx)), to = shift_of(m_new, scale2), corr = rescale_factor(m, m_new, scale2);
            m = m_new;
            shift = is_far(to) ? 0.f : to;
            far = __any(is_far(to));
            l *= corr;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) acc[dt] *= corr;
        }
        if (far) {
            const float less = is_far(shift_of(m, scale2)) ? m : 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t) c[t] -= less;
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        uint32_t part[PP][4];
        auto weigh = [&](int g) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float p[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    p[x] = __builtin_amdgcn_exp2f(fmaf(c[g / 2][8 * (g % 2) + 2 * e + x], scale2, shift));       // masked scores give 0
                    sum[(2 * e + x) % 4] += p[x];
                }
#pragma unroll
                for (int t = 0; t < PP; ++t) {
                    part[t][e] = pack_bf16(p[0], p[1]);
                    p[0] -= __uint_as_float(part[t][e] << 16);
                    p[1] -= __uint_as_float(part[t][e] & 0xffff0000u);
                }
            }
        };
        auto product = [&](const uint4 &v, const uint32_t (&p)[4], floatx16 to) {
            return score_mfma(v, make_uint4(p[0], p[1], p[2], p[3]), to);
        };
        weigh(0);
#pragma unroll
        for (int g = 0; g < 2 * NT; ++g) {
            __builtin_amdgcn_sched_barrier(0);
            uint4(&v)[DT] = vop[g % 2];
            if (g + 1 < 2 * NT) read_v(g + 1, vop[(g + 1) % 2]);
            if constexpr (MASKED && !kCodes) {
                // rows behind the end become 0 (a weight of 0 does not keep an infinity out); infinities and NaN of drafted rows are taken
                // out (OddSeen brings them to the rows that see them)
                const int left = span.end - (tok + 16 * g + 4 * hw);            // the lane's tokens: 0..3 and 8..11 of them
                uint32_t odd = 0;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    uint32_t x[4] = {v[dt].x, v[dt].y, v[dt].z, v[dt].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int first = 8 * (i / 2) + 2 * (i % 2);
                        x[i] = left > first + 1 ? x[i] : left > first ? x[i] & 0xffffu : 0u;
                        odd |= odd_carry(x[i]);
                    }
                    v[dt] = make_uint4(x[0], x[1], x[2], x[3]);
                }
                if (a.mask && __any((odd & kSigns) != 0)) {
                    met_odd = true;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        uint4 &x = v[dt];
                        x = make_uint4(x.x & ~odd_halves(x.x), x.y & ~odd_halves(x.y), x.z & ~odd_halves(x.z), x.w & ~odd_halves(x.w));
                    }
                }
            }
            uint32_t now[PP][4];
#pragma unroll
            for (int t = 0; t < PP; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) now[t][e] = part[t][e];
#pragma unroll
            for (int t = 0; t < PP; ++t)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) acc[dt] = product(v[dt], now[t], acc[dt]);
            if (g + 1 < 2 * NT) weigh(g + 1);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };

    const int total = span.end - span.begin, sub_len = pass_length(a.kv, total);
    for (int sub0 = 0; sub0 < total; sub0 += sub_len) {
        const int nsub = min(sub_len, total - sub0), first = span.begin + sub0, steps = (nsub + kStepTokens - 1) / kStepTokens;
        // steps of the pass that end before the drafted tokens and the end need no mask
        const int plain = max(min(min(tail, span.end) - first, nsub), 0) / kStepTokens;
        __syncthreads();                         // the previous table and stages are no longer in use
        const BlockRows where = make_block_rows<kTreeBlock>(s_row, a.kv, a.sh.n_kv_heads, b, kvh, first, nsub);
        CodesInFlight<kCodes ? D : 64> codes;
        auto request = [&](int s, char *k, char *v) {
            if constexpr (kCodes) codes.load(a, where, s, nsub);
            else if (streamed) dma_step<D, kNW, kNonTemporal, kNonTemporal>(a.kv, where, s, nsub, k, v);
            else dma_step<D, kNW, 0, 0>(a.kv, where, s, nsub, k, v);
        };
        auto arrive = [&](char *k, char *v) {    // what was requested is in its stage once all waves have passed a barrier
            if constexpr (kCodes) codes.store(k, v);
        };
        request(0, s_k0, s_v0);
        arrive(s_k0, s_v0);
        // Step s reads the stages of its parity, and the rows of step s + 1 go to those of the other parity, which were last read in
        // step s - 1: the barrier at its top orders both.
        auto step = [&](auto masked, int s, const char *k_cur, const char *v_cur, char *k_next, char *v_next) {
            if constexpr (!kCodes) wait_for_own_loads();         // the barrier alone does not wait for LDS-direct loads
            __syncthreads();
            if (s + 1 < steps) request(s + 1, k_next, v_next);
            // the further a workgroup is in its pass, the lower its priority: of two on a unit the older would finish far ahead
            const int left = steps - s;
            if (2 * left > steps) __builtin_amdgcn_s_setprio(3);
            else if (4 * left > steps) __builtin_amdgcn_s_setprio(2);
            else if (8 * left > steps) __builtin_amdgcn_s_setprio(1);
            else __builtin_amdgcn_s_setprio(0);
            if (wave_live) body(masked, k_cur, v_cur, first + s * kStepTokens);
            if (s + 1 < steps) arrive(k_next, v_next);
        };
        int s = 0;
        for (; s + 1 < plain; s += 2) {
            step(std::false_type{}, s, s_k0, s_v0, s_k1, s_v1);
            step(std::false_type{}, s + 1, s_k1, s_v1, s_k0, s_v0);
        }
        for (; s < steps; ++s)                   // at most one step here needs no mask
            step(std::true_type{}, s, s % 2 ? s_k1 : s_k0, s % 2 ? s_v1 : s_v0, s % 2 ? s_k0 : s_k1, s % 2 ? s_v0 : s_v1);
    }

    l = halves_sum(l);
    shift = shift_of(m, scale2);
    if constexpr (!kCodes) {                     // (codes are finite or NaN, and a NaN stays one in every product)
        float z[4] = {0.f, 0.f, 0.f, 0.f};       // NaN where a sum is not finite
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) z[r % 4] = fmaf(acc[dt][r], 0.f, z[r % 4]);
        const float all = (z[0] + z[1]) + (z[2] + z[3]);
        met_odd = __any(all != all) || met_odd;
        if (lane == 0) s_odd[w] = met_odd;
    }
    if constexpr (HALVES || !kCodes) __syncthreads();            // all waves have read the stages
    OddSeen<D> &seen_odd = *reinterpret_cast<OddSeen<D> *>(s_v1);
    static_assert(sizeof(OddSeen<D>) <= sizeof(s_v1), "the notes lie in a stage");
    bool any_odd = false;                        // uniform over the workgroup
    if constexpr (!kCodes) {
#pragma unroll
        for (int i = 0; i < kNW; ++i) any_odd = any_odd || s_odd[i];
        if (any_odd) seen_odd.template collect<ST, kTreeBlock>(s_row, a, b, kvh, span.begin, span.end, tail);
    }
    if constexpr (HALVES) {                      // the two waves of a row: the second one's results by way of the stages
        float *const box = reinterpret_cast<float *>(w % 2 ? s_k1 : s_k0);
        float *const stats = reinterpret_cast<float *>(s_v0) + 2 * kWave * (w % 2);
        if (half) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) box[(16 * dt + r) * kWave + lane] = acc[dt][r];
            stats[lane] = shift;
            stats[kWave + lane] = l;
        }
        __syncthreads();
        if (half) return;
        const float shift2 = stats[lane], l2 = stats[kWave + lane];
        const bool none = l == 0.f, none2 = l2 == 0.f;           // (with only NaN seen l is NaN)
        const float to = none ? shift2 : none2 ? shift : fminf(shift, shift2);                   // of the larger maximum
        const float f1 = none ? 0.f : __builtin_amdgcn_exp2f(to - shift), f2 = none2 ? 0.f : __builtin_amdgcn_exp2f(to - shift2);
        l = none2 ? l : fmaf(l2, f2, l * f1);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float x = box[(16 * dt + r) * kWave + lane];
                acc[dt][r] = none2 ? acc[dt][r] : none ? x : fmaf(x, f2, acc[dt][r] * f1);
            }
        shift = to;
    }
    // the lane holds columns 32 dt + 8 q + 4 hw .. + 3 of its row
    if (!row_exists) return;
    if constexpr (!kCodes) {
        if (any_odd) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[dt][r] = seen_odd.result(32 * dt + 8 * (r / 4) + 4 * hw + r % 4, mask, acc[dt][r]);
        }
    }
    const bool whole = a.n_splits == 1;
    const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
    const int64_t at = whole ? out_row : partial_row(a, slot, kvh, row);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            const int64_t to = at * D + 32 * dt + 8 * q4 + 4 * hw;
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = whole && l == 0.f ? 0.f : acc[dt][4 * q4 + i] * inv;
            if (whole && a.o_bf16)
                *reinterpret_cast<uint2 *>(static_cast<char *>(a.o) + 2 * to) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
            else
                *reinterpret_cast<float4 *>((whole ? static_cast<float *>(a.o) : a.part_o) + to) = make_float4(x[0], x[1], x[2], x[3]);
        }
    if (hw == 0) {
        if (whole) {
            a.lse[at] = l == 0.f ? -INFINITY : (__builtin_amdgcn_logf(l) - shift) * kLn2;
        } else {
            a.part_m[at] = l == 0.f ? -INFINITY : -shift;
            a.part_l[at] = l;
        }
    }
}

}  // namespace

hipError_t launch_tree_rows(int head_dim, bool kv8, const TreeArgs &a, int batch, hipStream_t s)
{
    const int64_t streams = (int64_t)a.n_splits * a.sh.n_kv_heads * batch;
    const int64_t blocks = (streams + kXcds - 1) / kXcds * kXcds * a.row_blocks;
    const int flat = a.row_blocks > 1 && blocks <= int64_t(1) << 23 ? 1 : 0;     // (threads of a flat grid are counted in 32 bits)
    const dim3 grid = flat ? dim3((unsigned)blocks) : dim3((unsigned)((int64_t)batch * a.n_splits * a.row_blocks), (unsigned)a.sh.n_kv_heads);
    // rows that pass once and are more than the last cache holds leave the caches alone
    const int streamed = a.row_blocks == 1 && (int64_t)batch * a.sh.n_kv_heads * a.kv.cap * head_dim * (kv8 ? 2 : 4) >= kLastCache ? 1 : 0;
    const bool halves = a.n_q * a.sh.group <= kRowsPerBlock / 2;
#define HGCA_MANY(ST, D)                                                                                                            \
    do {                                                                                                                            \
        if (halves && a.o_bf16) hipLaunchKernelGGL((many_rows_attn_kernel<ST, D, 2, true>), grid, block, 0, s, a, flat, streamed);  \
        else if (halves) hipLaunchKernelGGL((many_rows_attn_kernel<ST, D, 3, true>), grid, block, 0, s, a, flat, streamed);         \
        else if (a.o_bf16) hipLaunchKernelGGL((many_rows_attn_kernel<ST, D, 2, false>), grid, block, 0, s, a, flat, streamed);      \
        else hipLaunchKernelGGL((many_rows_attn_kernel<ST, D, 3, false>), grid, block, 0, s, a, flat, streamed);                    \
    } while (0)
    const dim3 block(kTreeBlock);
    if (kv8 && head_dim == 64) HGCA_MANY(kv8_t, 64);
    else if (kv8) HGCA_MANY(kv8_t, 128);
    else if (head_dim == 64) HGCA_MANY(bf16_t, 64);
    else HGCA_MANY(bf16_t, 128);
#undef HGCA_MANY
    return hipGetLastError();
}

}  // namespace hgca
