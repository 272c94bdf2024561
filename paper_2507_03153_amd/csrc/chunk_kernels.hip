// Attention of packed new tokens, any number per sequence, over one tier, in bf16: causal or not, with a window, a prefix that all see, a
// first token per row (documents), scores capped by a tanh, a bias by distance; and the fold of the shares that several workgroups went
// through.
//
// Work unit: 128 rows (a row is one query of one head of the group), 32 per wave, and a share of the tokens that they see
// (chunk_device.hpp).  K and V of a 64-token step go through a double-buffered LDS stage that all four waves read, brought in by LDS-direct
// loads while the step before is worked on.  Products are 32 x 32 tiles of the matrix cores with the rows in the columns,
//   S^T[token, row] = K . Q^T,  O^T[col, row] += V^T . P^T,
// so that a lane's column is its row in both, a row's maximum and sum need one exchange between the wave's halves, and the scores as they come
// out of the first product are the operand of the second.
// A wave tells by its rows' ranges which steps all of them see (no mask), and which none (left out).
//
// What bounds it: matrix and vector instructions (a weight is an exponential, nine others and a conversion for 768 products), and power, at
// 2.0 GHz of 2.4 on long prompts: two of 4096 tokens, 64 / 8 heads, 562 GFLOP, 795 to 825 us, 680 to 710 TFLOP/s, matrix units busy 48 % of the
// cycles, vector units 54 %.  Capped scores cost eight instructions each (four prompts of 864 tokens over 4096: 329 us, 411 capped; heads of 128 then need all
// 256 registers, and three to eight values wait in scratch memory, outside of the loops).  32 rows
// per wave: with 64 the compiler has no registers left (640 -> 995 us); four waves per workgroup, two workgroups per compute unit: eight waves and
// 256 rows read K and V half as often (661 : 679).  (These with weights of one part.)  Weights enter the second product as two bf16 parts for bf16 O, 16 bits, far
// below its rounding, as three for fp32 O (the same prompts 953 us).  One part, 2^-9 of a weight and with it as much error again as the rounding of O, is there for
// callers that ask for it: prompts 795 -> 655 us (38 % and 49 % busy), mixed step 502 -> 408, documents 495 -> 417; single tokens, whose bound is memory, 169 : 169.
#include <algorithm>

#include "chunk_few.hpp"

namespace hgca {

namespace {

// kinds of instructions for sched_group_barrier: the matrix ones, the other vector ones, LDS reads
constexpr int kSchedMatrix = 0x8, kSchedVector = 0x402, kSchedLds = 0x100;

// Takes infinities and NaN out of a step's V rows, for all waves; true if there were any (settle_odd brings them to the rows that see them).
// Called by waves of which some row does not see all of the step; one that reads the rows before or while they change has sums that are
// not finite.
template <int D> __device__ __forceinline__ bool clean_stage(char *v_stage)
{
    constexpr int kPieces = kChunkStep * 2 * D / 16;
    uint32_t odd = 0;
#pragma unroll 4
    for (int i = threadIdx.x % kWave; i < kPieces; i += kWave) {
        const uint4 x = *reinterpret_cast<const uint4 *>(v_stage + 16 * i);
        odd |= odd_carry(x.x) | odd_carry(x.y) | odd_carry(x.z) | odd_carry(x.w);
    }
    if (!any_lane((odd & kSigns) != 0)) return false;
    for (int i = threadIdx.x % kWave; i < kPieces; i += kWave) {
        uint4 &x = *reinterpret_cast<uint4 *>(v_stage + 16 * i);
        x = make_uint4(x.x & ~odd_halves(x.x), x.y & ~odd_halves(x.y), x.z & ~odd_halves(x.z), x.w & ~odd_halves(x.w));
    }
    return true;
}

// Requests K and V rows of tokens tok .. tok + 63, `there` of which exist (the others repeat the last one).  A load of a wave covers kGroupRows
// rows of one granule, so that in a full step its address is a scalar and an offset that is the lane's for good.
template <int D>
__device__ __forceinline__ void request_step(const ChunkArgs &a, const GranuleRows &rows, int tok, int there, char *k_stage, char *v_stage)
{
    using S = DmaStage<D, kChunkWaves>;
    static_assert(16 % S::kSwizzled == 0 && kChunkWaves * S::kGroupRows % kGranule == 0, "the lane's offsets are those of every group of the wave");
    constexpr int kQuadLanes = 4 * S::kRowBytes / 16;
    typedef const __attribute__((address_space(1))) char *GlobalBytes;
    typedef const __attribute__((address_space(1))) void *GlobalPtr;
    typedef __attribute__((address_space(3))) void *LdsPtr;
    const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), granule = tok / kGranule;
    // what lands at byte 16 * lane of a group: the row inside the group and the byte of the row
    const int k_row = lane / S::kPieces, v_row = 4 * (lane / kQuadLanes) + (lane % 8) / 2;
    const int k_byte = 16 * ((lane % S::kPieces) ^ S::k_swizzle(w * S::kGroupRows + k_row)), v_byte = 16 * (2 * ((lane % kQuadLanes) / 8) + lane % 2);
    const GlobalBytes k = (GlobalBytes)a.kv.k, v = (GlobalBytes)a.kv.v;
    auto scalar = [](GlobalBytes p) {            // keeps the address in scalar registers: the compiler adds the lane's offset to it first
        uint64_t x = (uint64_t)p;
        asm("" : "+s"(x));
        return (GlobalBytes)x;
    };
    if (there >= kChunkStep) {                   // uniform over the workgroup
        const uint32_t k_off = k_row * S::kRowBytes + k_byte, v_off = v_row * S::kRowBytes + v_byte;
#pragma unroll
        for (int u = 0; u < S::kLoads; ++u) {
            const int group = w + kChunkWaves * u, first = group * S::kGroupRows;
            const size_t at = (size_t)(rows.row(granule + first / kGranule) + first % kGranule) * S::kRowBytes;
            __builtin_amdgcn_global_load_lds((GlobalPtr)(scalar(k + at) + k_off), (LdsPtr)(k_stage + group * 1024), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((GlobalPtr)(scalar(v + at) + v_off), (LdsPtr)(v_stage + group * 1024), 16, 0, 0);
        }
        return;
    }
#pragma unroll
    for (int u = 0; u < S::kLoads; ++u) {
        const int group = w + kChunkWaves * u;
        const int kt = min(group * S::kGroupRows + k_row, there - 1), vt = min(group * S::kGroupRows + v_row, there - 1);
        const uint32_t kr = __shfl(rows.now, granule + kt / kGranule - rows.base) + kt % kGranule;
        const uint32_t vr = __shfl(rows.now, granule + vt / kGranule - rows.base) + vt % kGranule;
        __builtin_amdgcn_global_load_lds((GlobalPtr)(k + (size_t)kr * S::kRowBytes + k_byte), (LdsPtr)(k_stage + group * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((GlobalPtr)(v + (size_t)vr * S::kRowBytes + v_byte), (LdsPtr)(v_stage + group * 1024), 16, 0, 0);
    }
}

template <int D, int PP, int MODE>
__global__ __launch_bounds__(kChunkBlock, 2) void chunk_attn_kernel(ChunkArgs a)
{
    using S = DmaStage<D, kChunkWaves>;
    constexpr int KK = D / 16, DT = D / 32, NT = kChunkStep / 32;
    constexpr int kV = 2 * S::kBytes;            // the stages: K of even and odd steps, V of even and odd steps
    __shared__ __attribute__((aligned(4 * S::kBytes))) char s_kv[4 * S::kBytes];
    __shared__ uint32_t s_row[kSub];
    __shared__ int s_odd[kChunkWaves], s_range[2];

    const int kvh = blockIdx.x % a.sh.n_kv_heads;
    Place at;
    at.find<false>(a, blockIdx.x / a.sh.n_kv_heads);
    if (at.idle) return;                         // uniform over the workgroup
    SeqWork seq(a, at.b);
    seq.unify();
    const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = lane % 32, hw = lane / 32;
    const RowPlace rp(a, seq, at.unit, kvh, 32 * w + n);
    const RowSees sees(a, seq, rp.query), all_sees[1] = {sees};
    const WaveSees wave(all_sees);
    int lo, hi;
    unit_range(wave, s_range, lo, hi);
    const Steps steps(seq.pre, lo, hi, at.share, at.n_shares);
    const int64_t unit_rows = ((int64_t)seq.nq << __builtin_ctz(a.sh.group)) - (int64_t)at.unit * kChunkRows;
    if (unit_rows <= kFewTile) {                 // uniform over the workgroup
        FewShared<D> &few = *reinterpret_cast<FewShared<D> *>(s_kv);
        static_assert(sizeof(FewShared<D>) <= sizeof(s_kv), "the waves' results lie in the stages");
        few_rows_bf16<D, PP, MODE>(few, s_row, a, at, seq, steps, kvh);
        return;
    }
    const bool wave_live = any_lane(rp.live);       // uniform over the wave
    uint4 qop[KK];
    {
        const char *const q = a.q + (seq.n0 + rp.query) * a.q_stride + (int64_t)rp.head * S::kRowBytes;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) qop[kk] = load16(q + 16 * (2 * kk + hw));
    }
    const int pos = seq.len - seq.nq + rp.query;
    const ScoreMap<MODE, PP != 1> map(a, rp.head);
    int k_lane[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) k_lane[kk] = S::k_offset(n, 2 * kk + hw);
    const int v_lane = S::v_offset(4 * hw + lane % 16 / 4, lane / 16 % 2) + 8 * (lane % 4);

    bool met_odd = false;                        // uniform over the wave
    Running<DT> run;
    floatx16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = floatx16{};

    // One step.  c[t][r] is the score of step token 32 t + 8 (r / 4) + 4 hw + r % 4; group g of the second product is 16 tokens, of
    // which the lane holds eight.
    auto body = [&](char *stage, int tok) {
        const bool masked = !wave.all(tok, kChunkStep);          // uniform over the wave
        floatx16 c[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) c[t] = floatx16{};
        uint4 kf[KK][NT];
        auto read_slice = [&](int kk) {
#pragma unroll
            for (int t = 0; t < NT; ++t) kf[kk][t] = *reinterpret_cast<const uint4 *>(stage + t * 32 * S::kRowBytes + k_lane[kk]);
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
        if (masked) met_odd = clean_stage<D>(stage + kV) || met_odd;
        uint4 vop[2][DT];
        auto read_v = [&](int g, uint4 (&x)[DT]) {
            const char *v = stage + kV + S::v_offset(16 * g, 0) + v_lane;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const short4v x0 = lds_read_tr16(v + 256 * dt), x1 = lds_read_tr16(v + S::v_offset(8, 0) + 256 * dt);
                const short8v both = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
                x[dt] = __builtin_bit_cast(uint4, both);
            }
        };
        read_v(0, vop[0]);
        __builtin_amdgcn_sched_barrier(0);
        map.apply(c, pos, tok + 4 * hw);
        if (masked) {
            const uint64_t seen = sees.mask(tok + 4 * hw);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(seen >> (32 * t + 8 * (r / 4) + r % 4) & 1)) c[t][r] = -INFINITY;
        }
        run.update(c, map.k2, acc);
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        uint32_t part[PP][4];
        auto weigh = [&](int g) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float p[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    p[x] = __builtin_amdgcn_exp2f(fmaf(c[g / 2][8 * (g % 2) + 2 * e + x], map.k2, run.shift));   // masked scores give 0
                    sum[(2 * e + x) % 4] += p[x];
                }
#pragma unroll
                for (int t = 0; t < PP; ++t) {
                    part[t][e] = pack_bf16(p[0], p[1]);
                    if (t + 1 < PP) {
                        p[0] -= __uint_as_float(part[t][e] << 16);
                        p[1] -= __uint_as_float(part[t][e] & 0xffff0000u);
                    }
                }
            }
        };
        weigh(0);
        // The weights of the next group are worked out between the matrix instructions of this one: left to itself the compiler puts these side by
        // side, and a wave waits for each.
#pragma unroll
        for (int g = 0; g < 2 * NT; ++g) {
            __builtin_amdgcn_sched_barrier(0);
            uint4(&v)[DT] = vop[g % 2];
            if (g + 1 < 2 * NT) read_v(g + 1, vop[(g + 1) % 2]);
            uint32_t now[PP][4];
#pragma unroll
            for (int t = 0; t < PP; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) now[t][e] = part[t][e];
#pragma unroll
            for (int t = 0; t < PP; ++t)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
                    acc[dt] = score_mfma(v[dt], make_uint4(now[t][0], now[t][1], now[t][2], now[t][3]), acc[dt]);
            if (g + 1 < 2 * NT) {
                weigh(g + 1);
                __builtin_amdgcn_sched_group_barrier(kSchedLds, 2 * DT, 0);
#pragma unroll
                for (int i = 0; i < PP * DT; ++i) {
                    __builtin_amdgcn_sched_group_barrier(kSchedMatrix, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kSchedVector, (20 + 16 * PP) / (PP * DT), 0);
                }
            }
        }
        run.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };

    GranuleRows rows(a, at.b, kvh, seq.len);
#pragma unroll 1
    for (int range = 0; range < 2; ++range) {
        const int begin = steps.begin(range), end = steps.end(range);
        if (begin >= end) continue;
        __syncthreads();                         // the stages are no longer in use
        rows.start(begin * (kChunkStep / kGranule));
        request_step<D>(a, rows, begin * kChunkStep, seq.len - begin * kChunkStep, s_kv, s_kv + kV);
        // A step reads the stages of its parity, and the rows of the next one go to those of the other parity, which were last read in
        // the step before: the barrier at its top orders both.
        char *stage = s_kv, *other = s_kv + S::kBytes;
#pragma unroll 1
        for (int s = begin; s < end; ++s) {
            const int tok = s * kChunkStep;
            wait_for_own_loads();                // the barrier alone does not wait for LDS-direct loads
            __syncthreads();
            if (s + 1 < end) {
                rows.reach((tok + kChunkStep) / kGranule);
                request_step<D>(a, rows, tok + kChunkStep, seq.len - tok - kChunkStep, other, other + kV);
            }
            if (wave_live && !wave.none(tok, kChunkStep)) body(stage, tok);
            char *const t = stage;
            stage = other;
            other = t;
        }
    }

    __syncthreads();                             // all waves have read the stages
    OddTokens<D> &notes = *reinterpret_cast<OddTokens<D> *>(s_kv);
    static_assert(sizeof(OddTokens<D>) <= sizeof(s_kv), "the notes lie in a stage");
    settle_odd<bf16_t, D>(a, at.b, kvh, sees, steps, seq.len, met_odd, s_odd, notes, acc);
    store_row<D>(a, at, kvh, rp, halves_sum(run.l), shift_of(run.m, map.k2), acc);
}

// ---- more than 64 sequences: the cut by a launch of its own ----
// (A wave's search of the lists is a chain of loads; 65 sequences over 4096 tokens 230 us, 64 189: the rest is the last round of workgroups.)

constexpr int kCutBlock = 1024, kCutWaves = kCutBlock / kWave;

__global__ __launch_bounds__(kCutBlock) void chunk_cut_kernel(ChunkArgs a)
{
    __shared__ float s_work[kCutWaves];
    __shared__ uint32_t s_sum[4][kCutWaves];
    const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave, B = a.sh.batch;
    auto over_all = [&](float x, bool largest) { // a workgroup's sum or maximum, in every thread
        x = largest ? wave_max(x) : wave_sum(x);
        __syncthreads();
        if (lane == 0) s_work[w] = x;
        __syncthreads();
        x = s_work[0];
#pragma unroll
        for (int i = 1; i < kCutWaves; ++i) x = largest ? fmaxf(x, s_work[i]) : x + s_work[i];
        return x;
    };
    float units = 0.f, work = 0.f, longest = 0.f;
    for (int b = tid; b < B; b += kCutBlock) {
        const SeqWork q(a, b);
        if (q.units == 0) continue;
        units += (float)q.units;
        work += (float)q.units * (float)q.steps;
        longest = fmaxf(longest, (float)q.steps);
    }
    const int c = share_steps(a, over_all(units, false), over_all(work, false), (int)over_all(longest, true), [&](int c) {
        float n = 0.f;
        for (int b = tid; b < B; b += kCutBlock) {
            const SeqWork q(a, b);
            n += (float)q.units * (float)shares_of(q, c);
        }
        return over_all(n, false);
    });
    int32_t *const lists = a.cut + 1;            // four lists of B + 1 beginnings: slots, partials, units with several shares, later slots
    if (tid == 0) a.cut[0] = c;
    if (tid < 4) lists[tid * (B + 1)] = 0;
    // Beginnings that do not ascend may count the same rows for every sequence: sums that no 32 bits hold.  A wave's end at kMost, which is beyond any slot
    // of a launch (2^23 at most), those before at 16 of them.  (A sequence has at most 2^24 shares.)
    constexpr uint32_t kMost = 1u << 26;
    uint32_t base[4] = {0, 0, 0, 0};
    for (int b0 = 0; b0 < B; b0 += kCutBlock) {
        const int b = b0 + tid;
        uint32_t v[4] = {0, 0, 0, 0};
        if (b < B) {
            const SeqWork q(a, b);
            const int n = shares_of(q, c);
            const uint32_t all = (uint32_t)q.units * n;
            v[0] = q.whole_units(a) ? all : 0;
            v[1] = n > 1 ? all : 0;
            v[2] = n > 1 ? q.units : 0;
            v[3] = all - v[0];
        }
        __syncthreads();
        for (int k = 0; k < 4; ++k) {
            v[k] = min(wave_inclusive_scan(v[k]), kMost);
            if (lane == kWave - 1) s_sum[k][w] = v[k];
        }
        __syncthreads();
        for (int k = 0; k < 4; ++k) {
            uint32_t before = base[k];
            for (int i = 0; i < kCutWaves; ++i) {
                before += i < w ? s_sum[k][i] : 0;
                base[k] += s_sum[k][i];
            }
            base[k] = min(base[k], kCutWaves * kMost);
            if (b < B) lists[k * (B + 1) + b + 1] = (int32_t)min(before + v[k], kCutWaves * kMost);
        }
    }
}

// ---- the fold ----
// Bound by memory, 67 MB of partials at most for 512 workgroups of the attention in fp32: 15 us for prompts of 758 tokens over 2048, 5 where few units
// have several shares.

constexpr int kChunkFoldRows = 8;                // rows of a workgroup

// Rows row0 .. of a unit that has several shares, kChunkFoldRows of them or as many as there are left: O = sum o_s 2^(m_s - M) / L, L = sum l_s 2^(m_s -
// M), m_s in powers of 2.  A row's columns are held by D / 4 lanes, four each; where there are fewer rows than a workgroup takes,
// several sets of lanes share a row's partials.
template <int D>
__device__ __forceinline__ void fold_rows(const ChunkArgs &a, const Place &at, const SeqWork &seq, int kvh, int row0, int rows)
{
    constexpr int C4 = D / 4;
    __shared__ float4 s_acc[kChunkFoldRows][C4];
    __shared__ float s_m[kChunkFoldRows], s_l[kChunkFoldRows];
    const int set = threadIdx.x / C4, c4 = threadIdx.x % C4;
    int per_row = 1;                             // sets of lanes that share a row
    while (per_row * 2 * rows <= kChunkFoldRows) per_row *= 2;
    const int mine = set / per_row, r = row0 + min(mine, rows - 1);
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    auto join = [](float &m0, float &l0, float4 &a0, float m1, float l1, const float4 &a1) {
        const float top = fmaxf(m0, m1), to = top == -INFINITY ? 0.f : top;
        const float f0 = __builtin_amdgcn_exp2f(m0 - to), f1 = __builtin_amdgcn_exp2f(m1 - to);
        // an infinity or NaN stays what it is, whatever its share weighs
        auto one = [&](float x, float y) {
            const float p = fabsf(x) < INFINITY ? x * f0 : x, q = fabsf(y) < INFINITY ? y * f1 : y;
            return p + q;
        };
        l0 = one(l0, l1);
        a0 = make_float4(one(a0.x, a1.x), one(a0.y, a1.y), one(a0.z, a1.z), one(a0.w, a1.w));
        m0 = top;
    };
#pragma unroll 4
    for (int s = set % per_row; s < at.n_shares; s += per_row) {
        const int64_t i = ((int64_t)(at.part + s) * a.sh.n_kv_heads + kvh) * kChunkRows + r;
        join(m, l, acc, a.part_m[i], a.part_l[i], *reinterpret_cast<const float4 *>(a.part_o + i * D + 4 * c4));
    }
    if (per_row > 1) {                           // uniform over the workgroup; then there are no further rows
        s_acc[set][c4] = acc;
        if (c4 == 0) {
            s_m[set] = m;
            s_l[set] = l;
        }
        __syncthreads();
        if (set % per_row) return;
        for (int i = 1; i < per_row; ++i) join(m, l, acc, s_m[set + i], s_l[set + i], s_acc[set + i][c4]);
    }
    if (mine >= rows) return;
    const RowPlace rp(a, seq, at.unit, kvh, r);
    const bool none = l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    const float x[4] = {none ? 0.f : acc.x * inv, none ? 0.f : acc.y * inv, none ? 0.f : acc.z * inv, none ? 0.f : acc.w * inv};
    if (a.o_bf16)
        *reinterpret_cast<uint2 *>(static_cast<char *>(a.o) + 2 * (rp.out * D + 4 * c4)) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    else
        *reinterpret_cast<float4 *>(static_cast<float *>(a.o) + rp.out * D + 4 * c4) = make_float4(x[0], x[1], x[2], x[3]);
    if (c4 == 0) a.lse[rp.out] = none ? -INFINITY : (__builtin_amdgcn_logf(l) + m) * kLn2;
}

template <int D>
__global__ __launch_bounds__(kChunkFoldRows * D / 4) void chunk_fold_kernel(ChunkArgs a)
{
    Place at;
    at.find<true>(a, blockIdx.x);
    if (at.idle) return;                         // uniform over the workgroup
    const SeqWork seq(a, at.b);
    const int rows = (int)min(((int64_t)seq.nq << __builtin_ctz(a.sh.group)) - (int64_t)at.unit * kChunkRows, (int64_t)kChunkRows);
    for (int row0 = blockIdx.z * kChunkFoldRows; row0 < rows; row0 += gridDim.z * kChunkFoldRows)
        fold_rows<D>(a, at, seq, blockIdx.y, row0, rows - row0);
}

}  // namespace

hipError_t launch_chunk_rows_bf16(int head_dim, const ChunkArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((int64_t)a.slots * a.sh.n_kv_heads)), block(kChunkBlock);
    const int mode = (a.slopes ? kBiased : 0) + (a.cap > 0.f ? kCapped : 0);
#define HGCA_CHUNK(D, PP)                                                                                          \
    do {                                                                                                           \
        if (mode == kPlainScores) hipLaunchKernelGGL((chunk_attn_kernel<D, PP, kPlainScores>), grid, block, 0, s, a); \
        else if (mode == kCapped) hipLaunchKernelGGL((chunk_attn_kernel<D, PP, kCapped>), grid, block, 0, s, a);   \
        else if (mode == kBiased) hipLaunchKernelGGL((chunk_attn_kernel<D, PP, kBiased>), grid, block, 0, s, a);   \
        else hipLaunchKernelGGL((chunk_attn_kernel<D, PP, kCapped + kBiased>), grid, block, 0, s, a);              \
    } while (0)
    const int parts = !a.o_bf16 ? 3 : a.one_part ? 1 : 2;
    if (head_dim == 64 && parts == 1) HGCA_CHUNK(64, 1);
    else if (head_dim == 64 && parts == 2) HGCA_CHUNK(64, 2);
    else if (head_dim == 64) HGCA_CHUNK(64, 3);
    else if (parts == 1) HGCA_CHUNK(128, 1);
    else if (parts == 2) HGCA_CHUNK(128, 2);
    else HGCA_CHUNK(128, 3);
#undef HGCA_CHUNK
    return hipGetLastError();
}

hipError_t launch_chunk_attn(int dtype, int head_dim, const ChunkArgs &a, hipStream_t s)
{
    hipError_t rc;
    if (a.sh.batch > kWave) {
        hipLaunchKernelGGL(chunk_cut_kernel, dim3(1), dim3(kCutBlock), 0, s, a);
        if ((rc = hipGetLastError()) != hipSuccess) return rc;
    }
    rc = dtype == 0 ? launch_chunk_rows_f32(head_dim, a, s) : launch_chunk_rows_bf16(head_dim, a, s);
    if (rc != hipSuccess || a.parts == 0) return rc;
    // a unit with several shares has two at least; how many there are is known on the device only, and most workgroups of a large grid leave
    // at once
    const int64_t rows = std::min<int64_t>(kChunkRows, (int64_t)a.n_tokens * a.sh.group), units = std::max(std::min(a.parts / 2, a.units), 1);
    int64_t z = (rows + kChunkFoldRows - 1) / kChunkFoldRows;
    while (z > 2 && units * a.sh.n_kv_heads * z > 2048) z = (z + 1) / 2;
    const dim3 grid((unsigned)units, (unsigned)a.sh.n_kv_heads, (unsigned)z);
    if (head_dim == 64) hipLaunchKernelGGL(chunk_fold_kernel<64>, grid, dim3(kChunkFoldRows * 64 / 4), 0, s, a);
    else hipLaunchKernelGGL(chunk_fold_kernel<128>, grid, dim3(kChunkFoldRows * 128 / 4), 0, s, a);
    return hipGetLastError();
}

}  // namespace hgca
