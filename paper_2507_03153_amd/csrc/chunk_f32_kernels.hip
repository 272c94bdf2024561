// Attention of packed new tokens over one tier in fp32 (chunk_kernels.hip has the same in bf16, and the fold): both products on the fp32 matrix
// instructions, whose products and sums are fp32 ones, over the whole range of the type.
//
// The unit of work and the tiles are those of the bf16 kernel, the stages half a step: 32 tokens of K and V, twice.  A lane reads 16 bytes of a
// K row, which are an operand of four instructions (the order of the columns is free), and one V value per instruction: register r of the
// scores is token 8 (r / 4) + 4 hw + r % 4, the two tokens of an instruction.
//
// What bounds it: the matrix cores, 64 cycles of a SIMD for 32 x 32 x 2.  A prompt of 4096 tokens, 32 / 8 heads, 137 GFLOP, 1220 us, 113 TFLOP/s of the 154
// that a large product reaches; four prompts, 758 tokens over 2048, 197 to 219 us, of which the fold is 15: matrix units are busy 69 % of the time that
// the compute units have work, which they have 81 % of the time, shares of five steps having a start and an end of their own.  (Operands read two pairs of pieces ahead: level, the
// other workgroup's waves fill the gaps.)
#include <algorithm>

#include "chunk_few.hpp"

namespace hgca {

namespace {

constexpr int kHalfStep = 32;

// 16-byte pieces of a row in LDS lie at (piece ^ row): the rows of an operand's lanes are on different banks.
template <int D> struct StageF32 {
    static constexpr int kRowBytes = 4 * D, kPieces = D / 4, kBytes = kHalfStep * kRowBytes;
    static constexpr int kGroupRows = 1024 / kRowBytes, kLoads = kHalfStep / kGroupRows / kChunkWaves;
    static __device__ __forceinline__ int offset(int row, int piece) { return row * kRowBytes + 16 * (piece ^ (row % kPieces)); }
};

// Tokens 32 step .. of the pass, by LDS-direct loads; tokens behind its end read its last row.
template <int D>
__device__ __forceinline__ void load_half_step(const KvDev &kv, const BlockRows &rows, int step, int nsub, char *k_stage, char *v_stage)
{
    using S = StageF32<D>;
    typedef const __attribute__((address_space(1))) void *GlobalPtr;
    typedef __attribute__((address_space(3))) void *LdsPtr;
    const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    uint32_t row[S::kLoads];
    int at[S::kLoads];
#pragma unroll
    for (int u = 0; u < S::kLoads; ++u) {
        const int r = (w + kChunkWaves * u) * S::kGroupRows + lane / S::kPieces;
        const uint32_t t = min(step * kHalfStep + r, nsub - 1);
        row[u] = rows.table ? rows.table[t / kGranule] + t % kGranule : rows.base + t;
        at[u] = 16 * (lane % S::kPieces ^ r % S::kPieces);
    }
#pragma unroll
    for (int u = 0; u < S::kLoads; ++u) {
        const size_t from = (size_t)row[u] * S::kRowBytes + at[u];
        __builtin_amdgcn_global_load_lds((GlobalPtr)(kv.k + from), (LdsPtr)(k_stage + (w + kChunkWaves * u) * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((GlobalPtr)(kv.v + from), (LdsPtr)(v_stage + (w + kChunkWaves * u) * 1024), 16, 0, 0);
    }
}

// Takes infinities and NaN out of a half step's V rows, for all waves; true if there were any (settle_odd brings them to the rows that see them).
// Called by waves of which some row does not see all of it; one that reads the rows before or while they change has sums that are not
// finite.
template <int D> __device__ __forceinline__ bool clean_half_stage(char *v_stage)
{
    constexpr int kPieces = kHalfStep * D / 4;
    bool odd = false;
#pragma unroll 4
    for (int i = threadIdx.x % kWave; i < kPieces; i += kWave) {
        const float4 x = *reinterpret_cast<const float4 *>(v_stage + 16 * i);
        odd = odd || !(fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(x.z), fabsf(x.w))) < INFINITY) || x.x != x.x || x.y != x.y || x.z != x.z || x.w != x.w;
    }
    if (!any_lane(odd)) return false;
    auto finite = [](float x) { return fabsf(x) < INFINITY ? x : 0.f; };
    for (int i = threadIdx.x % kWave; i < kPieces; i += kWave) {
        float4 &x = *reinterpret_cast<float4 *>(v_stage + 16 * i);
        x = make_float4(finite(x.x), finite(x.y), finite(x.z), finite(x.w));
    }
    return true;
}

template <int D, int MODE>
__global__ __launch_bounds__(kChunkBlock, 2) void chunk_attn_f32_kernel(ChunkArgs a)
{
    using S = StageF32<D>;
    constexpr int KP = D / 8, DT = D / 32;       // pairs of pieces of a row, column tiles
    constexpr int kV = 2 * S::kBytes;            // the stages: K of even and odd half steps, V of even and odd ones
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
    if (unit_rows <= kFewRows) {                 // uniform over the workgroup
        FewShared<D> &few = *reinterpret_cast<FewShared<D> *>(s_kv);
        static_assert(sizeof(FewShared<D>) <= sizeof(s_kv), "the waves' results lie in the stages");
        if (unit_rows <= kFewTile) few_rows_f32<D, MODE, 1>(few, s_row, a, at, seq, steps, kvh);
        else few_rows_f32<D, MODE, 2>(few, s_row, a, at, seq, steps, kvh);
        return;
    }
    const bool wave_live = any_lane(rp.live);       // uniform over the wave
    float4 qop[KP];
    {
        const char *const q = a.q + (seq.n0 + rp.query) * a.q_stride + (int64_t)rp.head * S::kRowBytes;
#pragma unroll
        for (int j = 0; j < KP; ++j) qop[j] = __builtin_bit_cast(float4, load16(q + 16 * (2 * j + hw)));
    }
    const int pos = seq.len - seq.nq + rp.query;
    const ScoreMap<MODE, true> map(a, rp.head);
    int v_lane[4];                               // of token 4 hw + i, columns n / 4 ..
#pragma unroll
    for (int i = 0; i < 4; ++i) v_lane[i] = (4 * hw + i) * S::kRowBytes + 16 * ((n / 4) ^ (4 * hw + i)) + 4 * (n % 4);

    bool met_odd = false;                        // uniform over the wave
    Running<DT> run;
    floatx16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = floatx16{};

    auto body = [&](char *stage, int tok) {
        const bool masked = !wave.all(tok, kHalfStep);           // uniform over the wave
        floatx16 c[1] = {floatx16{}};
#pragma unroll
        for (int j = 0; j < KP; ++j) {
            const float4 k = *reinterpret_cast<const float4 *>(stage + S::offset(n, 2 * j + hw));
            c[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.x, qop[j].x, c[0], 0, 0, 0);
            c[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.y, qop[j].y, c[0], 0, 0, 0);
            c[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.z, qop[j].z, c[0], 0, 0, 0);
            c[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.w, qop[j].w, c[0], 0, 0, 0);
        }
        map.apply(c, pos, tok + 4 * hw);
        if (masked) {
            met_odd = clean_half_stage<D>(stage + kV) || met_odd;
            const uint64_t seen = sees.mask(tok + 4 * hw);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (!(seen >> (8 * (r / 4) + r % 4) & 1)) c[0][r] = -INFINITY;
        }
        run.update(c, map.k2, acc);
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float p = __builtin_amdgcn_exp2f(fmaf(c[0][r], map.k2, run.shift));            // masked scores give 0
            sum[r % 4] += p;
            // piece 8 dt + n / 4 of row 8 (r / 4) + 4 hw + r % 4 lies at their exclusive or
            const char *const v = stage + kV + 8 * (r / 4) * S::kRowBytes + v_lane[r % 4];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const float x = *reinterpret_cast<const float *>(v + 128 * (dt ^ (r / 4) % (S::kPieces / 8)));
                acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, p, acc[dt], 0, 0, 0);
            }
        }
        run.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };

#pragma unroll 1
    for (int range = 0; range < 2; ++range) {
        const int from = steps.begin(range) * kChunkStep, total = min(steps.end(range) * kChunkStep, seq.len) - from;
        const int sub_len = pass_length(a.kv, total);
#pragma unroll 1
        for (int sub0 = 0; sub0 < total; sub0 += sub_len) {
            const int nsub = min(sub_len, total - sub0), first = from + sub0, count = (nsub + kHalfStep - 1) / kHalfStep;
            __syncthreads();                     // the previous table and stages are no longer in use
            const BlockRows where = make_block_rows<kChunkBlock>(s_row, a.kv, a.sh.n_kv_heads, at.b, kvh, first, nsub);
            load_half_step<D>(a.kv, where, 0, nsub, s_kv, s_kv + kV);
            // Half step s reads the stages of its parity, and the rows of s + 1 go to those of the other parity, which were last read in
            // s - 1: the barrier at its top orders both.
#pragma unroll 1
            for (int s = 0; s < count; ++s) {
                wait_for_own_loads();            // the barrier alone does not wait for LDS-direct loads
                __syncthreads();
                char *const next = s_kv + (s + 1) % 2 * S::kBytes;
                if (s + 1 < count) load_half_step<D>(a.kv, where, s + 1, nsub, next, next + kV);
                const int tok = first + s * kHalfStep;
                if (wave_live && !wave.none(tok, kHalfStep)) body(s_kv + s % 2 * S::kBytes, tok);
            }
        }
    }

    __syncthreads();                             // all waves have read the stages
    OddTokens<D> &notes = *reinterpret_cast<OddTokens<D> *>(s_kv);
    static_assert(sizeof(OddTokens<D>) <= sizeof(s_kv), "the notes lie in a stage");
    settle_odd<float, D>(a, at.b, kvh, sees, steps, seq.len, met_odd, s_odd, notes, acc);
    store_row<D>(a, at, kvh, rp, halves_sum(run.l), shift_of(run.m, map.k2), acc);
}

}  // namespace

hipError_t launch_chunk_rows_f32(int head_dim, const ChunkArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((int64_t)a.slots * a.sh.n_kv_heads)), block(kChunkBlock);
    const int mode = (a.slopes ? kBiased : 0) + (a.cap > 0.f ? kCapped : 0);
#define HGCA_CHUNK(D)                                                                                                \
    do {                                                                                                             \
        if (mode == kPlainScores) hipLaunchKernelGGL((chunk_attn_f32_kernel<D, kPlainScores>), grid, block, 0, s, a); \
        else if (mode == kCapped) hipLaunchKernelGGL((chunk_attn_f32_kernel<D, kCapped>), grid, block, 0, s, a);     \
        else if (mode == kBiased) hipLaunchKernelGGL((chunk_attn_f32_kernel<D, kBiased>), grid, block, 0, s, a);     \
        else hipLaunchKernelGGL((chunk_attn_f32_kernel<D, kCapped + kBiased>), grid, block, 0, s, a);                \
    } while (0)
    if (head_dim == 64) HGCA_CHUNK(64);
    else HGCA_CHUNK(128);
#undef HGCA_CHUNK
    return hipGetLastError();
}

}  // namespace hgca
