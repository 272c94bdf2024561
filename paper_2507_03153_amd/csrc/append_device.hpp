// What the append kernels in bf16 and in fp32 share: where rows live, which row of the launch is which query and head, the
// layouts of the tiles in LDS that the matrix operands are read from.
#pragma once

#include "hgca_launch.hpp"
#include "row_map.hpp"

namespace hgca {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));

constexpr int kStepBlocks = 2;                   // 32-token contraction blocks per step
constexpr int kStepTokens = 32 * kStepBlocks;
constexpr int kRowsPerBlock = 128;               // query rows of a workgroup
constexpr int kAttnWaves = kRowsPerBlock / 32, kAttnBlock = kAttnWaves * kWave;   // of the attention: a wave owns 32 of them
constexpr int kSub = kMaxChunk;                  // entries of the table of rows (paged tiers)
static_assert(kStepTokens == kLineStep, "shares of a line are whole steps");
static_assert(kSub * 16 % kStepTokens == 0, "a pass is a whole number of steps");

// Where the rows of a pass over part of a split live.  A contiguous tier is plain arithmetic.  A paged tier gets a
// table in LDS with one entry per 16 tokens (block sizes are multiples of 16: the row of the granule's first token for
// this KV head), so a lookup is a shift, whatever the block size, and one filling of kSub entries covers a whole split
// and the load pipeline is not drained for refills.
constexpr int kGranule = 16;
struct BlockRows {
    const uint32_t *table;                       // LDS; nullptr => row = base + j
    uint32_t base;
};

// tokens a pass may cover so that its granules fit the table, a multiple of the step
__device__ __forceinline__ int pass_length(const KvDev &kv, int nt_total) {
    return kv.block_table ? kSub * kGranule : max(nt_total, 1);
}

// `first` is the tier position of the pass's first token, a multiple of kGranule (splits and passes are cut at whole
// steps), nt the number of tokens; contains a barrier iff the tier is paged (uniform over the workgroup).
template <int BLOCK>
__device__ __forceinline__ BlockRows make_block_rows(uint32_t *s_tab, const KvDev &kv, int n_kv_heads, int b, int kvh,
                                                     int first, int nt)
{
    BlockRows m;
    if (!kv.block_table) {
        m.table = nullptr;
        m.base = (uint32_t)(((int64_t)b * n_kv_heads + kvh) * kv.cap + first);
        return m;
    }
    const int32_t *blocks = kv.block_table + (int64_t)b * kv.max_blocks + (kv.first_block ? kv.first_block[b] : 0);
    const int n_gr = (nt + kGranule - 1) / kGranule;             // <= kSub by pass_length
    for (int i = threadIdx.x; i < n_gr; i += BLOCK) {
        const int tok = first + i * kGranule;
        s_tab[i] = (uint32_t)(((int64_t)blocks[tok / kv.block_size] * n_kv_heads + kvh) * kv.block_size + tok % kv.block_size);
    }
    __syncthreads();
    m.table = s_tab;
    m.base = 0;
    return m;
}

// Reductions over the two halves of a wave (lanes n and n + 32 hold partial results of one query row):
// v_permlane32_swap of a register with itself returns the lower half twice and the upper half twice, one VALU
// instruction where a lane shuffle would go through the LDS pipeline.
__device__ __forceinline__ float halves_max(float x) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Where a query row of a (sequence, KV head) pair lives: query r / G, head r % G of the group.
struct RowInfo {
    bool valid;
    int query;
    int64_t out_row;                             // (b * N + query) * Hq + head
};

template <int G>
__device__ __forceinline__ RowInfo row_info(const AppendArgs &a, int b, int kvh, int r) {
    RowInfo ri;
    ri.valid = r < a.n_q * G;
    ri.query = ri.valid ? r / G : 0;
    ri.out_row = ((int64_t)b * a.n_q + ri.query) * a.sh.n_q_heads + kvh * G + (ri.valid ? r % G : 0);
    return ri;
}

constexpr int kXcds = 8;                         // workgroups of a launch are dealt to the XCDs in turn
constexpr int kWTile = 32;                       // tokens of a wave's tile in the weights pass
constexpr int kWManyRowTokens = 2048;            // tokens of a block that more than one pass over the rows goes through

// LDS stage of the attention kernel: the rows of a step are brought in by LDS-direct loads (global_load_lds, 16
// bytes per lane, no registers in between).  One such instruction fills 1024 consecutive bytes of LDS with whatever
// 64 pieces its lanes address, so the layout inside each 1 KB group is chosen by the lane -> global address map:
//   K: row-major rows with the 16-byte pieces of a row XOR-swizzled by the row, so that the 16 rows an A-operand
//      read touches land on different banks without padding;
//   V: quads of four rows, interleaved in 32-byte chunks ([quad][column chunk][row of the quad][32 bytes]), so that
//      the 4 rows x 32 bytes a 16-lane group takes with one transpose read are 128 consecutive bytes and the two
//      groups of a half wave, which take neighbouring chunks, 256.
template <int D, int NW> struct DmaStage {
    static constexpr int kRowBytes = D * 2;
    static constexpr int kPieces = kRowBytes / 16;               // 16-byte pieces per row
    static constexpr int kSwizzled = kPieces < 16 ? kPieces : 16;
    static constexpr int kGroupRows = 1024 / kRowBytes;          // rows per load instruction of a wave
    static constexpr int kGroups = kStepTokens / kGroupRows;     // per step and tensor
    static constexpr int kLoads = kGroups / NW;                  // per wave, step and tensor
    static constexpr int kBytes = kStepTokens * kRowBytes;       // per step and tensor
    static_assert(kGroups % NW == 0 && kLoads >= 1, "the waves share the groups of a step evenly");

    static __device__ __forceinline__ int k_swizzle(int row) { return (row / (16 / kSwizzled)) % kSwizzled; }
    // byte offset, in a K stage, of logical piece `piece` of step row `row`
    static __device__ __forceinline__ int k_offset(int row, int piece) {
        return row * kRowBytes + 16 * (piece ^ k_swizzle(row));
    }
    // byte offset, in a V stage, of the 32-byte column chunk `dt` of step row `row`
    static __device__ __forceinline__ int v_offset(int row, int dt) {
        return (row / 4) * (4 * kRowBytes) + dt * 128 + (row % 4) * 32;
    }
};

constexpr int kNonTemporal = 2;                  // cache policy of a load: streamed once
constexpr int64_t kLastCache = int64_t(256) << 20;

// s_waitcnt vmcnt(0) (expcnt and lgkmcnt fields at their maxima = no wait): an LDS-direct load has landed in LDS
// when the wave's memory-load counter has counted it down.  Every wave does this before the barrier after which
// other waves read what it loaded.
__device__ __forceinline__ void wait_for_own_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// Requests the K and the V rows of a step.  A load instruction of a wave covers kGroupRows rows of one granule, so in
// a full step its address is a scalar (the granule's row) plus an offset that is the lane's for good; only a step
// that the pass's end cuts computes rows per lane (tokens behind the end read the last row).  The row numbers of a
// paged tier are looked up before the first load is issued: an LDS read placed after an LDS-direct load waits for it.
// POLICY_K and POLICY_V are the loads' cache policies: 0, or kNonTemporal where the rows are not to stay in the caches.
template <int D, int NW, int POLICY_K, int POLICY_V>
__device__ __forceinline__ void dma_step(const KvDev &kv, const BlockRows &rows, int step, int nsub, char *k_stage,
                                         char *v_stage)
{
    using S = DmaStage<D, NW>;
    static_assert(kGranule % S::kGroupRows == 0, "a load stays inside a granule");
    constexpr int kQuadLanes = 4 * S::kRowBytes / 16;
    const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    // what lands at byte 16 * lane of the wave's u-th group: the row inside the group and the byte of the row
    const int k_row = lane / S::kPieces, v_row = 4 * (lane / kQuadLanes) + (lane % 8) / 2;
    auto k_byte = [&](int u) { return 16 * ((lane % S::kPieces) ^ S::k_swizzle((w + NW * u) * S::kGroupRows + k_row)); };
    const int v_byte = 16 * (2 * ((lane % kQuadLanes) / 8) + lane % 2);
    typedef const __attribute__((address_space(1))) void *GlobalPtr;
    typedef __attribute__((address_space(3))) void *LdsPtr;
    if ((step + 1) * kStepTokens <= nsub) {                      // uniform over the workgroup
        const int first = step * kStepTokens + w * S::kGroupRows;                        // of the wave's first load
        uint32_t row[S::kLoads];                                 // uniform over the wave
#pragma unroll
        for (int u = 0; u < S::kLoads; ++u) row[u] = rows.base + first + NW * S::kGroupRows * u;
        if (rows.table) {
#pragma unroll
            for (int u = 0; u < S::kLoads; ++u) row[u] = rows.table[(first + NW * S::kGroupRows * u) / kGranule];
#pragma unroll
            for (int u = 0; u < S::kLoads; ++u)
                row[u] = __builtin_amdgcn_readfirstlane(row[u]) + (first + NW * S::kGroupRows * u) % kGranule;
        }
#pragma unroll
        for (int u = 0; u < S::kLoads; ++u) {
            const size_t at = (size_t)row[u] * S::kRowBytes;
            const uint32_t k_off = k_row * S::kRowBytes + k_byte(u), v_off = v_row * S::kRowBytes + v_byte;
            __builtin_amdgcn_global_load_lds((GlobalPtr)(kv.k + at + k_off), (LdsPtr)(k_stage + (w + NW * u) * 1024), 16, 0, POLICY_K);
            __builtin_amdgcn_global_load_lds((GlobalPtr)(kv.v + at + v_off), (LdsPtr)(v_stage + (w + NW * u) * 1024), 16, 0, POLICY_V);
        }
        return;
    }
    uint32_t kr[S::kLoads], vr[S::kLoads];
#pragma unroll
    for (int u = 0; u < S::kLoads; ++u) {
        const int first = step * kStepTokens + (w + NW * u) * S::kGroupRows;
        const uint32_t kt = min(first + k_row, nsub - 1), vt = min(first + v_row, nsub - 1);
        kr[u] = rows.table ? rows.table[kt / kGranule] + kt % kGranule : rows.base + kt;
        vr[u] = rows.table ? rows.table[vt / kGranule] + vt % kGranule : rows.base + vt;
    }
#pragma unroll
    for (int u = 0; u < S::kLoads; ++u) {
        __builtin_amdgcn_global_load_lds((GlobalPtr)(kv.k + (size_t)kr[u] * S::kRowBytes + k_byte(u)),
                                         (LdsPtr)(k_stage + (w + NW * u) * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((GlobalPtr)(kv.v + (size_t)vr[u] * S::kRowBytes + v_byte),
                                         (LdsPtr)(v_stage + (w + NW * u) * 1024), 16, 0, 0);
    }
}

// One 16-byte slice of the score contraction in bf16: C[32 x 32] += A . B over 16 columns.  A lane holds 16 bytes of row
// lane % 32 of either operand, the lower half of the wave one piece and the upper half the next.
__device__ __forceinline__ floatx16 score_mfma(const uint4 &a, const uint4 &b, floatx16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

}  // namespace

}  // namespace hgca
