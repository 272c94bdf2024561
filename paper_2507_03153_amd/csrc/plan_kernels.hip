// Block tables and slot maps from the requests' lengths, and rows of packed tokens written by slot.
//
// A plan: sequence b, len tokens in held blocks, is to get n more, so it needs ceil((len + n) / block_size) - held blocks.  Two
// prefix sums over the sequences say who gets what; the k-th granted block is free_blocks[count - 1 - k] (a stack), token t of
// a sequence lies in slot table[pos / block_size] * block_size + pos % block_size with pos = len + t.  A release is the way back:
// the k-th of R blocks goes to free_blocks[count + R - 1 - k], so that a release undoes a plan.
//
// Nothing here has bytes to speak of; a chain of loads, sums and barriers bounds it.  One workgroup does the sums, and the tokens too where they
// are few; more tokens are a second launch of as many workgroups as they fill, which goes by what the first left in scratch.  64 sequences
// with a token each: plan 3.5 us, release 2.6 (with 1024 threads 14.9 for both at first, most of it sums in 64 bits and barriers of 16 waves); 512 of
// up to 512 tokens: 4.9 + 5.3 and 6.0.
#include <algorithm>

#include "hgca_launch.hpp"

namespace hgca {

namespace {

// threads of the workgroup of the sums, and the sequences of one round of them (64 tokens of 64 sequences 3.5 : 4.9 us)
constexpr int kPlanSmall = 256, kPlanLarge = 1024;
// tokens that the workgroup of the sums maps itself (1024 of 64 sequences 5.5 us, by two launches 7.0; 4096 9.2 : 7.6; 16 384 of 512 23.7 : 9.2)
constexpr int kPlanOneLaunch = 2048;

constexpr int kContextFull = 2, kBlocksOut = 8, kTokensFull = 16;        // HGCA_CACHE_* bits of the status

// Inclusive prefix sums over the workgroup of N values, and their totals, in 32 bits; contains barriers, all threads take part.
template <int BLOCK, int N>
__device__ __forceinline__ void scan(uint32_t (&v)[N], uint32_t (&total)[N], uint32_t (&s)[N][BLOCK / kWave]) {
    constexpr int W = BLOCK / kWave;
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_inclusive_scan(v[k]);
    __syncthreads();                             // the last use of s is over
    if (lane == kWave - 1) {
#pragma unroll
        for (int k = 0; k < N; ++k) s[k][w] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        total[k] = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            v[k] += i < w ? s[k][i] : 0;
            total[k] += s[k][i];
        }
    }
}

// The same of two values below 2^31 each, whose sums may need more bits: in parts of 20 and 11 bits.
struct TwoSums {
    int64_t a, b;
};
template <int BLOCK>
__device__ __forceinline__ TwoSums scan_two(int64_t a, int64_t b, uint32_t (&s)[4][BLOCK / kWave], TwoSums &total) {
    uint32_t v[4] = {(uint32_t)a & 0xfffffu, (uint32_t)(a >> 20), (uint32_t)b & 0xfffffu, (uint32_t)(b >> 20)}, t[4];
    scan<BLOCK, 4>(v, t, s);
    total = TwoSums{((int64_t)t[1] << 20) + t[0], ((int64_t)t[3] << 20) + t[2]};
    return TwoSums{((int64_t)v[1] << 20) + v[0], ((int64_t)v[3] << 20) + v[2]};
}

// The first index i of ascending at[0 .. n] with at[i + 1] > t, for at[0] <= t < at[n].
template <typename At>
__device__ __forceinline__ int segment_of(At at, int n, int t) {
    int lo = 0, hi = n;                          // at[lo] <= t < at[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (at(mid) <= t) lo = mid; else hi = mid;
    }
    return lo;
}

// Token `i` of a sequence's new ones (len tokens in `held` blocks before, its grant beginning at the `first`-th granted block):
// its position and slot; the first token in a granted block enters the block in the table.
__device__ __forceinline__ void place_token(const PlanArgs &a, int b, int i, int len, int held, int first, int count, int t) {
    const int pos = len + i, blk = pos / a.block_size, off = pos - blk * a.block_size;
    int32_t *const entry = a.table + (int64_t)b * a.max_blocks + blk;
    int32_t where;
    if (blk >= held) {
        where = a.free_blocks[count - 1 - (first + blk - held)];
        if (off == 0 || i == 0) *entry = where;
    } else {
        where = *entry;
    }
    a.positions[t] = pos;
    a.slots[t] = where < 0 ? -1 : where * a.block_size + off;
}

// MAP: the workgroup maps the tokens itself, else it leaves each sequence's old length, old number of blocks and first granted block in scratch.
template <int BLOCK, bool MAP>
__global__ __launch_bounds__(BLOCK) void kv_plan_kernel(PlanArgs a)
{
    __shared__ uint32_t s_sums[4][BLOCK / kWave], s_got[2][BLOCK / kWave];
    __shared__ int32_t s_cu[BLOCK + 1], s_len[BLOCK], s_held[BLOCK], s_first[BLOCK];
    const int tid = threadIdx.x, bs = a.block_size;
    const int64_t count = min(max(a.free_count[0], 0), a.n_blocks), room = (int64_t)a.max_blocks * bs;
    TwoSums asked{0, 0}, granted{0, 0};          // of the sequences before this round's; a: blocks, b: tokens
    int32_t bits = 0;
    for (int b0 = 0; b0 < a.batch; b0 += BLOCK) {
        const int b = b0 + tid;
        const bool real = b < a.batch;
        const int64_t len = real ? max(a.lens[b], 0) : 0, held = real ? min(max(a.held[b], 0), a.max_blocks) : 0;
        int64_t n = real ? max(a.n_new[b], 0) : 0;
        const bool fits = len + n <= room;
        if (!fits) {
            n = 0;
            bits |= kContextFull;
        }
        int64_t need = fits ? max((len + n + bs - 1) / bs - held, (int64_t)0) : 0;
        TwoSums all;
        const TwoSums upto = scan_two<BLOCK>(need, n, s_sums, all);
        // first come, first served: a sequence that is refused keeps later ones from what it asked for
        const bool blocks = need == 0 || asked.a + upto.a <= count, tokens = n == 0 || asked.b + upto.b <= a.max_tokens;
        if (!blocks) bits |= kBlocksOut;
        if (!tokens) bits |= kTokensFull;
        if (!blocks || !tokens) need = n = 0;
        asked = TwoSums{asked.a + all.a, asked.b + all.b};
        // what is granted is at most the free blocks and max_tokens
        uint32_t got[2] = {(uint32_t)need, (uint32_t)n}, sum[2];
        scan<BLOCK, 2>(got, sum, s_got);
        const int64_t first = granted.a + got[0] - need, cu = granted.b + got[1];
        if (real) {
            a.cu[b + 1] = (int32_t)cu;
            if (n > 0) a.lens[b] = (int32_t)(len + n);
            if (need > 0) a.held[b] = (int32_t)(held + need);
            if (!MAP) {
                a.scratch[b] = (int32_t)len;
                a.scratch[a.batch + b] = (int32_t)held;
                a.scratch[2 * a.batch + b] = (int32_t)first;
            }
        }
        if (MAP) {
            s_cu[tid + 1] = (int32_t)cu;
            if (tid == 0) s_cu[0] = (int32_t)granted.b;
            s_len[tid] = (int32_t)len;
            s_held[tid] = (int32_t)held;
            s_first[tid] = (int32_t)first;
            __syncthreads();
            const int end = (int)(granted.b + sum[1]);
            for (int t = (int)granted.b + tid; t < end; t += BLOCK) {
                const int i = segment_of([&](int x) { return s_cu[x]; }, BLOCK, t);
                place_token(a, b0 + i, t - s_cu[i], s_len[i], s_held[i], s_first[i], (int)count, t);
            }
        }
        granted = TwoSums{granted.a + sum[0], granted.b + sum[1]};
    }
    if (bits && a.status) atomicOr(a.status, bits);
    if (tid == 0) {
        a.cu[0] = 0;
        a.free_count[0] = (int32_t)(count - granted.a);
        if (!MAP) a.scratch[3 * a.batch] = (int32_t)count;
    }
    if (MAP) {
        for (int t = (int)granted.b + tid; t < a.max_tokens; t += BLOCK) {
            a.positions[t] = 0;
            a.slots[t] = -1;
        }
    }
}

constexpr int kMapBlock = 256;

__global__ __launch_bounds__(kMapBlock) void kv_plan_tokens_kernel(PlanArgs a)
{
    const int t = blockIdx.x * kMapBlock + threadIdx.x, B = a.batch;
    if (t >= a.max_tokens) return;
    if (t >= a.cu[B]) {
        a.positions[t] = 0;
        a.slots[t] = -1;
        return;
    }
    const int b = segment_of([&](int x) { return a.cu[x]; }, B, t);
    place_token(a, b, t - a.cu[b], a.scratch[b], a.scratch[B + b], a.scratch[2 * B + b], a.scratch[3 * B], t);
}

// What each sequence gives back is counted first: the stack's new top decides where the first block goes.
template <int BLOCK>
__global__ __launch_bounds__(BLOCK) void kv_release_kernel(PlanArgs a)
{
    __shared__ uint32_t s_sums[4][BLOCK / kWave];
    __shared__ int32_t s_upto[BLOCK + 1], s_keep[BLOCK];
    const int tid = threadIdx.x, bs = a.block_size;
    const int64_t count = min(max(a.free_count[0], 0), a.n_blocks);
    auto share = [&](int b, int32_t &len, int32_t &keep) {       // blocks that sequence b gives back
        len = keep = 0;
        if (b >= a.batch) return 0;
        const int held = min(max(a.held[b], 0), a.max_blocks);
        len = min(max(a.new_lens[b], 0), max(a.lens[b], 0));
        keep = min((int)(((int64_t)len + bs - 1) / bs), held);
        return held - keep;
    };
    int64_t total = 0;
    for (int b0 = 0; a.batch > BLOCK && b0 < a.batch; b0 += BLOCK) {         // (one round finds the total on its way)
        int32_t len, keep;
        TwoSums all;
        scan_two<BLOCK>(share(b0 + tid, len, keep), 0, s_sums, all);
        total += all.a;
    }
    int64_t before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += BLOCK) {
        const int b = b0 + tid;
        int32_t len, keep;
        TwoSums all;
        const int give = share(b, len, keep);
        const TwoSums upto = scan_two<BLOCK>(give, 0, s_sums, all);
        if (a.batch <= BLOCK) total = all.a;
        s_upto[tid + 1] = (int32_t)upto.a;
        if (tid == 0) s_upto[0] = 0;
        s_keep[tid] = keep;
        if (b < a.batch) {
            a.lens[b] = len;
            if (give > 0) a.held[b] = keep;
        }
        __syncthreads();
        for (int k = tid; k < (int)all.a; k += BLOCK) {
            const int i = segment_of([&](int x) { return s_upto[x]; }, BLOCK, k);
            const int64_t to = count + total - 1 - (before + k);
            if (to < a.n_blocks)                 // (more blocks than there are: held or count is wrong)
                a.free_blocks[to] = a.table[(int64_t)(b0 + i) * a.max_blocks + s_keep[i] + (k - s_upto[i])];
        }
        before += all.a;
    }
    if (tid == 0) a.free_count[0] = (int32_t)min(count + total, (int64_t)a.n_blocks);
}

// ---- rows of packed tokens ----

constexpr int kWriteBlock = 256;

// Bound by memory: 32 MB of 16 sequences' prompts, 8 heads of 128, bf16, 6.8 us, 4.7 TB/s; 64 tokens 2.4 us, a launch.
// A token's rows of all KV heads are `pieces` of 16 bytes; `lanes` adjacent lanes (a power of two) take a token.  K and V are the grid's
// second dimension.
__global__ __launch_bounds__(kWriteBlock) void kv_write_kernel(WriteArgs a, int lg_lanes, int lg_row_pieces)
{
    const bool value = blockIdx.y != 0;
    const int64_t t = ((int64_t)blockIdx.x * kWriteBlock + threadIdx.x) >> lg_lanes;
    if (t >= a.n_tokens) return;
    const int slot = a.slots[t];
    if (slot < 0 || slot >= a.n_slots) return;   // a token that is not kept
    const int lanes = 1 << lg_lanes, pieces = a.n_kv_heads << lg_row_pieces;
    const int blk = slot / a.per_block, off = slot - blk * a.per_block;
    const char *const in = value ? a.v_in + t * a.v_stride : a.k_in + t * a.k_stride;
    char *const out = value ? a.v : a.k;
    for (int p = threadIdx.x & (lanes - 1); p < pieces; p += lanes) {
        const int head = p >> lg_row_pieces, at = p & ((1 << lg_row_pieces) - 1);
        const int64_t row = ((int64_t)blk * a.n_kv_heads + head) * a.per_block + off;
        *reinterpret_cast<uint4 *>(out + row * a.row_bytes + 16 * at) = load16(in + 16 * p);
    }
}

int log2_up(int64_t x) {
    int lg = 0;
    while ((int64_t(1) << lg) < x) ++lg;
    return lg;
}

}  // namespace

hipError_t launch_kv_plan(const PlanArgs &a, hipStream_t s)
{
    const bool one = a.max_tokens <= kPlanOneLaunch, small = a.batch <= kPlanSmall && a.max_tokens <= kPlanSmall;
    if (small) hipLaunchKernelGGL((kv_plan_kernel<kPlanSmall, true>), dim3(1), dim3(kPlanSmall), 0, s, a);
    else if (one) hipLaunchKernelGGL((kv_plan_kernel<kPlanLarge, true>), dim3(1), dim3(kPlanLarge), 0, s, a);
    else hipLaunchKernelGGL((kv_plan_kernel<kPlanLarge, false>), dim3(1), dim3(kPlanLarge), 0, s, a);
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess || one) return rc;
    hipLaunchKernelGGL(kv_plan_tokens_kernel, dim3((unsigned)(((int64_t)a.max_tokens + kMapBlock - 1) / kMapBlock)), dim3(kMapBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_kv_release(const PlanArgs &a, hipStream_t s)
{
    if (a.batch <= kPlanSmall) hipLaunchKernelGGL(kv_release_kernel<kPlanSmall>, dim3(1), dim3(kPlanSmall), 0, s, a);
    else hipLaunchKernelGGL(kv_release_kernel<kPlanLarge>, dim3(1), dim3(kPlanLarge), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_kv_write(const WriteArgs &a, hipStream_t s)
{
    const int lg_row = log2_up(a.row_bytes / 16);                // rows have 128, 256 or 512 bytes
    const int lg_lanes = std::min(log2_up((int64_t)a.n_kv_heads << lg_row), log2_up(kWriteBlock));
    const int64_t blocks = (((int64_t)a.n_tokens << lg_lanes) + kWriteBlock - 1) / kWriteBlock;
    hipLaunchKernelGGL(kv_write_kernel, dim3((unsigned)blocks, 2), dim3(kWriteBlock), 0, s, a, lg_lanes, lg_row);
    return hipGetLastError();
}

}  // namespace hgca
