// Block tables and slot maps from the requests' lengths, and rows of packed tokens written by slot.
//
// A plan: sequence b, len tokens in held blocks, is to get n more, so it needs ceil((len + n) / block_size) - held blocks.  Two
// prefix sums over the sequences say who gets what; the k-th granted block is free_blocks[count - 1 - k] (a stack), token t of
// a sequence lies in slot table[pos / block_size] * block_size + pos % block_size with pos = len + t.  A release is the way back:
// the k-th of R blocks goes to free_blocks[count + R - 1 - k], so that a release undoes a plan.
//
// Nothing here has bytes to speak of: one workgroup does the sums (1024 sequences at a time), and the tokens too where they are
// few; more tokens are a second launch of as many workgroups as they fill, which goes by what the first left in scratch.
#include <algorithm>

#include "hgca_launch.hpp"

namespace hgca {

namespace {

constexpr int kPlanBlock = 1024, kPlanWaves = kPlanBlock / kWave;
constexpr int kPlanOneLaunch = 4096;             // tokens that the workgroup of the sums maps itself

constexpr int kContextFull = 2, kBlocksOut = 8, kTokensFull = 16;        // HGCA_CACHE_* bits of the status

__device__ __forceinline__ int64_t wave_scan64(int64_t v) {
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int step = 1; step < kWave; step *= 2) {
        const int64_t o = __shfl_up(v, step);
        if (lane >= step) v += o;
    }
    return v;
}

// Inclusive prefix sums of two values over the workgroup; contains barriers, all threads take part.
struct TwoSums {
    int64_t a, b;
};
__device__ TwoSums scan_two(int64_t a, int64_t b, int64_t (&s)[2][kPlanWaves], TwoSums &total) {
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
    a = wave_scan64(a);
    b = wave_scan64(b);
    __syncthreads();                             // the last use of s is over
    if (lane == kWave - 1) {
        s[0][w] = a;
        s[1][w] = b;
    }
    __syncthreads();
    TwoSums before{0, 0};
    total = TwoSums{0, 0};
#pragma unroll
    for (int i = 0; i < kPlanWaves; ++i) {
        if (i < w) before = TwoSums{before.a + s[0][i], before.b + s[1][i]};
        total = TwoSums{total.a + s[0][i], total.b + s[1][i]};
    }
    return TwoSums{before.a + a, before.b + b};
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
template <bool MAP>
__global__ __launch_bounds__(kPlanBlock) void kv_plan_kernel(PlanArgs a)
{
    __shared__ int64_t s_sums[2][kPlanWaves];
    __shared__ int32_t s_cu[kPlanBlock + 1], s_len[kPlanBlock], s_held[kPlanBlock], s_first[kPlanBlock];
    const int tid = threadIdx.x, bs = a.block_size;
    const int64_t count = min(max(a.free_count[0], 0), a.n_blocks), room = (int64_t)a.max_blocks * bs;
    TwoSums asked{0, 0}, granted{0, 0};          // of the sequences before this round's; a: blocks, b: tokens
    int32_t bits = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kPlanBlock) {
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
        const TwoSums upto = scan_two(need, n, s_sums, all);
        // first come, first served: a sequence that is refused keeps later ones from what it asked for
        const bool blocks = need == 0 || asked.a + upto.a <= count, tokens = n == 0 || asked.b + upto.b <= a.max_tokens;
        if (!blocks) bits |= kBlocksOut;
        if (!tokens) bits |= kTokensFull;
        if (!blocks || !tokens) need = n = 0;
        asked = TwoSums{asked.a + all.a, asked.b + all.b};
        const TwoSums got = scan_two(need, n, s_sums, all);
        const int64_t first = granted.a + got.a - need, cu = granted.b + got.b;
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
            const int end = (int)(granted.b + all.b);
            for (int t = (int)granted.b + tid; t < end; t += kPlanBlock) {
                const int i = segment_of([&](int x) { return s_cu[x]; }, kPlanBlock, t);
                place_token(a, b0 + i, t - s_cu[i], s_len[i], s_held[i], s_first[i], (int)count, t);
            }
        }
        granted = TwoSums{granted.a + all.a, granted.b + all.b};
    }
    if (bits && a.status) atomicOr(a.status, bits);
    if (tid == 0) {
        a.cu[0] = 0;
        a.free_count[0] = (int32_t)(count - granted.a);
        if (!MAP) a.scratch[3 * a.batch] = (int32_t)count;
    }
    if (MAP) {
        for (int t = (int)granted.b + tid; t < a.max_tokens; t += kPlanBlock) {
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
__global__ __launch_bounds__(kPlanBlock) void kv_release_kernel(PlanArgs a)
{
    __shared__ int64_t s_sums[2][kPlanWaves];
    __shared__ int32_t s_upto[kPlanBlock + 1], s_keep[kPlanBlock];
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
    for (int b0 = 0; b0 < a.batch; b0 += kPlanBlock) {
        int32_t len, keep;
        TwoSums all;
        scan_two(share(b0 + tid, len, keep), 0, s_sums, all);
        total += all.a;
    }
    int64_t before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kPlanBlock) {
        const int b = b0 + tid;
        int32_t len, keep;
        TwoSums all;
        const int give = share(b, len, keep);
        const TwoSums upto = scan_two(give, 0, s_sums, all);
        s_upto[tid + 1] = (int32_t)upto.a;
        if (tid == 0) s_upto[0] = 0;
        s_keep[tid] = keep;
        if (b < a.batch) {
            a.lens[b] = len;
            if (give > 0) a.held[b] = keep;
        }
        __syncthreads();
        for (int k = tid; k < (int)all.a; k += kPlanBlock) {
            const int i = segment_of([&](int x) { return s_upto[x]; }, kPlanBlock, k);
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
    const bool one = a.max_tokens <= kPlanOneLaunch;
    if (one) hipLaunchKernelGGL(kv_plan_kernel<true>, dim3(1), dim3(kPlanBlock), 0, s, a);
    else hipLaunchKernelGGL(kv_plan_kernel<false>, dim3(1), dim3(kPlanBlock), 0, s, a);
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess || one) return rc;
    hipLaunchKernelGGL(kv_plan_tokens_kernel, dim3((unsigned)(((int64_t)a.max_tokens + kMapBlock - 1) / kMapBlock)), dim3(kMapBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_kv_release(const PlanArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL(kv_release_kernel, dim3(1), dim3(kPlanBlock), 0, s, a);
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
