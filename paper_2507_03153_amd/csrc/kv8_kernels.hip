// An older pool in 8 bits: rows of K and V as E4M3 values with one power of two per 32 adjacent columns (E8M0), 1.03 bytes per
// element, the block format whose conversions gfx950 has as instructions.
//
// The scale of a block is the least 2^e, e >= -110, with amax <= 448 * 2^e (448 is E4M3's largest value): nothing is cut off
// and a value of the upper binades keeps 4 significant bits.  x * 2^-e is exact, so the one rounding is E4M3's (half a
// step, 2^-4 of a normal value, 2^(e - 10) below 2^(e - 6)).  With e >= -110 every code stands for a normal bf16 and fp32 number,
// which is what makes reading back, as rows or as matrix operands, exact; at the other end what would round to
// 2^128 is 240 * 2^120.  An infinity or NaN becomes NaN and leaves
// the scale of its block alone.
#include <algorithm>

#include "hgca_launch.hpp"
#include "kv8_device.hpp"

namespace hgca {

namespace {

constexpr int kKv8Block = 256;

// Rows in bf16 are streamed past the caches on their way in and out (codes, which attention reads next, are not): 8 x 4096 tokens of 8
// heads of 128 written and read back 95.5 -> 76.8 us (407 MB, 5.3 TB/s; only in or only out 79 and 80), new tokens 89.2 -> 70.6.
// (fp32 is not: a lane has 32 bytes, each of its two accesses meets half of a line; 4 x 2000 tokens 34.9 -> 45.4.)
template <typename T> __device__ __forceinline__ void load8(const char *p, float *f);
template <> __device__ __forceinline__ void load8<float>(const char *p, float *f) {
    Elem<float>::expand(load16(p), f);
    Elem<float>::expand(load16(p + 16), f + 4);
}
template <> __device__ __forceinline__ void load8<bf16_t>(const char *p, float *f) { Elem<bf16_t>::expand(load16_stream(p), f); }

// Eight adjacent columns of a row per lane, a block of 32 per quad of lanes: its largest magnitude takes two lane exchanges.
__device__ __forceinline__ uint2 encode8(const float *x, uint32_t &code) {
    uint32_t top = 0;                            // magnitudes as integers are ordered as the numbers are
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t m = __float_as_uint(x[i]) & 0x7fffffffu;
        top = max(top, m < 0x7f800000u ? m : 0u);
    }
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, kDppXor1, 0xf, 0xf, true));
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, kDppXor2, 0xf, 0xf, true));
    // biased exponent of amax, less 8 (2^8 <= 448 < 2^9), one more where its significand is above 448 / 256 = 1.75
    const int e = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    code = (uint32_t)max(e, kKv8LeastScale);
    const float inv = __uint_as_float((254u - code) << 23);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i] * inv;
    if (code == kKv8TopScale) {                  // 256 * 2^120 is no fp32 number (infinities and NaN are not touched)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (fabsf(y[i]) <= 256.f) y[i] = fminf(fmaxf(y[i], -240.f), 240.f);
    }
    int w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], w[i], false);
        w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w[i], true);
    }
    return make_uint2((uint32_t)w[0], (uint32_t)w[1]);
}

// The scales of a row's blocks as one word, in every lane of the row: quad q of the D / 8 lanes holds block q's.
template <int D> __device__ __forceinline__ uint32_t row_scales(uint32_t code, int lane) {
    uint32_t s = code << (8 * (lane % (D / 8) / 4));
    s |= (uint32_t)__builtin_amdgcn_mov_dpp((int)s, kDppHalfMirror, 0xf, 0xf, true);
    if (D == 128) s |= (uint32_t)__builtin_amdgcn_mov_dpp((int)s, kDppRor8, 0xf, 0xf, true);
    return s;
}

// Row of position p of a sequence and KV head, counted over the whole tier.
__device__ __forceinline__ uint32_t row_of(const KvDev &kv, const int32_t *blocks, int n_kv_heads, int b, int h, int p) {
    if (!blocks) return (uint32_t)(((int64_t)b * n_kv_heads + h) * kv.cap + p);
    return (uint32_t)(((int64_t)blocks[p / kv.block_size] * n_kv_heads + h) * kv.block_size + p % kv.block_size);
}

__device__ __forceinline__ const int32_t *blocks_of(const KvDev &kv, int b) {
    return kv.block_table ? kv.block_table + (int64_t)b * kv.max_blocks + (kv.first_block ? kv.first_block[b] : 0) : nullptr;
}

// positions a sequence's tier has room for: its capacity, or what is left of its table row
__device__ __forceinline__ int room_of(const KvDev &kv, int b) {
    if (!kv.block_table) return kv.cap;
    const int64_t left = (int64_t)(kv.max_blocks - (kv.first_block ? kv.first_block[b] : 0)) * kv.block_size;
    return (int)min((int64_t)kv.cap, max(left, (int64_t)0));
}

// Which rows a workgroup goes through: D / 8 lanes per row of K and of V, so 16 or 32 rows at a time, of `tokens_at_once` tokens (a
// power of two) of one KV head, or of few tokens of several heads; then the next ones, gridDim.x workgroups apart.  No division
// but the one by the block size.
template <int D> struct RowWalk {
    static constexpr int kRows = kKv8Block / (D / 8);
    int head, token, step;
    __device__ __forceinline__ explicit RowWalk(int lg_tokens) {
        const int row = threadIdx.x / (D / 8), at_once = 1 << lg_tokens;
        head = (int)blockIdx.y * (kRows >> lg_tokens) + (row >> lg_tokens);
        token = (int)blockIdx.x * at_once + (row & (at_once - 1));
        step = (int)gridDim.x * at_once;
    }
};
// Rows of a thread whose loads are in flight together; rows of fp32 are long enough one at a time.  8 x 4096 tokens of 8 heads of 128 written
// and read back, 4 : 2 : 1 rows, us: bf16 90 to 97 : 94 to 96 : 94 to 97 (with a division per row 99 to 105), heads of 64 40.8 : 43.6 : 43;
// 4 x 2000 tokens in fp32 41.6 : 36.6 : 34.9.
template <typename T> constexpr int kTogether = sizeof(T) == 2 ? 4 : 1;

// FROM_TIER: rows of the same positions of another tier; else rows [B, n, Hkv, d].
template <typename T, int D, bool FROM_TIER>
__global__ __launch_bounds__(kKv8Block) void kv8_write_kernel(Kv8WriteArgs a)
{
    constexpr int LR = D / 8, RB = D * (int)sizeof(T);
    const int b = blockIdx.z, lane = threadIdx.x % kWave, sub = threadIdx.x % LR;
    const int first = max(a.first ? a.first[b] : 0, 0);
    int n = a.n_tokens;
    if (FROM_TIER) n = min(n, max(tier_len(a.src, b) - first, 0));
    const int room = max(room_of(a.dst, b) - first, 0);
    if (n > room) {
        if (a.status && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(a.status, kCacheContextFull);
        n = room;
    }
    const int32_t *to = blocks_of(a.dst, b), *from = FROM_TIER ? blocks_of(a.src, b) : nullptr;
    const RowWalk<D> walk(a.lg_tokens);
    if (walk.head >= a.n_kv_heads) return;
    for (int64_t t0 = walk.token; t0 < n; t0 += (int64_t)kTogether<T> * walk.step) {
        float k[kTogether<T>][8], v[kTogether<T>][8];
#pragma unroll
        for (int u = 0; u < kTogether<T>; ++u) {    // (behind the last token: the last one again)
            const int t = (int)min(t0 + (int64_t)u * walk.step, (int64_t)n - 1);
            const size_t row = FROM_TIER ? row_of(a.src, from, a.n_kv_heads, b, walk.head, first + t)
                                         : ((size_t)b * a.n_tokens + t) * a.n_kv_heads + walk.head;
            load8<T>(a.src.k + row * RB + sub * 8 * sizeof(T), k[u]);
            load8<T>(a.src.v + row * RB + sub * 8 * sizeof(T), v[u]);
        }
#pragma unroll
        for (int u = 0; u < kTogether<T>; ++u) {
            const int64_t t = t0 + (int64_t)u * walk.step;
            if (t >= n) break;                   // (the lanes of a row agree)
            const size_t out = row_of(a.dst, to, a.n_kv_heads, b, walk.head, first + (int)t);
            uint32_t kc, vc;
            const uint2 k8 = encode8(k[u], kc), v8 = encode8(v[u], vc);
            *reinterpret_cast<uint2 *>(const_cast<char *>(a.dst.k) + out * D + sub * 8) = k8;
            *reinterpret_cast<uint2 *>(const_cast<char *>(a.dst.v) + out * D + sub * 8) = v8;
            const uint32_t ks = row_scales<D>(kc, lane), vs = row_scales<D>(vc, lane);
            if (sub == 0) {
                typedef typename Kv8Scales<D>::Word Word;
                reinterpret_cast<Word *>(a.k_scale)[out] = (Word)ks;
                reinterpret_cast<Word *>(a.v_scale)[out] = (Word)vs;
            }
        }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kKv8Block) void kv8_read_kernel(Kv8ReadArgs a)
{
    constexpr int LR = D / 8, E = sizeof(T);
    typedef typename Kv8Scales<D>::Word Word;
    const int b = blockIdx.z, sub = threadIdx.x % LR;
    const int first = max(a.first ? a.first[b] : 0, 0);
    const int n = min(a.n_tokens, max(min(tier_len(a.src, b), room_of(a.src, b)) - first, 0));
    const int32_t *from = blocks_of(a.src, b);
    const RowWalk<D> walk(a.lg_tokens);
    if (walk.head >= a.n_kv_heads) return;
    for (int64_t t0 = walk.token; t0 < n; t0 += (int64_t)kTogether<T> * walk.step) {
        uint2 c[kTogether<T>][2];
        Word scales[kTogether<T>][2];
#pragma unroll
        for (int u = 0; u < kTogether<T>; ++u) {
            const int t = (int)min(t0 + (int64_t)u * walk.step, (int64_t)n - 1);
            const size_t row = row_of(a.src, from, a.n_kv_heads, b, walk.head, first + t);
            c[u][0] = *reinterpret_cast<const uint2 *>(a.src.k + row * D + sub * 8);
            c[u][1] = *reinterpret_cast<const uint2 *>(a.src.v + row * D + sub * 8);
            scales[u][0] = reinterpret_cast<const Word *>(a.k_scale)[row];
            scales[u][1] = reinterpret_cast<const Word *>(a.v_scale)[row];
        }
#pragma unroll
        for (int u = 0; u < kTogether<T>; ++u) {
            const int64_t t = t0 + (int64_t)u * walk.step;
            if (t >= n) break;
            const size_t out = (((size_t)b * a.n_tokens + t) * a.n_kv_heads + walk.head) * D + sub * 8;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const float scale = kv8_scale((uint32_t)scales[u][x], sub / 4);
                char *dst = (x ? a.v_out : a.k_out) + out * E;
                if constexpr (E == 4) {
                    const FloatPair p0 = kv8_pair_f32<false>(c[u][x].x, scale), p1 = kv8_pair_f32<true>(c[u][x].x, scale);
                    const FloatPair p2 = kv8_pair_f32<false>(c[u][x].y, scale), p3 = kv8_pair_f32<true>(c[u][x].y, scale);
                    *reinterpret_cast<float4 *>(dst) = make_float4(p0[0], p0[1], p1[0], p1[1]);
                    *reinterpret_cast<float4 *>(dst + 16) = make_float4(p2[0], p2[1], p3[0], p3[1]);
                } else {
                    store16_stream(
                        dst, make_uint4(kv8_pair_bf16<false>(c[u][x].x, scale), kv8_pair_bf16<true>(c[u][x].x, scale),
                                        kv8_pair_bf16<false>(c[u][x].y, scale), kv8_pair_bf16<true>(c[u][x].y, scale)));
                }
            }
        }
    }
}

// Rows first + i of a tier from row path[i] of [B, n, Hkv, d], 16 bytes per thread and tensor; the new length.  A copy: 64
// sequences x 64 drafts of 40 heads of 128, 1 to 33 of them accepted, 8.7 to 10.3 us (drafts and rows stay in the last cache),
// 8 x 8 drafts of 8 heads 3.1 us, the launch.
__global__ __launch_bounds__(kKv8Block) void kv_commit_kernel(CommitArgs a)
{
    const int b = blockIdx.y, pieces = a.row_bytes / 16;
    const int first = max(a.first ? a.first[b] : 0, 0);
    const int room = max(room_of(a.tier, b) - first, 0);
    int n = a.cnt ? min(max(a.cnt[b], 0), a.n_tokens) : a.n_tokens;
    if (n > room) {
        if (a.status && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.status, kCacheContextFull);
        n = room;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) a.lens_out[b] = first + n;
    const int32_t *to = blocks_of(a.tier, b);
    const int per_token = a.n_kv_heads * pieces;
    const int64_t total = (int64_t)n * per_token;
    for (int64_t i = (int64_t)blockIdx.x * kKv8Block + threadIdx.x; i < total; i += (int64_t)gridDim.x * kKv8Block) {
        const int t = (int)(i / per_token), r = (int)(i % per_token), h = r / pieces, p = r % pieces;
        const int s = a.path ? min(max(a.path[(int64_t)b * a.n_tokens + t], 0), a.n_tokens - 1) : t;
        const size_t src = (((size_t)b * a.n_tokens + s) * a.n_kv_heads + h) * a.row_bytes + 16 * p;
        const size_t dst = (size_t)row_of(a.tier, to, a.n_kv_heads, b, h, first + t) * a.row_bytes + 16 * p;
        const uint4 k = load16(a.k_in + src), v = load16(a.v_in + src);
        *reinterpret_cast<uint4 *>(const_cast<char *>(a.tier.k) + dst) = k;
        *reinterpret_cast<uint4 *>(const_cast<char *>(a.tier.v) + dst) = v;
    }
}

// workgroups per sequence: one round of the launch's work, 2048 workgroups of all sequences at most
unsigned share_of(int64_t units, int batch) {
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>(units, std::max<int64_t>(1, 2048 / batch)));
}

// Rows of a workgroup by tokens and heads (RowWalk), and the grid: 2048 workgroups at most where a sequence has more tokens
dim3 walk_grid(int head_dim, int n_tokens, int n_kv_heads, int batch, int32_t &lg_tokens)
{
    const int rows = kKv8Block / (head_dim / 8);
    lg_tokens = 0;
    while ((1 << lg_tokens) < rows && (1 << lg_tokens) < n_tokens) ++lg_tokens;
    const int heads = rows >> lg_tokens;
    const unsigned y = (unsigned)((n_kv_heads + heads - 1) / heads);
    const int64_t x = ((int64_t)n_tokens + (1 << lg_tokens) - 1) >> lg_tokens;
    return dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(x, 2048 / std::max<int64_t>(1, (int64_t)y * batch))), y, (unsigned)batch);
}

}  // namespace

hipError_t launch_kv8_write(int dtype, int head_dim, bool from_tier, Kv8WriteArgs a, int batch, hipStream_t s)
{
    const dim3 grid = walk_grid(head_dim, a.n_tokens, a.n_kv_heads, batch, a.lg_tokens), block(kKv8Block);
#define HGCA_KV8_WRITE(T, D)                                                                         \
    do {                                                                                             \
        if (from_tier) hipLaunchKernelGGL((kv8_write_kernel<T, D, true>), grid, block, 0, s, a);     \
        else hipLaunchKernelGGL((kv8_write_kernel<T, D, false>), grid, block, 0, s, a);              \
    } while (0)
    if (dtype == 0 && head_dim == 64) HGCA_KV8_WRITE(float, 64);
    else if (dtype == 0) HGCA_KV8_WRITE(float, 128);
    else if (head_dim == 64) HGCA_KV8_WRITE(bf16_t, 64);
    else HGCA_KV8_WRITE(bf16_t, 128);
#undef HGCA_KV8_WRITE
    return hipGetLastError();
}

hipError_t launch_kv8_read(int dtype, int head_dim, Kv8ReadArgs a, int batch, hipStream_t s)
{
    const dim3 grid = walk_grid(head_dim, a.n_tokens, a.n_kv_heads, batch, a.lg_tokens), block(kKv8Block);
    if (dtype == 0 && head_dim == 64) hipLaunchKernelGGL((kv8_read_kernel<float, 64>), grid, block, 0, s, a);
    else if (dtype == 0) hipLaunchKernelGGL((kv8_read_kernel<float, 128>), grid, block, 0, s, a);
    else if (head_dim == 64) hipLaunchKernelGGL((kv8_read_kernel<bf16_t, 64>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((kv8_read_kernel<bf16_t, 128>), grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_kv_commit(const CommitArgs &a, int batch, hipStream_t s)
{
    const int64_t per_seq = ((int64_t)a.n_tokens * a.n_kv_heads * (a.row_bytes / 16) + kKv8Block - 1) / kKv8Block;
    hipLaunchKernelGGL(kv_commit_kernel, dim3(share_of(per_seq, batch), batch), dim3(kKv8Block), 0, s, a);
    return hipGetLastError();
}

}  // namespace hgca
