// What stands before a step: queries and keys are normed per head (y = w * x / sqrt(mean x^2 + eps)) and their columns
// rotated in pairs by the token's position, (a, b) -> (a cos t - b sin t, a sin t + b cos t) with t = position * inv_freq[j].
//
// Everything between the load and the one rounding of the result is fp32, the angle fp64: a position of a million times a
// frequency near 1 has no digits left in fp32 (its fraction of a turn would be off by 2^-4); the fp64 product is brought into
// half a turn before it becomes fp32, and what that leaves of it turns the sine and cosine a little further (worst error 1.9 -> 1.3
// units of 2^-24, level in time).
//
// Bound by memory, each row read and written once: 2 x 4096 tokens of 64 + 8 heads of 128 52.5 us, 302 MB at 5.75 TB/s (a large
// copy: 5.16); one token x 8 sequences of 32 + 8 heads 3.5 us, the launch and a load's way.
#include <algorithm>

#include "hgca_launch.hpp"

namespace hgca {

namespace {

constexpr int kRopeBlock = 256, kRopeWaves = kRopeBlock / kWave;

// 8 adjacent elements as floats, and back with one rounding each.  Streamed stores: 2 x 4096 tokens of 64 + 8 heads 60.0 -> 54.5 us (302 MB,
// 5.5 TB/s), 2 x 1024 of 32 + 8 heads 10.8 -> 9.7; loads streamed as well 56.0 and 11.0.  (fp32 is not streamed: a lane
// has 32 bytes, and each of its two accesses would meet half of a line.)
template <typename T> struct Eight;
template <> struct Eight<float> {
    uint4 r[2];
    __device__ __forceinline__ void load(const char *p) { r[0] = load16(p); r[1] = load16(p + 16); }
    __device__ __forceinline__ void expand(float *f) const { Elem<float>::expand(r[0], f); Elem<float>::expand(r[1], f + 4); }
    static __device__ __forceinline__ void store(char *p, const float *f) {
        *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
        *reinterpret_cast<float4 *>(p + 16) = make_float4(f[4], f[5], f[6], f[7]);
    }
};
template <> struct Eight<bf16_t> {
    uint4 r;
    __device__ __forceinline__ void load(const char *p) { r = load16(p); }
    __device__ __forceinline__ void expand(float *f) const { Elem<bf16_t>::expand(r, f); }
    static __device__ __forceinline__ void store(char *p, const float *f) {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        typedef float f2 __attribute__((ext_vector_type(2)));
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{f[2 * i], f[2 * i + 1]}), bf2));
        store16_stream(p, make_uint4(w[0], w[1], w[2], w[3]));
    }
};

// A row of a head is held by D / 16 lanes, 16 columns each: 8 pairs of the rotation, or 16 columns behind it, so that both
// members of a pair are in one lane for either pairing and every load is 16 bytes.  A wave takes 64 / (D / 16) rows of one
// token at a time; the token's sines and cosines are formed once, one pair per lane, and go through LDS to the lanes that need
// them, eight adjacent pairs each.
template <typename T, int D, bool INTERLEAVED>
__global__ __launch_bounds__(kRopeBlock) void qk_norm_rope_kernel(RopeArgs a)
{
    constexpr int LR = D / 16, RPW = kWave / LR, E = sizeof(T);
    __shared__ float s_cos[kRopeWaves][D / 2], s_sin[kRopeWaves][D / 2];
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave, c = lane % LR;
    const int half = a.rot / 2;
    const bool turns = 8 * c < half;
    // first column of the lane's two runs of 8: halves pair j with j + rot/2, interleaved 2j with 2j + 1
    const int c0 = !turns ? a.rot + 16 * (c - half / 8) : INTERLEAVED ? 16 * c : 8 * c;
    const int c1 = turns && !INTERLEAVED ? half + 8 * c : c0 + 8;
    const int rows = a.n_q_heads + a.n_kv_heads;

    for (int64_t tok = blockIdx.x; tok < a.tokens; tok += gridDim.x) {
        const int b = (int)(tok / a.n_tokens), i = (int)(tok % a.n_tokens);
        const double pos = a.positions ? a.positions[tok] : (double)(a.first_pos ? a.first_pos[b] : 0) + i;
        if (lane < half) {
            double turn = pos * (double)a.inv_freq[lane] * 0.15915494309189533577;       // 1 / 2 pi
            turn -= rint(turn);
            const float part = (float)turn, rest = (float)(turn - part) * 6.283185307f;  // what fp32 leaves of the angle
            float sn, cs;
            sincospif(2.f * part, &sn, &cs);
            s_cos[w][lane] = fmaf(-sn, rest, cs);
            s_sin[w][lane] = fmaf(cs, rest, sn);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // written and read by the lanes of one wave only
        float cs[8], sn[8];
        if (turns) {
#pragma unroll
            for (int u = 0; u < 8; ++u) { cs[u] = s_cos[w][8 * c + u]; sn[u] = s_sin[w][8 * c + u]; }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        for (int r0 = (blockIdx.y * kRopeWaves + w) * RPW; r0 < rows; r0 += gridDim.y * kRopeWaves * RPW) {
            const int r = r0 + lane / LR;
            const bool live = r < rows, is_q = r < a.n_q_heads;
            const int rc = live ? r : rows - 1;
            const int64_t in = rc < a.n_q_heads ? tok * a.q_stride + (int64_t)rc * D : tok * a.k_stride + (int64_t)(rc - a.n_q_heads) * D;
            const char *src = (rc < a.n_q_heads ? a.q : a.k) + in * E;
            Eight<T> x0, x1;
            x0.load(src + c0 * E);
            x1.load(src + c1 * E);
            float x[16];
            x0.expand(x);
            x1.expand(x + 8);
            const char *weight = rc < a.n_q_heads ? a.q_weight : a.k_weight;
            if (weight) {
                float sum = 0.f;               // (the lanes of a row take the same branch)
#pragma unroll
                for (int u = 0; u < 16; ++u) sum = fmaf(x[u], x[u], sum);
                sum = group_sum<LR>(sum);
                const float inv = rsqrtf(sum * (1.f / D) + a.eps);
                Eight<T> w0, w1;
                w0.load(weight + c0 * E);
                w1.load(weight + c1 * E);
                float wt[16];
                w0.expand(wt);
                w1.expand(wt + 8);
#pragma unroll
                for (int u = 0; u < 16; ++u) x[u] *= inv * wt[u];
            }
            if (turns) {
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    float &p = x[INTERLEAVED ? 2 * u : u], &q = x[INTERLEAVED ? 2 * u + 1 : 8 + u];
                    const float p0 = p, q0 = q;
                    p = p0 * cs[u] - q0 * sn[u];
                    q = p0 * sn[u] + q0 * cs[u];
                }
            }
            if (live) {
                char *dst = is_q ? a.q_out + (tok * a.n_q_heads + r) * D * E
                                 : a.k_out + (tok * a.n_kv_heads + (r - a.n_q_heads)) * D * E;
                Eight<T>::store(dst + c0 * E, x);
                Eight<T>::store(dst + c1 * E, x + 8);
            }
        }
    }
}

}  // namespace

hipError_t launch_qk_norm_rope(int dtype, int head_dim, const RopeArgs &a, hipStream_t s)
{
    const int rows = a.n_q_heads + a.n_kv_heads, per_pass = kRopeWaves * (kWave / (head_dim / 16));
    // few tokens: a workgroup per pass over the heads of a token; many: one per token, which forms its angles once
    const int y = a.tokens < 1024 ? std::min((rows + per_pass - 1) / per_pass, 64) : 1;
    const dim3 grid((unsigned)std::min<int64_t>(a.tokens, 1 << 20), y);
#define HGCA_ROPE(T, D)                                                                                             \
    do {                                                                                                            \
        if (a.interleaved) hipLaunchKernelGGL((qk_norm_rope_kernel<T, D, true>), grid, dim3(kRopeBlock), 0, s, a);  \
        else hipLaunchKernelGGL((qk_norm_rope_kernel<T, D, false>), grid, dim3(kRopeBlock), 0, s, a);               \
    } while (0)
    if (dtype == 0 && head_dim == 64) HGCA_ROPE(float, 64);
    else if (dtype == 0) HGCA_ROPE(float, 128);
    else if (head_dim == 64) HGCA_ROPE(bf16_t, 64);
    else HGCA_ROPE(bf16_t, 128);
#undef HGCA_ROPE
    return hipGetLastError();
}

}  // namespace hgca
