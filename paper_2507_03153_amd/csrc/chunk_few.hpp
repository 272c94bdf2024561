// Units of up to 16 rows of a chunk call (a token's heads, a few tokens), in fp32 of up to 32: a wave is the 16 rows (RT = 1) or 32 (RT = 2) against
// tokens of its own at a time, straight from memory to the operands of 16 x 16 tiles, the next ones requested while these are worked on; the workgroup's four
// waves take turns and join what they found at the end.  Nothing waits at a barrier, all four waves work, and 16 rows take a quarter of
// the 32 x 32 tiles' arithmetic.
//   S^T[token, row] = K . Q^T,  O^T[col, row] += V^T . P^T,
// lane n + 16 g has row n of a tile in both: scores of tokens 4 g .. 4 g + 3 of a tile of 16, and columns e of E = D / 16 adjacent ones, product e, at
// E m + e with m = 4 g + i.
//
// What bounds it: memory.  One token of 8 sequences over 28 672, 32 / 8 heads of 128, bf16: 940 MB in 163 us, 5.8 TB/s, and 5 for the fold (through
// LDS 174; heads of 64 89 : 102; a mixed step, whose single tokens it is, 441 : 488).  Units of 9 to 16 rows are
// level (171 : 167).  17 to 32 rows in bf16 lose (169 -> 177), in fp32 they gain, as a unit through LDS does the arithmetic of 128 rows (8 tokens x
// 8 over 14 K, groups of 4: 377 -> 196).  (bf16 figures with weights of one part; with two the units of up to 16 rows take 164 and 174 us.)
#pragma once

#include "chunk_device.hpp"

namespace hgca {

namespace {

constexpr int kFewRows = 32;

__device__ __forceinline__ floatx4 few_mfma(const uint4 &a, const uint4 &b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// over the four rows of 16 lanes
__device__ __forceinline__ float few_max(float x) {
    const LanePair r = rows_of(x);
    const LanePair h = halves_of(fmaxf(r.a, r.b));
    return fmaxf(h.a, h.b);
}

// The waves' results on their way to one.
template <int D> struct FewShared {
    float m[kChunkWaves][kFewRows], l[kChunkWaves][kFewRows];
    float o[kChunkWaves][kFewTile][D + 4];       // a tile at a time
    int odd[kChunkWaves];
    OddTokens<D> notes;
};

template <int E> struct FewState {
    float m = -INFINITY, shift = 0.f, l = 0.f;   // shift: 0 for far rows (shift_of); l: over the lane's own tokens
    bool far = false;                            // uniform over the wave: a row of it is
    floatx4 o[E];
    __device__ __forceinline__ FewState() {
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = floatx4{};
    }
    // scores become weights
    template <int NT> __device__ __forceinline__ void weigh(floatx4 (&s)[NT], float k2) {
        float mx = s[0][0];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[t][i]);
        if (any_lane(mx > m)) {
            const float m_new = fmaxf(m, few_max(mx)), to = shift_of(m_new, k2), corr = rescale_factor(m, m_new, k2);
            m = m_new;
            shift = is_far(to) ? 0.f : to;
            far = any_lane(is_far(to));
            l *= corr;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] *= corr;
        }
        if (far) {
            const float less = is_far(shift_of(m, k2)) ? m : 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t] -= less;
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], k2, shift));      // masked scores give 0
                l += s[t][i];
            }
    }
};

// What the waves found becomes one result per row, a tile of 16 at a time: its row r is lane group r of the workgroup, 16 lanes with E columns each.
template <typename T, int D, int RT>
__device__ __forceinline__ void few_join(FewShared<D> &sh, const ChunkArgs &a, const Place &at, const SeqWork &seq, const Steps &steps, int kvh,
                                         FewState<D / 16> (&st)[RT], float k2, bool odd)
{
    constexpr int E = D / 16;
    const int tid = threadIdx.x, w = tid / kWave, lane = tid % kWave, n = lane % 16, g = lane / 16;
    float z[4] = {0.f, 0.f, 0.f, 0.f};           // NaN where a sum is not finite
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const float lw = strided_sum<16>(st[t].l);
        if (g == 0) {
            sh.m[w][kFewTile * t + n] = lw == 0.f ? -INFINITY : -shift_of(st[t].m, k2);
            sh.l[w][kFewTile * t + n] = lw;
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = fmaf(st[t].o[e][i], 0.f, z[i]);
    }
    const float all = (z[0] + z[1]) + (z[2] + z[3]);
    odd = any_lane(all != all || odd);
    if (lane == 0) sh.odd[w] = odd;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if (t > 0) __syncthreads();              // the tile before has been read
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < E; e += 4)
                *reinterpret_cast<float4 *>(&sh.o[w][n][(4 * g + i) * E + e]) =
                    make_float4(st[t].o[e][i], st[t].o[e + 1][i], st[t].o[e + 2][i], st[t].o[e + 3][i]);
        __syncthreads();
        const int r = tid / 16, c = tid % 16, row = kFewTile * t + r;
        const RowPlace rp(a, seq, at.unit, kvh, row);
        float M = -INFINITY, L = 0.f, x[E];
#pragma unroll
        for (int i = 0; i < kChunkWaves; ++i) M = fmaxf(M, sh.m[i][row]);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = 0.f;
#pragma unroll
        for (int i = 0; i < kChunkWaves; ++i) {
            const float m = sh.m[i][row];
            if (m == -INFINITY) continue;        // the wave saw nothing of the row
            const float f = __builtin_amdgcn_exp2f(m - M);
            L = fmaf(sh.l[i][row], f, L);
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const float4 o = *reinterpret_cast<const float4 *>(&sh.o[i][r][c * E + e]);
                x[e] = fmaf(o.x, f, x[e]);
                x[e + 1] = fmaf(o.y, f, x[e + 1]);
                x[e + 2] = fmaf(o.z, f, x[e + 2]);
                x[e + 3] = fmaf(o.w, f, x[e + 3]);
            }
        }
        bool any = false;
#pragma unroll
        for (int i = 0; i < kChunkWaves; ++i) any = any || sh.odd[i];
        if (any) {                               // uniform over the workgroup
            const RowSees sees(a, seq, rp.query);
            uint32_t kinds[E];
#pragma unroll
            for (int e = 0; e < E; ++e) kinds[e] = 0;
            for (int part = 0; part < 2; ++part)
                for (int s = steps.begin(part); s < steps.end(part); ++s) {
                    sh.notes.template note<T>(a, at.b, kvh, s * kChunkStep, seq.len);
                    const uint64_t seen = sees.mask(s * kChunkStep);
#pragma unroll
                    for (int e = 0; e < E; ++e)
#pragma unroll
                        for (int k = 0; k < 3; ++k) kinds[e] |= sh.notes.bits[k][c * E + e] & seen ? 1u << k : 0u;
                }
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = kinds[e] == 0 ? x[e] : kinds[e] == 1 ? INFINITY : kinds[e] == 2 ? -INFINITY : NAN;
        }
        if (!rp.live) continue;                  // (barriers are reached by all: the loop is unrolled and uniform)
        auto store = [&](auto four) {
#pragma unroll
            for (int e = 0; e < E; e += 4) four(c * E + e, make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]));
        };
        if (at.n_shares > 1) {
            const int64_t to = ((int64_t)(at.part + at.share) * a.sh.n_kv_heads + kvh) * kChunkRows + row;
            store([&](int col, const float4 &y) { *reinterpret_cast<float4 *>(a.part_o + to * D + col) = y; });
            if (c == 0) {
                a.part_m[to] = M;
                a.part_l[to] = L;
            }
            continue;
        }
        const float inv = L == 0.f ? 0.f : 1.f / L;
        store([&](int col, const float4 &y) {
            const float4 v = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
            if (a.o_bf16)
                *reinterpret_cast<uint2 *>(static_cast<char *>(a.o) + 2 * (rp.out * D + col)) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
            else
                *reinterpret_cast<float4 *>(static_cast<float *>(a.o) + rp.out * D + col) = v;
        });
        if (c == 0) a.lse[rp.out] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
    }
}

// What both types' loops go through: the share in passes that the table of a paged tier covers; of every kChunkWaves * kTokens tokens a wave takes
// its kTokens.  fetch(rows, tok, nsub) requests those from token tok of the pass on; use(tok, next) goes through them, tok being the tier's.
template <int kTokens, typename Fetch, typename Use>
__device__ __forceinline__ void few_tokens(uint32_t *s_row, const ChunkArgs &a, const Place &at, const SeqWork &seq, const Steps &steps, int kvh,
                                           Fetch fetch, Use use)
{
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll 1
    for (int range = 0; range < 2; ++range) {
        const int from = steps.begin(range) * kChunkStep, total = min(steps.end(range) * kChunkStep, seq.len) - from;
        const int sub_len = pass_length(a.kv, total);
#pragma unroll 1
        for (int sub0 = 0; sub0 < total; sub0 += sub_len) {
            const int nsub = min(sub_len, total - sub0), first = from + sub0;
            __syncthreads();                     // the table of the pass before is no longer in use
            const BlockRows where = make_block_rows<kChunkBlock>(s_row, a.kv, a.sh.n_kv_heads, at.b, kvh, first, nsub);
            int tok = kTokens * w;
            if (tok < nsub) fetch(where, tok, nsub);
#pragma unroll 1
            for (; tok < nsub; tok += kTokens * kChunkWaves)
                use(first + tok, [&](auto request) {
                    const int next = tok + kTokens * kChunkWaves;
                    if (next < nsub) request(where, next, nsub);
                });
        }
    }
}

constexpr uint32_t kFewLow = 0x05040100u, kFewHigh = 0x07060302u;                // byte selectors: (b.lo, a.lo) and (b.hi, a.hi)

// bf16: one tile of 16 rows and 32 tokens of a wave at a time.  V needs tokens side by side where rows have columns side by side: pairs of tokens are put together by
// byte permutations.
template <int D, int PP, int MODE>
__device__ __forceinline__ void few_rows_bf16(FewShared<D> &sh, uint32_t *s_row, const ChunkArgs &a, const Place &at, const SeqWork &seq,
                                              const Steps &steps, int kvh)
{
    constexpr int KS = D / 32, E = D / 16, W = E / 2, RT = 1;
    const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
    uint4 q[RT][KS];
    RowSees sees[RT];
    int pos[RT];
    float slope[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const RowPlace rp(a, seq, at.unit, kvh, kFewTile * r + n);
        const char *const qp = a.q + (seq.n0 + rp.query) * a.q_stride + (int64_t)rp.head * (2 * D) + 16 * g;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[r][s] = load16(qp + 64 * s);
        sees[r] = RowSees(a, seq, rp.query);
        pos[r] = seq.len - seq.nq + rp.query;
        slope[r] = ScoreMap<MODE, PP != 1>::slope_of(a, rp.head);
    }
    const WaveSees wave(sees);
    ScoreMap<MODE, PP != 1> map(a);
    FewState<E> st[RT];
    bool met_odd = false;                        // of the lane
    uint4 k[2][KS];
    uint32_t v[2][4][W];
    auto tile = [&](const BlockRows &rows, int tok, int nsub, int t, int &nv) {
        const int gr = min(tok / 16 + t, (nsub - 1) / 16);
        nv = min(16, nsub - 16 * gr);            // tokens that exist; the others repeat the last one
        return (size_t)(uint32_t)__builtin_amdgcn_readfirstlane(rows.table ? rows.table[gr] : rows.base + 16 * gr) * (2 * D);
    };
    auto fetch_k = [&](const BlockRows &rows, int tok, int nsub) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            int nv;
            const char *const p = a.kv.k + tile(rows, tok, nsub, t, nv) + (uint32_t)(min(n, nv - 1) * (2 * D) + 16 * g);
#pragma unroll
            for (int s = 0; s < KS; ++s) k[t][s] = load16(p + 64 * s);
        }
    };
    auto fetch_v = [&](const BlockRows &rows, int tok, int nsub) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            int nv;
            const char *const vp = a.kv.v + tile(rows, tok, nsub, t, nv);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const char *const p = vp + (uint32_t)(min(4 * g + j, nv - 1) * (2 * D) + n * 2 * E);
                if constexpr (D == 128) *reinterpret_cast<uint4 *>(v[t][j]) = load16(p);
                else *reinterpret_cast<uint2 *>(v[t][j]) = *reinterpret_cast<const uint2 *>(p);
            }
        }
    };
    auto use = [&](int tok, auto next) {
        floatx4 s[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r) s[r][0] = s[r][1] = floatx4{};
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < RT; ++r) s[r][t] = few_mfma(k[t][i], q[r][i], s[r][t]);
        next(fetch_k);
        const bool masked = !wave.all(tok, 32);
        uint32_t part[RT][PP][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            map.slope2 = slope[r];
            map.template each<8>([&](int i) { return s[r][i / 4][i % 4]; }, [&](int i, float x) { s[r][i / 4][i % 4] = x; },
                                 [](int i) { return 16 * (i / 4) + i % 4; }, pos[r], tok + 4 * g);
            if (masked) {
                const uint32_t seen = (uint32_t)sees[r].mask(tok + 4 * g);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(seen >> (16 * t + i) & 1u)) s[r][t][i] = -INFINITY;
            }
            st[r].weigh(s[r], map.k2);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float x0 = s[r][c / 2][2 * (c % 2)], x1 = s[r][c / 2][2 * (c % 2) + 1];
#pragma unroll
                for (int t = 0; t < PP; ++t) {
                    part[r][t][c] = pack_bf16(x0, x1);
                    x0 -= __uint_as_float(part[r][t][c] << 16);
                    x1 -= __uint_as_float(part[r][t][c] & 0xffff0000u);
                }
            }
        }
        if (masked) {                            // infinities and NaN are taken out (few_join brings them to the rows that see them)
            uint32_t odd = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < W; ++i) odd |= odd_carry(v[t][j][i]);
            if (odd & kSigns) {
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
        for (int e = 0; e < E; ++e) {            // eight tokens of column n * E + e
            const uint32_t sel = e % 2 ? kFewHigh : kFewLow;
            const uint4 op = make_uint4(__builtin_amdgcn_perm(v[0][1][e / 2], v[0][0][e / 2], sel), __builtin_amdgcn_perm(v[0][3][e / 2], v[0][2][e / 2], sel),
                                        __builtin_amdgcn_perm(v[1][1][e / 2], v[1][0][e / 2], sel), __builtin_amdgcn_perm(v[1][3][e / 2], v[1][2][e / 2], sel));
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int t = PP - 1; t >= 0; --t)
                    st[r].o[e] = few_mfma(op, make_uint4(part[r][t][0], part[r][t][1], part[r][t][2], part[r][t][3]), st[r].o[e]);
        }
        next(fetch_v);
    };
    few_tokens<32>(s_row, a, at, seq, steps, kvh,
                   [&](const BlockRows &rows, int tok, int nsub) {
                       fetch_k(rows, tok, nsub);
                       fetch_v(rows, tok, nsub);
                   },
                   use);
    few_join<bf16_t, D, RT>(sh, a, at, seq, steps, kvh, st, map.k2, met_odd);
}

// fp32: 16 tokens of a wave at a time; a lane's four tokens are the four slices of the second product.
template <int D, int MODE, int RT>
__device__ __forceinline__ void few_rows_f32(FewShared<D> &sh, uint32_t *s_row, const ChunkArgs &a, const Place &at, const SeqWork &seq,
                                             const Steps &steps, int kvh)
{
    constexpr int U = D / 16, E = D / 16, RB = 4 * D;
    const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
    float q[RT][U][4];
    RowSees sees[RT];
    int pos[RT];
    float slope[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const RowPlace rp(a, seq, at.unit, kvh, kFewTile * r + n);
        const char *const qp = a.q + (seq.n0 + rp.query) * a.q_stride + (int64_t)rp.head * RB + 16 * g;
#pragma unroll
        for (int u = 0; u < U; ++u) Elem<float>::expand(load16(qp + 64 * u), q[r][u]);
        sees[r] = RowSees(a, seq, rp.query);
        pos[r] = seq.len - seq.nq + rp.query;
        slope[r] = ScoreMap<MODE, true>::slope_of(a, rp.head);
    }
    const WaveSees wave(sees);
    ScoreMap<MODE, true> map(a);
    FewState<E> st[RT];
    bool met_odd = false;                        // of the lane
    float k[U][4], v[4][E];
    auto first_row = [&](const BlockRows &rows, int tok) {
        return (size_t)(uint32_t)__builtin_amdgcn_readfirstlane(rows.table ? rows.table[tok / 16] : rows.base + tok) * RB;
    };
    auto fetch_k = [&](const BlockRows &rows, int tok, int nsub) {
        const char *const p = a.kv.k + first_row(rows, tok) + (uint32_t)(min(n, min(16, nsub - tok) - 1) * RB + 16 * g);
#pragma unroll
        for (int u = 0; u < U; ++u) Elem<float>::expand(load16(p + 64 * u), k[u]);
    };
    auto fetch_v = [&](const BlockRows &rows, int tok, int nsub) {
        const char *const vp = a.kv.v + first_row(rows, tok);
        const int last = min(16, nsub - tok) - 1;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < E; e += 4)
                Elem<float>::expand(load16(vp + (uint32_t)(min(4 * g + j, last) * RB + n * 4 * E + 4 * e)), v[j] + e);
    };
    auto use = [&](int tok, auto next) {
        floatx4 s[RT][1], s2[RT];                // two chains
#pragma unroll
        for (int r = 0; r < RT; ++r) s[r][0] = s2[r] = floatx4{};
#pragma unroll
        for (int u = 0; u < U; u += 2)
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    s[r][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[u][c], q[r][u][c], s[r][0], 0, 0, 0);
                    s2[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[u + 1][c], q[r][u + 1][c], s2[r], 0, 0, 0);
                }
        next(fetch_k);
        const bool masked = !wave.all(tok, 16);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            s[r][0] += s2[r];
            map.slope2 = slope[r];
            map.template each<4>([&](int i) { return s[r][0][i]; }, [&](int i, float x) { s[r][0][i] = x; }, [](int i) { return i; }, pos[r],
                                 tok + 4 * g);
            if (masked) {
                const uint32_t seen = (uint32_t)sees[r].mask(tok + 4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(seen >> i & 1u)) s[r][0][i] = -INFINITY;
            }
            st[r].weigh(s[r], map.k2);
        }
        if (masked) {                            // as above
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const bool bad = !(fabsf(v[j][e]) < INFINITY);
                    met_odd = met_odd || bad;
                    v[j][e] = bad ? 0.f : v[j][e];
                }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int r = 0; r < RT; ++r) st[r].o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j][e], s[r][0][j], st[r].o[e], 0, 0, 0);
        next(fetch_v);
    };
    few_tokens<16>(s_row, a, at, seq, steps, kvh,
                   [&](const BlockRows &rows, int tok, int nsub) {
                       fetch_k(rows, tok, nsub);
                       fetch_v(rows, tok, nsub);
                   },
                   use);
    few_join<float, D, RT>(sh, a, at, seq, steps, kvh, st, map.k2, met_odd);
}

}  // namespace

}  // namespace hgca
