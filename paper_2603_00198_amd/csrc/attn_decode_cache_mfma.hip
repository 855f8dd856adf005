// One token's attention over a 4-bit or a plain bf16 cache on the matrix cores (heads of 64 or 128 channels, up to 16 query heads
// to a kv head, in 4 bits up to 8 of 128 channels): pass 1 of attn_decode_cache.hip, whose pass 2 joins the splits.
//
// The step is bound by reading the cache -- 5 bits per element -- if the vector instructions per element stay below about two:
// turning codes into numbers and multiplying them into up to 8 heads one by one takes six.  So both products are matrix products,
// on codes as they are:
//  * A code n becomes the bf16 number 16 + n by a shift and one instruction (its bits are the upper mantissa bits; exact).
//  * Scores: A = the codes of 16 rows, B = the query heads, a column for every (group of channels, head) with zeros outside the group.
//    The product leaves every group's sum of q (16 + n) apart; with the group's s and z it becomes s * sum + (z - 24 s) * sum q,
//    and the groups of a head, columns 4 (8) lanes apart, are added by two rotations of the 16 lanes.  An accumulator's rows are
//    rows of the cache, four to a lane: the next product's operand as it stands.
//  * Values: A = the codes of V with the cache's rows as the contraction index, B = p * s, rounded to bf16 -- the one rounding of
//    the path beside the output's -- for every (group, head).  A lane collects 8 rows' codes and
//    regroups their halves.  What the 24 too many and z add does not depend on the channel: each lane sums p z - 24 (the rounded
//    p s) in fp32.  Rows (channels) of the product and columns of another group belong to nobody.
//  * A plain cache goes the same way without groups: columns are heads, values are regrouped halves.
// A wave takes 32 rows at a time, the next ones on their way; its softmax has one reference per head that moves when a score is
// 2^8 above it.  Weights: the scores go to the workspace as they come.
#include "attn_decode_cache.h"

namespace strd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4, kTrip = 32, kRound = kWaves * kTrip;
constexpr float kLog2e = 1.4426950408889634f, kLazy = 8.f;

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
template <int N>
__device__ __forceinline__ float row_ror(float v) {  // of the lane N places on in the row of 16, round its end
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xF, 0xF, true));
}
__device__ __forceinline__ float quarters_sum(float v) {
    v += __shfl_xor(v, 16, kWave);
    return v + __shfl_xor(v, 32, kWave);
}
__device__ __forceinline__ float quarters_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, bf16x2{(bf16_t)lo, (bf16_t)hi});
}
// Codes at bits 4 J and 16 + 4 J as a pair of bf16 numbers 16 + n: n belongs at bits 3 .. 6 of each half.
template <int J>
__device__ __forceinline__ uint32_t code_pair(uint32_t x) {
    const uint32_t y = J == 0 ? x << 3 : x >> (4 * J - 3);
    return (y & 0x00780078u) | 0x41804180u;
}

template <int D, bool KV4>
struct Shape {
    static constexpr int kGroupsOfD = KV4 ? D / kKv4Group : 1;
    static constexpr int kHeads = 16 / kGroupsOfD;      // query heads per set of columns
    static constexpr int kKSteps = D / 32;              // products per 16 rows of keys
    static constexpr int kVTiles = D / 16;              // products per 32 rows of values
    static constexpr int kKDwords = KV4 ? D / 32 : D / 8;  // of a lane, per 16 rows
    static constexpr int kVDwords = KV4 ? 1 : D / 32;      // of a lane, per row (4 bits, D = 64: half of one)
};

template <int D, bool KV4, int NP, bool BIAS>
__global__ __launch_bounds__(kWaves *kWave) __attribute__((amdgpu_waves_per_eu(NP == 1 && !BIAS && (KV4 || D == 64) ? 3 : 2))) void decode_cache_mfma_kernel(
    const bf16_t *__restrict__ q, CacheView cv, DecWs ws, int Tn, int Hq, int Hkv, int tps, int nsplit, ScoreMod mod) {
    using S = Shape<D, KV4>;
    constexpr int NG = S::kGroupsOfD, HP = S::kHeads, KS = S::kKSteps, VT = S::kVTiles, KD = S::kKDwords, VD = S::kVDwords;
    __shared__ __attribute__((aligned(16))) float sm_o[kWaves][HP][D];
    __shared__ float sm_m[kWaves][HP], sm_l[kWaves][HP];
    int hk, split;
    dec_place(blockIdx.x, Hkv, hk, split);
    if (split >= nsplit) return;  // uniform
    const int rep = Hq / Hkv;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int lr = lane & 15, c = lane >> 4;
    const int grp = lr / HP, hcol = lr % HP;               // this lane's column: group of channels, head
    const int kgrp = KV4 ? c * (D / 4) / kKv4Group : 0;    // group of the channels this lane holds of a key
    const long long begin = (long long)split * tps;
    const int t_end = (int)min((long long)Tn, begin + tps);

    struct Rows {
        uint32_t k[2][KD], v[8][VD], km[KV4 ? 8 : 1], vm[KV4 ? 8 : 1];
        int32_t pos[BIAS ? 8 : 1];
    };
    // Rows t0 .. t0 + 31 of this kv head; rows past the last one are read as that one, and masked.
    const uint32_t k_stride = (uint32_t)Hkv * (KV4 ? D / 2 : D * 2), m_stride = (uint32_t)Hkv * (NG * 4);
    auto load = [&](int t0, Rows &x) __attribute__((always_inline)) {
        t0 = min(t0, Tn - 1);  // uniform
        const int last = Tn - 1 - t0;
        const char *kb = (const char *)cv.k + (size_t)t0 * k_stride + (size_t)hk * (k_stride / Hkv);
        const char *vb = (const char *)cv.v + (size_t)t0 * k_stride + (size_t)hk * (k_stride / Hkv);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t off = (uint32_t)min(16 * u + lr, last) * k_stride;
            if constexpr (KV4 && D == 128) {
                const u32x4 d = *reinterpret_cast<const u32x4 *>(kb + off + 16 * c);
#pragma unroll
                for (int i = 0; i < 4; ++i) x.k[u][i] = d[i];
            } else if constexpr (KV4) {
                const u32x2 d = *reinterpret_cast<const u32x2 *>(kb + off + 8 * c);
                x.k[u][0] = d[0];
                x.k[u][1] = d[1];
            } else {
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    const u32x4 d = *reinterpret_cast<const u32x4 *>(kb + off + 64 * i + 16 * c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.k[u][4 * i + e] = d[e];
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t row = (uint32_t)min(16 * (e >> 2) + 4 * c + (e & 3), last);
            const uint32_t off = row * k_stride;
            if constexpr (KV4 && D == 128) {
                x.v[e][0] = *reinterpret_cast<const uint32_t *>(vb + off + 4 * lr);
            } else if constexpr (KV4) {
                x.v[e][0] = *reinterpret_cast<const uint16_t *>(vb + off + 2 * lr);
            } else if constexpr (D == 128) {
                const u32x4 d = *reinterpret_cast<const u32x4 *>(vb + off + 16 * lr);
#pragma unroll
                for (int i = 0; i < 4; ++i) x.v[e][i] = d[i];
            } else {
                const u32x2 d = *reinterpret_cast<const u32x2 *>(vb + off + 8 * lr);
                x.v[e][0] = d[0];
                x.v[e][1] = d[1];
            }
            if constexpr (KV4) {
                const uint32_t mo = row * m_stride + 4 * grp;
                x.km[e] = *reinterpret_cast<const uint32_t *>((const char *)cv.km + ((size_t)t0 * Hkv + hk) * (NG * 4) + mo);
                x.vm[e] = *reinterpret_cast<const uint32_t *>((const char *)cv.vm + ((size_t)t0 * Hkv + hk) * (NG * 4) + mo);
            }
        }
        if constexpr (BIAS) {
            if (mod.pos) {  // uniform
#pragma unroll
                for (int e = 0; e < 8; ++e) x.pos[e] = mod.pos[t0 + min(16 * (e >> 2) + 4 * c + (e & 3), last)];
            }
        }
    };

    // the query heads: B operand, column (grp, hcol), k slots as the keys' codes come (the pairs of code_pair), zeros outside
    // the column's group
    bf16x8 bq[NP][KS];
    float qsum[NP], slope[NP], m[NP], l[NP], corr[NP];
    f32x4 oacc[NP][VT];
    const bf16_t one = (bf16_t)1.f;
    const bf16x8 ones = {one, one, one, one, one, one, one, one};
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int hh = p * HP + hcol;
        const bool live = hh < rep && (!KV4 || grp == kgrp);
        const bf16_t *qh = q + (size_t)(hk * rep + min(hh, rep - 1)) * D;
        f32x4 z = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const bf16x8 x = *reinterpret_cast<const bf16x8 *>(qh + (KV4 ? c * (D / 4) + 8 * i : 32 * i + 8 * c));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int from = KV4 ? (e >> 1) + 4 * (e & 1) : e;
                bq[p][i][e] = live ? x[from] : (bf16_t)0.f;
            }
            if constexpr (KV4) z = mfma16(ones, bq[p][i], z);
        }
        qsum[p] = z[0];
        slope[p] = BIAS && hh < rep ? mod.slopes[hk * rep + hh] : 0.f;
        m[p] = kDecNegBig;
        l[p] = corr[p] = 0.f;
#pragma unroll
        for (int j = 0; j < VT; ++j) oacc[p][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float pos_q = 0.f;
    if constexpr (BIAS) pos_q = mod.pos ? (float)mod.pos[Tn - 1] : (float)(Tn - 1);

    auto fold = [&](int t0, const Rows &x) __attribute__((always_inline)) {
        const bool tail = t0 + kTrip > t_end;  // uniform
        bf16x8 pb[NP];                         // p (4 bits: p * s of the column's group) of the 32 rows, the next product's operand
        float pr[NP][2][4];
        // ---- scores ----
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            bf16x8 ka[KS];
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                if constexpr (KV4)
                    ka[i] = __builtin_bit_cast(bf16x8, u32x4{code_pair<0>(x.k[u][i]), code_pair<1>(x.k[u][i]), code_pair<2>(x.k[u][i]), code_pair<3>(x.k[u][i])});
                else
                    ka[i] = __builtin_bit_cast(bf16x8, u32x4{x.k[u][4 * i], x.k[u][4 * i + 1], x.k[u][4 * i + 2], x.k[u][4 * i + 3]});
            }
            float far[4];
            if constexpr (BIAS) {
#pragma unroll
                for (int i = 0; i < 4; ++i) far[i] = fabsf(pos_q - (float)(mod.pos ? x.pos[4 * u + i] : t0 + 16 * u + 4 * c + i));
            }
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                f32x4 z = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < KS; ++i) z = mfma16(ka[i], bq[p][i], z);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float s = z[i];
                    if constexpr (KV4) {
                        const Kv4Group g = kv4_meta(x.km[4 * u + i]);
                        s = fmaf(g.s, s, fmaf(-24.f, g.s, g.z) * qsum[p]);
                        s += row_ror<8>(s);
                        if constexpr (NG == 4) s += row_ror<4>(s);
                    }
                    pr[p][u][i] = s * mod.scale;
                }
            }
            if (mod.cap > 0.f) {  // uniform
                bool wide = false;
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        pr[p][u][i] *= mod.inv_cap;
                        wide |= fabsf(pr[p][u][i]) > 0.5f;
                    }
                if (__any(wide)) {
#pragma unroll
                    for (int p = 0; p < NP; ++p)
#pragma unroll
                        for (int i = 0; i < 4; ++i) pr[p][u][i] = mod.cap * tanhf(pr[p][u][i]);
                } else {
                    // tanh(y) / y up to y = 0.5, as a polynomial in y^2 of least relative error (1.3e-8)
#pragma unroll
                    for (int p = 0; p < NP; ++p)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float y = pr[p][u][i], w = y * y;
                            float r = fmaf(w, 0.0171347708f, -0.0529858599f);
                            r = fmaf(w, r, 0.133247737f);
                            r = fmaf(w, r, -0.333330689f);
                            r = fmaf(w, r, 0.999999987f);
                            pr[p][u][i] = mod.cap * (y * r);
                        }
                }
            }
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float s = pr[p][u][i];
                    if constexpr (BIAS) s = fmaf(-slope[p], far[i], s);
                    s *= kLog2e;
                    pr[p][u][i] = tail && t0 + 16 * u + 4 * c + i >= t_end ? -INFINITY : s;
                }
            if (ws.scores) {  // uniform; a head's four rows are one vector, from the lanes of its first group
#pragma unroll
                for (int p = 0; p < NP; ++p)
                    if (grp == 0 && p * HP + hcol < rep && t0 + 16 * u + 4 * c < t_end)
                        *reinterpret_cast<f32x4 *>(ws.scores + (size_t)(hk * rep + p * HP + hcol) * ws.ldt + t0 + 16 * u + 4 * c) =
                            f32x4{pr[p][u][0], pr[p][u][1], pr[p][u][2], pr[p][u][3]};
            }
        }
        // ---- softmax ----
        float tm[NP];
        bool moves = false;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            tm[p] = pr[p][0][0];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) tm[p] = fmaxf(tm[p], pr[p][u][i]);
            moves |= tm[p] > m[p] + kLazy;
        }
        if (__any(moves)) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const float nm = fmaxf(m[p], quarters_max(tm[p])), f = ex2(m[p] - nm);
                m[p] = nm;
                l[p] *= f;
                corr[p] *= f;
#pragma unroll
                for (int j = 0; j < VT; ++j) oacc[p][j] *= f;
            }
        }
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            uint32_t w[4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float ps[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = ex2(pr[p][u][i] - m[p]);
                    l[p] += e;
                    ps[i] = e;
                    if constexpr (KV4) {
                        const Kv4Group g = kv4_meta(x.vm[4 * u + i]);
                        const bool out = tail && t0 + 16 * u + 4 * c + i >= t_end;  // (a group behind the last row may hold NaN)
                        ps[i] = out ? 0.f : e * g.s;
                        corr[p] = out ? corr[p] : fmaf(e, g.z, corr[p]);
                    }
                }
                w[2 * u] = bf16_pair(ps[0], ps[1]);
                w[2 * u + 1] = bf16_pair(ps[2], ps[3]);
            }
            if constexpr (KV4) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    corr[p] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[i]), bf16x2{(bf16_t)-24.f, (bf16_t)-24.f}, corr[p], false);
            }
            pb[p] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
        }
        // ---- values ----
        // halves of two rows' dwords side by side: lo of both, hi of both
        auto pair_lo = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); };
        auto pair_hi = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); };
        uint32_t va[8][VD];
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < VD; ++i)
                va[e][i] = !KV4 && tail && t0 + 16 * (e >> 2) + 4 * c + (e & 3) >= t_end ? 0u : x.v[e][i];  // (0 times what is not finite)
        uint32_t lo[4][VD], hi[4][VD];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < VD; ++i) {
                lo[e][i] = pair_lo(va[2 * e][i], va[2 * e + 1][i]);
                hi[e][i] = pair_hi(va[2 * e][i], va[2 * e + 1][i]);
            }
        auto product = [&](auto jc) __attribute__((always_inline)) {
            constexpr int J = decltype(jc)::value;
            if constexpr (J < VT) {
                u32x4 a;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (KV4)
                        a[e] = code_pair<J % 4>(J < 4 ? lo[e][0] : hi[e][0]);
                    else
                        a[e] = J % 2 ? hi[e][J / 2] : lo[e][J / 2];
                }
#pragma unroll
                for (int p = 0; p < NP; ++p) oacc[p][J] = mfma16(__builtin_bit_cast(bf16x8, a), pb[p], oacc[p][J]);
            }
        };
        product(std::integral_constant<int, 0>());
        product(std::integral_constant<int, 1>());
        product(std::integral_constant<int, 2>());
        product(std::integral_constant<int, 3>());
        product(std::integral_constant<int, 4>());
        product(std::integral_constant<int, 5>());
        product(std::integral_constant<int, 6>());
        product(std::integral_constant<int, 7>());
    };

    {
        Rows a, b;
        int t0 = (int)min(begin + kTrip * wave, (long long)Tn);
        load(t0, a);
        for (; t0 < t_end; t0 += 2 * kRound) {
            load(min(t0 + kRound, Tn), b);
            fold(t0, a);
            if (t0 + kRound < t_end) {
                load(min(t0 + 2 * kRound, Tn), a);
                fold(t0 + kRound, b);
            }
        }
    }

    // ---- the four waves join, one set of heads at a time ----
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int nh = min(HP, rep - p * HP);
        if (nh <= 0) break;  // uniform
        if (p) __syncthreads();
        l[p] = quarters_sum(l[p]);
        corr[p] = quarters_sum(corr[p]);
        // rows 4 c + i of product j are channels VT (4 c + i) + j; a lane's column counts for its own group's channels
        if (!KV4 || grp == VT * 4 * c / kKv4Group) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < VT; j += 4)
                    *reinterpret_cast<f32x4 *>(&sm_o[wave][hcol][VT * (4 * c + i) + j]) =
                        f32x4{oacc[p][j][i] + corr[p], oacc[p][j + 1][i] + corr[p], oacc[p][j + 2][i] + corr[p], oacc[p][j + 3][i] + corr[p]};
        }
        if (lane < HP) {
            sm_m[wave][hcol] = m[p];
            sm_l[wave][hcol] = l[p];
        }
        __syncthreads();
        for (int e = threadIdx.x; e < nh * D; e += kWaves * kWave) {
            const int r = e / D, ch = e % D;
            float mx = sm_m[0][r], num = 0.f, den = 0.f;
#pragma unroll
            for (int w = 1; w < kWaves; ++w) mx = fmaxf(mx, sm_m[w][r]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = ex2(sm_m[w][r] - mx);
                num = fmaf(f, sm_o[w][r][ch], num);
                den = fmaf(f, sm_l[w][r], den);
            }
            const size_t ph = (size_t)split * Hq + hk * rep + p * HP + r;
            ws.part[ph * D + ch] = num;
            if (ch == 0) {
                ws.ml[2 * ph] = mx;
                ws.ml[2 * ph + 1] = den;
            }
        }
    }
}

template <int D, bool KV4, int NP>
void launch_bias(const DecCall &a, const DecWs &ws, int nsplit, int tps, hipStream_t st) {
    const int grid = dec_grid(a.Hkv, nsplit);
    if (a.mod.slopes)
        decode_cache_mfma_kernel<D, KV4, NP, true><<<grid, kWaves * kWave, 0, st>>>((const bf16_t *)a.q, a.c, ws, a.T, a.Hq, a.Hkv, tps, nsplit, a.mod);
    else
        decode_cache_mfma_kernel<D, KV4, NP, false><<<grid, kWaves * kWave, 0, st>>>((const bf16_t *)a.q, a.c, ws, a.T, a.Hq, a.Hkv, tps, nsplit, a.mod);
}

}  // namespace

// Rows are read at 32-bit offsets from the first of 32: any that fit a GPU's memory.
bool dec_mfma_supported(int Hq, int Hkv, int d, bool kv4, strd_dtype io) {
    if (io != STRD_BF16 || (d != 64 && d != 128) || Hkv > 8192) return false;
    const int rep = Hq / Hkv;
    return rep <= (kv4 && d == 128 ? 8 : 16);
}

// About 768 workgroups -- three on every CU, what their registers allow -- and 32 rows for each of their waves at least.
int dec_mfma_splits(int T, int Hkv, int &tps) {
    const int want = min(kDecMaxSplits, max(1, 768 / Hkv));
    tps = (int)(((long long)ceil_div(T, want) + kRound - 1) / kRound * kRound);
    return (int)(((long long)T + tps - 1) / tps);
}

void dec_mfma(const DecCall &a, const DecWs &ws, int nsplit, int tps, hipStream_t st) {
    const int rep = a.Hq / a.Hkv;
    if (a.kv4) {
        if (a.d == 128) {
            if (rep <= 4) launch_bias<128, true, 1>(a, ws, nsplit, tps, st);
            else launch_bias<128, true, 2>(a, ws, nsplit, tps, st);
        } else {
            if (rep <= 8) launch_bias<64, true, 1>(a, ws, nsplit, tps, st);
            else launch_bias<64, true, 2>(a, ws, nsplit, tps, st);
        }
    } else {
        if (a.d == 128) launch_bias<128, false, 1>(a, ws, nsplit, tps, st);
        else launch_bias<64, false, 1>(a, ws, nsplit, tps, st);
    }
}

}  // namespace strd
