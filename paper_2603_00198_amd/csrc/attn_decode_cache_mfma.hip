// One token's attention over a 4-bit or a plain bf16 cache on the matrix cores (heads of 64 or 128 channels, up to 16 query heads
// to a kv head, in 4 bits up to 8 of 128 channels): pass 1 of attn_decode_cache.hip, whose pass 2 joins the splits.
//
// The step is bound by reading the cache -- 5 bits per element -- if the vector instructions per element stay below about two:
// turning codes into numbers and multiplying them into up to 8 heads one by one takes six.  So both products are matrix products,
// on codes as they are:
//  * A code n becomes the bf16 number 16 + n by a shift and one instruction (its bits are the upper mantissa bits; exact).
//  * Scores: A = the codes of 16 rows, B = the query heads, a column for every (head, group of channels) with zeros outside the
//    group, and -24 sum q to start from.  The product leaves every group's sum of q (n - 8) apart; with the group's s and z it becomes
//    s * sum + z * sum q.  An accumulator's rows are rows of the cache, four to a lane, and the groups of a head are neighbouring
//    lanes: they exchange their parts so that each ends up with the whole score of one row of the four (two with two groups), whose cap, bias and
//    exponential only it computes.
//  * Values: A = the codes of V with the cache's rows as the contraction index, B = p * s -- p comes from the lane that has it with the
//    multiplication itself -- for every (head, group), as two bf16 numbers, its upper 8 bits and the rest, in two products: what is left out is
//    2^-16 of a weight, where bf16 alone left 2^-8 (a step over 131627 rows 59.4 -> 59.6 us, over 8491 plain ones 11.9 -> 12.0, with 8 heads to a kv head
//    71.6 -> 73.2).  A lane collects 8 rows' codes and regroups their halves.  What the 24 too many and z add does not depend on the channel: each lane sums
//    p z - 24 (both parts of p s) in fp32.  Rows (channels) of the product and columns of another group belong to nobody.
//  * A plain cache goes the same way without groups: columns are heads, values are regrouped halves.  The lower part is 2^-24 of the weight
//    at least there: where it is 0 an infinite value would become NaN.
// A wave takes 32 rows at a time, the next ones on their way; its softmax has one reference per head that moves when a score is
// 2^8 above it.  The last rows are read as the last 32 of the cache, those before them masked (their scores are -inf; a row that holds NaN has
// made the result NaN already), so that no read is clamped.  Weights: the scores go to the workspace as they come.
// 131627 rows of 8 heads of 128 in 4 bits, 32 query heads, cap, bias and weights: 51 us (170 MB, 3.3 TB/s), the reads alone 37 to 44;
// 843 rows 6.3 us.  Three trips on their way, or (s, z) read once for the heads and handed round, do not pass this (54 and 52 us).
#include "attn_decode_cache.h"

namespace strd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x2u __attribute__((ext_vector_type(2), aligned(4)));

constexpr int kTrip = 32;
constexpr float kLog2e = 1.4426950408889634f, kLazy = 8.f;
constexpr float kLeast = 0x1p-24f;  // least share of the lower part in a plain cache's weight

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
template <int P0, int P1, int P2, int P3>
__device__ __forceinline__ float quad(float v) {  // of lane P(its place) of this lane's quad
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), P0 | P1 << 2 | P2 << 4 | P3 << 6, 0xF, 0xF, true));
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
// Codes at bits 4 J and 16 + 4 J as a pair of bf16 numbers 16 + n: n belongs at bits 3 .. 6 of each half.  A bit-field insert into
// a register whose value the compiler does not know -- with a constant it comes out as an and and an or.  (The statement that hides it
// holds no instruction: one in inline assembly that writes a vector register is not kept apart from a matrix product's late write.)
struct CodeBits {
    uint32_t sixteen = 0x41804180u;
    __device__ __forceinline__ CodeBits() { asm("" : "+v"(sixteen)); }
    template <int J>
    __device__ __forceinline__ uint32_t pair(uint32_t x) const {
        constexpr uint32_t kMask = 0x00780078u;
        return ((J == 0 ? x << 3 : x >> (4 * J - 3)) & kMask) | (sixteen & ~kMask);
    }
};

template <int D, bool KV4>
struct Shape {
    static constexpr int kGroupsOfD = KV4 ? D / kKv4Group : 1;
    static constexpr int kHeads = 16 / kGroupsOfD;      // query heads per set of columns
    static constexpr int kKSteps = D / 32;              // products per 16 rows of keys
    static constexpr int kVTiles = D / 16;              // products per 32 rows of values
    static constexpr int kKDwords = KV4 ? D / 32 : D / 8;  // of a lane, per 16 rows
    static constexpr int kVDwords = KV4 ? 1 : D / 32;      // of a lane, per row (4 bits, D = 64: half of one)
};

// Long caches, from about 16 MB on: a workgroup is as many waves as a CU holds of them (three on a SIMD, or two), on `hw` neighbouring
// kv heads and the same rows: what heads share of a line of the cache -- two heads' codes, eight heads' (s, z) -- one CU fetches once.
// Shorter ones: four waves on one kv head, which start and join sooner.  us of a step with four waves / as many as fit: 8 heads of 128 in 4 bits,
// 843 rows 12.1 / 14.9, 6000 (8 MB) 15.9 / 16.9, 12000 (15 MB) 19.5 / 19.2, 131627 64.3 / 59.5; plain, 2500 (10 MB) 14.4 / 17.5, 6000
// (25 MB) 21.4 / 18.6, 131627 143 / 127; 4 heads of 64 in 4 bits, 50000 (16 MB) 21.2 / 21.2; plain, 12000 (12 MB) 16.6 / 17.3.
template <int D, bool KV4, int NP>
constexpr int dec_waves() { return NP == 1 && (KV4 || D == 64) ? 12 : 8; }
inline bool dec_long(int T, int Hkv, int d, bool kv4) { return (long long)T * Hkv * d * (kv4 ? 10 : 32) >= 8LL << 24; }
inline int dec_heads(int T, int Hkv, int d, bool kv4) { return !dec_long(T, Hkv, d, kv4) ? 1 : Hkv % 4 == 0 ? 4 : Hkv % 2 == 0 ? 2 : 1; }

template <int D, bool KV4, int NP, bool BIAS, int kWaves>
__global__ __launch_bounds__(kWaves * kWave) __attribute__((amdgpu_waves_per_eu(NP == 1 && (KV4 || D == 64) ? 3 : 2))) void decode_cache_mfma_kernel(
    const bf16_t *__restrict__ q, CacheView cv, DecWs ws, int Tn, int Hq, int Hkv, int hw, int tps, int nsplit, ScoreMod mod) {
    using S = Shape<D, KV4>;
    constexpr int NG = S::kGroupsOfD, HP = S::kHeads, KS = S::kKSteps, VT = S::kVTiles, KD = S::kKDwords, VD = S::kVDwords;
    constexpr int RL = 4 / NG;  // rows of a lane's four whose scores it ends up with
    extern __shared__ __attribute__((aligned(16))) float sm[];  // [kWaves][hs][D] values, [kWaves][hs] references and sums
    int hg, split;
    dec_place(blockIdx.x, Hkv / hw, hg, split);
    if (split >= nsplit) return;  // uniform
    const int rep = Hq / Hkv, hs = min(HP, rep);
    float *const sm_m = sm + kWaves * hs * D, *const sm_l = sm_m + kWaves * hs;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int hk = hg * hw + wave % hw, round = kWaves / hw * kTrip;  // this wave's kv head; rows of all waves' trips
    const int lr = lane & 15, c = lane >> 4;
    const int grp = lr % NG, hcol = lr / NG;             // this lane's column: head, group of channels
    const int kgrp = KV4 ? c * (D / 4) / kKv4Group : 0;  // group of the channels this lane holds of a key
    const int row_l = 4 * c + RL * grp;                   // first of its rows, of 16
    const int begin = split * tps, t_end = min(Tn, begin + tps);

    struct Rows {
        uint32_t k[2][KD], v[8][VD], km[KV4 ? 8 : 1], vm[KV4 ? 8 : 1];
        int32_t pos[BIAS ? 2 : 1][RL];
    };
    // 32 rows of this kv head from `base` on, all of them in the cache: a buffer of 32 rows for each side (whose size bounds every
    // read), one offset a lane, and a uniform one for the row; no address is computed by a vector instruction.
    const uint32_t kv_row = (uint32_t)Hkv * (KV4 ? D / 2 : D * 2), m_row = (uint32_t)Hkv * (NG * 4);
    const uint32_t koff = hk * (KV4 ? D / 2 : D * 2) + lr * kv_row + (KV4 ? c * (D / 8) : 16 * c);
    const uint32_t voff = hk * (KV4 ? D / 2 : D * 2) + 4 * c * kv_row + lr * (KV4 ? D / 32 : D / 8), moff = hk * (NG * 4) + 4 * c * m_row + 4 * grp;
    auto rows_of = [&](const void *p, int base, uint32_t row) __attribute__((always_inline)) {
        return __builtin_amdgcn_make_buffer_rsrc((char *)const_cast<void *>(p) + (size_t)base * row, (short)0, (int)(kTrip * row), 0x00027000);
    };
    auto load = [&](int base, Rows &x) __attribute__((always_inline)) {
        const auto kb = rows_of(cv.k, base, kv_row), vb = rows_of(cv.v, base, kv_row);
        const auto kmb = rows_of(cv.km, base, m_row), vmb = rows_of(cv.vm, base, m_row);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t at = 16 * u * kv_row;
            if constexpr (KV4 && D == 128) {
                const u32x4 d = __builtin_amdgcn_raw_buffer_load_b128(kb, koff, at, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) x.k[u][i] = d[i];
            } else if constexpr (KV4) {
                const u32x2 d = __builtin_amdgcn_raw_buffer_load_b64(kb, koff, at, 0);
                x.k[u][0] = d[0];
                x.k[u][1] = d[1];
            } else {
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    const u32x4 d = __builtin_amdgcn_raw_buffer_load_b128(kb, koff + 64 * i, at, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.k[u][4 * i + e] = d[e];
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t row = 16 * (e >> 2) + (e & 3);
            if constexpr (KV4 && D == 128) {
                x.v[e][0] = __builtin_amdgcn_raw_buffer_load_b32(vb, voff, row * kv_row, 0);
            } else if constexpr (KV4) {
                x.v[e][0] = __builtin_amdgcn_raw_buffer_load_b16(vb, voff, row * kv_row, 0);
            } else if constexpr (D == 128) {
                const u32x4 d = __builtin_amdgcn_raw_buffer_load_b128(vb, voff, row * kv_row, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) x.v[e][i] = d[i];
            } else {
                const u32x2 d = __builtin_amdgcn_raw_buffer_load_b64(vb, voff, row * kv_row, 0);
                x.v[e][0] = d[0];
                x.v[e][1] = d[1];
            }
            if constexpr (KV4) {
                x.km[e] = __builtin_amdgcn_raw_buffer_load_b32(kmb, moff, row * m_row, 0);
                x.vm[e] = __builtin_amdgcn_raw_buffer_load_b32(vmb, moff, row * m_row, 0);
            }
        }
        if constexpr (BIAS) {
            // (without positions a buffer of no bytes: reads that return 0 and are not looked at, but no branch, behind which every
            // outstanding read would be waited for)
            const auto pb = __builtin_amdgcn_make_buffer_rsrc((char *)const_cast<int32_t *>(mod.pos) + (mod.pos ? (size_t)base * 4 : 0), (short)0,
                                                              mod.pos ? kTrip * 4 : 0, 0x00027000);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < RL; ++k) x.pos[u][k] = __builtin_amdgcn_raw_buffer_load_b32(pb, 4 * row_l + 4 * k, 64 * u, 0);
        }
    };
    Rows xa, xb;
    const CodeBits bits;
    // trips from the last to the first: with a bias from far to near the softmax reference would move in every one
    const int t_first = begin + kTrip * (wave / hw), trips = t_first < t_end ? (t_end - t_first + round - 1) / round : 0;
    auto trip_at = [&](int i) { return t_first + max(trips - 1 - i, 0) * round; };
    load(min(trip_at(0), Tn - kTrip), xa);

    // the query heads: B operand, column (hcol, grp), k slots as the keys' codes come (the pairs of CodeBits), zeros outside
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
        slope[p] = BIAS && hh < rep ? fminf(fmaxf(mod.slopes[hk * rep + hh] * kLog2e, -1e30f), 1e30f) : 0.f;  // (infinity times 0 is NaN)
        m[p] = kDecNegBig;
        l[p] = corr[p] = 0.f;
#pragma unroll
        for (int j = 0; j < VT; ++j) oacc[p][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float pos_q = 0.f;
    if constexpr (BIAS) pos_q = mod.pos ? (float)mod.pos[Tn - 1] : (float)(Tn - 1);
    const size_t soff = (size_t)hcol * ws.ldt + row_l;
    const bool capped = mod.cap > 0.f;  // uniform
    const float dot_scale = capped ? mod.scale * mod.inv_cap : mod.scale * kLog2e, cap2 = mod.cap * kLog2e;

    // the 32 rows from t0 on, in x those from min(t0, Tn - 32) on
    auto fold = [&](int t0, const Rows &x) __attribute__((always_inline)) {
        const int base = min(t0, Tn - kTrip);
        const bool all = base == t0;  // uniform
        bf16x8 pb[NP], pl[NP];        // p (4 bits: p * s of the column's group) of the 32 rows, the next product's operand: upper and lower bits
        float pr[NP][2][RL];
        // ---- scores ----
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            bf16x8 ka[KS];
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                if constexpr (KV4)
                    ka[i] = __builtin_bit_cast(bf16x8, u32x4{bits.pair<0>(x.k[u][i]), bits.pair<1>(x.k[u][i]), bits.pair<2>(x.k[u][i]), bits.pair<3>(x.k[u][i])});
                else
                    ka[i] = __builtin_bit_cast(bf16x8, u32x4{x.k[u][4 * i], x.k[u][4 * i + 1], x.k[u][4 * i + 2], x.k[u][4 * i + 3]});
            }
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const float start = KV4 ? -24.f * qsum[p] : 0.f;
                f32x4 z = f32x4{start, start, start, start};
#pragma unroll
                for (int i = 0; i < KS; ++i) z = mfma16(ka[i], bq[p][i], z);
                if constexpr (KV4) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const Kv4Group g = kv4_meta(x.km[4 * u + i]);
                        z[i] = fmaf(g.s, z[i], g.z * qsum[p]);
                    }
                }
                // the groups' parts meet: a lane keeps its rows and hands the others on
                if constexpr (NG == 4) {
                    const bool hi = grp & 2, odd = grp & 1;
                    float k0 = hi ? z[2] : z[0], k1 = hi ? z[3] : z[1];
                    const float g0 = hi ? z[0] : z[2], g1 = hi ? z[1] : z[3];
                    k0 += quad<2, 3, 0, 1>(g0);
                    k1 += quad<2, 3, 0, 1>(g1);
                    pr[p][u][0] = (odd ? k1 : k0) + quad<1, 0, 3, 2>(odd ? k0 : k1);
                } else if constexpr (NG == 2) {
                    const bool odd = grp & 1;
                    pr[p][u][0] = (odd ? z[2] : z[0]) + quad<1, 0, 3, 2>(odd ? z[0] : z[2]);
                    pr[p][u][1] = (odd ? z[3] : z[1]) + quad<1, 0, 3, 2>(odd ? z[1] : z[3]);
                } else {
#pragma unroll
                    for (int k = 0; k < RL; ++k) pr[p][u][k] = z[k];
                }
            }
        }
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < RL; ++k) pr[p][u][k] *= dot_scale;
        if (capped) {
            float far = 0.f;
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int k = 0; k < RL; ++k) far = fmaxf(far, fabsf(pr[p][u][k]));
            // tanh(y) / y up to y = 0.5, as a polynomial in y^2 of least relative error (1.3e-8)
            auto capped = [&](auto beyond) __attribute__((always_inline)) {
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int k = 0; k < RL; ++k) {
                            const float y = pr[p][u][k], w = y * y;
                            float r = fmaf(w, 0.0171347708f, -0.0529858599f);
                            r = fmaf(w, r, 0.133247737f);
                            r = fmaf(w, r, -0.333330689f);
                            r = fmaf(w, r, 0.999999987f);
                            pr[p][u][k] = cap2 * y * r;
                            if constexpr (beyond) pr[p][u][k] = fabsf(y) <= 0.5f ? pr[p][u][k] : cap2 * tanhf(y);
                        }
            };
            if (__any(far > 0.5f)) capped(std::true_type());
            else capped(std::false_type());
        }
        if constexpr (BIAS) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < RL; ++k) {
                    const float far = fabsf(pos_q - (float)(mod.pos ? x.pos[u][k] : base + 16 * u + row_l + k));
#pragma unroll
                    for (int p = 0; p < NP; ++p) pr[p][u][k] = fmaf(-slope[p], far, pr[p][u][k]);
                }
        }
        if (!all) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < RL; ++k)
#pragma unroll
                    for (int p = 0; p < NP; ++p) pr[p][u][k] = base + 16 * u + row_l + k < t0 ? -INFINITY : pr[p][u][k];
        }
        if (ws.scores) {  // uniform
            float *const sc = ws.scores + (size_t)(hk * rep) * ws.ldt + base;  // uniform
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (p * HP + hcol < rep)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        float *const at = sc + (size_t)(p * HP) * ws.ldt + 16 * u + soff;
                        if (all) {
                            if constexpr (RL == 4) *reinterpret_cast<f32x4u *>(at) = f32x4u{pr[p][u][0], pr[p][u][1], pr[p][u][2], pr[p][u][3]};
                            else if constexpr (RL == 2) *reinterpret_cast<f32x2u *>(at) = f32x2u{pr[p][u][0], pr[p][u][1]};
                            else at[0] = pr[p][u][0];
                        } else {
#pragma unroll
                            for (int k = 0; k < RL; ++k)
                                if (base + 16 * u + row_l + k >= t0) at[k] = pr[p][u][k];
                        }
                    }
        }
        // halves of two dwords side by side: lo of both, hi of both
        auto pair_lo = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); };
        auto pair_hi = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); };
        // ---- softmax ----
        float tm[NP];
        bool moves = false;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            tm[p] = pr[p][0][0];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < RL; ++k) tm[p] = fmaxf(tm[p], pr[p][u][k]);
            moves |= tm[p] > m[p] + kLazy;
        }
        if (__any(moves)) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                float t = tm[p];
                if constexpr (NG >= 2) t = fmaxf(t, quad<1, 0, 3, 2>(t));
                if constexpr (NG == 4) t = fmaxf(t, quad<2, 3, 0, 1>(t));
                const float nm = fmaxf(m[p], quarters_max(t)), f = ex2(m[p] - nm);
                m[p] = nm;
                l[p] *= f;
                corr[p] *= f;
#pragma unroll
                for (int j = 0; j < VT; ++j) oacc[p][j] *= f;
            }
        }
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            uint32_t w[4], wl[4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float e[RL], ps[4];
#pragma unroll
                for (int k = 0; k < RL; ++k) {
                    e[k] = ex2(pr[p][u][k] - m[p]);
                    l[p] += e[k];
                }
                auto of_row = [&](auto ic) __attribute__((always_inline)) {
                    constexpr int I = decltype(ic)::value;
                    float pi;
                    if constexpr (NG == 4) pi = quad<I, I, I, I>(e[0]);
                    else if constexpr (NG == 2) pi = quad<I / 2, I / 2, 2 + I / 2, 2 + I / 2>(e[I % 2]);
                    else pi = e[I % RL];
                    if constexpr (KV4) {
                        const Kv4Group g = kv4_meta(x.vm[4 * u + I]);
                        ps[I] = pi * g.s;
                        corr[p] = fmaf(pi, g.z, corr[p]);
                    } else {
                        ps[I] = pi;
                    }
                };
                of_row(std::integral_constant<int, 0>());
                of_row(std::integral_constant<int, 1>());
                of_row(std::integral_constant<int, 2>());
                of_row(std::integral_constant<int, 3>());
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t a = __builtin_bit_cast(uint32_t, ps[2 * i]), b = __builtin_bit_cast(uint32_t, ps[2 * i + 1]);
                    float la = ps[2 * i] - __builtin_bit_cast(float, a & 0xFFFF0000u), lb = ps[2 * i + 1] - __builtin_bit_cast(float, b & 0xFFFF0000u);
                    if constexpr (!KV4) la = fmaxf(la, kLeast * ps[2 * i]), lb = fmaxf(lb, kLeast * ps[2 * i + 1]);
                    w[2 * u + i] = pair_hi(a, b);
                    wl[2 * u + i] = bf16_pair(la, lb);
                }
            }
            if constexpr (KV4) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    corr[p] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[i]), bf16x2{(bf16_t)-24.f, (bf16_t)-24.f}, corr[p], false);
                    corr[p] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, wl[i]), bf16x2{(bf16_t)-24.f, (bf16_t)-24.f}, corr[p], false);
                }
            }
            pb[p] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
            pl[p] = __builtin_bit_cast(bf16x8, u32x4{wl[0], wl[1], wl[2], wl[3]});
        }
        // ---- values ----
        uint32_t lo[4][VD], hi[4][VD];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < VD; ++i) {
                uint32_t a = x.v[2 * e][i], b = x.v[2 * e + 1][i];
                if (!KV4 && !all) {  // (a probability of 0 times what is not finite)
                    const int row = base + 16 * (e >> 1) + 4 * c + 2 * (e & 1);
                    a = row < t0 ? 0u : a;
                    b = row + 1 < t0 ? 0u : b;
                }
                lo[e][i] = pair_lo(a, b);
                hi[e][i] = pair_hi(a, b);
            }
        auto product = [&](auto jc) __attribute__((always_inline)) {
            constexpr int J = decltype(jc)::value;
            if constexpr (J < VT) {
                u32x4 a;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (KV4)
                        a[e] = bits.template pair<J % 4>(J < 4 ? lo[e][0] : hi[e][0]);
                    else
                        a[e] = J % 2 ? hi[e][J / 2] : lo[e][J / 2];
                }
#pragma unroll
                for (int p = 0; p < NP; ++p) oacc[p][J] = mfma16(__builtin_bit_cast(bf16x8, a), pb[p], oacc[p][J]);
#pragma unroll
                for (int p = 0; p < NP; ++p) oacc[p][J] = mfma16(__builtin_bit_cast(bf16x8, a), pl[p], oacc[p][J]);
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

    for (int i = 0; i < trips; i += 2) {
        load(min(trip_at(i + 1), Tn - kTrip), xb);
        fold(trip_at(i), xa);
        load(min(trip_at(i + 2), Tn - kTrip), xa);
        if (i + 1 < trips) fold(trip_at(i + 1), xb);
    }

    // ---- the waves of a kv head join, one set of query heads at a time ----
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int nh = min(HP, rep - p * HP);
        if (nh <= 0) break;  // uniform
        if (p) __syncthreads();
        if constexpr (NG >= 2) l[p] += quad<1, 0, 3, 2>(l[p]);
        if constexpr (NG == 4) l[p] += quad<2, 3, 0, 1>(l[p]);
        l[p] = quarters_sum(l[p]);
        corr[p] = quarters_sum(corr[p]);
        // rows 4 c + i of product j are channels VT (4 c + i) + j; a lane's column counts for its own group's channels
        if (hcol < nh && (!KV4 || grp == VT * 4 * c / kKv4Group)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < VT; j += 4)
                    *reinterpret_cast<f32x4 *>(sm + (wave * hs + hcol) * D + VT * (4 * c + i) + j) =
                        f32x4{oacc[p][j][i] + corr[p], oacc[p][j + 1][i] + corr[p], oacc[p][j + 2][i] + corr[p], oacc[p][j + 3][i] + corr[p]};
        }
        if (c == 0 && grp == 0 && hcol < nh) {
            sm_m[wave * hs + hcol] = m[p];
            sm_l[wave * hs + hcol] = l[p];
        }
        __syncthreads();
        for (int e = threadIdx.x; e < hw * nh * D; e += kWaves * kWave) {
            const int r = e / D % nh, ch = e % D, hl = e / (D * nh);
            float mx = kDecNegBig, num = 0.f, den = 0.f;
            for (int w = hl; w < kWaves; w += hw) mx = fmaxf(mx, sm_m[w * hs + r]);
            for (int w = hl; w < kWaves; w += hw) {
                const float f = ex2(sm_m[w * hs + r] - mx);
                num = fmaf(f, sm[(w * hs + r) * D + ch], num);
                den = fmaf(f, sm_l[w * hs + r], den);
            }
            const size_t ph = (size_t)split * Hq + (hg * hw + hl) * rep + p * HP + r;
            ws.part[ph * D + ch] = num;
            if (ch == 0) {
                ws.ml[2 * ph] = mx;
                ws.ml[2 * ph + 1] = den;
            }
        }
    }
}

template <int D, bool KV4, int NP, int kWaves>
int launch_waves(const DecCall &a, const DecWs &ws, int nsplit, int tps, hipStream_t st) {
    const int hw = dec_heads(a.T, a.Hkv, D, KV4), grid = dec_grid(a.Hkv / hw, nsplit), hs = min(Shape<D, KV4>::kHeads, a.Hq / a.Hkv);
    const size_t smem = (size_t)kWaves * hs * (D + 2) * sizeof(float);
    auto launch = [&](auto kernel) {
        if (smem > 65536 && !allow_dynamic_lds(reinterpret_cast<const void *>(kernel), (size_t)kWaves * Shape<D, KV4>::kHeads * (D + 2) * sizeof(float)))
            return (int)STRD_EHIP;
        kernel<<<grid, kWaves * kWave, smem, st>>>((const bf16_t *)a.q, a.c, ws, a.T, a.Hq, a.Hkv, hw, tps, nsplit, a.mod);
        return launch_status();
    };
    return a.mod.slopes ? launch(&decode_cache_mfma_kernel<D, KV4, NP, true, kWaves>) : launch(&decode_cache_mfma_kernel<D, KV4, NP, false, kWaves>);
}
template <int D, bool KV4, int NP>
int launch_bias(const DecCall &a, const DecWs &ws, int nsplit, int tps, hipStream_t st) {
    return dec_long(a.T, a.Hkv, D, KV4) ? launch_waves<D, KV4, NP, dec_waves<D, KV4, NP>()>(a, ws, nsplit, tps, st) : launch_waves<D, KV4, NP, 4>(a, ws, nsplit, tps, st);
}

}  // namespace

// 32 rows are read at a time, at 32-bit offsets from the first: caches of 32 rows at least (fewer: the launches' latency, whatever
// is launched), of up to 8192 heads.
bool dec_mfma_supported(int T, int Hq, int Hkv, int d, bool kv4, strd_dtype io) {
    if (T < kTrip || io != STRD_BF16 || (d != 64 && d != 128) || Hkv > 8192) return false;
    const int rep = Hq / Hkv;
    return rep <= (kv4 && d == 128 ? 8 : 16);
}

// Long: a workgroup on every CU.  Short: a trip for each of the four waves, up to three workgroups on every CU.
int dec_mfma_splits(int T, int Hkv, int d, bool kv4, int &tps) {
    const bool longer = dec_long(T, Hkv, d, kv4);
    const int hw = dec_heads(T, Hkv, d, kv4), round = (longer ? 12 / hw : 4) * kTrip;
    const int want = min(kDecMaxSplits, max(1, (longer ? 256 * hw : 768) / Hkv));
    tps = (int)(((long long)ceil_div(T, want) + round - 1) / round * round);
    return (int)(((long long)T + tps - 1) / tps);
}

int dec_mfma(const DecCall &a, const DecWs &ws, int nsplit, int tps, hipStream_t st) {
    const int rep = a.Hq / a.Hkv;
    if (a.kv4 && a.d == 128)
        return rep <= 4 ? launch_bias<128, true, 1>(a, ws, nsplit, tps, st) : launch_bias<128, true, 2>(a, ws, nsplit, tps, st);
    if (a.kv4) return rep <= 8 ? launch_bias<64, true, 1>(a, ws, nsplit, tps, st) : launch_bias<64, true, 2>(a, ws, nsplit, tps, st);
    return a.d == 128 ? launch_bias<128, false, 1>(a, ws, nsplit, tps, st) : launch_bias<64, false, 1>(a, ws, nsplit, tps, st);
}

}  // namespace strd
