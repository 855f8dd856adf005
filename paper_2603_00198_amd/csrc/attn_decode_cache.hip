// One token's attention over a cache, plain or in 4 bits, with capped scores, a bias by distance and the attention weight that
// every row has gathered (the cap, the bias and the weights: strd.h).  Any head size up to 256, any number of heads, fp32
// arithmetic; the shapes of attn_decode_cache_mfma.hip run there.
//
// Pass 1: a workgroup takes one kv head's share of the tokens, and up to 8 of its query heads.  16 lanes hold a token's
// row, 8 neighbouring channels each (two such pieces above 128 channels), and 4 tokens are on their way together; a lane
// group has a softmax of its own, and the 16 of a workgroup meet in LDS.  Where weights are wanted the scores go to the workspace.
// Pass 2: a workgroup per 32 output channels of a head joins the splits; others turn the scores of 1024 tokens into weights,
// once the heads' references and sums over all splits are known: w = w_in + mean over the heads of 2^(score - ref) / sum.
#include "attn_decode_cache.h"

namespace strd {
namespace {

constexpr int kThreads = 256, kLanes = 16, kGroups = kThreads / kLanes, kTok = 4;
constexpr float kLog2e = 1.4426950408889634f;

template <typename T> struct Vec8;
template <> struct Vec8<bf16_t> {
    typedef __bf16 type __attribute__((ext_vector_type(8)));
};
template <> struct Vec8<float> {
    typedef float type __attribute__((ext_vector_type(8)));
};

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

// Channels 8 c .. 8 c + 7 of row `row` (a row of all heads is Hkv * d channels, `at` the head's first channel).
template <typename T, bool KV4, bool VEC>
__device__ __forceinline__ void load8(const void *rows, const void *meta, size_t at, int c, int d, float (&x)[8]) {
    if constexpr (KV4) {
        const size_t u = at / 8 + c;
        const uint32_t codes = reinterpret_cast<const uint32_t *>(rows)[u];
        const Kv4Group g = kv4_meta(reinterpret_cast<const uint32_t *>(meta)[u / 4]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = kv4_value(codes, e, g);
    } else if constexpr (VEC) {
        typedef typename Vec8<T>::type V;
        const V t = *reinterpret_cast<const V *>((const T *)rows + at + 8 * c);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = to_f32((T)t[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 8 * c + e < d ? to_f32(((const T *)rows + at)[min(8 * c + e, d - 1)]) : 0.f;
    }
}

template <typename T, bool KV4, bool VEC, int RP, int NC>
__global__ __launch_bounds__(kThreads) void decode_cache_kernel(const T *__restrict__ q, CacheView c, DecWs ws, int Tn, int Hq, int Hkv,
                                                                int d, int tps, ScoreMod mod) {
    extern __shared__ float sm_acc[];  // [kGroups][d]
    __shared__ float sm_m[kGroups][RP], sm_l[kGroups][RP];
    const int hk = blockIdx.x, split = blockIdx.y, rep = Hq / Hkv, r0 = blockIdx.z * RP;
    const int grp = threadIdx.x / kLanes, sub = threadIdx.x % kLanes;
    const int nh = min(RP, rep - r0), h0 = hk * rep + r0;
    float qv[RP][NC][8], acc[RP][NC][8], m[RP], l[RP], slope[RP];
#pragma unroll
    for (int r = 0; r < RP; ++r) {
        m[r] = kDecNegBig;
        l[r] = 0.f;
        slope[r] = mod.slopes && r < nh ? mod.slopes[h0 + r] : 0.f;
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const int ch = 8 * (sub + kLanes * n);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                qv[r][n][e] = r < nh && ch + e < d ? to_f32(q[(size_t)(h0 + r) * d + ch + e]) : 0.f;
                acc[r][n][e] = 0.f;
            }
        }
    }
    const int t_begin = split * tps, t_end = (int)min((long long)Tn, (long long)t_begin + tps);
    const float pos_q = mod.pos ? (float)mod.pos[Tn - 1] : (float)(Tn - 1);
    for (int t0 = t_begin + grp; t0 < t_end; t0 += kGroups * kTok) {
        float kx[kTok][NC][8], vx[kTok][NC][8], far[kTok];
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            const int t = min(t0 + kGroups * u, t_end - 1);  // rows behind the split's last are read again, and not counted
            const size_t at = ((size_t)t * Hkv + hk) * d;
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                const int cc = sub + kLanes * n, cl = min(cc, (d - 1) / 8);  // (lanes behind the row re-read its last piece)
                load8<T, KV4, VEC>(c.k, c.km, at, cl, d, kx[u][n]);
                load8<T, KV4, VEC>(c.v, c.vm, at, cl, d, vx[u][n]);
            }
            far[u] = mod.pos ? fabsf(pos_q - (float)mod.pos[t]) : fabsf(pos_q - (float)t);
        }
        float x[kTok][RP];
#pragma unroll
        for (int r = 0; r < RP; ++r) {
            float mn = m[r];
#pragma unroll
            for (int u = 0; u < kTok; ++u) {
                float dot = 0.f;
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    if (8 * (sub + kLanes * n) < d)
#pragma unroll
                        for (int e = 0; e < 8; ++e) dot = fmaf(qv[r][n][e], kx[u][n][e], dot);
                const int t = t0 + kGroups * u;
                x[u][r] = (capped_score(mod, group_sum(dot)) - slope[r] * far[u]) * kLog2e;
                if (ws.scores && sub == 0 && r < nh && t < t_end) ws.scores[(size_t)(h0 + r) * ws.ldt + t] = x[u][r];
                if (t < t_end) mn = fmaxf(mn, x[u][r]);
            }
            const float corr = ex2(m[r] - mn);
            m[r] = mn;
            l[r] *= corr;
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[r][n][e] *= corr;
#pragma unroll
            for (int u = 0; u < kTok; ++u) {
                if (t0 + kGroups * u >= t_end) continue;
                const float p = ex2(x[u][r] - mn);
                l[r] += p;
#pragma unroll
                for (int n = 0; n < NC; ++n)
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[r][n][e] = fmaf(p, vx[u][n][e], acc[r][n][e]);
            }
        }
    }
    if (sub == 0)
#pragma unroll
        for (int r = 0; r < RP; ++r) {
            sm_m[grp][r] = m[r];
            sm_l[grp][r] = l[r];
        }
#pragma unroll
    for (int r = 0; r < RP; ++r) {
        if (r >= nh) break;  // uniform
        if (r) __syncthreads();
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int ch = 8 * (sub + kLanes * n) + e;
                if (ch < d) sm_acc[grp * d + ch] = acc[r][n][e];
            }
        __syncthreads();
        float mx = sm_m[0][r];
#pragma unroll
        for (int g = 1; g < kGroups; ++g) mx = fmaxf(mx, sm_m[g][r]);
        float wt[kGroups], den = 0.f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            wt[g] = ex2(sm_m[g][r] - mx);
            den = fmaf(wt[g], sm_l[g][r], den);
        }
        const size_t ph = (size_t)split * Hq + h0 + r;
        for (int ch = threadIdx.x; ch < d; ch += kThreads) {
            float num = 0.f;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) num = fmaf(wt[g], sm_acc[g * d + ch], num);  // fixed order
            ws.part[ph * d + ch] = num;
        }
        if (threadIdx.x == 0) {
            ws.ml[2 * ph] = mx;
            ws.ml[2 * ph + 1] = den;
        }
    }
}

// Reference and reciprocal sum of one head over all splits, by the 64 lanes of a wave.
__device__ __forceinline__ void head_total(const float *__restrict__ ml, int nsplit, int Hq, int h, float &mx, float &den) {
    const int lane = threadIdx.x % kWave;
    float2 pr[kDecMaxSplits / kWave];
    mx = kDecNegBig;
#pragma unroll
    for (int i = 0; i < kDecMaxSplits / kWave; ++i) {
        if (i * kWave >= nsplit) break;  // uniform
        pr[i] = *reinterpret_cast<const float2 *>(ml + ((size_t)min(lane + kWave * i, nsplit - 1) * Hq + h) * 2);
        mx = fmaxf(mx, pr[i].x);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, kWave));
    den = 0.f;
#pragma unroll
    for (int i = 0; i < kDecMaxSplits / kWave; ++i) {
        if (i * kWave >= nsplit) break;
        if (lane + kWave * i < nsplit) den = fmaf(ex2(pr[i].x - mx), pr[i].y, den);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) den += __shfl_xor(den, o, kWave);
}

constexpr int kHeadsAtOnce = 64, kTokPerBlock = 4 * kThreads;

template <typename T>
__global__ __launch_bounds__(kThreads) void decode_combine_kernel(DecWs ws, T *__restrict__ o, const float *__restrict__ w_in,
                                                                  float *__restrict__ w_out, int nsplit, int Tn, int Hq, int d,
                                                                  int o_blocks) {
    __shared__ float wts[kDecMaxSplits], tot[2], sums[8][33], hm[kHeadsAtOnce], hl[kHeadsAtOnce];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    if ((int)blockIdx.x < o_blocks) {
        const int per = (d + 31) / 32, h = blockIdx.x / per, c = (blockIdx.x % per) * 32 + tid % 32, sg = tid / 32;
        if (wave == 0) {
            float mx, den;
            head_total(ws.ml, nsplit, Hq, h, mx, den);
            for (int s = lane; s < nsplit; s += kWave) wts[s] = ex2(ws.ml[((size_t)s * Hq + h) * 2] - mx);
            if (lane == 0) tot[0] = den;
        }
        __syncthreads();
        float acc = 0.f;
        if (c < d)
            for (int s = sg; s < nsplit; s += 8) acc = fmaf(wts[s], ws.part[((size_t)s * Hq + h) * d + c], acc);
        sums[sg][tid % 32] = acc;
        __syncthreads();
        if (tid < 32 && c < d) {
            float num = 0.f;
#pragma unroll
            for (int g = 0; g < 8; ++g) num += sums[g][tid];  // fixed order
            o[(size_t)h * d + c] = from_f32<T>(num / tot[0]);
        }
        return;
    }
    const long long t0 = (long long)(blockIdx.x - o_blocks) * kTokPerBlock + tid;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int h0 = 0; h0 < Hq; h0 += kHeadsAtOnce) {
        const int nh = min(kHeadsAtOnce, Hq - h0);
        __syncthreads();
        for (int h = wave; h < nh; h += kThreads / kWave) {
            float mx, den;
            head_total(ws.ml, nsplit, Hq, h0 + h, mx, den);
            if (lane == 0) {
                hm[h] = mx;
                hl[h] = 1.f / den;
            }
        }
        __syncthreads();
        for (int h = 0; h < nh; ++h) {
            const float *s = ws.scores + (size_t)(h0 + h) * ws.ldt;
#pragma unroll
            for (int u = 0; u < 4; ++u) acc[u] = fmaf(ex2(s[min(t0 + kThreads * u, (long long)Tn - 1)] - hm[h]), hl[h], acc[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const long long t = t0 + kThreads * u;
        if (t < Tn) w_out[t] = (w_in ? w_in[t] : 0.f) + acc[u] / (float)Hq;
    }
}

template <typename T, bool KV4, bool VEC, int RP>
void launch_rp(const DecCall &a, const DecWs &ws, int nsplit, int tps, hipStream_t st) {
    const dim3 grid(a.Hkv, nsplit, ceil_div(a.Hq / a.Hkv, RP));
    const size_t smem = (size_t)kGroups * a.d * sizeof(float);
    if (a.d <= 128)
        decode_cache_kernel<T, KV4, VEC, RP, 1><<<grid, kThreads, smem, st>>>((const T *)a.q, a.c, ws, a.T, a.Hq, a.Hkv, a.d, tps, a.mod);
    else
        decode_cache_kernel<T, KV4, VEC, RP, 2><<<grid, kThreads, smem, st>>>((const T *)a.q, a.c, ws, a.T, a.Hq, a.Hkv, a.d, tps, a.mod);
}

template <typename T, bool KV4, bool VEC>
void launch_cache(const DecCall &a, const DecWs &ws, int nsplit, int tps, hipStream_t st) {
    const int rep = a.Hq / a.Hkv;
    if (rep == 1) launch_rp<T, KV4, VEC, 1>(a, ws, nsplit, tps, st);
    else if (rep == 2) launch_rp<T, KV4, VEC, 2>(a, ws, nsplit, tps, st);
    else launch_rp<T, KV4, VEC, 4>(a, ws, nsplit, tps, st);
}

template <typename T>
void launch_typed(const DecCall &a, const DecWs &ws, int nsplit, int tps, hipStream_t st) {
    const size_t al = 8 * sizeof(T);
    if (a.kv4) launch_cache<T, true, true>(a, ws, nsplit, tps, st);
    else if (a.d % 8 == 0 && !((uintptr_t)a.c.k % al) && !((uintptr_t)a.c.v % al)) launch_cache<T, false, true>(a, ws, nsplit, tps, st);
    else launch_cache<T, false, false>(a, ws, nsplit, tps, st);
}

}  // namespace

// About 512 workgroups, and a trip of all lane groups for each at least.
int dec_splits_general(int T, int Hq, int Hkv, int &tps) {
    const int passes = ceil_div(Hq / Hkv, 4);
    const int want = min(kDecMaxSplits, max(1, (int)(512 / min(512LL, (long long)Hkv * passes))));
    tps = (int)(((long long)ceil_div(T, want) + kGroups * kTok - 1) / (kGroups * kTok) * (kGroups * kTok));
    return (int)(((long long)T + tps - 1) / tps);
}

int dec_combine(const DecCall &a, const DecWs &ws, int nsplit, hipStream_t st) {
    const int o_blocks = a.Hq * ceil_div(a.d, 32), w_blocks = a.w_out ? (int)(((long long)a.T + kTokPerBlock - 1) / kTokPerBlock) : 0;
    if (a.io == STRD_BF16)
        decode_combine_kernel<bf16_t><<<o_blocks + w_blocks, kThreads, 0, st>>>(ws, (bf16_t *)a.o, a.w_in, a.w_out, nsplit, a.T, a.Hq, a.d, o_blocks);
    else
        decode_combine_kernel<float><<<o_blocks + w_blocks, kThreads, 0, st>>>(ws, (float *)a.o, a.w_in, a.w_out, nsplit, a.T, a.Hq, a.d, o_blocks);
    return launch_status();
}

size_t attn_decode_cache_ws(int T, int Hq, int Hkv, int d, bool kv4, bool weights, strd_dtype io) {
    // (a plain cache that 16-byte reads do not fit takes the general kernel whatever its shape: room for either's splits)
    int tps, n = dec_splits_general(T, Hq, Hkv, tps);
    if (dec_mfma_supported(Hq, Hkv, d, kv4, io)) n = kv4 ? dec_mfma_splits(T, Hkv, tps) : max(n, dec_mfma_splits(T, Hkv, tps));
    return dec_ws_bytes(n, Hq, d, dec_ldt(T), weights);
}

int attn_decode_cache(const DecCall &a, void *wsp, hipStream_t st) {
    const bool mfma = dec_mfma_supported(a.Hq, a.Hkv, a.d, a.kv4, a.io) && (((uintptr_t)a.q | (uintptr_t)a.c.k | (uintptr_t)a.c.v) & 15) == 0;
    DecWs ws;
    int tps;
    const int nsplit = mfma ? dec_mfma_splits(a.T, a.Hkv, tps) : dec_splits_general(a.T, a.Hq, a.Hkv, tps);
    ws.ml = (float *)wsp;  // (pairs: they come first)
    ws.part = ws.ml + (size_t)nsplit * a.Hq * 2;
    ws.ldt = dec_ldt(a.T);
    ws.scores = a.w_out ? (float *)((char *)wsp + align_up((size_t)nsplit * a.Hq * (a.d + 2) * sizeof(float), 256)) : nullptr;
    if (mfma) dec_mfma(a, ws, nsplit, tps, st);
    else if (a.io == STRD_BF16) launch_typed<bf16_t>(a, ws, nsplit, tps, st);
    else launch_typed<float>(a, ws, nsplit, tps, st);
    if (hipGetLastError() != hipSuccess) return STRD_EHIP;
    return dec_combine(a, ws, nsplit, st);
}

}  // namespace strd
