// One token's attention over a cache, plain or in 4 bits, with capped scores, a bias by distance and the attention weight that
// every row has gathered (the cap, the bias and the weights: strd.h).  Any head size up to 256, any number of heads, fp32
// arithmetic; the shapes of attn_decode_cache_mfma.hip run there.
//
// Pass 1: a workgroup takes one kv head's share of the tokens, and up to 4 of its query heads (more: the cache is read again).  16 lanes hold a token's
// row, 8 neighbouring channels each (two such pieces above 128 channels), and 4 tokens are on their way together; a lane
// group has a softmax of its own, and the 16 of a workgroup meet in LDS.  Where weights are wanted the scores go to the workspace.
// Pass 2: a workgroup per 32 output channels of a head joins the splits; others turn the scores of 256 or 512 tokens into weights,
// once the heads' references and sums over all splits are known: w = w_in + mean over the heads of 2^(score - ref) / sum.
// Pass 2 is a launch and two round trips to memory, 3.8 us up to some ten thousand tokens, 8.5 at 131627 (17 MB of scores).
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
                                                                int d, int tps, int nsplit, ScoreMod mod) {
    extern __shared__ float sm_acc[];  // [kGroups][d]
    __shared__ float sm_m[kGroups][RP], sm_l[kGroups][RP];
    int hk, split;
    dec_place(blockIdx.x, Hkv, hk, split);
    if (split >= nsplit) return;  // uniform
    const int rep = Hq / Hkv, r0 = blockIdx.y * RP;
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
                x[u][r] = (capped_score(group_sum(dot), mod.scale, mod.cap, mod.inv_cap) - slope[r] * far[u]) * kLog2e;
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

// References and reciprocal sums of 32 heads from h0 on over all splits, 8 lanes a head, by a workgroup: everything is asked
// for before the first maximum, and what `ask` reads behind that (loads return in order).  hm, hl hold them behind the barrier at the end.
constexpr int kHeadsAtOnce = kThreads / 8, kSplitLoads = 16;
template <class ASK>
__device__ __forceinline__ void head_totals(const float *__restrict__ ml, int nsplit, int Hq, int h0, float *hm, float *hl, ASK &&ask) {
    const int h = min(h0 + (int)threadIdx.x / 8, Hq - 1), sub = threadIdx.x % 8;
    const float2 *pairs = reinterpret_cast<const float2 *>(ml) + h;
    float mx = kDecNegBig, den = 0.f;
    for (int s0 = 0; s0 < nsplit; s0 += 8 * kSplitLoads) {  // (one round up to 128 splits)
        float2 pr[kSplitLoads];
#pragma unroll
        for (int i = 0; i < kSplitLoads; ++i) pr[i] = pairs[(size_t)min(s0 + sub + 8 * i, nsplit - 1) * Hq];
        if (s0 == 0) ask();
        float nm = mx;
#pragma unroll
        for (int i = 0; i < kSplitLoads; ++i) nm = fmaxf(nm, pr[i].x);
        den *= ex2(mx - nm);
#pragma unroll
        for (int i = 0; i < kSplitLoads; ++i)
            den = fmaf(s0 + sub + 8 * i < nsplit ? ex2(pr[i].x - nm) : 0.f, pr[i].y, den);
        mx = nm;
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
        const float om = __shfl_xor(mx, o, kWave), od = __shfl_xor(den, o, kWave), nm = fmaxf(mx, om);
        den = den * ex2(mx - nm) + od * ex2(om - nm);
        mx = nm;
    }
    if (sub == 0) {
        hm[threadIdx.x / 8] = mx;
        hl[threadIdx.x / 8] = 1.f / den;
    }
    __syncthreads();
}

// One workgroup per 32 channels of a head (8 lane groups share the splits), then one per NT * 256 tokens' weights.
constexpr int kPartLoads = 16;
static_assert(kThreads == 4 * kWave, "four tokens a lane of a wave, then one a lane of all");

template <typename T, int NT>
__global__ __launch_bounds__(kThreads) void decode_combine_kernel(DecWs ws, T *__restrict__ o, const float *__restrict__ w_in,
                                                                  float *__restrict__ w_out, int nsplit, int Tn, int Hq, int d,
                                                                  int o_blocks) {
    __shared__ float sums[8][33], dens[8], maxs[8], hm[kHeadsAtOnce], hl[kHeadsAtOnce];
    __shared__ __attribute__((aligned(16))) float shares[NT][kThreads / kWave][kThreads];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < o_blocks) {
        const int per = (d + 31) / 32, h = blockIdx.x / per, c = (blockIdx.x % per) * 32 + tid % 32, sg = tid / 32;
        const float2 *pairs = reinterpret_cast<const float2 *>(ws.ml) + h;
        const float *part = ws.part + (size_t)h * d + min(c, d - 1);
        float mx = kDecNegBig, den = 0.f, acc = 0.f;  // of this lane group's splits; everything is asked for before the first sum
        for (int s0 = sg; s0 < nsplit; s0 += 8 * kPartLoads) {
            float2 pr[kPartLoads];
            float v[kPartLoads];
#pragma unroll
            for (int i = 0; i < kPartLoads; ++i) {
                const size_t at = (size_t)min(s0 + 8 * i, nsplit - 1) * Hq;
                pr[i] = pairs[at];
                v[i] = part[at * d];
            }
            float nm = mx;
#pragma unroll
            for (int i = 0; i < kPartLoads; ++i) nm = fmaxf(nm, pr[i].x);
            const float corr = ex2(mx - nm);
            den *= corr;
            acc *= corr;
#pragma unroll
            for (int i = 0; i < kPartLoads; ++i) {
                const float f = s0 + 8 * i < nsplit ? ex2(pr[i].x - nm) : 0.f;
                den = fmaf(f, pr[i].y, den);
                acc = fmaf(f, s0 + 8 * i < nsplit ? v[i] : 0.f, acc);
            }
            mx = nm;
        }
        sums[sg][tid % 32] = acc;
        if (tid % 32 == 0) {
            dens[sg] = den;
            maxs[sg] = mx;
        }
        __syncthreads();
        if (tid < 32 && c < d) {
            float top = maxs[0], num = 0.f, all = 0.f;
#pragma unroll
            for (int g = 1; g < 8; ++g) top = fmaxf(top, maxs[g]);
#pragma unroll
            for (int g = 0; g < 8; ++g) {  // fixed order
                const float f = ex2(maxs[g] - top);
                num = fmaf(f, sums[g][tid], num);
                all = fmaf(f, dens[g], all);
            }
            o[(size_t)h * d + c] = from_f32<T>(num / all);
        }
        return;
    }
    // a wave has a quarter of the heads at once and 4 tokens a lane; the scores are asked for before the totals are known
    const int lane = tid % kWave, wave = tid / kWave;
    const long long tb = (long long)(blockIdx.x - o_blocks) * (NT * kThreads);
    float before[NT];
    float4 acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = make_float4(0.f, 0.f, 0.f, 0.f), before[n] = 0.f;
    for (int h0 = 0; h0 < Hq; h0 += kHeadsAtOnce) {
        constexpr int kOwn = kHeadsAtOnce / (kThreads / kWave);
        float4 x[NT][kOwn];
        if (h0) __syncthreads();
        head_totals(ws.ml, nsplit, Hq, h0, hm, hl, [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const long long ts = min(tb + n * kThreads + 4 * lane, ws.ldt - 4);  // (rows of scores are padded to 64)
#pragma unroll
                for (int i = 0; i < kOwn; ++i)
                    x[n][i] = *reinterpret_cast<const float4 *>(ws.scores + (size_t)min(h0 + kOwn * wave + i, Hq - 1) * ws.ldt + ts);
                if (h0 == 0 && w_in && tb + n * kThreads + tid < Tn) before[n] = w_in[tb + n * kThreads + tid];
            }
        });
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            if (h0 + kOwn * wave + i >= Hq) break;  // uniform
            const float m = hm[kOwn * wave + i], l = hl[kOwn * wave + i];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                acc[n].x = fmaf(ex2(x[n][i].x - m), l, acc[n].x);
                acc[n].y = fmaf(ex2(x[n][i].y - m), l, acc[n].y);
                acc[n].z = fmaf(ex2(x[n][i].z - m), l, acc[n].z);
                acc[n].w = fmaf(ex2(x[n][i].w - m), l, acc[n].w);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) *reinterpret_cast<float4 *>(&shares[n][wave][4 * lane]) = acc[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const long long t = tb + n * kThreads + tid;
        if (t < Tn) {
            float sum = shares[n][0][tid];
#pragma unroll
            for (int w = 1; w < kThreads / kWave; ++w) sum += shares[n][w][tid];
            w_out[t] = before[n] + sum / (float)Hq;
        }
    }
}

template <typename T, bool KV4, bool VEC, int RP>
void launch_rp(const DecCall &a, const DecWs &ws, int nsplit, int tps, hipStream_t st) {
    const dim3 grid(dec_grid(a.Hkv, nsplit), ceil_div(a.Hq / a.Hkv, RP));
    const size_t smem = (size_t)kGroups * a.d * sizeof(float);
    if (a.d <= 128)
        decode_cache_kernel<T, KV4, VEC, RP, 1><<<grid, kThreads, smem, st>>>((const T *)a.q, a.c, ws, a.T, a.Hq, a.Hkv, a.d, tps, nsplit, a.mod);
    else
        decode_cache_kernel<T, KV4, VEC, RP, 2><<<grid, kThreads, smem, st>>>((const T *)a.q, a.c, ws, a.T, a.Hq, a.Hkv, a.d, tps, nsplit, a.mod);
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

template <typename T, int NT>
static void launch_combine(const DecCall &a, const DecWs &ws, int nsplit, hipStream_t st) {
    const int o_blocks = a.Hq * ceil_div(a.d, 32), w_blocks = a.w_out ? (int)(((long long)a.T + NT * kThreads - 1) / (NT * kThreads)) : 0;
    decode_combine_kernel<T, NT><<<o_blocks + w_blocks, kThreads, 0, st>>>(ws, (T *)a.o, a.w_in, a.w_out, nsplit, a.T, a.Hq, a.d, o_blocks);
}
// 256 tokens a workgroup; 512 where that is more than one for every CU, each of which reads all totals (32 heads: 8491 tokens 4.0 / 4.8 us,
// 131627 9.8 / 8.5).
int dec_combine(const DecCall &a, const DecWs &ws, int nsplit, hipStream_t st) {
    const bool two = a.w_out && a.T > 256 * kThreads;
    if (a.io == STRD_BF16) two ? launch_combine<bf16_t, 2>(a, ws, nsplit, st) : launch_combine<bf16_t, 1>(a, ws, nsplit, st);
    else two ? launch_combine<float, 2>(a, ws, nsplit, st) : launch_combine<float, 1>(a, ws, nsplit, st);
    return launch_status();
}

size_t attn_decode_cache_ws(int T, int Hq, int Hkv, int d, bool kv4, bool weights, strd_dtype io) {
    // (a query or a plain cache that 16-byte reads do not fit takes the general kernel whatever its shape: room for either's splits)
    int tps, n = dec_splits_general(T, Hq, Hkv, tps);
    if (dec_mfma_supported(T, Hq, Hkv, d, kv4, io)) n = max(n, dec_mfma_splits(T, Hkv, d, kv4, tps));
    return dec_ws_bytes(n, Hq, d, dec_ldt(T), weights);
}

int attn_decode_cache(const DecCall &a, void *wsp, hipStream_t st) {
    const bool mfma = dec_mfma_supported(a.T, a.Hq, a.Hkv, a.d, a.kv4, a.io) && (((uintptr_t)a.q | (uintptr_t)a.c.k | (uintptr_t)a.c.v) & 15) == 0;
    DecWs ws;
    int tps;
    const int nsplit = mfma ? dec_mfma_splits(a.T, a.Hkv, a.d, a.kv4, tps) : dec_splits_general(a.T, a.Hq, a.Hkv, tps);
    ws.ml = (float *)wsp;  // (pairs: they come first)
    ws.part = ws.ml + (size_t)nsplit * a.Hq * 2;
    ws.ldt = dec_ldt(a.T);
    ws.scores = a.w_out ? (float *)((char *)wsp + align_up((size_t)nsplit * a.Hq * (a.d + 2) * sizeof(float), 256)) : nullptr;
    if (mfma) {
        const int rc = dec_mfma(a, ws, nsplit, tps, st);
        if (rc != STRD_OK) return rc;
    } else if (a.io == STRD_BF16) launch_typed<bf16_t>(a, ws, nsplit, tps, st);
    else launch_typed<float>(a, ws, nsplit, tps, st);
    if (hipGetLastError() != hipSuccess) return STRD_EHIP;
    return dec_combine(a, ws, nsplit, st);
}

}  // namespace strd
