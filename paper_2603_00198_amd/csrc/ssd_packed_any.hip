// ssd_prefill_varlen in fp32 products: the Mamba-2 recurrence (paper Eqs. "ssm_state_update", "ssm_output") over a packed batch, for the shapes and types
// that ssd_packed_mfma.hip does not take, and for small batches.  Sequences are cut into chunks of 64 tokens, all of them side by side:
//     (1) E_c = sum_{j in c} (dt_j 2^(l_end - l_j) x_j) b_j^T                       what a chunk leaves in the state behind it
//     (2) S_c = the state before chunk c;  S_{c+1} = 2^(l_end) S_c + E_c            runs of chunks at a time, then the runs where there are several
//     (3) y_t = 2^(l_t) S_c c_t + sum_{j <= t in c} 2^(l_t - l_j) dt_j (c_t . b_j) x_j + D x_t
// with l the sums of dt A log2 e from the chunk's start.  Products are v_mfma_f32_16x16x4_f32; l is added up in 64 bits and kept as two fp32 numbers, so
// that differences of far sums are good to 32 bits.  (1) and (3) are bound by their reads and products, (2) by HBM or, where states are small, by the
// latency of a run: 4160 fp32 tokens of 128 heads of 64 x 128 140 + 100 (5.5 TB/s) + 255 us, 33280 of 8 heads of 64 x 64 35 + 31 + 71.  Side by side, not one
// sequence after the other on the vector units (general.hip): those 694 -> 465 and 270 -> 139 us, three clips of 86 tokens together 18.6 -> 13.4; one sequence
// of 4160 tokens of 8 small heads takes the same 23 either way.
#include <algorithm>

#include "carry.h"

namespace strd {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float read_lane_f32(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

constexpr int kQ = 64, kThreads = 256, kSlab = 64;  // tokens of a chunk; channels of a workgroup
constexpr int kXPitch = kSlab + 4;
constexpr size_t kMostStates = (size_t)8 << 30;     // bytes of states between the kernels

struct AnyArgs {
    CarryTab tab;  // tiles: chunks
    const void *x, *B, *C;
    const float *dt, *A, *D, *S_in;
    float *S_out;
    void *y;
    float *states;  // [chunks, H, P, n]: E, then the states before chunks (of a run other than a sequence's first: without what came before the run)
    float *runs;    // [runs, H, P, n]: what a run leaves, then the states before runs
    float *total;   // [chunks, H]: log2 decay over a chunk
    float *lead;    // [chunks, H]: from its run's start to a chunk
    float *run_total;  // [runs, H]
    int H, P, G, n, run, slabs;  // run: chunks of one
    int run0[kMaxSeqs + 1];      // runs before a sequence's
    __device__ __forceinline__ bool history(int s) const { return S_in && !(tab.fresh >> s & 1); }
};

// One workgroup's chunk, head and slab of channels; heads of a chunk are neighbours.
struct Unit {
    int chunk, h, g, s, slab, row0, rows, first;  // first: of the sequence
    template <typename A>
    __device__ __forceinline__ bool find(const A &a, int nunits) {
        const int u = xcd_swizzle(blockIdx.x, nunits);
        if (u >= nunits) return false;
        slab = u % a.slabs;
        h = u / a.slabs % a.H;
        chunk = u / a.slabs / a.H;
        g = h / (a.H / a.G);
        s = a.tab.find(chunk);
        first = a.tab.base[s];
        row0 = a.tab.row0[s] + (chunk - first) * kQ;
        rows = min(kQ, a.tab.row0[s] + a.tab.len[s] - row0);
        return true;
    }
};

// Sums of a chunk's decays, in lane t those up to token t: l = hi + lo; rows past the end have dt = 0.
struct Decays {
    float dt, A;
    template <int CTRL, int ROWS>
    __device__ static __forceinline__ double from_lane(double v) {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xF, true);
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xF, true);
        return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    }
    __device__ __forceinline__ Decays(const AnyArgs &a, const Unit &u)
        : dt(a.dt[(size_t)(u.row0 + min((int)threadIdx.x & 63, u.rows - 1)) * a.H + u.h]), A(a.A[u.h]) {}
    __device__ __forceinline__ void sums(const Unit &u, float &mine, float &hi, float &lo) const {
        const int lane = threadIdx.x & 63;
        mine = lane < u.rows ? dt : 0.f;
        double l = (double)mine * ((double)A * 1.4426950408889634);
        l += from_lane<0x111, 0xF>(l);  // row_shr:1
        l += from_lane<0x112, 0xF>(l);  // row_shr:2
        l += from_lane<0x114, 0xF>(l);  // row_shr:4
        l += from_lane<0x118, 0xF>(l);  // row_shr:8
        l += from_lane<0x142, 0xA>(l);  // row_bcast:15 into rows 1 and 3
        l += from_lane<0x143, 0xC>(l);  // row_bcast:31 into rows 2 and 3
        hi = (float)l;
        lo = hi - hi == 0.f ? (float)(l - (double)hi) : 0.f;
    }
};

// Rows of a matrix on their way to LDS: W columns (a multiple of 16), four to a thread.  WHOLE: rows are read four numbers at a time, all of them at once;
// those past the end are read from its last ones and left out later.
template <typename T, int W, bool WHOLE>
struct Rows {
    typedef T V4 __attribute__((ext_vector_type(4)));
    static constexpr int kPer = kQ * W / 4 / kThreads;
    V4 v[kPer];
    __device__ static __forceinline__ int row(int i) { return (i * kThreads + (int)threadIdx.x) / (W / 4); }
    __device__ static __forceinline__ int col(int i) { return (i * kThreads + (int)threadIdx.x) % (W / 4) * 4; }
    __device__ __forceinline__ void load(const T *p, size_t pitch, int rows, int width) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const T *const from = p + min(row(i), rows - 1) * pitch;
            if constexpr (WHOLE) {
                v[i] = *reinterpret_cast<const V4 *>(from + min(col(i), width - 4));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i][e] = from[min(col(i) + e, width - 1)];
            }
        }
    }
    __device__ __forceinline__ f32x4 get(int i, int rows, int width) const {
        f32x4 f;
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = row(i) < rows && col(i) + e < width ? to_f32((T)v[i][e]) : 0.f;
        return f;
    }
    __device__ __forceinline__ void store(float *lds, int pitch, int rows, int width) const {
#pragma unroll
        for (int i = 0; i < kPer; ++i) *reinterpret_cast<f32x4 *>(lds + row(i) * pitch + col(i)) = get(i, rows, width);
    }
};

__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// ---- (1): a wave has 16 channels, the columns of S^T; rows are the state's columns; a k slot is a token ----------------------------------------------
template <typename T, int NT, bool WHOLE>
__global__ __launch_bounds__(kThreads) void ssd_any_states_kernel(AnyArgs a, int nunits) {
    constexpr int kPitch = 16 * NT + 4;
    extern __shared__ __attribute__((aligned(16))) float sm[];
    float *const bs = sm, *const xs = bs + kQ * kPitch, *const ws = xs + kQ * kXPitch;
    Unit u;
    if (!u.find(a, nunits)) return;
    const int lane = threadIdx.x & 63, lr = lane & 15, lb = lane >> 4, wave = threadIdx.x >> 6;
    const int p0 = u.slab * kSlab, width = min(kSlab, a.P - p0);
    Rows<T, 16 * NT, WHOLE> b;
    Rows<T, kSlab, WHOLE> x;
    float dt, hi, lo;
    Decays d(a, u);
    x.load((const T *)a.x + ((size_t)u.row0 * a.H + u.h) * a.P + p0, (size_t)a.H * a.P, u.rows, width);
    b.load((const T *)a.B + ((size_t)u.row0 * a.G + u.g) * a.n, (size_t)a.G * a.n, u.rows, a.n);
    d.sums(u, dt, hi, lo);
    const float end_hi = read_lane_f32(hi, 63), end_lo = read_lane_f32(lo, 63);
    if (wave == 0) {
        ws[lane] = dt == 0.f ? 0.f : dt * fast_exp2((end_hi - hi) + (end_lo - lo));
        if (lane == 0 && u.slab == 0) a.total[(size_t)u.chunk * a.H + u.h] = end_hi;
    }
    b.store(bs, kPitch, u.rows, a.n);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < x.kPer; ++i) *reinterpret_cast<f32x4 *>(xs + x.row(i) * kXPitch + x.col(i)) = x.get(i, u.rows, width) * ws[x.row(i)];
    __syncthreads();
    if (16 * wave >= width) return;
    f32x4 acc[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int j0 = 4 * lb; j0 < 4 * lb + u.rows; j0 += 16) {  // (whole tiles of 16 tokens)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float xv = xs[(j0 + e) * kXPitch + 16 * wave + lr];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[nt] = mfma4(bs[(j0 + e) * kPitch + 16 * nt + lr], xv, acc[nt]);
        }
    }
    const int p = p0 + 16 * wave + lr;
    if (p >= a.P) return;
    float *const out = a.states + (((size_t)u.chunk * a.H + u.h) * a.P + p) * a.n;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int c = 16 * nt + 4 * lb;
        if (a.n % 4 == 0) {  // uniform
            if (c < a.n) *reinterpret_cast<f32x4 *>(out + c) = acc[nt];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < a.n) out[c + e] = acc[nt][e];
        }
    }
}

// ---- (2): a thread has VW entries of a state, over the chunks of a run --------------------------------------------------------------------------------
template <int VW>
__global__ __launch_bounds__(kThreads) void ssd_any_runs_kernel(AnyArgs a) {
    typedef float F __attribute__((ext_vector_type(VW)));
    const size_t state = (size_t)a.H * a.P * a.n, at = ((size_t)blockIdx.x * kThreads + threadIdx.x) * VW;
    if (at >= state) return;
    int s = 0;
    while (s + 1 < a.tab.nseq && (int)blockIdx.y >= a.run0[s + 1]) ++s;  // uniform
    const int r = blockIdx.y - a.run0[s], nrun = a.run0[s + 1] - a.run0[s], c0 = a.tab.base[s] + r * a.run, c1 = min(c0 + a.run, a.tab.base[s + 1]);
    const int h = (int)(at / ((size_t)a.P * a.n));
    const bool from = r == 0 && a.history(s), teller = at % ((size_t)a.P * a.n) == 0;
    const bool wants_end = nrun > 1 || a.S_out;
    F run = {};
    if (from) run = *reinterpret_cast<const F *>(a.S_in + (size_t)a.tab.slot[s] * state + at);
    float lead = 0.f;
    constexpr int kAhead = 8;
    for (int c = c0; c < c1; c += kAhead) {
        F e[kAhead];
        float t[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int ci = min(c + i, c1 - 1);
            e[i] = *reinterpret_cast<const F *>(a.states + (size_t)ci * state + at);
            t[i] = a.total[(size_t)ci * a.H + h];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (c + i < c1) {
                *reinterpret_cast<F *>(a.states + (size_t)(c + i) * state + at) = run;
                if (teller) a.lead[(size_t)(c + i) * a.H + h] = lead;
                run = run * fast_exp2(t[i]) + e[i];
                lead += t[i];
            }
    }
    if (nrun > 1) {
        *reinterpret_cast<F *>(a.runs + (size_t)blockIdx.y * state + at) = run;
        if (teller) a.run_total[(size_t)blockIdx.y * a.H + h] = lead;
    } else if (wants_end) {
        *reinterpret_cast<F *>(a.S_out + (size_t)a.tab.slot[s] * state + at) = run;
    }
}

// The states before a sequence's runs.
template <int VW>
__global__ __launch_bounds__(kThreads) void ssd_any_join_kernel(AnyArgs a) {
    typedef float F __attribute__((ext_vector_type(VW)));
    const int s = blockIdx.y, r0 = a.run0[s], r1 = a.run0[s + 1];
    const size_t state = (size_t)a.H * a.P * a.n, at = ((size_t)blockIdx.x * kThreads + threadIdx.x) * VW;
    if (at >= state || r1 - r0 < 2) return;
    const int h = (int)(at / ((size_t)a.P * a.n));
    F run = *reinterpret_cast<const F *>(a.runs + (size_t)r0 * state + at);  // (the first run's end has what it set out from in it)
    constexpr int kAhead = 8;
    for (int r = r0 + 1; r < r1; r += kAhead) {
        F e[kAhead];
        float t[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int ri = min(r + i, r1 - 1);
            e[i] = *reinterpret_cast<const F *>(a.runs + (size_t)ri * state + at);
            t[i] = a.run_total[(size_t)ri * a.H + h];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (r + i < r1) {
                *reinterpret_cast<F *>(a.runs + (size_t)(r + i) * state + at) = run;
                run = run * fast_exp2(t[i]) + e[i];
            }
    }
    if (a.S_out) *reinterpret_cast<F *>(a.S_out + (size_t)a.tab.slot[s] * state + at) = run;
}

// ---- (3): a wave has 16 tokens, the columns of Y^T and of the products c . b; rows are channels (16 PT of them) and earlier tokens -------------------------
template <typename T, int NT, int PT, bool WHOLE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(WHOLE ? 3 : 2))) void ssd_any_out_kernel(AnyArgs a, int nunits) {
    constexpr int kPitch = 16 * NT + 4, kXP = 16 * PT + 4;
    typedef T V4 __attribute__((ext_vector_type(4)));
    extern __shared__ __attribute__((aligned(16))) float sm[];
    float *const tile = sm, *const xs = tile + kQ * kPitch, *const his = xs + kQ * kXP, *const los = his + kQ, *const dts = los + kQ;
    Unit u;
    if (!u.find(a, nunits)) return;
    const int lane = threadIdx.x & 63, lr = lane & 15, lb = lane >> 4, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    // A wave's work grows with its tokens' place in the chunk, and wave w of every workgroup is on one of the CU's four SIMDs: every other head the other way.
    const int wave = u.h & 1 ? kThreads / 64 - 1 - w : w;
    const int p0 = u.slab * kSlab, width = min(16 * PT, a.P - p0), t = 16 * wave + lr;
    const int run = (u.chunk - u.first) / a.run;              // of the sequence
    const bool before = u.chunk > u.first || a.history(u.s);  // uniform: there is a state
    Rows<T, 16 * NT, WHOLE> b;
    Rows<T, 16 * PT, WHOLE> x;
    Rows<float, 16 * NT, WHOLE> st;
    V4 craw[NT];
    const size_t head = (size_t)u.h * a.P + p0, state = (size_t)a.H * a.P * a.n;
    const Decays d(a, u);
    const float skip = a.D ? a.D[u.h] : 0.f;
    if (before) st.load(a.states + u.chunk * state + head * a.n, a.n, width, a.n);
    x.load((const T *)a.x + (size_t)u.row0 * a.H * a.P + head, (size_t)a.H * a.P, u.rows, width);
    const T *const cp = (const T *)a.C + ((size_t)(u.row0 + min(t, u.rows - 1)) * a.G + u.g) * a.n;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int col = 16 * j + 4 * lb;
        if constexpr (WHOLE) {
            craw[j] = *reinterpret_cast<const V4 *>(cp + min(col, a.n - 4));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) craw[j][e] = cp[min(col + e, a.n - 1)];
        }
    }
    b.load((const T *)a.B + ((size_t)u.row0 * a.G + u.g) * a.n, (size_t)a.G * a.n, u.rows, a.n);
    float dt, hi, lo;
    d.sums(u, dt, hi, lo);
    if (w == 0) his[lane] = hi, los[lane] = lo, dts[lane] = dt;
    if (before) {
        if (run) {  // uniform: and what came before the run
            Rows<float, 16 * NT, WHOLE> rs;
            rs.load(a.runs + (size_t)(a.run0[u.s] + run) * state + head * a.n, a.n, width, a.n);
            const float f = fast_exp2(a.lead[(size_t)u.chunk * a.H + u.h]);
#pragma unroll
            for (int i = 0; i < st.kPer; ++i) st.v[i] += f * rs.v[i];
        }
        st.store(tile, kPitch, width, a.n);
    }
    x.store(xs, kXP, u.rows, width);
    f32x4 c[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[j][e] = 16 * j + 4 * lb + e < a.n ? to_f32((T)craw[j][e]) : 0.f;
    __syncthreads();
    const float hi_t = his[t], lo_t = los[t];
    // acc[pt][e]: channel 16 pt + 4 lb + e, token t
    f32x4 acc[PT];
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) acc[pt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bool live = 16 * wave < u.rows;
    if (before) {
        if (live) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                f32x4 s4[PT];
#pragma unroll
                for (int pt = 0; pt < PT; ++pt) s4[pt] = *reinterpret_cast<const f32x4 *>(&tile[(16 * pt + lr) * kPitch + 16 * j + 4 * lb]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int pt = 0; pt < PT; ++pt) acc[pt] = mfma4(s4[pt][e], c[j][e], acc[pt]);
            }
            const float decay = fast_exp2(hi_t + lo_t);
#pragma unroll
            for (int pt = 0; pt < PT; ++pt) acc[pt] *= decay;
        }
        __syncthreads();
    }
    b.store(tile, kPitch, u.rows, a.n);
    __syncthreads();
    if (!live) return;
    for (int jt = 0; jt <= wave; ++jt) {
        const int j0 = 16 * jt + 4 * lb;
        const f32x4 hj = *reinterpret_cast<const f32x4 *>(&his[j0]), lj = *reinterpret_cast<const f32x4 *>(&los[j0]), dj = *reinterpret_cast<const f32x4 *>(&dts[j0]);
        f32x4 g[2] = {};
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const f32x4 b4 = *reinterpret_cast<const f32x4 *>(&tile[(16 * jt + lr) * kPitch + 16 * j + 4 * lb]);
#pragma unroll
            for (int e = 0; e < 4; ++e) g[e & 1] = mfma4(b4[e], c[j][e], g[e & 1]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float m = j0 + e <= t ? (g[0][e] + g[1][e]) * dj[e] * fast_exp2((hi_t - hj[e]) + (lo_t - lj[e])) : 0.f;
#pragma unroll
            for (int pt = 0; pt < PT; ++pt) acc[pt] = mfma4(xs[(j0 + e) * kXP + 16 * pt + lr], m, acc[pt]);
        }
    }
    if (t >= u.rows) return;
    T *const out = (T *)a.y + (size_t)(u.row0 + t) * a.H * a.P + head;
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) {
        const int p = 16 * pt + 4 * lb;
        if (p >= width) continue;
        if (a.D) {
            const f32x4 xv = *reinterpret_cast<const f32x4 *>(&xs[t * kXP + p]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[pt][e] = fmaf(skip, xv[e], acc[pt][e]);
        }
        if constexpr (WHOLE) {
            V4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = from_f32<T>(acc[pt][e]);
            *reinterpret_cast<V4 *>(out + p) = o;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (p + e < width) out[p + e] = from_f32<T>(acc[pt][e]);
        }
    }
}

struct AnyPlan {
    CarryTab tab;
    int run, runs, run0[kMaxSeqs + 1];
    size_t state, states, run_states, totals, run_totals;  // bytes
    size_t bytes() const { return states + run_states + 2 * totals + run_totals; }
};

// Runs are as long as leaves a thousand workgroups of 1024 entries, and 32 chunks at least, which take as long as the launch that joins runs; states that
// give as many workgroups by themselves have one run to a sequence.
AnyPlan plan_any(const CarryTab &t, int H, int P, int n) {
    AnyPlan p;
    p.tab = t;
    int chunks = 0;
    for (int s = 0; s < t.nseq; ++s) {
        p.tab.base[s] = chunks;
        chunks += ceil_div(t.len[s], kQ);
    }
    p.tab.base[t.nseq] = chunks;
    const long long entries = (long long)H * P * n;
    p.run = (int)std::max<long long>(32, std::min<long long>(chunks, (chunks * ((entries + 1023) / 1024) + 1023) / 1024));
    p.runs = 0;
    int several = 0;
    for (int s = 0; s < t.nseq; ++s) {
        p.run0[s] = p.runs;
        const int k = ceil_div(ceil_div(t.len[s], kQ), p.run);
        p.runs += k;
        if (k > 1) several = 1;
    }
    p.run0[t.nseq] = p.runs;
    p.state = entries * sizeof(float);
    p.states = align_up(chunks * p.state, 256);
    p.run_states = several ? align_up(p.runs * p.state, 256) : 0;
    p.totals = align_up((size_t)chunks * H * sizeof(float), 256);
    p.run_totals = several ? align_up((size_t)p.runs * H * sizeof(float), 256) : 0;
    return p;
}

template <typename T, int NT, bool WHOLE>
int launch(const AnyArgs &a, const AnyPlan &p, bool vec, hipStream_t st) {
    const int nunits = p.tab.base[p.tab.nseq] * a.H * a.slabs;
    const size_t state = p.state / sizeof(float), lds = ((size_t)kQ * (16 * NT + 4) + kQ * kXPitch) * sizeof(float);
    if (!allow_dynamic_lds((const void *)&ssd_any_states_kernel<T, NT, WHOLE>, lds + kQ * 4)) return STRD_EHIP;
    bool several_chunks = false;
    for (int s = 0; s < p.tab.nseq; ++s) several_chunks |= p.tab.len[s] > kQ;
    if (several_chunks || a.S_in || a.S_out) {
        ssd_any_states_kernel<T, NT, WHOLE><<<xcd_grid(nunits), kThreads, lds + kQ * 4, st>>>(a, nunits);
        const int per = vec ? 4 : 1;
        const dim3 grid((unsigned)((state + kThreads * per - 1) / (kThreads * per)), p.runs), join(grid.x, p.tab.nseq);
        if (vec) ssd_any_runs_kernel<4><<<grid, kThreads, 0, st>>>(a);
        else ssd_any_runs_kernel<1><<<grid, kThreads, 0, st>>>(a);
        if (p.run_states) {
            if (vec) ssd_any_join_kernel<4><<<join, kThreads, 0, st>>>(a);
            else ssd_any_join_kernel<1><<<join, kThreads, 0, st>>>(a);
        }
    }
    auto out = [&](auto *kernel) {
        if (!allow_dynamic_lds((const void *)kernel, lds + 3 * kQ * 4)) return (int)STRD_EHIP;
        kernel<<<xcd_grid(nunits), kThreads, lds + 3 * kQ * 4, st>>>(a, nunits);
        return launch_status();
    };
    if constexpr (WHOLE)
        if (a.P <= 32) return out(&ssd_any_out_kernel<T, NT, 2, WHOLE>);
    return out(&ssd_any_out_kernel<T, NT, kSlab / 16, WHOLE>);
}

}  // namespace

// Batches of the bf16 matrix cores' shapes that are too small for the five launches and serial steps there (us, there / here; rows, heads, columns of a
// state): 57 in three sequences, 128, 128 44 / 41, 64, 64 28 / 19; 200, 128, 128 54 / 47; 490, 128, 128 65 / 68; 1000, 128, 128 73 / 115, 64, 64 54 / 47, 16,
// 128 58 / 34.
bool ssd_any_wanted(const CarryTab &t, int H, int n) {
    double chunks = 0;
    for (int s = 0; s < t.nseq; ++s) chunks += ceil_div(t.len[s], kQ);
    return chunks * kQ * H * n <= 5 << 20;
}

// States of up to 128 columns, as long as what lies between the kernels takes no more than 8 GB.
bool ssd_any_supported(const CarryTab &t, int H, int P, int n) {
    long long chunks = 0;
    for (int s = 0; s < t.nseq; ++s) chunks += ceil_div(t.len[s], kQ);
    return n <= 128 && chunks / 32 + t.nseq <= 65535 && (double)chunks * H * P * n * 4 <= (double)kMostStates && chunks * H * ceil_div(P, kSlab) <= (1 << 24) - kXcd;
}

size_t ssd_any_ws(const CarryTab &t, int H, int P, int n) { return plan_any(t, H, P, n).bytes(); }

int ssd_any(const void *x, const float *dt, const float *A, const void *B, const void *C, const float *D, const float *S_in, float *S_out, const CarryTab &t,
            void *y, int H, int P, int G, int n, strd_dtype io, void *ws, hipStream_t st) {
    const AnyPlan p = plan_any(t, H, P, n);
    AnyArgs a = {};
    a.tab = p.tab;
    a.x = x, a.B = B, a.C = C, a.dt = dt, a.A = A, a.D = D, a.S_in = S_in, a.S_out = S_out, a.y = y;
    char *w = (char *)ws;
    a.states = (float *)w, w += p.states;
    a.runs = (float *)w, w += p.run_states;
    a.total = (float *)w, w += p.totals;
    a.lead = (float *)w, w += p.totals;
    a.run_total = (float *)w;
    a.H = H, a.P = P, a.G = G, a.n = n, a.run = p.run, a.slabs = ceil_div(P, kSlab);
    for (int s = 0; s <= t.nseq; ++s) a.run0[s] = p.run0[s];
    const size_t es = io == STRD_F32 ? 4 : 2;
    const bool whole = P % 4 == 0 && n % 4 == 0 && (((uintptr_t)x | (uintptr_t)B | (uintptr_t)C | (uintptr_t)y) & (4 * es - 1)) == 0;
    const bool vec = (long long)P * n % 4 == 0 && (((uintptr_t)S_in | (uintptr_t)S_out) & 15) == 0;
    if (S_out) {
        const int rc = copy_empty_slots(t, S_in, S_out, (size_t)H * P * n, st);
        if (rc != STRD_OK) return rc;
    }
    if (p.tab.base[t.nseq] == 0) return launch_status();
    auto by_n = [&](auto *tag) {
        using T = std::remove_pointer_t<decltype(tag)>;
        return !whole    ? launch<T, 8, false>(a, p, vec, st)
               : n <= 16 ? launch<T, 1, true>(a, p, vec, st)
               : n <= 32 ? launch<T, 2, true>(a, p, vec, st)
               : n <= 64 ? launch<T, 4, true>(a, p, vec, st)
                         : launch<T, 8, true>(a, p, vec, st);
    };
    return io == STRD_F32 ? by_n((float *)nullptr) : by_n((bf16_t *)nullptr);
}

}  // namespace strd
