// The short causal convolution of a Mamba-2 layer with SiLU where sequences come in parts: over a packed batch, each sequence going on
// from its window, the W - 1 input rows that its last part ended with; and one token each of many sequences.
//     o[t, c] = silu(b[c] + sum_{k < W} w[c, k] u[t - (W - 1) + k, c]),   u[t < 0] = window row W - 1 + t (zeros for a sequence that begins)
//     window' = the last W - 1 rows of (window, u)
// Bound by HBM: an element is read and written once for 2 W + 6 operations.  fp32 arithmetic, one rounding.  Instantiated per W:
// a tap that is not there multiplies nothing, so what is not finite reaches W rows and no more.  33280 rows of 10240 channels: 252 us, 5.4 TB/s (its
// vector instructions take half the time beside that); one token of 48 sequences 4.0 us in the kernel, a launch and two trips to memory.
#include "carry.h"

namespace strd {
namespace {

constexpr int kThreads = 256;
// Tokens per thread, which also reads the W - 1 rows before them (33280 rows of 10240 channels: 4 tokens 301 us, 8 259, 16 257 and half the threads); four
// where eight leave less than 200 000 threads (8 / 4, us: 309 rows fp32 10.7 / 8.5, 1009 bf16 12.2 / 11.2, 2009 17.1 / 17.2).
constexpr int kTok = 8, kFewTok = 4, kFewThreads = 200000;
static_assert(kFewTok >= 3, "only the thread of a sequence's first tokens reads its window");

// VW adjacent channels of a row
template <typename T, int VW> struct Chan {
    typedef T type __attribute__((ext_vector_type(VW), aligned(VW * sizeof(T) < 16 ? VW * sizeof(T) : 16)));
};

// (the reciprocal instruction, off by a step, not the ten instructions of a division: 33280 rows of 10240 channels 283 -> 255 us)
__device__ __forceinline__ float silu(float v) { return v * __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

template <typename T>
struct ConvArgs {
    const T *u, *w, *b, *win_in;
    T *win_out, *xo, *Bo, *Co;
    long long ld;
    int Cx, Cb;
};

// The channels' taps and biases
template <typename T, int W, int VW>
struct Taps {
    float w[VW][W], b[VW];
    __device__ __forceinline__ Taps(const T *wp, const T *bp, int c0) {
        typedef typename Chan<T, VW>::type V;
        T flat[VW * W];  // the taps of adjacent channels are adjacent
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const V v = *reinterpret_cast<const V *>(wp + (size_t)c0 * W + VW * i);
#pragma unroll
            for (int e = 0; e < VW; ++e) flat[VW * i + e] = v[e];
        }
        V bv = {};
        if (bp) bv = *reinterpret_cast<const V *>(bp + c0);
#pragma unroll
        for (int e = 0; e < VW; ++e) {
            b[e] = to_f32((T)bv[e]);
#pragma unroll
            for (int k = 0; k < W; ++k) w[e][k] = to_f32(flat[W * e + k]);
        }
    }
    template <typename V>
    __device__ __forceinline__ V apply(const V (&rows)[W]) const {
        V o;
#pragma unroll
        for (int e = 0; e < VW; ++e) {
            float acc = b[e];
#pragma unroll
            for (int k = 0; k < W; ++k) acc = fmaf(w[e][k], to_f32((T)rows[k][e]), acc);
            o[e] = from_f32<T>(silu(acc));
        }
        return o;
    }
};

// Where channel c0 of an output row goes, and that tensor's pitch
template <typename T>
__device__ __forceinline__ T *out_of(const ConvArgs<T> &a, int c0, int &pitch) {
    pitch = c0 < a.Cx ? a.Cx : a.Cb;
    return c0 < a.Cx ? a.xo + c0 : c0 < a.Cx + a.Cb ? a.Bo + (c0 - a.Cx) : a.Co + (c0 - a.Cx - a.Cb);
}

// One thread: VW adjacent channels of TOK consecutive tokens of one sequence.  All rows are requested before any arithmetic.  The thread of a
// sequence's first tokens alone reads the old window, and it writes the new one afterwards, so the two may be one buffer.
template <typename T, int W, int VW, int TOK>
__global__ __launch_bounds__(kThreads) void conv_varlen_kernel(ConvArgs<T> a, CarryTab tab, int vecs, int nunits) {
    typedef typename Chan<T, VW>::type V;
    const int unit = xcd_swizzle(blockIdx.x, nunits);
    const long long gid = (long long)unit * kThreads + threadIdx.x;
    const int tile = (int)(gid / vecs), c0 = (int)(gid % vecs) * VW;
    if (unit >= nunits || tile >= tab.base[tab.nseq]) return;
    const int s = tab.find(tile), t0 = (tile - tab.base[s]) * TOK, len = tab.len[s];
    const int Ct = a.Cx + 2 * a.Cb;
    const T *u = a.u + (size_t)tab.row0[s] * a.ld + c0;
    const bool history = a.win_in && !(tab.fresh >> s & 1);
    const size_t win = (size_t)tab.slot[s] * (W - 1) * Ct + c0;
    auto row = [&](int t) -> V {  // row t of the sequence, from its window below 0
        if (t >= 0) return *reinterpret_cast<const V *>(u + (size_t)t * a.ld);
        if (history) return *reinterpret_cast<const V *>(a.win_in + win + (size_t)(W - 1 + t) * Ct);
        return V{};
    };
    if (t0 < len) {
        V rows[TOK + W - 1];
        if (t0 > 0) {  // rows past the end: the last one again, not used
#pragma unroll
            for (int j = 0; j < TOK + W - 1; ++j) rows[j] = *reinterpret_cast<const V *>(u + (size_t)min(t0 - (W - 1) + j, len - 1) * a.ld);
        } else {
#pragma unroll
            for (int j = 0; j < TOK + W - 1; ++j) rows[j] = row(min(t0 - (W - 1) + j, len - 1));
        }
        const Taps<T, W, VW> taps(a.w, a.b, c0);
        int pitch;
        T *dst = out_of(a, c0, pitch) + (size_t)(tab.row0[s] + t0) * pitch;
#pragma unroll
        for (int i = 0; i < TOK; ++i)
            if (t0 + i < len) {
                V now[W];
#pragma unroll
                for (int k = 0; k < W; ++k) now[k] = rows[i + k];
                *reinterpret_cast<V *>(dst + (size_t)i * pitch) = taps.template apply<V>(now);
            }
    }
    if (t0 == 0 && a.win_out) {
        V last[W > 1 ? W - 1 : 1];
#pragma unroll
        for (int r = 0; r < W - 1; ++r) last[r] = row(len - (W - 1) + r);
#pragma unroll
        for (int r = 0; r < W - 1; ++r) *reinterpret_cast<V *>(a.win_out + win + (size_t)r * Ct) = last[r];
    }
}

// One token each of many sequences: a workgroup takes VW channels per thread of one entry; the last workgroups of an entry its dt,
//     dt[e, h] = log(1 + exp(row[e, Ct + h] + dt_bias[h])).
// An entry without a slot of its own gets zeros, its window is left alone.
template <typename T, int W, int VW>
__global__ __launch_bounds__(kThreads) void conv_step_kernel(ConvArgs<T> a, const int32_t *__restrict__ slots, int nslots, const float *__restrict__ dt_bias,
                                                             float *__restrict__ dt, int H, int conv_wgs) {
    typedef typename Chan<T, VW>::type V;
    const int e = blockIdx.y, Ct = a.Cx + 2 * a.Cb;
    const int slot = slot_of_entry(slots, e, nslots);
    const T *u = a.u + (size_t)e * a.ld;
    if ((int)blockIdx.x >= conv_wgs) {  // uniform
        const int h = ((int)blockIdx.x - conv_wgs) * kThreads + threadIdx.x;
        if (h >= H) return;
        const float v = to_f32(u[Ct + h]) + (dt_bias ? dt_bias[h] : 0.f);
        dt[(size_t)e * H + h] = slot < 0 ? 0.f : v > 20.f ? v : log1pf(__expf(v));
        return;
    }
    const int c0 = ((int)blockIdx.x * kThreads + (int)threadIdx.x) * VW;
    if (c0 >= Ct) return;
    int pitch;
    T *dst = out_of(a, c0, pitch) + (size_t)e * pitch;
    if (slot < 0) {
        *reinterpret_cast<V *>(dst) = V{};
        return;
    }
    const size_t win = (size_t)slot * (W - 1) * Ct + c0;
    V rows[W];
#pragma unroll
    for (int k = 0; k < W - 1; ++k) rows[k] = *reinterpret_cast<const V *>(a.win_in + win + (size_t)k * Ct);
    rows[W - 1] = *reinterpret_cast<const V *>(u + c0);
    const Taps<T, W, VW> taps(a.w, a.b, c0);
    *reinterpret_cast<V *>(dst) = taps.template apply<V>(rows);
#pragma unroll
    for (int k = 0; k < W - 1; ++k) *reinterpret_cast<V *>(a.win_out + win + (size_t)k * Ct) = rows[k + 1];
}

template <typename F> void by_width(int W, F &&f) {
    if (W == 4) f(std::integral_constant<int, 4>());
    else if (W == 3) f(std::integral_constant<int, 3>());
    else if (W == 2) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 1>());
}

// 16 bytes of channels at a time (fp32: 8000 rows with 32 bytes 145 us, 16 125) where column ranges, pitches and addresses keep them whole, else one.
template <typename... P>
bool whole_vectors(int vw, int Cx, int Cb, long long ld, const P *...p) {
    return Cx % vw == 0 && Cb % vw == 0 && ld % vw == 0 && ((... | (uintptr_t)p) & 15u) == 0;
}

}  // namespace

int conv_varlen(const void *xbc, long long ld, const void *w, const void *b, const void *window_in, void *window_out, const strd_seq *seqs, int nseq,
                int nslots, const int32_t *slots, const uint8_t *fresh, void *xo, void *Bo, void *Co, int Cx, int Cb, int W, strd_dtype io, hipStream_t st) {
    CarryTab tab;
    long long rows;
    const bool always = window_out != nullptr && W > 1;
    if (!plan_carry(seqs, nseq, window_in || window_out, nslots, slots, fresh, kTok, always, tab, rows)) return STRD_EINVAL;
    if (rows > 0 && (!xbc || !w || (Cx && !xo) || (Cb && (!Bo || !Co)))) return STRD_EINVAL;
    if (tab.base[nseq] == 0) return STRD_OK;
    const int whole = io == STRD_F32 ? 4 : 8, Ct = Cx + 2 * Cb;
    const bool vec = whole_vectors(whole, Cx, Cb, ld, xbc, w, b, window_in, window_out, xo, Bo, Co);
    const int vecs = vec ? Ct / whole : Ct;
    const bool few = (long long)tab.base[nseq] * vecs < kFewThreads;
    if (few) plan_carry(seqs, nseq, false, nslots, slots, fresh, kFewTok, always, tab, rows);
    const int tiles = tab.base[nseq];
    const long long units = ((long long)tiles * vecs + kThreads - 1) / kThreads;
    if (units > (1 << 24) - kXcd) return STRD_EUNSUPPORTED;  // threads of a launch have 32 bits
    auto run = [&](auto *tag) {
        using T = std::remove_pointer_t<decltype(tag)>;
        const ConvArgs<T> a = {(const T *)xbc, (const T *)w, (const T *)b, (const T *)window_in, (T *)window_out, (T *)xo, (T *)Bo, (T *)Co, ld, Cx, Cb};
        by_width(W, [&](auto width) {
            constexpr int VW = 16 / sizeof(T);
            auto go = [&](auto *kernel) { kernel<<<xcd_grid((int)units), kThreads, 0, st>>>(a, tab, vecs, (int)units); };
            if (vec && few) go(&conv_varlen_kernel<T, width.value, VW, kFewTok>);
            else if (vec) go(&conv_varlen_kernel<T, width.value, VW, kTok>);
            else if (few) go(&conv_varlen_kernel<T, width.value, 1, kFewTok>);
            else go(&conv_varlen_kernel<T, width.value, 1, kTok>);
        });
    };
    if (io == STRD_F32) run((float *)nullptr);
    else run((bf16_t *)nullptr);
    return launch_status();
}

int conv_step(const void *row, long long ld, const void *w, const void *b, const float *dt_bias, const void *window_in, void *window_out, int nslots,
              const int32_t *slots, void *xo, void *Bo, void *Co, float *dt, int batch, int Cx, int Cb, int H, int W, strd_dtype io, hipStream_t st) {
    if (batch == 0) return STRD_OK;
    const int whole = io == STRD_F32 ? 4 : 8;
    const bool vec = whole_vectors(whole, Cx, Cb, ld, row, w, b, window_in, window_out, xo, Bo, Co);
    const int wgs = ceil_div(Cx + 2 * Cb, kThreads * (vec ? whole : 1));
    const dim3 grid(wgs + ceil_div(H, kThreads), batch);
    auto run = [&](auto *tag) {
        using T = std::remove_pointer_t<decltype(tag)>;
        const ConvArgs<T> a = {(const T *)row, (const T *)w, (const T *)b, (const T *)window_in, (T *)window_out, (T *)xo, (T *)Bo, (T *)Co, ld, Cx, Cb};
        by_width(W, [&](auto width) {
            if (vec) conv_step_kernel<T, width.value, 16 / sizeof(T)><<<grid, kThreads, 0, st>>>(a, slots, nslots, dt_bias, dt, H, wgs);
            else conv_step_kernel<T, width.value, 1><<<grid, kThreads, 0, st>>>(a, slots, nslots, dt_bias, dt, H, wgs);
        });
    };
    if (io == STRD_F32) run((float *)nullptr);
    else run((bf16_t *)nullptr);
    return launch_status();
}

}  // namespace strd
