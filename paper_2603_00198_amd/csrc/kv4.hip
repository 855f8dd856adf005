// Rows of keys and values into the 4-bit cache (kv4.h) and back.  Both are bound by HBM: a row is read once and
// written once, 2 + 5/8 bytes per bf16 element either way.  A lane takes 8 neighbouring channels (16 bytes of bf16, 32 of fp32, one
// dword of codes), the four lanes of a group exchange their smallest and largest value by quad permutations, and one of
// them stores the group's step and middle.  Keys and values go in one launch.
#include "kv4.h"

namespace strd {
namespace {

constexpr int kThreads = 256;

template <typename T> struct Vec8;
template <> struct Vec8<bf16_t> {
    typedef __bf16 type __attribute__((ext_vector_type(8)));
};
template <> struct Vec8<float> {
    typedef float type __attribute__((ext_vector_type(8)));
};

template <int CTRL>
__device__ __forceinline__ float quad(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E;  // quad permutations [1,0,3,2] and [2,3,0,1]

// bits of a bf16 number, rounded to nearest even
__device__ __forceinline__ uint32_t bf16_bits(float v) { return __builtin_bit_cast(uint16_t, (bf16_t)v); }
__device__ __forceinline__ float bf16_round(float v) { return (float)(bf16_t)v; }

struct Side {
    const void *rows;    // [R rows of pitch ld]: this side's keys or values
    void *codes, *meta;  // the cache's rows from the first one on
    long long ld;        // elements between rows
};

// VEC: 8 elements of a row can be read as one vector.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void kv4_store_kernel(Side k, Side v, long long units, int upr) {
    typedef typename Vec8<T>::type V;
    const Side &sd = blockIdx.y ? v : k;
    const long long u = (long long)blockIdx.x * kThreads + threadIdx.x;  // 8 channels; 4 lanes a group, never half of one
    if (u >= units) return;
    const long long row = u / upr;
    const int c = (int)(u - row * upr);
    const T *src = (const T *)sd.rows + row * sd.ld + 8 * c;
    float x[8];
    if constexpr (VEC) {
        const V t = *reinterpret_cast<const V *>(src);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = to_f32((T)t[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = to_f32(src[e]);
    }
    float lo = x[0], hi = x[0], odd = 0.f;  // odd: NaN if a value is not finite
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        lo = fminf(lo, x[e]);
        hi = fmaxf(hi, x[e]);
        odd = fmaf(x[e], 0.f, odd);
    }
    lo = fminf(lo, quad<kSwap1>(lo));
    hi = fmaxf(hi, quad<kSwap1>(hi));
    odd += quad<kSwap1>(odd);
    lo = fminf(lo, quad<kSwap2>(lo));
    hi = fmaxf(hi, quad<kSwap2>(hi));
    odd += quad<kSwap2>(odd);
    float s = bf16_round((hi - lo) / 15.f);
    const bool off = !(odd == 0.f) || !(s < INFINITY);
    s = s < kKv4Tiny ? 0.f : s;
    const float z = bf16_round(lo + 8.f * s);
    const bool bad = off || !(fabsf(z) < INFINITY);  // (bf16 ends below fp32's largest numbers)
    // (x - z) / s, correctly rounded: s has 8 bits and is no denormal, r is its correctly rounded reciprocal, and one residual
    // of the first quotient gives the second (Markstein), which is what a division would return
    const float r = s > 0.f ? 1.f / s : 0.f;
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = x[e] - z, q0 = d * r, q = fmaf(fmaf(-q0, s, d), r, q0);
        const float n = fminf(fmaxf(rintf(q) + 8.f, 0.f), 15.f);  // (NaN becomes 0)
        codes |= (uint32_t)n << (4 * e);
    }
    reinterpret_cast<uint32_t *>(sd.codes)[u] = codes;
    if ((c & 3) == 0)
        reinterpret_cast<uint32_t *>(sd.meta)[u / 4] = bad ? 0x7FC07FC0u : bf16_bits(s) | bf16_bits(z) << 16;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void kv4_load_kernel(const uint32_t *__restrict__ kc, const uint32_t *__restrict__ km,
                                                            const uint32_t *__restrict__ vc, const uint32_t *__restrict__ vm,
                                                            T *__restrict__ k, T *__restrict__ v, long long units) {
    typedef typename Vec8<T>::type V;
    const long long u = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (u >= units) return;
    const uint32_t codes = (blockIdx.y ? vc : kc)[u];
    const Kv4Group g = kv4_meta((blockIdx.y ? vm : km)[u / 4]);
    V out;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = from_f32<T>(kv4_value(codes, e, g));
    *reinterpret_cast<V *>((blockIdx.y ? v : k) + 8 * u) = out;
}

}  // namespace

int kv4_store_launch(const void *k, long long ldk, const void *v, long long ldv, const strd_kv4 &c, int row0, int R, int Hkv, int d,
                     strd_dtype io, hipStream_t st) {
    const int upr = Hkv * (d / 8);
    const long long units = (long long)R * upr, first = (long long)row0 * upr;
    const dim3 grid((unsigned)((units + kThreads - 1) / kThreads), 2);
    const Side sk = {k, (uint32_t *)c.k_codes + first, (uint32_t *)c.k_meta + first / 4, ldk};
    const Side sv = {v, (uint32_t *)c.v_codes + first, (uint32_t *)c.v_meta + first / 4, ldv};
    const size_t al = 8 * (io == STRD_BF16 ? 2 : 4);
    const bool vec = !((uintptr_t)k % al) && !((uintptr_t)v % al) && ldk % 8 == 0 && ldv % 8 == 0;
    if (io == STRD_BF16) {
        if (vec) kv4_store_kernel<bf16_t, true><<<grid, kThreads, 0, st>>>(sk, sv, units, upr);
        else kv4_store_kernel<bf16_t, false><<<grid, kThreads, 0, st>>>(sk, sv, units, upr);
    } else {
        if (vec) kv4_store_kernel<float, true><<<grid, kThreads, 0, st>>>(sk, sv, units, upr);
        else kv4_store_kernel<float, false><<<grid, kThreads, 0, st>>>(sk, sv, units, upr);
    }
    return launch_status();
}

int kv4_load_launch(const strd_kv4 &c, int row0, int R, void *k, void *v, int Hkv, int d, strd_dtype io, hipStream_t st) {
    const int upr = Hkv * (d / 8);
    const long long units = (long long)R * upr, first = (long long)row0 * upr;
    const dim3 grid((unsigned)((units + kThreads - 1) / kThreads), 2);
    const uint32_t *kc = (const uint32_t *)c.k_codes + first, *km = (const uint32_t *)c.k_meta + first / 4;
    const uint32_t *vc = (const uint32_t *)c.v_codes + first, *vm = (const uint32_t *)c.v_meta + first / 4;
    if (io == STRD_BF16)
        kv4_load_kernel<bf16_t><<<grid, kThreads, 0, st>>>(kc, km, vc, vm, (bf16_t *)k, (bf16_t *)v, units);
    else
        kv4_load_kernel<float><<<grid, kThreads, 0, st>>>(kc, km, vc, vm, (float *)k, (float *)v, units);
    return launch_status();
}

}  // namespace strd
