// Rows of keys and values into the 4-bit cache (kv4.h) and back.  Both are bound by HBM: a row is read once and
// written once, 2 + 5/8 bytes per bf16 element either way.  A lane takes 8 neighbouring channels (16 bytes of bf16, 32 of fp32, one
// dword of codes), the four lanes of a group exchange their smallest and largest value by quad permutations, and one of
// them stores the group's step and middle.  Keys and values go in one launch.  33024 rows of 8 heads of 128 bf16 channels: store 40 us
// (177 MB, 4.4 TB/s; a large copy reaches 5.1), load 26 us; one row 2.0 and 1.6 us.
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

constexpr int kUnits = 2;  // pieces of 8 channels a lane has on their way

// The dword of codes of this lane's 8 values; (s, z) of its group, which it shares with the other lanes of its quad.
__device__ __forceinline__ uint32_t quantize(const float (&x)[8], uint32_t &meta) {
    // (minimum and maximum that keep a NaN: two values an instruction, and no look at single values)
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        lo = __builtin_elementwise_minimum(lo, x[e]);
        hi = __builtin_elementwise_maximum(hi, x[e]);
    }
    lo = __builtin_elementwise_minimum(lo, quad<kSwap1>(lo));
    hi = __builtin_elementwise_maximum(hi, quad<kSwap1>(hi));
    lo = __builtin_elementwise_minimum(lo, quad<kSwap2>(lo));
    hi = __builtin_elementwise_maximum(hi, quad<kSwap2>(hi));
    float s = bf16_round((hi - lo) / 15.f);
    const bool off = !(s < INFINITY);  // infinities and NaN are in the difference
    s = s < kKv4Tiny ? 0.f : s;
    const float z = bf16_round(lo + 8.f * s);
    const bool bad = off || !(fabsf(z) < INFINITY);  // (bf16 ends below fp32's largest numbers)
    // (x - z) / s, correctly rounded: s has 8 bits and is no denormal, r is its correctly rounded reciprocal, and one residual
    // of the first quotient gives the second (Markstein), which is what a division would return.  Clamped to -8 .. 7 it is
    // rounded to a whole number, ties to even, by adding 1.5 * 2^23; that and 8 leaves the code in the sum's low bits, and the eight
    // sums, shifted to their places, add up to the dword and a constant.
    const float r = s > 0.f ? 1.f / s : 0.f;
    constexpr float kRound = 12582912.f + 8.f;
    uint32_t codes = 0u - 0x4B400000u * 0x11111111u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = x[e] - z, q0 = d * r, q = fmaf(fmaf(-q0, s, d), r, q0);
        codes += __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(q, -8.f, 7.f) + kRound) << (4 * e);
    }
    meta = bad ? 0x7FC07FC0u : bf16_bits(s) | bf16_bits(z) << 16;
    return codes;
}

// VEC: 8 elements of a row can be read as one vector.  DENSE: rows lie one behind the other, and a lane's pieces need no division.
template <typename T, bool VEC, bool DENSE>
__global__ __launch_bounds__(kThreads) void kv4_store_kernel(Side k, Side v, long long units, int upr) {
    typedef typename Vec8<T>::type V;
    const Side &sd = blockIdx.y ? v : k;
    const long long u0 = (long long)blockIdx.x * (kThreads * kUnits) + threadIdx.x;  // 8 channels; 4 lanes a group, never half of one
    V t[kUnits];
    float x[kUnits][8];
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const long long u = min(u0 + kThreads * i, units - 1);
        const T *src = (const T *)sd.rows + 8 * u;
        if constexpr (!DENSE) {
            const long long row = u / upr;
            src = (const T *)sd.rows + row * sd.ld + 8 * (u - row * upr);
        }
        if constexpr (VEC) {
            t[i] = *reinterpret_cast<const V *>(src);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = to_f32(src[e]);
        }
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const long long u = u0 + kThreads * i;
        if constexpr (VEC)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = to_f32((T)t[i][e]);
        uint32_t meta;
        const uint32_t codes = quantize(x[i], meta);
        if (u >= units) continue;  // (the four lanes of a group are on one side of the end)
        reinterpret_cast<uint32_t *>(sd.codes)[u] = codes;
        if ((u & 3) == 0) reinterpret_cast<uint32_t *>(sd.meta)[u / 4] = meta;
    }
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
    const dim3 grid((unsigned)((units + kThreads * kUnits - 1) / (kThreads * kUnits)), 2);
    const Side sk = {k, (uint32_t *)c.k_codes + first, (uint32_t *)c.k_meta + first / 4, ldk};
    const Side sv = {v, (uint32_t *)c.v_codes + first, (uint32_t *)c.v_meta + first / 4, ldv};
    const size_t al = 8 * (io == STRD_BF16 ? 2 : 4);
    const bool dense = (ldk == (long long)Hkv * d && ldv == ldk) || R == 1;
    const bool vec = !((uintptr_t)k % al) && !((uintptr_t)v % al) && (dense || (ldk % 8 == 0 && ldv % 8 == 0));
    auto launch = [&](auto *tag) {
        using T = std::remove_pointer_t<decltype(tag)>;
        if (vec && dense) kv4_store_kernel<T, true, true><<<grid, kThreads, 0, st>>>(sk, sv, units, upr);
        else if (vec) kv4_store_kernel<T, true, false><<<grid, kThreads, 0, st>>>(sk, sv, units, upr);
        else kv4_store_kernel<T, false, false><<<grid, kThreads, 0, st>>>(sk, sv, units, upr);
    };
    if (io == STRD_BF16) launch((bf16_t *)nullptr);
    else launch((float *)nullptr);
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
