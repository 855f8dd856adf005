// The 4-bit cache: what a group of 32 channels of one (row, kv head) is held as.
//   32 codes n in 0..15, channel 2 i in the low half of byte i, channel 2 i + 1 in the high half (16 bytes), and
//   two bf16 numbers, the step s and the value z of code 8 (4 bytes); a code stands for z + s (n - 8).
// Of the group's smallest and largest value lo, hi, in fp32:
//   s = bf16((hi - lo) / 15), 0 if that is below 2^-100;  z = bf16(lo + 8 s);
//   n = clamp(rint((x - z) / s) + 8, 0, 15), ties of the quotient to the even side; 8 where s = 0.
// A group with a value that is not finite, or whose s or z is not, has s = z = NaN: it reads back as NaN and can be
// told from every other, where single codes could not carry one.
#pragma once
#include "common.h"

namespace strd {

constexpr int kKv4Group = 32;
constexpr float kKv4Tiny = 7.888609052210118e-31f;  // 2^-100

struct Kv4Group {
    float s, z;
};
__device__ __forceinline__ Kv4Group kv4_meta(uint32_t m) {  // s in the low half
    return {__builtin_bit_cast(float, m << 16), __builtin_bit_cast(float, m & 0xFFFF0000u)};
}
__device__ __forceinline__ float kv4_value(uint32_t codes, int i, Kv4Group g) {
    return fmaf(g.s, (float)((codes >> (4 * i)) & 15u) - 8.f, g.z);  // (s times a small integer is exact: one rounding)
}

}  // namespace strd
