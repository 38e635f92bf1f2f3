// 4-bit operands of the warp MMA: unpacking without arithmetic (fp16 subnormals), and activations brought into fp16's range.
#pragma once
#include "element.cuh"

namespace coral {

__device__ __forceinline__ void q4_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// A word's eight weights as four MMA operands: (0,4), 16 (1,5), (2,6), 16 (3,7), in units of 2^-24.
__device__ __forceinline__ void q4_spread(uint32_t w, uint32_t (&v)[4]) {
    v[0] = w & 0x000f000fu;
    v[1] = w & 0x00f000f0u;
    w >>= 8;
    v[2] = w & 0x000f000fu;
    v[3] = w & 0x00f000f0u;
}

// The power of two that brings the largest absolute value (as bits) to 2^14..2^15 (below that, subnormal bf16 numbers: at least
// to 2^8, all of them whole); 1 for a row that is not finite.
__device__ __forceinline__ int q4_exponent(uint32_t max_bits) { return max_bits >= 0x7f800000u ? 0 : 141 - (int)(max_bits >> 23); }
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// v 2^e for e from -252 to 254: as two factors, since rows of bf16 want exponents from -113 to 141 and those that undo them.
// Neither product leaves the range of fp32 unless the result does.
struct Q4Power {
    float a, b;
    Q4Power() = default;
    __device__ __forceinline__ explicit Q4Power(int e) : a(exp2_int(e / 2)), b(exp2_int(e - e / 2)) {}
    __device__ __forceinline__ float operator()(float v) const { return v * a * b; }
};

// Eight scaled activations in the order of q4_spread.
__device__ __forceinline__ uint4 q4_operand(const float (&f)[8]) {
    uint4 v;
    const __half2 h[4] = {__floats2half2_rn(f[0], f[4]), __floats2half2_rn(f[1] * 0.0625f, f[5] * 0.0625f),
                          __floats2half2_rn(f[2], f[6]), __floats2half2_rn(f[3] * 0.0625f, f[7] * 0.0625f)};
    v.x = *reinterpret_cast<const uint32_t*>(&h[0]);
    v.y = *reinterpret_cast<const uint32_t*>(&h[1]);
    v.z = *reinterpret_cast<const uint32_t*>(&h[2]);
    v.w = *reinterpret_cast<const uint32_t*>(&h[3]);
    return v;
}

}  // namespace coral
