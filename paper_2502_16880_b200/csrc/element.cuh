// Element types of the operators that take bf16, fp16 or fp32 rows: eight elements at a time, widened to fp32 and
// rounded back once (round to nearest even).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace coral {

template <typename T> struct Elem;

template <> struct Elem<float> {
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
    static __device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    static __device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
};

template <> struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 down(float v) { return __float2bfloat16_rn(v); }
    static __device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
        v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
    }
    static __device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
        uint4 a;
        __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&a);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<uint4*>(p) = a;
    }
};

template <> struct Elem<__half> {
    static __device__ __forceinline__ float up(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half down(float v) { return __float2half_rn(v); }
    static __device__ __forceinline__ void load8(const __half* p, float (&v)[8]) {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        const __half2* h = reinterpret_cast<const __half2*>(&a);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(h[i]);
            v[2 * i] = f.x; v[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ void store8(__half* p, const float (&v)[8]) {
        uint4 a;
        __half2* h = reinterpret_cast<__half2*>(&a);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<uint4*>(p) = a;
    }
};

// Eight fp32 values as four pairs: the two-wide instructions do the arithmetic of a pair at once (each half rounds as the
// scalar instruction does).
struct V8 {
    unsigned long long p[4];
};
__device__ __forceinline__ unsigned long long pair_of(float lo, float hi) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 halves(unsigned long long p) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p));
    return f;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ V8 operator*(const V8& a, const V8& b) {
    V8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.p[i] = mul2(a.p[i], b.p[i]);
    return r;
}
__device__ __forceinline__ V8 fma8(const V8& a, const V8& b, const V8& c) {
    V8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.p[i] = fma2(a.p[i], b.p[i], c.p[i]);
    return r;
}
__device__ __forceinline__ V8 splat8(float v) {
    const unsigned long long p = pair_of(v, v);
    return V8{{p, p, p, p}};
}
// acc + a b, the products added up over four pairs
__device__ __forceinline__ unsigned long long dot8v(const V8& a, const V8& b, unsigned long long acc) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = fma2(a.p[i], b.p[i], acc);
    return acc;
}
template <typename T>
__device__ __forceinline__ V8 load8v(const T* p) {
    float f[8];
    Elem<T>::load8(p, f);
    return V8{{pair_of(f[0], f[1]), pair_of(f[2], f[3]), pair_of(f[4], f[5]), pair_of(f[6], f[7])}};
}
template <typename T>
__device__ __forceinline__ void store8v(T* p, const V8& v) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 h = halves(v.p[i]);
        f[2 * i] = h.x;
        f[2 * i + 1] = h.y;
    }
    Elem<T>::store8(p, f);
}

}  // namespace coral
