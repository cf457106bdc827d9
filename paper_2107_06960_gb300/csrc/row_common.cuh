// What the kernels that go over rows of channels share: accesses of some channels, overlapped launches, results in 8 bits.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "attention.h"

namespace {

constexpr float kE4m3Max = 448.f;

__device__ __forceinline__ float max_nan(float x, float y) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
    return r;
}

// V channels as one access of V elements; loaded as they are and widened later, so that what is in
// flight takes few registers
template <class T, int V>
struct Vec;
template <>
struct Vec<float, 4> {
    float4 u;
    __device__ __forceinline__ void load(const float* p, bool on) {
        u = on ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w; }
    static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
};
template <>
struct Vec<__nv_bfloat16, 8> {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool on) {
        u = on ? *reinterpret_cast<const uint4*>(p) : make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Vec<__nv_bfloat16, 4> {
    uint2 u;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool on) {
        u = on ? *reinterpret_cast<const uint2*>(p) : make_uint2(0u, 0u);
    }
    __device__ __forceinline__ void get(float (&v)[4]) const {
        v[0] = __uint_as_float(u.x << 16);
        v[1] = __uint_as_float(u.x & 0xFFFF0000u);
        v[2] = __uint_as_float(u.y << 16);
        v[3] = __uint_as_float(u.y & 0xFFFF0000u);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[4]) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
        *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    }
};
template <>
struct Vec<float, 2> {
    float2 u;
    __device__ __forceinline__ void load(const float* p, bool on) {
        u = on ? *reinterpret_cast<const float2*>(p) : make_float2(0.f, 0.f);
    }
    __device__ __forceinline__ void get(float (&v)[2]) const { v[0] = u.x; v[1] = u.y; }
    static __device__ __forceinline__ void store(float* p, const float (&v)[2]) {
        *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
    }
};
template <>
struct Vec<__nv_bfloat16, 2> {
    uint32_t u;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool on) {
        u = on ? *reinterpret_cast<const uint32_t*>(p) : 0u;
    }
    __device__ __forceinline__ void get(float (&v)[2]) const {
        v[0] = __uint_as_float(u << 16);
        v[1] = __uint_as_float(u & 0xFFFF0000u);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[2]) {
        *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(v[0], v[1]);
    }
};
template <>
struct Vec<float, 1> {
    float u;
    __device__ __forceinline__ void load(const float* p, bool on) { u = on ? *p : 0.f; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = u; }
    static __device__ __forceinline__ void store(float* p, const float (&v)[1]) { *p = v[0]; }
};
template <>
struct Vec<__nv_bfloat16, 1> {
    __nv_bfloat16 u;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool on) { u = on ? *p : __float2bfloat16_rn(0.f); }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = __bfloat162float(u); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[1]) { *p = __float2bfloat16_rn(v[0]); }
};
// V values in 8 bits; past the largest value the conversion saturates, a NaN stays one
template <int V>
__device__ __forceinline__ void store8(uint8_t* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = (uint8_t)__nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
    } else if constexpr (V == 2) {
        *reinterpret_cast<uint16_t*>(p) = __nv_cvt_float2_to_fp8x2(make_float2(v[0], v[1]), __NV_SATFINITE, __NV_E4M3);
    } else {
        uint32_t w[V / 4];
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
            w[i] = lo | hi << 16;
        }
        if constexpr (V == 8)
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else
            *reinterpret_cast<uint32_t*>(p) = w[0];
    }
}

// The launch may start while the one before it ends.
__device__ __forceinline__ void launch_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// of values that are not negative, whose bits are ordered as they are and a NaN's are above all
template <int WIDTH>
__device__ __forceinline__ float max_over(float v) {
    if constexpr (WIDTH == 32) return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
#pragma unroll
    for (int w = 1; w < WIDTH; w *= 2) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, w));
    return v;
}
// v / s by the reciprocal, whose error of 2^-23 is far below a step of 8 bits; for scales so small that it
// could overflow, by division
template <int V>
__device__ __forceinline__ void divide(float (&v)[V], float s) {
    if (s < 0x1p-100f) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = v[j] / s;
    } else {
        const float r = 1.f / s;
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] *= r;
    }
}
// 1 where the quotient is 0, which it also is for values below 448 * 2^-150
__device__ __forceinline__ float scale_of(float top) {
    const float s = top / kE4m3Max;
    return s == 0.f ? 1.f : s;
}

// Writes a row's norm h * inv * weight, with its scales where it is in 8 bits.  The thread has N accesses of V channels from
// c0, 32 * V apart; `part`: room for a value of each of the row's warps.
template <class T, int V, int N, MafatNormQuant Q>
__device__ __forceinline__ void finish_row(const MafatNormArgs& a, int64_t row, int c0, float (&h)[N][V], const Vec<T, V> (&vw)[N],
                                           float inv, float* part, int warps) {
    const int lane = threadIdx.x, warp = threadIdx.y;
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = c0 + i * 32 * V;
        float w[V];
        vw[i].get(w);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            h[i][j] = h[i][j] * inv * w[j];
            if (Q == MAFAT_NORM_ROW && c < a.cols) top = max_nan(top, fabsf(h[i][j]));
        }
    }
    if constexpr (Q == MAFAT_NORM_PLAIN) {
        T* y = (T*)a.y + row * a.y_s;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = c0 + i * 32 * V;
            if (c < a.cols) Vec<T, V>::store(y + c, h[i]);
        }
        return;
    }
    uint8_t* y = (uint8_t*)a.y + row * a.y_s;
    if constexpr (Q == MAFAT_NORM_ROW) {
        top = max_over<32>(top);
        if (warps > 1) {
            if (lane == 0) part[warp] = top;
            __syncthreads();
            top = max_over<32>(lane < warps ? part[lane] : 0.f);
        }
        const float s = scale_of(top);
        if (lane == 0 && warp == 0) a.scales[row] = s;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = c0 + i * 32 * V;
            divide(h[i], s);
            if (c < a.cols) store8<V>(y + c, h[i]);
        }
    } else {
        constexpr int kLanes = 128 / V < 32 ? 128 / V : 32;  // lanes that share a block of channels
        constexpr int kRuns = 128 / V / kLanes;              // accesses of a lane in one block
        static_assert(N % kRuns == 0, "whole blocks in a warp");
        float* scales = a.scales + row * a.groups;
#pragma unroll
        for (int g = 0; g < N / kRuns; ++g) {
            float t = 0.f;
#pragma unroll
            for (int i = 0; i < kRuns; ++i)
                if (c0 + (g * kRuns + i) * 32 * V < a.cols)
#pragma unroll
                    for (int j = 0; j < V; ++j) t = max_nan(t, fabsf(h[g * kRuns + i][j]));
            const float s = scale_of(max_over<kLanes>(t));
#pragma unroll
            for (int i = 0; i < kRuns; ++i) {
                const int k = g * kRuns + i, c = c0 + k * 32 * V;
                divide(h[k], s);
                if (c < a.cols) {
                    store8<V>(y + c, h[k]);
                    if (c % 128 == 0) scales[c / 128] = s;
                }
            }
        }
    }
}

}  // namespace
