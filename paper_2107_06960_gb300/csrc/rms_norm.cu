// Root-mean-square norm with the residual's addition:
//   h = x + r,  y = h / sqrt(mean(h^2) + eps) * w,
// y in the inputs' type or in 8 bits: y / s rounded to e4m3 with s = max |y| / 448 over the row or
// over each 128 channels (s = 1 where that is 0 in fp32).
//
// One pass: a row's sums stay in registers between the sum of squares and the output, so that x, r
// are read and h, y written once; bound by those bytes.  Everything is fp32 until a result is
// rounded, once; the norm is taken of the unrounded h.  A warp takes a row where its registers hold
// one (no barrier), several warps of a block where they do not.  Each warp has a contiguous run
// of channels, a multiple of 128 long, so that a block of 128 channels lies in one warp.
//
// An access has 16 bytes of a row, or two channels or one where the rows' starts allow no more.  46208 rows of
// 1024 bf16, to e4m3 by blocks: 50 us or 6.7 TB/s, what a copy takes.  16244 rows of 1568, 1570 and 1571 channels: 31, 31
// and 41 us in bf16 (6.5, 6.5 and 5.0 TB/s); by blocks 34, 48 and 69 (issue: an access, a bound and a byte's store for
// every channel).  16 rows take 5 us: the launch and three round trips.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "attention.h"

namespace {

constexpr int kRowWarps = 4;   // rows of a block whose rows take one warp each
constexpr int kMaxWarps = 16;  // of a row
constexpr int kMaxThread = 32; // channels of a thread
constexpr int kFewRows = 2048;
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

// V channels an access, N accesses a thread.  blockDim = (32, warps of a row, rows).
template <class T, int V, int N, MafatNormQuant Q>
__global__ void __launch_bounds__(kMaxWarps * 32) rms_norm_kernel(const __grid_constant__ MafatNormArgs a) {
    __shared__ float part[2][kMaxWarps];
    const int lane = threadIdx.x, warp = threadIdx.y, warps = blockDim.y;
    const int64_t row = (int64_t)blockIdx.x * blockDim.z + threadIdx.z;
    if (row >= a.rows) return;  // only blocks whose rows take one warp each have several rows: no barrier follows
    const T* x = (const T*)a.x + row * a.x_s;
    const T* r = a.residual ? (const T*)a.residual + row * a.r_s : nullptr;
    const int c0 = (warp * 32 * N + lane) * V;
    Vec<T, V> vx[N], vr[N], vw[N];
    launch_wait();
#pragma unroll
    for (int i = 0; i < N; ++i) vx[i].load(x + c0 + i * 32 * V, c0 + i * 32 * V < a.cols);
#pragma unroll
    for (int i = 0; i < N; ++i) vr[i].load(r + c0 + i * 32 * V, r && c0 + i * 32 * V < a.cols);
#pragma unroll
    for (int i = 0; i < N; ++i) vw[i].load((const T*)a.weight + c0 + i * 32 * V, c0 + i * 32 * V < a.cols);
    launch_next();
    float h[N][V];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[V];
        vx[i].get(h[i]);
        vr[i].get(v);
#pragma unroll
        for (int j = 0; j < V; ++j) h[i][j] += v[j];
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) sum = fmaf(h[i][j], h[i][j], sum);
    if (a.residual_out) {
        T* ro = (T*)a.residual_out + row * a.ro_s;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = c0 + i * 32 * V;
            if (c < a.cols) Vec<T, V>::store(ro + c, h[i]);
        }
    }
#pragma unroll
    for (int w = 1; w < 32; w *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    if (warps > 1) {
        if (lane == 0) part[0][warp] = sum;
        __syncthreads();
        sum = lane < warps ? part[0][lane] : 0.f;
#pragma unroll
        for (int w = 1; w < 32; w *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    }
    const float inv = 1.f / sqrtf(sum / (float)a.cols + a.eps);
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
            if (lane == 0) part[1][warp] = top;
            __syncthreads();
            top = max_over<32>(lane < warps ? part[1][lane] : 0.f);
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

template <class T, int V, int N>
cudaError_t launch(const MafatNormArgs& a, MafatNormQuant q, int warps, cudaStream_t s) {
    const int rows = warps == 1 ? kRowWarps : 1;
    const dim3 block(32, warps, rows);
    const unsigned grid = (unsigned)((a.rows + rows - 1) / rows);
    return mafat_launch_overlapped(q == MAFAT_NORM_PLAIN ? rms_norm_kernel<T, V, N, MAFAT_NORM_PLAIN>
                                   : q == MAFAT_NORM_ROW ? rms_norm_kernel<T, V, N, MAFAT_NORM_ROW>
                                                         : rms_norm_kernel<T, V, N, MAFAT_NORM_BLOCK>,
                                   grid, block, 0, s, a);
}

// Accesses of a thread: with rows enough to fill the GPU, the fewest that leave a row to one warp (no
// barrier, more in flight a thread), as far as its registers go (with block scales fewer channels: in us, at 16244
// rows of 1568 fp32 64.6 with 32 a thread, 52.6 with 16, 53.2 with 8; of 1571 bf16 98.7, 83.2, 71.9); with few rows
// as few as 16 warps allow (a row is there sooner).
template <class T, int V, int N>
cudaError_t launch_v(const MafatNormArgs& a, MafatNormQuant q, cudaStream_t s) {
    const int per_warp = 32 * V * N;
    const int most = q != MAFAT_NORM_BLOCK ? kMaxThread : V == 1 ? 8 : 16;
    const bool one_warp = a.rows >= kFewRows && 2 * N * V <= most;
    if constexpr (2 * N * V <= kMaxThread)
        if (a.cols > per_warp * (one_warp ? 1 : kMaxWarps)) return launch_v<T, V, 2 * N>(a, q, s);
    return launch<T, V, N>(a, q, (a.cols + per_warp - 1) / per_warp, s);
}

}  // namespace

int mafat_norm_max_cols() { return kMaxWarps * 32 * kMaxThread; }

cudaError_t mafat_launch_norm(const MafatNormArgs& a, bool bf16, int vec, MafatNormQuant quant, cudaStream_t s) {
    // a warp has 128 channels at least: 4 accesses of one, 2 of two
    if (bf16)
        return vec >= 8   ? launch_v<__nv_bfloat16, 8, 1>(a, quant, s)
               : vec >= 2 ? launch_v<__nv_bfloat16, 2, 2>(a, quant, s)
                          : launch_v<__nv_bfloat16, 1, 4>(a, quant, s);
    return vec >= 4   ? launch_v<float, 4, 1>(a, quant, s)
           : vec >= 2 ? launch_v<float, 2, 2>(a, quant, s)
                      : launch_v<float, 1, 4>(a, quant, s);
}
