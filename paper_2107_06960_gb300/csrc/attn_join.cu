// Joins the parts of each row: O = sum_i w_i O_i / sum_i w_i with w_i = 2^(lse_i - max lse).
//
// A warp takes a row; a lane four channels, of every second part where a row has 64 channels at
// most.  The weights are made first, a lane each, so that the loads of eight parts are on their way
// together: the kernel is bound by those round trips for few rows, by the parts' bytes (in L2, just
// written) for many.  The order of the sums is fixed, so results do not change from run to run.
#include <cuda_bf16.h>

#include "attn_common.cuh"

namespace {

constexpr int kWarps = 4;

__device__ __forceinline__ void put(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float4 v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2*>(p) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// WAYS parts at a time: 2 with rows of up to 64 channels, 1 of up to 128
template <class T, int WAYS>
__global__ void __launch_bounds__(kWarps * 32) attn_join_kernel(const __grid_constant__ MafatAttnArgs a) {
    constexpr int kLanes = 32 / WAYS, kUnroll = 8;
    mafat_attn::launch_begin(a);
    const int64_t row = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    const int lane = threadIdx.x % 32;
    if (row >= a.rows_total) return;
    const int way = lane / kLanes, d = lane % kLanes * 4;
    const bool in_dim = d < a.dim;
    // log2 sums of the parts, 32 at a time in the lanes: at most MAFAT_ATTN_MAX_SPLITS of each set of keys
    constexpr int kSets = 8;
    float lse[kSets], top = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
        const int p = i * 32 + lane;
        lse[i] = p < a.parts ? a.part_lse[(int64_t)p * a.rows_total + row] : -CUDART_INF_F;
        top = mafat_attn::max_nan(top, lse[i]);
    }
#pragma unroll
    for (int w = 1; w < 32; w *= 2) top = mafat_attn::max_nan(top, __shfl_xor_sync(0xffffffffu, top, w));
    const float base = top == -CUDART_INF_F ? 0.f : top;
    float sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
        if (i * 32 >= a.parts) break;
        const float w = mafat_attn::exp2_fast(lse[i] - base);
        sum += w;
        const int n = min(32, a.parts - i * 32);
        const float* src = a.part_o + ((int64_t)(i * 32) * a.rows_total + row) * a.dim + d;
#pragma unroll 1
        for (int p0 = 0; p0 < n; p0 += kUnroll * WAYS) {
            float4 v[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int p = p0 + u * WAYS + way;
                v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (p < n && in_dim) v[u] = *reinterpret_cast<const float4*>(src + (int64_t)p * a.rows_total * a.dim);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const float x = __shfl_sync(0xffffffffu, w, (p0 + u * WAYS + way) & 31);  // past n: v is zero
                acc.x = fmaf(x, v[u].x, acc.x);
                acc.y = fmaf(x, v[u].y, acc.y);
                acc.z = fmaf(x, v[u].z, acc.z);
                acc.w = fmaf(x, v[u].w, acc.w);
            }
        }
    }
#pragma unroll
    for (int w = 1; w < 32; w *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    if (WAYS == 2) {
        acc.x += __shfl_xor_sync(0xffffffffu, acc.x, 16);
        acc.y += __shfl_xor_sync(0xffffffffu, acc.y, 16);
        acc.z += __shfl_xor_sync(0xffffffffu, acc.z, 16);
        acc.w += __shfl_xor_sync(0xffffffffu, acc.w, 16);
    }
    const float inv = mafat_attn::inverse_sum(sum);
    const uint32_t u = a.heads_q_div.div((uint32_t)row), req = a.n_q_div.div(u);
    const int h = (int)((uint32_t)row - u * (uint32_t)a.heads_q), t = (int)(u - req * (uint32_t)a.n_q);
    if (way == 0 && in_dim)
        put((T*)a.out + (int64_t)req * a.o_sb + (int64_t)t * a.o_st + (int64_t)h * a.o_sh + d,
            make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
    if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -CUDART_INF_F : (base + log2f(sum)) * CUDART_LN2_F;
}

template <class T>
cudaError_t launch(const MafatAttnArgs& a, cudaStream_t s) {
    const unsigned blocks = (unsigned)((a.rows_total + kWarps - 1) / kWarps);
    return a.dim <= 64 ? mafat_launch_overlapped(attn_join_kernel<T, 2>, blocks, kWarps * 32, 0, s, a)
                       : mafat_launch_overlapped(attn_join_kernel<T, 1>, blocks, kWarps * 32, 0, s, a);
}

}  // namespace

cudaError_t mafat_launch_attn_join(const MafatAttnArgs& a, bool bf16, cudaStream_t s) {
    return bf16 ? launch<__nv_bfloat16>(a, s) : launch<float>(a, s);
}
