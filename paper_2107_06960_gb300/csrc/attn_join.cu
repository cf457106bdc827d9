// Joins the parts of each row: O = sum_i w_i O_i / sum_i w_i with w_i = 2^(lse_i - max lse).
//
// A warp takes a row.  Bound by the bytes of the parts (they are in L2, just written) and, for few
// rows, by the launch.  The order of the sum is fixed, so results do not change from run to run.
#include <cuda_bf16.h>

#include "attn_common.cuh"

namespace {

constexpr int kWarps = 4;

__device__ __forceinline__ void put(float* p, float2 v) { *reinterpret_cast<float2*>(p) = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float2 v) {
    *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(v.x, v.y);
}

template <class T>
__global__ void __launch_bounds__(kWarps * 32) attn_join_kernel(const __grid_constant__ MafatAttnArgs a) {
    const int64_t row = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    const int lane = threadIdx.x % 32;
    if (row >= a.rows_total) return;
    float top = -CUDART_INF_F;
    for (int p = lane; p < a.parts; p += 32) top = mafat_attn::max_nan(top, a.part_lse[p * a.rows_total + row]);
#pragma unroll
    for (int w = 1; w < 32; w *= 2) top = mafat_attn::max_nan(top, __shfl_xor_sync(0xffffffffu, top, w));
    const float base = top == -CUDART_INF_F ? 0.f : top;
    float2 acc[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    float sum = 0.f;
#pragma unroll 4
    for (int p = 0; p < a.parts; ++p) {
        const float w = mafat_attn::exp2_fast(a.part_lse[p * a.rows_total + row] - base);
        sum += w;
        const float* src = a.part_o + (p * a.rows_total + row) * a.dim;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int d = c * 64 + lane * 2;
            if (d < a.dim) {
                const float2 v = *reinterpret_cast<const float2*>(src + d);
                acc[c].x = fmaf(w, v.x, acc[c].x);
                acc[c].y = fmaf(w, v.y, acc[c].y);
            }
        }
    }
    const float inv = mafat_attn::inverse_sum(sum);
    const int h = (int)(row % a.heads_q), t = (int)(row / a.heads_q % a.n_q);
    const int64_t req = row / a.heads_q / a.n_q;
    T* out = (T*)a.out + req * a.o_sb + (int64_t)t * a.o_st + (int64_t)h * a.o_sh;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int d = c * 64 + lane * 2;
        if (d < a.dim) put(out + d, make_float2(acc[c].x * inv, acc[c].y * inv));
    }
    if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -CUDART_INF_F : (base + log2f(sum)) * CUDART_LN2_F;
}

}  // namespace

cudaError_t mafat_launch_attn_join(const MafatAttnArgs& a, bool bf16, cudaStream_t s) {
    const int64_t blocks = (a.rows_total + kWarps - 1) / kWarps;
    if (bf16)
        attn_join_kernel<__nv_bfloat16><<<(unsigned)blocks, kWarps * 32, 0, s>>>(a);
    else
        attn_join_kernel<float><<<(unsigned)blocks, kWarps * 32, 0, s>>>(a);
    return cudaGetLastError();
}
