// The norms around a block, with its gate and the residual's scale:
//   n = x / sqrt(mean(x^2) + eps) * w1;  h = a r + b g n;  y = h / sqrt(mean(h^2) + eps) * w2,
// y in the inputs' type or in 8 bits with scales, as the norm alone has them.
//
// One pass: a row stays in registers between its two sums of squares and the output, so that x, r are read and h, y
// written once; bound by those bytes.  All is fp32 until a result is rounded, once; y is of the unrounded h.  A row is one warp's
// where its registers hold it, as in the norm alone; the second sum of squares waits for the first, not for memory.
//
// 46208 rows of 1024 bf16, a gate for each 5776: 56.5 us or 6.7 TB/s, what a copy takes.  1443 rows of 1001 fp32 6.3 us: a launch, two
// round trips and accesses of one channel.  16 rows of 1024 to e4m3 2.1 us.
#include "row_common.cuh"

namespace {

constexpr int kRowWarps = 4;   // rows of a block whose rows take one warp each
constexpr int kMaxWarps = 16;  // of a row
constexpr int kMaxThread = 32; // channels of a thread
// Rows have few warps where the GPU is full of them: from so many rows on, or, with accesses of 16 bytes and where no more than a quarter
// of what a row's warps have room for is lost by it, from so many such warps on.  In us, with as many warps as rows can have and with few:
// 750 rows of 4096 bf16 8.6, 7.0, 2000 of 2048 10.3, 9.9, 1100 of 512 3.14, 2.98, 520 of 1024 3.03, 3.32, 750 of 600 to e4m3 by blocks 3.25, 3.53; in
// accesses of one channel 1443 of 1001 fp32 6.3, 7.1; 17146 of 1312 bf16 44.1, 37.8.
constexpr int kManyRows = 2048, kManyWarps = 1024;

// Sum over the row's warps; `part` is not used by another sum of the row.
__device__ __forceinline__ float row_sum(float v, float* part, int warps) {
#pragma unroll
    for (int w = 1; w < 32; w *= 2) v += __shfl_xor_sync(0xffffffffu, v, w);
    if (warps > 1) {
        if (threadIdx.x == 0) part[threadIdx.y] = v;
        __syncthreads();
        v = (int)threadIdx.x < warps ? part[threadIdx.x] : 0.f;
#pragma unroll
        for (int w = 1; w < 32; w *= 2) v += __shfl_xor_sync(0xffffffffu, v, w);
    }
    return v;
}

// V channels an access, N accesses a thread.  blockDim = (32, warps of a row, rows).
template <class T, int V, int N, MafatNormQuant Q>
__global__ void __launch_bounds__(kMaxWarps * 32) block_norm_kernel(const __grid_constant__ MafatBlockNormArgs a) {
    __shared__ float part[3][kMaxWarps];
    const int lane = threadIdx.x, warp = threadIdx.y, warps = blockDim.y;
    const int64_t row = (int64_t)blockIdx.x * blockDim.z + threadIdx.z;
    if (row >= a.n.rows) return;  // only blocks whose rows take one warp each have several rows: no barrier follows
    const int cols = a.n.cols;
    const int c0 = (warp * 32 * N + lane) * V;
    Vec<T, V> vx[N], vr[N], vw[N];
    launch_wait();
    const T* x = (const T*)a.n.x + row * a.n.x_s;
    const T* r = (const T*)a.n.residual + row * a.n.r_s;
#pragma unroll
    for (int i = 0; i < N; ++i) vx[i].load(x + c0 + i * 32 * V, c0 + i * 32 * V < cols);
#pragma unroll
    for (int i = 0; i < N; ++i) vr[i].load(r + c0 + i * 32 * V, c0 + i * 32 * V < cols);
    launch_next();
    float h[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i) vx[i].get(h[i]);
    if (a.post_weight) {
#pragma unroll
        for (int i = 0; i < N; ++i) vw[i].load((const T*)a.post_weight + c0 + i * 32 * V, c0 + i * 32 * V < cols);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) sum = fmaf(h[i][j], h[i][j], sum);
        const float inv = 1.f / sqrtf(row_sum(sum, part[0], warps) / (float)cols + a.n.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float w[V];
            vw[i].get(w);
#pragma unroll
            for (int j = 0; j < V; ++j) h[i][j] = h[i][j] * inv * w[j];
        }
    }
    if (a.gate) {
        const T* gate = (const T*)a.gate + (int64_t)a.gate_div.div((uint32_t)row) * a.g_s;
#pragma unroll
        for (int i = 0; i < N; ++i) vw[i].load(gate + c0 + i * 32 * V, c0 + i * 32 * V < cols);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float w[V];
            vw[i].get(w);
#pragma unroll
            for (int j = 0; j < V; ++j) h[i][j] *= w[j];
        }
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[V];
        vr[i].get(v);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            h[i][j] = fmaf(a.branch, h[i][j], a.keep * v[j]);
            sum = fmaf(h[i][j], h[i][j], sum);
        }
    }
    if (a.n.residual_out) {
        T* ro = (T*)a.n.residual_out + row * a.n.ro_s;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = c0 + i * 32 * V;
            if (c < cols) Vec<T, V>::store(ro + c, h[i]);
        }
    }
    if (!a.n.y) return;
#pragma unroll
    for (int i = 0; i < N; ++i) vw[i].load((const T*)a.n.weight + c0 + i * 32 * V, c0 + i * 32 * V < cols);
    const float inv = 1.f / sqrtf(row_sum(sum, part[1], warps) / (float)cols + a.n.eps);
    finish_row<T, V, N, Q>(a.n, row, c0, h, vw, inv, part[2], warps);
}

template <class T, int V, int N>
cudaError_t launch(const MafatBlockNormArgs& a, MafatNormQuant q, int warps, cudaStream_t s) {
    const int rows = warps == 1 ? kRowWarps : 1;
    const dim3 block(32, warps, rows);
    const unsigned grid = (unsigned)((a.n.rows + rows - 1) / rows);
    return mafat_launch_overlapped(q == MAFAT_NORM_PLAIN ? block_norm_kernel<T, V, N, MAFAT_NORM_PLAIN>
                                   : q == MAFAT_NORM_ROW ? block_norm_kernel<T, V, N, MAFAT_NORM_ROW>
                                                         : block_norm_kernel<T, V, N, MAFAT_NORM_BLOCK>,
                                   grid, block, 0, s, a);
}

// Accesses of a thread, twice as many until the row's warps hold it: all that it can have, or with `few` the fewest warps.
template <class T, int V, int N>
cudaError_t launch_v(const MafatBlockNormArgs& a, MafatNormQuant q, bool few, int most, cudaStream_t s) {
    const int per_warp = 32 * V * N;
    if constexpr (2 * N * V <= kMaxThread)
        if (a.n.cols > per_warp * (few && 2 * N * V <= most ? 1 : kMaxWarps)) return launch_v<T, V, 2 * N>(a, q, few, most, s);
    return launch<T, V, N>(a, q, (a.n.cols + per_warp - 1) / per_warp, s);
}
template <class T, int V, int N>
cudaError_t launch_rows(const MafatBlockNormArgs& a, MafatNormQuant q, cudaStream_t s) {
    const int most = q != MAFAT_NORM_BLOCK ? kMaxThread : V == 1 ? 8 : 16;  // channels of a thread
    constexpr int kLeast = 32 * V * N;
    const int64_t warps = (a.n.cols + 32 * most - 1) / (32 * most), held = (a.n.cols + kLeast - 1) / kLeast * kLeast;
    const bool few = a.n.rows >= kManyRows ||
                     (V * sizeof(T) == 16 && a.n.rows * warps >= kManyWarps && (warps == 1 || warps * 32 * most * 4 <= held * 5));
    return launch_v<T, V, N>(a, q, few, most, s);
}

}  // namespace

cudaError_t mafat_launch_block_norm(const MafatBlockNormArgs& a, bool bf16, int vec, MafatNormQuant quant, cudaStream_t s) {
    // A warp has 128 channels at least: 4 accesses of one, 2 of two.  20000 rows of 1004 bf16 26.6 us with accesses of four, of two
    // 28.1; to e4m3 by blocks 31.9, 37.3.
    if (bf16)
        return vec >= 8   ? launch_rows<__nv_bfloat16, 8, 1>(a, quant, s)
               : vec >= 4 ? launch_rows<__nv_bfloat16, 4, 1>(a, quant, s)
               : vec >= 2 ? launch_rows<__nv_bfloat16, 2, 2>(a, quant, s)
                          : launch_rows<__nv_bfloat16, 1, 4>(a, quant, s);
    return vec >= 4   ? launch_rows<float, 4, 1>(a, quant, s)
           : vec >= 2 ? launch_rows<float, 2, 2>(a, quant, s)
                      : launch_rows<float, 1, 4>(a, quant, s);
}
