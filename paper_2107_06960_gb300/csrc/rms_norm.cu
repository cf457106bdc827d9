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
#include "row_common.cuh"

namespace {

constexpr int kRowWarps = 4;   // rows of a block whose rows take one warp each
constexpr int kMaxWarps = 16;  // of a row
constexpr int kMaxThread = 32; // channels of a thread
constexpr int kFewRows = 2048;

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
    finish_row<T, V, N, Q>(a, row, c0, h, vw, inv, part[1], warps);
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
