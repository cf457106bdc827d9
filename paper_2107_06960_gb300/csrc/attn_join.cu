// Joins the parts of each row, a warp a row, where the CTAs that made them leave that to a launch of its own.
//
// With the parts' results O_p, each normalised, and their log2 sums z_p:  O = sum_p 2^(z_p - z) O_p / sum_p 2^(z_p - z),
// z = max z_p: three fp32 operations for 4 bytes read.  Bound by the round trips of its loads for few rows (a warp a row
// has the loads of 16 or 32 parts on their way together, 1.6 us a round), by the parts' bytes (in L2, just written) for
// many: 8192 rows of 128 channels add 13 us with 2 parts and 26 with 8, 1.3 to 2.6 TB/s there and back.
#include "attn_common.cuh"

namespace {

constexpr int kWarps = 4;

template <class T, int WAYS>
__global__ void __launch_bounds__(kWarps * 32) attn_join_kernel(const __grid_constant__ MafatAttnArgs a) {
    mafat_attn::launch_begin(a);
    const int64_t row = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    // at most MAFAT_ATTN_MAX_SPLITS parts of each of two sets of keys
    if (row < a.rows_total) mafat_attn::join_row<T, WAYS, 8>(a, row);
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
