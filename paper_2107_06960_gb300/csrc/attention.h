// Launch interface of the language operators: attention to one or two sets of keys, the join of
// its parts, and the root-mean-square norm (host and device visible).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

// Division by a number known at launch, for dividends below 2^31: a product and a shift (Granlund
// and Montgomery, "Division by invariant integers using multiplication", 1994).
struct MafatDiv {
    uint32_t d = 1, mul = 1, shift = 0;
    __host__ __device__ MafatDiv() {}
    explicit MafatDiv(uint32_t n) : d(n) {
        while (shift < 32 && (1ull << shift) < n) ++shift;
        mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - n)) / n + 1);
    }
    __device__ __forceinline__ uint32_t div(uint32_t x) const {
#ifdef __CUDA_ARCH__
        return (__umulhi(x, mul) + x) >> shift;
#else
        return x / d;
#endif
    }
};

// One set of keys and values: n_seq sequences, each read by the n_q queries of `reqs` requests.
// The rows of a (sequence, key head) are its queries, row = (request * n_q + token) * group + head.
// A CTA takes one tile of rows and one of `splits` parts of the readable keys.
struct MafatAttnSeg {
    const void* k;
    const void* v;
    int64_t k_sb, k_ss, k_sh;   // strides in elements: sequence, key, head (the channels are contiguous)
    int64_t v_sb, v_ss, v_sh;
    const int32_t* len;         // [n_seq] readable keys (null: n)
    const uint8_t* mask;        // [n_seq][n] 0: the key is not readable (null: all are)
    int32_t n;                  // keys that a sequence has room for
    int32_t causal;             // 1: token t of n_q sees keys 0 .. len - n_q + t
    int32_t reqs;
    int32_t n_seq;
    int32_t rows;               // reqs * n_q * group
    int32_t row_tiles;
    int32_t splits;
    MafatDiv row_tiles_div, splits_div;
    int32_t part0;              // first of its splits among the parts of a row
    int32_t items;              // n_seq * heads_kv * splits * row_tiles
};

constexpr int kMafatMostOrdered = 128;

struct MafatAttnArgs {
    const void* q;
    void* out;
    float* lse;                 // [batch][n_q][heads_q] natural logarithm (null: not wanted)
    int64_t q_sb, q_st, q_sh;
    int64_t o_sb, o_st, o_sh;
    int32_t n_q, group, heads_q, heads_kv, dim;
    MafatDiv n_q_div, group_div, heads_q_div, heads_kv_div;
    int32_t parts;              // parts of a row, over all segments
    // 1: the CTA that has the row writes its result, joined with the `join` parts of an earlier launch; 0: it writes a part
    int32_t direct, join;
    // more than 1: the CTAs with a row's parts are a cluster of this many, and join them among themselves
    int32_t cluster;
    int32_t ordered;            // 1: attn_rows takes the longest of the n_seq sequences (at most kMafatMostOrdered) first
    float scale_log2;           // softmax scale times log2(e)
    float* part_o;              // [parts][rows_total][dim] results of the parts, each normalised
    float* part_lse;            // [parts][rows_total] their log2 of the sum of exponentials
    int64_t rows_total;         // batch * n_q * heads_q, row index = (request * n_q + token) * heads_q + head
    // 1: an earlier launch of the same run, which has waited for what came before, is all that this one
    // follows: it waits for its results, or at its end for those that join both
    int32_t overlap;
    uint32_t* status;           // [2] status and abort words, as the plans' counter block starts
    int64_t timeout_ns;
    MafatAttnSeg seg;
};

// fp32 on the CUDA cores, tiles of 4, 8 or 64 rows.
cudaError_t mafat_launch_attn_simt(const MafatAttnArgs& a, int rows, cudaStream_t s);
cudaError_t mafat_prepare_attn_simt();
int mafat_attn_simt_keys();

// bf16, tiles of 16 rows by runs of 64 keys, ctas CTAs that take one item after another.
cudaError_t mafat_launch_attn_rows(const MafatAttnArgs& a, int ctas, cudaStream_t s);
cudaError_t mafat_prepare_attn_rows();
int mafat_attn_rows_keys();
int mafat_attn_rows_join();  // most parts of an earlier launch that it joins

// bf16 on the tensor cores: tiles of 128 * slots rows (slots 1 or 2) by 128 keys.  The maps are 4-D over {channel, head,
// key, sequence}, boxes of 64 channels x 128 keys, 128-byte swizzle.
// prefix: null, or keys that come before the segment's own and that `per` of its sequences after another share.
struct MafatAttnPrefix {
    CUtensorMap k, v;
    const int32_t* len;         // of each prefix (null: n)
    int32_t n;
    MafatDiv per;
};
cudaError_t mafat_launch_attn_tc(const MafatAttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int slots,
                                 const MafatAttnPrefix* prefix, cudaStream_t s);
cudaError_t mafat_prepare_attn_tc();

// Joins the parts of each row.
cudaError_t mafat_launch_attn_join(const MafatAttnArgs& a, bool bf16, cudaStream_t s);

struct MafatNormArgs {
    const void* x;
    const void* residual;       // null: none
    const void* weight;         // [cols]
    void* residual_out;         // x + residual (null: not wanted)
    void* y;
    float* scales;              // [rows][groups]
    int64_t rows;
    int64_t x_s, r_s, ro_s, y_s;  // row strides in elements
    int32_t cols;
    int32_t groups;             // scales of a row
    float eps;
};
// Launches fn with programmatic stream serialisation: it may start while the launch before it ends,
// and waits (griddepcontrol.wait) before it touches memory.
// Clusters of `cluster` CTAs along x.
template <class... P, class... A>
cudaError_t mafat_launch_clusters(int cluster, void (*fn)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s,
                                  const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, fn, P(args)...);
}
template <class... P, class... A>
cudaError_t mafat_launch_overlapped(void (*fn)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, const A&... args) {
    return mafat_launch_clusters(1, fn, grid, block, smem, s, args...);
}

enum MafatNormQuant { MAFAT_NORM_PLAIN = 0, MAFAT_NORM_ROW = 1, MAFAT_NORM_BLOCK = 2 };

int mafat_norm_max_cols();  // of a row
// vec: a power of two that divides cols and every matrix's row stride: the rows can be accessed by as many channels
cudaError_t mafat_launch_norm(const MafatNormArgs& a, bool bf16, int vec, MafatNormQuant quant, cudaStream_t s);
