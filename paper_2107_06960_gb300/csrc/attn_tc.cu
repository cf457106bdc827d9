// Attention of many rows in bf16 on the tensor cores: the forms without trees (apart from those with, so that both compile at once).
#include "attn_tc.cuh"

cudaError_t mafat_launch_attn_tc(const MafatAttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int slots,
                                 const MafatAttnPrefix* prefix, cudaStream_t s) {
    return a.tree ? mafat_launch_attn_tc_tree(a, k, v, slots, prefix, s) : launch_tc<false>(a, k, v, slots, prefix, s);
}

cudaError_t mafat_prepare_attn_tc(bool tree, int dim) { return tree ? mafat_prepare_attn_tc_tree(dim) : prepare_tc<false>(dim); }
