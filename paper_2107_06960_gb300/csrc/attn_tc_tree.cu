// Attention of many rows in bf16 on the tensor cores: the forms whose rows are nodes of trees.
#include "attn_tc.cuh"

cudaError_t mafat_launch_attn_tc_tree(const MafatAttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int slots,
                                      const MafatAttnPrefix* prefix, cudaStream_t s) {
    return launch_tc<true>(a, k, v, slots, prefix, s);
}

cudaError_t mafat_prepare_attn_tc_tree(int dim) { return prepare_tc<true>(dim); }
