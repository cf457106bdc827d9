// Launch interface of the operators of a decoding step beside attention and norms: rotary positions and
// adjusted logits (host and device visible).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "attention.h"

// One of a call's tensors and where it goes; strides in elements: sequence, token or place, head.
struct MafatRotaryTensor {
    const void* in;
    void* out;
    int64_t in_sb, in_st, in_sh;
    int64_t out_sb, out_st, out_sh;
    int32_t heads;              // 0: not given
};

struct MafatRotaryArgs {
    MafatRotaryTensor t[3];     // queries; keys and values, which go to the tokens' places
    const uint64_t* turns;      // [rot / 2] fractions of a turn a position, times 2^64
    const int32_t* positions;   // [tokens]
    const int32_t* places;      // [tokens] (null: each token's own)
    int64_t tokens;
    MafatDiv n_q_div;
    int32_t n_q, room;
    int32_t dim, rot;
    float magnitude;
    // set by the launch: items of a head (pairs, then channels that stay), tokens of a CTA, heads that it has at a time
    int32_t pairs, lanes, per_block, steps;
    MafatDiv lanes_div, steps_div, half_div;
};
int mafat_rotary_most_dim();
cudaError_t mafat_launch_rotary(MafatRotaryArgs& a, bool bf16, bool interleaved, cudaStream_t s);

struct MafatLogitsArgs {
    const void* logits;
    void* out;
    int64_t in_s, out_s;        // of rows, in elements
    const int32_t* tokens;      // [batch][room] (null: none)
    const int32_t* lengths;     // null: room
    const int32_t* prompt;      // null: 0
    const float *repetition, *presence, *frequency;
    const int32_t* drafts;      // [batch][n_q] (null: none)
    const uint32_t* tree;       // null: a chain
    int64_t tree_s;             // words of a request (0: all share one tree)
    const int32_t* bias_ids;
    const float* bias;
    int64_t bias_s;             // entries of a request (0: all share them)
    const uint32_t* masks;
    const int32_t* mask_rows;
    // set by the launch: runs of the vocabulary, groups of a request's rows; rows of a group
    MafatDiv items_div, groups_div;
    int32_t rows_of_cta;
    int32_t pass;               // 0: out is logits and nothing is masked: only what is noted is written
    int32_t n_q, vocab, room, n_bias, n_masks, tree_words, mask_words;
};
cudaError_t mafat_launch_logits(MafatLogitsArgs& a, bool bf16, bool out_bf16, int64_t batch, cudaStream_t s);
int mafat_logits_run();  // tokens of a row that a CTA has at least
