// What the attention kernels share: which rows and keys a CTA has, where its results go.
#pragma once
#include <math_constants.h>

#include "attention.h"

namespace mafat_attn {

// The work of one CTA.  Row tiles of one part of the keys are neighbours in the grid, so that CTAs
// that run together read the same keys.
struct Block {
    int seg, seq, head, split, row0;
    int len;         // readable keys of the sequence
    int key0, key1;  // its part of them: a run of whole tiles

    __device__ __forceinline__ Block(const MafatAttnArgs& a, int tile_rows, int tile_keys) {
        int i = (int)blockIdx.x;
        seg = 0;
        if (i >= a.seg[0].blocks) {
            i -= a.seg[0].blocks;
            seg = 1;
        }
        const MafatAttnSeg& g = a.seg[seg];
        row0 = (i % g.row_tiles) * tile_rows;
        i /= g.row_tiles;
        split = i % g.splits;
        i /= g.splits;
        head = i % a.heads_kv;
        seq = i / a.heads_kv;
        len = g.n;
        if (g.len) len = min(max(g.len[seq], 0), g.n);
        // the keys that some row of the tile sees
        int last = len;
        if (g.causal) {
            const int r1 = min(row0 + tile_rows, g.rows);
            const int per = a.n_q * a.group;  // rows of a request
            // the latest token among the tile's rows
            const int t = (row0 / per != (r1 - 1) / per) ? a.n_q - 1 : (r1 - 1) % per / a.group;
            last = min(max(len - a.n_q + t + 1, 0), len);
        }
        const int64_t tiles = (last + tile_keys - 1) / tile_keys;
        key0 = (int)(tiles * split / g.splits) * tile_keys;
        key1 = min((int)(tiles * (split + 1) / g.splits) * tile_keys, last);
    }
};

// Where row r of the CTA's (sequence, key head) has its query.
__device__ __forceinline__ int64_t q_offset(const MafatAttnArgs& a, const MafatAttnSeg& g, const Block& b, int r) {
    const int h = r % a.group, u = r / a.group, t = u % a.n_q;
    const int64_t req = (int64_t)b.seq * g.reqs + u / a.n_q;
    return req * a.q_sb + (int64_t)t * a.q_st + (int64_t)(b.head * a.group + h) * a.q_sh;
}

// Row r sees the keys below this one.
__device__ __forceinline__ int row_limit(const MafatAttnArgs& a, const MafatAttnSeg& g, const Block& b, int r) {
    if (!g.causal) return b.len;
    const int t = r / a.group % a.n_q;
    return min(max(b.len - a.n_q + t + 1, 0), b.len);
}

// Where row r's results go.
struct Out {
    int64_t o;     // element of out
    int64_t row;   // row among all
    int64_t part;  // row of the parts' arrays

    __device__ __forceinline__ Out(const MafatAttnArgs& a, const MafatAttnSeg& g, const Block& b, int r) {
        const int h = b.head * a.group + r % a.group, u = r / a.group, t = u % a.n_q;
        const int64_t req = (int64_t)b.seq * g.reqs + u / a.n_q;
        o = req * a.o_sb + (int64_t)t * a.o_st + (int64_t)h * a.o_sh;
        row = (req * a.n_q + t) * a.heads_q + h;
        part = (int64_t)(g.part0 + b.split) * a.rows_total + row;
    }
};

// Maximum that keeps a NaN, so that a NaN score reaches the result.
__device__ __forceinline__ float max_nan(float x, float y) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
    return r;
}

// 2^x by the special function unit (2 ulp; results below the normal range become zero, as a
// share of a sum that is at least one).
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// 1 / sum, and 0 for a row that no key is readable for: its result is zero.
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.f ? 0.f : 1.f / l; }

// The row's log2 of its sum of exponentials, -inf where no key is readable.
__device__ __forceinline__ void store_lse(const MafatAttnArgs& a, const Out& w, float m, float l) {
    const float lse2 = l == 0.f ? -CUDART_INF_F : fmaf(m, a.scale_log2, log2f(l));
    if (a.parts > 1)
        a.part_lse[w.part] = lse2;
    else if (a.lse)
        a.lse[w.row] = lse2 * CUDART_LN2_F;
}

}  // namespace mafat_attn
