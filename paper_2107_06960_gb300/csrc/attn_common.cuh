// What the attention kernels share: which rows and keys a CTA has, where its results go.
#pragma once
#include <math_constants.h>

#include "attention.h"

namespace mafat_attn {

// One item of work.  Row tiles of one part of the keys are neighbours, so that CTAs that run together
// read the same keys.
struct Block {
    int seq, head, split, row0;
    int len;         // readable keys of the sequence
    int key0, key1;  // its part of them: a run of whole tiles

    // Reads the sequence's length: after launch_begin.
    __device__ __forceinline__ Block(const MafatAttnArgs& a, uint32_t i, int tile_rows, int tile_keys) {
        const MafatAttnSeg& g = a.seg;
        uint32_t next = g.row_tiles_div.div(i);
        row0 = (int)(i - next * (uint32_t)g.row_tiles) * tile_rows;
        i = next;
        next = g.splits_div.div(i);
        split = (int)(i - next * (uint32_t)g.splits);
        i = next;
        next = a.heads_kv_div.div(i);
        head = (int)(i - next * (uint32_t)a.heads_kv);
        seq = (int)next;
        len = g.n;
        if (g.len) len = min(max(g.len[seq], 0), g.n);
        // the keys that some row of the tile sees
        int last = len;
        if (g.causal) {
            const int r1 = min(row0 + tile_rows, g.rows);
            // the latest token among the tile's rows
            const uint32_t u0 = a.group_div.div((uint32_t)row0), u1 = a.group_div.div((uint32_t)(r1 - 1));
            const uint32_t q0 = a.n_q_div.div(u0), q1 = a.n_q_div.div(u1);
            const int t = q0 != q1 ? a.n_q - 1 : (int)(u1 - q1 * (uint32_t)a.n_q);
            last = min(max(len - a.n_q + t + 1, 0), len);
        }
        const uint32_t tiles = ((uint32_t)last + (uint32_t)tile_keys - 1) / (uint32_t)tile_keys;
        // tiles * split / splits without 64 bits: whole tiles a split, and the rest's share
        const uint32_t each = g.splits_div.div(tiles), rest = tiles - each * (uint32_t)g.splits;
        const uint32_t s0 = (uint32_t)split, s1 = s0 + 1;
        key0 = (int)(each * s0 + g.splits_div.div(rest * s0)) * tile_keys;
        key1 = min((int)(each * s1 + g.splits_div.div(rest * s1)) * tile_keys, last);
    }
};

// Row r of a (sequence, key head): its request among all, token and query head.
struct Row {
    int64_t req;
    int t, h;
    __device__ __forceinline__ Row(const MafatAttnArgs& a, const Block& b, int r) {
        const uint32_t u = a.group_div.div((uint32_t)r), q = a.n_q_div.div(u);
        h = b.head * a.group + (r - (int)u * a.group);
        t = (int)u - (int)q * a.n_q;
        req = (int64_t)b.seq * a.seg.reqs + q;
    }
    __device__ __forceinline__ int64_t query(const MafatAttnArgs& a) const {
        return req * a.q_sb + (int64_t)t * a.q_st + (int64_t)h * a.q_sh;
    }
    // it sees the keys below this one
    __device__ __forceinline__ int limit(const MafatAttnArgs& a, const Block& b) const {
        return a.seg.causal ? min(max(b.len - a.n_q + t + 1, 0), b.len) : b.len;
    }
};

// Where a row's results go.
struct Out {
    int64_t o;     // element of out
    int64_t row;   // row among all
    int64_t part;  // row of the parts' arrays

    __device__ __forceinline__ Out(const MafatAttnArgs& a, const Block& b, const Row& r) {
        o = r.req * a.o_sb + (int64_t)r.t * a.o_st + (int64_t)r.h * a.o_sh;
        row = (r.req * a.n_q + r.t) * a.heads_q + r.h;
        part = (int64_t)(a.seg.part0 + b.split) * a.rows_total + row;
    }
};

// A launch may start while the one before it ends: it waits before it touches memory that others
// write, then lets the next one start.  One that follows a launch of its own run, whose results it does not
// use at first, waits for them before it joins them, or at its end, so that its own end means the end of both.
__device__ __forceinline__ void launch_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void launch_begin(const MafatAttnArgs& a) {
    if (!a.overlap) launch_wait();
    launch_next();
}
__device__ __forceinline__ void launch_end(const MafatAttnArgs& a) {
    if (a.overlap) launch_wait();
}

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
    if (!a.direct)
        a.part_lse[w.part] = lse2;
    else if (a.lse)
        a.lse[w.row] = lse2 * CUDART_LN2_F;
}

// How a row's result is joined with its parts of an earlier launch:
// out = own * O + sum_p 2^(lse_p - top) * inv * O_p.
struct Join {
    float top, own, inv;
    __device__ __forceinline__ Join(const MafatAttnArgs& a, const Out& w, float m, float l) {
        const float mine = l == 0.f ? -CUDART_INF_F : fmaf(m, a.scale_log2, log2f(l));
        top = mine;
        for (int p = 0; p < a.join; ++p) top = max_nan(top, a.part_lse[(int64_t)p * a.rows_total + w.row]);
        if (top == -CUDART_INF_F) top = 0.f;  // no readable key anywhere: all factors are zero
        const float x = exp2_fast(mine - top);
        float sum = x;
        for (int p = 0; p < a.join; ++p) sum += exp2_fast(a.part_lse[(int64_t)p * a.rows_total + w.row] - top);
        inv = inverse_sum(sum);
        own = l == 0.f ? 0.f : x * inv / l;
        lse2 = sum == 0.f ? -CUDART_INF_F : top + log2f(sum);
    }
    float lse2;
};

}  // namespace mafat_attn
