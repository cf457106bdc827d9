// What the attention kernels share: which rows and keys a CTA has, where its results go.
#pragma once
#include <cuda_bf16.h>
#include <math_constants.h>

#include "attention.h"

namespace mafat_attn {

__device__ __forceinline__ int length_of(const MafatAttnSeg& g, int seq) {
    return g.len ? min(max(g.len[seq], 0), g.n) : g.n;
}

// The j-th sequence and its length, as they are given.
struct AsGiven {
    const MafatAttnSeg& g;
    __device__ __forceinline__ int operator()(int j, int& len) const {
        len = length_of(g, j);
        return j;
    }
};

// One item of work.  Row tiles of one part of the keys are neighbours, so that CTAs that run together
// read the same keys.
struct Block {
    int seq, head, split, row0;
    int len;         // readable keys of the sequence
    int key0, key1;  // its part of them: a run of whole tiles

    // Reads the sequence's length: after launch_begin.
    __device__ __forceinline__ Block(const MafatAttnArgs& a, uint32_t i, int tile_rows, int tile_keys)
        : Block(a, i, tile_rows, tile_keys, AsGiven{a.seg}) {}
    template <class Seq>
    __device__ __forceinline__ Block(const MafatAttnArgs& a, uint32_t i, int tile_rows, int tile_keys, Seq seq_of)
        : Block(a, i, tile_rows) {
        seq = seq_of(seq, len);
        set_keys(a, tile_rows, tile_keys);
    }
    // The item alone, with its sequence as they are given; set_keys follows once len is there.
    __device__ __forceinline__ Block(const MafatAttnArgs& a, uint32_t i, int tile_rows) {
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
    }
    __device__ __forceinline__ void set_keys(const MafatAttnArgs& a, int tile_rows, int tile_keys) {
        const MafatAttnSeg& g = a.seg;
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

// The running maximum of a row is kept as `base`, its score times c = scale log2(e) in fp32, rounded once; weights are
// 2^(fma(s, c, -base)), and what was summed at another base is multiplied by 2^(base - new base), which is 1
// where it did not move.  (Making both from the score would be off by the product's rounding, a share of 2^-24 of the
// exponent in every tile, always the same way: 8e-6 of the result after some hundred tiles.)
// Before the first readable key base is -inf, and nothing is to be subtracted: 2^-inf = 0.
__device__ __forceinline__ float subtrahend(float base) { return base == -CUDART_INF_F ? 0.f : base; }

// The row's log2 of its sum of exponentials, -inf where no key is readable.
__device__ __forceinline__ float row_lse2(float base, float l) { return l == 0.f ? -CUDART_INF_F : base + log2f(l); }
__device__ __forceinline__ void store_lse(const MafatAttnArgs& a, const Out& w, float base, float l) {
    const float lse2 = row_lse2(base, l);
    if (!a.direct)
        a.part_lse[w.part] = lse2;
    else if (a.lse)
        a.lse[w.row] = lse2 * CUDART_LN2_F;
}

// How a row's result is joined with its parts of an earlier launch:
// out = own * O + sum_p 2^(lse_p - top) * inv * O_p.
struct Join {
    float top, own, inv;
    __device__ __forceinline__ Join(const MafatAttnArgs& a, const Out& w, float base, float l) {
        const float mine = row_lse2(base, l);
        top = mine;
#pragma unroll 4
        for (int p = 0; p < a.join; ++p) top = max_nan(top, a.part_lse[(int64_t)p * a.rows_total + w.row]);
        if (top == -CUDART_INF_F) top = 0.f;  // no readable key anywhere: all factors are zero
        const float x = exp2_fast(mine - top);
        float sum = x;
#pragma unroll 4
        for (int p = 0; p < a.join; ++p) sum += exp2_fast(a.part_lse[(int64_t)p * a.rows_total + w.row] - top);
        inv = inverse_sum(sum);
        own = l == 0.f ? 0.f : x * inv / l;
        lse2 = sum == 0.f ? -CUDART_INF_F : top + log2f(sum);
    }
    float lse2;
};

__device__ __forceinline__ void put4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void put4(__nv_bfloat16* p, float4 v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2*>(p) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// A warp joins the parts of a row: O = sum_i w_i O_i / sum_i w_i with w_i = 2^(lse_i - max lse).  A lane
// has four channels, of every WAYS-th part (2 where a row has 64 channels at most, else 1).  The weights are
// made first, a lane each, so that the loads of sixteen parts a lane are on their way together.  The order of the sums is
// fixed, so results do not change from run to run.  SETS: a row has 32 * SETS parts at most.
template <class T, int WAYS, int SETS>
__device__ __forceinline__ void join_row(const MafatAttnArgs& a, int64_t row) {
    constexpr int kLanes = 32 / WAYS, kUnroll = 16;
    const int lane = threadIdx.x % 32, way = lane / kLanes, d = lane % kLanes * 4;
    const bool in_dim = d < a.dim;
    float lse[SETS], top = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
        const int p = i * 32 + lane;
        lse[i] = p < a.parts ? __ldcg(a.part_lse + (int64_t)p * a.rows_total + row) : -CUDART_INF_F;
        top = max_nan(top, lse[i]);
    }
#pragma unroll
    for (int w = 1; w < 32; w *= 2) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, w));
    const float base = top == -CUDART_INF_F ? 0.f : top;
    float sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
        if (i * 32 >= a.parts) break;
        const float w = exp2_fast(lse[i] - base);
        sum += w;
        const int n = min(32, a.parts - i * 32);
        const float* src = a.part_o + ((int64_t)(i * 32) * a.rows_total + row) * a.dim + d;
#pragma unroll 1
        for (int p0 = 0; p0 < n; p0 += kUnroll * WAYS) {
            float4 v[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int p = p0 + u * WAYS + way;
                v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (p < n && in_dim)
                    v[u] = __ldcg(reinterpret_cast<const float4*>(src + (int64_t)p * a.rows_total * a.dim));
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const float x = __shfl_sync(0xffffffffu, w, (p0 + u * WAYS + way) & 31);  // past n: v is zero
                acc.x = fmaf(x, v[u].x, acc.x);
                acc.y = fmaf(x, v[u].y, acc.y);
                acc.z = fmaf(x, v[u].z, acc.z);
                acc.w = fmaf(x, v[u].w, acc.w);
            }
        }
    }
#pragma unroll
    for (int w = 1; w < 32; w *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    if (WAYS == 2) {
        acc.x += __shfl_xor_sync(0xffffffffu, acc.x, 16);
        acc.y += __shfl_xor_sync(0xffffffffu, acc.y, 16);
        acc.z += __shfl_xor_sync(0xffffffffu, acc.z, 16);
        acc.w += __shfl_xor_sync(0xffffffffu, acc.w, 16);
    }
    const float inv = inverse_sum(sum);
    const uint32_t u = a.heads_q_div.div((uint32_t)row), req = a.n_q_div.div(u);
    const int h = (int)((uint32_t)row - u * (uint32_t)a.heads_q), t = (int)(u - req * (uint32_t)a.n_q);
    if (way == 0 && in_dim)
        put4((T*)a.out + (int64_t)req * a.o_sb + (int64_t)t * a.o_st + (int64_t)h * a.o_sh + d,
             make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
    if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -CUDART_INF_F : (base + log2f(sum)) * CUDART_LN2_F;
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The place of shared memory p in the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t in_cluster(const void* p, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}

// Joins an item's parts among the CTAs of a cluster (2, 4 or 8, a part each): every CTA writes its rows, each normalised,
// and their log2 sums into the shared memory of the CTA that joins the row, every a.cluster-th of ROWS; that one finds
// all parts at home, and joins them in their order, a warp a row.  No launch, no trip through memory, and one way
// across the cluster (reading the others' parts took two, and a barrier more: 5.3 us against 5.1 for one token of 8
// heads over 1444 keys, 4.3 against 4.0 over 200).
constexpr int kMostCluster = 8;
template <int ROWS, int DP>
struct ClusterParts {
    static constexpr int kPitch = DP + 4;  // the sum stands behind the channels
    static constexpr int kBytes = (ROWS > kMostCluster ? ROWS : kMostCluster) * kPitch * 4;
    float* area;   // the same place in each CTA, which nothing else uses
    int cluster, shift, per;  // rows of a CTA
    uint32_t rank;
    __device__ __forceinline__ ClusterParts(const MafatAttnArgs& a, void* p) : area((float*)p), cluster(a.cluster) {
        shift = 31 - __clz(cluster);
        per = (ROWS + cluster - 1) >> shift;
        rank = cluster_rank();
    }
    // at the CTA's start; and before the first part is written, when all CTAs have to have started
    static __device__ __forceinline__ void start() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
    static __device__ __forceinline__ void started() { asm volatile("barrier.cluster.wait;" ::: "memory"); }
    __device__ __forceinline__ uint32_t place(int r, int d) const {
        return in_cluster(area + ((int)rank * per + (r >> shift)) * kPitch + d, (uint32_t)(r & (cluster - 1)));
    }
    __device__ __forceinline__ void put(int r, int d, float4 v) const {
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(place(r, d)), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
                     : "memory");
    }
    __device__ __forceinline__ void put_sum(int r, float lse2) const {
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(place(r, DP)), "f"(lse2) : "memory");
    }
    template <class T, int WARPS>
    __device__ __forceinline__ void join(const MafatAttnArgs& a, const Block& b, int rows) const {
        asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, d = lane * 4;
        for (int i = warp; (int)rank + (i << shift) < rows; i += WARPS) {
            float4 v[kMostCluster];
            float x[kMostCluster], top = -CUDART_INF_F;
#pragma unroll
            for (int p = 0; p < kMostCluster; ++p) {
                x[p] = -CUDART_INF_F;
                v[p] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (p < cluster) {
                    const float* part = area + (p * per + i) * kPitch;
                    x[p] = part[DP];
                    if (d < a.dim) v[p] = *reinterpret_cast<const float4*>(part + d);
                }
            }
#pragma unroll
            for (int p = 0; p < kMostCluster; ++p) top = max_nan(top, x[p]);
            const float base = subtrahend(top);
            float sum = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int p = 0; p < kMostCluster; ++p) {
                const float w = exp2_fast(x[p] - base);
                sum += w;
                acc = make_float4(fmaf(w, v[p].x, acc.x), fmaf(w, v[p].y, acc.y), fmaf(w, v[p].z, acc.z), fmaf(w, v[p].w, acc.w));
            }
            const float inv = inverse_sum(sum);
            const Out out(a, b, Row(a, b, b.row0 + (int)rank + (i << shift)));
            if (d < a.dim) put4((T*)a.out + out.o + d, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
            if (lane == 0 && a.lse) a.lse[out.row] = row_lse2(base, sum) * CUDART_LN2_F;
        }
    }
};

}  // namespace mafat_attn
