// Attention of few rows in bf16: the queries of a single token (or of a few), up to 16 rows of one
// (sequence, key head).
//
// Bound by reading K and V once: 16 rows give each 16-byte vector 16 x 16 operations, far from
// what the tensor core could do, so the work is to keep copies in flight.  A warp has every fourth run of 16
// keys of an item's part, a ring of kStages runs of its own in shared memory (cp.async, no barrier between
// warps) and its own running maximum, sum and O; the four are joined once, at the item's end.  A CTA
// takes one item after another, and its copies run ahead into the next one: without that every item began with an empty
// ring.  The products are the 16 x 8 x 16 ones of a single warp, whose operands are registers: S's
// accumulators are P's operand as they are.  P is rounded to bf16 for its product; all else is fp32.
//
// Items of the longest sequences are taken first, and a CTA's next from the other end of the order: 64 sequences of half
// to all of 1444 keys (one token, 32 query and 8 key heads) take 48 us, as they are given 54, 128 channels; 29 and
// 31.5 with 64.  (In the kernels whose CTAs have one item each, finding its sequence cost what it brought.)
//
// Keys that are not readable are not copied but filled with zeros, so that 0 x NaN cannot reach O.
//
// One token of 64 sequences, 32 query and 8 key heads, 1444 keys: 59 us or 6.4 TB/s with 128 channels, 34 us or 5.5 TB/s
// with 64; under 40 % of the issue slots are taken.  One token of one sequence (8 query and 4 key heads, 1444 keys) is
// bound by round trips: 5.1 us in 4 clusters of 8 CTAs, 5.8 with a launch that joins the parts.
//
// Trees: the bits of a row are looked at in the runs that have nodes' keys, the first word read ahead.  Where there is little to do
// a cluster splits the keys of both sets, the prefix's and the request's own, as if they were one: a tree of 8 nodes over 1444
// + 96 keys (16 query and 4 key heads of 64 channels) 7.0 us, in two launches 7.5.
#include <type_traits>

#include "attn_common.cuh"

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kRun = 16;                // keys of a warp at a time
constexpr int kBN = kWarps * kRun;
constexpr int kMostJoin = 32;           // parts of the launch before

template <int DP, bool CLUSTER>
struct Cfg {
    static constexpr int kStages = DP == 128 ? 2 : 4;
    static constexpr int kMatrix = kRun * DP * 2;       // bytes of a run of K or V
    static constexpr int kRing = kStages * 2 * kMatrix;  // of a warp
    static constexpr int kOffQ = kWarps * kRing;         // queries of this item and of the next
    static constexpr int kQ = 16 * DP * 2;
    // in a cluster there is no next item: the others' parts of rows come to where its queries would be, and beyond
    static constexpr int kOffParts = kOffQ + kQ, kParts = mafat_attn::ClusterParts<16, DP>::kBytes;
    static constexpr int kOffJoin = kOffQ + (CLUSTER ? kQ + kParts : 2 * kQ);
    static constexpr int kPitch = DP + 4;                // floats of a row of O while the warps are joined
    static constexpr int kSmem = kOffJoin + kWarps * 16 * (kPitch + 2) * 4;
    static_assert(kSmem + 1024 <= 115712, "two CTAs on an SM, with the order's table");
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// also for those that are in no group yet
__device__ __forceinline__ void wait_all_copies() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldm4_t(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// The CTA's items: one of every round of gridDim.x, from one end of a round and from the other in turn, so that with the
// longest sequences first each has long ones and short ones.
struct Items {
    uint32_t item, edge;
    __device__ __forceinline__ Items() : item(blockIdx.x), edge(2 * gridDim.x - 1) {}
    __device__ __forceinline__ uint32_t next() const { return edge - item; }
    __device__ __forceinline__ void step() {
        item = edge - item;
        edge += 2 * gridDim.x;
    }
};
// The j-th sequence and its length; with a table of them the j-th longest.
struct Table {
    const MafatAttnSeg& g;
    const int2* order;  // null: as they are given
    __device__ __forceinline__ int operator()(int j, int& len) const {
        const int2 x = order ? order[j] : make_int2(j, mafat_attn::length_of(g, j));
        len = x.y;
        return x.x;
    }
};
// Fills the table, longest first, by counting for each sequence those before it: a ballot of each 32, for kTogether
// sequences of a warp at a time.
__device__ __forceinline__ void order_sequences(const MafatAttnSeg& g, int2* order) {
    constexpr int kSets = kMafatMostOrdered / 32, kTogether = 4, kStep = kTogether * kWarps;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int len[kSets];
#pragma unroll
    for (int i = 0; i < kSets; ++i) len[i] = i * 32 + lane < g.n_seq ? mafat_attn::length_of(g, i * 32 + lane) : -1;
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
        const int n = min(32, g.n_seq - i * 32);
#pragma unroll 1
        for (int s0 = warp; s0 < n; s0 += kStep) {
            int mine[kTogether], place[kTogether];
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
                mine[k] = __shfl_sync(0xffffffffu, len[i], (s0 + k * kWarps) & 31);
                place[k] = 0;
            }
#pragma unroll
            for (int u = 0; u < kSets; ++u)
                if (u * 32 < g.n_seq)
#pragma unroll
                    for (int k = 0; k < kTogether; ++k)
                        place[k] += __popc(__ballot_sync(
                            0xffffffffu, len[u] > mine[k] || (len[u] == mine[k] && u * 32 + lane < i * 32 + s0 + k * kWarps)));
#pragma unroll
            for (int k = 0; k < kTogether; ++k)
                if (lane == 0 && s0 + k * kWarps < n) order[place[k]] = make_int2(i * 32 + s0 + k * kWarps, mine[k]);
        }
    }
    __syncthreads();
}

struct NoPrefix {};

// Keys of two sets as one: first the prefix's tiles, of which the last may be partly empty, then the own keys.
template <class Prefix>
struct Sets {
    static constexpr bool kBoth = std::is_same<Prefix, MafatRowsPrefix>::value;
    int seq, len0, own0;  // of the prefix: which, readable keys; where own keys begin
    __device__ __forceinline__ Sets() : seq(0), len0(0), own0(0) {}
    // the item's keys, a run of whole tiles of both sets' (splits: the cluster's CTAs, or 1: all of them)
    __device__ __forceinline__ Sets(const MafatAttnArgs& a, mafat_attn::Block& b, const Prefix& prefix) : Sets() {
        if constexpr (kBoth) {
            seq = (int)prefix.per.div((uint32_t)b.seq);
            len0 = prefix.len ? min(max(prefix.len[seq], 0), prefix.n) : prefix.n;
            own0 = (len0 + kBN - 1) / kBN * kBN;
            const uint32_t tiles = (uint32_t)(own0 + b.len + kBN - 1) / kBN, s = (uint32_t)b.split;
            b.key0 = (int)a.seg.splits_div.div(tiles * s) * kBN;
            b.key1 = min((int)a.seg.splits_div.div(tiles * (s + 1u)) * kBN, own0 + b.len);
        }
    }
    __device__ __forceinline__ bool of_prefix(int key) const { return kBoth && key < own0; }
    // The item of a CTA: a cluster's are the parts of one tile of rows, which are not neighbours where there are more tiles.
    static __device__ __forceinline__ uint32_t item(const MafatAttnArgs& a, uint32_t i) {
        if constexpr (!kBoth) return i;
        const MafatAttnSeg& g = a.seg;
        const uint32_t tile = g.splits_div.div(i), pair = g.row_tiles_div.div(tile);
        return (pair * (uint32_t)g.splits + i - tile * (uint32_t)g.splits) * (uint32_t)g.row_tiles + tile - pair * (uint32_t)g.row_tiles;
    }
};

// The copying side's place: a run of an item.
struct Ahead : Items {
    int run, runs, first, len, head;
    const __nv_bfloat16 *k, *v;
    const uint8_t* mask;

    template <bool TREE, class Prefix>
    __device__ __forceinline__ void open(const MafatAttnArgs& a, int warp, Table table, const Prefix& prefix, Sets<Prefix>& sets) {
        run = runs = 0;
        if (item >= (uint32_t)a.seg.items) return;
        const MafatAttnSeg& g = a.seg;
        mafat_attn::Block b(a, Sets<Prefix>::item(a, item), 16, kBN, table);
        sets = Sets<Prefix>(a, b, prefix);
        mafat_attn::leave_dead<TREE>(a, b);
        first = b.key0 + warp * kRun;
        runs = b.key1 > first ? (b.key1 - first + kBN - 1) / kBN : 0;
        len = b.len;
        head = b.head;
        k = (const __nv_bfloat16*)g.k + (int64_t)b.seq * g.k_sb + (int64_t)b.head * g.k_sh;
        v = (const __nv_bfloat16*)g.v + (int64_t)b.seq * g.v_sb + (int64_t)b.head * g.v_sh;
        mask = g.mask ? g.mask + (int64_t)b.seq * g.n : nullptr;
    }
};

// CLUSTER: a cluster's CTAs have an item's parts and join them (an instance of its own: in one kernel it cost the
// other form's inner loop 20 %).  TREE: queries are nodes of trees, whose bits are looked at in runs that have such keys.
// Prefix: MafatRowsPrefix where both sets of keys are read as one.
template <int DP, bool CLUSTER, bool TREE, class Prefix>
__global__ void __launch_bounds__(kThreads) attn_rows_kernel(const __grid_constant__ MafatAttnArgs a, const __grid_constant__ Prefix prefix) {
    constexpr bool kBoth = Sets<Prefix>::kBoth;
    using C = Cfg<DP, CLUSTER>;
    using Parts = mafat_attn::ClusterParts<16, DP>;
    constexpr int kChunks = DP / 8;        // 16-byte chunks of a row
    constexpr int kRows = 32 / kChunks;    // rows of one access of a warp
    constexpr int kSteps = DP / 16;
    extern __shared__ __align__(128) uint8_t sm[];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const MafatAttnSeg& g = a.seg;
    const uint32_t smem = (uint32_t)__cvta_generic_to_shared(sm), ring = smem + warp * C::kRing;
    const int cc = lane % kChunks, cr = lane / kChunks;
    const bool in_dim = cc * 8 < a.dim;
    if constexpr (CLUSTER) Parts::start();
    mafat_attn::launch_begin(a);

    __shared__ int2 order[kMafatMostOrdered];
    const Table table{g, a.ordered ? order : nullptr};
    if (a.ordered) order_sequences(g, order);

    // the next run into its stage: chunk c of key r at chunk c ^ (r % 8) of its row; empty past the last item
    Ahead ld;
    Sets<Prefix> sets;
    ld.open<TREE>(a, warp, table, prefix, sets);
    uint32_t ld_stage = 0u, stage = 0u;
    auto load = [&]() {
        while (ld.run == ld.runs && ld.item < (uint32_t)g.items) {
            ld.step();
            ld.open<TREE>(a, warp, table, prefix, sets);
        }
        if (ld.run < ld.runs) {
            int key = ld.first + ld.run * kBN, len = ld.len;
            const uint32_t st = ring + ld_stage * (2 * C::kMatrix);
            const __nv_bfloat16 *k_from = ld.k, *v_from = ld.v;
            int64_t k_step = g.k_ss, v_step = g.v_ss;
            if constexpr (kBoth) {
                if (sets.of_prefix(key)) {
                    k_from = (const __nv_bfloat16*)prefix.k + (int64_t)sets.seq * prefix.k_sb + (int64_t)ld.head * prefix.k_sh;
                    v_from = (const __nv_bfloat16*)prefix.v + (int64_t)sets.seq * prefix.v_sb + (int64_t)ld.head * prefix.v_sh;
                    k_step = prefix.k_ss;
                    v_step = prefix.v_ss;
                    len = sets.len0;
                } else {
                    key -= sets.own0;
                }
            }
#pragma unroll
            for (int r0 = 0; r0 < kRun; r0 += kRows) {
                const int r = r0 + cr, k = key + r;
                const bool on = in_dim && k < len && (!ld.mask || ld.mask[k] != 0);
                const uint32_t at = st + (uint32_t)(r * (DP * 2) + ((cc ^ (r % 8)) * 16));
                // a place that is not read still gets an address inside the tensor
                const int64_t kk = on ? k : 0;
                copy16(at, k_from + (on ? kk * k_step + cc * 8 : 0), on);
                copy16(at + C::kMatrix, v_from + (on ? kk * v_step + cc * 8 : 0), on);
            }
            ++ld.run;
            if (++ld_stage == (uint32_t)C::kStages) ld_stage = 0u;
        }
        copies_done();
    };
    // a warp's share of an item's queries, rows past the last zero
    auto load_queries = [&](uint32_t item, uint32_t which) {
        if (item < (uint32_t)g.items) {
            const mafat_attn::Block b(a, Sets<Prefix>::item(a, item), 16, kBN, table);
#pragma unroll
            for (int r0 = 0; r0 < 16 / kWarps; r0 += kRows) {
                const int r = warp * (16 / kWarps) + r0 + cr, row = min(b.row0 + r, g.rows - 1);
                const bool on = in_dim && b.row0 + r < g.rows;
                const int64_t off = mafat_attn::Row(a, b, row).query(a);
                copy16(smem + C::kOffQ + which * C::kQ + (uint32_t)(r * (DP * 2) + ((cc ^ (r % 8)) * 16)),
                       (const __nv_bfloat16*)a.q + off + (on ? cc * 8 : 0), on);
            }
        }
    };
    load_queries(blockIdx.x, 0u);
#pragma unroll
    for (int i = 0; i < C::kStages - 1; ++i) load();
    bool waited = !a.overlap;  // for the launch whose parts are joined

    // ldmatrix addresses: lane 8i + j gives row j of matrix i
    const int mi = lane / 8, mj = lane % 8;
    const int k_row = (mi / 2) * 8 + mj, k_chunk = mi % 2;   // K: keys 0-7 and 8-15, each with channels 0-7 and 8-15
    const int v_row = (mi % 2) * 8 + mj, v_chunk = mi / 2;   // V: channels 0-7 and 8-15, each with keys 0-7 and 8-15
    float* so = (float*)(sm + C::kOffJoin);
    float* sml = so + kWarps * 16 * C::kPitch;
    const Parts parts(a, sm + C::kOffParts);

    uint32_t which = 0u;
#pragma unroll 1
    for (Items it; it.item < (uint32_t)g.items; it.step(), which ^= 1u) {
        mafat_attn::Block b(a, Sets<Prefix>::item(a, it.item), 16, kBN, table);
        const Sets<Prefix> now(a, b, prefix);  // the copies may be at the next item's
        mafat_attn::leave_dead<TREE>(a, b);
        const uint8_t* mask = g.mask ? g.mask + (int64_t)b.seq * g.n : nullptr;
        const int first = b.key0 + warp * kRun;
        const int runs = b.key1 > first ? (b.key1 - first + kBN - 1) / kBN : 0;
        // this item's queries are there (each warp's share), and the item before is joined.  Their copies are in the
        // group of the run after them; a warp that had no run in the item before has closed no group since.
        wait_all_copies();
        __syncthreads();
        uint32_t q[kSteps][4];
#pragma unroll
        for (int t = 0; t < kSteps; ++t)  // rows 0-7 and 8-15 with channels 0-7, then with 8-15
            ldm4(q[t], smem + C::kOffQ + which * C::kQ + (uint32_t)(v_row * (DP * 2) + (((2 * t + v_chunk) ^ (v_row % 8)) * 16)));
        load_queries(it.next(), which ^ 1u);  // lands with the next run
        int limit[2];
        mafat_attn::WayAhead way[2];
        const int first_node = TREE ? mafat_attn::tree_first(a, b) : 0x7fffffff;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = b.row0 + lane / 4 + 8 * h;
            limit[h] = 0x7fffffff;
            if (!TREE || r < g.rows) {
                const mafat_attn::Row row(a, b, r);
                if (r < g.rows) limit[h] = mafat_attn::limit_of<TREE>(a, b, row);
                if (kBoth && r < g.rows) limit[h] = mafat_attn::live<TREE>(a, row) ? 0x7fffffff : 0;  // the length bounds them
                if (TREE && g.tree) way[h] = mafat_attn::WayAhead(a, b, row);
            }
        }
        float base[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};
        float o[DP / 8][4];
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] = 0.f;

#pragma unroll 1
        for (int i = 0; i < runs; ++i) {
            load();
            wait_copies<C::kStages - 1>();
            __syncwarp();
            int key = first + i * kBN, len = b.len;
            bool own = true;  // the request's keys
            if constexpr (kBoth) {
                own = !now.of_prefix(key);
                if (own)
                    key -= now.own0;
                else
                    len = now.len0;
            }
            const uint32_t st = ring + stage * (2 * C::kMatrix);
            if (++stage == (uint32_t)C::kStages) stage = 0u;
            float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                uint32_t f[4];
                ldm4(f, st + (uint32_t)(k_row * (DP * 2) + (((2 * t + k_chunk) ^ (k_row % 8)) * 16)));
                mma(s[0], q[t], f[0], f[1]);
                mma(s[1], q[t], f[2], f[3]);
            }
            // of two sets a row sees either's keys, or none
            const int most[2] = {kBoth ? min(limit[0], len) : limit[0], kBoth ? min(limit[1], len) : limit[1]};
            if (mask || key + kRun > most[0] || key + kRun > most[1]) {
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int k = key + n * 8 + (lane % 4) * 2 + e % 2;
                        if (k >= len || k >= most[e / 2] || (mask && mask[k] == 0)) s[n][e] = -CUDART_INF_F;
                    }
            }
            if (TREE && own && key + kRun > first_node) {
                uint32_t held[2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    held[h] = way[h].bits ? way[h].from(key, first_node, g.tree_words) >> (lane % 4 * 2) : 0xffffffffu;
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if ((held[e / 2] >> (n * 8 + e % 2) & 1u) == 0u) s[n][e] = -CUDART_INF_F;
            }
            float keep[2], off[2];
            bool up = false;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float top = mafat_attn::max_nan(mafat_attn::max_nan(s[0][2 * h], s[0][2 * h + 1]),
                                                mafat_attn::max_nan(s[1][2 * h], s[1][2 * h + 1]));
                top = mafat_attn::max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = mafat_attn::max_nan(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const float next = mafat_attn::max_nan(base[h], top * a.scale_log2);
                up = up || next != base[h];
                off[h] = -mafat_attn::subtrahend(next);
                keep[h] = mafat_attn::exp2_fast(base[h] + off[h]);
                base[h] = next;
            }
            if (__any_sync(0xffffffffu, up)) {
#pragma unroll
                for (int h = 0; h < 2; ++h) l[h] *= keep[h];
#pragma unroll
                for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[n][e] *= keep[e / 2];
            }
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[n][e] = mafat_attn::exp2_fast(fmaf(s[n][e], a.scale_log2, off[e / 2]));
                    l[e / 2] += s[n][e];
                }
            const uint32_t p[4] = {pack(s[0][0], s[0][1]), pack(s[0][2], s[0][3]), pack(s[1][0], s[1][1]), pack(s[1][2], s[1][3])};
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                uint32_t f[4];
                ldm4_t(f, st + C::kMatrix + (uint32_t)(v_row * (DP * 2) + (((2 * t + v_chunk) ^ (v_row % 8)) * 16)));
                mma(o[2 * t], p, f[0], f[1]);
                mma(o[2 * t + 1], p, f[2], f[3]);
            }
            __syncwarp();  // the stage is written again by a later copy
        }

        // join the warps: O, base and l of each in shared memory
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            const int r = lane / 4 + 8 * h;
            if (lane % 4 == 0) {
                sml[(warp * 16 + r) * 2] = base[h];
                sml[(warp * 16 + r) * 2 + 1] = l[h];
            }
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
                *reinterpret_cast<float2*>(so + (warp * 16 + r) * C::kPitch + n * 8 + (lane % 4) * 2) =
                    make_float2(o[n][2 * h], o[n][2 * h + 1]);
        }
        __syncthreads();
        if (a.join && !waited) {
            mafat_attn::launch_wait();
            waited = true;
        }
        if constexpr (CLUSTER) Parts::started();
        const int rows = min(16, g.rows - b.row0);
        constexpr int kQuads = DP / 4, kSets = 32 / kQuads;  // lanes of a row; rows of a warp, and parts of a lane
        const int d = lane % kQuads * 4;
#pragma unroll 1
        for (int r0 = warp * kSets; r0 < rows; r0 += kWarps * kSets) {
            const int r = min(r0 + lane / kQuads, rows - 1);
            const bool mine = r0 + lane / kQuads < rows;
            float top = -CUDART_INF_F, mw[kWarps];
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                mw[w] = sml[(w * 16 + r) * 2];
                top = mafat_attn::max_nan(top, mw[w]);
            }
            const float off = mafat_attn::subtrahend(top);
            float sum = 0.f;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float x = mafat_attn::exp2_fast(mw[w] - off);
                sum = fmaf(x, sml[(w * 16 + r) * 2 + 1], sum);
                const float4 u = *reinterpret_cast<const float4*>(so + (w * 16 + r) * C::kPitch + d);
                v.x = fmaf(x, u.x, v.x);
                v.y = fmaf(x, u.y, v.y);
                v.z = fmaf(x, u.z, v.z);
                v.w = fmaf(x, u.w, v.w);
            }
            const mafat_attn::Out out(a, b, mafat_attn::Row(a, b, b.row0 + r));
            float inv = mafat_attn::inverse_sum(sum);
            if (a.join) {  // with the parts of the launch before: a lane has the weight of every kQuads-th
                // sixteen parts' loads on their way together, the first with those of the weights
                constexpr int kTogether = 16;
                const float* src = a.part_o + out.row * a.dim + d;
                float4 u[kTogether];
                auto load_parts = [&](int p0) {
#pragma unroll
                    for (int e = 0; e < kTogether; ++e) {
                        u[e] = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (p0 + e < a.join && d < a.dim)
                            u[e] = *reinterpret_cast<const float4*>(src + (int64_t)(p0 + e) * a.rows_total * a.dim);
                    }
                };
                load_parts(0);
                const float own = mafat_attn::row_lse2(top, sum);
                float lse[kSets], best = own;
#pragma unroll
                for (int k = 0; k < kSets; ++k) {
                    const int p = k * kQuads + lane % kQuads;
                    lse[k] = p < a.join ? a.part_lse[(int64_t)p * a.rows_total + out.row] : -CUDART_INF_F;
                    best = mafat_attn::max_nan(best, lse[k]);
                }
#pragma unroll
                for (int w = 1; w < kQuads; w *= 2) best = mafat_attn::max_nan(best, __shfl_xor_sync(0xffffffffu, best, w));
                const float base = best == -CUDART_INF_F ? 0.f : best;
                float total = 0.f;
#pragma unroll
                for (int k = 0; k < kSets; ++k) total += lse[k] = mafat_attn::exp2_fast(lse[k] - base);
#pragma unroll
                for (int w = 1; w < kQuads; w *= 2) total += __shfl_xor_sync(0xffffffffu, total, w);
                const float x = mafat_attn::exp2_fast(own - base);
                total += x;
                inv = sum == 0.f ? 0.f : x / sum;  // then all are divided by the total
                v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
#pragma unroll
                for (int p0 = 0; p0 < kMostJoin; p0 += kTogether) {
                    if (p0 >= a.join) break;
                    if (p0 > 0) load_parts(p0);
#pragma unroll
                    for (int e = 0; e < kTogether; ++e) {  // past the last part: u is zero
                        const float f =
                            __shfl_sync(0xffffffffu, lse[p0 / kQuads], (lane & ~(kQuads - 1)) + (p0 + e) % kQuads);
                        v = make_float4(fmaf(f, u[e].x, v.x), fmaf(f, u[e].y, v.y), fmaf(f, u[e].z, v.z),
                                        fmaf(f, u[e].w, v.w));
                    }
                }
                inv = mafat_attn::inverse_sum(total);
                if (mine && d == 0 && a.lse)
                    a.lse[out.row] = total == 0.f ? -CUDART_INF_F : (base + log2f(total)) * CUDART_LN2_F;
            } else if (mine && d == 0) {
                if constexpr (CLUSTER)
                    parts.put_sum(r, mafat_attn::row_lse2(top, sum));
                else
                    mafat_attn::store_lse(a, out, top, sum);
            }
            if (!mine || d >= a.dim) continue;
            v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
            if constexpr (CLUSTER)
                parts.put(r, d, v);
            else if (a.direct)
                *reinterpret_cast<uint2*>((__nv_bfloat16*)a.out + out.o + d) = make_uint2(pack(v.x, v.y), pack(v.z, v.w));
            else
                *reinterpret_cast<float4*>(a.part_o + out.part * a.dim + d) = v;
        }
        if constexpr (CLUSTER) parts.template join<__nv_bfloat16, kWarps>(a, b, rows);
    }
    wait_copies<0>();
    mafat_attn::launch_end(a);
}

template <int DP, bool TREE>
cudaError_t launch_form(const MafatAttnArgs& a, int ctas, cudaStream_t s) {
    return mafat_launch_clusters(a.cluster, a.cluster > 1 ? attn_rows_kernel<DP, true, TREE, NoPrefix> : attn_rows_kernel<DP, false, TREE, NoPrefix>,
                                 (unsigned)ctas, kThreads, a.cluster > 1 ? Cfg<DP, true>::kSmem : Cfg<DP, false>::kSmem, s, a, NoPrefix());
}
template <int DP>
cudaError_t launch(const MafatAttnArgs& a, int ctas, const MafatRowsPrefix* prefix, cudaStream_t s) {
    if (prefix)
        return mafat_launch_clusters(
            a.cluster, a.cluster > 1 ? attn_rows_kernel<DP, true, true, MafatRowsPrefix> : attn_rows_kernel<DP, false, true, MafatRowsPrefix>,
            (unsigned)ctas, kThreads, a.cluster > 1 ? Cfg<DP, true>::kSmem : Cfg<DP, false>::kSmem, s, a, *prefix);
    return a.tree ? launch_form<DP, true>(a, ctas, s) : launch_form<DP, false>(a, ctas, s);
}
template <int DP, bool TREE>
cudaError_t prepare_form() {
    const cudaError_t e = cudaFuncSetAttribute(attn_rows_kernel<DP, false, TREE, NoPrefix>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               Cfg<DP, false>::kSmem);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(attn_rows_kernel<DP, true, TREE, NoPrefix>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<DP, true>::kSmem);
}
template <int DP>
cudaError_t prepare(bool tree) {
    if (!tree) return prepare_form<DP, false>();
    cudaError_t e = prepare_form<DP, true>();
    if (e != cudaSuccess) return e;
    e = cudaFuncSetAttribute(attn_rows_kernel<DP, false, true, MafatRowsPrefix>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             Cfg<DP, false>::kSmem);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(attn_rows_kernel<DP, true, true, MafatRowsPrefix>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                Cfg<DP, true>::kSmem);
}

}  // namespace

int mafat_attn_rows_keys() { return kBN; }
int mafat_attn_rows_join() { return kMostJoin; }

cudaError_t mafat_launch_attn_rows(const MafatAttnArgs& a, int ctas, const MafatRowsPrefix* prefix, cudaStream_t s) {
    return a.dim <= 64 ? launch<64>(a, ctas, prefix, s) : launch<128>(a, ctas, prefix, s);
}

cudaError_t mafat_prepare_attn_rows(bool tree, int dim) { return dim <= 64 ? prepare<64>(tree) : prepare<128>(tree); }
