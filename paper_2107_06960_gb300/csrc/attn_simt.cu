// Attention in fp32 on the CUDA cores, for fp32 plans.
//
// For a row with query q and readable keys s:  O = sum_s exp(c q.k_s) v_s / sum_s exp(c q.k_s), with
// the running maximum b of c log2(e) q.k_s, the sum l and the unnormalised O of each row, all fp32: a tile's
// scores raise b to b', and l and O are multiplied by 2^(b - b').
//
// Two neighbouring products are one packed instruction (fma.rn.f32x2, each rounded as alone), which
// leaves issue slots to the shared-memory reads.  Keys that are not readable are not read: zeros stand in the places of
// a tile without a key (cp.async fills them), so that 0 x NaN cannot reach O.
//
// Many rows (attn_simt_kernel): bound by shared-memory reads (81 % of their rate with 61 % of the FMAs'): 2 x 1024
// tokens, 16 query and 4 key heads of 128 channels, 2888 keys take 1136 us or 43 TFLOP/s.  A CTA takes 64 rows, 64 keys at a time, two CTAs an SM; a thread has 4 rows x 4 keys of the scores, then 4
// rows x DP / 16 channels of O.  K's and V's tiles are single buffers: the next K is copied while the
// values are summed, the next V while the scores are made.  With a mask the tiles are of readable keys alone: one warp
// lists the next tile's while the scores are made (8 x 1024 tokens, 8 heads of 64 channels over 1444 states, in us:
// half of them readable 339, all 633; 643 with tiles of all keys either way).  A warp with 16 rows x 64 keys (queries and
// weights broadcast, fewer reads an FMA, 8 warps instead of 16) was 4 % slower.
//
// Few rows (attn_simt_few_kernel): bound by reading K and V.  The warps of a CTA share the R rows and split the
// keys, each with a ring of runs of 8 keys of its own and its own maximum, sum and O, joined at the end.  One token of 64
// sequences, 32 query and 8 key heads, 1444 keys: 131 us or 5.8 TB/s with 128 channels, 66 us with 64.
#include "attn_common.cuh"

namespace {

constexpr int kBN = 64;

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }

__device__ __forceinline__ void copy16(float* dst, const float* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
                 "r"(on ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// r += a * b, two values at once
__device__ __forceinline__ void fma2(float2& r, float2 a, float2 b) {
    asm("{\n\t.reg .b64 x, y, z;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%0, %1};\n\t"
        "fma.rn.f32x2 z, x, y, z;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "+f"(r.x), "+f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
}

// One row's share of the online softmax for the score of a lane, whose WIDTH neighbours have the row's others:
// s becomes the weight; returns the factor of what was summed before.
template <int WIDTH>
__device__ __forceinline__ float softmax_step(float& s, float& base, float& l, float scale_log2) {
    float top = s;
#pragma unroll
    for (int w = 1; w < WIDTH; w *= 2) top = mafat_attn::max_nan(top, __shfl_xor_sync(0xffffffffu, top, w));
    const float next = mafat_attn::max_nan(base, top * scale_log2), off = mafat_attn::subtrahend(next);
    const float keep = mafat_attn::exp2_fast(base - off);
    base = next;
    s = mafat_attn::exp2_fast(fmaf(s, scale_log2, -off));
    l = l * keep + s;  // of the lane's keys
    return keep;
}

// Writes a row's four channels from d, joined with the parts of the launch before.
struct Writer {
    mafat_attn::Out at;
    float own, top, inv;
    __device__ __forceinline__ Writer(const MafatAttnArgs& a, const mafat_attn::Block& b, int r, float base, float l, bool first)
        : at(a, b, mafat_attn::Row(a, b, r)), own(mafat_attn::inverse_sum(l)), top(0.f), inv(0.f) {
        if (a.join) {
            mafat_attn::launch_wait();
            const mafat_attn::Join jn(a, at, base, l);
            own = jn.own;
            top = jn.top;
            inv = jn.inv;
            if (first && a.lse) a.lse[at.row] = jn.lse2 * CUDART_LN2_F;
        } else if (first) {
            mafat_attn::store_lse(a, at, base, l);
        }
    }
    __device__ __forceinline__ void put(const MafatAttnArgs& a, int d, float4 v) const {
        if (d >= a.dim) return;
        v = make_float4(v.x * own, v.y * own, v.z * own, v.w * own);
        for (int p = 0; p < a.join; ++p) {
            const int64_t row = (int64_t)p * a.rows_total + at.row;
            const float f = mafat_attn::exp2_fast(a.part_lse[row] - top) * inv;
            const float4 u = load4(a.part_o + row * a.dim + d);
            v = make_float4(fmaf(f, u.x, v.x), fmaf(f, u.y, v.y), fmaf(f, u.z, v.z), fmaf(f, u.w, v.w));
        }
        store4(a.direct ? (float*)a.out + at.o + d : a.part_o + at.part * a.dim + d, v);
    }
};

// ---- many rows --------------------------------------------------------------------------------

constexpr int kTX = 16;  // threads along the keys / channels
constexpr int kBM = 64;

template <int DP>
struct Tile {
    static constexpr int kThreads = kBM / 4 * kTX;
    static constexpr int kPitch = DP + 4;  // K rows: 16-byte reads of 8 rows hit all banks
    static constexpr int kSmem = (kBM * DP + kBN * kPitch + kBN * DP + kBM * kBN) * 4;
    static_assert(kSmem <= 115712, "two CTAs on an SM");
};
// Queries and weights have no padding: a warp reads two rows four apart, whose quads are swapped in one of them so
// that they lie in different banks.
__device__ __forceinline__ int quad_of(int row, int quad) { return quad ^ (row / 4 % 2); }

// copies rows of a matrix with `stride` elements between rows, the r-th from row key(r); channels past dim and rows
// whose key is negative become zero
template <int ROWS, int DP, int PITCH, int THREADS, class Key>
__device__ __forceinline__ void copy_rows(float* dst, const float* src, int64_t stride, int dim, Key key) {
    constexpr int kChunks = DP / 4;
#pragma unroll 8
    for (int i = threadIdx.x; i < ROWS * kChunks; i += THREADS) {
        const int r = i / kChunks, c = (i % kChunks) * 4, k = key(r);
        const bool on = c < dim && k >= 0;
        copy16(dst + r * PITCH + c, src + (on ? (int64_t)k * stride + c : 0), on);
    }
    copies_done();
}

// Lists the readable keys of a part, kBN at a time, by one warp.  The bytes of the mask that a list starts with are
// read before they are used.
struct Readable {
    static constexpr int kBytes = 4;  // of a lane
    const uint8_t* mask;
    int pos, end, lane;
    uint8_t m[kBytes];
    __device__ __forceinline__ void read() {
#pragma unroll
        for (int i = 0; i < kBytes; ++i) m[i] = pos + 32 * i + lane < end ? mask[pos + 32 * i + lane] : 0;
    }
    // the key of place r goes to list[r * PITCH], -1 to the places after the last; returns how many there are
    template <int PITCH>
    __device__ __forceinline__ int list(int* list) {
        int n = 0;
#pragma unroll 1
        for (;;) {
#pragma unroll
            for (int i = 0; i < kBytes; ++i) {
                const uint32_t on = __ballot_sync(0xffffffffu, m[i] != 0);
                const int at = n + __popc(on & ((1u << lane) - 1u));
                if (m[i] != 0 && at < kBN) list[at * PITCH] = pos + 32 * i + lane;
                n += __popc(on);
            }
            if (n >= kBN) {
                __syncwarp();
                pos = list[(kBN - 1) * PITCH] + 1;
                return kBN;
            }
            pos += 32 * kBytes;
            if (pos >= end) break;
            read();
        }
        for (int r = n + lane; r < kBN; r += 32) list[r * PITCH] = -1;
        return n;
    }
};

template <int DP, bool MASK>
__global__ void __launch_bounds__(kBM / 4 * kTX, 2) attn_simt_kernel(const __grid_constant__ MafatAttnArgs a) {
    using L = Tile<DP>;
    extern __shared__ __align__(16) float sm[];
    float* sq = sm;
    float* sk = sq + kBM * DP;
    float* sv = sk + kBN * L::kPitch;
    float* sp = sv + kBN * DP;
    mafat_attn::launch_begin(a);
    const mafat_attn::Block b(a, blockIdx.x, kBM, kBN);
    const MafatAttnSeg& g = a.seg;
    const int tx = threadIdx.x % kTX, ty = threadIdx.x / kTX;
    const float* kp = (const float*)g.k + (int64_t)b.seq * g.k_sb + (int64_t)b.head * g.k_sh;
    const float* vp = (const float*)g.v + (int64_t)b.seq * g.v_sb + (int64_t)b.head * g.v_sh;
    // MASK: tiles are of readable keys alone, whose numbers stand in two lists in the padding of K's rows
    int* lists = (int*)(sk + DP);
    Readable readable{MASK ? g.mask + (int64_t)b.seq * g.n : nullptr, b.key0, min(b.key1, b.len), (int)threadIdx.x, {}};
    auto list_next = [&](int buf) {
        const int n = readable.list<L::kPitch>(lists + buf);
        if (threadIdx.x == 0) lists[2 + buf] = n;
    };
    int tile = 0, key0 = b.key0;
    bool more = b.key0 < b.key1;
    auto key_of = [&](int r) {  // of the tile's place r; negative: none
        if constexpr (MASK) return lists[r * L::kPitch + (tile & 1)];
        return key0 + r < b.len ? key0 + r : -1;
    };
    auto copy_k = [&]() {
        copy_rows<kBN, DP, L::kPitch, L::kThreads>(sk, kp, g.k_ss, a.dim, key_of);
    };
    auto copy_v = [&]() {
        copy_rows<kBN, DP, DP, L::kThreads>(sv, vp, g.v_ss, a.dim, key_of);
    };

    // queries, then the first keys
    {
        constexpr int kChunks = DP / 4;
#pragma unroll 4
        for (int i = threadIdx.x; i < kBM * kChunks; i += L::kThreads) {
            const int r = i / kChunks, c = (i % kChunks) * 4;
            const bool on = c < a.dim && b.row0 + r < g.rows;
            copy16(sq + r * DP + quad_of(r, c / 4) * 4,
                   (const float*)a.q + (on ? mafat_attn::Row(a, b, b.row0 + r).query(a) + c : 0), on);
        }
        if constexpr (MASK) {
            if (threadIdx.x < 32) {
                readable.read();
                list_next(0);
            }
            __syncthreads();
            more = lists[2] > 0;
        }
        if (more) copy_k();
        copies_done();
    }
    constexpr int kO = DP / kTX / 2;  // pairs of channels: c * 64 + tx * 4 + {0, 1}, {2, 3}
    int limit[4];
    float base[4], l[4];
    float2 o[4][kO];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        limit[i] = mafat_attn::Row(a, b, b.row0 + ty * 4 + i).limit(a, b);
        base[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int d = 0; d < kO; ++d) o[i][d] = make_float2(0.f, 0.f);
    }

#pragma unroll 1
    while (more) {
        wait_copies<0>();
        __syncthreads();  // K is there, and all are done with V
        copy_v();
        if (MASK && threadIdx.x < 32) readable.read();
        float2 acc[4][4];  // sums over even and odd channels
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int d = 0; d < DP; d += 4) {
            float4 x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = load4(sq + (ty * 4 + i) * DP + quad_of(ty * 4, d / 4) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = load4(sk + (tx + kTX * j) * L::kPitch + d);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    fma2(acc[i][j], make_float2(x[i].x, x[i].y), make_float2(y[j].x, y[j].y));
                    fma2(acc[i][j], make_float2(x[i].z, x[i].w), make_float2(y[j].z, y[j].w));
                }
        }
        int key[4];
        float keep[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) key[j] = key_of(tx + kTX * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float s[4], top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[j] = acc[i][j].x + acc[i][j].y;
                if (key[j] < 0 || key[j] >= limit[i]) s[j] = -INFINITY;
                top = mafat_attn::max_nan(top, s[j]);
            }
#pragma unroll
            for (int w = 1; w < kTX; w *= 2) top = mafat_attn::max_nan(top, __shfl_xor_sync(0xffffffffu, top, w));
            const float next = mafat_attn::max_nan(base[i], top * a.scale_log2), off = mafat_attn::subtrahend(next);
            keep[i] = mafat_attn::exp2_fast(base[i] - off);
            base[i] = next;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[j] = mafat_attn::exp2_fast(fmaf(s[j], a.scale_log2, -off));
                sum += s[j];
                sp[(ty * 4 + i) * kBN + quad_of(ty * 4, (tx + kTX * j) / 4) * 4 + tx % 4] = s[j];
            }
            l[i] = l[i] * keep[i] + sum;
        }
        if (MASK && threadIdx.x < 32) list_next((tile & 1) ^ 1);
        wait_copies<0>();
        __syncthreads();  // V is there, and all are done with K (P is read by the half warp that wrote it)
        ++tile;
        key0 += kBN;
        if constexpr (MASK)
            more = lists[2 + (tile & 1)] > 0;
        else
            more = key0 < b.key1;
        if (more) copy_k();
        // the tile's sum by itself, then added: O's size sets the rounding of one addition a tile, not of 64 (6000 keys
        // in one part: 1.4e-6 of the result without it, the weights' 3e-7 with it)
        float2 sum[4][kO];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < kO; ++d) sum[i][d] = make_float2(0.f, 0.f);
#pragma unroll 2
        for (int k = 0; k < kBN; k += 4) {
            float4 p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = load4(sp + (ty * 4 + i) * kBN + quad_of(ty * 4, k / 4) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
                for (int c = 0; c < DP / 64; ++c) {
                    const float4 v = load4(sv + (k + e) * DP + c * 64 + tx * 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float w = e == 0 ? p[i].x : e == 1 ? p[i].y : e == 2 ? p[i].z : p[i].w;
                        fma2(sum[i][2 * c], make_float2(w, w), make_float2(v.x, v.y));
                        fma2(sum[i][2 * c + 1], make_float2(w, w), make_float2(v.z, v.w));
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < kO; ++d)
                o[i][d] = make_float2(fmaf(o[i][d].x, keep[i], sum[i][d].x), fmaf(o[i][d].y, keep[i], sum[i][d].y));
    }
    wait_copies<0>();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int w = 1; w < kTX; w *= 2) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
        const int r = b.row0 + ty * 4 + i;
        if (r >= g.rows) continue;
        const Writer w(a, b, r, base[i], l[i], tx == 0);
#pragma unroll
        for (int c = 0; c < DP / 64; ++c)
            w.put(a, c * 64 + tx * 4, make_float4(o[i][2 * c].x, o[i][2 * c].y, o[i][2 * c + 1].x, o[i][2 * c + 1].y));
    }
    mafat_attn::launch_end(a);
}

// ---- few rows -----------------------------------------------------------------------------------

constexpr int kFewWarps = 8, kRun = 8;  // keys of a warp at a time

template <int R, int DP, bool CLUSTER>
struct Few {
    static constexpr int kThreads = kFewWarps * 32;
    static constexpr int kStages = 3;  // with 64 channels two CTAs share an SM
    static constexpr int kPitch = DP + 4;
    static constexpr int kStage = kRun * (kPitch + DP);               // floats of a run of K and V
    static constexpr int kWarp = kStages * kStage + R * kRun;         // and the weights
    static constexpr int kOffParts = (R * DP + kFewWarps * kWarp) * 4;
    static constexpr int kSmem = kOffParts + (CLUSTER ? mafat_attn::ClusterParts<R, DP>::kBytes : 0);
    static_assert(kFewWarps * R * (DP + 2) <= kFewWarps * kWarp, "the join's space is the rings'");
};

template <int R, int DP, bool CLUSTER>
__global__ void __launch_bounds__(kFewWarps * 32, DP == 64 ? 2 : 1) attn_simt_few_kernel(const __grid_constant__ MafatAttnArgs a) {
    using L = Few<R, DP, CLUSTER>;
    using Parts = mafat_attn::ClusterParts<R, DP>;
    constexpr int kCh = DP / 32;
    extern __shared__ __align__(16) float sm[];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    float* sq = sm;
    float* ring = sm + R * DP + warp * L::kWarp;
    float* sp = ring + L::kStages * L::kStage;
    if constexpr (CLUSTER) Parts::start();
    mafat_attn::launch_begin(a);
    const mafat_attn::Block b(a, blockIdx.x, R, kBN);
    const MafatAttnSeg& g = a.seg;
    const float* kp = (const float*)g.k + (int64_t)b.seq * g.k_sb + (int64_t)b.head * g.k_sh;
    const float* vp = (const float*)g.v + (int64_t)b.seq * g.v_sb + (int64_t)b.head * g.v_sh;
    const uint8_t* mask = g.mask ? g.mask + (int64_t)b.seq * g.n : nullptr;
    const int first = b.key0 + warp * kRun;
    const int runs = b.key1 > first ? (b.key1 - first + kBN - 1) / kBN : 0;
    constexpr int kChunks = DP / 4, kRows = 32 / kChunks;  // 1 row of an access, or 2
    const int cc = lane % kChunks * 4, cr = lane / kChunks;
    auto load = [&](int i) {
        if (i < runs) {
            const int key = first + i * kBN;
            float* k_dst = ring + (i % L::kStages) * L::kStage;
            float* v_dst = k_dst + kRun * L::kPitch;
#pragma unroll
            for (int r0 = 0; r0 < kRun; r0 += kRows) {
                const int r = r0 + cr, k = key + r;
                const bool on = cc < a.dim && k < b.len && (!mask || mask[k] != 0);
                copy16(k_dst + r * L::kPitch + cc, kp + (on ? (int64_t)k * g.k_ss + cc : 0), on);
                copy16(v_dst + r * DP + cc, vp + (on ? (int64_t)k * g.v_ss + cc : 0), on);
            }
        }
        copies_done();
    };
    for (int i = threadIdx.x; i < R * kChunks; i += L::kThreads) {
        const int r = i / kChunks, c = i % kChunks * 4;
        const bool on = c < a.dim && b.row0 + r < g.rows;
        copy16(sq + r * DP + c, (const float*)a.q + (on ? mafat_attn::Row(a, b, b.row0 + r).query(a) + c : 0), on);
    }
#pragma unroll
    for (int i = 0; i < L::kStages - 1; ++i) load(i);
    wait_copies<L::kStages - 2>();
    __syncthreads();  // the queries came with the first run

    float base[R], l[R];
    float2 o[R][kCh / 2];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        base[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int d = 0; d < kCh / 2; ++d) o[i][d] = make_float2(0.f, 0.f);
    }
    // scores: a lane has one key and every fourth quad of channels
    const int key_of = lane % kRun, part = lane / kRun;
#pragma unroll 1
    for (int i = 0; i < runs; ++i) {
        load(i + L::kStages - 1);
        wait_copies<L::kStages - 1>();
        __syncwarp();
        const int key = first + i * kBN;
        const float* sk = ring + (i % L::kStages) * L::kStage;
        const float* sv = sk + kRun * L::kPitch;
        float2 acc[R];
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r] = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int d = part * 4; d < DP; d += 4 * (32 / kRun)) {
            const float4 y = load4(sk + key_of * L::kPitch + d);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float4 x = load4(sq + r * DP + d);
                fma2(acc[r], make_float2(x.x, x.y), make_float2(y.x, y.y));
                fma2(acc[r], make_float2(x.z, x.w), make_float2(y.z, y.w));
            }
        }
        const int k = key + key_of;
        const bool seen = k < b.len && (!mask || mask[k] != 0);
        float keep[R];
        bool moved = false;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int limit = g.causal ? mafat_attn::Row(a, b, b.row0 + r).limit(a, b) : b.len;
            float s = acc[r].x + acc[r].y;
#pragma unroll
            for (int w = kRun; w < 32; w *= 2) s += __shfl_xor_sync(0xffffffffu, s, w);
            if (!seen || k >= limit) s = -INFINITY;
            keep[r] = softmax_step<kRun>(s, base[r], l[r], a.scale_log2);  // l: each key in four lanes
            moved = moved || keep[r] != 1.f;
            if (part == 0) sp[r * kRun + key_of] = s;
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int d = 0; d < kCh / 2; ++d) o[r][d] = make_float2(o[r][d].x * keep[r], o[r][d].y * keep[r]);
        }
        __syncwarp();
#pragma unroll
        for (int e0 = 0; e0 < kRun; e0 += 4) {
            float2 v[4][kCh / 2];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (kCh == 4) {
                    const float4 u = load4(sv + (e0 + e) * DP + lane * 4);
                    v[e][0] = make_float2(u.x, u.y);
                    v[e][1] = make_float2(u.z, u.w);
                } else {
                    v[e][0] = *reinterpret_cast<const float2*>(sv + (e0 + e) * DP + lane * 2);
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float4 p = load4(sp + r * kRun + e0);
#pragma unroll
                for (int d = 0; d < kCh / 2; ++d) {
                    fma2(o[r][d], make_float2(p.x, p.x), v[0][d]);
                    fma2(o[r][d], make_float2(p.y, p.y), v[1][d]);
                    fma2(o[r][d], make_float2(p.z, p.z), v[2][d]);
                    fma2(o[r][d], make_float2(p.w, p.w), v[3][d]);
                }
            }
        }
        __syncwarp();  // the stage is written again by the next copies, the weights by the next run
    }
    wait_copies<0>();
    __syncthreads();
    // join the warps: O, base and l of each in shared memory
    float* so = sm + R * DP;
    float* sml = so + kFewWarps * R * DP;
    const Parts parts(a, (uint8_t*)sm + L::kOffParts);
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int w = 1; w < kRun; w *= 2) l[r] += __shfl_xor_sync(0xffffffffu, l[r], w);
        if (lane == 0) {
            sml[(warp * R + r) * 2] = base[r];
            sml[(warp * R + r) * 2 + 1] = l[r];
        }
#pragma unroll
        for (int d = 0; d < kCh / 2; ++d)
            *reinterpret_cast<float2*>(so + (warp * R + r) * DP + lane * kCh + 2 * d) = o[r][d];
    }
    __syncthreads();
    const int rows = min(R, g.rows - b.row0);
    if constexpr (CLUSTER) Parts::started();
    for (int i = threadIdx.x; i < rows * kChunks; i += L::kThreads) {
        const int r = i / kChunks, d = i % kChunks * 4;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) top = mafat_attn::max_nan(top, sml[(w * R + r) * 2]);
        const float off = mafat_attn::subtrahend(top);
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) {
            const float x = mafat_attn::exp2_fast(sml[(w * R + r) * 2] - off);
            sum = fmaf(x, sml[(w * R + r) * 2 + 1], sum);
            const float4 u = load4(so + (w * R + r) * DP + d);
            v = make_float4(fmaf(x, u.x, v.x), fmaf(x, u.y, v.y), fmaf(x, u.z, v.z), fmaf(x, u.w, v.w));
        }
        if constexpr (CLUSTER) {
            const float inv = mafat_attn::inverse_sum(sum);
            if (d < a.dim) parts.put(r, d, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
            if (d == 0) parts.put_sum(r, mafat_attn::row_lse2(top, sum));
        } else {
            const Writer w(a, b, b.row0 + r, top, sum, d == 0);
            w.put(a, d, v);
        }
    }
    if constexpr (CLUSTER) parts.template join<float, kFewWarps>(a, b, rows);
    mafat_attn::launch_end(a);
}

template <int DP>
cudaError_t launch(const MafatAttnArgs& a, cudaStream_t s) {
    return mafat_launch_overlapped(a.seg.mask ? attn_simt_kernel<DP, true> : attn_simt_kernel<DP, false>, a.seg.items,
                                   Tile<DP>::kThreads, Tile<DP>::kSmem, s, a);
}
template <int R, int DP>
cudaError_t launch_few(const MafatAttnArgs& a, cudaStream_t s) {
    return mafat_launch_clusters(a.cluster,
                                 a.cluster > 1 ? attn_simt_few_kernel<R, DP, true> : attn_simt_few_kernel<R, DP, false>,
                                 a.seg.items, kFewWarps * 32,
                                 a.cluster > 1 ? Few<R, DP, true>::kSmem : Few<R, DP, false>::kSmem, s, a);
}
cudaError_t prepare(const void* fn, int smem) {
    return cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
}
template <int DP>
cudaError_t prepare_tiles() {
    const cudaError_t e = prepare((const void*)attn_simt_kernel<DP, false>, Tile<DP>::kSmem);
    return e != cudaSuccess ? e : prepare((const void*)attn_simt_kernel<DP, true>, Tile<DP>::kSmem);
}
template <int R, int DP>
cudaError_t prepare_few() {
    const cudaError_t e = prepare((const void*)attn_simt_few_kernel<R, DP, false>, Few<R, DP, false>::kSmem);
    return e != cudaSuccess ? e : prepare((const void*)attn_simt_few_kernel<R, DP, true>, Few<R, DP, true>::kSmem);
}

}  // namespace

int mafat_attn_simt_keys() { return kBN; }

cudaError_t mafat_prepare_attn_simt() {
    cudaError_t e;
    if ((e = prepare_few<4, 64>()) != cudaSuccess || (e = prepare_few<4, 128>()) != cudaSuccess) return e;
    if ((e = prepare_few<8, 64>()) != cudaSuccess || (e = prepare_few<8, 128>()) != cudaSuccess) return e;
    if ((e = prepare_tiles<64>()) != cudaSuccess) return e;
    return prepare_tiles<128>();
}

cudaError_t mafat_launch_attn_simt(const MafatAttnArgs& a, int rows, cudaStream_t s) {
    if (rows == 4) return a.dim <= 64 ? launch_few<4, 64>(a, s) : launch_few<4, 128>(a, s);
    if (rows == 8) return a.dim <= 64 ? launch_few<8, 64>(a, s) : launch_few<8, 128>(a, s);
    return a.dim <= 64 ? launch<64>(a, s) : launch<128>(a, s);
}
