// Attention in fp32 on the CUDA cores, for fp32 plans.
//
// For a row with query q and readable keys s:  O = sum_s exp(c q.k_s) v_s / sum_s exp(c q.k_s).
// A CTA takes BM rows of one (sequence, key head) and one part of its keys, 64 keys at a time, and
// keeps for each row the running maximum m of q.k_s, the sum l and the unnormalised O, all fp32:
// a tile's scores raise m to m', and l and O are multiplied by 2^(c' (m - m')), c' = c log2(e).
//
// A thread owns 4 rows x 4 keys of the scores and 4 rows x 2 quarters of the channels of O, so that a
// 16-byte shared-memory read feeds 8 FMAs; K's and V's tiles are single buffers.
#include "attn_common.cuh"

namespace {

constexpr int kBN = 64;
constexpr int kTX = 16;  // threads along the keys / channels

template <int BM, int DP>
struct Tile {
    static constexpr int kThreads = BM / 4 * kTX;
    static constexpr int kPitch = DP + 4;        // K and Q rows: 16-byte reads of 8 rows hit all banks
    static constexpr int kPPitch = kBN + 4;
    static constexpr int kFloats = BM * kPitch + kBN * kPitch + kBN * DP + BM * kPPitch;
    static constexpr int kSmem = kFloats * 4;
};

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }

// rows [0, count) of a matrix with `stride` elements between rows into smem; channels past dim and
// rows that are not readable become zero
template <int ROWS, int DP, int PITCH, int THREADS, class Ok>
__device__ __forceinline__ void load_rows(float* dst, const float* src, int64_t stride, int dim, Ok ok) {
    constexpr int kChunks = DP / 4;
#pragma unroll 4
    for (int i = threadIdx.x; i < ROWS * kChunks; i += THREADS) {
        const int r = i / kChunks, c = (i % kChunks) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < dim && ok(r)) v = load4(src + (int64_t)r * stride + c);
        *reinterpret_cast<float4*>(dst + r * PITCH + c) = v;
    }
}

template <int BM, int DP>
__global__ void __launch_bounds__(BM / 4 * kTX) attn_simt_kernel(const __grid_constant__ MafatAttnArgs a) {
    using L = Tile<BM, DP>;
    extern __shared__ __align__(16) float sm[];
    float* sq = sm;
    float* sk = sq + BM * L::kPitch;
    float* sv = sk + kBN * L::kPitch;
    float* sp = sv + kBN * DP;
    mafat_attn::launch_begin(a);
    const mafat_attn::Block b(a, blockIdx.x, BM, kBN);
    const MafatAttnSeg& g = a.seg;
    const int tx = threadIdx.x % kTX, ty = threadIdx.x / kTX;

    // queries
    {
        constexpr int kChunks = DP / 4;
        for (int i = threadIdx.x; i < BM * kChunks; i += L::kThreads) {
            const int r = i / kChunks, c = (i % kChunks) * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (c < a.dim && b.row0 + r < g.rows)
                v = load4((const float*)a.q + mafat_attn::Row(a, b, b.row0 + r).query(a) + c);
            *reinterpret_cast<float4*>(sq + r * L::kPitch + c) = v;
        }
    }
    int limit[4];
    float m[4], l[4], o[4][DP / kTX];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        limit[i] = mafat_attn::Row(a, b, b.row0 + ty * 4 + i).limit(a, b);
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int d = 0; d < DP / kTX; ++d) o[i][d] = 0.f;
    }
    const float* kp = (const float*)g.k + (int64_t)b.seq * g.k_sb + (int64_t)b.head * g.k_sh;
    const float* vp = (const float*)g.v + (int64_t)b.seq * g.v_sb + (int64_t)b.head * g.v_sh;
    const uint8_t* mask = g.mask ? g.mask + (int64_t)b.seq * g.n : nullptr;

    for (int key0 = b.key0; key0 < b.key1; key0 += kBN) {
        auto ok = [&](int r) { return key0 + r < b.len && (!mask || mask[key0 + r] != 0); };
        __syncthreads();
        load_rows<kBN, DP, L::kPitch, L::kThreads>(sk, kp + (int64_t)key0 * g.k_ss, g.k_ss, a.dim, ok);
        load_rows<kBN, DP, DP, L::kThreads>(sv, vp + (int64_t)key0 * g.v_ss, g.v_ss, a.dim, ok);
        __syncthreads();
        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
        for (int d = 0; d < DP; d += 4) {
            float4 x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4*>(sq + (ty * 4 + i) * L::kPitch + d);
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(sk + (tx + kTX * j) * L::kPitch + d);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[i][j] = fmaf(x[i].x, y[j].x, s[i][j]);
                    s[i][j] = fmaf(x[i].y, y[j].y, s[i][j]);
                    s[i][j] = fmaf(x[i].z, y[j].z, s[i][j]);
                    s[i][j] = fmaf(x[i].w, y[j].w, s[i][j]);
                }
        }
        bool seen[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) seen[j] = ok(tx + kTX * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!seen[j] || key0 + tx + kTX * j >= limit[i]) s[i][j] = -INFINITY;
                top = mafat_attn::max_nan(top, s[i][j]);
            }
#pragma unroll
            for (int w = 1; w < kTX; w *= 2) top = mafat_attn::max_nan(top, __shfl_xor_sync(0xffffffffu, top, w));
            const float mn = mafat_attn::max_nan(m[i], top);
            const float base = mn == -INFINITY ? 0.f : mn * a.scale_log2;  // no readable key yet: 2^-inf = 0
            const float keep = mafat_attn::exp2_fast(fmaf(m[i], a.scale_log2, -base));
            m[i] = mn;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = mafat_attn::exp2_fast(fmaf(s[i][j], a.scale_log2, -base));
                sum += s[i][j];
                sp[(ty * 4 + i) * L::kPPitch + tx + kTX * j] = s[i][j];
            }
            l[i] = l[i] * keep + sum;
#pragma unroll
            for (int d = 0; d < DP / kTX; ++d) o[i][d] *= keep;
        }
        __syncwarp();  // a row's scores are written and read by the 16 threads of one half warp
#pragma unroll 2
        for (int k = 0; k < kBN; k += 4) {
            float4 p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = *reinterpret_cast<const float4*>(sp + (ty * 4 + i) * L::kPPitch + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
                for (int c = 0; c < DP / 64; ++c) {
                    const float4 v = *reinterpret_cast<const float4*>(sv + (k + e) * DP + c * 64 + tx * 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float w = e == 0 ? p[i].x : e == 1 ? p[i].y : e == 2 ? p[i].z : p[i].w;
                        o[i][c * 4 + 0] = fmaf(w, v.x, o[i][c * 4 + 0]);
                        o[i][c * 4 + 1] = fmaf(w, v.y, o[i][c * 4 + 1]);
                        o[i][c * 4 + 2] = fmaf(w, v.z, o[i][c * 4 + 2]);
                        o[i][c * 4 + 3] = fmaf(w, v.w, o[i][c * 4 + 3]);
                    }
                }
            }
        }
        __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int w = 1; w < kTX; w *= 2) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
        const int r = b.row0 + ty * 4 + i;
        if (r >= g.rows) continue;
        float inv = mafat_attn::inverse_sum(l[i]), top = 0.f, scale = 0.f;
        const mafat_attn::Out w(a, b, mafat_attn::Row(a, b, r));
        if (a.join) {
            mafat_attn::launch_wait();
            const mafat_attn::Join jn(a, w, m[i], l[i]);
            inv = jn.own;
            top = jn.top;
            scale = jn.inv;
            if (tx == 0 && a.lse) a.lse[w.row] = jn.lse2 * CUDART_LN2_F;
        } else if (tx == 0) {
            mafat_attn::store_lse(a, w, m[i], l[i]);
        }
#pragma unroll
        for (int c = 0; c < DP / 64; ++c) {
            const int d = c * 64 + tx * 4;
            if (d >= a.dim) continue;
            float4 v = make_float4(o[i][c * 4] * inv, o[i][c * 4 + 1] * inv, o[i][c * 4 + 2] * inv,
                                   o[i][c * 4 + 3] * inv);
            for (int p = 0; p < a.join; ++p) {
                const int64_t at = (int64_t)p * a.rows_total + w.row;
                const float f = mafat_attn::exp2_fast(a.part_lse[at] - top) * scale;
                const float4 u = load4(a.part_o + at * a.dim + d);
                v = make_float4(fmaf(f, u.x, v.x), fmaf(f, u.y, v.y), fmaf(f, u.z, v.z), fmaf(f, u.w, v.w));
            }
            store4(a.direct ? (float*)a.out + w.o + d : a.part_o + w.part * a.dim + d, v);
        }
    }
    mafat_attn::launch_end(a);
}

template <int BM, int DP>
cudaError_t launch(const MafatAttnArgs& a, cudaStream_t s) {
    return mafat_launch_overlapped(attn_simt_kernel<BM, DP>, a.seg.items, Tile<BM, DP>::kThreads, Tile<BM, DP>::kSmem, s, a);
}
template <int BM, int DP>
cudaError_t prepare() {
    return cudaFuncSetAttribute(attn_simt_kernel<BM, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                Tile<BM, DP>::kSmem);
}
}  // namespace

int mafat_attn_simt_rows(bool wide) { return wide ? 64 : 16; }
int mafat_attn_simt_keys() { return kBN; }

cudaError_t mafat_prepare_attn_simt() {
    cudaError_t e;
    if ((e = prepare<64, 64>()) != cudaSuccess) return e;
    if ((e = prepare<64, 128>()) != cudaSuccess) return e;
    if ((e = prepare<16, 64>()) != cudaSuccess) return e;
    return prepare<16, 128>();
}

cudaError_t mafat_launch_attn_simt(const MafatAttnArgs& a, bool wide, cudaStream_t s) {
    if (wide) return a.dim <= 64 ? launch<64, 64>(a, s) : launch<64, 128>(a, s);
    return a.dim <= 64 ? launch<16, 64>(a, s) : launch<16, 128>(a, s);
}
