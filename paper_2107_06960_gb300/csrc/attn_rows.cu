// Attention of few rows in bf16: the queries of a single token (or of a few), up to 16 rows of one
// (sequence, key head).
//
// Bound by reading K and V once: 16 rows give each 16-byte vector 16 x 16 operations, far from
// what the tensor core could do, so the work is to keep copies in flight.  A warp has every fourth run of 16
// keys of its CTA's part, a ring of STAGES runs of its own in shared memory (cp.async, no barrier between
// warps) and its own running maximum, sum and O; the four are joined once, at the end.  The products
// are the 16 x 8 x 16 ones of a single warp, whose operands are registers: S's accumulators are
// P's operand as they are.  P is rounded to bf16 for its product; all else is fp32.
//
// Keys that are not readable are not copied but filled with zeros, so that 0 x NaN cannot reach O.
#include <cuda_bf16.h>

#include "attn_common.cuh"

namespace {

constexpr int kWarps = 4;
constexpr int kRun = 16;                // keys of a warp at a time
constexpr int kBN = kWarps * kRun;

template <int DP>
struct Cfg {
    static constexpr int kStages = DP == 128 ? 3 : 4;
    static constexpr int kMatrix = kRun * DP * 2;       // bytes of a run of K or V
    static constexpr int kRing = kStages * 2 * kMatrix;  // of a warp
    static constexpr int kSmem = kWarps * kRing;
    static constexpr int kPitch = DP + 4;                // floats of a row of O while the warps are joined
    static_assert(kWarps * 16 * (kPitch + 2) * 4 <= kSmem, "the join's space is the rings'");
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

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

template <int DP>
__global__ void __launch_bounds__(kWarps * 32) attn_rows_kernel(const __grid_constant__ MafatAttnArgs a) {
    using C = Cfg<DP>;
    constexpr int kChunks = DP / 8;        // 16-byte chunks of a row
    constexpr int kSteps = DP / 16;
    extern __shared__ __align__(128) uint8_t sm[];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    mafat_attn::launch_begin(a);
    const mafat_attn::Block b(a, 16, kBN);
    const MafatAttnSeg& g = a.seg[b.seg];
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(sm) + warp * C::kRing;
    const __nv_bfloat16* kp = (const __nv_bfloat16*)g.k + (int64_t)b.seq * g.k_sb + (int64_t)b.head * g.k_sh;
    const __nv_bfloat16* vp = (const __nv_bfloat16*)g.v + (int64_t)b.seq * g.v_sb + (int64_t)b.head * g.v_sh;
    const uint8_t* mask = g.mask ? g.mask + (int64_t)b.seq * g.n : nullptr;
    const int first = b.key0 + warp * kRun;
    const int runs = b.key1 > first ? (b.key1 - first + kBN - 1) / kBN : 0;

    // run i into its stage: chunk c of key r at chunk c ^ (r % 8) of its row
    constexpr int kRows = 32 / kChunks;  // keys of one access of the warp
    const int cc = lane % kChunks, cr = lane / kChunks;
    const bool in_dim = cc * 8 < a.dim;
    auto load = [&](int i) {
        if (i < runs) {
            const int key = first + i * kBN;
            const uint32_t st = ring + (uint32_t)(i % C::kStages) * (2 * C::kMatrix);
#pragma unroll
            for (int r0 = 0; r0 < kRun; r0 += kRows) {
                const int r = r0 + cr, k = key + r;
                const bool on = in_dim && k < b.len && (!mask || mask[k] != 0);
                const uint32_t at = st + (uint32_t)(r * (DP * 2) + ((cc ^ (r % 8)) * 16));
                // a place that is not read still needs an address inside the tensor
                const int64_t kk = on ? k : 0;
                copy16(at, kp + (on ? kk * g.k_ss + cc * 8 : 0), on);
                copy16(at + C::kMatrix, vp + (on ? kk * g.v_ss + cc * 8 : 0), on);
            }
        }
        copies_done();
    };
#pragma unroll
    for (int i = 0; i < C::kStages - 1; ++i) load(i);

    // queries: operand rows lane / 4 and lane / 4 + 8
    uint32_t q[kSteps][4];
    int limit[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = b.row0 + lane / 4 + 8 * h;
        const mafat_attn::Row row(a, g, b, r);
        limit[h] = r < g.rows ? row.limit(a, g, b) : 0x7fffffff;
        const __nv_bfloat16* src = r < g.rows ? (const __nv_bfloat16*)a.q + row.query(a) : nullptr;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int d = s * 16 + e * 8 + (lane % 4) * 2;
                q[s][h + 2 * e] = src && d < a.dim ? *reinterpret_cast<const uint32_t*>(src + d) : 0u;
            }
    }

    float m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};
    float o[DP / 8][4];
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][e] = 0.f;

    // ldmatrix addresses: lane 8i + j gives row j of matrix i
    const int mi = lane / 8, mj = lane % 8;
    const int k_row = (mi / 2) * 8 + mj, k_chunk = mi % 2;   // K: keys 0-7 and 8-15, each with channels 0-7 and 8-15
    const int v_row = (mi % 2) * 8 + mj, v_chunk = mi / 2;   // V: channels 0-7 and 8-15, each with keys 0-7 and 8-15

#pragma unroll 1
    for (int i = 0; i < runs; ++i) {
        load(i + C::kStages - 1);
        wait_copies<C::kStages - 1>();
        __syncwarp();
        const int key = first + i * kBN;
        const uint32_t st = ring + (uint32_t)(i % C::kStages) * (2 * C::kMatrix);
        float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int t = 0; t < kSteps; ++t) {
            uint32_t f[4];
            ldm4(f, st + (uint32_t)(k_row * (DP * 2) + (((2 * t + k_chunk) ^ (k_row % 8)) * 16)));
            mma(s[0], q[t], f[0], f[1]);
            mma(s[1], q[t], f[2], f[3]);
        }
        if (mask || key + kRun > limit[0] || key + kRun > limit[1]) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int k = key + n * 8 + (lane % 4) * 2 + e % 2;
                    if (k >= b.len || k >= limit[e / 2] || (mask && mask[k] == 0)) s[n][e] = -CUDART_INF_F;
                }
        }
        float keep[2], off[2];
        bool up = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float top = mafat_attn::max_nan(mafat_attn::max_nan(s[0][2 * h], s[0][2 * h + 1]),
                                            mafat_attn::max_nan(s[1][2 * h], s[1][2 * h + 1]));
            top = mafat_attn::max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = mafat_attn::max_nan(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const float mn = mafat_attn::max_nan(m[h], top);
            up = up || mn != m[h];
            off[h] = mn == -CUDART_INF_F ? 0.f : -mn * a.scale_log2;
            keep[h] = mafat_attn::exp2_fast(fmaf(m[h], a.scale_log2, off[h]));
            m[h] = mn;
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
        __syncwarp();  // the stage is written again by the next iteration's copies
    }
    wait_copies<0>();
    __syncthreads();

    // join the warps: O, m and l of each in shared memory
    float* so = (float*)sm;
    float* sml = so + kWarps * 16 * C::kPitch;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        const int r = lane / 4 + 8 * h;
        if (lane % 4 == 0) {
            sml[(warp * 16 + r) * 2] = m[h];
            sml[(warp * 16 + r) * 2 + 1] = l[h];
        }
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
            *reinterpret_cast<float2*>(so + (warp * 16 + r) * C::kPitch + n * 8 + (lane % 4) * 2) =
                make_float2(o[n][2 * h], o[n][2 * h + 1]);
    }
    __syncthreads();
    const int rows = min(16, g.rows - b.row0);
    constexpr int kQuads = DP / 4;
    for (int i = threadIdx.x; i < rows * kQuads; i += kWarps * 32) {
        const int r = i / kQuads, d = i % kQuads * 4;
        float top = -CUDART_INF_F, mw[kWarps];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            mw[w] = sml[(w * 16 + r) * 2];
            top = mafat_attn::max_nan(top, mw[w]);
        }
        const float off = top == -CUDART_INF_F ? 0.f : -top * a.scale_log2;
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float x = mafat_attn::exp2_fast(fmaf(mw[w], a.scale_log2, off));
            sum = fmaf(x, sml[(w * 16 + r) * 2 + 1], sum);
            const float4 u = *reinterpret_cast<const float4*>(so + (w * 16 + r) * C::kPitch + d);
            v.x = fmaf(x, u.x, v.x);
            v.y = fmaf(x, u.y, v.y);
            v.z = fmaf(x, u.z, v.z);
            v.w = fmaf(x, u.w, v.w);
        }
        const mafat_attn::Out out(a, g, b, mafat_attn::Row(a, g, b, b.row0 + r));
        if (d == 0) mafat_attn::store_lse(a, out, top, sum);
        if (d >= a.dim) continue;
        const float inv = mafat_attn::inverse_sum(sum);
        v.x *= inv;
        v.y *= inv;
        v.z *= inv;
        v.w *= inv;
        if (a.parts == 1)
            *reinterpret_cast<uint2*>((__nv_bfloat16*)a.out + out.o + d) = make_uint2(pack(v.x, v.y), pack(v.z, v.w));
        else
            *reinterpret_cast<float4*>(a.part_o + out.part * a.dim + d) = v;
    }
    mafat_attn::launch_end(a);
}

template <int DP>
cudaError_t launch(const MafatAttnArgs& a, cudaStream_t s) {
    int blocks = 0;
    for (int i = 0; i < a.n_seg; ++i) blocks += a.seg[i].blocks;
    return mafat_launch_overlapped(attn_rows_kernel<DP>, blocks, kWarps * 32, Cfg<DP>::kSmem, s, a);
}
template <int DP>
cudaError_t prepare() {
    return cudaFuncSetAttribute(attn_rows_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<DP>::kSmem);
}

}  // namespace

int mafat_attn_rows_keys() { return kBN; }

cudaError_t mafat_launch_attn_rows(const MafatAttnArgs& a, cudaStream_t s) {
    return a.dim <= 64 ? launch<64>(a, s) : launch<128>(a, s);
}

cudaError_t mafat_prepare_attn_rows() {
    const cudaError_t e = prepare<64>();
    return e != cudaSuccess ? e : prepare<128>();
}
