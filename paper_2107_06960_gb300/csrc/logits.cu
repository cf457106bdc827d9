// What requests ask of their next token, for each row of logits:
//   x = logit;  said: x / r (x > 0) or x r;  x - f n - p [n > 0];  x + bias;  -inf where the grammar's mask forbids,
// in fp32, rounded once.
//
// Bound by reading a row and writing it once.  A CTA has a run of a row's tokens.  Their logits are asked for first; while
// they are on their way, the CTA goes over what the request has said and notes what falls into its run in a table in shared
// memory, a word a token: how often the answer has it, whether the prompt does, and its bias.  The sums are of whole numbers, so
// that their order does not matter.
#include <cuda_bf16.h>
#include <math_constants.h>

#include "decode.h"
#include "row_common.cuh"

namespace {

constexpr int kThreads = 256;
// a token's word: entry of the biases (number + 1) | the prompt has it | how often the answer has it
constexpr int kBiasShift = 20;
constexpr uint32_t kPrompt = 1u << 19, kCount = kPrompt - 1u;

struct Row {
    float repetition, presence, frequency;
    const float* bias;

    __device__ __forceinline__ float adjust(float x, uint32_t word) const {
        if (word == 0u) return x;
        const uint32_t n = word & kCount;
        if ((word & (kPrompt | kCount)) != 0u) x = x > 0.f ? x / repetition : x * repetition;
        x -= frequency * (float)n;
        if (n > 0u) x -= presence;
        if (word >> kBiasShift != 0u) x += bias[(word >> kBiasShift) - 1u];
        return x;
    }
};

template <int V>
__device__ __forceinline__ void store_all(float* p, const float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
}
template <int V>
__device__ __forceinline__ void store_all(__nv_bfloat16* p, const float (&v)[V]) { Vec<__nv_bfloat16, V>::store(p, v); }

__device__ __forceinline__ float wide(float x) { return x; }
__device__ __forceinline__ float wide(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void narrow(float* p, float x) { *p = x; }
__device__ __forceinline__ void narrow(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// N accesses of 16 bytes a thread
template <class T, class O, int N>
__global__ void __launch_bounds__(kThreads) logits_kernel(const __grid_constant__ MafatLogitsArgs a, MafatDiv chunks) {
    constexpr int V = 16 / sizeof(T), kRun = kThreads * N * V;
    __shared__ __align__(16) uint32_t table[kRun];
    const uint32_t row = chunks.div(blockIdx.x), chunk = blockIdx.x - row * chunks.d;
    const uint32_t b = a.n_q_div.div(row), t = row - b * (uint32_t)a.n_q;
    const T* in = (const T*)a.logits + (int64_t)row * a.in_s;
    O* out = (O*)a.out + (int64_t)row * a.out_s;
    // the run starts on 16 bytes of the input, before the row's first token where that is not there
    const int first = (int)(chunk * kRun) - (int)((uintptr_t)in / sizeof(T) % V);
    const int tid = threadIdx.x;
    launch_wait();
    launch_next();
    Vec<T, V> v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = first + (i * kThreads + tid) * V;
        v[i].load(in + e, e >= 0 && e + V <= a.vocab);
    }
#pragma unroll
    for (int i = tid; i < kRun / 4; i += kThreads) *reinterpret_cast<uint4*>(table + 4 * i) = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    Row r{1.f, 0.f, 0.f, a.bias ? a.bias + (int64_t)b * a.bias_s : nullptr};
    if (a.repetition) r.repetition = a.repetition[b];
    if (a.presence) r.presence = a.presence[b];
    if (a.frequency) r.frequency = a.frequency[b];
    if (a.bias_ids) {
        const int32_t* ids = a.bias_ids + (int64_t)b * a.bias_s;
        for (int i = tid; i < a.n_bias; i += kThreads) {
            const uint32_t at = (uint32_t)ids[i] - (uint32_t)first;
            if (at < (uint32_t)kRun) atomicMax(table + at, (uint32_t)(i + 1) << kBiasShift);  // the last of an id
        }
        __syncthreads();
    }
    if (a.tokens) {
        const int32_t* ids = a.tokens + (int64_t)b * a.room;
        const int len = a.lengths ? min(max(a.lengths[b], 0), a.room) : a.room;
        const int prompt = a.prompt ? a.prompt[b] : 0;
#pragma unroll 4
        for (int i = tid; i < len; i += kThreads) {
            const uint32_t at = (uint32_t)ids[i] - (uint32_t)first;
            if (at >= (uint32_t)kRun) continue;
            if (i < prompt)
                atomicOr(table + at, kPrompt);
            else
                atomicAdd(table + at, 1u);
        }
    }
    if (a.drafts) {
        const uint32_t* bits = a.tree ? a.tree + (int64_t)b * a.tree_s + (int64_t)t * a.tree_words : nullptr;
        for (int i = tid; i < a.n_q; i += kThreads) {
            const uint32_t at = (uint32_t)a.drafts[(int64_t)b * a.n_q + i] - (uint32_t)first;
            const bool held = bits ? (bits[i / 32] >> (i % 32) & 1u) != 0u : i <= (int)t;
            if (held && at < (uint32_t)kRun) atomicAdd(table + at, 1u);
        }
    }
    const uint32_t* mask = nullptr;
    if (a.masks) {
        const int64_t m = a.mask_rows ? a.mask_rows[row] : (int64_t)row;
        if (m >= 0 && m < a.n_masks) mask = a.masks + m * a.mask_words;
    }
    __syncthreads();
    const bool whole = ((uintptr_t)(out + first) & 15u) == 0u;  // the output can be written 16 bytes at a time
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int at = (i * kThreads + tid) * V, e = first + at;
        if (e >= a.vocab) break;
        if (e >= 0 && e + V <= a.vocab) {
            uint32_t allowed = 0xffffffffu;
            if (mask) {
                const uint32_t lo = mask[e >> 5], hi = (e & 31) + V > 32 ? mask[(e >> 5) + 1] : 0u;
                allowed = __funnelshift_r(lo, hi, (uint32_t)e & 31u);
            }
            float x[V];
            v[i].get(x);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[j] = r.adjust(x[j], table[at + j]);
                if ((allowed >> j & 1u) == 0u) x[j] = -CUDART_INF_F;
            }
            if (whole) {
                store_all<V>(out + e, x);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) narrow(out + e + j, x[j]);
            }
        } else {
            for (int j = 0; j < V; ++j) {
                const int k = e + j;
                if (k < 0 || k >= a.vocab) continue;
                float x = r.adjust(wide(in[k]), table[at + j]);
                if (mask && (mask[k >> 5] >> (k & 31) & 1u) == 0u) x = -CUDART_INF_F;
                narrow(out + k, x);
            }
        }
    }
}

template <class T, class O, int N>
cudaError_t launch(const MafatLogitsArgs& a, int64_t rows, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T), kRun = kThreads * N * V;
    const int64_t chunks = ((int64_t)a.vocab + V - 1 + kRun - 1) / kRun;  // a row may start V - 1 tokens late
    return mafat_launch_overlapped(logits_kernel<T, O, N>, (unsigned)(rows * chunks), kThreads, 0, s, a, MafatDiv((uint32_t)chunks));
}
template <class T, class O>
cudaError_t launch_n(const MafatLogitsArgs& a, int64_t rows, cudaStream_t s) {
    return launch<T, O, 4>(a, rows, s);
}

}  // namespace

int mafat_logits_run() { return kThreads * 4; }

cudaError_t mafat_launch_logits(const MafatLogitsArgs& a, bool bf16, bool out_bf16, int64_t rows, cudaStream_t s) {
    if (!bf16) return launch_n<float, float>(a, rows, s);
    return out_bf16 ? launch_n<__nv_bfloat16, __nv_bfloat16>(a, rows, s) : launch_n<__nv_bfloat16, float>(a, rows, s);
}
