// Rotary positions: pair i of a head's rotated channels is turned by angle = position * frequency[i],
//   (a, b) -> m (a cos - b sin, a sin + b cos),
// and keys go, with their values, to the tokens' places in a cache.
//
// Bound by reading and writing queries, keys and values once.  A frequency is a 64-bit fraction of a turn: its product with the
// position, modulo 2^64, is the fraction past whole turns, to 2^-33 of a turn whatever the position; sine and
// cosine are taken of that fraction in fp32, on -1/2 .. 1/2.  A thread has V channels and their partners of a token, and turns
// those of one head after another by the same sines and cosines.
#include <cuda_bf16.h>

#include "decode.h"
#include "row_common.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kTogether = 4;  // heads whose loads are on their way together

// V channels that are copied as they are
template <class T, int V>
__device__ __forceinline__ void copy(T* out, const T* in) {
    struct alignas(sizeof(T) * V) Piece {
        T v[V];
    };
    *reinterpret_cast<Piece*>(out) = *reinterpret_cast<const Piece*>(in);
}

template <class T, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const __grid_constant__ MafatRotaryArgs a) {
    // the block's tensor and group of heads
    int group = blockIdx.y, which = 0;
    while (group >= a.t[which].groups) group -= a.t[which++].groups;
    const MafatRotaryTensor& x = a.t[which];
    const int slot = (int)a.lanes_div.div(threadIdx.x), lane = (int)threadIdx.x - slot * a.lanes;
    const int64_t token = (int64_t)blockIdx.x * a.per_block + slot;
    if (slot >= a.per_block || token >= a.tokens) return;
    const int64_t b = a.n_q_div.div((uint32_t)token), t = token - b * a.n_q;
    launch_wait();
    launch_next();
    const int64_t place = x.placed && a.places ? a.places[token] : t;
    if (place < 0 || (x.placed && place >= a.room)) return;
    const T* in = (const T*)x.in + b * x.in_sb + t * x.in_st;
    T* out = (T*)x.out + b * x.out_sb + place * x.out_st;
    const int h0 = group * a.per_group, h1 = min(h0 + a.per_group, x.heads);
    if (which == 2) {  // values, 16 bytes at a time
        constexpr int kWide = 16 / sizeof(T);
        for (int h = h0; h < h1; ++h)
            for (int c = lane * kWide; c < a.dim; c += a.lanes * kWide) copy<T, kWide>(out + h * x.out_sh + c, in + h * x.in_sh + c);
        return;
    }
    if (lane >= a.pairs) {  // channels that stay
        const int c = a.rot + (lane - a.pairs) * V;
        for (int h = h0; h < h1; ++h) copy<T, V>(out + h * x.out_sh + c, in + h * x.in_sh + c);
        return;
    }
    // an access has V pairs' first channels, and V on their second ones; neighbours: V / 2 pairs each
    const int c0 = INTERLEAVED ? lane * 2 * V : lane * V, c1 = INTERLEAVED ? c0 + V : c0 + a.rot / 2;
    float cs[V], sn[V];
    const int64_t position = a.positions[token];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int i = lane * V + j;
        // past the last pair where an odd number of them is interleaved
        const uint64_t turn = !INTERLEAVED || i < a.rot / 2 ? a.turns[i] * (uint64_t)position : 0u;
        const int32_t top = (int32_t)((turn + 0x80000000u) >> 32);  // of half turns 2^-31
        sincospif((float)top * 0x1p-31f, &sn[j], &cs[j]);
        sn[j] *= a.magnitude;
        cs[j] *= a.magnitude;
    }
    const bool second = !INTERLEAVED || c1 < a.rot;
#pragma unroll 1
    for (int h = h0; h < h1; h += kTogether) {
        Vec<T, V> va[kTogether], vb[kTogether];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const T* p = in + min(h + u, h1 - 1) * x.in_sh;
            va[u].load(p + c0, h + u < h1);
            vb[u].load(p + c1, h + u < h1 && second);
        }
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            if (h + u >= h1) break;
            float p[V], q[V], y[V], z[V];
            va[u].get(p);
            vb[u].get(q);
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int j = 0; j < V; j += 2) {
                    const int k = j / 2, l = V / 2 + j / 2;
                    y[j] = p[j] * cs[k] - p[j + 1] * sn[k];
                    y[j + 1] = p[j] * sn[k] + p[j + 1] * cs[k];
                    z[j] = q[j] * cs[l] - q[j + 1] * sn[l];
                    z[j + 1] = q[j] * sn[l] + q[j + 1] * cs[l];
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    y[j] = p[j] * cs[j] - q[j] * sn[j];
                    z[j] = p[j] * sn[j] + q[j] * cs[j];
                }
            }
            T* o = out + (h + u) * x.out_sh;
            Vec<T, V>::store(o + c0, y);
            if (second) Vec<T, V>::store(o + c1, z);
        }
    }
}

template <class T, int V, bool INTERLEAVED>
cudaError_t launch(const MafatRotaryArgs& a, cudaStream_t s) {
    const dim3 grid((unsigned)((a.tokens + a.per_block - 1) / a.per_block), a.t[0].groups + a.t[1].groups + a.t[2].groups);
    return mafat_launch_overlapped(rotary_kernel<T, V, INTERLEAVED>, grid, kThreads, 0, s, a);
}
template <class T, bool INTERLEAVED>
cudaError_t launch_v(const MafatRotaryArgs& a, int vec, cudaStream_t s) {
    if constexpr (sizeof(T) == 2)
        if (vec >= 8) return launch<T, 8, INTERLEAVED>(a, s);
    if (vec >= 4) return launch<T, 4, INTERLEAVED>(a, s);
    if (INTERLEAVED || vec >= 2) return launch<T, 2, INTERLEAVED>(a, s);
    if constexpr (!INTERLEAVED) return launch<T, 1, INTERLEAVED>(a, s);
}

}  // namespace

cudaError_t mafat_launch_rotary(const MafatRotaryArgs& a, bool bf16, bool interleaved, int vec, cudaStream_t s) {
    if (bf16) return interleaved ? launch_v<__nv_bfloat16, true>(a, vec, s) : launch_v<__nv_bfloat16, false>(a, vec, s);
    return interleaved ? launch_v<float, true>(a, vec, s) : launch_v<float, false>(a, vec, s);
}
