// Rotary positions: pair i of a head's rotated channels is turned by angle = position * frequency[i],
//   (a, b) -> m (a cos - b sin, a sin + b cos),
// and keys go, with their values, to the tokens' places in a cache.
//
// Bound by reading and writing queries, keys and values once.  A frequency is a 64-bit fraction of a turn: its product with the
// position, modulo 2^64, is the fraction past whole turns, to 2^-33 of a turn whatever the position; sine and
// cosine are taken of that fraction in fp32, on -1/2 .. 1/2.  A CTA has a few tokens with all their heads: their sines and
// cosines are made once, while the first channels are on their way.  A thread has the same pairs of one head after another.
//
// 8 x 2048 tokens of 32 query and 8 key heads of 128 channels, bf16, with their values: 63 us or 6.4 TB/s; a form whose
// threads made the sines of their own pairs before they asked for channels took 77.6.  64 tokens of as many heads: 2.4 us,
// a launch and two round trips (the tokens' positions, then their angles' table, beside the channels).
#include <cuda_bf16.h>

#include <algorithm>

#include "decode.h"
#include "row_common.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kMostTokens = 16;  // of a CTA, where there are heads enough
constexpr int kTogether = 4;     // accesses of pairs of a thread that are on their way together
constexpr int kMostPairs = 128;  // of a head
constexpr int kAngles = 2048;    // of a CTA's tokens

// room for a token's angles: in accesses of 16 bytes
__host__ __device__ constexpr int angles_of(int rot) { return (rot / 2 + 3) / 4 * 4; }

// 16 bytes that are copied as they are
template <class T>
struct alignas(16) Piece {
    T v[16 / sizeof(T)];
};

// V channels an access; an item is two accesses, of pairs of channels or of neighbours that stay.
template <class T, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads, 3) rotary_kernel(const __grid_constant__ MafatRotaryArgs a) {
    __shared__ __align__(16) float cosines[kAngles + 8], sines[kAngles + 8];
    const int tid = threadIdx.x, half = a.rot / 2, stride = angles_of(a.rot);
    const int64_t token0 = (int64_t)blockIdx.x * a.per_block;
    const int tokens = (int)min((int64_t)a.per_block, a.tokens - token0);
    // the thread's token, first head and item; threads past the last token have none
    const int row = (int)a.lanes_div.div((uint32_t)tid), lane = tid - row * a.lanes;
    const int slot = (int)a.steps_div.div((uint32_t)row), head0 = row - slot * a.steps;
    const bool mine = slot < tokens;
    const uint32_t token = (uint32_t)token0 + (uint32_t)(mine ? slot : 0);
    const int64_t b = a.n_q_div.div(token), t = (int64_t)token - b * a.n_q;
    launch_wait();
    launch_next();
    int64_t place = t;
    if (a.places) place = a.places[token];
    const bool kept = place >= 0 && place < a.room;  // there is a place for the key and the value
    const MafatRotaryTensor &tq = a.t[0], &tk = a.t[1], &tv = a.t[2];
    const int heads = mine ? tq.heads + tk.heads : 0;
    const bool turned = lane < a.pairs;
    const int c0 = !turned ? a.rot + (lane - a.pairs) * 2 * V : INTERLEAVED ? lane * 2 * V : lane * V;
    const int c1 = turned && !INTERLEAVED ? c0 + half : c0 + V;
    // of an odd number of neighbouring accesses the last item has one
    const bool two = c1 < (turned ? a.rot : a.dim);
    const T* q_in = (const T*)tq.in + b * tq.in_sb + t * tq.in_st;
    const T* k_in = (const T*)tk.in + b * tk.in_sb + t * tk.in_st;
    Vec<T, V> va[kTogether], vb[kTogether];
    auto load = [&](int h0) {
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int h = h0 + u * a.steps;
            const T* in = h < tq.heads ? q_in + h * tq.in_sh : k_in + (h - tq.heads) * tk.in_sh;
            va[u].load(in + c0, h < heads);
            vb[u].load(in + c1, h < heads && two);
        }
    };
    load(head0);
    for (int i = tid; i < tokens * half; i += kThreads) {
        const int of = (int)a.half_div.div((uint32_t)i), pair = i - of * half;
        const uint64_t turn = a.turns[pair] * (uint64_t)(int64_t)a.positions[token0 + of];
        const int32_t top = (int32_t)((turn + 0x80000000u) >> 32);  // of half turns 2^-31
        float s, c;
        sincospif((float)top * 0x1p-31f, &s, &c);
        cosines[of * stride + pair] = c * a.magnitude;
        sines[of * stride + pair] = s * a.magnitude;
    }
    if (mine && kept && tv.heads > 0) {  // values, 16 bytes at a time
        constexpr int kWide = 16 / sizeof(T);
        const T* in = (const T*)tv.in + b * tv.in_sb + t * tv.in_st;
        T* out = (T*)tv.out + b * tv.out_sb + place * tv.out_st;
#pragma unroll 1
        for (int h = head0; h < tv.heads; h += a.steps)
#pragma unroll 1
            for (int d = lane * kWide; d < a.dim; d += a.lanes * kWide * 2) {
                const int e = d + a.lanes * kWide;
                const Piece<T> x = *reinterpret_cast<const Piece<T>*>(in + h * tv.in_sh + d);
                Piece<T> y;
                if (e < a.dim) y = *reinterpret_cast<const Piece<T>*>(in + h * tv.in_sh + e);
                *reinterpret_cast<Piece<T>*>(out + h * tv.out_sh + d) = x;
                if (e < a.dim) *reinterpret_cast<Piece<T>*>(out + h * tv.out_sh + e) = y;
            }
    }
    __syncthreads();  // sines and cosines are there
    if (head0 >= heads) return;
    constexpr int kRun = V < 4 ? V : 4;
    float cs[V], sn[V];
    if (turned) {
#pragma unroll
        for (int j = 0; j < V; j += kRun) {  // past the last pair of an item with one access, up to 7 past the end: not used
            Vec<float, kRun> x, y;
            x.load(cosines + slot * stride + lane * V + j, true);
            y.load(sines + slot * stride + lane * V + j, true);
            float p[kRun], q[kRun];
            x.get(p), y.get(q);
#pragma unroll
            for (int k = 0; k < kRun; ++k) cs[j + k] = p[k], sn[j + k] = q[k];
        }
    }
    T* q_out = (T*)tq.out + b * tq.out_sb + t * tq.out_st;
    T* k_out = (T*)tk.out + b * tk.out_sb + place * tk.out_st;
#pragma unroll 1
    for (int h0 = head0;;) {
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int h = h0 + u * a.steps;
            if (h >= heads || (h >= tq.heads && !kept)) break;
            T* out = h < tq.heads ? q_out + h * tq.out_sh : k_out + (h - tq.heads) * tk.out_sh;
            if (!turned) {
                *reinterpret_cast<Vec<T, V>*>(out + c0) = va[u];
                if (two) *reinterpret_cast<Vec<T, V>*>(out + c1) = vb[u];
                continue;
            }
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
            Vec<T, V>::store(out + c0, y);
            if (two) Vec<T, V>::store(out + c1, z);
        }
        h0 += kTogether * a.steps;
        if (h0 >= heads) break;
        load(h0);
    }
}

template <class T, int V, bool INTERLEAVED>
cudaError_t launch(const MafatRotaryArgs& a, cudaStream_t s) {
    return mafat_launch_overlapped(rotary_kernel<T, V, INTERLEAVED>, (unsigned)((a.tokens + a.per_block - 1) / a.per_block), kThreads, 0, s, a);
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

int mafat_rotary_most_dim() { return 2 * kMostPairs; }

cudaError_t mafat_launch_rotary(MafatRotaryArgs& a, bool bf16, bool interleaved, cudaStream_t s) {
    // an access is inside the rotated channels, and inside each half of them
    const int run = interleaved ? a.rot : a.rot / 2, vec = std::min(run & -run, bf16 ? 8 : 4);
    a.pairs = interleaved ? (a.rot + 2 * vec - 1) / (2 * vec) : a.rot / 2 / vec;
    a.lanes = a.pairs + (a.dim - a.rot + 2 * vec - 1) / (2 * vec);
    a.lanes_div = MafatDiv((uint32_t)a.lanes);
    a.half_div = MafatDiv((uint32_t)a.rot / 2);
    // A thread has 8 heads of a token (8 x 2048 tokens of 32 + 8 heads of 128 channels: 62.8 us, with 4 heads 68.0, with 2 116.8),
    // fewer where that leaves CTAs for all SMs (5 x 676 tokens of 8 + 2 heads: a CTA an SM 8.1, two 8.7, four 12.6).  Of few heads more tokens
    // are a CTA's: 44 x 2615 tokens of 2 + 1 heads of 64 channels 27.4, 16 at a time 39.6; of 4 + 4 heads of 128, 4 x 3844, 23.6 and 20.
    constexpr int kHeads = 8, kSms = 152;
    const int heads = std::max(a.t[0].heads + a.t[1].heads, a.t[2].heads), rows = kThreads / a.lanes;
    const int angles = kAngles / angles_of(a.rot), most = heads < 4 ? angles : std::min(angles, kMostTokens);
    a.per_block = std::max(1, std::min(rows / ((heads + kHeads - 1) / kHeads), most));
    while (a.per_block > 1 && a.tokens < (int64_t)kSms * a.per_block) a.per_block = (a.per_block + 1) / 2;
    a.steps = std::min(heads, rows / a.per_block);
    a.steps_div = MafatDiv((uint32_t)a.steps);
    if (bf16) return interleaved ? launch_v<__nv_bfloat16, true>(a, vec, s) : launch_v<__nv_bfloat16, false>(a, vec, s);
    return interleaved ? launch_v<float, true>(a, vec, s) : launch_v<float, false>(a, vec, s);
}
