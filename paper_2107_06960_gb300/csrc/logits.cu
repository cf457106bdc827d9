// What requests ask of their next token, for each row of logits:
//   x = logit;  said: x / r (x > 0) or x r;  x - f n - p [n > 0];  x + bias;  -inf where the grammar's mask forbids,
// in fp32, rounded once.
//
// Bound by reading a row and writing it once: nearly all logits pass as they are, or as the mask's -inf.  A CTA has a run of
// the vocabulary for some rows of a request.  While the first row's logits are on their way it goes over what the request
// has said, drafted and biased, and notes what falls into its run in a table in shared memory, a word a token, and each token
// there once in a list; when all rows have passed, the tokens of the list are written again, a lane each.  (Common tokens are
// neighbours in a vocabulary: in the pass over all of them their divisions fell to a few warps.)  The table's sums are
// of whole numbers, so that their order does not matter.
//
// 64 trees of 16 nodes, 131072 bf16 logits each, half of them with a mask, 2048 said: 100 us or 5.4 TB/s; with each next row in registers
// 103, with two on their way in shared memory as it is.  20 x 35 rows of 119808 from bf16 to fp32, 140 said: 80 us or 6.2 TB/s.  7 rows
// of 50001 fp32 with 20000 said: 7.7 us, going over the lists.  16 rows of 32000 bf16 with 512 said: 3.6 us, a launch and three round trips.
#include <cuda_bf16.h>
#include <math_constants.h>

#include "decode.h"
#include "row_common.cuh"

#include <algorithm>

namespace {

constexpr int kMostRows = 16;  // of a CTA
constexpr int kFewDrafts = 128;  // of a request, that a thread goes over for each token that it writes
constexpr int kAhead = 8;  // tokens of a history that a thread asks for at once
// a token's word: entry of the biases (number + 1) | a draft has it | the prompt has it | how often the answer has it
constexpr int kBiasShift = 20;
constexpr uint32_t kDraft = 1u << 19, kPrompt = 1u << 18, kCount = kPrompt - 1u;

__device__ __forceinline__ float wide(float x) { return x; }
__device__ __forceinline__ float wide(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void narrow(float* p, float x) { *p = x; }
__device__ __forceinline__ void narrow(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// Logits on their way to 16 bytes of `out`, at once where `whole`; MASK: those without a bit in `allowed` as -inf
template <bool MASK, class T>
__device__ __forceinline__ void put(float* out, const Vec<T, 4>& v, uint32_t allowed, bool whole) {
    float x[4];
    v.get(x);
    if constexpr (MASK)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if ((allowed >> j & 1u) == 0u) x[j] = -CUDART_INF_F;
    if (whole) {
        Vec<float, 4>::store(out, x);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = x[j];
    }
}
template <bool MASK>
__device__ __forceinline__ void put(__nv_bfloat16* out, const Vec<__nv_bfloat16, 8>& v, uint32_t allowed, bool whole) {
    uint32_t w[4] = {v.u.x, v.u.y, v.u.z, v.u.w};
    if constexpr (MASK)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t two = allowed >> (2 * j), keep = (two & 1u) * 0xffffu + (two & 2u) * 0x7fff8000u;
            w[j] = (w[j] & keep) | (0xff80ff80u & ~keep);  // -inf
        }
    if (whole) {
        *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            out[2 * j] = __ushort_as_bfloat16((unsigned short)w[j]);
            out[2 * j + 1] = __ushort_as_bfloat16((unsigned short)(w[j] >> 16));
        }
    }
}

__device__ __forceinline__ bool allows(const uint32_t* mask, int token) {
    return !mask || (mask[token >> 5] >> (token & 31) & 1u) != 0u;
}

// A CTA's run of a row: THREADS threads of accesses of V tokens, 16 bytes of the output, in all of N * 16 bytes of the input.  It
// starts on a whole access of the input, before the row's first token where that does not.  (With accesses of 16 bytes of the input
// and 32 of the output, in two halves, 20 x 35 rows of 119808 from bf16 to fp32 took 98 us instead of 80.)
template <class T, class O, int THREADS, int N>
struct Run {
    static constexpr int V = 16 / sizeof(O), kBytes = V * sizeof(T), A = N * 16 / kBytes, kTokens = THREADS * A * V, kStep = THREADS * V;
    // Rows that are asked for before they are needed, in shared memory (none: the next one alone, in registers)
    static constexpr int kAsked = THREADS * N <= 1024 ? 2 : 0;
    static_assert(kTokens <= 65536 && kStep % 32 == 0, "places in 16 bits; a thread's accesses begin at one bit of a word");
    int first, mine, vocab;  // the run's first token, that of the thread's first access
    bool inner;              // all of the run are the row's
    __device__ __forceinline__ Run(const MafatLogitsArgs& a, int run, const T* in)
        : first(run * kTokens - (int)((uintptr_t)in / sizeof(T) % V)), mine(first + (int)threadIdx.x * V), vocab(a.vocab),
          inner(first >= 0 && first + kTokens <= a.vocab) {}
    __device__ __forceinline__ bool inside(int i) const { return inner || (mine + i * kStep >= 0 && mine + i * kStep + V <= vocab); }
    __device__ __forceinline__ void load(const T* in, Vec<T, V> (&v)[A]) const {
#pragma unroll
        for (int i = 0; i < A; ++i) v[i].load(in + mine + i * kStep, inside(i));
    }
    // A later row's on their way to the thread's places in shared memory.
    __device__ __forceinline__ void ask(const T* in, uint32_t to, bool on) const {
#pragma unroll
        for (int i = 0; i < A; ++i)
            if (on && inside(i)) {
                if constexpr (kBytes == 16)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * THREADS * kBytes), "l"(in + mine + i * kStep) : "memory");
                else
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to + i * THREADS * kBytes), "l"(in + mine + i * kStep) : "memory");
            }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // the words with the thread's bits of a mask; from the second on where an access can pass a word's end
    struct Bits {
        uint32_t lo[A], hi[A];
    };
    __device__ __forceinline__ void look(const uint32_t* mask, Bits& bits) const {
        const uint32_t* words = mask + (mine >> 5);
        const bool two = (mine & 31) + V > 32;
#pragma unroll
        for (int i = 0; i < A; ++i) {
            const bool on = mask && inside(i);
            bits.lo[i] = on ? words[i * (kStep / 32)] : 0u;
            bits.hi[i] = on && two ? words[i * (kStep / 32) + 1] : 0u;
        }
    }
    template <bool MASK>
    __device__ __forceinline__ void pass(const T* in, O* out, const uint32_t* mask, const Vec<T, V> (&v)[A], const Bits& bits) const {
        const bool whole = ((uintptr_t)(out + first) & 15u) == 0u;
#pragma unroll
        for (int i = 0; i < A; ++i) {
            const int e = mine + i * kStep;
            if (inside(i)) {
                put<MASK>(out + e, v[i], MASK ? __funnelshift_r(bits.lo[i], bits.hi[i], (uint32_t)mine & 31u) : 0u, whole);
            } else if (e < vocab) {
#pragma unroll 1
                for (int k = max(e, 0); k < min(e + V, vocab); ++k) narrow(out + k, !MASK || allows(mask, k) ? wide(in[k]) : -CUDART_INF_F);
            }
        }
    }
};

// MANY: of drafts so many that a row's are counted in the table, which then is that row's; else a drafted token's count is made where it
// is written, going over all drafts.
template <class T, class O, int THREADS, int N, int BLOCKS, bool MANY>
__global__ void __launch_bounds__(THREADS, BLOCKS) logits_kernel(const __grid_constant__ MafatLogitsArgs a) {
    using S = Run<T, O, THREADS, N>;
    // Where histories are long the list is made of the whole table, not with each token, whose addition then has to come back
    // first: 7 rows of 50001 with 20000 said 7.7 us instead of 10.3, 95 of 128890 with 21842 and masks 53 instead of 59, as the rows passed then (16 rows of 32000 with
    // 512, in 256 threads: 3.8 instead of 3.6).
    constexpr bool kScan = THREADS > 256;
    constexpr int kAsked = S::kAsked;
    constexpr int kRow = THREADS * S::A;  // places of a row
    using Places = Vec<T, S::V>;
    extern __shared__ __align__(16) uint4 shared[];
    Places* const asked = (Places*)shared + threadIdx.x;  // the thread's of later rows
    uint32_t* const table = (uint32_t*)((Places*)shared + (a.rows_of_cta > 1 ? kAsked * kRow : 0));
    uint16_t* list = (uint16_t*)(table + S::kTokens);
    __shared__ int listed, masks[kMostRows];
    const int tid = threadIdx.x;
    // All requests' first runs, then their second ones: CTAs of one run have alike much to write again, which tends to be most where
    // a vocabulary begins, and the last CTAs short.  21 x 8 rows of 123520 with 8271 said 38.8 us, request by request 42.6, as the rows passed then.
    const uint32_t run = a.items_div.div(blockIdx.x), i0 = blockIdx.x - run * a.items_div.d, b = a.groups_div.div(i0);
    const int t0 = (int)(i0 - b * a.groups_div.d) * a.rows_of_cta, rows = min(a.rows_of_cta, a.n_q - t0);
    const int64_t row0 = (int64_t)b * a.n_q + t0;
    const T* in = (const T*)a.logits + row0 * a.in_s;
    O* out = (O*)a.out + row0 * a.out_s;
    const S s(a, (int)run, in);
    launch_wait();
    launch_next();
    Places v[S::A];
    if (a.pass) {
        s.load(in, v);
#pragma unroll
        for (int r = 1; r <= kAsked; ++r) s.ask(in + r * a.in_s, (uint32_t)__cvta_generic_to_shared(asked + (r - 1) * kRow), r < rows);
    }
    // what the CTA needs of the request is asked for together: the first of each list before the first barrier
    const bool any = a.tokens || a.drafts || a.bias_ids;
    const int32_t* bias_ids = a.bias_ids + (int64_t)b * a.bias_s;
    const int32_t* drafts = a.drafts + (int64_t)b * a.n_q;
    int32_t said[kAhead];
    auto look = [&](int from) {  // up to the room, so that the length is not waited for
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = from + i * THREADS + tid;
            said[i] = a.tokens && k < a.room ? a.tokens[(int64_t)b * a.room + k] : -1;
        }
    };
    look(0);
    const int32_t bias_id = a.bias_ids && tid < a.n_bias ? bias_ids[tid] : -1, draft = a.drafts && tid < a.n_q ? drafts[tid] : -1;
    int len = 0, prompt = 0;
    if (a.tokens) {
        len = a.lengths ? min(max(a.lengths[b], 0), a.room) : a.room;
        prompt = a.prompt ? a.prompt[b] : 0;
    }
    if (tid < rows) {  // the number of each row's mask, or -1
        int64_t m = -1;
        if (a.masks) m = a.mask_rows ? a.mask_rows[row0 + tid] : row0 + tid;
        masks[tid] = m < a.n_masks ? (int)m : -1;
    }
    if (any) {
#pragma unroll
        for (int i = tid * 4; i < S::kTokens; i += THREADS * 4) *reinterpret_cast<uint4*>(table + i) = make_uint4(0u, 0u, 0u, 0u);
        if (tid == 0) listed = 0;
    }
    __syncthreads();
    auto mask_of = [&](int t) -> const uint32_t* { return masks[t] < 0 ? nullptr : a.masks + (int64_t)masks[t] * a.mask_words; };
    typename S::Bits bits;
    s.look(a.pass ? mask_of(0) : nullptr, bits);
    auto place = [&](int32_t id) { return (uint32_t)id - (uint32_t)s.first; };  // kTokens and more: elsewhere
    if (any) {
        auto note = [&](uint32_t at, uint32_t was) {
            if (!kScan && was == 0u) list[atomicAdd(&listed, 1)] = (uint16_t)at;
        };
        if (a.bias_ids) {
            for (int i = tid; i < a.n_bias; i += THREADS) {
                const uint32_t at = place(i == tid ? bias_id : bias_ids[i]);
                if (at < (uint32_t)S::kTokens) note(at, atomicMax(table + at, (uint32_t)(i + 1) << kBiasShift));  // the last of an id
            }
            __syncthreads();
        }
        for (int from = 0; from < len; from += kAhead * THREADS) {
            if (from > 0) look(from);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int k = from + i * THREADS + tid;
                const uint32_t at = place(said[i]);
                if (at < (uint32_t)S::kTokens && k < len)
                    note(at, k < prompt ? atomicOr(table + at, kPrompt) : atomicAdd(table + at, 1u));
            }
        }
        if (a.drafts)
            for (int i = tid; i < a.n_q; i += THREADS) {
                const uint32_t at = place(i == tid ? draft : drafts[i]);
                if (at < (uint32_t)S::kTokens) note(at, atomicOr(table + at, kDraft));
            }
    }
    // The noted tokens of all rows, kTogether of a thread at a time.  The logits of the first ones are asked for before
    // the rows pass.
    constexpr int kTogether = N < 4 ? N : 4;
    struct Patch {
        float x[kTogether];
        int at[kTogether], row[kTogether];  // row: negative where there is nothing to write
    } patch;
    int t = 0, i = tid, n = 0;
    auto fetch = [&]() {
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            while (i >= n && t < rows) i -= n, ++t;
            patch.row[u] = -1;
            if (t < rows) {
                patch.at[u] = list[i];
                const int token = s.first + patch.at[u];
                // an id may be past the row's ends, and still in the run
                if (token >= 0 && token < a.vocab) {
                    patch.x[u] = wide(in[t * a.in_s + token]);
                    if (allows(mask_of(t), token)) patch.row[u] = t;
                }
            }
            i += THREADS;
        }
    };
    if (any) {
        __syncthreads();  // table and list are there
        if constexpr (kScan) {
            uint32_t hits = 0u;  // of the thread's words
            static_assert(S::A * S::V <= 32, "a bit each");
#pragma unroll
            for (int k = 0; k < S::A * S::V / 4; ++k) {
                const uint4 w = *reinterpret_cast<const uint4*>(table + (k * THREADS + tid) * 4);
                hits |= ((w.x ? 1u : 0u) | (w.y ? 2u : 0u) | (w.z ? 4u : 0u) | (w.w ? 8u : 0u)) << (4 * k);
            }
            const int mine = __popc(hits);
            if (__any_sync(0xffffffffu, mine)) {
                int upto = mine;
#pragma unroll
                for (int w = 1; w < 32; w *= 2) {
                    const int x = __shfl_up_sync(0xffffffffu, upto, w);
                    if (tid % 32 >= w) upto += x;
                }
                int at = 0;
                if (tid % 32 == 31) at = atomicAdd(&listed, upto);
                at = __shfl_sync(0xffffffffu, at, 31) + upto - mine;
                for (uint32_t left = hits; left; left &= left - 1u) {
                    const int bit = __ffs(left) - 1;
                    list[at++] = (uint16_t)((bit / 4 * THREADS + tid) * 4 + bit % 4);
                }
            }
            __syncthreads();
        }
        n = listed;
        if (n == 0) t = rows;
        if constexpr (!MANY) fetch();
    }
    if (a.pass) {
#pragma unroll 1
        for (int r = 0;; ++r) {
            const T* from = in + r * a.in_s;
            O* to = out + r * a.out_s;
            Places next[S::A];
            typename S::Bits next_bits;
            if (r + 1 < rows) {
                if constexpr (kAsked == 0) s.load(from + a.in_s, next);
                s.look(mask_of(r + 1), next_bits);
            }
            const uint32_t* mask = mask_of(r);
            if (mask)
                s.template pass<true>(from, to, mask, v, bits);
            else
                s.template pass<false>(from, to, mask, v, bits);
            if (r + 1 == rows) break;
            bits = next_bits;
            if constexpr (kAsked > 0) {
                Places* at = asked + r % kAsked * kRow;
                asm volatile("cp.async.wait_group %0;" ::"n"(kAsked - 1) : "memory");
#pragma unroll
                for (int k = 0; k < S::A; ++k) v[k] = at[k * THREADS];
                // its places are free: what was read is in registers when the copy is asked for
                s.ask(from + (1 + kAsked) * a.in_s, (uint32_t)__cvta_generic_to_shared(at), r + 1 + kAsked < rows);
            } else {
#pragma unroll
                for (int k = 0; k < S::A; ++k) v[k] = next[k];
            }
        }
    }
    if (n == 0) return;
    const float repetition = a.repetition ? a.repetition[b] : 1.f, presence = a.presence ? a.presence[b] : 0.f,
                frequency = a.frequency ? a.frequency[b] : 0.f;
    const float* bias = a.bias + (int64_t)b * a.bias_s;
    const uint32_t* tree = a.tree + (int64_t)b * a.tree_s;
    auto write = [&](int row, int at, float x, uint32_t drafted) {
        const uint32_t word = table[at], count = (word & kCount) + drafted;
        float y = x;
        if (count > 0u || (word & kPrompt)) y = y > 0.f ? y / repetition : y * repetition;
        y -= frequency * (float)count;
        if (count > 0u) y -= presence;
        if (word >> kBiasShift) y += bias[(word >> kBiasShift) - 1u];
        narrow(out + row * a.out_s + s.first + at, y);
    };
    if constexpr (MANY) {
        // From one row to the next a chain has a draft more; of a tree all are looked at, those that the row before had and this one
        // has not fall away.
#pragma unroll 1
        for (int row = 0; row < rows; ++row) {
            const int own = t0 + row;
            const uint32_t* way = a.tree ? tree + (int64_t)own * a.tree_words : nullptr;
            const int from = a.tree || row == 0 ? 0 : own, end = a.tree ? a.n_q : own + 1;
            for (int j = from + tid; j < end; j += THREADS) {
                const uint32_t at = place(drafts[j]);
                if (at >= (uint32_t)S::kTokens) continue;
                const bool now = !way || (way[j / 32] >> (j % 32) & 1u), was = way && row > 0 && ((way - a.tree_words)[j / 32] >> (j % 32) & 1u);
                if (now != was) atomicAdd(table + at, now ? 1u : 0xffffffffu);
            }
            __syncthreads();  // the row's counts are there, and before the first row what is written over
            const uint32_t* mask = mask_of(row);
            for (int k = tid; k < n; k += THREADS) {
                const int token = s.first + list[k];
                if (token >= 0 && token < a.vocab && allows(mask, token)) write(row, list[k], wide(in[row * a.in_s + token]), 0u);
            }
            __syncthreads();
        }
        return;
    }
    __syncthreads();  // what is written over is there
#pragma unroll 1
    for (;;) {
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int row = patch.row[u];
            if (row < 0) continue;
            uint32_t drafted = 0u;
            if (table[patch.at[u]] & kDraft) {  // those that the row's bits name, or up to its own
                const int token = s.first + patch.at[u];
                const uint32_t* way = a.tree ? tree + (int64_t)(t0 + row) * a.tree_words : nullptr;
                const int end = way ? a.n_q : t0 + row + 1;
                for (int j = 0; j < end; ++j) drafted += drafts[j] == token && (!way || (way[j / 32] >> (j % 32) & 1u));
            }
            write(row, patch.at[u], patch.x[u], drafted);
        }
        if (t >= rows) break;
        fetch();
    }
}

bool noted(const MafatLogitsArgs& a) { return a.tokens || a.drafts || a.bias_ids; }

// A request's rows are shared by as many CTAs as leave `least` in all, so that the table serves several rows.
template <class T, class O, int THREADS, int N, int BLOCKS, bool MANY = false>
cudaError_t launch(MafatLogitsArgs& a, int64_t batch, int64_t least, cudaStream_t s) {
    using S = Run<T, O, THREADS, N>;
    // rows that start alike share a CTA; a row may start V - 1 tokens late
    const bool alike = a.in_s % S::V == 0;
    const int late = alike && (uintptr_t)a.logits % S::kBytes == 0 ? 0 : S::V - 1;
    const int64_t runs = ((int64_t)a.vocab + late + S::kTokens - 1) / S::kTokens;
    int rows = alike ? kMostRows : 1;
    while (rows > 1 && (rows >= 2 * a.n_q || batch * ((a.n_q + rows - 1) / rows) * runs < least)) rows /= 2;
    const int64_t groups = (a.n_q + rows - 1) / rows;
    a.rows_of_cta = rows;
    a.items_div = MafatDiv((uint32_t)(batch * groups));
    a.groups_div = MafatDiv((uint32_t)groups);
    const int64_t listed = (a.tokens ? a.room : 0) + (int64_t)(a.drafts ? a.n_q : 0) + (a.bias_ids ? a.n_bias : 0);
    const size_t ahead = rows > 1 ? S::kAsked * THREADS * N * 16 : 0;
    const size_t smem = ahead + (noted(a) ? S::kTokens * 4 + (std::min<int64_t>(S::kTokens, listed) * 2 + 15) / 16 * 16 : 0);
    if (smem > 40 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(logits_kernel<T, O, THREADS, N, BLOCKS, MANY>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   S::kAsked * THREADS * N * 16 + S::kTokens * 6);
        if (e != cudaSuccess) return e;
    }
    return mafat_launch_overlapped(logits_kernel<T, O, THREADS, N, BLOCKS, MANY>, (unsigned)(batch * groups * runs), THREADS, smem, s, a);
}

// Each CTA goes over the whole history: the longer that is, the more threads it has, and the more tokens where there are many
// logits.  256, 512 and 1024 threads (1024 with one access each, with four), in us:
//   64 x 16 rows of 131072 bf16, 2048 said          94.4, 108, 114, 119      16 rows of 32000 bf16, 512 said   3.3, 4.0, 4.3, 9.8
//   102 rows of 111872 bf16, 6305 said             28.5, 27.1, 41.3, 32.7    4 x 27 of 8892 fp32, 5139        12.7,  9.3,  9.7,  9.3
//   7 rows of 50001 fp32, 20000 said               17.6,  8.4,  7.2, 11.2    57 of 25809 bf16, 24721          30.0, 16.8, 15.3, 21.2
//   95 rows of 128890 fp32, 21842 said             90.6, 65.9, 98.8, 46.5    40 x 36 of 21617 bf16, 8686       145,  127,  182,  154
//   5 x 24 rows of 40256 bf16, 16270 said          32.8, 22.0, 20.8, 29.3    15 x 24 of 11386 bf16, 13653     37.5, 29.0, 36.1, 44.0
// (without masks and biases, to fp32 but for the first)
// 2048 ids are one round of kAhead for 256 threads; the other steps lie between the calls above.
template <class T, class O>
cudaError_t launch_all(MafatLogitsArgs& a, int64_t batch, cudaStream_t s) {
    constexpr int kSms = 152;
    const int said = a.tokens ? a.room : 0;
    // Drafts counted in the table, and for each token that is written, in us; all are written in each row, and a token's drafts gone
    // over take as long as there are drafts.  Chains and trees, rows of 32000 bf16: 16 x 65 drafts 31, 32 and 32, 37; 8 x 128
    // 31, 32 and 34, 45; 4 x 256 31, 33 and 38, 62; 2048 87, 136 and 707, 2152; fp32: 16 x 96 87, 90 and 70, 76; 8 x 128 53, 55 and 51, 59;
    // 4 x 256 54, 57 and 54, 73.  4096 of 8192 bf16: 83, 132 in 512 threads, 160, 228 in 256; 4162, 13666.
    if (a.drafts && a.n_q > kFewDrafts)
        return said <= 2048 && a.n_q <= 2048 ? launch<T, O, 256, 2, 5, true>(a, batch, 4 * 5 * kSms, s) : launch<T, O, 512, 2, 2, true>(a, batch, 4 * kSms, s);
    if (said <= 2048) return launch<T, O, 256, 2, 5>(a, batch, 4 * 5 * kSms, s);
    const int64_t bytes = batch * a.n_q * a.vocab * (int64_t)sizeof(T);
    if (said > 8192 && bytes <= 4 << 20) return launch<T, O, 1024, 1, 1>(a, batch, kSms * 9 / 10, s);
    if (said > 16384 && bytes > 32 << 20) return launch<T, O, 1024, 4, 1>(a, batch, 4 * kSms, s);
    return launch<T, O, 512, 2, 2>(a, batch, 4 * kSms, s);
}

}  // namespace

int mafat_logits_run() { return 256 * 2 * 4; }

cudaError_t mafat_launch_logits(MafatLogitsArgs& a, bool bf16, bool out_bf16, int64_t batch, cudaStream_t s) {
    if (!bf16) return launch_all<float, float>(a, batch, s);
    return out_bf16 ? launch_all<__nv_bfloat16, __nv_bfloat16>(a, batch, s) : launch_all<__nv_bfloat16, float>(a, batch, s);
}
