// Attention of many rows in bf16 on the tensor cores (tcgen05, sm_103a): tiles of 128 rows by 128 keys.
//
// For a tile of queries Q and each tile of keys K and values V of the CTA's part:
//   S = Q K^T;  b' = max(b, c max S);  P = 2^(c S - b');  O = 2^(b - b') O + P V;  l alike,
// with c = scale log2(e).  S and O are fp32 accumulators in tensor memory; b and l are fp32 registers
// of the thread that has the row.  P is rounded to bf16 for its product (l sums it unrounded) and written
// over S in tensor memory, from where the second product reads it; nothing of S leaves the SM.
//
// A CTA has SLOTS tiles of rows that read the same keys: while the softmax of one runs, the tensor
// core works for the other.  Warps: 8 for each of two slots (two threads a row, each half of the keys), 4 for a
// single one (a thread a row), one that issues the products, one
// that loads K and V by TMA into a ring of tiles, and one that zeroes the values past the length, since
// 0 x NaN would reach O.  With a mask the last two and a third instead copy the readable keys alone, one
// after another (cp.async): keys that are not readable cost no product.
//
// O is rescaled only where b' is more than 8 above the b in use (a power that cancels in O / l and
// leaves P at most 256, well inside bf16), so that few tiles touch O outside the products.  That, and weights in the
// scores' place in tensor memory, are published methods of attention on this hardware.
//
// Rows whose keys are a shared prefix and then their own are done in one launch where that is better (attention.cpp has
// the rule): the tiles of the prefix come first, each set with its own maps, length and partial last tile.
//
// Bound, for long sequences, by the softmax between the two products: with 128 channels the tensor pipe is busy 74 % of
// the time, with 64, whose products take half as long for the same exponentials, 50 %, the special function unit
// as much and the issue slots 63 %.  8 x 2048 tokens, 16 query and 4 key heads, 5776 keys: 480 us or 1.61 PFLOP/s with 128
// channels, 339 us or 1.14 with 64.  For few keys by the round trips of an item's start and end, about 5 us: of two
// CTAs on an SM, one slot each, one works meanwhile.
//
// Shared-memory operands are in the 128-byte-swizzled layout: rows of 64 channels, 16-byte chunk c
// of row r at chunk c ^ (r % 8).  K is read K-major (its channels are the reduction), V MN-major (its keys
// are), from the same layout.
#include <type_traits>

#include "attn_common.cuh"
#include "device_types.h"

namespace {

constexpr int kKeys = 128;
constexpr float kRescaleLog2 = 8.f;

template <int DP, int SLOTS>
struct Cfg {
    static constexpr int kSub = 128 * 128;                 // one 128-row x 64-channel block
    static constexpr int kTileBytes = DP / 64 * kSub;      // a tile of Q, K or V
    static constexpr int kStages = SLOTS == 2 ? (DP == 128 ? 5 : 8) : (DP == 128 ? 2 : 5);
    // warps that share a row of scores: two halves of its keys, where the CTA has the SM to itself
    static constexpr int kHalves = SLOTS;
    static constexpr int kCols = kKeys / kHalves;          // scores of a thread
    static constexpr int kSlotWarps = 4 * kHalves;
    static constexpr int kSoftmaxWarps = kSlotWarps * SLOTS;
    static constexpr int kMmaWarp = kSoftmaxWarps, kLoadWarp = kSoftmaxWarps + 1, kMaskWarp = kSoftmaxWarps + 2;
    static constexpr int kThreads = (kSoftmaxWarps + 4) * 32;  // whole warpgroups: the last warp is idle
    // registers of a thread: at launch (the most that the occupancy leaves), then by role
    static constexpr int kRegs = SLOTS == 2 ? 96 : 128, kRegsSoftmax = SLOTS == 2 ? 96 : 192,
                         kRegsOther = SLOTS == 2 ? 88 : 64;
    static_assert(kRegsSoftmax * kSoftmaxWarps + kRegsOther * 4 <= kRegs * kThreads / 32,
                  "setmaxnreg draws on the launch's registers");
    // a row's results leave in passes of this many bytes a thread
    static constexpr int kOutBytes = DP * 2 / kHalves;
    // Tensor memory: buffers of 128 columns for scores and weights, then the slots' O.  Item n of the CTA
    // (tile n / live, slot n % live) has buffer n % kBufs; with more buffers than slots a slot's next scores
    // are there when its softmax comes to them.
    static constexpr int kTmemCols = 256 * SLOTS;
    static constexpr int kBufs = SLOTS == 2 && DP == 64 ? 3 : SLOTS;
    static_assert(kBufs * 128 + SLOTS * DP <= kTmemCols, "tensor memory");
    // Without a buffer more than slots the product with V starts when half of each thread's weights are there: 2 x 1216
    // tokens of 16 heads of 128 channels over 5776 keys take 67.4 us, with whole weights 70.1; with a buffer more (two
    // slots of 64 channels) the other slot's products fill that time, and halves cost 50.7 against 49.7.
    static constexpr int kPParts = kBufs > SLOTS ? 1 : 2;
    // shared memory, from a 1024-byte boundary
    static constexpr int kOffKv = SLOTS * kTileBytes;
    static constexpr int kOffBar = kOffKv + kStages * kTileBytes;
    static constexpr int kBarFull = 0, kBarEmpty = kStages, kBarS = 2 * kStages, kBarP = kBarS + kBufs,
                         kBarO = kBarP + kPParts * kBufs, kBarEnd = kBarO + SLOTS, kBarMask = kBarEnd + SLOTS, kBars = kBarMask + 2;
    static constexpr int kOffTmem = kOffBar + (kBars * 8 + 15) / 16 * 16;
    static constexpr int kOffBroken = kOffTmem + 4;
    static constexpr int kOffCount = kOffBroken + 4;                   // readable keys that each warp counted
    static constexpr int kOffList = kOffCount + kThreads / 32 * 4;     // keys of two tiles, then those left over
    static constexpr int kOffShare = (kOffList + 3 * kKeys * 4 + 15) / 16 * 16;  // a value of each row, between its halves
    static constexpr int kSmem = kOffShare + (kHalves == 2 ? SLOTS * 128 * 4 : 0);
    static_assert(kSmem <= (SLOTS == 2 ? 232448 : 116224), "shared memory");
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

struct Ctl {
    uint32_t* status;
    int64_t limit_ns;
    volatile int* broken;
};

__device__ __noinline__ void give_up(uint32_t* status, volatile int* broken) {
    atomicCAS(status, 0u, (uint32_t)MAFAT_DEV_PIPE);
    *broken = 1;
}

// Bounded wait for a barrier's phase.  All waits are for work inside the CTA and end by themselves;
// one that does not records it, after which every wait of the CTA gives up after 1 ms.  The poll is inside
// one asm statement: a polling loop in the instruction stream of the issuing warp slows its products.
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, const Ctl& c) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred P1, P2;\n\t.reg .u64 dl, t;\n\t.reg .b32 br;\n\t"
        "mov.u32 %0, 1;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 P1, [%1], %2;\n\t"
        "@P1 bra AW_DONE_%=;\n\t"
        "ld.volatile.shared.b32 br, [%4];\n\t"
        "setp.ne.b32 P2, br, 0;\n\t"
        "selp.b64 t, 1000000, %3, P2;\n\t"
        "mov.u64 dl, %%globaltimer;\n\t"
        "add.u64 dl, dl, t;\n\t"
        "AW_POLL_%=:\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 P1, [%1], %2;\n\t"
        "@P1 bra AW_DONE_%=;\n\t"
        "mov.u64 t, %%globaltimer;\n\t"
        "setp.lt.u64 P2, t, dl;\n\t"
        "@P2 bra AW_POLL_%=;\n\t"
        "mov.u32 %0, 0;\n\t"
        "AW_DONE_%=:\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "l"(c.limit_ns), "r"(smem_u32(const_cast<int*>(c.broken)))
        : "memory");
    if (ok == 0u) give_up(c.status, c.broken);
}

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// One lane of the converged warp, the same on every call.
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t el;
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(el));
    return el;
}
__device__ __forceinline__ void commit_el(uint32_t el, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %0, 0;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%1];\n\t}" ::"r"(el), "r"(bar)
        : "memory");
}
// D = A B (+ D) with A and B in shared memory
__device__ __forceinline__ void mma_ss(uint32_t el, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi,
                                       uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 e, %0, 0;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "mov.b64 da, {%2, %4};\n\tmov.b64 db, {%3, %4};\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%1], da, db, %5, p;\n\t}" ::"r"(el),
        "r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(acc)
        : "memory");
}
// the same with A in tensor memory: lane = row, two bf16 a column
__device__ __forceinline__ void mma_ts(uint32_t el, uint32_t d, uint32_t a, uint32_t b_lo, uint32_t hi, uint32_t idesc,
                                       uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 db;\n\t"
        "setp.ne.b32 e, %0, 0;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "mov.b64 db, {%3, %4};\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%1], [%2], db, %5, p;\n\t}" ::"r"(el),
        "r"(d), "r"(a), "r"(b_lo), "r"(hi), "r"(idesc), "r"(acc)
        : "memory");
}
// Matrix descriptor, 128-byte swizzle (layout 2 in bits 61-63, version 1 in bits 46-47): start >> 4 in
// bits 0-13, then leading and stride byte offsets >> 4 in bits 16-29 and 32-45.  K-major: the stride
// offset is that between groups of 8 rows, the leading one is not used.  MN-major: the stride offset is that between
// groups of 8 along the reduction, the leading one that between blocks of 64 along N.
__device__ __forceinline__ uint32_t desc_hi() { return (1024u >> 4) | (1u << 14) | (2u << 29); }
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t leading) {
    return ((addr & 0x3FFFFu) >> 4) | ((leading >> 4) << 16);
}
// fp32 accumulator, bf16 operands; bit 16: B is MN-major
__device__ __forceinline__ uint32_t instr_desc(int n, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}

__device__ __forceinline__ void tma_tile(uint32_t el, uint32_t dst, const CUtensorMap* map, int c, int head, int key,
                                         int seq, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %7, 0;\n\t"
        "@e cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c), "r"(head), "r"(key), "r"(seq), "r"(bar), "r"(el)
        : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void expect_el(uint32_t el, uint32_t bar, uint32_t bytes) {
    asm volatile(
        "{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %2, 0;\n\t"
        "@e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes), "r"(el)
        : "memory");
}

// 32 columns of the thread's lane; valid after ld_wait
__device__ __forceinline__ void tmem_ld32(uint32_t t, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(t)
        : "memory");
}
// The wait passes the registers through, so that no use of them moves ahead of it (29 a statement).
__device__ __forceinline__ void ld_wait32(uint32_t* v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
    asm volatile(""
                 : "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]),
                   "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]),
                   "+r"(v[30]), "+r"(v[31])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t t, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(t)
        : "memory");
}
__device__ __forceinline__ void ld_wait16(uint32_t* v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t t, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15, %16};" ::"r"(t),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// a * s + b for two values
__device__ __forceinline__ void fma2(uint32_t a0, uint32_t a1, float s, float b, float& r0, float& r1) {
    asm("{\n\t.reg .b64 a, s, b, r;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 s, {%4, %4};\n\tmov.b64 b, {%5, %5};\n\t"
        "fma.rn.f32x2 r, a, s, b;\n\tmov.b64 {%0, %1}, r;\n\t}"
        : "=f"(r0), "=f"(r1)
        : "r"(a0), "r"(a1), "f"(s), "f"(b));
}
__device__ __forceinline__ void add2(float& r0, float& r1, float a0, float a1) {
    asm("{\n\t.reg .b64 a, r;\n\t"
        "mov.b64 r, {%0, %1};\n\tmov.b64 a, {%2, %3};\n\t"
        "add.rn.f32x2 r, r, a;\n\tmov.b64 {%0, %1}, r;\n\t}"
        : "+f"(r0), "+f"(r1)
        : "f"(a0), "f"(a1));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// The CTA's tiles of keys.  Without a mask they are runs of 128 keys, of which the last may pass the
// length; with one they are the readable keys of its part one after another, gathered, numbered from 0.
template <bool BOTH>
struct Tiles {
    int key0, n, len;
    bool gather;
    int n0, len0;  // BOTH: the tiles and keys of the prefix, which come first
    __device__ __forceinline__ bool of_prefix(int j) const { return BOTH && j < n0; }
    // place of tile j's first key in its set
    __device__ __forceinline__ int first(int j) const {
        return of_prefix(j) ? j * kKeys : key0 + (BOTH ? j - n0 : j) * kKeys;
    }
    __device__ __forceinline__ int length(int j) const { return of_prefix(j) ? len0 : len; }
    // some keys of tile j are not readable, and their values have to be zeroed (gathered ones are)
    __device__ __forceinline__ bool partial(int j) const { return !gather && first(j) + kKeys > length(j); }
};

struct NoPrefix {};

// Prefix: MafatAttnPrefix where the rows' keys are those of a prefix and then their own
template <int DP, int SLOTS, class Prefix>
__global__ void __launch_bounds__(Cfg<DP, SLOTS>::kThreads, SLOTS == 2 ? 1 : 2)
    attn_tc_kernel(const __grid_constant__ MafatAttnArgs a, const __grid_constant__ CUtensorMap kmap,
                   const __grid_constant__ CUtensorMap vmap, const __grid_constant__ Prefix prefix) {
    using C = Cfg<DP, SLOTS>;
    constexpr bool kBoth = std::is_same<Prefix, MafatAttnPrefix>::value;
    extern __shared__ __align__(1024) uint8_t sm[];
    const uint32_t base = smem_u32(sm);
    if (base & 1023u) {  // the swizzled layouts need it; the declaration asks for it
        if (threadIdx.x == 0) atomicCAS(a.status, 0u, (uint32_t)MAFAT_DEV_PIPE);
        return;
    }
    const uint32_t bars = base + C::kOffBar;
    auto bar = [&](int i) { return bars + (uint32_t)i * 8u; };
    uint32_t* tmem_slot = (uint32_t*)(sm + C::kOffTmem);
    volatile int* broken = (volatile int*)(sm + C::kOffBroken);
    const Ctl ctl{a.status, a.timeout_ns, broken};
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const MafatAttnSeg& g = a.seg;
    const bool gather = !kBoth && g.mask != nullptr;

    if (warp == C::kLoadWarp && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&kmap)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&vmap)) : "memory");
        for (int i = 0; i < C::kStages; ++i) {
            // gathered tiles are filled by three warps' threads; others by TMA, and are also looked at by the mask warp
            bar_init(bar(C::kBarFull + i), gather ? 96 : 1);
            bar_init(bar(C::kBarEmpty + i), gather ? 1 : 2);
        }
        for (int i = 0; i < SLOTS; ++i) {
            bar_init(bar(C::kBarO + i), 1);
            bar_init(bar(C::kBarEnd + i), 1);
        }
        for (int i = 0; i < C::kBufs; ++i) {
            bar_init(bar(C::kBarS + i), 1);
            for (int part = 0; part < C::kPParts; ++part) bar_init(bar(C::kBarP + i * C::kPParts + part), C::kSlotWarps);
        }
        for (int i = 0; i < 2; ++i) bar_init(bar(C::kBarMask + i), 1);
        *broken = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == C::kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                     "r"(C::kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    __syncwarp();
    // queries, whose places are known before the launch before has ended; they and the length come together
    mafat_attn::Block b(a, blockIdx.x, 128 * SLOTS);
    constexpr int kChunks = DP / 8, kRows = 32 / kChunks;  // 16-byte chunks of a row; rows of a warp's access
    constexpr int kLoads = 32 / kRows / C::kHalves;
    const int q_slot = warp / C::kSlotWarps, q_half = warp / 4 % C::kHalves, q_quarter = warp % 4;
    const int q_row0 = b.row0 + q_slot * 128 + q_quarter * 32, cc = lane % kChunks, cr = lane / kChunks;
    const bool q_any = warp < C::kSoftmaxWarps && q_row0 < g.rows;
    const int64_t q_off = q_any && q_row0 + lane < g.rows ? mafat_attn::Row(a, b, q_row0 + lane).query(a) : -1;
    uint4 q[kLoads];
    mafat_attn::launch_begin(a);
    if (q_any) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int64_t o = __shfl_sync(0xffffffffu, q_off, (q_half * kLoads + i) * kRows + cr);
            q[i] = make_uint4(0u, 0u, 0u, 0u);
            if (o >= 0 && cc * 8 < a.dim) q[i] = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)a.q + o + cc * 8);
        }
    }
    b.len = mafat_attn::length_of(g, b.seq);
    Tiles<kBoth> t;
    t.n0 = t.len0 = 0;
    int prefix_seq = 0;
    if constexpr (kBoth) {
        prefix_seq = (int)prefix.per.div((uint32_t)b.seq);
        t.len0 = prefix.len ? min(max(prefix.len[prefix_seq], 0), prefix.n) : prefix.n;
        t.n0 = (t.len0 + kKeys - 1) / kKeys;
    }
    b.set_keys(a, 128 * SLOTS, kKeys);
    t.gather = gather;
    t.key0 = b.key0;
    t.len = b.len;
    t.n = t.n0 + (b.key1 > b.key0 ? (b.key1 - b.key0 + kKeys - 1) / kKeys : 0);
    const uint8_t* mask = gather ? g.mask + (int64_t)b.seq * g.n : nullptr;
    if (gather) {
        int n = 0;
#pragma unroll 8
        for (int k = b.key0 + (int)threadIdx.x; k < b.key1; k += C::kThreads) n += mask[k] != 0;
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) *(volatile int*)(sm + C::kOffCount + warp * 4) = n;
    }
    // K and V can be on their way, and the queries be loaded, before all warps are here
    uint32_t ahead_loads = 0u;
    auto load_tile = [&](uint32_t el, int i, uint32_t stage) {
        const uint32_t full = bar(C::kBarFull) + stage * 8u, dst = base + C::kOffKv + stage * C::kTileBytes;
        expect_el(el, full, C::kTileBytes);
#pragma unroll
        for (int c = 0; c < DP / 64; ++c) {
            if constexpr (kBoth)
                if (t.of_prefix(i / 2)) {
                    tma_tile(el, dst + c * C::kSub, (i & 1) ? &prefix.v : &prefix.k, c * 64, b.head, t.first(i / 2), prefix_seq, full);
                    continue;
                }
            tma_tile(el, dst + c * C::kSub, (i & 1) ? &vmap : &kmap, c * 64, b.head, t.first(i / 2), b.seq, full);
        }
    };
    if (!gather && warp == C::kLoadWarp && t.n > 0) {
        const uint32_t el = elect_one();
        ahead_loads = 2u;
        load_tile(el, 0, 0u);
        load_tile(el, 1, 1u);
    }
    if (q_any) {
        uint8_t* to = sm + q_slot * C::kTileBytes;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = q_quarter * 32 + (q_half * kLoads + i) * kRows + cr;
            *reinterpret_cast<uint4*>(to + (cc / 8) * C::kSub + r * 128 + ((cc % 8) ^ (r % 8)) * 16) = q[i];
        }
        fence_async();
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_slot;
    if (gather) {
        int n = lane < C::kThreads / 32 ? *(volatile int*)(sm + C::kOffCount + lane * 4) : 0;
        n = __reduce_add_sync(0xffffffffu, n);
        t.key0 = 0;
        t.len = n;
        t.n = (n + kKeys - 1) / kKeys;
    }
    const int live = SLOTS == 2 && b.row0 + 128 < g.rows ? 2 : 1;  // slots that have rows
    // Buffers in use: the scores of tile j wait for the slot's product of tile j - 2 at the least, so that who waits for
    // that of tile j - 1 is less than two phases of its barrier behind.
    const int bufs = C::kBufs > 2 && live == 1 ? 2 : C::kBufs;
    // Scores of a slot are made before its product before them has ended: O is then waited for by a barrier
    // of its own, else the scores' says that it is there.
    const bool ahead = live < bufs;

    if (warp < C::kSoftmaxWarps) {
        if constexpr (C::kRegsSoftmax > C::kRegs) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegsSoftmax));
        const int slot = warp / C::kSlotWarps, half = warp / 4 % C::kHalves, quarter = warp % 4;
        const int row0 = b.row0 + slot * 128 + quarter * 32;  // the warp's first row
        const int row = row0 + lane;
        const bool any = row0 < g.rows && t.n > 0;
        const mafat_attn::Row at(a, b, min(row, g.rows - 1));
        uint8_t* mine = sm + slot * C::kTileBytes;  // the slot's queries; at the end, its results on their way out
        // the two warps that have halves of the same rows
        const int pair = 2 + slot * 4 + quarter;
        volatile float* share = (volatile float*)(sm + C::kOffShare) + slot * 128 + quarter * 32 + lane;
        auto joined = [&](float x, auto op) {  // op of both halves' values, in both
            if constexpr (C::kHalves == 2) {
                if (half == 1) *share = x;
                asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory");
                if (half == 0) *share = x = op(x, *share);
                asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory");
                if (half == 1) x = *share;
            }
            return x;
        };
        auto either = [&](bool x) {  // whether it holds for a row of the warp, in either half
            if constexpr (C::kHalves == 2) {
                uint32_t r;
                asm volatile(
                    "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %2, 0;\n\t"
                    "bar.red.or.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                    : "=r"(r)
                    : "r"(pair), "r"((uint32_t)x)
                    : "memory");
                return r != 0u;
            }
            return __any_sync(0xffffffffu, x) != 0;
        };

        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t to = tmem + lanes + (uint32_t)(C::kBufs * 128 + slot * DP + half * (DP / C::kHalves));
        const int limit = row >= g.rows ? 0x7fffffff : gather ? t.len : at.limit(a, b);
        const float c = a.scale_log2;
        const int n_tiles = slot < live ? t.n : 0;
        float from = -CUDART_INF_F, l0 = 0.f, l1 = 0.f;  // the base in use: at most 2^8 below the maximum
        int buf = slot;
        uint32_t uses = 0u;  // parity of the buffer's uses
        for (int j = 0; j < n_tiles; ++j) {
            wait(bar(C::kBarS) + (uint32_t)buf * 8u, uses, ctl);
            const uint32_t ts = tmem + lanes + (uint32_t)(buf * 128);
            __syncwarp();  // tensor memory is read by converged warps
            if (any) {
                fence_after();
                uint32_t s[C::kCols];
#pragma unroll
                for (int i = 0; i < C::kCols / 32; ++i) tmem_ld32(ts + (uint32_t)(half * C::kCols + 32 * i), s + 32 * i);
                // readable keys of the thread's
                const int left = (t.of_prefix(j) ? t.len0 : limit) - t.first(j) - half * C::kCols;
#pragma unroll
                for (int i = 0; i < C::kCols / 32; ++i) ld_wait32(s + 32 * i);
                if (left < C::kCols) {
#pragma unroll
                    for (int i = 0; i < C::kCols; ++i)
                        if (i >= left) s[i] = 0xff800000u;  // -inf
                }
                float top[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    top[i] = __uint_as_float(s[i]);
#pragma unroll
                    for (int k = i + 4; k < C::kCols; k += 8)
                        top[i] = k + 4 < C::kCols ? max3(top[i], __uint_as_float(s[k]), __uint_as_float(s[k + 4]))
                                                  : mafat_attn::max_nan(top[i], __uint_as_float(s[k]));
                }
                const float mt = max3(mafat_attn::max_nan(top[0], top[1]), top[2], top[3]);
                // also where the base is -inf and mt is not.  After it both halves have read their scores: P may be
                // written over them.
                if (either(j == 0 || mt * c - from > kRescaleLog2)) {
                    const float next = joined(mt, [](float x, float y) { return mafat_attn::max_nan(x, y); }) * c;
                    if (j == 0) {
                        from = next;  // there is no O yet
                    } else {
                        const bool up = next - from > kRescaleLog2;
                        const float keep = up ? mafat_attn::exp2_fast(from - next) : 1.f;
                        if (up) from = next;
                        l0 *= keep;
                        l1 *= keep;
                        if (ahead) {  // the scores were made before the product that O waits for
                            wait(bar(C::kBarO + slot), (uint32_t)(j - 1) & 1u, ctl);
                            __syncwarp();
                            fence_after();
                        }
#pragma unroll
                        for (int i = 0; i < DP / C::kHalves / 16; ++i) {
                            uint32_t o[16];
                            tmem_ld16(to + 16u * i, o);
                            ld_wait16(o);
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * keep);
                            tmem_st16(to + 16u * i, o);
                        }
                    }
                }
                const float off = -mafat_attn::subtrahend(from);
#pragma unroll
                for (int h = 0; h < C::kCols / 32; ++h) {
                    uint32_t p[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float x, y;
                        fma2(s[32 * h + 2 * i], s[32 * h + 2 * i + 1], c, off, x, y);
                        x = mafat_attn::exp2_fast(x);
                        y = mafat_attn::exp2_fast(y);
                        add2(l0, l1, x, y);
                        p[i] = pack(x, y);
                    }
                    tmem_st16(ts + (uint32_t)(half * (C::kCols / 2) + 16 * h), p);
                    if (C::kPParts == 2 && h == C::kCols / 64 - 1) {  // the product with half of the thread's keys can begin
                        st_wait();
                        fence_before();
                        __syncwarp();
                        if (lane == 0) arrive(bar(C::kBarP) + (uint32_t)(buf * C::kPParts) * 8u);
                    }
                }
                st_wait();
                fence_before();
            } else if (C::kPParts == 2 && lane == 0) {
                arrive(bar(C::kBarP) + (uint32_t)(buf * C::kPParts) * 8u);
            }
            __syncwarp();
            if (lane == 0) arrive(bar(C::kBarP) + (uint32_t)(buf * C::kPParts + C::kPParts - 1) * 8u);
            buf += live;
            if (buf >= bufs) buf -= bufs, uses ^= 1u;
        }
        // Through shared memory, 16-byte chunks swizzled over the rows, so that a row leaves in whole pieces:
        // kOutBytes of each row at a time, bf16 results at once, fp32 parts in two passes.  joins: with the parts of
        // the launch before (apart, so that the form without them stays short).
        auto results = [&](auto joins) {
            constexpr bool kJoins = decltype(joins)::value;
            constexpr int kWide = DP / C::kHalves;           // columns of the thread
            constexpr int kStep = kWide >= 64 ? 32 : 16;     // read at a time
            constexpr int kChunks = C::kOutBytes / 16, kRows = 32 / kChunks, kSwz = kChunks < 8 ? kChunks : 8;
            const int cc = lane % kChunks, cr = lane / kChunks;
            const float l = joined(l0 + l1, [](float x, float y) { return x + y; });
            float inv = mafat_attn::inverse_sum(l), join_top = 0.f, join_inv = 0.f;
            const mafat_attn::Out w(a, b, at);
            if constexpr (kJoins) {
                mafat_attn::launch_wait();
                const mafat_attn::Join jn(a, w, from, l);
                inv = jn.own;
                join_top = jn.top;
                join_inv = jn.inv;
                if (row < g.rows && half == 0 && a.lse) a.lse[w.row] = jn.lse2 * CUDART_LN2_F;
            } else if (row < g.rows && half == 0) {
                mafat_attn::store_lse(a, w, from, l);
            }
            const bool part = !a.direct || kJoins, none = t.n == 0 || l == 0.f;  // fp32 on the way
            uint8_t* buf = mine + (quarter * C::kHalves + half) * 32 * C::kOutBytes;
            const int64_t dst = row >= g.rows ? -1 : a.direct ? w.o : w.part * a.dim;
            uint8_t* my = buf + lane * C::kOutBytes;
            if (n_tiles > 0) {
                wait(bar(C::kBarEnd + slot), 0u, ctl);
                __syncwarp();
                fence_after();
            }
            auto put = [&](int chunk, uint4 v) { *reinterpret_cast<uint4*>(my + ((chunk ^ (lane % kSwz)) * 16)) = v; };
#pragma unroll
            for (int pass = 0; pass < 2; ++pass) {
                if (pass == 1 && !part) break;
                const int cols = part ? kWide / 2 : kWide;  // of this pass
#pragma unroll
                for (int i = 0; i < kWide / kStep; ++i) {
                    if (i * kStep >= cols) break;
                    uint32_t o[kStep];
                    if (t.n > 0) {
                        const uint32_t src = to + (uint32_t)(pass * (kWide / 2) + kStep * i);
                        if constexpr (kStep == 32) {
                            tmem_ld32(src, o);
                            ld_wait32(o);
                        } else {
                            tmem_ld16(src, o);
                            ld_wait16(o);
                        }
                    }
                    // a row without readable keys: 0, whatever the products left
#pragma unroll
                    for (int k = 0; k < kStep; ++k) o[k] = none ? 0u : __float_as_uint(__uint_as_float(o[k]) * inv);
                    if (part) {
#pragma unroll
                        for (int k = 0; k < kStep / 4; ++k)
                            put(kStep / 4 * i + k, make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]));
                    } else {
                        uint32_t p[kStep / 2];
#pragma unroll
                        for (int k = 0; k < kStep / 2; ++k) p[k] = pack(__uint_as_float(o[2 * k]), __uint_as_float(o[2 * k + 1]));
#pragma unroll
                        for (int k = 0; k < kStep / 8; ++k)
                            put(kStep / 8 * i + k, make_uint4(p[4 * k], p[4 * k + 1], p[4 * k + 2], p[4 * k + 3]));
                    }
                }
                __syncwarp();
                // channel of the lane's chunk
                const int d = half * kWide + (part ? pass * (kWide / 2) + cc * 4 : cc * 8);
                constexpr int kPieces = 32 / kRows;  // rows of a lane
                if constexpr (kJoins) {
                    float4 v[kPieces];
#pragma unroll
                    for (int i = 0; i < kPieces; ++i) {
                        const int r = i * kRows + cr;
                        v[i] = *reinterpret_cast<const float4*>(buf + r * C::kOutBytes + ((cc ^ (r % kSwz)) * 16));
                    }
#pragma unroll 1
                    for (int p = 0; p < a.join; ++p) {  // a part of all rows at a time, whole rows of it
                        const float mine_f = mafat_attn::exp2_fast(a.part_lse[(int64_t)p * a.rows_total + w.row] - join_top) * join_inv;
                        const float* src = a.part_o + (int64_t)p * a.rows_total * a.dim + d;
#pragma unroll
                        for (int i = 0; i < kPieces; ++i) {
                            const int r = i * kRows + cr;
                            const float f = __shfl_sync(0xffffffffu, mine_f, r);
                            const int64_t at_row = __shfl_sync(0xffffffffu, w.row, r);
                            float4 u = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (d < a.dim) u = *reinterpret_cast<const float4*>(src + at_row * a.dim);
                            v[i] = make_float4(fmaf(f, u.x, v[i].x), fmaf(f, u.y, v[i].y), fmaf(f, u.z, v[i].z), fmaf(f, u.w, v[i].w));
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kPieces; ++i) {
                        const int64_t o = __shfl_sync(0xffffffffu, dst, i * kRows + cr);
                        if (o >= 0 && d < a.dim) mafat_attn::put4((__nv_bfloat16*)a.out + o + d, v[i]);
                    }
                } else {
                    constexpr int kTogether = kPieces < 8 ? kPieces : 8;  // read before they are written: writes might be to what is read
                    uint8_t* to_out = part ? (uint8_t*)(a.part_o + d) : (uint8_t*)((__nv_bfloat16*)a.out + d);
#pragma unroll
                    for (int i0 = 0; i0 < kPieces; i0 += kTogether) {
                        int64_t o[kTogether];
                        uint4 v[kTogether];
#pragma unroll
                        for (int i = 0; i < kTogether; ++i) {
                            const int r = (i0 + i) * kRows + cr;
                            o[i] = __shfl_sync(0xffffffffu, dst, r);
                            v[i] = *reinterpret_cast<const uint4*>(buf + r * C::kOutBytes + ((cc ^ (r % kSwz)) * 16));
                        }
#pragma unroll
                        for (int i = 0; i < kTogether; ++i)
                            if (o[i] >= 0 && d < a.dim) *reinterpret_cast<uint4*>(to_out + o[i] * (part ? 4 : 2)) = v[i];
                    }
                }
                __syncwarp();
            }
        };
        if (row0 < g.rows) {
            if (a.join)
                results(std::true_type());
            else
                results(std::false_type());
        }
        fence_before();
    } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegsOther));
    if (warp == C::kMmaWarp) {
        const uint32_t el = elect_one();
        const uint32_t id_s = instr_desc(kKeys, false), id_o = instr_desc(DP, true), hi = desc_hi();
        const uint32_t q_lo = desc_lo(base, 16u), k_lo = desc_lo(base + C::kOffKv, 16u),
                       v_lo = desc_lo(base + C::kOffKv, C::kSub);
        constexpr uint32_t kTile16 = C::kTileBytes / 16, kSub16 = C::kSub / 16;
        auto scores = [&](int slot, uint32_t stage, int buf) {
            const uint32_t qa = q_lo + (uint32_t)slot * kTile16, kb = k_lo + stage * kTile16;
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
                const uint32_t step = (uint32_t)(k / 4) * kSub16 + (uint32_t)(k % 4) * 2u;  // 32 bytes along a row
                mma_ss(el, tmem + (uint32_t)(buf * 128), qa + step, kb + step, hi, id_s, k > 0);
            }
            commit_el(el, bar(C::kBarS) + (uint32_t)buf * 8u);
        };
        uint32_t uses = 0u;  // parity of the uses of P's buffers
        auto values = [&](int slot, uint32_t stage, int buf, uint32_t acc, bool last) {
            const uint32_t vb = v_lo + stage * kTile16;
#pragma unroll
            for (int part = 0; part < C::kPParts; ++part) {  // of each softmax thread's keys
                wait(bar(C::kBarP) + (uint32_t)(buf * C::kPParts + part) * 8u, uses, ctl);
                fence_after();
                constexpr int kRun = C::kCols / 16 / C::kPParts;  // steps of a thread's keys in the part
#pragma unroll
                for (int i = 0; i < kKeys / 16 / C::kPParts; ++i) {  // 16 keys: 8 columns of P, two 8-key groups of V
                    const int k = i / kRun * (C::kCols / 16) + part * kRun + i % kRun;
                    mma_ts(el, tmem + (uint32_t)(C::kBufs * 128 + slot * DP), tmem + (uint32_t)(buf * 128 + 8 * k),
                           vb + (uint32_t)k * (2048u / 16u), hi, id_o, part + i > 0 ? 1u : acc);
                }
            }
            commit_el(last || ahead ? el : 0u, bar(last ? C::kBarEnd : C::kBarO) + (uint32_t)slot * 8u);
        };
        // The scores of item n + kBufs follow the values of item n: products run in the order of issue,
        // so that its buffer is free.  Two places in the ring, each of K or V of a tile and the item's slot.
        struct Place {
            uint32_t stage, phase;
            int slot, tile;
            __device__ __forceinline__ bool next(int live) {  // true: the tile is done with
                if (++slot < live) return false;
                slot = 0;
                ++tile;
                stage += 2u;
                if (stage >= (uint32_t)C::kStages) stage -= (uint32_t)C::kStages, phase ^= 1u;
                return true;
            }
        };
        Place ps{0u, 0u, 0, 0}, pv{1u, 0u, 0, 0};
        int bs = 0, bv = 0;
        auto wait_tile = [&](uint32_t stage, uint32_t phase) {
            wait(bar(C::kBarFull) + stage * 8u, phase, ctl);
            if (gather) fence_async();  // the copies' threads have not waited for them
        };
        auto next_scores = [&]() {
            if (ps.tile >= t.n) return;
            if (ps.slot == 0) wait_tile(ps.stage, ps.phase);
            fence_after();
            scores(ps.slot, ps.stage, bs);
            if (++bs == bufs) bs = 0;
            const uint32_t empty = bar(C::kBarEmpty) + ps.stage * 8u;
            if (ps.next(live)) commit_el(el, empty);
        };
#pragma unroll 1
        for (int i = 0; i < bufs; ++i) next_scores();
#pragma unroll 1
        while (pv.tile < t.n) {
            if (pv.slot == 0) {
                wait_tile(pv.stage, pv.phase);
                if (t.partial(pv.tile)) wait(bar(C::kBarMask + t.of_prefix(pv.tile)), 0u, ctl);
            }
            values(pv.slot, pv.stage, bv, pv.tile > 0, pv.tile == t.n - 1);
            if (++bv == bufs) bv = 0, uses ^= 1u;
            const uint32_t empty = bar(C::kBarEmpty) + pv.stage * 8u;
            if (pv.next(live)) commit_el(el, empty);
            next_scores();
        }
    } else if (gather) {
        // Three warps copy the readable keys of the part, 128 at a time, as they are found: the first
        // lists their numbers, all copy every third group of rows, and their copies' landing says that a tile is there.
        const int who = warp - C::kLoadWarp;
        int* list = (int*)(sm + C::kOffList);  // [2][kKeys], then [kKeys] left over
        constexpr int kChunks = DP / 8, kRows = 32 / kChunks;
        constexpr int kSets = 8 / kRows, kGroups = (kKeys / 8 + 2) / 3;  // accesses of 8 rows; groups of 8 rows of a warp
        const int cc = lane % kChunks, cr = lane / kChunks;
        const __nv_bfloat16* src[2] = {
            (const __nv_bfloat16*)g.k + (int64_t)b.seq * g.k_sb + (int64_t)b.head * g.k_sh + (cc * 8 < a.dim ? cc * 8 : 0),
            (const __nv_bfloat16*)g.v + (int64_t)b.seq * g.v_sb + (int64_t)b.head * g.v_sh + (cc * 8 < a.dim ? cc * 8 : 0)};
        const int64_t step[2] = {g.k_ss, g.v_ss};
        uint32_t at8[kSets];  // place of the lane's chunk in a group of 8 rows
#pragma unroll
        for (int i = 0; i < kSets; ++i) {
            const int r = i * kRows + cr;
            at8[i] = (uint32_t)(cc / 8 * C::kSub + r * 128 + ((cc % 8) ^ r) * 16);
        }
        const bool in_dim = cc * 8 < a.dim;
        int pos = b.key0, rest = 0;
        uint32_t seen[4];  // the next 128 bytes of the mask
        auto look = [&](int at) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = at + i * 32 + lane;
                seen[i] = k < b.key1 ? mask[k] : 0u;
            }
        };
        if (who == 0) look(pos);
        uint32_t stage = 0u, phase = 1u;
#pragma unroll 1
        for (int j = 0; j < t.n; ++j) {
            int* keys = list + (j & 1) * kKeys;
            if (who == 0) {
                int n = rest;
                for (int k = lane; k < n; k += 32) keys[k] = list[2 * kKeys + k];
                __syncwarp();
                while (n < kKeys && pos < b.key1) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const bool on = seen[k] != 0u;
                        const uint32_t bits = __ballot_sync(0xffffffffu, on);
                        const int at = n + __popc(bits & ((1u << lane) - 1u));
                        if (on) (at < kKeys ? keys : list + kKeys)[at] = pos + k * 32 + lane;
                        n += __popc(bits);
                    }
                    pos += kKeys;
                    look(pos);
                }
                rest = max(n - kKeys, 0);
                for (int k = n + lane; k < kKeys; k += 32) keys[k] = -1;
            }
            asm volatile("bar.sync 1, 96;" ::: "memory");
            int key[kGroups][kSets];
#pragma unroll
            for (int q = 0; q < kGroups; ++q)
#pragma unroll
                for (int i = 0; i < kSets; ++i) {
                    const int r = (q * 3 + who) * 8 + i * kRows + cr;
                    key[q][i] = r < kKeys && in_dim ? keys[r] : -1;
                }
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                wait(bar(C::kBarEmpty) + stage * 8u, phase, ctl);
                __syncwarp();
                const uint32_t dst = base + C::kOffKv + stage * C::kTileBytes;
#pragma unroll
                for (int q = 0; q < kGroups; ++q)
                    if (q * 3 + who < kKeys / 8)
#pragma unroll
                        for (int i = 0; i < kSets; ++i) {
                            const int k = key[q][i];
                            copy16(dst + (uint32_t)(q * 3 + who) * 1024u + at8[i],
                                   src[kv] + (int64_t)max(k, 0) * step[kv], k >= 0);
                        }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar(C::kBarFull) + stage * 8u)
                             : "memory");
                if (++stage == (uint32_t)C::kStages) stage = 0u, phase ^= 1u;
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp == C::kLoadWarp) {
        const uint32_t el = elect_one();
        uint32_t stage = ahead_loads % (uint32_t)C::kStages;
        uint32_t phase = ahead_loads < (uint32_t)C::kStages ? 1u : 0u;  // the first wait on an empty stage is over at once
#pragma unroll 1
        for (int i = (int)ahead_loads; i < 2 * t.n; ++i) {
            wait(bar(C::kBarEmpty) + stage * 8u, phase, ctl);
            load_tile(el, i, stage);
            if (++stage == (uint32_t)C::kStages) stage = 0u, phase ^= 1u;
        }
    } else if (warp == C::kMaskWarp) {
        // zeroes the values past the length in the tile that has some
        uint32_t stage = 0u, phase = 0u;
#pragma unroll 1
        for (int i = 0; i < 2 * t.n; ++i) {
            wait(bar(C::kBarFull) + stage * 8u, phase, ctl);
            __syncwarp();
            if ((i & 1) && t.partial(i / 2)) {
                uint8_t* v = sm + C::kOffKv + stage * C::kTileBytes;
                for (int r = t.length(i / 2) - t.first(i / 2) + lane / 8; r < kKeys; r += 4)
#pragma unroll
                    for (int c = 0; c < DP / 64; ++c)
                        *reinterpret_cast<uint4*>(v + c * C::kSub + r * 128 + (lane % 8) * 16) = make_uint4(0u, 0u, 0u, 0u);
                fence_async();
                __syncwarp();
                if (lane == 0) arrive(bar(C::kBarMask + t.of_prefix(i / 2)));
            }
            if (lane == 0) arrive(bar(C::kBarEmpty) + stage * 8u);
            if (++stage == (uint32_t)C::kStages) stage = 0u, phase ^= 1u;
        }
    }
    }
    __syncthreads();
    if (warp == C::kMmaWarp) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols));
    }
    mafat_attn::launch_end(a);
}

template <int DP, int SLOTS>
cudaError_t launch(const MafatAttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, const MafatAttnPrefix* prefix,
                   cudaStream_t s) {
    using C = Cfg<DP, SLOTS>;
    if (prefix)
        return mafat_launch_overlapped(attn_tc_kernel<DP, SLOTS, MafatAttnPrefix>, a.seg.items, C::kThreads, C::kSmem, s, a,
                                       k, v, *prefix);
    return mafat_launch_overlapped(attn_tc_kernel<DP, SLOTS, NoPrefix>, a.seg.items, C::kThreads, C::kSmem, s, a, k, v,
                                   NoPrefix());
}
template <int DP, int SLOTS, class Prefix>
cudaError_t prepare_form() {
    using C = Cfg<DP, SLOTS>;
    cudaFuncAttributes at;
    cudaError_t e = cudaFuncGetAttributes(&at, attn_tc_kernel<DP, SLOTS, Prefix>);
    if (e != cudaSuccess) return e;
    // with fewer registers at launch than the roles' shares add up to, setmaxnreg.inc would wait forever
    if (at.numRegs < C::kRegs) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(attn_tc_kernel<DP, SLOTS, Prefix>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
}
template <int DP, int SLOTS>
cudaError_t prepare() {
    const cudaError_t e = prepare_form<DP, SLOTS, NoPrefix>();
    return e != cudaSuccess ? e : prepare_form<DP, SLOTS, MafatAttnPrefix>();
}

}  // namespace

cudaError_t mafat_launch_attn_tc(const MafatAttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int slots,
                                 const MafatAttnPrefix* prefix, cudaStream_t s) {
    if (slots == 2) return a.dim <= 64 ? launch<64, 2>(a, k, v, prefix, s) : launch<128, 2>(a, k, v, prefix, s);
    return a.dim <= 64 ? launch<64, 1>(a, k, v, prefix, s) : launch<128, 1>(a, k, v, prefix, s);
}

cudaError_t mafat_prepare_attn_tc() {
    cudaError_t e;
    if ((e = prepare<64, 1>()) != cudaSuccess) return e;
    if ((e = prepare<128, 1>()) != cudaSuccess) return e;
    if ((e = prepare<64, 2>()) != cudaSuccess) return e;
    return prepare<128, 2>();
}
