// C ABI of the language operators: checks of arguments, plans (workspace and the split of the
// work) and launches.  See include/mafat.h.
#include <cuda.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/mafat.h"
#include "attention.h"
#include "device_types.h"
#include "lm_checks.h"

void* mafat_internal_encode_tiled();

// A kernel, the shape of its work and the time that it takes, in us, measured on GB300 with launches back to back over
// 16 to 400 sequences of 32 to 1444 keys: the terms of Model::us.
enum AttnKernel { kSimt4, kSimt8, kSimt64, kRows, kTc1, kTc2 };
struct AttnShape {
    int rows, keys;  // of a CTA's tile
    int ctas;        // of an SM
    double fixed;    // a launch
    double setup;    // start and end of an item
    double tile;     // a tile of keys, for a CTA that has its SM alone
    double shared;   // the same with another CTA on the SM
    double sm_item, sm_tile;  // an SM's time for an item and a tile when it has many (0: as above)
    double part;     // writing a part instead of a result
};

// One set of keys as a plan sees it.
struct AttnSegPlan {
    int32_t n_seq = 0, reqs = 0, n = 0, causal = 0;
    int64_t k[3] = {0, 0, 0}, v[3] = {0, 0, 0};  // strides: sequence, key, head
    int32_t rows = 0, row_tiles = 0, splits = 0, part0 = 0, items = 0, ctas = 0;
    uint32_t cut = 0;  // as MafatAttnSeg's
    AttnKernel kernel = kRows;
    double us = 0.;  // by the model
};

enum AttnKind { kCross, kPrefix, kTree };
const char* const kAttnPlans[] = {"mafat_cross_plan", "mafat_prefix_plan", "mafat_tree_plan"};

struct mafat_attn_s {
    AttnKind kind = kCross;
    bool dry_run = false;
    int device = 0, sms = 0;
    int32_t dtype = 0, batch = 0, n_q = 0, heads_q = 0, heads_kv = 0, dim = 0;
    float scale = 0.f;
    int64_t q[3] = {0, 0, 0}, o[3] = {0, 0, 0};
    int n_seg = 0;
    AttnSegPlan seg[2];
    // launches: the segments that have room for keys, or the first if none has
    int n_run = 0, run[2] = {0, 0};
    // the own keys' work when one launch of the tensor-core kernel does both sets (a run without a mask); items 0: never
    AttnSegPlan both;
    int parts = 0;
    int cluster = 1;      // CTAs of a cluster that joins its parts itself
    int both_cluster = 1;  // the same where one launch does both sets
    bool joined = false;  // the second launch joins the first one's parts with its own results
    int64_t rows_total = 0, workspace_bytes = 0;
    void* workspace = nullptr;
    float* part_o = nullptr;
    float* part_lse = nullptr;
    uint32_t* status = nullptr;
};

namespace {

using namespace mafat_lm;

constexpr int kStatusBytes = 256;
// rows and keys: a tile past the last still has a number in 32 bits
constexpr int64_t kMostCounted = kMaxI32 - 65536;
constexpr int kMaxDim = 128;

int sm_count(int device) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n <= 0) n = 152;
    return n;
}

struct Common {
    int32_t dtype, batch, n_q, heads_q, heads_kv, dim, kernel, splits, dry_run;
    float scale;
    const int64_t *q, *o;
};

mafat_status check_common(const Common& c) {
    if (c.dtype != MAFAT_BF16 && c.dtype != MAFAT_FP32) return fail(MAFAT_EINVAL, "dtype must be MAFAT_BF16 or MAFAT_FP32");
    if (c.batch < 1 || c.n_q < 1) return fail(MAFAT_EINVAL, "batch and n_q must be positive");
    if (c.heads_q < 1 || c.heads_kv < 1 || c.heads_q % c.heads_kv != 0)
        return fail(MAFAT_EINVAL, "heads_q must be a positive multiple of heads_kv");
    if (c.dim < 1) return fail(MAFAT_EINVAL, "head_dim must be positive");
    if (c.dim > kMaxDim || c.dim % 8 != 0)
        return fail(MAFAT_EUNSUPPORTED, "head_dim must be a multiple of 8 and at most 128");
    if (!(c.scale >= 0.f) || std::isinf(c.scale)) return fail(MAFAT_EINVAL, "scale must be positive, or 0 for 1/sqrt(head_dim)");
    if (c.kernel < MAFAT_ATTN_AUTO || c.kernel > MAFAT_ATTN_TILES) return fail(MAFAT_EINVAL, "unknown kernel");
    if (c.splits < 0 || c.splits > MAFAT_ATTN_MAX_SPLITS) return fail(MAFAT_EINVAL, "splits out of range");
    if ((int64_t)c.batch * c.n_q > kMostCounted / c.heads_q) return fail(MAFAT_EUNSUPPORTED, "too many rows");
    return MAFAT_OK;
}

// Each kernel where it is the quickest; in us, with as many parts as are best for each:
//   bf16, 64 sequences of 1444 keys, one key head of 128 channels   16 rows: kRows 10.5, kTc1 15.7; 32 rows: 18.7, 16.0
//   bf16, 152 sequences of 256 rows, one head   64 channels, 128 keys: kTc1 4.9, kTc2 5.2; 2048 keys: 23.7, 19.9;
//                                               128 channels, 128 keys: 7.0, 6.8; 2048 keys: 37.3, 35.4
//   fp32, 64 sequences of 1444 keys, 8 key heads of 128 channels    4 rows: kSimt4 130, kSimt8 172, kSimt64 573;
//                                               8 rows: 224, 173, 573; 16 rows: 442, 314, 577; 32 rows: 856, 622, 583
// The terms are those of earlier forms of the kernels.  146 drawn plans (1 to 64 sequences, 30 to 6000 keys, 1 to 1024
// tokens) take, as shares of the model's time, quartiles and ends: kTc1 0.95 0.98 1.05 (0.89 to 1.12), kTc2 0.92 0.97 1.04
// (0.90 to 1.13), kRows 0.83 0.93 1.00 (0.70 to 1.30), kSimt64 0.92 0.97 1.09 (0.88 to 1.77: a last wave of few CTAs, which
// the model takes for one an SM), kSimt4 and kSimt8 0.78 to 0.87, 0.82 to 0.93, 0.99 (0.70 to 1.24).
AttnShape shape_of(AttnKernel k, int dim) {
    const bool wide = dim > 64;
    const int simt = mafat_attn_simt_keys(), rows = mafat_attn_rows_keys();
    switch (k) {
        case kRows:
            return wide ? AttnShape{16, rows, 2, 3.2, 0.4, 0.87, 1.05, 1.1, 0.63, 0} : AttnShape{16, rows, 2, 2.7, 0.3, 0.5, 0.72, 0.65, 0.36, 0};
        case kTc1: return wide ? AttnShape{128, 128, 2, 0.2, 4.5, 1.15, 2.3, 0, 0, 1.5} : AttnShape{128, 128, 2, 0.7, 2.8, 0.96, 1.45, 0, 0, 1.0};
        case kTc2: return wide ? AttnShape{256, 128, 1, 0.35, 5.25, 1.45, 1.45, 0, 0, 1.5} : AttnShape{256, 128, 1, 0.5, 4.2, 1.05, 1.05, 0, 0, 1.0};
        case kSimt64: return wide ? AttnShape{64, simt, 1, 2.0, 1.2, 7.8, 7.8, 0, 0, 0} : AttnShape{64, simt, 1, 2.0, 1.2, 4.4, 4.4, 0, 0, 0};
        case kSimt8: return wide ? AttnShape{8, simt, 1, 2.8, 0.8, 1.9, 1.9, 0, 0, 0} : AttnShape{8, simt, 2, 2.5, 0.5, 1.17, 2.0, 1.0, 1.02, 0};
        default: return wide ? AttnShape{4, simt, 1, 2.8, 0.8, 1.2, 1.2, 0, 0, 0} : AttnShape{4, simt, 2, 2.5, 0.5, 0.7, 1.2, 0.8, 0.6, 0};
    }
}
bool is_tc(AttnKernel k) { return k == kTc1 || k == kTc2; }

bool is_rows(AttnKernel k) { return k == kSimt4 || k == kSimt8 || k == kRows; }

// What a segment asks of a kernel, and how long that takes.
struct Model {
    AttnShape sh;
    int sms;
    int64_t items, tiles;  // (sequence, key head, tile of rows); tiles of keys of each
    double bytes;          // of all keys and values, once
    double part_bytes;     // of one part of all rows
    int join_round;        // parts of a row that a join reads together

    // n parts: waves of CTAs, the SMs' throughput or the memory's, whichever is longest
    double us(int32_t n) const {
        const int64_t ctas = items * n, slots = (int64_t)sms * sh.ctas, waves = (ctas + slots - 1) / slots;
        const double each = (double)((tiles + n - 1) / n);
        double t = sh.fixed + (double)waves * (sh.setup + each * (ctas <= sms ? sh.tile : sh.shared));
        if (sh.sm_tile > 0) t = std::max(t, sh.fixed + (double)ctas / sms * (sh.sm_item + each * sh.sm_tile));
        return std::max(t, sh.fixed + sh.setup + bytes / 6.2e6);
    }
    // a launch that joins n parts: round trips, and the parts' bytes there and back
    double join_us(int32_t n) const {
        return sh.part + 0.2 + 1.6 * ((n + join_round - 1) / join_round) + 2. * n * part_bytes / 6e6;
    }
};
struct Choice {
    int32_t n;       // parts
    int cluster;     // CTAs of a cluster that joins them, or 1
    double us;
};

// The number of parts of the least time; fewer win a tie (1 %).
Choice choose_splits(const Model& m) {
    Choice best{1, 1, m.us(1)};
    for (int32_t n = 2; n <= MAFAT_ATTN_MAX_SPLITS && n <= m.tiles; ++n) {
        const double us = m.us(n) + m.join_us(n);
        if (us < 0.99 * best.us) best = {n, 1, us};
    }
    return best;
}

// Most parts that a tile of many rows joins at its end, and that a cluster has.  2 x 8 requests of 40 tokens about 3000
// states, 100 own keys, 16 query and 4 key heads, in us: three parts joined by the own keys' tiles 22.5 (64 channels) and
// 32.5 (128), by a launch 24.6 and 33.6.
constexpr int kTileJoin = 16, kMostCluster = 8;
// What a cluster's join takes (one token over 1444 states in clusters of 8: 4.9 us, the same work without a join 4.4), and
// the joining of another launch's parts is worth (above: 1.1 to 2.1 us).
constexpr double kClusterJoinUs = 0.7, kOwnJoinUs = 1.0;

int64_t row_tiles(const AttnShape& sh, int32_t rows) { return (rows + sh.rows - 1) / sh.rows; }

// One CTA an SM that leaves SMs idle: those take the last keys of all items, in as many rounds as that needs, while the others
// have the rest.  64 trees of 16 nodes about 23104 states (128 items of 181 tiles on 152 SMs), with their own keys: 263 us, 280 with
// whole items, in turn on one GPU; 265 to 287 on others, by their power.  For trees alone, as are the clusters over both sets below:
// nothing here needs one, but requests without keep the launches that they were measured with.
struct Cut {
    uint32_t share;  // of the first part; 0: whole items
    double us;
};
Cut choose_cut(const AttnShape& sh, int sms, int64_t items, int64_t tiles, double part_bytes) {
    const int64_t idle = sms - items;
    if (sh.ctas != 1 || idle < 1 || items < idle) return {0, 0.};
    const double rounds = (double)((items + idle - 1) / idle), whole = sh.setup + (double)tiles * sh.tile;
    const int64_t second = (int64_t)((whole - rounds * sh.setup) / ((rounds + 1.) * sh.tile));
    if (second < 1) return {0, 0.};
    const double us = sh.fixed + std::max(sh.setup + (double)(tiles - second) * sh.tile, rounds * (sh.setup + (double)second * sh.tile)) +
                      2. * part_bytes / 6e6 + 0.3;  // a part more there and back
    if (us > 0.98 * (sh.fixed + whole)) return {0, 0.};
    return {(uint32_t)std::ceil((double)(tiles - second) / (double)tiles * 4294967296.), us};
}

// The work of a segment: the kernel, tiles of rows, parts of the keys.
mafat_status plan_segment(mafat_attn_s& p, AttnSegPlan& g, const Common& c, int sms, bool second) {
    if (g.n > kMostCounted) return fail(MAFAT_EUNSUPPORTED, "too many keys");
    g.rows = g.reqs * p.n_q * (p.heads_q / p.heads_kv);
    const bool bf16 = p.dtype == MAFAT_BF16;
    AttnKernel kernels[3];
    int n_kernels = 0;
    if (c.kernel != MAFAT_ATTN_TILES || g.n == 0) {  // without keys there is nothing to map
        if (bf16)
            kernels[n_kernels++] = kRows;
        else
            kernels[n_kernels++] = g.rows <= 4 ? kSimt4 : kSimt8;
    }
    if (c.kernel != MAFAT_ATTN_ROWS && g.n > 0) {
        kernels[n_kernels++] = bf16 ? kTc1 : kSimt64;
        if (bf16 && g.rows > 128) kernels[n_kernels++] = kTc2;
    }
    Choice best{0, 1, 0.};
    for (int i = 0; i < n_kernels; ++i) {
        Model m;
        m.sh = shape_of(kernels[i], p.dim);
        m.sms = sms;
        m.items = (int64_t)g.n_seq * p.heads_kv * row_tiles(m.sh, g.rows);
        m.tiles = std::max<int64_t>(1, ((int64_t)g.n + m.sh.keys - 1) / m.sh.keys);
        m.bytes = 2. * g.n_seq * g.n * p.heads_kv * p.dim * (bf16 ? 2 : 4);
        m.part_bytes = 4. * p.dim * (double)p.rows_total;
        m.join_round = p.n_run == 2 || p.dim <= 64 ? 32 : 16;
        Choice x = choose_splits(m);
        if (c.splits) {
            x = {(int32_t)std::min<int64_t>(c.splits, m.tiles), 1, 0.};
            x.us = m.us(x.n);
        } else if (second && m.us(1) <= x.us + kOwnJoinUs) {
            x = {1, 1, m.us(1)};  // whole: it then joins the first launch's parts itself
        } else if (p.n_run == 1 && is_rows(kernels[i]) && m.items == (int64_t)g.n_seq * p.heads_kv && x.n > 1) {
            // A cluster joins its parts itself, which saves the launch for it: 5.1 us against 5.8 for one token of 8
            // heads over 1444 states, 7.2 against 8.7 for 16 requests, 6.3 against 7.4 for 4 over 676 of 32 heads.
            for (int32_t n = kMostCluster; n > 1 && x.cluster == 1; n /= 2)
                // clusters of CTAs that fill their SM find half of the SMs, not all, side by side
                if (n <= m.tiles && m.items * n <= (int64_t)sms * m.sh.ctas / (m.sh.ctas == 1 ? 2 : 1) &&
                    m.us(n) + kClusterJoinUs <= x.us)
                    x = {n, n, m.us(n) + kClusterJoinUs};
        }
        if (best.n == 0 || x.us < best.us) {
            best = x;
            g.kernel = kernels[i];
        }
    }
    g.us = best.us;
    const AttnShape sh = shape_of(g.kernel, p.dim);
    g.row_tiles = (int32_t)row_tiles(sh, g.rows);
    g.cut = 0;
    if (p.kind == kTree && p.n_run == 2 && !second && c.splits == 0 && g.kernel == kTc2 && best.n == 1) {
        Cut cut = choose_cut(sh, sms, (int64_t)g.n_seq * p.heads_kv * g.row_tiles, (g.n + sh.keys - 1) / sh.keys,
                             4. * p.dim * (double)p.rows_total);
        if (cut.share) {
            best.n = 2;
            g.cut = cut.share;
            g.us = cut.us;
        }
    }
    g.splits = best.n;
    p.cluster = best.cluster;
    const int64_t items = (int64_t)g.n_seq * p.heads_kv * g.row_tiles * g.splits;
    if (items > kMaxI32 / 4) return fail(MAFAT_EUNSUPPORTED, "too many items of work");
    g.items = (int32_t)items;
    // the kernel for few rows takes item after item
    g.ctas = g.kernel == kRows ? std::min(g.items, sms * sh.ctas) : g.items;
    g.part0 = p.parts;
    p.parts += g.splits;
    return MAFAT_OK;
}

// Whether both sets of keys of a prefix plan are better read by the same tiles of rows, of one request each: no parts and
// no second launch, where requests have rows enough to fill tiles or there is little to do.  In us, two launches and one:
// 8 requests of 61 tokens about each of 4 frames of 5776 states (16 query and 4 key heads, 128 channels) 78.4, 68.0;
// 32 of 46 tokens over 4 x 103 (8 and 4 heads of 80) 34.6, 18.7; 3 of a token over 2 x 100 (8 and 2 of 64) 6.1, 5.4; 16 of
// a token over 1444 (16 and 4 of 64) 7.3, 15.5; 8 of 64 over 3 x 13852 (8 and 4 of 128) 75, 133.
// Two launches whose first has whole results were measured to take 1 to 1.45 times what the model has for them (with
// parts, the launch to join them, which it counts, falls away).
constexpr double kTwoLaunches = 1.2, kClusterShare = 0.8, kShortShare = 0.9, kShortItemUs = 1.9;
void plan_both(mafat_attn_s& p, const Common& c, int sms) {
    if (p.dtype != MAFAT_BF16 || p.n_run != 2 || c.splits != 0 || c.kernel == MAFAT_ATTN_ROWS) return;
    const AttnSegPlan &first = p.seg[p.run[0]], &own = p.seg[p.run[1]];
    double best = first.us + own.us;
    if (first.splits == 1) best = kTwoLaunches * (best + kOwnJoinUs);
    for (AttnKernel k : {kTc1, kTc2}) {
        if (k == kTc2 && own.rows <= 128) continue;
        Model m{};
        m.sh = shape_of(k, p.dim);
        m.sms = sms;
        m.items = (int64_t)own.n_seq * p.heads_kv * row_tiles(m.sh, own.rows);
        m.tiles = ((int64_t)first.n + m.sh.keys - 1) / m.sh.keys + ((int64_t)own.n + m.sh.keys - 1) / m.sh.keys;
        m.bytes = 4. * p.heads_kv * p.dim * ((double)first.n_seq * first.n + (double)own.n_seq * own.n);
        if (m.items > kMaxI32 / 4 || m.us(1) >= best) continue;
        best = m.us(1);
        p.both = own;
        p.both.cut = 0;
        p.both.kernel = k;
        p.both.row_tiles = (int32_t)row_tiles(m.sh, own.rows);
        p.both.splits = 1;
        p.both.part0 = 0;
        p.both.items = p.both.ctas = (int32_t)m.items;
    }
    // Few rows of trees: clusters that split both sets' keys.  In us, as above (no clusters) and in clusters: a tree of 8 nodes over
    // 1444 + 96 keys (16 and 4 heads of 64) 7.5, 6.9; 8 of them (8 and 2 of 128) 13.4, 10.1; 4 x 2 trees of 3 over 96 + 116 (8 and 2 of
    // 64) 6.0, 5.4; 5 of 3 over 4663 + 4 (8 and 1 of 40) 9.8, 11.3.  Of 35 drawn plans they were slower in all whose time by the
    // model was more than kClusterShare of the others', and in 3 of the 28 below it, by up to 0.8.  Many short items, one after another
    // in a CTA, also in one launch: 8 x 30 trees of a node over 50 + 40 (8 and 2 of 64) 13.2, 8.7; 4 x 13 of 2 over 18 + 8 (8 heads of
    // 128) 14.2, 11.2; 43 of 5 over 22 + 41 (32 and 8 of 64) 11.8, 13.8.
    if (p.kind != kTree || c.kernel == MAFAT_ATTN_TILES || (int64_t)first.n + own.n > kMaxI32 / 16) return;
    Model m{};
    m.sh = shape_of(kRows, p.dim);
    m.sms = sms;
    m.items = (int64_t)own.n_seq * p.heads_kv * row_tiles(m.sh, own.rows);
    m.tiles = ((int64_t)first.n + m.sh.keys - 1) / m.sh.keys + ((int64_t)own.n + m.sh.keys - 1) / m.sh.keys;
    m.bytes = 4. * p.heads_kv * p.dim * ((double)own.n_seq * first.n + (double)own.n_seq * own.n);
    double least = best;
    for (int32_t n = kMostCluster; n > 0; n /= 2) {
        const int64_t slots = (int64_t)sms * m.sh.ctas;
        if (n > 1 ? n > m.tiles || m.items * n > slots : m.items > kMaxI32 / 4) continue;
        // of items of few tiles the start and the end are not hidden behind each other's copies
        const double us = n > 1 ? m.us(n) + kClusterJoinUs : m.us(1) + (double)((m.items + slots - 1) / slots) * kShortItemUs;
        if (us >= least || us >= (n > 1 ? kClusterShare : kShortShare) * best) continue;
        least = us;
        p.both = own;
        p.both.kernel = kRows;
        p.both.row_tiles = (int32_t)row_tiles(m.sh, own.rows);
        p.both.splits = p.both_cluster = n;
        p.both.part0 = 0;
        p.both.cut = 0;
        p.both.items = (int32_t)(m.items * n);
        p.both.ctas = n > 1 ? p.both.items : std::min(p.both.items, sms * m.sh.ctas);
    }
}

// 4-D map {channel, head, key, sequence} of keys or values; boxes of 64 channels x 128 keys of one head.
// Places past a dimension's end read as zero.
mafat_status encode_map(CUtensorMap* m, const void* base, const AttnSegPlan& g, const int64_t st[3], int heads, int dim) {
    const auto fn = (PFN_cuTensorMapEncodeTiled_v12000)mafat_internal_encode_tiled();
    if (!fn) return fail(MAFAT_ECUDA, "cuTensorMapEncodeTiled unavailable");
    const cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)g.n, (cuuint64_t)g.n_seq};
    const cuuint64_t strides[3] = {(cuuint64_t)st[2] * 2, (cuuint64_t)st[1] * 2, (cuuint64_t)st[0] * 2};
    const cuuint32_t box[4] = {64, 1, 128, 1}, estr[4] = {1, 1, 1, 1};
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(MAFAT_ECUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
    return MAFAT_OK;
}

mafat_status finish_plan(mafat_attn_s* p, const Common& c, mafat_attn_t** out) {
    p->dtype = c.dtype;
    p->batch = c.batch;
    p->n_q = c.n_q;
    p->heads_q = c.heads_q;
    p->heads_kv = c.heads_kv;
    p->dim = c.dim;
    p->scale = c.scale == 0.f ? 1.f / std::sqrt((float)c.dim) : c.scale;
    p->dry_run = c.dry_run != 0;
    p->rows_total = (int64_t)c.batch * c.n_q * c.heads_q;
    const int64_t esz = c.dtype == MAFAT_BF16 ? 2 : 4;
    const int64_t n[3] = {c.batch, c.n_q, c.heads_q};
    mafat_status st;
    if ((st = take_strides("q_strides", c.q, n, c.dim, esz, p->q)) != MAFAT_OK) return st;
    if ((st = take_strides("out_strides", c.o, n, c.dim, esz, p->o)) != MAFAT_OK) return st;
    if (!places_distinct(n, p->o, c.dim)) return fail(MAFAT_EINVAL, "out_strides: elements share a place");
    int sms = 152;
    cudaError_t e;
    if (!p->dry_run) {
        if ((e = cudaGetDevice(&p->device)) != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
        sms = sm_count(p->device);
    }
    p->sms = sms;
    for (int i = 0; i < p->n_seg; ++i)
        if (p->seg[i].n > 0) p->run[p->n_run++] = i;
    if (p->n_run == 0) p->run[p->n_run++] = 0;
    for (int i = 0; i < p->n_run; ++i)
        if ((st = plan_segment(*p, p->seg[p->run[i]], c, sms, i > 0)) != MAFAT_OK) return st;
    if (p->n_run == 2) {
        const AttnSegPlan &first = p->seg[p->run[0]], &last = p->seg[p->run[1]];
        p->joined = last.splits == 1 && first.splits <= (last.kernel == kRows ? mafat_attn_rows_join() : kTileJoin);
        if (p->joined) p->parts = first.splits;
        plan_both(*p, c, sms);
    }
    if (p->cluster > 1) p->parts = 1;  // none goes through the workspace
    const int64_t lse_bytes = (p->rows_total * p->parts * 4 + 255) / 256 * 256;
    p->workspace_bytes = kStatusBytes + (p->parts > 1 || p->joined ? lse_bytes + p->rows_total * p->parts * p->dim * 4 : 0);
    if (!p->dry_run) {
        // what the plan can launch, of its type, kind and channels alone: a plan takes 18 us, with all kernels 39, and a program's first
        // one, which loads them, 1.5 ms instead of 3.7
        const bool tree = p->kind == kTree;
        if (c.dtype == MAFAT_FP32)
            e = mafat_prepare_attn_simt(tree, p->dim);
        else if ((e = mafat_prepare_attn_rows(tree, p->dim)) == cudaSuccess)
            e = mafat_prepare_attn_tc(tree, p->dim);
        if (e != cudaSuccess)
            return cuda_fail(e, "attention kernels");
        if ((e = cudaMalloc(&p->workspace, (size_t)p->workspace_bytes)) != cudaSuccess) return cuda_fail(e, "cudaMalloc");
        p->status = (uint32_t*)p->workspace;
        p->part_lse = (float*)((char*)p->workspace + kStatusBytes);
        p->part_o = (float*)((char*)p->workspace + kStatusBytes + lse_bytes);
        if ((e = cudaMemset(p->status, 0, kStatusBytes)) != cudaSuccess) return cuda_fail(e, "cudaMemset");
        if ((e = transfers_done()) != cudaSuccess) return cuda_fail(e, "cudaStreamSynchronize");
    }
    *out = p;
    mafat_internal_clear_error();
    return MAFAT_OK;
}

struct SegData {
    const void *k, *v;
    const int32_t* len;
    const uint8_t* mask;
};

// What a tree's run has more.
struct TreeData {
    const int32_t* nodes = nullptr;
    const uint32_t* tree = nullptr;
    bool shared = false;
};

mafat_status run(const mafat_attn_s* p, AttnKind kind, const void* q, const SegData* d, const TreeData& tree, void* out,
                 float* lse, cudaStream_t s) {
    if (p->kind != kind) return fail(MAFAT_EINVAL, "the plan is one of %s", kAttnPlans[p->kind]);
    if (p->dry_run) return fail(MAFAT_EINVAL, "plan was created with dry_run");
    if (!q || !out) return fail(MAFAT_EINVAL, "null q or out");
    if (!aligned(q) || !aligned(out) || !aligned(lse, 4)) return fail(MAFAT_EINVAL, "q and out must be 16-byte aligned, lse 4-byte");
    const int64_t esz = p->dtype == MAFAT_BF16 ? 2 : 4;
    const int64_t nq[3] = {p->batch, p->n_q, p->heads_q};
    const int64_t out_bytes = extent(nq, p->o, p->dim, esz), lse_bytes = lse ? p->rows_total * 4 : 0;
    auto clear = [&](const void* x, int64_t bytes) {
        return !overlap(out, out_bytes, x, bytes) && !overlap(lse, lse_bytes, x, bytes);
    };
    if (overlap(out, out_bytes, lse, lse_bytes) || !clear(q, extent(nq, p->q, p->dim, esz)))
        return fail(MAFAT_EINVAL, "an output overlaps another tensor");
    MafatAttnArgs a{};
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.q_sb = p->q[0]; a.q_st = p->q[1]; a.q_sh = p->q[2];
    a.o_sb = p->o[0]; a.o_st = p->o[1]; a.o_sh = p->o[2];
    a.n_q = p->n_q;
    a.group = p->heads_q / p->heads_kv;
    a.heads_q = p->heads_q;
    a.heads_kv = p->heads_kv;
    a.dim = p->dim;
    a.n_q_div = MafatDiv((uint32_t)a.n_q);
    a.group_div = MafatDiv((uint32_t)a.group);
    a.heads_q_div = MafatDiv((uint32_t)a.heads_q);
    a.heads_kv_div = MafatDiv((uint32_t)a.heads_kv);
    a.parts = p->parts;
    a.scale_log2 = (float)((double)p->scale * 1.4426950408889634);
    a.part_o = p->part_o;
    a.part_lse = p->part_lse;
    a.rows_total = p->rows_total;
    a.status = p->status;
    a.timeout_ns = 2000000000LL;
    for (int i = 0; i < p->n_seg; ++i) {
        const AttnSegPlan& g = p->seg[i];
        const int64_t nk[3] = {g.n_seq, g.n, p->heads_kv};
        if (g.n > 0) {
            if (!d[i].k || !d[i].v) return fail(MAFAT_EINVAL, "null keys or values");
            if (!aligned(d[i].k) || !aligned(d[i].v)) return fail(MAFAT_EINVAL, "keys and values must be 16-byte aligned");
            if (!clear(d[i].k, extent(nk, g.k, p->dim, esz)) || !clear(d[i].v, extent(nk, g.v, p->dim, esz)) ||
                !clear(d[i].mask, (int64_t)g.n_seq * g.n))
                return fail(MAFAT_EINVAL, "an output overlaps another tensor");
        }
        if (!aligned(d[i].len, 4)) return fail(MAFAT_EINVAL, "lengths must be 4-byte aligned");
        if (!clear(d[i].len, (int64_t)g.n_seq * 4)) return fail(MAFAT_EINVAL, "an output overlaps another tensor");
    }
    const int32_t tree_words = (p->n_q + 31) / 32;
    if (kind == kTree) {
        if (!tree.tree) return fail(MAFAT_EINVAL, "null tree");
        if (!aligned(tree.tree, 4) || !aligned(tree.nodes, 4)) return fail(MAFAT_EINVAL, "tree and nodes must be 4-byte aligned");
        if (!clear(tree.tree, (int64_t)(tree.shared ? 1 : p->batch) * p->n_q * tree_words * 4) ||
            !clear(tree.nodes, (int64_t)p->batch * 4))
            return fail(MAFAT_EINVAL, "an output overlaps another tensor");
        a.tree = 1;
        a.nodes = tree.nodes;
    }
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    if (dev != p->device) return fail(MAFAT_EINVAL, "the current device is not the plan's");
    const bool both = p->both.items > 0 && !d[p->run[0]].mask;
    for (int r = both ? 1 : 0; r < p->n_run; ++r) {
        const int i = p->run[r];
        const AttnSegPlan& g = both ? p->both : p->seg[i];
        MafatAttnSeg& x = a.seg;
        x.k = d[i].k;
        x.v = d[i].v;
        x.k_sb = g.k[0]; x.k_ss = g.k[1]; x.k_sh = g.k[2];
        x.v_sb = g.v[0]; x.v_ss = g.v[1]; x.v_sh = g.v[2];
        x.len = d[i].len;
        x.mask = d[i].mask;
        x.tree = i == 1 ? tree.tree : nullptr;
        x.tree_s = tree.shared ? 0 : (int64_t)p->n_q * tree_words;
        x.tree_words = tree_words;
        x.n = g.n;
        x.causal = g.causal;
        x.reqs = g.reqs;
        x.n_seq = g.n_seq;
        x.rows = g.rows;
        x.row_tiles = g.row_tiles;
        x.splits = g.splits;
        x.row_tiles_div = MafatDiv((uint32_t)g.row_tiles);
        x.splits_div = MafatDiv((uint32_t)g.splits);
        x.part0 = g.part0;
        x.items = g.items;
        x.cut = g.cut;
        a.overlap = r > 0 && !both;
        // Fewer CTAs than SMs, of which two fit an SM: launched while the call before ends, they would gather on the SMs that are free
        // first.  fp32 in us, one call behind another and two programs' calls from two streams, by themselves and two an SM:
        // 6 x 7 requests of 24 tokens over 13517 + 40 keys (4 and 2 heads of 64) 490, 957 and 837, 883; 4 x 64 tokens of 16 heads of 64 over
        // 676 34, 63 and 54, 58.  As many as the SMs gain nothing by it (19 x 64 tokens of 8 heads over 5776: 412, 821 and 410, 734), nor does
        // a launch that runs beside the one before it (4 x 8 requests of 8 over 5776 + 200, 16 and 4 heads of 128: 331, 626 and 323, 597), nor
        // bf16 tiles of 128 rows (19 x 128 tokens of 8 heads over 676: 9.5, 18.4 and 10.0, 12.4).
        a.alone = g.kernel == kSimt64 && !a.overlap && g.items < p->sms;
        a.join = r > 0 && p->joined && !both ? p->parts : 0;
        a.cluster = both ? p->both_cluster : p->cluster;
        // where a CTA has several items; of more sequences it has so many that they level it
        a.ordered = g.kernel == kRows && x.len && g.n_seq > 1 && g.n_seq <= kMafatMostOrdered && g.items > g.ctas;
        a.direct = both || a.join || (p->parts == 1 && !p->joined);
        if (is_tc(g.kernel)) {
            CUtensorMap k, v;
            mafat_status st;
            if ((st = encode_map(&k, d[i].k, g, g.k, p->heads_kv, p->dim)) != MAFAT_OK ||
                (st = encode_map(&v, d[i].v, g, g.v, p->heads_kv, p->dim)) != MAFAT_OK)
                return st;
            MafatAttnPrefix prefix;
            if (both) {
                const AttnSegPlan& f = p->seg[p->run[0]];
                const SegData& fd = d[p->run[0]];
                if ((st = encode_map(&prefix.k, fd.k, f, f.k, p->heads_kv, p->dim)) != MAFAT_OK ||
                    (st = encode_map(&prefix.v, fd.v, f, f.v, p->heads_kv, p->dim)) != MAFAT_OK)
                    return st;
                prefix.len = fd.len;
                prefix.n = f.n;
                prefix.per = MafatDiv((uint32_t)f.reqs);
            }
            e = mafat_launch_attn_tc(a, k, v, g.kernel == kTc2 ? 2 : 1, both ? &prefix : nullptr, s);
        } else {
            MafatRowsPrefix prefix;
            if (both) {
                const AttnSegPlan& f = p->seg[p->run[0]];
                const SegData& fd = d[p->run[0]];
                prefix = {fd.k, fd.v, f.k[0], f.k[1], f.k[2], f.v[0], f.v[1], f.v[2], fd.len, f.n, MafatDiv((uint32_t)f.reqs)};
            }
            e = g.kernel == kRows ? mafat_launch_attn_rows(a, g.ctas, both ? &prefix : nullptr, s) : mafat_launch_attn_simt(a, shape_of(g.kernel, p->dim).rows, s);
        }
        if (e != cudaSuccess) return cuda_fail(e, "attention launch");
    }
    if (p->parts > 1 && !p->joined && !both) {
        a.overlap = 0;
        e = mafat_launch_attn_join(a, p->dtype == MAFAT_BF16, s);
        if (e != cudaSuccess) return cuda_fail(e, "join launch");
    }
    return MAFAT_OK;
}

// kind: kPrefix, or kTree, whose own keys each row reads by its bits
mafat_status prefix_plan(const mafat_prefix_desc* d, AttnKind kind, mafat_attn_t** out) {
    if (!d || !out) return fail(MAFAT_EINVAL, "null argument");
    *out = nullptr;
    if (d->struct_size != (int32_t)sizeof(mafat_prefix_desc)) return fail(MAFAT_EINVAL, "struct_size is not the descriptor's");
    if (d->prefixes < 1 || d->requests < 1) return fail(MAFAT_EINVAL, "prefixes and requests must be positive");
    if (d->prefixes > kMaxI32 / d->requests) return fail(MAFAT_EUNSUPPORTED, "too many requests");
    const Common c{d->dtype, d->prefixes * d->requests, d->n_q, d->heads_q, d->heads_kv, d->head_dim, d->kernel,
                   d->splits, d->dry_run, d->scale, d->q_strides, d->out_strides};
    mafat_status st = check_common(c);
    if (st != MAFAT_OK) return st;
    if (d->n_prefix < 0 || d->n_own < 0) return fail(MAFAT_EINVAL, "n_prefix and n_own must not be negative");
    mafat_attn_s* p = new (std::nothrow) mafat_attn_s();
    if (!p) return fail(MAFAT_ENOMEM, "host allocation failed");
    p->kind = kind;
    p->n_seg = 2;
    AttnSegPlan &g = p->seg[0], &w = p->seg[1];
    g.n_seq = d->prefixes;
    g.reqs = d->requests;
    g.n = d->n_prefix;
    w.n_seq = c.batch;
    w.reqs = 1;
    w.n = d->n_own;
    w.causal = kind == kPrefix;
    const int64_t esz = d->dtype == MAFAT_BF16 ? 2 : 4;
    const int64_t np[3] = {d->prefixes, d->n_prefix, d->heads_kv}, no[3] = {c.batch, d->n_own, d->heads_kv};
    if ((st = take_strides("prefix_k_strides", d->prefix_k_strides, np, d->head_dim, esz, g.k)) != MAFAT_OK ||
        (st = take_strides("prefix_v_strides", d->prefix_v_strides, np, d->head_dim, esz, g.v)) != MAFAT_OK ||
        (st = take_strides("own_k_strides", d->own_k_strides, no, d->head_dim, esz, w.k)) != MAFAT_OK ||
        (st = take_strides("own_v_strides", d->own_v_strides, no, d->head_dim, esz, w.v)) != MAFAT_OK ||
        (st = finish_plan(p, c, out)) != MAFAT_OK)
        mafat_attn_destroy(p);
    return st;
}

}  // namespace

extern "C" {

mafat_status mafat_cross_plan(const mafat_cross_desc* d, mafat_attn_t** out) {
    if (!d || !out) return fail(MAFAT_EINVAL, "null argument");
    *out = nullptr;
    if (d->struct_size != (int32_t)sizeof(mafat_cross_desc)) return fail(MAFAT_EINVAL, "struct_size is not the descriptor's");
    const Common c{d->dtype, d->batch, d->n_q, d->heads_q, d->heads_kv, d->head_dim, d->kernel, d->splits, d->dry_run,
                   d->scale, d->q_strides, d->out_strides};
    mafat_status st = check_common(c);
    if (st != MAFAT_OK) return st;
    if (d->n_kv < 0) return fail(MAFAT_EINVAL, "n_kv must not be negative");
    mafat_attn_s* p = new (std::nothrow) mafat_attn_s();
    if (!p) return fail(MAFAT_ENOMEM, "host allocation failed");
    p->n_seg = 1;
    AttnSegPlan& g = p->seg[0];
    g.n_seq = d->batch;
    g.reqs = 1;
    g.n = d->n_kv;
    const int64_t esz = d->dtype == MAFAT_BF16 ? 2 : 4, n[3] = {d->batch, d->n_kv, d->heads_kv};
    if ((st = take_strides("k_strides", d->k_strides, n, d->head_dim, esz, g.k)) != MAFAT_OK ||
        (st = take_strides("v_strides", d->v_strides, n, d->head_dim, esz, g.v)) != MAFAT_OK ||
        (st = finish_plan(p, c, out)) != MAFAT_OK)
        mafat_attn_destroy(p);
    return st;
}

mafat_status mafat_cross_run(const mafat_attn_t* p, const void* q, const void* k, const void* v, const int32_t* kv_len,
                             const uint8_t* kv_mask, void* out, float* lse, void* stream) {
    if (!p) return fail(MAFAT_EINVAL, "null plan");
    const SegData d[1] = {{k, v, kv_len, kv_mask}};
    return run(p, kCross, q, d, TreeData(), out, lse, (cudaStream_t)stream);
}

mafat_status mafat_prefix_plan(const mafat_prefix_desc* d, mafat_attn_t** out) { return prefix_plan(d, kPrefix, out); }

mafat_status mafat_prefix_run(const mafat_attn_t* p, const void* q, const void* prefix_k, const void* prefix_v,
                              const int32_t* prefix_len, const uint8_t* prefix_mask, const void* own_k,
                              const void* own_v, const int32_t* own_len, void* out, float* lse, void* stream) {
    if (!p) return fail(MAFAT_EINVAL, "null plan");
    const SegData d[2] = {{prefix_k, prefix_v, prefix_len, prefix_mask}, {own_k, own_v, own_len, nullptr}};
    return run(p, kPrefix, q, d, TreeData(), out, lse, (cudaStream_t)stream);
}

mafat_status mafat_tree_plan(const mafat_prefix_desc* d, mafat_attn_t** out) { return prefix_plan(d, kTree, out); }

mafat_status mafat_tree_run(const mafat_attn_t* p, const void* q, const void* prefix_k, const void* prefix_v,
                            const int32_t* prefix_len, const uint8_t* prefix_mask, const void* own_k, const void* own_v,
                            const int32_t* own_len, const int32_t* nodes, const uint32_t* tree, int32_t tree_shared,
                            void* out, float* lse, void* stream) {
    if (!p) return fail(MAFAT_EINVAL, "null plan");
    const SegData d[2] = {{prefix_k, prefix_v, prefix_len, prefix_mask}, {own_k, own_v, own_len, nullptr}};
    return run(p, kTree, q, d, TreeData{nodes, tree, tree_shared != 0}, out, lse, (cudaStream_t)stream);
}

mafat_status mafat_attn_stats(const mafat_attn_t* p, mafat_attn_stats_t* out) {
    if (!p || !out) return fail(MAFAT_EINVAL, "null argument");
    if (out->struct_size < (int32_t)sizeof(mafat_attn_stats_t)) return fail(MAFAT_EINVAL, "struct_size too small");
    mafat_attn_stats_t s{};
    s.struct_size = (int32_t)sizeof(mafat_attn_stats_t);
    for (int r = 0; r < p->n_run; ++r) {
        const int i = p->run[r];
        s.kernel[i] = is_rows(p->seg[i].kernel) ? MAFAT_ATTN_ROWS : MAFAT_ATTN_TILES;
        s.splits[i] = p->seg[i].splits;
        s.ctas[i] = p->seg[i].ctas;
    }
    s.parts = p->parts;
    s.launches_per_run = p->n_run + (p->parts > 1 && !p->joined ? 1 : 0);
    s.whole_ctas = p->both.ctas;
    s.workspace_bytes = p->workspace_bytes;
    *out = s;
    return MAFAT_OK;
}

mafat_status mafat_attn_sync_status(const mafat_attn_t* p, void* stream) {
    if (!p) return fail(MAFAT_EINVAL, "null plan");
    if (p->dry_run) return fail(MAFAT_EINVAL, "plan was created with dry_run");
    cudaError_t e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(e, "cudaStreamSynchronize");
    uint32_t st = 0;
    if ((e = cudaMemcpy(&st, p->status, sizeof(st), cudaMemcpyDeviceToHost)) != cudaSuccess) return cuda_fail(e, "cudaMemcpy");
    if (st == MAFAT_DEV_OK) return MAFAT_OK;
    if ((e = cudaMemset(p->status, 0, kStatusBytes)) != cudaSuccess) return cuda_fail(e, "cudaMemset");
    if ((e = transfers_done()) != cudaSuccess) return cuda_fail(e, "cudaStreamSynchronize");
    return fail(MAFAT_EDEVICE, "a device pipeline wait ran out");
}

void mafat_attn_destroy(mafat_attn_t* p) {
    if (!p) return;
    if (p->workspace) cudaFree(p->workspace);
    delete p;
}

mafat_status mafat_rms_norm(const mafat_norm_desc* d, const void* x, const void* residual, const void* weight,
                            void* residual_out, void* y, float* scales, void* stream) {
    if (!d) return fail(MAFAT_EINVAL, "null argument");
    if (d->struct_size != (int32_t)sizeof(mafat_norm_desc)) return fail(MAFAT_EINVAL, "struct_size is not the descriptor's");
    if (d->dtype != MAFAT_BF16 && d->dtype != MAFAT_FP32) return fail(MAFAT_EINVAL, "dtype must be MAFAT_BF16 or MAFAT_FP32");
    if (d->out_dtype != d->dtype && d->out_dtype != MAFAT_E4M3) return fail(MAFAT_EINVAL, "out_dtype must be dtype or MAFAT_E4M3");
    const bool quant = d->out_dtype == MAFAT_E4M3;
    if (d->rows < 0 || d->cols < 1) return fail(MAFAT_EINVAL, "rows must not be negative and cols must be positive");
    if (d->cols > mafat_norm_max_cols()) return fail(MAFAT_EUNSUPPORTED, "at most %d cols", mafat_norm_max_cols());
    if (d->rows > kMaxI32) return fail(MAFAT_EUNSUPPORTED, "too many rows");
    if (!(d->eps >= 0.f) || std::isinf(d->eps)) return fail(MAFAT_EINVAL, "eps must be finite and not negative");
    if (quant && d->scale_group != 0 && d->scale_group != 128)
        return fail(MAFAT_EUNSUPPORTED, "scale_group must be 0 (the row) or 128");
    if (!quant && d->scale_group != 0) return fail(MAFAT_EINVAL, "scale_group without an 8-bit output");
    if (d->rows == 0) {
        mafat_internal_clear_error();
        return MAFAT_OK;
    }
    if (!x || !weight || !y) return fail(MAFAT_EINVAL, "null x, weight or y");
    if (quant != (scales != nullptr)) return fail(MAFAT_EINVAL, "an 8-bit output takes scales, others take none");
    const int64_t esz = d->dtype == MAFAT_BF16 ? 2 : 4, osz = quant ? 1 : esz;
    const int64_t st[4] = {d->x_stride, d->residual_stride, d->residual_out_stride, d->y_stride};
    int64_t row[4];
    for (int i = 0; i < 4; ++i) {
        row[i] = st[i] == 0 ? d->cols : st[i];
        if (row[i] < d->cols) return fail(MAFAT_EINVAL, "a row stride is smaller than cols");
        if (row[i] > (int64_t)1 << 40) return fail(MAFAT_EUNSUPPORTED, "a row stride is too large");
    }
    const void* t[6] = {x, residual, residual_out, y, weight, scales};
    for (int i = 0; i < 6; ++i)
        if (!aligned(t[i], i == 5 ? 4 : 16)) return fail(MAFAT_EINVAL, "tensors must be 16-byte aligned (scales: 4-byte)");
    MafatNormArgs a{};
    a.groups = !quant ? 0 : d->scale_group == 0 ? 1 : (d->cols + 127) / 128;
    int64_t bytes[6];
    for (int i = 0; i < 4; ++i) bytes[i] = t[i] ? ((d->rows - 1) * row[i] + d->cols) * (i == 3 ? osz : esz) : 0;
    bytes[4] = d->cols * esz;
    bytes[5] = d->rows * a.groups * 4;
    // an output may be an input in place: the same rows, of the same type
    for (int o : {2, 3, 5})
        for (int i = 0; i < 6; ++i) {
            if (i == o || !overlap(t[o], bytes[o], t[i], bytes[i])) continue;
            const bool in_place = i < 2 && o != 5 && t[i] == t[o] && row[i] == row[o] && (o != 3 || osz == esz);
            if (!in_place) return fail(MAFAT_EINVAL, "an output overlaps another tensor");
        }
    int64_t steps = d->cols;  // rows start and end on multiples of its lowest bit
    for (int i = 0; i < 4; ++i)
        if (t[i]) steps |= row[i];
    const int vec = (int)std::min<int64_t>(steps & -steps, 8);
    a.x = x;
    a.residual = residual;
    a.weight = weight;
    a.residual_out = residual_out;
    a.y = y;
    a.scales = scales;
    a.rows = d->rows;
    a.x_s = row[0];
    a.r_s = row[1];
    a.ro_s = row[2];
    a.y_s = row[3];
    a.cols = d->cols;
    a.eps = d->eps;
    const cudaError_t e = mafat_launch_norm(a, d->dtype == MAFAT_BF16, vec,
                                            !quant ? MAFAT_NORM_PLAIN : d->scale_group == 0 ? MAFAT_NORM_ROW : MAFAT_NORM_BLOCK,
                                            (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(e, "norm launch");
    return MAFAT_OK;
}

}  // extern "C"
