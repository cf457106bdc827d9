// C ABI of the operators of a decoding step beside attention: the norms around a block, rotary positions,
// adjusted logits.  Checks of arguments and launches.  See include/mafat.h.
#include <cuda_runtime.h>

#include <cmath>
#include <new>

#include "../../include/mafat.h"
#include "attention.h"
#include "decode.h"
#include "lm_checks.h"

struct mafat_rotary_s {
    bool dry_run = false, interleaved = false;
    int device = 0;
    int32_t dtype = 0, dim = 0, rot = 0;
    double magnitude = 1.;
    double* frequencies = nullptr;  // [rot / 2]
    uint64_t* turns = nullptr;      // device: of a turn, times 2^64
};

namespace {

using namespace mafat_lm;

constexpr double kTurn = 6.283185307179586476925286766559;

// [rot / 2] radians a position
void fill_frequencies(const mafat_rotary_desc& d, int rot, double base, double factor, double fast, double slow, double* f) {
    if (d.scaling == MAFAT_ROTARY_BASE) base *= std::pow(factor, (double)rot / (rot - 2));
    for (int i = 0; i < rot / 2; ++i) {
        f[i] = d.frequencies ? d.frequencies[i] : std::pow(base, -2. * i / rot);
        if (d.scaling == MAFAT_ROTARY_LINEAR) f[i] /= factor;
        if (d.scaling == MAFAT_ROTARY_BLEND) {
            const double turns = d.first_positions * f[i] / kTurn;
            const double keep = std::min(std::max((turns - slow) / (fast - slow), 0.), 1.);
            f[i] *= keep + (1. - keep) / factor;
        }
    }
}

// Radians as a fraction of a turn, times 2^64; whole turns fall away.  1 / 2 pi in two doubles and the product's own rounding
// error by an fma, so that the fraction is good to its last places and the angle at the farthest position to 2^-32 of a turn.
uint64_t turn_of(double radians) {
    constexpr double kInv = 0.15915494309189535, kInvLow = -9.839338337591243e-18;
    const double high = radians * kInv, low = std::fma(radians, kInv, -high) + radians * kInvLow;
    const double part = high - std::floor(high);
    const uint64_t x = part < 1. ? (uint64_t)(part * 18446744073709551616.) : 0u;  // a tiny negative one rounds to 1
    return x + (uint64_t)(int64_t)std::llround(low * 18446744073709551616.);
}

// Whether two tensors of [n0][n1][heads][dim] share no element, as far as strides show it: their extents are apart, or there is a step of
// which all strides that reach it are multiples, and past whole steps the elements of each lie in a run of their own.  (Keys and
// values of one cache, or of one matrix, in any order of its dimensions.)
struct Placed {
    const void* p;
    const int64_t* n;
    const int64_t* st;
    bool steps(int i) const { return n[i] > 1; }
    // what the strides below the step span, 0 where one that reaches it is no multiple
    int64_t run(int64_t step, int64_t dim) const {
        int64_t r = dim;
        for (int i = 0; i < 3; ++i) {
            if (!steps(i)) continue;
            if (st[i] < step)
                r += (n[i] - 1) * st[i];
            else if (st[i] % step != 0)
                return 0;
        }
        return r;
    }
};
bool apart(const Placed& a, const Placed& b, int64_t dim, int64_t esz) {
    if (!overlap(a.p, extent(a.n, a.st, dim, esz), b.p, extent(b.n, b.st, dim, esz))) return true;
    const int64_t off = ((const char*)b.p - (const char*)a.p) / esz;
    for (const Placed* t : {&a, &b})
        for (int i = 0; i < 3; ++i) {
            if (!t->steps(i)) continue;
            const int64_t step = t->st[i], ra = a.run(step, dim), rb = b.run(step, dim), at = (off % step + step) % step;
            if (ra && rb && at >= ra && at + rb <= step) return true;
        }
    return false;
}

int32_t lowest_bit(int64_t x, int64_t most) { return (int32_t)std::min<int64_t>(x & -x, most); }

}  // namespace

extern "C" {

mafat_status mafat_block_norm(const mafat_block_norm_desc* d, const void* x, const void* residual, const void* post_weight,
                              const void* gate, const void* weight, void* residual_out, void* y, float* scales, void* stream) {
    if (!d) return fail(MAFAT_EINVAL, "null argument");
    if (d->struct_size != (int32_t)sizeof(mafat_block_norm_desc)) return fail(MAFAT_EINVAL, "struct_size is not the descriptor's");
    if (d->dtype != MAFAT_BF16 && d->dtype != MAFAT_FP32) return fail(MAFAT_EINVAL, "dtype must be MAFAT_BF16 or MAFAT_FP32");
    if (d->out_dtype != d->dtype && d->out_dtype != MAFAT_E4M3) return fail(MAFAT_EINVAL, "out_dtype must be dtype or MAFAT_E4M3");
    const bool quant = d->out_dtype == MAFAT_E4M3;
    if (d->rows < 0 || d->cols < 1) return fail(MAFAT_EINVAL, "rows must not be negative and cols must be positive");
    if (d->cols > mafat_norm_max_cols()) return fail(MAFAT_EUNSUPPORTED, "at most %d cols", mafat_norm_max_cols());
    if (d->rows > kMaxI32) return fail(MAFAT_EUNSUPPORTED, "too many rows");
    if (!(d->eps >= 0.f) || std::isinf(d->eps)) return fail(MAFAT_EINVAL, "eps must be finite and not negative");
    if (!std::isfinite(d->branch_scale) || !std::isfinite(d->residual_scale)) return fail(MAFAT_EINVAL, "scales must be finite");
    if (quant && d->scale_group != 0 && d->scale_group != 128)
        return fail(MAFAT_EUNSUPPORTED, "scale_group must be 0 (the row) or 128");
    if (!quant && d->scale_group != 0) return fail(MAFAT_EINVAL, "scale_group without an 8-bit output");
    if (d->gate_rows < 0) return fail(MAFAT_EINVAL, "gate_rows must not be negative");
    if (d->rows == 0) {
        mafat_internal_clear_error();
        return MAFAT_OK;
    }
    const int64_t per_gate = d->gate_rows == 0 ? d->rows : d->gate_rows;
    if (d->rows % per_gate != 0) return fail(MAFAT_EINVAL, "gate_rows must divide rows");
    if (!x || !residual) return fail(MAFAT_EINVAL, "null x or residual");
    if ((y != nullptr) != (weight != nullptr)) return fail(MAFAT_EINVAL, "weight and y are given together");
    if (!y && !residual_out) return fail(MAFAT_EINVAL, "neither residual_out nor y");
    if (quant && !y) return fail(MAFAT_EINVAL, "an 8-bit output without y");
    if (quant != (scales != nullptr)) return fail(MAFAT_EINVAL, "an 8-bit output takes scales, others take none");
    const int64_t esz = d->dtype == MAFAT_BF16 ? 2 : 4, osz = quant ? 1 : esz;
    const int64_t st[5] = {d->x_stride, d->residual_stride, d->residual_out_stride, d->y_stride, d->gate_stride};
    int64_t row[5];
    for (int i = 0; i < 5; ++i) {
        row[i] = st[i] == 0 ? d->cols : st[i];
        if (row[i] < d->cols) return fail(MAFAT_EINVAL, "a row stride is smaller than cols");
        if (row[i] > (int64_t)1 << 40) return fail(MAFAT_EUNSUPPORTED, "a row stride is too large");
    }
    enum { kX, kResidual, kH, kY, kGate, kWeight, kPostWeight, kScales, kTensors };
    const void* t[kTensors] = {x, residual, residual_out, y, gate, weight, post_weight, scales};
    for (int i = 0; i < kTensors; ++i)
        if (!aligned(t[i], i == kScales ? 4 : 16)) return fail(MAFAT_EINVAL, "tensors must be 16-byte aligned (scales: 4-byte)");
    MafatBlockNormArgs a{};
    a.n.groups = !quant ? 0 : d->scale_group == 0 ? 1 : (d->cols + 127) / 128;
    int64_t bytes[kTensors];
    for (int i = 0; i < 5; ++i) {
        const int64_t n = i == kGate ? d->rows / per_gate : d->rows;
        if (t[i] && (__int128)(n - 1) * row[i] * esz > (__int128)1 << 62) return fail(MAFAT_EUNSUPPORTED, "a tensor spans more than 2^62 bytes");
        bytes[i] = t[i] ? ((n - 1) * row[i] + d->cols) * (i == kY ? osz : esz) : 0;
    }
    bytes[kWeight] = bytes[kPostWeight] = d->cols * esz;
    bytes[kScales] = d->rows * a.n.groups * 4;
    // an output may be an input in place: the same rows, of the same type
    for (int o : {(int)kH, (int)kY, (int)kScales})
        for (int i = 0; i < kTensors; ++i) {
            if (i == o || !overlap(t[o], bytes[o], t[i], bytes[i])) continue;
            const bool in_place = i <= kResidual && o != kScales && t[i] == t[o] && row[i] == row[o] && (o != kY || osz == esz);
            if (!in_place) return fail(MAFAT_EINVAL, "an output overlaps another tensor");
        }
    int64_t steps = d->cols;  // rows start and end on multiples of its lowest bit
    for (int i = 0; i < 5; ++i)
        if (t[i]) steps |= row[i];
    a.n.x = x;
    a.n.residual = residual;
    a.n.weight = weight;
    a.n.residual_out = residual_out;
    a.n.y = y;
    a.n.scales = scales;
    a.n.rows = d->rows;
    a.n.x_s = row[kX];
    a.n.r_s = row[kResidual];
    a.n.ro_s = row[kH];
    a.n.y_s = row[kY];
    a.n.cols = d->cols;
    a.n.eps = d->eps;
    a.post_weight = post_weight;
    a.gate = gate;
    a.g_s = row[kGate];
    a.gate_div = MafatDiv((uint32_t)per_gate);
    a.branch = d->branch_scale;
    a.keep = d->residual_scale;
    const cudaError_t e = mafat_launch_block_norm(a, d->dtype == MAFAT_BF16, lowest_bit(steps, 8),
                                                  !quant ? MAFAT_NORM_PLAIN : d->scale_group == 0 ? MAFAT_NORM_ROW : MAFAT_NORM_BLOCK,
                                                  (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(e, "norm launch");
    return MAFAT_OK;
}

mafat_status mafat_rotary_plan(const mafat_rotary_desc* d, mafat_rotary_t** out) {
    if (!d || !out) return fail(MAFAT_EINVAL, "null argument");
    *out = nullptr;
    if (d->struct_size != (int32_t)sizeof(mafat_rotary_desc)) return fail(MAFAT_EINVAL, "struct_size is not the descriptor's");
    if (d->dtype != MAFAT_BF16 && d->dtype != MAFAT_FP32) return fail(MAFAT_EINVAL, "dtype must be MAFAT_BF16 or MAFAT_FP32");
    if (d->head_dim < 1) return fail(MAFAT_EINVAL, "head_dim must be positive");
    if (d->head_dim > mafat_rotary_most_dim() || d->head_dim % 8 != 0)
        return fail(MAFAT_EUNSUPPORTED, "head_dim must be a multiple of 8 and at most %d", mafat_rotary_most_dim());
    const int32_t rot = d->rot_dim == 0 ? d->head_dim : d->rot_dim;
    if (rot < 2 || rot > d->head_dim || rot % 2 != 0) return fail(MAFAT_EINVAL, "rot_dim must be even, and at most head_dim");
    if (d->scaling < MAFAT_ROTARY_PLAIN || d->scaling > MAFAT_ROTARY_BLEND) return fail(MAFAT_EINVAL, "unknown scaling");
    const double base = d->base == 0. ? 10000. : d->base, factor = d->factor == 0. ? 1. : d->factor;
    const bool chosen = d->fast == 0. && d->slow == 0.;
    const double fast = chosen ? 32. : d->fast, slow = chosen ? 1. : d->slow;
    if (!(base > 1.) || !std::isfinite(base)) return fail(MAFAT_EINVAL, "base must be finite and above 1");
    if (!(factor >= 1.) || !std::isfinite(factor)) return fail(MAFAT_EINVAL, "factor must be finite and at least 1");
    if (d->scaling == MAFAT_ROTARY_PLAIN && factor != 1.) return fail(MAFAT_EINVAL, "a factor without a scaling");
    if (d->scaling == MAFAT_ROTARY_BASE && rot == 2) return fail(MAFAT_EINVAL, "a larger base scales no single pair");
    if (d->scaling == MAFAT_ROTARY_BLEND &&
        (!(d->first_positions > 0.) || !std::isfinite(d->first_positions) || !(slow > 0.) || !(fast > slow) || !std::isfinite(fast)))
        return fail(MAFAT_EINVAL, "first_positions must be positive, and slow between 0 and fast");
    if (!(d->magnitude >= 0.) || !std::isfinite(d->magnitude)) return fail(MAFAT_EINVAL, "magnitude must be positive, or 0 for the scaling's");
    if (d->frequencies) {
        if (d->scaling != MAFAT_ROTARY_PLAIN || d->base != 0.) return fail(MAFAT_EINVAL, "frequencies instead of a base and a scaling");
        for (int i = 0; i < rot / 2; ++i)
            if (!(std::fabs(d->frequencies[i]) <= 65536.)) return fail(MAFAT_EINVAL, "frequencies must be at most 65536 radians a position");
    }
    mafat_rotary_s* p = new (std::nothrow) mafat_rotary_s();
    uint64_t* turns = new (std::nothrow) uint64_t[rot / 2];
    if (p) p->frequencies = new (std::nothrow) double[rot / 2];
    mafat_status st = MAFAT_OK;
    cudaError_t e = cudaSuccess;
    if (!p || !turns || !p->frequencies) {
        st = fail(MAFAT_ENOMEM, "host allocation failed");
    } else {
        p->dry_run = d->dry_run != 0;
        p->interleaved = d->interleaved != 0;
        p->dtype = d->dtype;
        p->dim = d->head_dim;
        p->rot = rot;
        p->magnitude = d->magnitude > 0.                   ? d->magnitude
                       : d->scaling == MAFAT_ROTARY_BLEND ? 0.1 * std::log(factor) + 1.
                                                          : 1.;
        fill_frequencies(*d, rot, base, factor, fast, slow, p->frequencies);
        for (int i = 0; i < rot / 2; ++i) turns[i] = turn_of(p->frequencies[i]);
        if (!p->dry_run) {
            if ((e = cudaGetDevice(&p->device)) != cudaSuccess)
                st = cuda_fail(e, "cudaGetDevice");
            else if ((e = cudaMalloc(&p->turns, rot / 2 * sizeof(uint64_t))) != cudaSuccess)
                st = cuda_fail(e, "cudaMalloc");
            else if ((e = cudaMemcpy(p->turns, turns, rot / 2 * sizeof(uint64_t), cudaMemcpyHostToDevice)) != cudaSuccess)
                st = cuda_fail(e, "cudaMemcpy");
            else if ((e = transfers_done()) != cudaSuccess)
                st = cuda_fail(e, "cudaStreamSynchronize");
        }
    }
    delete[] turns;
    if (st != MAFAT_OK) {
        mafat_rotary_destroy(p);
        return st;
    }
    *out = p;
    mafat_internal_clear_error();
    return MAFAT_OK;
}

mafat_status mafat_rotary_run(const mafat_rotary_t* p, const mafat_rotary_call* c, const int32_t* positions,
                              const int32_t* places, const void* q, void* q_out, const void* k, void* k_out, const void* v,
                              void* v_out, void* stream) {
    if (!p || !c) return fail(MAFAT_EINVAL, "null argument");
    if (c->struct_size != (int32_t)sizeof(mafat_rotary_call)) return fail(MAFAT_EINVAL, "struct_size is not the call's");
    if (c->batch < 0 || c->n_q < 0) return fail(MAFAT_EINVAL, "batch and n_q must not be negative");
    if (c->heads_q < 0 || c->heads_kv < 0 || c->room < 0) return fail(MAFAT_EINVAL, "heads and room must not be negative");
    if (c->batch == 0 || c->n_q == 0) {
        mafat_internal_clear_error();
        return MAFAT_OK;
    }
    if (c->room == 0 && places) k = v = k_out = v_out = nullptr;  // no place: nothing of them is written
    if ((q != nullptr) != (q_out != nullptr) || (k != nullptr) != (k_out != nullptr) || (v != nullptr) != (v_out != nullptr))
        return fail(MAFAT_EINVAL, "a tensor and its output are given together");
    if (q && c->heads_q < 1) return fail(MAFAT_EINVAL, "heads_q must be positive");
    if ((k || v) && c->heads_kv < 1) return fail(MAFAT_EINVAL, "heads_kv must be positive");
    if ((k || v) && !places && c->room != c->n_q) return fail(MAFAT_EINVAL, "without places room is n_q");
    if (!q && !k && !v) {
        if (c->room > 0) return fail(MAFAT_EINVAL, "no tensor");
        mafat_internal_clear_error();
        return MAFAT_OK;
    }
    const int64_t tokens = (int64_t)c->batch * c->n_q;
    if (tokens > kMaxI32) return fail(MAFAT_EUNSUPPORTED, "too many tokens");
    if (c->heads_q > 32768 || c->heads_kv > 16384) return fail(MAFAT_EUNSUPPORTED, "too many heads");
    if (!positions) return fail(MAFAT_EINVAL, "null positions");
    if (!aligned(positions, 4) || !aligned(places, 4)) return fail(MAFAT_EINVAL, "positions and places must be 4-byte aligned");
    const int64_t esz = p->dtype == MAFAT_BF16 ? 2 : 4;
    const void* in[3] = {q, k, v};
    void* out[3] = {q_out, k_out, v_out};
    const int64_t* const given[3] = {c->q_strides, c->k_strides, c->v_strides};
    const int64_t* const given_out[3] = {c->q_out_strides, c->k_out_strides, c->v_out_strides};
    static const char* const names[3][2] = {{"q_strides", "q_out_strides"}, {"k_strides", "k_out_strides"}, {"v_strides", "v_out_strides"}};
    int64_t n[3][3], n_out[3][3], st[3][3], st_out[3][3];
    mafat_status s;
    for (int i = 0; i < 3; ++i) {
        if (!in[i]) continue;
        if (!aligned(in[i]) || !aligned(out[i])) return fail(MAFAT_EINVAL, "tensors must be 16-byte aligned");
        const int64_t heads = i == 0 ? c->heads_q : c->heads_kv;
        for (int j = 0; j < 3; ++j) n[i][j] = n_out[i][j] = j == 0 ? c->batch : j == 1 ? c->n_q : heads;
        if (i > 0) n_out[i][1] = c->room;
        if ((s = take_strides(names[i][0], given[i], n[i], p->dim, esz, st[i])) != MAFAT_OK ||
            (s = take_strides(names[i][1], given_out[i], n_out[i], p->dim, esz, st_out[i])) != MAFAT_OK)
            return s;
        if (!places_distinct(n_out[i], st_out[i], p->dim)) return fail(MAFAT_EINVAL, "%s: elements share a place", names[i][1]);
    }
    auto same = [&](int i) {  // the output is the tensor itself
        if (in[i] != out[i] || (i > 0 && places)) return false;
        for (int j = 0; j < 3; ++j)
            if (n[i][j] > 1 && st[i][j] != st_out[i][j]) return false;
        return true;
    };
    for (int o = 0; o < 3; ++o) {
        if (!out[o]) continue;
        const Placed to{out[o], n_out[o], st_out[o]};
        for (int i = 0; i < 3; ++i) {
            if (in[i] && !(i == o && same(o)) && !apart(to, Placed{in[i], n[i], st[i]}, p->dim, esz))
                return fail(MAFAT_EINVAL, "an output overlaps another tensor");
            if (i > o && out[i] && !apart(to, Placed{out[i], n_out[i], st_out[i]}, p->dim, esz))
                return fail(MAFAT_EINVAL, "an output overlaps another tensor");
        }
        const int64_t bytes = extent(n_out[o], st_out[o], p->dim, esz);
        if (overlap(out[o], bytes, positions, tokens * 4) || overlap(out[o], bytes, places, tokens * 4))
            return fail(MAFAT_EINVAL, "an output overlaps another tensor");
    }
    if (p->dry_run) return fail(MAFAT_EINVAL, "plan was created with dry_run");
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    if (dev != p->device) return fail(MAFAT_EINVAL, "the current device is not the plan's");
    MafatRotaryArgs a{};
    for (int i = 0; i < 3; ++i) {
        if (!in[i]) continue;
        MafatRotaryTensor& t = a.t[i];
        t.in = in[i];
        t.out = out[i];
        t.in_sb = st[i][0]; t.in_st = st[i][1]; t.in_sh = st[i][2];
        t.out_sb = st_out[i][0]; t.out_st = st_out[i][1]; t.out_sh = st_out[i][2];
        t.heads = (int32_t)n[i][2];
    }
    a.turns = p->turns;
    a.positions = positions;
    a.places = places;
    a.tokens = tokens;
    a.n_q = c->n_q;
    a.n_q_div = MafatDiv((uint32_t)c->n_q);
    a.room = c->room;
    a.dim = p->dim;
    a.rot = p->rot;
    a.magnitude = (float)p->magnitude;
    e = mafat_launch_rotary(a, p->dtype == MAFAT_BF16, p->interleaved, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(e, "rotary launch");
    return MAFAT_OK;
}

mafat_status mafat_rotary_frequencies(const mafat_rotary_t* p, double* frequencies, double* magnitude) {
    if (!p) return fail(MAFAT_EINVAL, "null plan");
    if (frequencies) std::copy(p->frequencies, p->frequencies + p->rot / 2, frequencies);
    if (magnitude) *magnitude = p->magnitude;
    return MAFAT_OK;
}

void mafat_rotary_destroy(mafat_rotary_t* p) {
    if (!p) return;
    if (p->turns) cudaFree(p->turns);
    delete[] p->frequencies;
    delete p;
}

mafat_status mafat_adjust_logits(const mafat_logits_desc* d, const void* logits, const int32_t* tokens, const int32_t* lengths,
                                 const int32_t* prompt_lengths, const float* repetition, const float* presence,
                                 const float* frequency, const int32_t* drafts, const uint32_t* tree, const int32_t* bias_ids,
                                 const float* bias, const uint32_t* masks, const int32_t* mask_rows, void* out, void* stream) {
    if (!d) return fail(MAFAT_EINVAL, "null argument");
    if (d->struct_size != (int32_t)sizeof(mafat_logits_desc)) return fail(MAFAT_EINVAL, "struct_size is not the descriptor's");
    if (d->dtype != MAFAT_BF16 && d->dtype != MAFAT_FP32) return fail(MAFAT_EINVAL, "dtype must be MAFAT_BF16 or MAFAT_FP32");
    if (d->out_dtype != d->dtype && d->out_dtype != MAFAT_FP32) return fail(MAFAT_EINVAL, "out_dtype must be dtype or MAFAT_FP32");
    if (d->batch < 0 || d->n_q < 0) return fail(MAFAT_EINVAL, "batch and n_q must not be negative");
    if (d->vocab < 1) return fail(MAFAT_EINVAL, "vocab must be positive");
    if (d->vocab > 1 << 30) return fail(MAFAT_EUNSUPPORTED, "too many tokens in the vocabulary");
    if (d->room < 0 || d->n_bias < 0 || d->n_masks < 0) return fail(MAFAT_EINVAL, "room, n_bias and n_masks must not be negative");
    if ((int64_t)d->room + d->n_q >= 1 << 18) return fail(MAFAT_EUNSUPPORTED, "at most 2^18 - 1 tokens of a request");
    if (d->n_bias > 4095) return fail(MAFAT_EUNSUPPORTED, "at most 4095 biases of a request");
    const int64_t rows = (int64_t)d->batch * d->n_q;
    if (rows == 0) {
        mafat_internal_clear_error();
        return MAFAT_OK;
    }
    const int64_t words = (d->n_q + 31) / 32, mask_words = (d->vocab + 31) / 32;
    if (rows > kMaxI32 || rows * (d->vocab / mafat_logits_run() + 2) > kMaxI32) return fail(MAFAT_EUNSUPPORTED, "too many rows");
    if (!logits || !out) return fail(MAFAT_EINVAL, "null logits or out");
    if ((bias_ids != nullptr) != (bias != nullptr)) return fail(MAFAT_EINVAL, "bias_ids and bias are given together");
    if (tree && !drafts) return fail(MAFAT_EINVAL, "a tree without drafts");
    // lists without an element may have no address
    if (mask_rows && !masks && d->n_masks > 0) return fail(MAFAT_EINVAL, "mask_rows without masks");
    if (masks && !mask_rows && d->n_masks != rows) return fail(MAFAT_EINVAL, "without mask_rows each row has its mask");
    if ((lengths || prompt_lengths) && !tokens && d->room > 0) return fail(MAFAT_EINVAL, "lengths without tokens");
    const int64_t esz = d->dtype == MAFAT_BF16 ? 2 : 4, osz = d->out_dtype == MAFAT_BF16 ? 2 : 4;
    const int64_t in_s = d->logits_stride == 0 ? d->vocab : d->logits_stride, out_s = d->out_stride == 0 ? d->vocab : d->out_stride;
    if (in_s < d->vocab || out_s < d->vocab) return fail(MAFAT_EINVAL, "a row stride is smaller than vocab");
    if (in_s > (int64_t)1 << 30 || out_s > (int64_t)1 << 30) return fail(MAFAT_EUNSUPPORTED, "a row stride is too large");
    if (!aligned(logits, esz) || !aligned(out, osz)) return fail(MAFAT_EINVAL, "logits and out must be aligned to their elements");
    const int64_t out_bytes = ((rows - 1) * out_s + d->vocab) * osz, requests = d->batch;
    const bool in_place = logits == out && osz == esz && in_s == out_s;
    if (!in_place && overlap(out, out_bytes, logits, ((rows - 1) * in_s + d->vocab) * esz))
        return fail(MAFAT_EINVAL, "an output overlaps another tensor");
    const int64_t biases = (d->bias_shared ? 1 : requests) * d->n_bias * 4;
    const struct {
        const void* p;
        int64_t bytes;
    } rest[] = {{tokens, requests * d->room * 4}, {lengths, requests * 4}, {prompt_lengths, requests * 4}, {repetition, requests * 4},
                {presence, requests * 4}, {frequency, requests * 4}, {drafts, rows * 4},
                {tree, (d->tree_shared ? 1 : requests) * d->n_q * words * 4}, {bias_ids, biases}, {bias, biases},
                {masks, d->n_masks * mask_words * 4}, {mask_rows, rows * 4}};
    for (const auto& t : rest) {
        if (!aligned(t.p, 4)) return fail(MAFAT_EINVAL, "tensors must be 4-byte aligned");
        if (overlap(out, out_bytes, t.p, t.bytes)) return fail(MAFAT_EINVAL, "an output overlaps another tensor");
    }
    MafatLogitsArgs a{};
    a.logits = logits;
    a.out = out;
    a.in_s = in_s;
    a.out_s = out_s;
    a.tokens = d->room > 0 ? tokens : nullptr;
    a.lengths = lengths;
    a.prompt = prompt_lengths;
    a.repetition = repetition;
    a.presence = presence;
    a.frequency = frequency;
    a.drafts = drafts;
    a.tree = tree;
    a.tree_s = d->tree_shared ? 0 : d->n_q * words;
    a.bias_ids = d->n_bias > 0 ? bias_ids : nullptr;
    a.bias = bias;
    a.bias_s = d->bias_shared ? 0 : d->n_bias;
    a.masks = masks;
    a.mask_rows = mask_rows;
    a.n_q = d->n_q;
    a.pass = !in_place || masks != nullptr;
    a.vocab = d->vocab;
    a.room = d->room;
    a.n_bias = d->n_bias;
    a.n_masks = d->n_masks;
    a.tree_words = (int32_t)words;
    a.mask_words = (int32_t)mask_words;
    const cudaError_t e = mafat_launch_logits(a, d->dtype == MAFAT_BF16, d->out_dtype == MAFAT_BF16, d->batch, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(e, "logits launch");
    return MAFAT_OK;
}

}  // extern "C"
