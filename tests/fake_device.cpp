// A CUDA runtime and kernels that only note what they are asked for, in order, so that the library's host side can be run and
// looked at without a GPU.  fake_fail: the named call fails once; fake_next_out: what the next copy to the host starts with.
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>

#include "attention.h"
#include "decode.h"
#include "kernels.h"

namespace {

std::string notes, failing;
uint32_t next_out;

cudaError_t note(const char* name, const char* format = "", ...) {
    char more[128];
    va_list args;
    va_start(args, format);
    vsnprintf(more, sizeof(more), format, args);
    va_end(args);
    notes += std::string(name) + more + "\n";
    if (failing != name) return cudaSuccess;
    failing.clear();
    return cudaErrorUnknown;
}

CUresult encode(...) { return CUDA_SUCCESS; }

}  // namespace

extern "C" {

const char* fake_notes() { return notes.c_str(); }
void fake_reset() { notes.clear(), failing.clear(); }
void fake_fail(const char* name) { failing = name; }
void fake_next_out(uint32_t word) { next_out = word; }

cudaError_t cudaDeviceGetAttribute(int* value, cudaDeviceAttr, int) { return *value = 152, cudaSuccess; }
cudaError_t cudaGetDevice(int* device) { return *device = 0, cudaSuccess; }
const char* cudaGetErrorString(cudaError_t) { return "made to fail"; }
cudaError_t cudaGetDriverEntryPointByVersion(const char*, void** fn, unsigned, unsigned long long, cudaDriverEntryPointQueryResult* found) {
    *fn = (void*)encode;
    if (found) *found = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
cudaError_t cudaMalloc(void** p, size_t n) { return *p = malloc(n < 4096 ? 4096 : n), note("malloc"); }
cudaError_t cudaFree(void* p) { return free(p), note("free"); }
cudaError_t cudaMemcpy(void* to, const void* from, size_t n, cudaMemcpyKind kind) {
    memcpy(to, from, n);
    if (kind == cudaMemcpyDeviceToHost && next_out) memcpy(to, &next_out, 4), next_out = 0u;
    return note(kind == cudaMemcpyHostToDevice ? "copy in" : "copy out");
}
cudaError_t cudaMemset(void* p, int v, size_t n) { return memset(p, v, n), note("set"); }
cudaError_t cudaMemcpyAsync(void*, const void*, size_t, cudaMemcpyKind, cudaStream_t) { return note("copy async"); }
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return note("set async"); }
cudaError_t cudaGetSymbolAddress(void** p, const void* symbol) { return *p = const_cast<void*>(symbol), cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t s) { return note("sync", " %llu", (unsigned long long)(uintptr_t)s); }
cudaError_t cudaStreamCreateWithFlags(cudaStream_t* s, unsigned) { return *s = nullptr, cudaSuccess; }
cudaError_t cudaStreamDestroy(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamWaitEvent(cudaStream_t, cudaEvent_t, unsigned) { return cudaSuccess; }
cudaError_t cudaEventCreateWithFlags(cudaEvent_t* e, unsigned) { return *e = nullptr, cudaSuccess; }
cudaError_t cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaEventSynchronize(cudaEvent_t) { return cudaSuccess; }

}  // extern "C"

int mafat_attn_rows_join() { return 32; }
int mafat_attn_rows_keys() { return 64; }
int mafat_attn_simt_keys() { return 64; }
int mafat_fp32_ctas_per_sm() { return 1; }
size_t mafat_fp32_smem_bytes() { return 1 << 17; }
size_t mafat_tc_smem_bytes() { return 1 << 17; }
int mafat_logits_run() { return 2048; }
int mafat_norm_max_cols() { return 16384; }
int mafat_rotary_most_dim() { return 256; }

cudaError_t mafat_prepare_attn_rows(bool tree, int dim) { return note("prepare rows", " %d %d", tree, dim); }
cudaError_t mafat_prepare_attn_simt(bool tree, int dim) { return note("prepare simt", " %d %d", tree, dim); }
cudaError_t mafat_prepare_attn_tc(bool tree, int dim) { return note("prepare tc", " %d %d", tree, dim); }
cudaError_t mafat_prepare_fp32() { return note("prepare fp32"); }
cudaError_t mafat_prepare_tc(bool, bool) { return note("prepare tc plan"); }

cudaError_t mafat_launch_attn_join(const MafatAttnArgs&, bool, cudaStream_t) { return note("launch join"); }
cudaError_t mafat_launch_attn_rows(const MafatAttnArgs&, int, const MafatRowsPrefix*, cudaStream_t) { return note("launch rows"); }
cudaError_t mafat_launch_attn_simt(const MafatAttnArgs& a, int rows, cudaStream_t) {
    return note("launch simt", " %d, CTAs %d, alone %d", rows, a.seg.items, a.alone);
}
cudaError_t mafat_launch_attn_tc(const MafatAttnArgs&, const CUtensorMap&, const CUtensorMap&, int, const MafatAttnPrefix*, cudaStream_t) {
    return note("launch tc");
}
cudaError_t mafat_launch_norm(const MafatNormArgs&, bool, int, MafatNormQuant, cudaStream_t) { return note("launch norm"); }
cudaError_t mafat_launch_block_norm(const MafatBlockNormArgs&, bool, int, MafatNormQuant, cudaStream_t) { return note("launch block norm"); }
cudaError_t mafat_launch_rotary(MafatRotaryArgs&, bool, bool, cudaStream_t) { return note("launch rotary"); }
cudaError_t mafat_launch_logits(MafatLogitsArgs&, bool, bool, int64_t, cudaStream_t) { return note("launch logits"); }
cudaError_t mafat_launch_fp32(const MafatKParams&, int, cudaStream_t) { return note("launch fp32"); }
cudaError_t mafat_launch_tc(const MafatKParams&, const CUtensorMap&, int, bool, cudaStream_t) { return note("launch tc plan"); }
cudaError_t mafat_launch_to_planar(const void*, void*, int, int, int, int, int, int, cudaStream_t) { return note("launch planar"); }
cudaError_t mafat_launch_diag_umma(const void*, const void*, float*, int, int, cudaStream_t) { return note("launch umma"); }
