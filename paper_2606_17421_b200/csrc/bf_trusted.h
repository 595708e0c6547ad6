// Host-side state of the trusted half (plaintext operators) and what its translation units share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstdio>

#include "../../include/bifrost.h"

struct bf_trusted {
    int device = 0, n_sm = 0;
    cudaStream_t stream = nullptr;
    unsigned char* base = nullptr;       // one allocation: status word, arrival counters, workspace
    int* status = nullptr;
    unsigned* arrivals = nullptr;        // ARRIVALS counters, zero between calls
    unsigned char* ws = nullptr;
    size_t ws_bytes = 0;
    char cuda_msg[256] = "";
};

namespace bft {

constexpr int ST_RANGE = 1, ST_OOM = 2, ST_TIMEOUT = 4;         // bits of the status word
constexpr unsigned ARRIVALS = 4096;

// The context's device current for the length of a call.
struct OnDevice {
    int before = -1;
    bool ok = true;
    explicit OnDevice(int device) {
        ok = cudaGetDevice(&before) == cudaSuccess && (before == device || cudaSetDevice(device) == cudaSuccess);
        if (before == device) before = -1;
    }
    ~OnDevice() {
        if (before >= 0) cudaSetDevice(before);
    }
};

inline int cuda_failed(bf_trusted* t, const char* what, cudaError_t e) {
    cudaGetLastError();
    snprintf(t->cuda_msg, sizeof(t->cuda_msg), "%s: %s", what, cudaGetErrorString(e));
    return BF_ERR_CUDA;
}
inline int launched(bf_trusted* t, const char* what) {
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? BF_OK : cuda_failed(t, what, e);
}

// Dynamic shared memory that a kernel may ask for: set once a device, since the call costs as much as a third of a launch.
template <auto KERNEL> cudaError_t room_for(const bf_trusted* t, size_t bytes) {
    static std::atomic<unsigned long long> done{0};
    const unsigned long long bit = t->device >= 0 && t->device < 64 ? 1ull << t->device : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

inline bool type_ok(int32_t type) { return type == BF_F32 || type == BF_F16 || type == BF_BF16; }
inline unsigned type_bytes(int32_t type) { return type == BF_F32 ? 4 : 2; }
inline bool rows_ok(const bf_rows* r) { return r && r->data && type_ok(r->type) && (uintptr_t)r->data % type_bytes(r->type) == 0; }
// every access of 16 bytes that starts at a multiple of 16 bytes within a (row, head) is aligned
inline bool rows_wide(const bf_rows* r, bool heads) {
    const int64_t per = 16 / type_bytes(r->type);
    return (uintptr_t)r->data % 16 == 0 && r->row_stride % per == 0 && (!heads || r->head_stride % per == 0);
}

// ---- q4.cu
int q4_check(const bf_q4_matrix* W);
cudaError_t launch_q4_expand(const bf_q4_matrix& W, float* out, cudaStream_t stream);      // out: [d_out][d_in]

// The cache as kernels take it.
struct Cache {
    unsigned char* pool;
    int* tables;
    int* lengths;
    int* refs;
    unsigned n_layers, n_pages, heads, page_tokens, n_seqs, max_pages;
    unsigned sub_bytes, block_bytes;             // bytes of 16 tokens, of a page of one head
    size_t layer_bytes;
};
int cache_check(const bf_kv4_cache* c, Cache* out);

__device__ __forceinline__ float load_as_float(const void* p, int type, int64_t i) {
    if (type == BF_F32) return static_cast<const float*>(p)[i];
    if (type == BF_F16) return __half2float(static_cast<const __half*>(p)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
__device__ __forceinline__ void store_from_float(void* p, int type, int64_t i, float v) {
    if (type == BF_F32) static_cast<float*>(p)[i] = v;
    else if (type == BF_F16) static_cast<__half*>(p)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

}  // namespace bft
