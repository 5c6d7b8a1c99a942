// The context behind the C ABI and what its entry points share: error text, the caller's device, allocations.
#pragma once

#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <string>
#include <vector>

#include <nvtx3/nvToolsExt.h>

#include "kvdro.h"
#include "kv.cuh"
#include "kvdro_internal.cuh"

namespace kvdro {

struct Buf {
    void* p = nullptr;
    size_t bytes = 0;
};

}  // namespace kvdro

struct kvdro_ctx {
    int device = 0;
    int sms = 0;  // of the device
    std::string err;
    int fail_after = -1;  // test hook: the fail_after-th allocation of this context fails
    int skip_chunk = -1;  // test hook: grid kernels never copy this chunk, so their waits run out
    int allocs = 0;
    cudaStream_t last_stream = nullptr;  // of the last call that is not one of the page cache's

    bool loaded = false;
    bool quads = false;  // the staged form of the loaded samples
    int32_t K = 0;
    int64_t total = 0, pair_total = 0, hist_total = 0;
    std::vector<int64_t> off, pair_off, hist_off, N;
    std::vector<int32_t> L, Lin, hist_blocks, exp_blocks;
    std::vector<double> inv_n;

    kvdro::Buf sorted, pairs, hist, cum, csum, sumx, meta, errs, in_stage, grid_in, keys, cost64, out_stage, ranks, scan_tot,
        tile_lo;
    void* pin = nullptr;  // pinned host staging
    size_t pin_bytes = 0;
    void* land = nullptr;  // pinned: small results and the status words land here on their way to the caller
    cudaEvent_t pin_free = nullptr;  // completes when the last copy out of `pin` is done
    cudaEvent_t grid_t0 = nullptr, grid_t1 = nullptr;  // around the last grid-kernel launches
    // Copies of host outputs back to the caller, overlapped with later grid launches
    cudaStream_t copy_stream = nullptr;
    cudaEvent_t copy_ready = nullptr, copy_done = nullptr;
    bool grid_timed = false;

    // device views into `meta`
    int64_t *d_off = nullptr, *d_pair_off = nullptr, *d_hist_off = nullptr, *d_N = nullptr;
    double* d_inv_n = nullptr;
    int32_t* d_cum = nullptr;  // cumulative counts
    int32_t *d_L = nullptr, *d_Lin = nullptr, *d_hist_blocks = nullptr, *d_exp_blocks = nullptr;

    // The page cache
    kvdro_kv* caches = nullptr;  // open handles
    kvdro::Buf kv_err;           // the word in which its kernels report what they met, and the one it is taken to
    kvdro::Buf kv_pieces, kv_tickets, kv_joins;  // scratch of the attention kernels
    cudaStream_t kv_side = nullptr;    // clears scratch and the status word; ordered with no caller's stream
    cudaEvent_t kv_done = nullptr;     // completes when the last attention call outside captures is done with it
    unsigned long long kv_stream = 0;  // that call's stream, by its number
    bool kv_used = false;
    cudaStream_t kv_last = nullptr;    // of the last page cache call
    bool kv_err_ready = false, kv_plan_ready = false, kv_ready = false;
};

// A page cache that the caller owns.
struct kvdro_kv {
    kvdro_ctx* ctx = nullptr;
    kvdro_kv *next = nullptr, *prev = nullptr;
    bool half = false;  // FP16, else BF16
    int32_t n_pages = 0, page_size = 0, page_shift = 0, heads = 0, head_dim = 0;
    void *k = nullptr, *v = nullptr;
    int64_t k_stride[3] = {}, v_stride[3] = {};  // page, slot, head; in elements
    kvdro::KvMaps maps;
};

namespace kvdro {

inline int fail(kvdro_ctx* c, int code, const char* fmt, ...) {
    if (c) {
        char buf[512];
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(buf, sizeof(buf), fmt, ap);
        va_end(ap);
        c->err = buf;
    }
    return code;
}

inline int cuda_fail(kvdro_ctx* c, cudaError_t e, const char* what) {
    return fail(c, KVDRO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

#define KV_CUDA(call, what)                            \
    do {                                               \
        cudaError_t e_ = (call);                       \
        if (e_ != cudaSuccess) return cuda_fail(ctx, e_, what); \
    } while (0)

// An NVTX range around one entry point (visible in Nsight timelines; a no-op without a tool).
struct NvtxRange {
    explicit NvtxRange(const char* name) { nvtxRangePushA(name); }
    ~NvtxRange() { nvtxRangePop(); }
};

// Keeps the caller's current device and restores it on exit.
struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        ok = cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard() {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

inline int ensure(kvdro_ctx* ctx, Buf& b, size_t bytes) {
    if (bytes == 0) bytes = 16;
    if (b.bytes >= bytes) return KVDRO_OK;
    if (b.p) {
        cudaFree(b.p);
        b.p = nullptr;
        b.bytes = 0;
    }
    ctx->allocs++;
    if (ctx->fail_after > 0 && ctx->allocs == ctx->fail_after)
        return fail(ctx, KVDRO_ENOMEM, "device allocation of %zu bytes failed (injected by KVDRO_TEST_FAIL_ALLOC)", bytes);
    cudaError_t e = cudaMalloc(&b.p, bytes);
    if (e != cudaSuccess) {
        cudaGetLastError();
        b.p = nullptr;
        return fail(ctx, KVDRO_ENOMEM, "cudaMalloc(%zu): %s", bytes, cudaGetErrorString(e));
    }
    b.bytes = bytes;
    return KVDRO_OK;
}

inline void release(Buf& b) {
    if (b.p) cudaFree(b.p);
    b.p = nullptr;
    b.bytes = 0;
}

// Device-accessible (device or managed memory) versus host memory (pinned or pageable).
inline bool is_device_ptr(const void* p) {
    cudaPointerAttributes at;
    cudaError_t e = cudaPointerGetAttributes(&at, p);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    return at.type == cudaMemoryTypeDevice || at.type == cudaMemoryTypeManaged;
}

int wait_kv(kvdro_ctx* ctx);  // kv_api.cu
int check_kv_errors(kvdro_ctx* ctx);

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace kvdro
