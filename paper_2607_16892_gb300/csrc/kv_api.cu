// C ABI of the page cache (declared in include/kvdro.h): argument validation and launches.
#include <cuda_runtime.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <iterator>
#include <new>

#include "context.cuh"

using kvdro::cuda_fail;
using kvdro::DeviceGuard;
using kvdro::ensure;
using kvdro::fail;
using kvdro::NvtxRange;

namespace {

constexpr int64_t kMaxStride = (int64_t)1 << 39;  // elements: what a tensor map's 40 bits of bytes hold
constexpr int32_t kMaxTokens = 1 << 30, kMaxPositions = 1 << 30, kMaxRows = 1 << 30;  // with room for a tile in 32 bits
constexpr int32_t kMaxHeads = 4096, kMaxKvHeads = 1024;
constexpr unsigned long long kWaitNs = 2000000000, kTestWaitNs = 1000000;
// Rows that share a key head, up to which the kernel for single tokens runs.  32 requests of 3000 positions, 8 key heads of 128:
// 12 rows 77 us there; 20 to 32 rows 140 us there, 85 on the kernel for chunks; 64 rows 249 and 85.
constexpr int64_t kFewRows = 16;

int log2_of(int32_t v) {
    int s = 0;
    while ((1 << s) < v) s++;
    return s;
}

int check_pages(kvdro_ctx* ctx, int32_t page_size, int32_t n_pages) {
    if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128)
        return fail(ctx, KVDRO_EINVAL, "page_size = %d is not 16, 32, 64 or 128", page_size);
    if (n_pages < 1 || (int64_t)n_pages * page_size > 0x7fffffffLL)
        return fail(ctx, KVDRO_EINVAL, "n_pages = %d: n_pages * page_size outside [page_size, 2^31)", n_pages);
    return KVDRO_OK;
}

int check_requests(kvdro_ctx* ctx, int32_t B, int32_t T, int32_t max_pages, int32_t page_size) {
    if (B < 1 || B > kvdro::kKvMaxRequests) return fail(ctx, KVDRO_EINVAL, "B = %d outside [1, %d]", B, kvdro::kKvMaxRequests);
    if (T < 0 || T > kMaxTokens) return fail(ctx, KVDRO_EINVAL, "T = %d outside [0, 2^30]", T);
    if (max_pages < 1 || (int64_t)max_pages * page_size > kMaxPositions)
        return fail(ctx, KVDRO_EINVAL, "max_pages = %d: max_pages * page_size outside [page_size, 2^30]", max_pages);
    return KVDRO_OK;
}

struct Arg {
    const char* name;
    const void* p;
};

int check_device(kvdro_ctx* ctx, std::initializer_list<Arg> args) {
    for (const Arg& x : args) {
        if (!x.p) return fail(ctx, KVDRO_EINVAL, "%s is required", x.name);
        cudaPointerAttributes at;
        if (cudaPointerGetAttributes(&at, x.p) != cudaSuccess) {
            cudaGetLastError();
            at = {};
        }
        if (const char* what = kvdro::kv_not_usable(at, ctx->device)) return fail(ctx, KVDRO_EINVAL, "%s must be %s", x.name, what);
    }
    return KVDRO_OK;
}

struct Extent {
    const char* name;
    const int32_t* p;
    int64_t n;
};

bool overlap(const Extent& x, const Extent& y) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
    return a < b + 4 * (uintptr_t)y.n && b < a + 4 * (uintptr_t)x.n && x.n > 0 && y.n > 0;
}

// Strides of rows of 16-byte vectors: `n` of them into `out`, from the caller's or the contiguous ones.
int rows(kvdro_ctx* ctx, const char* name, const void* p, const int64_t* stride, int n, const int64_t* dense, int64_t* out) {
    if (reinterpret_cast<uintptr_t>(p) % 16) return fail(ctx, KVDRO_EINVAL, "%s is not 16-byte aligned", name);
    for (int i = 0; i < n; i++) {
        out[i] = stride ? stride[i] : dense[i];
        if (out[i] < 1 || out[i] >= kMaxStride || out[i] % 8)
            return fail(ctx, KVDRO_EINVAL, "%s: stride %lld is not a positive multiple of 8 elements below 2^39", name,
                        (long long)out[i]);
    }
    return KVDRO_OK;
}

// A tensor map of k or v for boxes of 64 elements by `slots` slots of one head and page, rows of 128 bytes permuted
// (128-byte swizzle) so that matrix loads meet no bank conflict.
int encode(kvdro_ctx* ctx, CUtensorMap* map, const kvdro_kv& c, void* p, const int64_t* stride, int slots) {
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
    }();
    if (!fn) return fail(ctx, KVDRO_ECUDA, "the driver has no cuTensorMapEncodeTiled");
    const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.heads, (cuuint64_t)c.n_pages};
    const cuuint64_t bytes[3] = {(cuuint64_t)stride[1] * 2, (cuuint64_t)stride[2] * 2, (cuuint64_t)stride[0] * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)slots, 1, 1}, one[4] = {1, 1, 1, 1};
    const CUresult r = fn(map, c.half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, p, dims, bytes, box, one,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(ctx, KVDRO_EINVAL, "these sizes and strides make no tensor map (driver error %d)", (int)r);
    return KVDRO_OK;
}

// Zeros, there when the call returns, whatever stream uses them next.  (A memset on the default stream is neither waited for
// by the host nor ordered with non-blocking streams, and would wait for the caller's work on that stream.)
int clear(kvdro_ctx* ctx, void* p, size_t bytes) {
    if (!ctx->kv_side) KV_CUDA(cudaStreamCreateWithFlags(&ctx->kv_side, cudaStreamNonBlocking), "creating a stream");
    KV_CUDA(cudaMemsetAsync(p, 0, bytes, ctx->kv_side), "clearing scratch");
    KV_CUDA(cudaStreamSynchronize(ctx->kv_side), "clearing scratch");
    return KVDRO_OK;
}

// What the attention kernels need once per context: attributes, scratch.
int prepare_attend(kvdro_ctx* ctx) {
    if (ctx->kv_ready) return KVDRO_OK;
    KV_CUDA(kvdro::kv_decode_prepare(), "preparing the attention kernels");
    KV_CUDA(kvdro::kv_chunk_prepare(), "preparing the attention kernels");
    if (!ctx->kv_done) KV_CUDA(cudaEventCreateWithFlags(&ctx->kv_done, cudaEventDisableTiming), "creating an event");
    const size_t pieces = kvdro::kv_decode_piece_bytes(ctx->sms) + kvdro::kv_chunk_piece_bytes(ctx->sms);
    if (int rc = ensure(ctx, ctx->kv_pieces, pieces)) return rc;
    if (int rc = ensure(ctx, ctx->kv_joins, sizeof(kvdro::Join) * (size_t)ctx->sms)) return rc;
    const size_t tickets = 4 * (size_t)kvdro::kv_decode_ctas(ctx->sms);
    if (int rc = ensure(ctx, ctx->kv_tickets, tickets)) return rc;
    if (int rc = clear(ctx, ctx->kv_tickets.p, tickets)) return rc;
    ctx->kv_ready = true;
    return KVDRO_OK;
}

// The word in which page cache kernels report what they met.
int error_word(kvdro_ctx* ctx) {
    if (ctx->kv_err_ready) return KVDRO_OK;
    if (int rc = ensure(ctx, ctx->kv_err, 16)) return rc;
    if (int rc = clear(ctx, ctx->kv_err.p, 16)) return rc;
    ctx->kv_err_ready = true;
    return KVDRO_OK;
}

}  // namespace

extern "C" {

int kvdro_kv_open(kvdro_ctx* ctx, kvdro_kv** out, int dtype, int32_t n_pages, int32_t page_size, int32_t n_kv_heads,
                  int32_t head_dim, void* k, const int64_t* k_stride, void* v, const int64_t* v_stride) {
    NvtxRange nvtx_("kvdro_kv_open");
    if (out) *out = nullptr;
    if (!ctx) return KVDRO_EINVAL;
    ctx->err.clear();
    if (!out) return fail(ctx, KVDRO_EINVAL, "out is required");
    if (dtype != KVDRO_BF16 && dtype != KVDRO_FP16) return fail(ctx, KVDRO_EINVAL, "dtype must be KVDRO_BF16 or KVDRO_FP16");
    if (int rc = check_pages(ctx, page_size, n_pages)) return rc;
    if (n_kv_heads < 1 || n_kv_heads > kMaxKvHeads)
        return fail(ctx, KVDRO_EINVAL, "n_kv_heads = %d outside [1, %d]", n_kv_heads, kMaxKvHeads);
    if (head_dim != 64 && head_dim != 128) return fail(ctx, KVDRO_EINVAL, "head_dim = %d is not 64 or 128", head_dim);
    DeviceGuard g(ctx->device);
    if (!g.ok) return fail(ctx, KVDRO_ECUDA, "cannot select device %d", ctx->device);
    if (int rc = check_device(ctx, {{"k", k}, {"v", v}})) return rc;
    const int64_t row = (int64_t)n_kv_heads * head_dim, dense[3] = {page_size * row, row, head_dim};
    kvdro_kv c;
    if (int rc = rows(ctx, "k", k, k_stride, 3, dense, c.k_stride)) return rc;
    if (int rc = rows(ctx, "v", v, v_stride, 3, dense, c.v_stride)) return rc;
    if (int rc = error_word(ctx)) return rc;
    if (int rc = prepare_attend(ctx)) return rc;
    c.ctx = ctx;
    c.half = dtype == KVDRO_FP16;
    c.n_pages = n_pages;
    c.page_size = page_size;
    c.page_shift = log2_of(page_size);
    c.heads = n_kv_heads;
    c.head_dim = head_dim;
    c.k = k;
    c.v = v;
    if (int rc = encode(ctx, &c.maps.k_slice, c, k, c.k_stride, std::min(page_size, 32))) return rc;
    if (int rc = encode(ctx, &c.maps.v_slice, c, v, c.v_stride, std::min(page_size, 32))) return rc;
    if (int rc = encode(ctx, &c.maps.k, c, k, c.k_stride, page_size)) return rc;
    if (int rc = encode(ctx, &c.maps.v, c, v, c.v_stride, page_size)) return rc;
    kvdro_kv* kv = new (std::nothrow) kvdro_kv(c);
    if (!kv) return fail(ctx, KVDRO_ENOMEM, "no memory for the handle");
    kv->next = ctx->caches;
    if (kv->next) kv->next->prev = kv;
    ctx->caches = kv;
    *out = kv;
    return KVDRO_OK;
}

int kvdro_kv_close(kvdro_kv* kv) {
    if (!kv) return KVDRO_OK;
    if (kv->prev) kv->prev->next = kv->next;
    else kv->ctx->caches = kv->next;
    if (kv->next) kv->next->prev = kv->prev;
    delete kv;
    return KVDRO_OK;
}

int kvdro_kv_plan(kvdro_ctx* ctx, int32_t page_size, int32_t n_pages, int32_t B, int32_t max_pages, int32_t T,
                  const int32_t* cached, const int32_t* new_len, const int32_t* reserve, const int32_t* held,
                  int32_t* table, int32_t* ring, const int32_t* pool, int32_t* held_out, int32_t* pool_out,
                  int32_t* q_off, int32_t* kv_len, int32_t* slot, int32_t* pos, void* stream) {
    NvtxRange nvtx_("kvdro_kv_plan");
    if (!ctx) return KVDRO_EINVAL;
    ctx->err.clear();
    if (int rc = check_pages(ctx, page_size, n_pages)) return rc;
    if (int rc = check_requests(ctx, B, T, max_pages, page_size)) return rc;
    DeviceGuard g(ctx->device);
    if (!g.ok) return fail(ctx, KVDRO_ECUDA, "cannot select device %d", ctx->device);
    if (int rc = check_device(ctx, {{"cached", cached}, {"new_len", new_len}, {"held", held}, {"table", table}, {"ring", ring},
                                    {"pool", pool}, {"held_out", held_out}, {"pool_out", pool_out}, {"q_off", q_off},
                                    {"kv_len", kv_len}}))
        return rc;
    if (reserve)
        if (int rc = check_device(ctx, {{"reserve", reserve}})) return rc;
    if (T > 0)
        if (int rc = check_device(ctx, {{"slot", slot}})) return rc;
    if (T > 0 && pos)
        if (int rc = check_device(ctx, {{"pos", pos}})) return rc;
    // CTAs read lengths again after others have written results, in no order.
    const Extent written[] = {{"held_out", held_out, B}, {"pool_out", pool_out, 2}, {"q_off", q_off, B + 1}, {"kv_len", kv_len, B},
                              {"slot", slot, T}, {"pos", pos, pos ? T : 0}, {"table", table, (int64_t)B * max_pages}, {"ring", ring, n_pages}};
    const Extent read[] = {{"held", held, B}, {"pool", pool, 2}, {"cached", cached, B}, {"new_len", new_len, B}, {"reserve", reserve, reserve ? B : 0}};
    for (const Extent* w = std::begin(written); w != std::end(written); w++) {
        for (const Extent& r : read)
            if (overlap(*w, r)) return fail(ctx, KVDRO_EINVAL, "%s overlaps %s", w->name, r.name);
        for (const Extent* o = std::begin(written); o != w; o++)
            if (overlap(*w, *o)) return fail(ctx, KVDRO_EINVAL, "%s overlaps %s", w->name, o->name);
    }
    if (!ctx->kv_plan_ready) {
        KV_CUDA(kvdro::kv_plan_prepare(), "preparing the plan kernel");
        ctx->kv_plan_ready = true;
    }
    if (int rc = error_word(ctx)) return rc;
    kvdro::PlanArgs a{log2_of(page_size), n_pages, B, max_pages, T, cached, new_len, reserve, held, pool, table, ring, held_out,
                      pool_out, q_off, kv_len, slot, pos, static_cast<int32_t*>(ctx->kv_err.p)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    ctx->kv_last = s;
    KV_CUDA(kvdro::launch_kv_plan(a, ctx->sms, s), "plan kernel");
    return KVDRO_OK;
}

int kvdro_kv_append(kvdro_kv* kv, int32_t T, const void* k, const int64_t* k_stride, const void* v,
                    const int64_t* v_stride, const int32_t* slot, void* stream) {
    NvtxRange nvtx_("kvdro_kv_append");
    if (!kv) return KVDRO_EINVAL;
    kvdro_ctx* ctx = kv->ctx;
    ctx->err.clear();
    if (T < 0 || T > kMaxTokens) return fail(ctx, KVDRO_EINVAL, "T = %d outside [0, 2^30]", T);
    if (T == 0) return KVDRO_OK;
    DeviceGuard g(ctx->device);
    if (!g.ok) return fail(ctx, KVDRO_ECUDA, "cannot select device %d", ctx->device);
    if (int rc = check_device(ctx, {{"k", k}, {"v", v}, {"slot", slot}})) return rc;
    const int64_t dense[2] = {(int64_t)kv->heads * kv->head_dim, kv->head_dim};
    int64_t ks[2] = {}, vs[2] = {};
    if (int rc = rows(ctx, "k", k, k_stride, 2, dense, ks)) return rc;
    if (int rc = rows(ctx, "v", v, v_stride, 2, dense, vs)) return rc;
    kvdro::AppendArgs a;
    a.k = static_cast<const uint4*>(k);
    a.v = static_cast<const uint4*>(v);
    a.kc = static_cast<uint4*>(kv->k);
    a.vc = static_cast<uint4*>(kv->v);
    a.k_tok = ks[0] / 8;
    a.k_head = ks[1] / 8;
    a.v_tok = vs[0] / 8;
    a.v_head = vs[1] / 8;
    a.kc_page = kv->k_stride[0] / 8;
    a.kc_slot = kv->k_stride[1] / 8;
    a.kc_head = kv->k_stride[2] / 8;
    a.vc_page = kv->v_stride[0] / 8;
    a.vc_slot = kv->v_stride[1] / 8;
    a.vc_head = kv->v_stride[2] / 8;
    a.slot = slot;
    a.T = T;
    a.n_slots = kv->n_pages << kv->page_shift;
    a.page_shift = kv->page_shift;
    a.heads = kv->heads;
    a.vec_shift = log2_of(kv->head_dim / 8);
    a.err = static_cast<int32_t*>(ctx->kv_err.p);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    ctx->kv_last = s;
    KV_CUDA(kvdro::launch_kv_append(a, s), "append kernel");
    return KVDRO_OK;
}

int kvdro_kv_attend(kvdro_kv* kv, int32_t B, int32_t T, int32_t n_heads, int32_t max_q, const void* q,
                    const int64_t* q_stride, const int32_t* q_off, const int32_t* kv_len, const int32_t* table,
                    int32_t max_pages, double scale, int causal, int32_t window, double softcap, void* out,
                    const int64_t* out_stride, float* lse, void* stream) {
    NvtxRange nvtx_("kvdro_kv_attend");
    if (!kv) return KVDRO_EINVAL;
    kvdro_ctx* ctx = kv->ctx;
    ctx->err.clear();
    if (int rc = check_requests(ctx, B, T, max_pages, kv->page_size)) return rc;
    if (n_heads < 1 || n_heads > kMaxHeads || n_heads % kv->heads)
        return fail(ctx, KVDRO_EINVAL, "n_heads = %d is not a multiple of n_kv_heads = %d up to %d", n_heads, kv->heads, kMaxHeads);
    if (max_q < 0) return fail(ctx, KVDRO_EINVAL, "max_q = %d is negative", max_q);
    if (!std::isfinite((float)scale)) return fail(ctx, KVDRO_EINVAL, "scale = %g is not finite", scale);
    if (!(softcap == 0.0 || (softcap >= 0x1p-20 && softcap <= 1000.0)))
        return fail(ctx, KVDRO_EINVAL, "softcap = %g is neither 0 nor in [2^-20, 1000]", softcap);
    if (causal != 0 && causal != 1) return fail(ctx, KVDRO_EINVAL, "causal must be 0 or 1");
    if (window < 0 || (window > 0 && !causal)) return fail(ctx, KVDRO_EINVAL, "window = %d: not negative, and with causal only", window);
    if (T == 0) return KVDRO_OK;
    if ((int64_t)T * n_heads > kMaxRows) return fail(ctx, KVDRO_EINVAL, "T * n_heads = %lld passes 2^30", (long long)T * n_heads);
    DeviceGuard g(ctx->device);
    if (!g.ok) return fail(ctx, KVDRO_ECUDA, "cannot select device %d", ctx->device);
    if (int rc = check_device(ctx, {{"q", q}, {"q_off", q_off}, {"kv_len", kv_len}, {"table", table}, {"out", out}})) return rc;
    if (lse)
        if (int rc = check_device(ctx, {{"lse", lse}})) return rc;
    const int64_t dense[2] = {(int64_t)n_heads * kv->head_dim, kv->head_dim};
    int64_t qs[2] = {}, os[2] = {};
    if (int rc = rows(ctx, "q", q, q_stride, 2, dense, qs)) return rc;
    if (int rc = rows(ctx, "out", out, out_stride, 2, dense, os)) return rc;
    kvdro::AttendArgs a;
    a.q = static_cast<const uint16_t*>(q);
    a.v = static_cast<const uint16_t*>(kv->v);
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.q_tok = qs[0];
    a.q_head = qs[1];
    a.out_tok = os[0];
    a.out_head = os[1];
    a.v_page = kv->v_stride[0];
    a.v_slot = kv->v_stride[1];
    a.v_head = kv->v_stride[2];
    a.q_off = q_off;
    a.kv_len = kv_len;
    a.table = table;
    a.B = B;
    a.T = T;
    a.heads = n_heads;
    a.kv_heads = kv->heads;
    a.group = n_heads / kv->heads;
    // p = 31 + ceil(log2 group), mul = ceil(2^p / group) < 2^32: row * mul >> p is exact for rows below 2^31, since
    // mul * group exceeds 2^p by less than group <= 2^(p - 31).
    a.group_shift = 31 + log2_of(a.group);
    a.group_mul = (uint32_t)((((uint64_t)1 << a.group_shift) + a.group - 1) / a.group);
    a.min_q = 0;
    a.max_q = 0x7fffffff;
    a.head_dim = kv->head_dim;
    a.n_pages = kv->n_pages;
    a.page_shift = kv->page_shift;
    a.max_pages = max_pages;
    a.window = window;
    a.half = kv->half;
    a.causal = causal != 0;
    a.scale = (float)scale;
    a.cap = (float)softcap;
    a.pieces = static_cast<float*>(ctx->kv_pieces.p);
    a.tickets = static_cast<unsigned*>(ctx->kv_tickets.p);
    a.joins = static_cast<kvdro::Join*>(ctx->kv_joins.p);
    a.wait_ns = ctx->skip_chunk >= 0 ? kTestWaitNs : kWaitNs;
    a.skip = ctx->skip_chunk;
    a.err = static_cast<int32_t*>(ctx->kv_err.p);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    ctx->kv_last = s;
    // Calls share the scratch: one on another stream than the last waits for that one.  (By the streams' numbers: a new stream
    // may have an old one's handle.  Waiting in every case cost a small call 2 us.)
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    KV_CUDA(cudaStreamIsCapturing(s, &capture), "asking for the stream's state");
    const bool captured = capture != cudaStreamCaptureStatusNone;
    unsigned long long number = 0;
    if (!captured) KV_CUDA(cudaStreamGetId(s, &number), "asking for the stream's number");
    if (!captured && ctx->kv_used && ctx->kv_stream != number) KV_CUDA(cudaStreamWaitEvent(s, ctx->kv_done, 0), "ordering streams");
    // Few rows that share a key head run on the kernel for single tokens, many on the one for chunks; a batch that may hold
    // both runs on both, each request on its own.
    const int64_t most = max_q > 0 ? max_q : T > B ? T : 1;  // new tokens of a request, as far as is known
    const bool eight = a.group <= 8 && most * a.group <= 8;
    if (most * a.group <= kFewRows) {
        KV_CUDA(kvdro::launch_kv_decode(a, kv->maps, eight, ctx->sms, s), "attention kernel");
    } else {
        const int32_t few = (a.group <= 8 ? 8 : kFewRows) / a.group;
        const bool both = few > 0 && (max_q == 0 || (int64_t)max_q * B != T);
        if (both) {
            a.max_q = few;
            KV_CUDA(kvdro::launch_kv_decode(a, kv->maps, a.group <= 8, ctx->sms, s), "attention kernel");
            a.min_q = few;
            a.max_q = 0x7fffffff;
            a.pieces += kvdro::kv_decode_piece_bytes(ctx->sms) / sizeof(float);
        }
        KV_CUDA(kvdro::launch_kv_chunk(a, kv->maps, both, ctx->sms, s), "attention kernel");
    }
    if (!captured) {
        KV_CUDA(cudaEventRecord(ctx->kv_done, s), "recording an event");
        ctx->kv_stream = number;
        ctx->kv_used = true;
    }
    return KVDRO_OK;
}

}  // extern "C"

namespace kvdro {

// What memory with these attributes should be for a context of this device, or null if it is that.
const char* kv_not_usable(const cudaPointerAttributes& at, int device) {
    if (at.type == cudaMemoryTypeManaged) return nullptr;
    if (at.type != cudaMemoryTypeDevice) return "device memory";
    return at.device == device ? nullptr : "memory of the context's device";
}

// Waits for the last page cache call, and for the last attention call, which may be on another stream.
int wait_kv(kvdro_ctx* ctx) {
    KV_CUDA(cudaStreamSynchronize(ctx->kv_last), "synchronising");
    if (ctx->kv_used) KV_CUDA(cudaEventSynchronize(ctx->kv_done), "synchronising");
    return KVDRO_OK;
}

// What the page cache's kernels reported, cleared.  They have been waited for, but earlier calls on other streams may still
// run: the word is taken in one step, so that what they report meanwhile is kept for the next time.
int check_kv_errors(kvdro_ctx* ctx) {
    if (!ctx->kv_err_ready) return KVDRO_OK;
    auto read = [&](int i, int32_t* to) {
        KV_CUDA(cudaMemcpyAsync(to, static_cast<int32_t*>(ctx->kv_err.p) + i, sizeof(*to), cudaMemcpyDeviceToHost, ctx->kv_side),
                "reading kernel status");
        KV_CUDA(cudaStreamSynchronize(ctx->kv_side), "reading kernel status");
        return (int)KVDRO_OK;
    };
    int32_t bits = 0;
    if (int rc = read(0, &bits)) return rc;
    if (!bits) return KVDRO_OK;
    KV_CUDA(launch_kv_take(static_cast<int32_t*>(ctx->kv_err.p), ctx->kv_side), "taking kernel status");
    if (int rc = read(1, &bits)) return rc;
    if (bits & kKvErrTimeout) {  // arrivals may be missing; replays of captured calls may be counting theirs
        KV_CUDA(cudaDeviceSynchronize(), "synchronising");
        if (int rc = clear(ctx, ctx->kv_tickets.p, ctx->kv_tickets.bytes)) return rc;
        return fail(ctx, KVDRO_ETIMEOUT, "an attention kernel gave up a bounded wait");
    }
    return fail(ctx, KVDRO_ERANGE, "a page cache kernel met a page number, slot or length outside its range");
}

}  // namespace kvdro
