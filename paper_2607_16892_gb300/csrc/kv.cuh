// Internal declarations of the page cache: the handle's description and the kernels' arguments.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace kvdro {

// Error bits that page cache kernels report in the first word of ctx->kv_err.
constexpr int kKvErrRange = 1;
constexpr int kKvErrTimeout = 2;

constexpr int kKvMaxRequests = 16384;

const char* kv_not_usable(const cudaPointerAttributes& at, int device);  // kv_api.cu

cudaError_t launch_kv_take(int32_t* err, cudaStream_t s);  // moves the first word to the second

struct PlanArgs {
    int32_t page_shift, n_pages, B, max_pages, T;
    const int32_t *cached, *new_len, *reserve, *held, *pool;
    int32_t *table, *ring, *held_out, *pool_out, *q_off, *kv_len, *slot, *pos;
    int32_t* err;
};
cudaError_t kv_plan_prepare();
cudaError_t launch_kv_plan(const PlanArgs& a, int sms, cudaStream_t s);

struct AppendArgs {
    const uint4 *k, *v;                      // caller's rows, in 16-byte units like every stride below
    uint4 *kc, *vc;                          // the cache
    int64_t k_tok, k_head, v_tok, v_head;
    int64_t kc_page, kc_slot, kc_head, vc_page, vc_slot, vc_head;
    const int32_t* slot;
    int32_t T, n_slots, page_shift, heads, vec_shift;  // 16-byte vectors of a head: 1 << vec_shift
    int32_t* err;
};
cudaError_t launch_kv_append(const AppendArgs& a, cudaStream_t s);

// Quantises as it copies: all strides in 16-byte units.
struct Append8Args {
    const uint4 *k, *v;
    uint4 *kc, *vc;
    uint8_t *k_exp, *v_exp;
    int64_t k_tok, k_head, v_tok, v_head;
    int64_t kc_page, kc_slot, kc_head, vc_page, vc_slot, vc_head;
    const int32_t* slot;
    int32_t T, n_slots, page_shift, heads, part_shift;  // parts of 16 elements of a head: 1 << part_shift
    bool half;
    int32_t* err;
};
cudaError_t launch_kv_append8(const Append8Args& a, cudaStream_t s);

struct ReadArgs {
    const char *kc, *vc;
    const uint8_t *k_exp, *v_exp;  // null: 16 bits
    uint4 *k, *v;                  // results
    int64_t k_tok, k_head, v_tok, v_head;                            // in 16-byte units
    int64_t kc_page, kc_slot, kc_head, vc_page, vc_slot, vc_head;  // in bytes
    const int32_t *q_off, *kv_len, *table;
    int32_t B, T, n_pages, page_shift, max_pages, heads, vec_shift;
    bool half;
    int32_t* err;
};
cudaError_t launch_kv_read(const ReadArgs& a, cudaStream_t s);

// Tensor maps of a cache (d, slot, head, page) for boxes of a page's slots by 64 elements of d, and of 32 slots at most.  8 bits: all
// of d in a box, the former not permuted, the latter of 64 slots where heads are of 64.
struct KvMaps {
    CUtensorMap k, v, k_slice, v_slice;
};

// A tile of the chunk kernel that several CTAs share, noted by the first of them.
struct Join {
    int32_t q0, h, row0, rows;  // the request's first token; key head; the tile's rows
    int32_t last;  // the last CTA with a piece; -1: no tile
};

enum class Part : int32_t { kWhole, kLeave, kJoin };

struct AttendArgs {
    const uint16_t* q;
    const void* v;
    uint16_t* out;
    float* lse;
    int64_t q_tok, q_head, out_tok, out_head, v_page, v_slot, v_head;  // in elements
    const int32_t *q_off, *kv_len, *table;
    int32_t B, T, heads, kv_heads, group, head_dim, n_pages, page_shift, max_pages, window;
    uint32_t group_mul;  // a row's token: row / group = row * group_mul >> group_shift, for rows below 2^31
    int32_t group_shift;
    int32_t min_q, max_q;  // a launch's requests: more than min_q tokens, at most max_q
    bool half, causal;
    float scale, cap;    // cap 0: none
    float* pieces;       // sums of tiles that several CTAs share
    unsigned* tickets;   // by CTA: arrivals at the tile that its stretch ends in, zero between calls
    Join* joins;         // by CTA
    const uint8_t *k_exp, *v_exp;  // 8 bits: a byte E + 127 per page, head and slot, in this order; null: 16 bits
    int32_t head_shift;  // 8 bits, eight rows: a tile of the kernel for few rows is of 2^head_shift key heads
    // Prefixes: a launch over them takes request g's tokens from those of requests share_off[g] .. share_off[g + 1] - 1 of
    // the caller's `share_n`, and leaves its sums; one over the requests' own pages joins those with its own.
    const int32_t* share_off;
    int32_t share_n;
    // Prefixes read by each of their requests, in front of its own tokens: as the call gives them.
    const int32_t *pre_off, *pre_len, *pre_table;
    int32_t pre_n, pre_pages;
    Part part;
    float* sums;         // [T][heads][head_dim]
    float2* sum_ml;      // [T][heads]: maximum (in log2) and sum of weights
    unsigned long long wait_ns;  // bound of a wait
    int32_t skip;        // test hook: each CTA leaves this copy out, so that the wait for it runs out; -1: none
    int32_t* err;
};
size_t kv_decode_piece_bytes(int sms);
int kv_decode_ctas(int sms);
cudaError_t kv_decode_prepare();
cudaError_t kv_decode8_prepare();
cudaError_t kv_direct_prepare();
cudaError_t kv_direct8_prepare();
// `rows`: that share a key head, at most (more are right, but slow).  `early`: may start while the launch before it, whose sums it
// joins, ends.
cudaError_t launch_kv_decode(const AttendArgs& a, const KvMaps& maps, int rows, bool early, int sms, cudaStream_t s);
cudaError_t launch_kv_decode8(const AttendArgs& a, const KvMaps& maps, int rows, bool early, int sms, cudaStream_t s);
// The same with a's prefixes in front of the requests' own tokens.
cudaError_t launch_kv_direct(const AttendArgs& a, const KvMaps& maps, int rows, int sms, cudaStream_t s);
cudaError_t launch_kv_direct8(const AttendArgs& a, const KvMaps& maps, int rows, int sms, cudaStream_t s);
size_t kv_chunk_piece_bytes(int sms);
bool kv_join_few(int64_t tiles, int sms);  // whether the launch that joins few tiles takes so many
cudaError_t kv_chunk_prepare();
cudaError_t kv_chunk8_prepare();
cudaError_t launch_kv_chunk8(const AttendArgs& a, const KvMaps& maps, bool after_few, int sms, cudaStream_t s);
// `after_few`: beside a launch of kv_decode for the requests of few rows, directly before it, on other scratch.
cudaError_t launch_kv_chunk(const AttendArgs& a, const KvMaps& maps, bool after_few, int sms, cudaStream_t s);

}  // namespace kvdro
