// Attention of few rows over pages: single tokens, drafted tokens.
//
// Bound by the bytes of the keys and values, each read once for the (at most 16; 8 bits: 24) rows that share a key head.  The line of
// all blocks of 128 positions is dealt to two to four CTAs per SM (kv_device.cuh); in a block each of a CTA's four warps has 32
// positions of its own, with its own ring of tensor copies, maxima, sums and weighted sums: nothing in the loop waits
// for another warp.  The warps are joined through shared memory at the end of a tile, pieces of a tile through
// global memory by the CTA that arrives last, both in a fixed order.
//
// Products run on mma.m16n8k16 with the positions (then the columns of V) as the 16 and the rows as the 8, so that up to
// eight rows fill what they are given: S^T = K Q^T, O^T += V^T P^T.  A tcgen05 tile would have 128 rows.  With eight to
// sixteen warps on an SM a warp's latency per slice counts, hence 32 positions at a time and a maximum that is raised only when a
// row's own passes it by 2^8 (O and the sum refer to the same one), which saves the shuffles in most slices.
// The weights are rounded to the cache's type for the second product, which adds about as much error as the result's own
// rounding.
//
// Measured (bf16, 8 key heads of 128, four query heads each): 64 requests of lognormal lengths up to 8192, 557 MB, 96 us =
// 5.8 TB/s; 4 requests of 131072 with eight query heads each, 2148 MB, 325 us = 6.6 TB/s (a copy runs at 6.8); one request of
// 1000, 10.4 us, all latency.
//
// Caches of 8 bits (Q): codes become FP16, exactly, two to an instruction, as they leave shared memory, whatever the type of the
// queries; BF16 queries become FP16 times a power of two per row.  A key's scale multiplies its scores.  A value's scale goes
// into its weight for O, 2^(s - m + E - c), beside 2^(s - m) in the sum: c, a whole number, follows the largest s - m + E as m follows the
// largest s, so that tokens' sizes may differ by any factor.  As weights are FP16, held 2^7 above 1 at the largest, what is below 2^-32 of a
// row's largest weight times 2^E is lost, also in columns where that token holds zeros.
// V is transposed in pairs of columns, as 16-bit elements, and a byte permutation per register parts them.
// Half the bytes leave half the time for as many positions, and what bounds such a kernel first is its own code: unrolled over 32
// positions it took 1050 instructions a slice (70 us for the batch below), over 64 1700 and as long, warps waiting for instructions
// more often than for data; the loop over 16 positions is rolled, 460 instructions with their share of a slice's, and the batch takes 61.  Copies without any
// products take 57: rows of 128 bytes are the least that DRAM gives, and rows of 64 are read in pairs of heads.
// Measured (8 bits): 64 requests of lognormal lengths up to 8192, 8 key heads of 128, 281 MB, 60 to 64 us from one GPU to the next = 4.7 to 4.4
// TB/s; 4 requests of 131071, 16 heads of 64, 1090 MB, 180 to 205 us = 6.1 to 5.3 TB/s; one request of 1000, 12.3 us, all latency.
//
// With prefixes in front (S) a request's line of blocks begins with its prefix's, and pages are looked up in the one table or the other:
// what it costs to read a short prefix once per request out of L2 is less than the launches that read it once for all.
#pragma once

#include "kv_device.cuh"

namespace kvdro {

namespace {

using namespace kv;

constexpr int kWarps = 4, kThreads = 32 * kWarps, kMostRows = 24;
constexpr int kMostCtas = 4;  // per SM
constexpr int kOver = 2;      // a tile's fixed cost, in blocks (0 / 1 / 2: window case 41.3 / 40.3 / 39.6 us)
constexpr int kAtOnce = 8;    // pieces read at a time
constexpr float kTop = kRaise + kLift<true>;  // 8 bits: weights are 2^15 at most, which FP16 holds

template <int D, int NR, bool Q>
struct Ring {  // a stage: K or V of a slice; 8 bits: both
    // What fits the registers and the shared memory.  Eight rows, D 128: 3 CTAs of 2 stages 95 us (64 requests), 2 of 3 stages 99;
    // D 64: 4 of 3 stages 41 us (window case), 3 of 4 stages 44, 2 of 6 stages 52.
    // 8 bits: keys and values of a slice together; of heads of 64, 64 positions (four requests of 131071: 215 us, 253 with 32).
    static constexpr int kSlice = Q && D == 64 ? 64 : 32;
    // Sixteen rows of 64: 3 CTAs of 2 stages 29.7 us (32 requests of 3000), 2 of 3 stages 31.5; of 128 3 CTAs spill, 47.4 us for 40.5.
    static constexpr int kCtas = D == 128 ? (NR == 1 ? 3 : 2) : (NR == 1 ? (Q ? 3 : 4) : Q && NR == 2 ? 3 : 2);  // per SM
    static constexpr int kBytes = kSlice * D * 2;
    static constexpr int kStages = D == 128 || Q ? (NR == 1 || (Q && D == 64 && NR == 2) ? 2 : 3) : (NR == 1 ? 3 : 6);
    static constexpr int kScales = Q ? kWarps * kStages * 2 * kSlice : 0;  // a byte per key and value, behind the ring
    // Queries in shared memory where they and the sums do not fit the registers (24 rows of 128, 32 requests of 3000: 78 us in registers, 52 so).
    static constexpr bool kHoldQ = Q && D == 128 && NR == 3;
    static constexpr int kQAt = kWarps * kStages * kBytes + kScales, kQueries = kHoldQ ? NR * (D / 16) * 32 * 8 : 0;
    static constexpr int kSmem = kQAt + kQueries + 1024;
    static_assert(Stretch<kThreads>::kScratch <= kSmem, "the ring is scratch first");
};
// A piece in global memory: rows (8 bits: of two heads, if of eight) of D sums, then their maxima and sums of weights.
template <int D>
constexpr int kPieceFloats = kMostRows * (D + 2);

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {  // an 8 x 8 matrix of 16-bit elements across the warp
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <bool H>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (H)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Byte offset of 16-byte chunk `c` of row `key` in a slice: rows of 128 bytes (halves of 64 elements; 8 bits: whole rows, which
// for heads of 64 have 64 bytes) whose chunks the tensor copy permutes by the row.
template <int D, bool Q>
__device__ __forceinline__ uint32_t chunk_at(int key, int c) {
    if constexpr (Q && D == 64) return (uint32_t)(key * 64 + ((c ^ (key >> 1 & 3)) << 4));
    if constexpr (Q) return (uint32_t)(key * 128 + ((c ^ (key & 7)) << 4));
    return (uint32_t)((c >> 3) * (32 * 128) + key * 128 + (((c & 7) ^ (key & 7)) << 4));
}
__device__ __forceinline__ uint32_t load_u8(uint32_t at) {
    uint32_t x;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x) : "r"(at));
    return x;
}

// 8 bits: rows are left in units of 2^k, which brings their sum of weights into [1/2, 1): sums of weights times values are then no larger than
// the values.  k for a sum that refers to m, or 0 where m + k is rounded.
__device__ __forceinline__ float unit_of(float m, float sum) {
    const float k = (float)((int)(__float_as_uint(sum) >> 23) - 126);
    return sum > 0.f && sum < INFINITY && (m + k) - m == k ? k : 0.f;
}
__device__ __forceinline__ float power_of(float k) { return __uint_as_float((uint32_t)(127 + (int)k) << 23); }  // 2^k, -126 to 127

// NR: groups of eight rows of a tile.
template <bool H, int D, int NR, bool Q, bool S>
__global__ void __launch_bounds__(kThreads, Ring<D, NR, Q>::kCtas)
    k_kv_decode(const AttendArgs a, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
    extern __shared__ __align__(16) char s_raw[];  // 64-bit words of the search first
    constexpr int kSlice = Ring<D, NR, Q>::kSlice, kKeys = kSlice * kWarps;
    constexpr int kStages = Ring<D, NR, Q>::kStages, kStage = Ring<D, NR, Q>::kBytes, KS = D / 16, DT = D / 16, MT = kSlice / 16;
    constexpr int kRows = 8 * NR;
    using DecodeLine = Line<kRows, kKeys, kSlice, kOver, Q && NR == 1, S>;
    constexpr bool kLifted = H && !Q;  // weights are 2^(s - m + kLift); 8 bits: 2^(s - m), of an m that lies below by that much
    // Where column c of row r of the sums stands in shared memory, without bank conflicts.
    auto sum_at = [](int r, int c) { return Q ? r * D + (c ^ (r >> 1 & 3) << 3) : r * (D + 4) + c; };
    __shared__ alignas(8) uint64_t s_bar[kWarps][kStages];
    __shared__ Stretch<kThreads> s_part;
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
    __shared__ float4 s_row[Q ? kRows * (NR == 1 ? 2 : 1) : 1];  // 8 bits, by head and row: maximum and sum in its unit, what that began from, the unit
    __shared__ int s_last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_u32(s_raw), ring = ((raw + 1023) & ~1023u) + warp * kStages * kStage;
    char* const ring_ptr = s_raw + (ring - raw);
    // A tile's heads, of which this warp has one, and its warps with the others of that head a block's slices.
    const int hs = Q && NR == 1 ? a.head_shift : 0, of_head = kWarps >> hs, my_head = warp / of_head, my_slice = (warp & (of_head - 1)) * kSlice;
    const uint32_t flip = (D == 128 ? lane & 7 : lane >> 1 & 3) << 4;  // 8 bits: how chunks of row lane & 15 of sixteen are permuted
    const uint32_t scales = ((raw + 1023) & ~1023u) + kWarps * kStages * kStage + warp * kStages * 2 * kSlice;
    constexpr bool kHoldQ = Ring<D, NR, Q>::kHoldQ;
    uint2* const s_q = reinterpret_cast<uint2*>(s_raw + (((raw + 1023) & ~1023u) - raw) + Ring<D, NR, Q>::kQAt) + lane;
    DecodeLine line(a);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // a launch for many rows may fill SMs that this one leaves

    if (lane < kStages) mbar_init(smem_u32(&s_bar[warp][lane]), 1);
    fence_mbar_init();

    s_part.find(line, s_raw);
    clear_rest<D, kThreads>(line);
    fence_proxy_async();  // the ring served as scratch
    __syncthreads();
    if (s_part.empty()) {
        if (line.bad && tid == 0) atomicOr(a.err, kKvErrRange);
        if (a.part == Part::kJoin) asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }

    // Units in the order K, V of a slice, K, V of the next; 8 bits: a unit is both.
    Walk<DecodeLine> in(line, s_part), w = in;  // of the copies, and of the sums
    int in_blk = in.p0;
    bool in_v = false;
    int fetched = 0;

    // Page numbers of this warp's slices of 32 blocks, one per lane; a slice has several pages if they have fewer slots.
    constexpr int NP = kSlice / 16;
    const int slots = min(kSlice, 1 << a.page_shift);
    int pg[NP], pg_b = -1, pg_rt = -1, pg_blk = -1;
#pragma unroll
    for (int i = 0; i < NP; i++) pg[i] = -1;
    bool range = false;
    uint32_t filled = 0, phase = 0;  // by stage: holds a slice; the parity to wait for
    uint32_t gaps = 0;               // by stage, a bit for each 16 positions whose page number is none
    constexpr uint32_t kAllGaps = (1u << NP) - 1;
    // The page numbers of the slices around the next one, unless they are there.
    auto look_up = [&] {
        if (in.at.b == pg_b && in.at.rt == pg_rt && (in_blk >> 5) == pg_blk) return;
        pg_b = in.at.b;
        pg_rt = in.at.rt;
        pg_blk = in_blk >> 5;
        const int j = in.at.t.lo + ((in_blk & ~31) + lane) * line.keys() + my_slice;
        const int seen_lo = line.seen(in.at.r, line.token(in.at.rt * kRows)).x;
#pragma unroll
        for (int i = 0; i < NP; i++) {
            pg[i] = -1;
            if (S && j < 0) {
                const int at = j + 16 * i + in.at.r.pad;
                if (at < in.at.r.pre) {
                    const int page = a.pre_table[(int64_t)in.at.r.prefix * a.pre_pages + (at >> a.page_shift)];
                    if ((uint32_t)page < (uint32_t)a.n_pages) pg[i] = page;
                    else range = true;
                }
            } else if (j + 16 * i < in.at.t.hi && ((j + 16 * i) | (slots - 1)) >= seen_lo) {  // else no row's business
                const int page = a.table[(int64_t)in.at.b * a.max_pages + ((j + 16 * i) >> a.page_shift)];
                if ((uint32_t)page < (uint32_t)a.n_pages) pg[i] = page;
                else range = true;
            }
        }
    };
    // 8 bits: the next slice's keys, values and scales.
    auto fetch8 = [&](int stage) {
        filled &= ~(1u << stage);
        if (!in.more) return;
        look_up();
        int p[NP];
        uint32_t gap = 0;
#pragma unroll
        for (int i = 0; i < NP; i++) {
            p[i] = __shfl_sync(~0u, pg[i], in_blk & 31);
            gap |= (p[i] < 0 ? 1u : 0u) << i;
        }
        gaps = (gaps & ~(kAllGaps << NP * stage)) | gap << NP * stage;
        if (gap != kAllGaps) {
            const int slot = __shfl_sync(~0u, (in.at.t.lo + in_blk * line.keys() + my_slice) & ((1 << a.page_shift) - 1), 0);
            const int head = __shfl_sync(~0u, (in.at.h << hs) + my_head, 0);
            const uint32_t bar = __shfl_sync(~0u, smem_u32(&s_bar[warp][stage]), 0), to = __shfl_sync(~0u, ring + stage * kStage, 0);
            const uint32_t scale_to = __shfl_sync(~0u, scales + stage * 2 * kSlice, 0);
            if (fetched != a.skip && elect_one()) {  // (left out: a test's wait runs out)
                mbar_expect(bar, kStage + 2 * kSlice);
                auto copy = [&](int at, int page) {  // a page that is none reads as zeros, with any page's scales
                    const int box_page = page >= 0 ? page : a.n_pages;
                    const int64_t e = (((int64_t)max(page, 0) * a.kv_heads + head) << a.page_shift) + slot;
                    load_box(to + at * D, &kmap, 0, slot, head, box_page, bar);
                    load_box(to + (kSlice + at) * D, &vmap, 0, slot, head, box_page, bar);
                    load_bytes(scale_to + at, a.k_exp + e, slots, bar);
                    load_bytes(scale_to + kSlice + at, a.v_exp + e, slots, bar);
                };
                if (slots == kSlice) {
                    copy(0, p[0]);
                } else if (slots == 16) {
#pragma unroll
                    for (int i = 0; i < NP; i++) copy(16 * i, p[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < NP; i += 2) copy(16 * i, p[i]);
                }
            }
            filled |= 1u << stage;
        }
        fetched++;
        if (++in_blk == in.p1) {
            in.next();
            in_blk = 0;
        }
    };
    auto fetch = [&](int stage) {
        filled &= ~(1u << stage);
        if (!in.more) return;
        look_up();
        const int p0 = __shfl_sync(~0u, pg[0], in_blk & 31), p1 = __shfl_sync(~0u, pg[1], in_blk & 31);
        gaps = (gaps & ~(3u << 2 * stage)) | ((p0 < 0 ? 1u : 0u) | (p1 < 0 ? 2u : 0u)) << 2 * stage;
        if (p0 >= 0 || p1 >= 0) {
            const int slot = __shfl_sync(~0u, (in.at.t.lo + in_blk * kKeys + warp * kSlice) & ((1 << a.page_shift) - 1), 0);
            const int head = __shfl_sync(~0u, in.at.h, 0);
            const uint32_t bar = __shfl_sync(~0u, smem_u32(&s_bar[warp][stage]), 0), to = __shfl_sync(~0u, ring + stage * kStage, 0);
            if (fetched != a.skip && elect_one()) {  // (left out: a test's wait runs out)
                const CUtensorMap* const map = in_v ? &vmap : &kmap;
                mbar_expect(bar, kStage);
#pragma unroll
                for (int d = 0; d < D / 64; d++) {  // a page that is none reads as zeros
                    load_box(to + d * (kSlice * 128), map, d * 64, slot, head, p0 >= 0 ? p0 : a.n_pages, bar);
                    if (slots < kSlice) load_box(to + d * (kSlice * 128) + 16 * 128, map, d * 64, slot, head, p1 >= 0 ? p1 : a.n_pages, bar);
                }
            }
            filled |= 1u << stage;
        }
        fetched++;
        in_v = !in_v;
        if (in_v) return;
        if (++in_blk == in.p1) {
            in.next();
            in_blk = 0;
        }
    };
#pragma unroll
    for (int s = 0; s < kStages; s++) {
        if constexpr (Q) fetch8(s);
        else fetch(s);
    }

    const float mul = a.cap > 0.f ? 2.f * kLog2e * a.scale / a.cap : kLog2e * a.scale, cap2 = a.cap * kLog2e;
    uint32_t qf[NR][KS][2];
    float o[NR][DT][4];  // columns 16 d + (lane >> 2) and 8 more (8 bits: 16 d + 2 (lane >> 2) and 1 more), of the rows
    float m[NR][2], l[NR][2];  // of rows 8 n + 2 (lane & 3) + i
    float qmul[NR][2];          // 8 bits: what turns products into scores
    float c[NR][2], up[NR][2];  // 8 bits: O refers to 2^(m + c), c a whole number; m is raised where s - m passes `up`
    int2 see[NR][2];
    int2 all_see, any_see;  // positions that every row of the tile sees, and that some row does
    int none = 0;           // S: from here to 0 there are no positions
    bool dead = false;
    int stage = 0;

    // The slice in `stage`, once it is there; false if there is none.
    auto ready = [&] {
        if (!(filled >> stage & 1) || dead) return false;
        const uint32_t bar = smem_u32(&s_bar[warp][stage]), parity = phase >> stage & 1;
        if (__all_sync(~0u, mbar_try(bar, parity) || mbar_wait_slow(bar, parity, a.wait_ns, nullptr))) phase ^= 1u << stage;
        else dead = true;
        return !dead;
    };
    auto advance = [&] {
        if constexpr (Q) {
            if (!dead) fetch8(stage);
        } else {
            if (!dead) fetch(stage);
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
    };

    bool waited = a.part != Part::kJoin;  // for the sums of the launch before, beside which this one may have started
    while (w.more) {
        Cursor& at = w.at;
        {  // a tile begins here, or this CTA's piece of it
            const int first = at.rt * kRows, rows = min(kRows, at.r.rows - first);
#pragma unroll
            for (int n = 0; n < NR; n++) {
                {
                    const int r = first + min(8 * n + (lane >> 2), rows - 1), tok = line.token(r), g = r - tok * a.group;
                    const uint16_t* const q = a.q + (int64_t)(at.r.q0 + tok) * a.q_tok + (int64_t)(((at.h << hs) + my_head) * a.group + g) * a.q_head + (Q ? 4 : 2) * (lane & 3);
#pragma unroll
                    for (int k = 0; k < KS; k++) {
                        if constexpr (Q) {  // a register of codes holds four neighbours: theirs
                            const uint2 x = *reinterpret_cast<const uint2*>(q + k * 16);
                            qf[n][k][0] = x.x;
                            qf[n][k][1] = x.y;
                        } else {
                            qf[n][k][0] = *reinterpret_cast<const uint32_t*>(q + k * 16);
                            qf[n][k][1] = *reinterpret_cast<const uint32_t*>(q + k * 16 + 8);
                        }
                    }
                    if constexpr (Q && !H) {
                        // BF16 to FP16 at a row's largest in [1, 2): exact down to 2^-17 of that, off by 2^-25 of it below.  Where a key's
                        // elements are of one size that is less than the FP32 sum's rounding; a key with one large element, on a small one of
                        // the query, has a score that is off by 2^-25 of the largest of each.  A NaN stays one, an infinity too.
                        float top = 0.f;
#pragma unroll
                        for (int k = 0; k < KS; k++)
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                const float2 x = unpack2<false>(qf[n][k][i]);
                                top = fmaxf(top, fmaxf(fabsf(x.x), fabsf(x.y)));
                            }
                        top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
                        const int e = min(max((int)(__float_as_uint(top) >> 23), 1), 253);
                        const float down = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
                        for (int k = 0; k < KS; k++)
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                const float2 x = unpack2<false>(qf[n][k][i]);
                                qf[n][k][i] = pack2<true>(x.x * down, x.y * down);
                            }
#pragma unroll
                        for (int i = 0; i < 2; i++) qmul[n][i] = mul * __uint_as_float((uint32_t)__shfl_sync(~0u, e, (2 * (lane & 3) + i) * 4) << 23);
                    } else {
                        qmul[n][0] = qmul[n][1] = mul;
                    }
                    if constexpr (kHoldQ) {
                        if (warp == 0) {
#pragma unroll
                            for (int k = 0; k < KS; k++) s_q[(n * KS + k) * 32] = make_uint2(qf[n][k][0], qf[n][k][1]);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    see[n][i] = line.seen(at.r, line.token(first + min(8 * n + 2 * (lane & 3) + i, rows - 1)));
                    m[n][i] = Q ? 0.f : -INFINITY;
                    c[n][i] = 0.f;
                    up[n][i] = -INFINITY;  // nothing seen so far
                    l[n][i] = 0.f;
                }
#pragma unroll
                for (int d = 0; d < DT; d++)
#pragma unroll
                    for (int i = 0; i < 4; i++) o[n][d][i] = 0.f;
            }
            const int2 s0 = line.seen(at.r, line.token(first)), s1 = line.seen(at.r, line.token(first + rows - 1));
            all_see = make_int2(s1.x, s0.y);
            any_see = make_int2(s0.x, s1.y);
            if constexpr (S) none = at.r.pre - at.r.pad;
            if constexpr (kHoldQ) __syncthreads();
        }
        for (int blk = w.p0; blk < w.p1; blk++) {
        const int j0 = at.t.lo + blk * line.keys() + my_slice;
        if constexpr (Q) {
            const uint32_t gap = gaps >> NP * stage & kAllGaps;
            const bool edge = j0 < all_see.x || j0 + kSlice > all_see.y || gap || (S && j0 < 0 && j0 + kSlice > none);
            if (ready()) {
                const uint32_t kt = ring + stage * kStage, vt = kt + kSlice * D, ke = scales + stage * 2 * kSlice + (lane >> 2), ve = ke + kSlice;
                auto seen = [&](int j) { return j >= any_see.x && j < any_see.y && !(S && j >= none && j < 0); };
                bool odd = false;  // a value that some rows see and others do not is NaN
                if (edge && (any_see.x != all_see.x || any_see.y != all_see.y)) {
#pragma unroll 1
                    for (int c = lane; c < kSlice * D / 16; c += 32) {
                        uint32_t w[4];
                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                                     : "r"(vt + c * 16));
                        odd |= (any_nan8(w[0]) || any_nan8(w[1]) || any_nan8(w[2]) || any_nan8(w[3])) && seen(j0 + c / (D / 16));
                    }
                    odd = __any_sync(~0u, odd);
                }
                // Sixteen positions at a time in a rolled loop: unrolled, what 64 or 32 of them take left the instruction cache.
#pragma unroll 1
                for (int t = 0; t < MT; t++) {
                    float s[NR][4];  // scores, then weights: position 16 t + (lane >> 2) + 8 (i >> 1), row 8 n + 2 (lane & 3) + (i & 1)
#pragma unroll
                    for (int n = 0; n < NR; n++)
#pragma unroll
                        for (int i = 0; i < 4; i++) s[n][i] = 0.f;
                    const uint32_t krow = kt + (16 * t + (lane & 15)) * D;
#pragma unroll
                    for (int k = 0; k < KS; k += 2) {
                        uint32_t x[4];
                        ldsm4(x, krow + ((k + (lane >> 4)) << 4 ^ flip));
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            const uint32_t kf[4] = {half2_of(x[2 * i]), half2_of(x[2 * i + 1]), half2_of(x[2 * i] >> 16), half2_of(x[2 * i + 1] >> 16)};
#pragma unroll
                            for (int n = 0; n < NR; n++) {
                                uint2 q = make_uint2(qf[n][k + i][0], qf[n][k + i][1]);
                                if constexpr (kHoldQ)
                                    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(q.x), "=r"(q.y) : "r"(smem_u32(s_q + (n * KS + k + i) * 32)));
                                mma<true>(s[n], kf, q.x, q.y);
                            }
                        }
                    }
                    // Scales of the keys, exponents of the values'.  A key's scale meets its query's first: one of 2^119 times a sum of codes, 2^17 at
                    // most, would pass FP32 before a query of 2^-110 brings it back.
                    float ks[2], vs[2];
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        ks[i] = scale_of(load_u8(ke + 16 * t + 8 * i));
                        vs[i] = (float)((int)load_u8(ve + 16 * t + 8 * i) - 127);
                    }
                    // Exponents of the weights in l, d = s - m, and of those in O, e = d + (E - c), whose factor is a power of two: whatever FP32
                    // made of s, both come from the same d, so that O / l is a mean.
                    float e[NR][4];
                    bool raise = false;
#pragma unroll
                    for (int n = 0; n < NR; n++) {
#pragma unroll
                        for (int i = 0; i < 4; i++) s[n][i] = score(s[n][i], ks[i >> 1] * qmul[n][i & 1], cap2);
                        if (edge) {
                            const int j = j0 + 16 * t + (lane >> 2);
#pragma unroll
                            for (int i = 0; i < 4; i++)
                                if (j + 8 * (i >> 1) < see[n][i & 1].x || j + 8 * (i >> 1) >= see[n][i & 1].y || (gap >> t & 1) ||
                                    (S && j + 8 * (i >> 1) >= none && j + 8 * (i >> 1) < 0))
                                    s[n][i] = -INFINITY;
                        }
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            s[n][i] -= m[n][i & 1];
                            e[n][i] = s[n][i] + (vs[i >> 1] - c[n][i & 1]);
                        }
#pragma unroll
                        for (int i = 0; i < 2; i++) raise |= fmaxf(s[n][i], s[n][i + 2]) > up[n][i] || fmaxf(e[n][i], e[n][i + 2]) > kTop;
                    }
                    if (__any_sync(~0u, raise)) {  // m by whatever brings the largest d to 7, c what brings the largest e there
#pragma unroll
                        for (int n = 0; n < NR; n++)
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                float top = fmaxf(s[n][i], s[n][i + 2]), tope = fmaxf(e[n][i], e[n][i + 2]);
#pragma unroll
                                for (int x = 4; x < 32; x <<= 1) {
                                    top = fmaxf(top, __shfl_xor_sync(~0u, top, x));
                                    tope = fmaxf(tope, __shfl_xor_sync(~0u, tope, x));
                                }
                                const bool first = up[n][i] == -INFINITY, some = !first || top != -INFINITY;
                                float by = top - kLift<true>;
                                if (!first) by = fmaxf(by, 0.f);
                                const float to = some ? m[n][i] + by : 0.f;
                                by = to - m[n][i];  // as it was rounded
                                float by_e = rintf(tope - by - kLift<true>);
                                if (!first) by_e = fmaxf(by_e, ceilf(-by));  // m + c never falls
                                if (!(fabsf(by_e) < INFINITY)) by_e = 0.f;   // nothing seen, or a row that is NaN
                                l[n][i] *= exp2_fast(fminf(-by, 0.f));
                                const float keep = exp2_fast(fminf(-(by + by_e), 0.f));
                                m[n][i] = to;
                                c[n][i] += by_e;
                                if (some) up[n][i] = kTop;
#pragma unroll
                                for (int k = 0; k < 4; k += 2) {
                                    s[n][i + k] -= by;
                                    e[n][i + k] = s[n][i + k] + (vs[k >> 1] - c[n][i]);
                                }
#pragma unroll
                                for (int d = 0; d < DT; d++) {
                                    o[n][d][i] *= keep;
                                    o[n][d][i + 2] *= keep;
                                }
                            }
                    }
                    uint32_t pf[NR][2];
#pragma unroll
                    for (int n = 0; n < NR; n++) {
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            l[n][i] += exp2_fast(s[n][i]) + exp2_fast(s[n][i + 2]);
                            e[n][i] = exp2_fast(e[n][i]);
                            e[n][i + 2] = exp2_fast(e[n][i + 2]);
                        }
                        pf[n][0] = transpose8(pack2<true>(e[n][0], e[n][1]));
                        pf[n][1] = transpose8(pack2<true>(e[n][2], e[n][3]));
                    }
                    if (!odd) {
                        uint32_t keep[2] = {~0u, ~0u};  // values of positions that no row sees are taken as zero, whatever is stored there
                        if (edge) {
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                const int j = j0 + 16 * t + 8 * i + 2 * (lane & 3);
                                keep[i] = (seen(j) ? 0xffffu : 0u) | (seen(j + 1) ? 0xffff0000u : 0u);
                            }
                        }
                        const uint32_t vrow = vt + (16 * t + (lane & 15)) * D;
#pragma unroll
                        for (int d = 0; d < DT; d += 2) {
                            // Transposed in pairs of columns: a register holds two columns of two positions.
                            uint32_t x[4];
                            ldsm4t(x, vrow + ((d + (lane >> 4)) << 4 ^ flip));
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                const uint32_t y = __byte_perm(x[2 * i] & keep[0], 0, 0x3120), z = __byte_perm(x[2 * i + 1] & keep[1], 0, 0x3120);
                                const uint32_t vf[4] = {half2_of(y), half2_of(y >> 16), half2_of(z), half2_of(z >> 16)};
#pragma unroll
                                for (int n = 0; n < NR; n++) mma<true>(o[n][d + i], vf, pf[n][0], pf[n][1]);
                            }
                        }
                    } else {  // row by row, over what each sees
#pragma unroll 1
                        for (int k = 0; k < 16; k++) {
                            const int from = (k & 7) * 4 + (lane & 3), j = j0 + 16 * t + k;
#pragma unroll
                            for (int n = 0; n < NR; n++) {
                                float w[2];
                                bool see_k[2];
#pragma unroll
                                for (int i = 0; i < 2; i++) {
                                    w[i] = __shfl_sync(~0u, k & 8 ? e[n][2 + i] : e[n][i], from);
                                    see_k[i] = j >= see[n][i].x && j < see[n][i].y && !(gap >> t & 1) && !(S && j >= none && j < 0);
                                }
#pragma unroll
                                for (int d = 0; d < 2 * DT; d++) {
                                    const uint32_t at = vt + chunk_at<D, Q>(16 * t + k, d >> 1) + 2 * (lane >> 2) + (d & 1);
                                    const float v = unpack2<true>(half2_of((uint16_t)load_u8(at))).x;
#pragma unroll
                                    for (int i = 0; i < 2; i++) {
                                        float& y = o[n][d >> 1][2 * (d & 1) + i];
                                        if (see_k[i]) y = fmaf(w[i], v, y);
                                    }
                                }
                            }
                        }
                    }
                }
            }
            if (blk + 1 < w.p1) {
                __syncwarp();
                advance();
            }
        } else {
        const bool edge = j0 < all_see.x || j0 + kSlice > all_see.y || (gaps >> 2 * stage & 3) || (S && j0 < 0 && j0 + kSlice > none);
        const uint32_t gap = gaps >> 2 * stage & 3;
        float s[NR][MT][4];  // scores, then weights: position 16 t + (lane >> 2) + 8 (i >> 1), row 8 n + 2 (lane & 3) + (i & 1)
        const bool some = ready();
        if (some) {
            const uint32_t st = ring + stage * kStage;
#pragma unroll
            for (int n = 0; n < NR; n++)
#pragma unroll
                for (int t = 0; t < MT; t++)
#pragma unroll
                    for (int i = 0; i < 4; i++) s[n][t][i] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; k++)
#pragma unroll
                for (int t = 0; t < MT; t++) {
                    uint32_t kf[4];
                    ldsm4(kf, st + chunk_at<D, Q>(16 * t + (lane & 15), 2 * k + (lane >> 4)));
#pragma unroll
                    for (int n = 0; n < NR; n++) mma<H>(s[n][t], kf, qf[n][k][0], qf[n][k][1]);
                }
        }
        __syncwarp();
        advance();
        const bool have = ready();
        const uint32_t st = ring + stage * kStage;
        if (some && have) {
            float top[NR][2];
#pragma unroll
            for (int n = 0; n < NR; n++) {
                top[n][0] = top[n][1] = -INFINITY;
#pragma unroll
                for (int t = 0; t < MT; t++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        float& x = s[n][t][i];
                        x = score(x, mul, cap2);
                        if (edge) {
                            const int j = j0 + 16 * t + (lane >> 2) + 8 * (i >> 1);
                            if (j < see[n][i & 1].x || j >= see[n][i & 1].y || (gap >> t & 1) || (S && j >= none && j < 0)) x = -INFINITY;
                        }
                        top[n][i & 1] = fmaxf(top[n][i & 1], x);
                    }
            }
            bool raise = false;
#pragma unroll
            for (int n = 0; n < NR; n++)
#pragma unroll
                for (int i = 0; i < 2; i++) raise |= raises<H>(top[n][i], m[n][i]);
            if (__any_sync(~0u, raise)) {
#pragma unroll
                for (int n = 0; n < NR; n++)
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        float to = top[n][i];
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) to = fmaxf(to, __shfl_xor_sync(~0u, to, x));
                        to = fmaxf(to, m[n][i]);
                        const float keep = m[n][i] == -INFINITY ? 0.f : exp2_fast(m[n][i] - to);
                        m[n][i] = to;
                        l[n][i] *= keep;
#pragma unroll
                        for (int d = 0; d < DT; d++) {
                            o[n][d][i] *= keep;
                            o[n][d][i + 2] *= keep;
                        }
                    }
            }
            uint32_t pf[NR][MT][2];
#pragma unroll
            for (int n = 0; n < NR; n++)
#pragma unroll
                for (int t = 0; t < MT; t++) {
                    const float shift[2] = {(m[n][0] == -INFINITY ? 0.f : m[n][0]) - kLift<H>, (m[n][1] == -INFINITY ? 0.f : m[n][1]) - kLift<H>};
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        s[n][t][i] = exp2_fast(s[n][t][i] - shift[i & 1]);
                        l[n][i & 1] += s[n][t][i];
                    }
                    pf[n][t][0] = transpose8(pack2<H>(s[n][t][0], s[n][t][1]));
                    pf[n][t][1] = transpose8(pack2<H>(s[n][t][2], s[n][t][3]));
                }
            // Values of positions that no row sees are taken as zero, whatever is stored there.
            uint32_t keep[MT][2];
            bool odd = false;
            if (edge) {
                auto seen = [&](int j) { return j >= any_see.x && j < any_see.y && !(S && j >= none && j < 0); };
#pragma unroll
                for (int t = 0; t < MT; t++)
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const int j = j0 + 16 * t + 8 * i + 2 * (lane & 3);
                        keep[t][i] = (seen(j) ? 0xffffu : 0u) | (seen(j + 1) ? 0xffff0000u : 0u);
                    }
                if (any_see.x != all_see.x || any_see.y != all_see.y) {  // a value that some rows see must be finite for the others
#pragma unroll 1
                    for (int c = lane; c < kSlice * D / 8; c += 32) {
                        uint32_t w[4];
                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                                     : "r"(st + c * 16));
                        bool x = false;
                        for (int i = 0; i < 4; i++) x |= any_nonfinite<H>(w[i]);
                        odd |= x && seen(j0 + (c >> 3) % kSlice);
                    }
                    odd = __any_sync(~0u, odd);
                }
            }
            if (!odd) {
#pragma unroll
                for (int d = 0; d < DT; d++)
#pragma unroll
                    for (int t = 0; t < MT; t++) {
                        uint32_t vf[4];
                        ldsm4t(vf, st + chunk_at<D, Q>(16 * t + ((lane >> 4) << 3) + (lane & 7), 2 * d + ((lane >> 3) & 1)));
                        if (edge) {
                            vf[0] &= keep[t][0];
                            vf[1] &= keep[t][0];
                            vf[2] &= keep[t][1];
                            vf[3] &= keep[t][1];
                        }
#pragma unroll
                        for (int n = 0; n < NR; n++) mma<H>(o[n][d], vf, pf[n][t][0], pf[n][t][1]);
                    }
            } else {  // row by row, over what each sees
#pragma unroll 1
                for (int k = 0; k < kSlice; k++) {
                    const int from = (k & 7) * 4 + (lane & 3);
#pragma unroll
                    for (int n = 0; n < NR; n++) {
                        float w[2];
                        bool see_k[2];
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            const float x = k & 16 ? (k & 8 ? s[n][1][2 + i] : s[n][1][i]) : (k & 8 ? s[n][0][2 + i] : s[n][0][i]);
                            w[i] = __shfl_sync(~0u, x, from);
                            see_k[i] = j0 + k >= see[n][i].x && j0 + k < see[n][i].y && !(gap >> (k >> 4) & 1) && !(S && j0 + k >= none && j0 + k < 0);
                        }
#pragma unroll
                        for (int d = 0; d < 2 * DT; d++) {
                            uint16_t x;
                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(st + chunk_at<D, Q>(k, d) + 2 * (lane >> 2)));
                            const float v = unpack2<H>(x).x;
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                float& y = o[n][d >> 1][2 * (d & 1) + i];
                                if (see_k[i]) y = fmaf(w[i], v, y);
                            }
                        }
                    }
                }
            }
        }

        if (blk + 1 < w.p1) {
            __syncwarp();
            advance();
        }
        }
        }
        {  // the end of a tile, or of this CTA's piece of it
            const int first = at.rt * kRows, rows = min(kRows, at.r.rows - first);
#pragma unroll
            for (int n = 0; n < NR; n++)
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    if (Q && up[n][i] == -INFINITY) m[n][i] = -INFINITY;
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) l[n][i] += __shfl_xor_sync(~0u, l[n][i], x);
                    if (lane < 4) {
                        s_m[warp][8 * n + 2 * lane + i] = m[n][i];
                        s_l[warp][8 * n + 2 * lane + i] = l[n][i];
                    }
                }
            __syncthreads();
            if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
            waited = true;
            const bool whole = w.whole(s_part);
            float* const piece = a.pieces + (int64_t)(2 * blockIdx.x + w.begins(s_part)) * kPieceFloats<D>;
            // N columns of a row of the tile's head `of`, whole.
            auto row_out = [&](int of, int r, int c, auto& x, float to, float sum) {
                constexpr int N = sizeof(x) / sizeof(float);
                const int tok = line.token(first + r), g = first + r - tok * a.group;
                const int64_t t = at.r.q0 + tok;
                const int h = ((at.h << hs) + of) * a.group + g;
                const int64_t row = t * a.heads + h;
                if (a.part == Part::kLeave) {
                    for (int i = 0; i < N; i += 2) *reinterpret_cast<float2*>(a.sums + row * D + c + i) = make_float2(x[i], x[i + 1]);
                    if (c == 0) leave_max<kLifted>(a, row, to, sum);
                    return;
                }
                if (a.part == Part::kJoin) {
                    float2 by = join_max<kLifted>(a, row, to, sum);
                    if constexpr (Q) {  // of two sums below 1, the half
                        by = make_float2(0.5f * by.x, 0.5f * by.y);
                        sum *= 0.5f;
                        to += 1.f;
                    }
                    join_sums<D, N>(a, row, c, by, x);
                }
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                uint32_t y[N / 2];
                for (int i = 0; i < N / 2; i++) y[i] = pack2<H>(x[2 * i] * inv, x[2 * i + 1] * inv);
                uint16_t* const to_out = a.out + t * a.out_tok + h * a.out_head + c;
                if constexpr (N == 4) *reinterpret_cast<uint2*>(to_out) = make_uint2(y[0], y[1]);
                else *reinterpret_cast<uint32_t*>(to_out) = y[0];
                if (a.lse && c == 0) a.lse[row] = log_sum<kLifted>(to, sum);
            };
            constexpr int kQuads = D / 4;
            // Each warp's sums go over its own last stage, whose next copy waits for that; eight rows at a time.
            float* const mine_o = reinterpret_cast<float*>(ring_ptr + stage * kStage);
            float by[NR][2];  // 8 bits: from what this warp's O refers to, to the row's unit
            if constexpr (Q) {
                // A thread to a row: this code runs once or twice in a CTA, and what it costs is its fetching (for each lane's rows, unrolled: 131.1
                // us instead of 128.6 for 90 requests of 21 rows behind five prefixes).
                if (tid < kRows << hs) {
                    const int of = NR == 1 ? tid / kRows : 0, r = tid - of * kRows, w0 = of * of_head;
                    float mw[kWarps], lw[kWarps], to = -INFINITY, sum = 0.f;
#pragma unroll
                    for (int w = 0; w < kWarps; w++) {
                        mw[w] = w < of_head ? s_m[w0 + w][r] : -INFINITY;
                        lw[w] = w < of_head ? s_l[w0 + w][r] : 0.f;
                        to = fmaxf(to, mw[w]);
                    }
                    const float shift = to == -INFINITY ? 0.f : to;
#pragma unroll
                    for (int w = 0; w < kWarps; w++) sum += lw[w] * exp2_fast(mw[w] - shift);
                    const float k = unit_of(to, sum);
                    s_row[tid] = make_float4(to + k, sum * power_of(-k), shift, k);
                }
                __syncthreads();
                bool far = false;
#pragma unroll
                for (int n = 0; n < NR; n++)
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const float4 row = s_row[my_head * kRows + 8 * n + 2 * (lane & 3) + i];
                        by[n][i] = m[n][i] - row.z + (c[n][i] - row.w);  // up to 127
                        far |= by[n][i] < -100.f && m[n][i] > -INFINITY;
                    }
                far = __any_sync(~0u, far);
#pragma unroll
                for (int n = 0; n < NR; n++)
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        if (far) {  // two steps, for 2^by may be far below FP32's numbers
                            const float g = exp2_fast(fminf(by[n][i] + 100.f, 0.f));
#pragma unroll
                            for (int d = 0; d < DT; d++) {
                                o[n][d][i] *= g;
                                o[n][d][i + 2] *= g;
                            }
                        }
                        by[n][i] = exp2_fast(fmaxf(by[n][i], -100.f));
                    }
            }
#pragma unroll
            for (int n = 0; n < NR; n++) {
                if (n > 0) __syncthreads();  // (the sums of the eight rows before have been read)
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const int r = 2 * (lane & 3) + i;
                    float f;
                    if constexpr (Q) {
                        f = by[n][i];
                    } else {
                        float to = s_m[my_head * of_head][8 * n + r];
                        for (int w = 1; w < of_head; w++) to = fmaxf(to, s_m[my_head * of_head + w][8 * n + r]);
                        f = exp2_fast(m[n][i] - (to == -INFINITY ? 0.f : to));
                    }
#pragma unroll
                    for (int d = 0; d < DT; d++) {
                        if constexpr (Q) {
                            *reinterpret_cast<float2*>(mine_o + sum_at(r, 16 * d + 2 * (lane >> 2))) = make_float2(o[n][d][i] * f, o[n][d][i + 2] * f);
                        } else {
                            mine_o[sum_at(r, 16 * d + (lane >> 2))] = o[n][d][i] * f;
                            mine_o[sum_at(r, 16 * d + 8 + (lane >> 2))] = o[n][d][i + 2] * f;
                        }
                    }
                }
                __syncthreads();
                for (int i = tid; i < (min(8, rows - 8 * n) << hs) * kQuads; i += kThreads) {
                    const int all = i / kQuads, r8 = all >> hs, of = all - (r8 << hs), c = 4 * (i % kQuads), r = 8 * n + r8, w0 = of * of_head, w1 = w0 + of_head;
                    float to, sum = 0.f;
                    if constexpr (Q) {
                        const float4 row = s_row[of * kRows + r];
                        to = row.x;
                        sum = row.y;
                    } else {
                        to = s_m[w0][r];
                        for (int w = w0 + 1; w < w1; w++) to = fmaxf(to, s_m[w][r]);
                    }
                    float x[4] = {};
                    for (int w = w0; w < w1; w++) {
                        const float4 y = *reinterpret_cast<const float4*>(ring_ptr + (w - warp) * kStages * kStage + stage * kStage + 4 * sum_at(r8, c));
                        x[0] += y.x;
                        x[1] += y.y;
                        x[2] += y.z;
                        x[3] += y.w;
                        if constexpr (!Q) sum += s_l[w][r] * exp2_fast(s_m[w][r] - (to == -INFINITY ? 0.f : to));
                    }
                    if (whole) {
                        row_out(of, r, c, x, to, sum);
                    } else {
                        const int pr = (r << hs) + of;
                        *reinterpret_cast<float4*>(piece + pr * D + c) = make_float4(x[0], x[1], x[2], x[3]);
                        if (c == 0) *reinterpret_cast<float2*>(piece + kMostRows * D + 2 * pr) = make_float2(to, sum);
                    }
                }
            }
            __syncthreads();
            if (!whole) {
                const int64_t c0 = divide(at.start, s_part.share), c1 = divide(at.start + at.t.blocks - 1, s_part.share);  // CTAs with a piece
                if (tid == 0) {
                    __threadfence();
                    const unsigned arrived = atomicAdd(a.tickets + c0, 1u);
                    s_last = arrived == (unsigned)(c1 - c0);
                    if (s_last) {
                        a.tickets[c0] = 0;
                        __threadfence();
                    }
                }
                __syncthreads();
                if (s_last) {
                    auto piece_of = [&](int64_t c) {
                        return a.pieces + (2 * c + (c == c0)) * kPieceFloats<D>;
                    };
                    // A warp to a row: the factors of 32 pieces at once, a piece per lane, then their sums, loads of several in
                    // flight.
                    constexpr int V = D / 32;
                    for (int r = warp; r < rows << hs; r += kWarps) {
                        float to = -INFINITY, sum = 0.f, x[V] = {};
                        for (int64_t p0 = c0; p0 <= c1; p0 += 32) {
                            const int n = (int)min((int64_t)32, c1 - p0 + 1);
                            float2 ml = make_float2(-INFINITY, 0.f);
                            if (lane < n) ml = __ldcg(reinterpret_cast<const float2*>(piece_of(p0 + lane) + kMostRows * D + 2 * r));
                            float up = ml.x;
                            for (int o = 16; o; o >>= 1) up = fmaxf(up, __shfl_xor_sync(~0u, up, o));
                            up = fmaxf(up, to);
                            const float shift = up == -INFINITY ? 0.f : up;
                            float keep = exp2_fast(to - shift), f = exp2_fast(ml.x - shift);
                            to = up;
                            float l = ml.y * f;
                            for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(~0u, l, o);
                            sum = sum * keep + l;
                            if constexpr (Q) {
                                const float k = unit_of(to, sum), by = power_of(-k);
                                sum *= by;
                                keep *= by;
                                f *= by;
                                to += k;
                            }
                            for (int i = 0; i < V; i++) x[i] *= keep;
                            for (int k0 = 0; k0 < n; k0 += kAtOnce) {
                                float y[kAtOnce][V];
#pragma unroll
                                for (int k = 0; k < kAtOnce; k++) {
                                    const float* const from = piece_of(p0 + min(k0 + k, n - 1)) + r * D + V * lane;
                                    if constexpr (V == 4) *reinterpret_cast<float4*>(y[k]) = __ldcg(reinterpret_cast<const float4*>(from));
                                    else *reinterpret_cast<float2*>(y[k]) = __ldcg(reinterpret_cast<const float2*>(from));
                                }
#pragma unroll
                                for (int k = 0; k < kAtOnce; k++) {
                                    const float fk = __shfl_sync(~0u, f, (k0 + k) & 31);
                                    for (int i = 0; i < V; i++)
                                        if (k0 + k < n) x[i] = fmaf(y[k][i], fk, x[i]);
                                }
                            }
                        }
                        row_out(r & ((1 << hs) - 1), r >> hs, V * lane, x, to, sum);
                    }
                }
            }
            w.next();
            fence_proxy_async();
            __syncwarp();
            advance();
        }
    }
    if (dead) {  // what is still in flight must land before the CTA's memory is given away
        for (int s = 0; s < kStages; s++) {
            const uint32_t bar = smem_u32(&s_bar[warp][s]), parity = phase >> s & 1;
            if ((filled >> s & 1) && !mbar_try(bar, parity)) mbar_wait_slow(bar, parity, a.wait_ns, nullptr);
        }
        if (lane == 0) atomicOr(a.err, kKvErrTimeout);
    }
    if (__any_sync(~0u, range || line.bad) && lane == 0) atomicOr(a.err, kKvErrRange);
}

template <bool H, int D, int NR, bool Q, bool S>
cudaError_t prepare() {
    return cudaFuncSetAttribute(k_kv_decode<H, D, NR, Q, S>, cudaFuncAttributeMaxDynamicSharedMemorySize, Ring<D, NR, Q>::kSmem);
}
template <bool H, int D, bool Q, bool S>
cudaError_t prepare() {
    cudaError_t e = prepare<H, D, 1, Q, S>();
    if (e == cudaSuccess) e = prepare<H, D, 2, Q, S>();
    if constexpr (Q)
        if (e == cudaSuccess) e = prepare<H, D, 3, Q, S>();
    return e;
}
template <bool Q, bool S>
cudaError_t prepare_all() {
    for (cudaError_t e : {prepare<false, 64, Q, S>(), prepare<true, 64, Q, S>(), prepare<false, 128, Q, S>(), prepare<true, 128, Q, S>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

template <bool H, int D, int NR, bool Q, bool S>
cudaError_t launch(const AttendArgs& a, const KvMaps& maps, bool early, int sms, cudaStream_t s) {
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(sms * Ring<D, NR, Q>::kCtas);
    c.blockDim = dim3(kThreads);
    c.dynamicSmemBytes = Ring<D, NR, Q>::kSmem;
    c.stream = s;
    c.attrs = at;
    c.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&c, k_kv_decode<H, D, NR, Q, S>, a, maps.k_slice, maps.v_slice);
}
template <bool H, int D, bool Q, bool S>
cudaError_t launch(const AttendArgs& a, const KvMaps& maps, int rows, bool early, int sms, cudaStream_t s) {
    if (rows <= 8) return launch<H, D, 1, Q, S>(a, maps, early, sms, s);
    if constexpr (Q)
        if (rows > 16) return launch<H, D, 3, Q, S>(a, maps, early, sms, s);
    return launch<H, D, 2, Q, S>(a, maps, early, sms, s);
}
template <bool Q, bool S>
cudaError_t launch_any(const AttendArgs& a, const KvMaps& maps, int rows, bool early, int sms, cudaStream_t s) {
    if (a.half)
        return a.head_dim == 128 ? launch<true, 128, Q, S>(a, maps, rows, early, sms, s) : launch<true, 64, Q, S>(a, maps, rows, early, sms, s);
    return a.head_dim == 128 ? launch<false, 128, Q, S>(a, maps, rows, early, sms, s) : launch<false, 64, Q, S>(a, maps, rows, early, sms, s);
}

}  // namespace

}  // namespace kvdro
