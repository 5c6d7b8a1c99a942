// Attention of few rows over pages: single tokens, drafted tokens.
//
// Bound by the bytes of the keys and values, each read once for the (at most 16) rows that share a key head.  The line of
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
#include "kv_device.cuh"

namespace kvdro {

namespace {

using namespace kv;

constexpr int kWarps = 4, kThreads = 32 * kWarps, kMostRows = 16, kSlice = 32, kKeys = kSlice * kWarps;
constexpr int kMostCtas = 4;  // per SM
constexpr int kOver = 2;      // a tile's fixed cost, in blocks (0 / 1 / 2: window case 41.3 / 40.3 / 39.6 us)
constexpr int kAtOnce = 8;    // pieces read at a time

template <int D, int NR>
struct Ring {  // a stage: K or V of a slice
    // What fits the registers and the shared memory.  Eight rows, D 128: 3 CTAs of 2 stages 95 us (64 requests), 2 of 3 stages 99;
    // D 64: 4 of 3 stages 41 us (window case), 3 of 4 stages 44, 2 of 6 stages 52.
    static constexpr int kCtas = D == 128 ? (NR == 1 ? 3 : 2) : (NR == 1 ? 4 : 2);  // per SM
    static constexpr int kBytes = kSlice * D * 2, kStages = D == 128 ? (NR == 1 ? 2 : 3) : (NR == 1 ? 3 : 6);
    static constexpr int kSmem = kWarps * kStages * kBytes + 1024;
    static_assert(Stretch<kThreads>::kScratch <= kSmem, "the ring is scratch first");
};
// A piece in global memory: rows of D sums, then their maxima and sums of weights.
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

// Byte offset of 16-byte chunk `c` of row `key` in a slice: halves of 64 elements, rows of 128 bytes whose chunks the
// tensor copy permutes by the row.
__device__ __forceinline__ uint32_t chunk_at(int key, int c) {
    return (uint32_t)((c >> 3) * (kSlice * 128) + key * 128 + (((c & 7) ^ (key & 7)) << 4));
}

// NR: groups of eight rows of a tile.
template <bool H, int D, int NR>
__global__ void __launch_bounds__(kThreads, Ring<D, NR>::kCtas)
    k_kv_decode(const AttendArgs a, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
    extern __shared__ __align__(16) char s_raw[];  // 64-bit words of the search first
    constexpr int kStages = Ring<D, NR>::kStages, kStage = Ring<D, NR>::kBytes, KS = D / 16, DT = D / 16, MT = kSlice / 16;
    constexpr int kRows = 8 * NR;
    using DecodeLine = Line<kRows, kKeys, kSlice, kOver>;
    constexpr int kRowFloats = D + 4;  // of a row of sums in shared memory: no bank conflicts
    __shared__ alignas(8) uint64_t s_bar[kWarps][kStages];
    __shared__ Stretch<kThreads> s_part;
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
    __shared__ int s_last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_u32(s_raw), ring = ((raw + 1023) & ~1023u) + warp * kStages * kStage;
    char* const ring_ptr = s_raw + (ring - raw);
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
        return;
    }

    // Units in the order K, V of a slice, K, V of the next.
    Walk<DecodeLine> in(line, s_part), w = in;  // of the copies, and of the sums
    int in_blk = in.p0;
    bool in_v = false;
    int fetched = 0;

    // Page numbers of this warp's slices of 32 blocks, one per lane; a slice has two pages if they have 16 slots.
    const int slots = min(kSlice, 1 << a.page_shift);
    int pg[2] = {-1, -1}, pg_b = -1, pg_rt = -1, pg_blk = -1;
    bool range = false;
    uint32_t filled = 0, phase = 0;  // by stage: holds a slice; the parity to wait for
    uint32_t gaps = 0;               // by stage, two bits: 16 positions whose page number is none
    auto fetch = [&](int stage) {
        filled &= ~(1u << stage);
        if (!in.more) return;
        if (in.at.b != pg_b || in.at.rt != pg_rt || (in_blk >> 5) != pg_blk) {
            pg_b = in.at.b;
            pg_rt = in.at.rt;
            pg_blk = in_blk >> 5;
            const int j = in.at.t.lo + ((in_blk & ~31) + lane) * kKeys + warp * kSlice;
            const int seen_lo = line.seen(in.at.r, line.token(in.at.rt * kRows)).x;
#pragma unroll
            for (int i = 0; i < 2; i++) {
                pg[i] = -1;
                if (j + 16 * i < in.at.t.hi && ((j + 16 * i) | (slots - 1)) >= seen_lo) {  // else no row's business
                    const int page = a.table[(int64_t)in.at.b * a.max_pages + ((j + 16 * i) >> a.page_shift)];
                    if ((uint32_t)page < (uint32_t)a.n_pages) pg[i] = page;
                    else range = true;
                }
            }
        }
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
    for (int s = 0; s < kStages; s++) fetch(s);

    const float mul = a.cap > 0.f ? 2.f * kLog2e * a.scale / a.cap : kLog2e * a.scale, cap2 = a.cap * kLog2e;
    uint32_t qf[NR][KS][2];
    float o[NR][DT][4];
    float m[NR][2], l[NR][2];  // of rows 8 n + 2 (lane & 3) + i
    int2 see[NR][2];
    int2 all_see, any_see;  // positions that every row of the tile sees, and that some row does
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
        if (!dead) fetch(stage);
        stage = stage + 1 == kStages ? 0 : stage + 1;
    };

    while (w.more) {
        Cursor& at = w.at;
        {  // a tile begins here, or this CTA's piece of it
            const int first = at.rt * kRows, rows = min(kRows, at.r.rows - first);
#pragma unroll
            for (int n = 0; n < NR; n++) {
                {
                    const int r = first + min(8 * n + (lane >> 2), rows - 1), tok = line.token(r), g = r - tok * a.group;
                    const uint16_t* const q = a.q + (int64_t)(at.r.q0 + tok) * a.q_tok + (int64_t)(at.h * a.group + g) * a.q_head + 2 * (lane & 3);
#pragma unroll
                    for (int k = 0; k < KS; k++) {
                        qf[n][k][0] = *reinterpret_cast<const uint32_t*>(q + k * 16);
                        qf[n][k][1] = *reinterpret_cast<const uint32_t*>(q + k * 16 + 8);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    see[n][i] = line.seen(at.r, line.token(first + min(8 * n + 2 * (lane & 3) + i, rows - 1)));
                    m[n][i] = -INFINITY;
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
        }
        for (int blk = w.p0; blk < w.p1; blk++) {
        const int j0 = at.t.lo + blk * kKeys + warp * kSlice;
        const bool edge = j0 < all_see.x || j0 + kSlice > all_see.y || (gaps >> 2 * stage & 3);
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
                    ldsm4(kf, st + chunk_at(16 * t + (lane & 15), 2 * k + (lane >> 4)));
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
                            if (j < see[n][i & 1].x || j >= see[n][i & 1].y || (gap >> t & 1)) x = -INFINITY;
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
                auto seen = [&](int j) { return j >= any_see.x && j < any_see.y; };
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
                        ldsm4t(vf, st + chunk_at(16 * t + ((lane >> 4) << 3) + (lane & 7), 2 * d + ((lane >> 3) & 1)));
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
                            see_k[i] = j0 + k >= see[n][i].x && j0 + k < see[n][i].y && !(gap >> (k >> 4) & 1);
                        }
#pragma unroll
                        for (int d = 0; d < 2 * DT; d++) {
                            uint16_t x;
                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(st + chunk_at(k, d) + 2 * (lane >> 2)));
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
        {  // the end of a tile, or of this CTA's piece of it
            const int first = at.rt * kRows, rows = min(kRows, at.r.rows - first);
#pragma unroll
            for (int n = 0; n < NR; n++)
#pragma unroll
                for (int i = 0; i < 2; i++) {
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) l[n][i] += __shfl_xor_sync(~0u, l[n][i], x);
                    if (lane < 4) {
                        s_m[warp][8 * n + 2 * lane + i] = m[n][i];
                        s_l[warp][8 * n + 2 * lane + i] = l[n][i];
                    }
                }
            __syncthreads();
            const bool whole = w.whole(s_part);
            float* const piece = a.pieces + (int64_t)(2 * blockIdx.x + w.begins(s_part)) * kPieceFloats<D>;
            auto row_out = [&](int r, int c, float4 x, float to, float sum) {
                const int tok = line.token(first + r), g = first + r - tok * a.group;
                const int64_t t = at.r.q0 + tok;
                const int h = at.h * a.group + g;
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                *reinterpret_cast<uint2*>(a.out + t * a.out_tok + h * a.out_head + c) =
                    make_uint2(pack2<H>(x.x * inv, x.y * inv), pack2<H>(x.z * inv, x.w * inv));
                if (a.lse && c == 0) a.lse[t * a.heads + h] = log_sum<H>(to, sum);
            };
            constexpr int kQuads = D / 4;
            // Each warp's sums go over its own last stage, whose next copy waits for that; eight rows at a time.
            float* const mine_o = reinterpret_cast<float*>(ring_ptr + stage * kStage);
#pragma unroll
            for (int n = 0; n < NR; n++) {
                if (n > 0) __syncthreads();
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const int r = 2 * (lane & 3) + i;
                    float to = s_m[0][8 * n + r];
                    for (int w = 1; w < kWarps; w++) to = fmaxf(to, s_m[w][8 * n + r]);
                    const float f = exp2_fast(m[n][i] - (to == -INFINITY ? 0.f : to));
#pragma unroll
                    for (int d = 0; d < DT; d++) {
                        mine_o[r * kRowFloats + 16 * d + (lane >> 2)] = o[n][d][i] * f;
                        mine_o[r * kRowFloats + 16 * d + 8 + (lane >> 2)] = o[n][d][i + 2] * f;
                    }
                }
                __syncthreads();
                for (int i = tid; i < min(8, rows - 8 * n) * kQuads; i += kThreads) {
                    const int r8 = i / kQuads, c = 4 * (i % kQuads), r = 8 * n + r8;
                    float to = s_m[0][r], sum = 0.f;
                    for (int w = 1; w < kWarps; w++) to = fmaxf(to, s_m[w][r]);
                    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int w = 0; w < kWarps; w++) {
                        const float4 y = *reinterpret_cast<const float4*>(ring_ptr + (w - warp) * kStages * kStage + stage * kStage +
                                                                          4 * (r8 * kRowFloats + c));
                        x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
                        sum += s_l[w][r] * exp2_fast(s_m[w][r] - (to == -INFINITY ? 0.f : to));
                    }
                    if (whole) {
                        row_out(r, c, x, to, sum);
                    } else {
                        *reinterpret_cast<float4*>(piece + r * D + c) = x;
                        if (c == 0) *reinterpret_cast<float2*>(piece + kMostRows * D + 2 * r) = make_float2(to, sum);
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
                    for (int r = warp; r < rows; r += kWarps) {
                        float to = -INFINITY, sum = 0.f, x[V] = {};
                        for (int64_t p0 = c0; p0 <= c1; p0 += 32) {
                            const int n = (int)min((int64_t)32, c1 - p0 + 1);
                            float2 ml = make_float2(-INFINITY, 0.f);
                            if (lane < n) ml = __ldcg(reinterpret_cast<const float2*>(piece_of(p0 + lane) + kMostRows * D + 2 * r));
                            float up = ml.x;
                            for (int o = 16; o; o >>= 1) up = fmaxf(up, __shfl_xor_sync(~0u, up, o));
                            up = fmaxf(up, to);
                            const float shift = up == -INFINITY ? 0.f : up, keep = exp2_fast(to - shift), f = exp2_fast(ml.x - shift);
                            to = up;
                            float l = ml.y * f;
                            for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(~0u, l, o);
                            sum = sum * keep + l;
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
                        const int tok = line.token(first + r), g = first + r - tok * a.group, h = at.h * a.group + g;
                        const int64_t t = at.r.q0 + tok;
                        const float inv = sum == 0.f ? 0.f : 1.f / sum;
                        uint32_t* const to_out = reinterpret_cast<uint32_t*>(a.out + t * a.out_tok + h * a.out_head + V * lane);
                        for (int i = 0; i < V; i += 2) to_out[i / 2] = pack2<H>(x[i] * inv, x[i + 1] * inv);
                        if (a.lse && lane == 0) a.lse[t * a.heads + h] = log_sum<H>(to, sum);
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

template <bool H, int D, int NR>
cudaError_t prepare() {
    return cudaFuncSetAttribute(k_kv_decode<H, D, NR>, cudaFuncAttributeMaxDynamicSharedMemorySize, Ring<D, NR>::kSmem);
}
template <bool H, int D>
cudaError_t prepare() {
    const cudaError_t e = prepare<H, D, 1>();
    return e == cudaSuccess ? prepare<H, D, 2>() : e;
}

template <bool H, int D>
cudaError_t launch(const AttendArgs& a, const KvMaps& maps, bool eight, int sms, cudaStream_t s) {
    if (eight) k_kv_decode<H, D, 1><<<sms * Ring<D, 1>::kCtas, kThreads, Ring<D, 1>::kSmem, s>>>(a, maps.k_slice, maps.v_slice);
    else k_kv_decode<H, D, 2><<<sms * Ring<D, 2>::kCtas, kThreads, Ring<D, 2>::kSmem, s>>>(a, maps.k_slice, maps.v_slice);
    return cudaGetLastError();
}

}  // namespace

size_t kv_decode_piece_bytes(int sms) { return (size_t)sms * kMostCtas * 2 * kPieceFloats<128> * sizeof(float); }
int kv_decode_ctas(int sms) { return sms * kMostCtas; }

cudaError_t kv_decode_prepare() {
    cudaError_t e;
    if ((e = prepare<false, 64>()) != cudaSuccess || (e = prepare<true, 64>()) != cudaSuccess ||
        (e = prepare<false, 128>()) != cudaSuccess)
        return e;
    return prepare<true, 128>();
}

cudaError_t launch_kv_decode(const AttendArgs& a, const KvMaps& maps, bool eight, int sms, cudaStream_t s) {
    if (a.half) return a.head_dim == 128 ? launch<true, 128>(a, maps, eight, sms, s) : launch<true, 64>(a, maps, eight, sms, s);
    return a.head_dim == 128 ? launch<false, 128>(a, maps, eight, sms, s) : launch<false, 64>(a, maps, eight, sms, s);
}

}  // namespace kvdro
