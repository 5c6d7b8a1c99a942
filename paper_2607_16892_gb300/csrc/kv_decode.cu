// Attention of few rows over pages: single tokens, drafted tokens.
//
// Bound by the bytes of the keys and values, each read once for the (at most 16) rows that share a key head.  The line of
// all blocks of 64 positions is dealt to two CTAs per SM (kv_device.cuh); in a block each of a CTA's four warps has 16
// positions of its own, with its own ring of tensor copies, running maxima, sums and weighted sums: nothing
// in the loop waits for another warp.  The warps are joined through shared memory at the end of a tile, pieces of a tile
// through global memory by the CTA that arrives last, both in a fixed order.
//
// Products run on mma.m16n8k16: a tcgen05 tile has 128 rows, and a slice's 32 mma take far less than its copy.  The weights are
// rounded to the cache's type for the second product, which adds about as much error as the result's own rounding.
#include "kv_device.cuh"

namespace kvdro {

namespace {

using namespace kv;

constexpr int kWarps = 4, kThreads = 32 * kWarps, kRows = 16, kSlice = 16, kKeys = kSlice * kWarps, kStages = 3;
constexpr int kCtasPerSm = 2;

template <int D>
constexpr int kStageBytes = 2 * kSlice * D * 2;
template <int D>
constexpr int kSmemBytes = kWarps * kStages * kStageBytes<D> + 1024;
// A piece in global memory: kRows rows of D sums, then their maxima and sums of weights.
template <int D>
constexpr int kPieceFloats = kRows * (D + 2);

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

using DecodeLine = Line<kRows, kKeys, kSlice>;

template <bool H, int D>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
    k_kv_decode(const AttendArgs a, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
    extern __shared__ char s_raw[];
    __shared__ alignas(8) uint64_t s_bar[kWarps][kStages];
    __shared__ int64_t s_base, s_warp_sum[kWarps];  // where the requests of thread `s_found` begin in the line
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
    __shared__ int s_found, s_last;
    constexpr int kStage = kStageBytes<D>, kHalf = kStage / 2, KS = D / 16, NT = D / 8;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_u32(s_raw), ring = ((raw + 1023) & ~1023u) + warp * kStages * kStage;
    char* const ring_ptr = s_raw + (ring - raw);
    DecodeLine line(a);

    if (lane < kStages) mbar_init(smem_u32(&s_bar[warp][lane]), 1);
    fence_mbar_init();

    // The line's length, and where each thread's requests begin in it.
    const int per = (a.B + kThreads - 1) / kThreads;
    int64_t mine = 0;
    for (int b = min(tid * per, a.B), b1 = min(b + per, a.B); b < b1; b++) mine += line.cost(line.request(b));
    int64_t incl = mine;
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(~0u, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) s_warp_sum[warp] = incl;
    __syncthreads();
    int64_t before = 0, total = 0;
    for (int w = 0; w < kWarps; w++) {
        if (w == warp) before = total;
        total += s_warp_sum[w];
    }
    before += incl - mine;
    const int64_t share = max((int64_t)1, (total + gridDim.x - 1) / gridDim.x);
    const int64_t u0 = blockIdx.x * share, u1 = min(u0 + share, total);
    if (u0 >= before && u0 < before + mine) {
        s_found = tid;
        s_base = before;
    }
    __syncthreads();

    // Tokens of no request: out = 0.
    {
        const int end = max(0, min(a.q_off[a.B], a.T));
        const int64_t vecs = (int64_t)(a.T - end) * a.heads * (D / 8);
        for (int64_t i = (int64_t)blockIdx.x * kThreads + tid; i < vecs; i += (int64_t)gridDim.x * kThreads) {
            const int64_t row = i / (D / 8);
            const int t = end + (int)(row / a.heads), h = (int)(row % a.heads), c = (int)(i % (D / 8));
            *reinterpret_cast<uint4*>(a.out + t * a.out_tok + h * a.out_head + c * 8) = make_uint4(0, 0, 0, 0);
            if (a.lse && c == 0) a.lse[(int64_t)t * a.heads + h] = -INFINITY;
        }
    }
    if (u0 >= u1) {
        if (line.bad && tid == 0) atomicOr(a.err, kKvErrRange);
        return;
    }

    Cursor<DecodeLine> in, at;  // of the copies, and of the sums
    in.seek(line, s_found * per, s_base, u0);
    at = in;
    int in_blk = (int)(u0 - in.start), in_left = (int)(u1 - u0);

    // Page numbers of this warp's slices of 32 blocks, one per lane.
    int pg = -1, pg_b = -1, pg_rt = -1, pg_blk = -1;
    bool range = false;
    uint32_t filled = 0, phase = 0;  // by stage: holds a slice; the parity to wait for
    auto fetch = [&](int stage) {
        if (in_left == 0) {
            filled &= ~(1u << stage);
            return;
        }
        if (in.b != pg_b || in.rt != pg_rt || (in_blk >> 5) != pg_blk) {
            pg_b = in.b;
            pg_rt = in.rt;
            pg_blk = in_blk >> 5;
            const int j = in.t.lo + ((in_blk & ~31) + lane) * kKeys + warp * kSlice;
            pg = -1;
            if (j < in.t.hi) {
                pg = a.table[(int64_t)in.b * a.max_pages + (j >> a.page_shift)];
                if ((uint32_t)pg >= (uint32_t)a.n_pages) {
                    pg = -1;
                    range = true;
                }
            }
        }
        const int page = __shfl_sync(~0u, pg, in_blk & 31);
        if (page >= 0) {
            if (lane == 0) {
                const int slot = (in.t.lo + in_blk * kKeys + warp * kSlice) & ((1 << a.page_shift) - 1);
                const uint32_t bar = smem_u32(&s_bar[warp][stage]), to = ring + stage * kStage;
                mbar_expect(bar, kStage);
#pragma unroll
                for (int d = 0; d < D / 64; d++) {
                    load_box(to + d * (kSlice * 128), &kmap, d * 64, slot, in.h, page, bar);
                    load_box(to + kHalf + d * (kSlice * 128), &vmap, d * 64, slot, in.h, page, bar);
                }
            }
            filled |= 1u << stage;
        } else {
            filled &= ~(1u << stage);
        }
        in_left--;
        if (++in_blk == in.t.blocks && in_left) {
            in.next(line);
            in_blk = 0;
        }
    };
#pragma unroll
    for (int s = 0; s < kStages; s++) fetch(s);

    const float mul = a.cap > 0.f ? 2.f * kLog2e * a.scale / a.cap : kLog2e * a.scale, cap2 = a.cap * kLog2e;
    const int r_lo = lane >> 2, r_hi = r_lo + 8;  // this thread's rows
    uint32_t qf[KS][4];
    float o[NT][4];
    float m[2], l[2];
    int2 see[2];
    int2 all_see;  // positions that every row sees
    bool alike = true;  // every row sees the same
    bool dead = false;
    int stage = 0, blk = (int)(u0 - at.start);
    bool fresh = true;

    for (int64_t u = u0; u < u1; u++) {
        if (fresh) {  // a tile begins here, or this CTA's piece of it
            fresh = false;
            const int first = at.rt * kRows, rows = min(kRows, at.r.rows - first);
            const uint16_t* qp[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const int r = first + min(i ? r_hi : r_lo, rows - 1), tok = r / a.group, g = r - tok * a.group;
                qp[i] = a.q + (int64_t)(at.r.q0 + tok) * a.q_tok + (int64_t)(at.h * a.group + g) * a.q_head;
                see[i] = line.seen(at.r, tok);
                m[i] = -INFINITY;
                l[i] = 0.f;
            }
            const int2 s0 = line.seen(at.r, first / a.group), s1 = line.seen(at.r, (first + rows - 1) / a.group);
            all_see = make_int2(s1.x, s0.y);
            alike = s0.x == s1.x && s0.y == s1.y;
#pragma unroll
            for (int k = 0; k < KS; k++) {
                const int c = k * 16 + 2 * (lane & 3);
                qf[k][0] = *reinterpret_cast<const uint32_t*>(qp[0] + c);
                qf[k][1] = *reinterpret_cast<const uint32_t*>(qp[1] + c);
                qf[k][2] = *reinterpret_cast<const uint32_t*>(qp[0] + c + 8);
                qf[k][3] = *reinterpret_cast<const uint32_t*>(qp[1] + c + 8);
            }
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int i = 0; i < 4; i++) o[n][i] = 0.f;
        }
        const uint32_t st = ring + stage * kStage;
        if ((filled >> stage & 1) && !dead) {
            if (__all_sync(~0u, mbar_wait(smem_u32(&s_bar[warp][stage]), phase >> stage & 1))) phase ^= 1u << stage;
            else dead = true;
        }
        if ((filled >> stage & 1) && !dead) {
            const int j0 = at.t.lo + blk * kKeys + warp * kSlice;
            const bool edge = j0 < all_see.x || j0 + kSlice > all_see.y;
            float s[2][4] = {};
#pragma unroll
            for (int k = 0; k < KS; k++) {
                uint32_t kf[4];
                ldsm4(kf, st + chunk_at((lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)));
                mma<H>(s[0], qf[k], kf[0], kf[1]);
                mma<H>(s[1], qf[k], kf[2], kf[3]);
            }
#pragma unroll
            for (int n = 0; n < 2; n++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    s[n][i] = score(s[n][i], mul, cap2);
                    if (edge) {
                        const int j = j0 + 8 * n + 2 * (lane & 3) + (i & 1);
                        if (j < see[i >> 1].x || j >= see[i >> 1].y) s[n][i] = -INFINITY;
                    }
                }
            float top[2];
            bool grows = false;
#pragma unroll
            for (int i = 0; i < 2; i++) {
                top[i] = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1]));
                top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], 2));
                top[i] = fmaxf(top[i], m[i]);
                grows |= top[i] > m[i];
            }
            if (__any_sync(~0u, grows)) {
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const float keep = m[i] == -INFINITY ? 0.f : exp2_fast(m[i] - top[i]);
                    m[i] = top[i];
                    l[i] *= keep;
#pragma unroll
                    for (int n = 0; n < NT; n++) {
                        o[n][2 * i] *= keep;
                        o[n][2 * i + 1] *= keep;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float shift = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
                for (int n = 0; n < 2; n++)
#pragma unroll
                    for (int c = 0; c < 2; c++) {
                        s[n][2 * i + c] = exp2_fast(s[n][2 * i + c] - shift);
                        l[i] += s[n][2 * i + c];
                    }
            }
            uint32_t pf[4];
#pragma unroll
            for (int i = 0; i < 4; i++) pf[i] = pack2<H>(s[i >> 1][2 * (i & 1)], s[i >> 1][2 * (i & 1) + 1]);
            // Values of positions that no row sees are taken as zero, whatever is stored there.
            uint32_t keep0 = ~0u, keep1 = ~0u;
            bool odd = false;
            if (edge) {
                const int j = j0 + 2 * (lane & 3);
                auto in_tile = [&](int x) {
                    const int lo = alike ? all_see.x : at.t.lo, hi = alike ? all_see.y : at.t.hi;
                    return x >= lo && x < hi;
                };
                keep0 = (in_tile(j) ? 0xffffu : 0u) | (in_tile(j + 1) ? 0xffff0000u : 0u);
                keep1 = (in_tile(j + 8) ? 0xffffu : 0u) | (in_tile(j + 9) ? 0xffff0000u : 0u);
                if (!alike) {  // a value that some rows see must be finite for the others
#pragma unroll 1
                    for (int c = lane; c < kSlice * D / 8; c += 32) {
                        uint32_t w[4];
                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                                     : "r"(st + kHalf + c * 16));
                        for (int i = 0; i < 4; i++) odd |= any_nonfinite<H>(w[i]);
                    }
                    odd = __any_sync(~0u, odd);
                }
            }
            if (!odd) {
#pragma unroll
                for (int n = 0; n < NT; n += 2) {
                    uint32_t vf[4];
                    ldsm4t(vf, st + kHalf + chunk_at((lane & 7) + (((lane >> 3) & 1) << 3), n + (lane >> 4)));
                    if (edge) {
                        vf[0] &= keep0;
                        vf[1] &= keep1;
                        vf[2] &= keep0;
                        vf[3] &= keep1;
                    }
                    mma<H>(o[n], pf, vf[0], vf[1]);
                    mma<H>(o[n + 1], pf, vf[2], vf[3]);
                }
            } else {  // row by row, over what each sees
#pragma unroll 1
                for (int k = 0; k < kSlice; k++) {
                    const int from = (lane & ~3) + ((k & 7) >> 1);
                    float w[2];
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const float x = k & 8 ? (k & 1 ? s[1][2 * i + 1] : s[1][2 * i]) : (k & 1 ? s[0][2 * i + 1] : s[0][2 * i]);
                        w[i] = __shfl_sync(~0u, x, from);
                    }
                    const bool v0 = j0 + k >= see[0].x && j0 + k < see[0].y, v1 = j0 + k >= see[1].x && j0 + k < see[1].y;
#pragma unroll
                    for (int n = 0; n < NT; n++) {
                        uint32_t x;
                        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(st + kHalf + chunk_at(k, n) + 4 * (lane & 3)));
                        const float2 v = unpack2<H>(x);
                        if (v0) {
                            o[n][0] = fmaf(w[0], v.x, o[n][0]);
                            o[n][1] = fmaf(w[0], v.y, o[n][1]);
                        }
                        if (v1) {
                            o[n][2] = fmaf(w[1], v.x, o[n][2]);
                            o[n][3] = fmaf(w[1], v.y, o[n][3]);
                        }
                    }
                }
            }
        }

        blk++;
        if (blk == at.t.blocks || u + 1 == u1) {  // the end of a tile, or of this CTA's piece of it
            const int first = at.rt * kRows, rows = min(kRows, at.r.rows - first);
#pragma unroll
            for (int i = 0; i < 2; i++) {
                l[i] += __shfl_xor_sync(~0u, l[i], 1);
                l[i] += __shfl_xor_sync(~0u, l[i], 2);
                if ((lane & 3) == 0) {
                    s_m[warp][i ? r_hi : r_lo] = m[i];
                    s_l[warp][i ? r_hi : r_lo] = l[i];
                }
            }
            __syncthreads();
            // Each warp's sums go over its own last stage, whose next copy waits for that.
            float* const mine_o = reinterpret_cast<float*>(ring_ptr + stage * kStage);
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const int r = i ? r_hi : r_lo;
                float to = s_m[0][r];
                for (int w = 1; w < kWarps; w++) to = fmaxf(to, s_m[w][r]);
                const float f = exp2_fast(m[i] - (to == -INFINITY ? 0.f : to));
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    const int c = (8 * n + 2 * (lane & 3)) ^ ((r & 3) << 3);
                    *reinterpret_cast<float2*>(mine_o + r * D + c) = make_float2(o[n][2 * i] * f, o[n][2 * i + 1] * f);
                }
            }
            __syncthreads();
            const int64_t c0 = at.start / share, c1 = (at.start + at.t.blocks - 1) / share;  // CTAs with a piece
            const int cta = blockIdx.x;
            float* const piece = a.pieces + (int64_t)(2 * cta + (c0 == cta)) * kPieceFloats<D>;
            auto row_out = [&](int r, int c, float4 x, float to, float sum) {
                const int tok = (first + r) / a.group, g = first + r - tok * a.group;
                const int64_t t = at.r.q0 + tok;
                const int h = at.h * a.group + g;
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                *reinterpret_cast<uint2*>(a.out + t * a.out_tok + h * a.out_head + c) =
                    make_uint2(pack2<H>(x.x * inv, x.y * inv), pack2<H>(x.z * inv, x.w * inv));
                if (a.lse && c == 0) a.lse[t * a.heads + h] = sum == 0.f ? -INFINITY : kLn2 * (to + log2f(sum));
            };
            constexpr int kQuads = D / 4;
            for (int i = tid; i < rows * kQuads; i += kThreads) {
                const int r = i / kQuads, c = 4 * (i % kQuads);
                float to = s_m[0][r], sum = 0.f;
                for (int w = 1; w < kWarps; w++) to = fmaxf(to, s_m[w][r]);
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int w = 0; w < kWarps; w++) {
                    const float4 y = *reinterpret_cast<const float4*>(ring_ptr + (w - warp) * kStages * kStage + stage * kStage +
                                                                      4 * (r * D + (c ^ ((r & 3) << 3))));
                    x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
                    sum += s_l[w][r] * exp2_fast(s_m[w][r] - (to == -INFINITY ? 0.f : to));
                }
                if (c0 == c1) {
                    row_out(r, c, x, to, sum);
                } else {
                    *reinterpret_cast<float4*>(piece + r * D + c) = x;
                    if (c == 0) *reinterpret_cast<float2*>(piece + kRows * D + 2 * r) = make_float2(to, sum);
                }
            }
            __syncthreads();
            if (c0 != c1) {
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
                    for (int i = tid; i < rows * kQuads; i += kThreads) {
                        const int r = i / kQuads, c = 4 * (i % kQuads);
                        float to = -INFINITY, sum = 0.f;
                        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                        for (int64_t p = c0; p <= c1; p++) {
                            const float2 ml = __ldcg(reinterpret_cast<const float2*>(piece_of(p) + kRows * D + 2 * r));
                            const float4 y = __ldcg(reinterpret_cast<const float4*>(piece_of(p) + r * D + c));
                            const float up = fmaxf(to, ml.x), shift = up == -INFINITY ? 0.f : up;
                            const float f = exp2_fast(to - shift), g = exp2_fast(ml.x - shift);
                            x = make_float4(x.x * f + y.x * g, x.y * f + y.y * g, x.z * f + y.z * g, x.w * f + y.w * g);
                            sum = sum * f + ml.y * g;
                            to = up;
                        }
                        row_out(r, c, x, to, sum);
                    }
                }
            }
            fence_proxy_async();
            __syncwarp();
            if (u + 1 < u1) {
                at.next(line);
                blk = 0;
                fresh = true;
            }
        }
        if (!dead) fetch(stage);
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    if (dead) {  // what is still in flight must land before the CTA's memory is given away
        for (int s = 0; s < kStages; s++)
            if (filled >> s & 1) mbar_wait(smem_u32(&s_bar[warp][s]), phase >> s & 1);
        if (lane == 0) atomicOr(a.err, kKvErrTimeout);
    }
    if (__any_sync(~0u, range || line.bad) && lane == 0) atomicOr(a.err, kKvErrRange);
}

template <bool H, int D>
cudaError_t prepare() {
    return cudaFuncSetAttribute(k_kv_decode<H, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes<D>);
}

template <bool H, int D>
cudaError_t launch(const AttendArgs& a, const KvMaps& maps, int sms, cudaStream_t s) {
    k_kv_decode<H, D><<<sms * kCtasPerSm, kThreads, kSmemBytes<D>, s>>>(a, maps.k16, maps.v16);
    return cudaGetLastError();
}

}  // namespace

size_t kv_decode_piece_bytes(int sms) { return (size_t)sms * kCtasPerSm * 2 * kPieceFloats<128> * sizeof(float); }
int kv_decode_ctas(int sms) { return sms * kCtasPerSm; }

cudaError_t kv_decode_prepare() {
    cudaError_t e;
    if ((e = prepare<false, 64>()) != cudaSuccess || (e = prepare<true, 64>()) != cudaSuccess ||
        (e = prepare<false, 128>()) != cudaSuccess)
        return e;
    return prepare<true, 128>();
}

cudaError_t launch_kv_decode(const AttendArgs& a, const KvMaps& maps, int sms, cudaStream_t s) {
    if (a.half) return a.head_dim == 128 ? launch<true, 128>(a, maps, sms, s) : launch<true, 64>(a, maps, sms, s);
    return a.head_dim == 128 ? launch<false, 128>(a, maps, sms, s) : launch<false, 64>(a, maps, sms, s);
}

}  // namespace kvdro
