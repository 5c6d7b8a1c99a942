// Device code shared by the page cache's attention kernels: 16-bit types, barriers and tensor copies, and the
// division of the work among CTAs.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv.cuh"

namespace kvdro {
namespace kv {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <bool H>
__device__ __forceinline__ uint32_t pack2(float x, float y) {  // x in the low half
    if constexpr (H) {
        const __half2 r = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&r);
    } else {
        const __nv_bfloat162 r = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&r);
    }
}
template <bool H>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
    if constexpr (H) return __half22float2(*reinterpret_cast<__half2*>(&w));
    else return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&w));
}
// Weights are 2^(s - m + kLift), and so are their sums.  FP16 has no weights below 2^-25, and 32768 of them may be a result's
// whole component: 2^7 moves that to 2^-32 of the row's largest, while the largest stays at or below 2^15 (m is raised
// when a row's maximum passes it by more than kRaise).  BF16 has FP32's exponents.
template <bool H>
constexpr float kLift = H ? 7.f : 0.f;
constexpr float kRaise = 8.f;
// Whether a maximum asks for m to be raised to it.  With FP16 every greater one does where scores are spaced by 1/8 and more: rounded
// differences of 8 may be 9, and 2^16 is an infinity.
template <bool H>
__device__ __forceinline__ bool raises(float top, float m) {
    const float slack = H && fabsf(top) > 0x1p20f ? 0.f : kRaise;
    return top > m + slack || (m == -INFINITY && top > m);
}
// The log sum of a row (natural), from the m that its sum refers to.
template <bool H>
__device__ __forceinline__ float log_sum(float m, float sum) {
    return sum == 0.f ? -INFINITY : kLn2 * (m + (log2f(sum) - kLift<H>));
}

// Whether either half is an infinity or NaN: all exponent bits set, so that one more carries into the sign's place.
template <bool H>
__device__ __forceinline__ bool any_nonfinite(uint32_t w) {
    constexpr uint32_t exponent = H ? 0x7c007c00u : 0x7f807f80u, one = H ? 0x04000400u : 0x00800080u;
    return ((w & exponent) + one) & 0x80008000u;
}

// 2^x.  Relative error 2^-22; 0 at -infinity.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// A score times log2(e), through the cap if there is one: cap tanh(y / cap) = cap (1 - 2 / (1 + exp(2 y / cap))), off by
// 2^-20 of cap at most: 2^-22 of a quotient of up to 2 from the division, 2^-24 of it from its sum, 2^-23 and 2^-24 from the
// exponential and its argument, 2^-24 from the difference.  `mul` is scale * log2(e), or 2 log2(e) scale / cap; `cap2` is cap * log2(e).
__device__ __forceinline__ float score(float dot, float mul, float cap2) {
    const float y = dot * mul;
    if (cap2 == 0.f) return y;
    return fmaf(-2.f * cap2, __fdividef(1.f, 1.f + exp2_fast(y)), cap2);
}

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void fence_mbar_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Waits for a phase, for `limit` ns of the GPU's timer at most (and, where that is long, 2^14 polls made while running);
// ends at once where `dead` (if there is one) says that another wait ran out.  False, and `dead` set, if it ran out.
static __device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity, unsigned long long limit, volatile int* dead) {
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    const unsigned least = limit > 100000000ull ? 1u << 14 : 16u;
    for (unsigned polls = 0; polls < (1u << 28); polls++) {
        if (mbar_try(bar, parity)) return true;
        if (dead && *dead) return false;
        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
        if (polls > least && t - t0 > limit) break;
    }
    if (dead) *dead = 1;
    return false;
}

// One lane of a whole warp, the same every time: what it issues takes its operands from uniform registers.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// A box of one page: coordinates d, slot, head, page.  Out-of-range pages read as zeros.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int d, int slot, int head, int page, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(map), "r"(d), "r"(slot), "r"(head), "r"(page), "r"(bar)
        : "memory");
}

// The requests' rows are dealt to tiles of `kRows` rows (a token's query heads of one key head are neighbours), and a tile's
// positions to blocks of `kKeys`.  All blocks of all tiles stand in one line -- request, row tile, key head, block --
// with kOver more places behind a tile's last block for what a tile costs beside its blocks (its Q, its results), and each
// CTA takes an equal stretch of the line, so that long contexts are shared by many CTAs and short ones share a CTA.
// A tile that crosses from one stretch into the next is joined from its pieces.
struct Request {
    int q0, n, rows, kv;  // first token, tokens, rows (tokens inside T times the group; 0: no positions, or not this launch's), positions
};

struct Tile {
    int lo, hi, blocks;  // positions [lo, hi), lo aligned
};

template <int kRowsOf, int kKeysOf, int kAlign, int kOverOf>
struct Line {
    static constexpr int kRows = kRowsOf, kKeys = kKeysOf, kOver = kOverOf;
    const AttendArgs& a;
    bool bad = false;

    __device__ __forceinline__ explicit Line(const AttendArgs& args) : a(args) {}

    __device__ __forceinline__ int token(int row) const { return (int)(((uint64_t)(uint32_t)row * a.group_mul) >> a.group_shift); }
    __device__ __forceinline__ Request request(int b) {
        Request r;
        r.q0 = a.q_off[b];
        const int q1 = a.q_off[b + 1];
        r.kv = a.kv_len[b];
        if (r.q0 < 0 || q1 < r.q0) {
            bad = true;
            r.q0 = r.n = r.rows = 0;
            return r;
        }
        r.n = q1 - r.q0;
        if (r.kv < 0 || (int64_t)r.kv > ((int64_t)a.max_pages << a.page_shift)) {
            bad = true;
            r.kv = 0;
        }
        r.rows = r.kv > 0 && r.n > a.min_q && r.n <= a.max_q ? max(0, min(q1, a.T) - r.q0) * a.group : 0;
        return r;
    }
    // Visible positions [lo, hi) of token i of a request.
    __device__ __forceinline__ int2 seen(const Request& r, int i) const {
        const int p = r.kv - r.n + i;  // kv and n are below 2^31, not negative
        const int hi = a.causal ? min(max(p + 1, 0), r.kv) : r.kv;
        const int lo = a.window > 0 && p >= a.window ? p - a.window + 1 : 0;
        return make_int2(min(lo, hi), hi);
    }
    __device__ __forceinline__ Tile tile(const Request& r, int rt) const {
        const int first = rt * kRows, last = min(first + kRows, r.rows) - 1;
        Tile t;
        t.hi = seen(r, token(last)).y;
        t.lo = min(seen(r, token(first)).x, t.hi) & ~(kAlign - 1);
        t.blocks = max(1, (t.hi - t.lo + kKeys - 1) / kKeys);
        return t;
    }
    __device__ __forceinline__ int row_tiles(const Request& r) const { return (r.rows + kRows - 1) / kRows; }
    // Places of row tiles first, first + step, ...
    __device__ __forceinline__ int64_t cost(const Request& r, int first = 0, int step = 1) const {
        int64_t c = 0;
        for (int rt = first, n = row_tiles(r); rt < n; rt += step) c += tile(r, rt).blocks + kOver;
        return c * a.kv_heads;
    }
};

// x / y for x >= 0, y > 0: a 64-bit division takes some 500 cycles, a 32-bit one a fifth of that.
__device__ __forceinline__ int64_t divide(int64_t x, int64_t y) {
    return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

__device__ __forceinline__ int64_t warp_sum(int64_t x) {
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    return x;
}

// A place in the line: a tile and where it begins.
struct Cursor {
    Request r;
    Tile t;
    int b, rt, h;
    int64_t start;

    // The tile that holds place `u`, walking from request `b0`, whose places begin at `base` (u lies in it or later).  By a
    // whole warp.
    template <class L>
    __device__ __forceinline__ void seek(L& line, int b0, int64_t base, int64_t u, int lane) {
        b = b0;
        for (;; b++) {
            r = line.request(b);
            const int64_t c = warp_sum(line.cost(r, lane, 32));
            if (u < base + c || b + 1 >= line.a.B) break;
            base += c;
        }
        for (rt = 0;; rt += 32) {  // 32 row tiles at a time
            const bool there = rt + lane < line.row_tiles(r);
            const int64_t mine = there ? (int64_t)(line.tile(r, rt + lane).blocks + L::kOver) * line.a.kv_heads : 0;
            int64_t incl = mine;
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t x = __shfl_up_sync(~0u, incl, o);
                if (lane >= o) incl += x;
            }
            const unsigned at = __ballot_sync(~0u, there && u < base + incl);
            if (at) {
                const int l = __ffs(at) - 1;
                base += __shfl_sync(~0u, incl - mine, l);
                rt += l;
                break;
            }
            base += __shfl_sync(~0u, incl, 31);
            if (rt + 32 >= line.row_tiles(r)) break;
        }
        t = line.tile(r, rt);
        h = (int)divide(u - base, t.blocks + L::kOver);
        start = base + (int64_t)h * (t.blocks + L::kOver);
    }
    // On to the next tile (there is one).
    template <class L>
    __device__ __forceinline__ void next(L& line) {
        start += t.blocks + L::kOver;
        if (++h < line.a.kv_heads) return;
        h = 0;
        if (++rt >= line.row_tiles(r)) {
            rt = 0;
            do {
                b++;
                r = line.request(b);
            } while (r.rows == 0 && b + 1 < line.a.B);
        }
        t = line.tile(r, rt);
    }
};

// A CTA's stretch of the line, in shared memory.
template <int kThreads>
struct Stretch {
    static constexpr int kScratch = 8 * kThreads + 2 * kKvMaxRequests;  // bytes that find() needs
    int64_t warp_sums[kThreads / 32];
    int many, found;
    int64_t base;
    Cursor first;
    int64_t u0, u1, share;

    // Finds it.  By all threads; `scratch`: shared memory that nothing else uses meanwhile.
    template <class L>
    __device__ __forceinline__ void find(L& line, char* scratch) {
        constexpr int kFew = 4;  // row tiles that one thread counts by itself
        const AttendArgs& a = line.a;
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, per = (a.B + kThreads - 1) / kThreads;
        unsigned long long* const more = reinterpret_cast<unsigned long long*>(scratch);  // places of a thread's requests of many row tiles
        uint16_t* const list = reinterpret_cast<uint16_t*>(more + kThreads);               // those requests
        if (tid == 0) many = 0;
        more[tid] = 0;
        __syncthreads();
        int64_t mine = 0;
        for (int b = min(tid * per, a.B), b1 = min(b + per, a.B); b < b1; b++) {
            const Request r = line.request(b);
            if (line.row_tiles(r) <= kFew) mine += line.cost(r);
            else list[atomicAdd(&many, 1)] = (uint16_t)b;
        }
        __syncthreads();
        for (int i = warp; i < many; i += kThreads / 32) {
            const int64_t c = warp_sum(line.cost(line.request(list[i]), lane, 32));
            if (lane == 0) atomicAdd(&more[list[i] / per], (unsigned long long)c);
        }
        __syncthreads();
        mine += (int64_t)more[tid];
        int64_t incl = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(~0u, incl, o);
            if (lane >= o) incl += x;
        }
        if (lane == 31) warp_sums[warp] = incl;
        __syncthreads();
        int64_t before = 0, total = 0;
        for (int w = 0; w < kThreads / 32; w++) {
            if (w == warp) before = total;
            total += warp_sums[w];
        }
        before += incl - mine;
        const int64_t each = max((int64_t)1, divide(total + gridDim.x - 1, gridDim.x)), at = blockIdx.x * each;
        const bool countable = each < 0x7fffffff;  // a stretch is counted in 32 bits; a longer one would take days
        if (!countable) line.bad = true;
        if (tid == 0) {
            share = each;
            u0 = at;
            u1 = countable ? min(at + each, total) : at;
        }
        if (at >= before && at < before + mine) {
            found = tid;
            base = before;
        }
        __syncthreads();
        if (warp == 0 && at < total) {
            Cursor c = {};
            c.seek(line, found * per, base, at, lane);
            if (lane == 0) first = c;
        }
        __syncthreads();
    }
    __device__ __forceinline__ bool empty() const { return u0 >= u1; }
};

// The pieces of a stretch, in order: the part of each tile's blocks [p0, p1) that lies in it.
template <class L>
struct Walk {
    L& line;
    Cursor at;
    int left;    // places of the stretch from this tile on
    int used;    // of them this tile's
    int p0, p1;
    int piece = 0;
    bool more;   // there is a piece

    template <class S>
    __device__ __forceinline__ Walk(L& l, const S& s) : line(l) {
        at = s.first;
        left = (int)(s.u1 - s.u0);
        const int from = (int)(s.u0 - at.start);
        p0 = min(from, at.t.blocks);
        used = min(at.t.blocks + L::kOver - from, left);
        p1 = min(from + used, at.t.blocks);
        more = true;
        if (p0 == p1) {  // places behind the last block alone
            next();
            piece = 0;
        }
    }
    __device__ __forceinline__ void next() {
        left -= used;
        piece++;
        if (left == 0) {
            more = false;
            return;
        }
        at.next(line);
        p0 = 0;
        used = min(at.t.blocks + L::kOver, left);
        p1 = min(used, at.t.blocks);
    }
    // Whether the tile begins in this stretch, and whether it lies in it whole.
    template <class S>
    __device__ __forceinline__ bool begins(const S& s) const {
        return at.start >= s.u0;
    }
    template <class S>
    __device__ __forceinline__ bool whole(const S& s) const {
        return at.start >= s.u0 && at.start + at.t.blocks <= s.u1;
    }
};

// Tokens of no request, and of requests without positions: out = 0.
template <int D, int kThreads, class L>
__device__ __forceinline__ void clear_rest(L& line) {
    const AttendArgs& a = line.a;
    auto clear = [&](int t0, int t1, int from, int step) {
        const int64_t vecs = (int64_t)(t1 - t0) * a.heads * (D / 8);
        for (int64_t i = (int64_t)from * kThreads + threadIdx.x; i < vecs; i += (int64_t)step * kThreads) {
            const int64_t row = i / (D / 8);
            const int t = t0 + (int)(row / a.heads), h = (int)(row % a.heads), c = (int)(i % (D / 8));
            *reinterpret_cast<uint4*>(a.out + t * a.out_tok + h * a.out_head + c * 8) = make_uint4(0, 0, 0, 0);
            if (a.lse && c == 0) a.lse[(int64_t)t * a.heads + h] = -INFINITY;
        }
    };
    const int end = max(0, min(a.q_off[a.B], a.T));
    if (end < a.T) clear(end, a.T, blockIdx.x, gridDim.x);
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        const Request r = line.request(b);
        if (r.kv == 0 && r.n > a.min_q && r.n <= a.max_q && r.q0 < a.T) clear(r.q0, min(r.q0 + r.n, a.T), 0, 1);
    }
}

}  // namespace kv
}  // namespace kvdro
