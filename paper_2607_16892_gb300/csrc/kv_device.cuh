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
// a few 2^-24 of cap.  `mul` is scale * log2(e), or 2 log2(e) scale / cap; `cap2` is cap * log2(e).
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
// Waits for a phase, for about 2 s at most: 2 s of the GPU's timer and 2^14 polls made while running.
static __device__ __forceinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity) {
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    for (unsigned polls = 0; polls < (1u << 28); polls++) {
        if (mbar_try(bar, parity)) return true;
        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
        if (polls > (1u << 14) && t - t0 > 2000000000ull) return false;
    }
    return false;
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {
    return mbar_try(bar, parity) || mbar_wait_slow(bar, parity);
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
// and each CTA takes an equal stretch of it, so that long contexts are shared by many CTAs and short ones share a CTA.
// A tile that crosses from one stretch into the next is joined from its pieces.
struct Request {
    int q0, n, rows, kv;  // first token, tokens, rows (tokens inside T times the group), positions
};

struct Tile {
    int lo, hi, blocks;  // positions [lo, hi), lo on a slice of 16
};

template <int kRows, int kKeys, int kAlign>
struct Line {
    const AttendArgs& a;
    bool bad = false;

    __device__ __forceinline__ explicit Line(const AttendArgs& args) : a(args) {}

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
        r.rows = max(0, min(q1, a.T) - r.q0) * a.group;
        if (r.kv < 0 || (int64_t)r.kv > ((int64_t)a.max_pages << a.page_shift)) {
            bad = true;
            r.kv = 0;
        }
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
        t.hi = seen(r, last / a.group).y;
        t.lo = min(seen(r, first / a.group).x, t.hi) & ~(kAlign - 1);
        t.blocks = max(1, (t.hi - t.lo + kKeys - 1) / kKeys);
        return t;
    }
    __device__ __forceinline__ int row_tiles(const Request& r) const { return (r.rows + kRows - 1) / kRows; }
    __device__ __forceinline__ int64_t cost(const Request& r) const {
        int64_t c = 0;
        for (int rt = 0, n = row_tiles(r); rt < n; rt++) c += tile(r, rt).blocks;
        return c * a.kv_heads;
    }
};

// A place in the line: a tile and where its blocks begin.
template <class L>
struct Cursor {
    Request r;
    Tile t;
    int b, rt, h;
    int64_t start;  // the tile's first block in the line

    // The tile that holds block `u`, walking from request `b0`, whose blocks begin at `base` (u lies in it or later).
    __device__ __forceinline__ void seek(L& line, int b0, int64_t base, int64_t u) {
        b = b0;
        for (;; b++) {
            r = line.request(b);
            const int64_t c = line.cost(r);
            if (u < base + c || b + 1 >= line.a.B) break;
            base += c;
        }
        for (rt = 0;; rt++) {
            t = line.tile(r, rt);
            const int64_t c = (int64_t)t.blocks * line.a.kv_heads;
            if (u < base + c || rt + 1 >= line.row_tiles(r)) break;
            base += c;
        }
        h = (int)((u - base) / t.blocks);
        start = base + (int64_t)h * t.blocks;
    }
    // On to the next tile (there is one).
    __device__ __forceinline__ void next(L& line) {
        start += t.blocks;
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

}  // namespace kv
}  // namespace kvdro
