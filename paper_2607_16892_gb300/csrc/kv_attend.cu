// Attention over pages (kvdro_kv_attend).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv.cuh"

namespace kvdro {

namespace {

constexpr int kWarps = 4;

template <bool H>
__device__ __forceinline__ float2 widen(uint32_t w) {
    if constexpr (H) return __half22float2(*reinterpret_cast<__half2*>(&w));
    else return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&w));
}
template <bool H>
__device__ __forceinline__ uint32_t narrow2(float x, float y) {
    if constexpr (H) {
        const __half2 r = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&r);
    } else {
        const __nv_bfloat162 r = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&r);
    }
}

// One warp per token and head, one key per lane: running maximum m, sum l and weighted sum o of the rows of v, each
// rescaled by exp(m - m') when the maximum grows to m'.
template <bool H, int D>
__global__ void __launch_bounds__(32 * kWarps) k_kv_attend(AttendArgs a) {
    __shared__ float s_q[kWarps][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * kWarps + warp;
    if (row >= (int64_t)a.T * a.heads) return;
    const int t = (int)(row / a.heads), h = (int)(row % a.heads), kh = h / a.group;
    constexpr int PER = D / 32;  // elements of o in a lane
    int b = -1;
    if (t < a.q_off[a.B]) {
        int lo = 0, hi = a.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.q_off[mid] <= t) lo = mid;
            else hi = mid;
        }
        b = lo;
    }
    int first = 0, last = 0;  // visible positions [first, last)
    if (b >= 0) {
        const int64_t n = a.kv_len[b], p = n - (a.q_off[b + 1] - t);
        const int64_t cap = (int64_t)a.max_pages << a.page_shift;
        if (n < 0 || n > cap) atomicOr(a.err, kKvErrRange);
        else {
            last = (int)(a.causal ? min(n, p + 1) : n);
            first = (int)(a.window > 0 ? max((int64_t)0, p - a.window + 1) : 0);
        }
    }
    const uint16_t* q = a.q + t * a.q_tok + h * a.q_head;
    if (lane < D / 8) {
        const uint4 x = reinterpret_cast<const uint4*>(q)[lane];
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        for (int i = 0; i < 4; i++) {
            const float2 f = widen<H>(w[i]);
            s_q[warp][lane * 8 + 2 * i] = f.x;
            s_q[warp][lane * 8 + 2 * i + 1] = f.y;
        }
    }
    __syncwarp();
    float m = -INFINITY, l = 0.f, o[PER];
    for (int i = 0; i < PER; i++) o[i] = 0.f;
    for (int j0 = first; j0 < last; j0 += 32) {
        const int j = j0 + lane;
        int page = -1;
        float s = -INFINITY;
        if (j < last) {
            page = a.table[(int64_t)b * a.max_pages + (j >> a.page_shift)];
            if ((uint32_t)page >= (uint32_t)a.n_pages) {
                atomicOr(a.err, kKvErrRange);
                page = -1;
            }
        }
        const int in = j & ((1 << a.page_shift) - 1);
        if (page >= 0) {
            const uint4* k = reinterpret_cast<const uint4*>(a.k + page * a.k_page + in * a.k_slot + kh * a.k_head);
            float dot = 0.f;
            for (int c = 0; c < D / 8; c++) {
                const uint4 x = k[c];
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                for (int i = 0; i < 4; i++) {
                    const float2 f = widen<H>(w[i]);
                    dot = fmaf(f.x, s_q[warp][c * 8 + 2 * i], dot);
                    dot = fmaf(f.y, s_q[warp][c * 8 + 2 * i + 1], dot);
                }
            }
            s = dot * a.scale;
            if (a.cap > 0.f) s = a.cap * tanhf(s / a.cap);
        }
        float top = s;
        for (int i = 16; i; i >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, i));
        const float to = fmaxf(m, top), shift = to == -INFINITY ? 0.f : to;
        const float w = page >= 0 ? expf(s - shift) : 0.f, keep = expf(m - shift);
        float sum = w;
        for (int i = 16; i; i >>= 1) sum += __shfl_xor_sync(~0u, sum, i);
        l = l * keep + sum;
        m = to;
        for (int i = 0; i < PER; i++) o[i] *= keep;
        for (int u = 0; u < 32 && j0 + u < last; u++) {
            const int pg = __shfl_sync(~0u, page, u), sl = __shfl_sync(~0u, in, u);
            const float wu = __shfl_sync(~0u, w, u);
            if (pg < 0) continue;
            const uint16_t* v = a.v + pg * a.v_page + sl * a.v_slot + kh * a.v_head + lane * PER;
            for (int i = 0; i < PER; i += 2) {
                const float2 f = widen<H>(*reinterpret_cast<const uint32_t*>(v + i));
                o[i] = fmaf(wu, f.x, o[i]);
                o[i + 1] = fmaf(wu, f.y, o[i + 1]);
            }
        }
    }
    const float r = l == 0.f ? 0.f : 1.f / l;
    uint16_t* out = a.out + t * a.out_tok + h * a.out_head + lane * PER;
    for (int i = 0; i < PER; i += 2) *reinterpret_cast<uint32_t*>(out + i) = narrow2<H>(o[i] * r, o[i + 1] * r);
    if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : m + logf(l);
}

template <bool H, int D>
cudaError_t launch(const AttendArgs& a, cudaStream_t s) {
    const int64_t rows = (int64_t)a.T * a.heads;
    k_kv_attend<H, D><<<(unsigned)((rows + kWarps - 1) / kWarps), 32 * kWarps, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv_attend(const AttendArgs& a, cudaStream_t s) {
    if (a.half) return a.head_dim == 128 ? launch<true, 128>(a, s) : launch<true, 64>(a, s);
    return a.head_dim == 128 ? launch<false, 128>(a, s) : launch<false, 64>(a, s);
}

}  // namespace kvdro
