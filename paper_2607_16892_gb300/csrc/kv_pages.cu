// Pages for requests (kvdro_kv_plan), the write into them (kvdro_kv_append, 16 and 8 bits) and the way back (kvdro_kv_read).
#include "kv_device.cuh"

#include <type_traits>

namespace kvdro {

namespace {

constexpr int kPlanThreads = 1024, kPer = 4;  // requests per thread at a time
constexpr int kPlanItems = 4096;  // tokens per CTA of a plan, about

// What the lengths of one request ask for.
struct Ask {
    int32_t q_len;   // tokens in the packed order
    int32_t need;    // pages beyond those held
    int32_t back;    // pages returned
    int32_t kv_len;  // tokens after the step
    bool fits;       // not refused by its own lengths
    bool bad;        // lengths that contradict each other
};

// max_pages << page_shift is below 2^31, so are all tokens held; cached + n is below 2^32.
__device__ __forceinline__ Ask ask(const PlanArgs& a, int32_t cached, int32_t n, int32_t held, int32_t reserve) {
    const uint32_t cap = (uint32_t)a.max_pages << a.page_shift;
    Ask r{max(n, 0), 0, 0, 0, false, false};
    r.bad = held < 0 || held > a.max_pages || cached < 0 || (n >= 0 && (uint32_t)cached > (uint32_t)held << a.page_shift);
    if (r.bad) return r;
    if (n < 0) {
        r.back = held;
        r.fits = true;
        return r;
    }
    const uint32_t total = (uint32_t)cached + (uint32_t)n;
    r.fits = total <= cap;
    if (!r.fits) return r;
    r.kv_len = (int32_t)total;
    const uint32_t want = max(total, min((uint32_t)max(reserve, 0), cap));
    if (n > 0) r.need = max(0, (int32_t)((want + (1u << a.page_shift) - 1) >> a.page_shift) - held);
    return r;
}

// Largest b in [0, B) with off[b] <= x (off ascending, off[0] <= x).
__device__ __forceinline__ int find(const int32_t* off, int B, int32_t x) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (off[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Sums up to 2^31 - 1, where they stay.  (64-bit ones took twice the shuffles, and those are what a scan waits for.)
__device__ __forceinline__ uint32_t plus(uint32_t x, uint32_t y) { return min(x + y, 0x7fffffffu); }
struct Sums {
    uint32_t q, need, back;
    __device__ __forceinline__ void add(const Sums& x) {
        q = plus(q, x.q);
        need = plus(need, x.need);
        back = plus(back, x.back);
    }
};
// Sums over the lanes before this one; `all`: over the warp.
__device__ __forceinline__ Sums scan(Sums x, int lane, Sums& all) {
    for (int o = 1; o < 32; o <<= 1) {
        const Sums y{__shfl_up_sync(~0u, x.q, o), __shfl_up_sync(~0u, x.need, o), __shfl_up_sync(~0u, x.back, o)};
        if (lane >= o) x.add(y);
    }
    all = x;  // in the last lane
    const Sums before{__shfl_up_sync(~0u, x.q, 1), __shfl_up_sync(~0u, x.need, 1), __shfl_up_sync(~0u, x.back, 1)};
    return lane ? before : Sums{0, 0, 0};
}

// Every CTA scans all requests, four per thread at a time (16 bytes each, out of L2 after the first CTA's reads), and
// keeps the prefix sums in shared memory; then the CTAs share the tokens and the pages, each found by a binary search there.
// One launch, and no CTA waits for another: nothing that a CTA writes is read by any (a new token's page is
// looked up in the ring, not in the table that another CTA may not have written yet).  Bound by the latency of its chain of
// dependent reads: lengths, sums, search, page.  8 requests 11 us a call (the host's share), 4096 requests with 424 k new tokens
// 12.4 us (17 with a request per thread and turn, 21 with 64-bit sums by every warp).
__global__ void __launch_bounds__(kPlanThreads) k_kv_plan(PlanArgs a) {
    extern __shared__ int32_t sm[];
    int32_t* s_q = sm;             // [B] first token
    int32_t* s_need = sm + a.B;    // [B] pages taken before this request
    int32_t* s_back = sm + 2 * a.B;  // [B] pages returned before this request; the sign: refused
    constexpr int kWarps = kPlanThreads / 32;
    static_assert(kWarps == 32, "one warp scans the warps' sums");
    __shared__ Sums s_warp[kWarps], s_all;
    __shared__ int32_t s_taken;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool first_cta = blockIdx.x == 0;
    if (tid == 0) s_taken = 0;

    struct Rows {
        int32_t cached[kPer], n[kPer], held[kPer], reserve[kPer];
    };
    const bool wide = ((reinterpret_cast<uintptr_t>(a.cached) | reinterpret_cast<uintptr_t>(a.new_len) | reinterpret_cast<uintptr_t>(a.held) |
                        reinterpret_cast<uintptr_t>(a.reserve)) & 15) == 0;
    auto load4 = [&](const int32_t* p, int b, int32_t (&x)[kPer]) {
        static_assert(kPer == 4, "one 16-byte load");
        if (wide && b + kPer <= a.B) {
            const int4 v = *reinterpret_cast<const int4*>(p + b);
            x[0] = v.x;
            x[1] = v.y;
            x[2] = v.z;
            x[3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < kPer; i++) x[i] = b + i < a.B ? p[b + i] : 0;
        }
    };
    auto load = [&](int b) {
        Rows x = {};
        if (b < a.B) {
            load4(a.cached, b, x.cached);
            load4(a.new_len, b, x.n);
            load4(a.held, b, x.held);
            if (a.reserve) load4(a.reserve, b, x.reserve);
        }
        return x;
    };
    Rows next = load(kPer * tid);
    int32_t head = a.pool[0], n_free = a.pool[1];
    const bool pool_bad = head < 0 || head >= a.n_pages || n_free < 0 || n_free > a.n_pages;
    if (pool_bad) head = n_free = 0;
    bool bad = pool_bad;
    const int32_t room = pool_bad ? 0 : a.n_pages - n_free;  // returned pages that the ring can hold

    // Pages are taken in the order of b while they last: the first request that does not fit ends it.
    Sums all{0, 0, 0};
    int32_t taken = 0;
    for (int b0 = 0; b0 < a.B; b0 += kPer * kPlanThreads) {
        const int first = b0 + kPer * tid;
        const bool writes = (b0 / (32 * kPer) + warp) % gridDim.x == blockIdx.x;  // the results by request, shared by warps
        const Rows x = next;
        next = load(first + kPer * kPlanThreads);
        Ask r[kPer];
        Sums mine{0, 0, 0};
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            r[i] = ask(a, x.cached[i], x.n[i], x.held[i], x.reserve[i]);
            mine.add(Sums{(uint32_t)r[i].q_len, (uint32_t)r[i].need, (uint32_t)r[i].back});
        }
        Sums sum;
        const Sums in_warp = scan(mine, lane, sum);
        if (lane == 31) s_warp[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            const Sums before = scan(s_warp[lane], lane, sum);
            s_warp[lane] = before;
            if (lane == 31) s_all = sum;
        }
        __syncthreads();
        Sums at = all;
        at.add(s_warp[warp]);
        at.add(in_warp);
        all.add(s_all);
#pragma unroll
        for (int i = 0; i < kPer; i++) {
            const int b = first + i;
            if (b >= a.B) break;
            const uint32_t need = plus(at.need, r[i].need);
            const bool full = r[i].need > 0 && need > (uint32_t)n_free, refused = !r[i].fits || full;
            if (r[i].need > 0 && !full) taken = (int32_t)need;
            // The place of a refused request among the pages does not matter, but ascends.
            s_q[b] = (int32_t)at.q;
            s_need[b] = (int32_t)min(at.need, (uint32_t)n_free);
            s_back[b] = (int32_t)(at.back | (refused ? 0x80000000u : 0u));
            if (writes) {
                a.q_off[b] = s_q[b];
                a.kv_len[b] = refused ? 0 : r[i].kv_len;
                a.held_out[b] = r[i].back ? 0 : x.held[i] + (refused ? 0 : r[i].need);
                bad |= r[i].bad;
            }
            at.add(Sums{(uint32_t)r[i].q_len, (uint32_t)r[i].need, (uint32_t)r[i].back});
        }
        __syncthreads();  // before the next turn's sums
    }
    taken = __reduce_max_sync(~0u, taken);
    if (lane == 0 && taken) atomicMax(&s_taken, taken);
    __syncthreads();
    taken = s_taken;
    const int32_t back = (int32_t)min(all.back, (uint32_t)room);
    if (first_cta && tid == 0) {
        a.q_off[a.B] = (int32_t)all.q;
        if (all.back > (uint32_t)room || all.q > (uint32_t)a.T) bad = true;
        if (pool_bad) {  // stays as it is
            a.pool_out[0] = a.pool[0];
            a.pool_out[1] = a.pool[1];
        } else {
            int64_t h = (int64_t)head + taken;
            a.pool_out[0] = (int32_t)(h >= a.n_pages ? h - a.n_pages : h);
            a.pool_out[1] = (int32_t)(n_free - taken + back);
        }
    }
    auto ring_at = [&](int64_t i) { return (int64_t)(i >= a.n_pages ? i - a.n_pages : i); };

    const int step = gridDim.x * kPlanThreads, id = blockIdx.x * kPlanThreads + tid;
    // A request's place is capped at n_free once the pages ran out: those places hold no page of its own.
    for (int i = id; i < taken; i += step) {
        const int b = find(s_need, a.B, i);
        int32_t page = a.ring[ring_at((int64_t)head + i)];
        if ((uint32_t)page >= (uint32_t)a.n_pages) {
            bad = true;
            page = -1;
        }
        a.table[(int64_t)b * a.max_pages + a.held[b] + (i - s_need[b])] = page;
    }
    for (int i = id; i < back; i += step) {
        int lo = 0, hi = a.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((s_back[mid] & 0x7fffffff) <= i) lo = mid;
            else hi = mid;
        }
        int64_t to = (int64_t)head + n_free;
        to = ring_at(ring_at(to) + i);
        int32_t page = a.table[(int64_t)lo * a.max_pages + (i - (s_back[lo] & 0x7fffffff))];
        if ((uint32_t)page >= (uint32_t)a.n_pages) {  // none, and stays none in the ring
            bad = true;
            page = -1;
        }
        a.ring[to] = page;
    }
    // Tokens four at a time: mostly of one request and one page, found once.
    const int tokens = (int)min(all.q, (uint32_t)a.T), mask = (1 << a.page_shift) - 1;
    const bool wide_out = reinterpret_cast<uintptr_t>(a.slot) % 16 == 0 && reinterpret_cast<uintptr_t>(a.pos) % 16 == 0;
    for (int t0 = 4 * id; t0 < a.T; t0 += 4 * step) {
        int32_t slot[4] = {-1, -1, -1, -1}, pos[4] = {-1, -1, -1, -1};
        if (t0 < tokens) {
            int b = find(s_q, a.B, t0), have_b = -1, have_j = -1;
            int32_t cached = 0, held = 0, page = -1;
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const int t = t0 + k;
                if (t >= tokens) break;
                while (b + 1 < a.B && s_q[b + 1] <= t) b++;
                if (s_back[b] < 0) continue;
                if (b != have_b) {
                    have_b = b;
                    have_j = -1;
                    cached = a.cached[b];
                    held = a.held[b];
                }
                pos[k] = cached + (t - s_q[b]);
                const int32_t j = pos[k] >> a.page_shift;
                if (j != have_j) {
                    have_j = j;
                    page = j < held ? a.table[(int64_t)b * a.max_pages + j] : a.ring[ring_at((int64_t)head + s_need[b] + (j - held))];
                }
                if ((uint32_t)page < (uint32_t)a.n_pages) slot[k] = (page << a.page_shift) + (pos[k] & mask);
                else bad = true;
            }
        }
        if (wide_out && t0 + 4 <= a.T) {
            *reinterpret_cast<int4*>(a.slot + t0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
            if (a.pos) *reinterpret_cast<int4*>(a.pos + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        } else {
            for (int k = 0; k < 4 && t0 + k < a.T; k++) {
                a.slot[t0 + k] = slot[k];
                if (a.pos) a.pos[t0 + k] = pos[k];
            }
        }
    }
    if (bad) atomicOr(a.err, kKvErrRange);
}

// A copy with a lookup: bound by the bytes read and written (65539 tokens of 8 heads of 128, 526 MB, 81 us = 6.5 TB/s; a copy runs
// at 6.8).  A token's row is dealt to 2^lanes_shift lanes, 16 bytes
// each at a time, keys and values together, so that a lane has up to eight loads in flight.
constexpr int kAppendThreads = 256, kAppendDeep = 4;

__global__ void __launch_bounds__(kAppendThreads) k_kv_append(AppendArgs a, int lanes_shift) {
    const int64_t id = (int64_t)blockIdx.x * kAppendThreads + threadIdx.x, t = id >> lanes_shift;
    const int lanes = 1 << lanes_shift;
    if (t >= a.T) return;
    const int32_t slot = a.slot[t];
    if (slot < 0 || slot >= a.n_slots) {
        if (slot != -1) atomicOr(a.err, kKvErrRange);
        return;
    }
    const int64_t page = slot >> a.page_shift, in = slot & ((1 << a.page_shift) - 1);
    const uint4 *k = a.k + t * a.k_tok, *v = a.v + t * a.v_tok;
    uint4 *kc = a.kc + page * a.kc_page + in * a.kc_slot, *vc = a.vc + page * a.vc_page + in * a.vc_slot;
    const int vecs = a.heads << a.vec_shift, mask = (1 << a.vec_shift) - 1;
    for (int i0 = (int)id & (lanes - 1); i0 < vecs; i0 += kAppendDeep * lanes) {
        uint4 x[kAppendDeep], y[kAppendDeep];
#pragma unroll
        for (int u = 0; u < kAppendDeep; u++) {
            const int i = i0 + u * lanes;
            if (i < vecs) {
                x[u] = k[(i >> a.vec_shift) * a.k_head + (i & mask)];
                y[u] = v[(i >> a.vec_shift) * a.v_head + (i & mask)];
            }
        }
#pragma unroll
        for (int u = 0; u < kAppendDeep; u++) {
            const int i = i0 + u * lanes;
            if (i < vecs) {
                kc[(i >> a.vec_shift) * a.kc_head + (i & mask)] = x[u];
                vc[(i >> a.vec_shift) * a.vc_head + (i & mask)] = y[u];
            }
        }
    }
}

// Sixteen elements of a row as codes, the row's others in the neighbouring `lanes` of `mask`: the scale is the least power of two
// 2^E, E >= -126, with max |x| <= 448 2^E over the row's finite elements, and each element is rounded once, to the nearest code.
// A power of two costs no precision (codes are floating-point numbers of three bits whatever their scale) and multiplies
// exactly.  Non-finite elements become NaN.  FP16 cannot hold 256 * 2^8, which its largest numbers would round to: 240 * 2^8.
// `e`: E + 127.
template <bool H>
__device__ __forceinline__ uint4 quantise(const uint4 (&x)[2], unsigned mask, int lanes, uint32_t& e) {
    constexpr uint32_t kInf = H ? 0x7c00u : 0x7f80u;
    const uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    uint32_t top2 = 0;  // magnitudes of 16-bit numbers are ordered as whole numbers, two at a time
#pragma unroll
    for (int i = 0; i < 8; i++) top2 = __vmaxu2(top2, w[i] & 0x7fff7fffu);
    for (int o = 1; o < lanes; o <<= 1) top2 = __vmaxu2(top2, __shfl_xor_sync(mask, top2, o));
    uint32_t top16 = max(top2 & 0xffffu, top2 >> 16);
    const bool odd = top16 >= kInf;
    if (odd) {  // the largest of the finite ones
        top2 = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t y = w[i] & 0x7fff7fffu;
            top2 = __vmaxu2(top2, ((y & 0xffffu) < kInf ? y & 0xffffu : 0u) | (y >> 16 < kInf ? y & 0xffff0000u : 0u));
        }
        for (int o = 1; o < lanes; o <<= 1) top2 = __vmaxu2(top2, __shfl_xor_sync(mask, top2, o));
        top16 = max(top2 & 0xffffu, top2 >> 16);
    }
    const uint32_t u = __float_as_uint(kv::unpack2<H>(top16).x);
    e = (uint32_t)max((int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), 1);  // 448 = 1.75 * 2^8
    const float down = __uint_as_float((254 - e) << 23);
    float2 y[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        y[i] = kv::unpack2<H>(w[i]);
        y[i].x *= down;
        y[i].y *= down;
    }
    if (odd || (H && e == 135)) {
        const float most = H && e == 135 ? 240.f : 448.f, nan = __uint_as_float(0x7fffffffu);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            y[i] = make_float2(fminf(fmaxf(y[i].x, -most), most), fminf(fmaxf(y[i].y, -most), most));
            if ((w[i] & 0x7fffu) >= kInf) y[i].x = nan;
            if ((w[i] >> 16 & 0x7fffu) >= kInf) y[i].y = nan;
        }
    }
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        uint16_t r[2];
#pragma unroll
        for (int k = 0; k < 2; k++) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r[k]) : "f"(y[2 * i + k].y), "f"(y[2 * i + k].x));
        c[i] = __byte_perm(r[0], r[1], 0x5410);
    }
    return make_uint4(c[0], c[1], c[2], c[3]);
}

// As the copy above, a row dealt to lanes of sixteen elements each.  Bound by the bytes: 65539 tokens of 8 heads of 128 in FP16, 396 MB
// read and written, 67.5 us = 5.9 TB/s.  On the way there: eight elements to a lane and addresses by products, 182 instructions for
// every eight elements, 115 us; addresses by steps 92; sixteen elements 87; 128 threads 76; ten CTAs per SM (48 registers,
// and 16 bytes spilled in BF16, 20 in FP16) 67.5, eight 73.6, twelve 70.9; two or four heads of a lane at once 84 and 98.
constexpr int kAppend8Deep = 1, kAppend8Threads = 128, kAppend8Ctas = 10;

template <bool H>
__global__ void __launch_bounds__(kAppend8Threads, kAppend8Ctas) k_kv_append8(Append8Args a, int lanes_shift) {
    const int64_t id = (int64_t)blockIdx.x * kAppend8Threads + threadIdx.x, t = id >> lanes_shift;
    const int lanes = 1 << lanes_shift;
    if (t >= a.T) return;
    const int32_t slot = a.slot[t];
    if (slot < 0 || slot >= a.n_slots) {
        if (slot != -1) atomicOr(a.err, kKvErrRange);
        return;
    }
    const int64_t page = slot >> a.page_shift, in = slot & ((1 << a.page_shift) - 1);
    // A lane has the same part of every head that it comes to: its addresses advance by the same steps.
    const int row = 1 << a.part_shift, c = (int)id & (row - 1), by = lanes >> a.part_shift;
    int h = ((int)id & (lanes - 1)) >> a.part_shift;
    const uint4 *k = a.k + t * a.k_tok + h * a.k_head + 2 * c, *v = a.v + t * a.v_tok + h * a.v_head + 2 * c;
    uint4 *kc = a.kc + page * a.kc_page + in * a.kc_slot + h * a.kc_head + c, *vc = a.vc + page * a.vc_page + in * a.vc_slot + h * a.vc_head + c;
    const int64_t k_by = by * a.k_head, v_by = by * a.v_head, kc_by = by * a.kc_head, vc_by = by * a.vc_head;
    int64_t at = ((page * a.heads + h) << a.page_shift) + in;
    const int64_t at_by = (int64_t)by << a.page_shift;
    const unsigned mask = ((1u << row) - 1u) << (threadIdx.x & 31 & ~(row - 1));  // 4 or 8 lanes, all of one token
    for (; h < a.heads; h += kAppend8Deep * by) {
        uint4 x[kAppend8Deep][2], y[kAppend8Deep][2];
#pragma unroll
        for (int u = 0; u < kAppend8Deep; u++) {
            if (h + u * by < a.heads) {
                x[u][0] = k[0];
                x[u][1] = k[1];
                y[u][0] = v[0];
                y[u][1] = v[1];
            }
            k += k_by;
            v += v_by;
        }
#pragma unroll
        for (int u = 0; u < kAppend8Deep; u++) {
            if (h + u * by < a.heads) {
                uint32_t ke, ve;
                *kc = quantise<H>(x[u], mask, row, ke);
                *vc = quantise<H>(y[u], mask, row, ve);
                if (c == 0) {
                    a.k_exp[at] = (uint8_t)ke;
                    a.v_exp[at] = (uint8_t)ve;
                }
            }
            kc += kc_by;
            vc += vc_by;
            at += at_by;
        }
    }
}

// Rows out of pages: a copy with two lookups, the request of a token and its page.  A token's row is dealt to lanes as above, eight
// elements each, of two heads at once.  Bound by the bytes: 64 requests of lognormal lengths up to 8192 out of 8 bits, 837 MB, 137 us =
// 6.1 TB/s (one head at once 149 us, three 143, four 145; CTAs of 256 139).
constexpr int kReadDeep = 2, kReadThreads = 128;

template <bool H, bool Q>
__global__ void __launch_bounds__(kReadThreads) k_kv_read(ReadArgs a, int lanes_shift) {
    const int64_t id = (int64_t)blockIdx.x * kReadThreads + threadIdx.x, t64 = id >> lanes_shift;
    const int lanes = 1 << lanes_shift;
    if (t64 >= a.T) return;
    const int t = (int)t64;
    int lo = 0, hi = a.B;  // the first request that ends behind t
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.q_off[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    int32_t page = -1, in = 0;
    bool bad = false;
    if (lo < a.B) {
        const int32_t q0 = a.q_off[lo], q1 = a.q_off[lo + 1], n = a.kv_len[lo];
        if (q0 < 0 || n < 0 || (int64_t)n > ((int64_t)a.max_pages << a.page_shift)) {
            bad = true;
        } else if (t >= q0 && n - (q1 - t) >= 0) {
            const int32_t p = n - (q1 - t);
            page = a.table[(int64_t)lo * a.max_pages + (p >> a.page_shift)];
            in = p & ((1 << a.page_shift) - 1);
            if ((uint32_t)page >= (uint32_t)a.n_pages) {
                bad = true;
                page = -1;
            }
        }
    }
    if (bad) atomicOr(a.err, kKvErrRange);
    uint4 *k = a.k + (int64_t)t * a.k_tok, *v = a.v + (int64_t)t * a.v_tok;
    const int64_t from = max(page, 0);
    const char *kc = a.kc + from * a.kc_page + in * a.kc_slot, *vc = a.vc + from * a.vc_page + in * a.vc_slot;
    const int vecs = a.heads << a.vec_shift, mask = (1 << a.vec_shift) - 1;
    using Vec = typename std::conditional<Q, uint2, uint4>::type;  // eight elements as they are stored
    for (int i0 = (int)id & (lanes - 1); i0 < vecs; i0 += kReadDeep * lanes) {
        Vec x[kReadDeep] = {}, y[kReadDeep] = {};
        uint32_t ke[kReadDeep] = {}, ve[kReadDeep] = {};
#pragma unroll
        for (int u = 0; u < kReadDeep; u++) {
            const int i = i0 + u * lanes, h = i >> a.vec_shift, c = i & mask;
            if (i < vecs && page >= 0) {
                x[u] = *reinterpret_cast<const Vec*>(kc + h * a.kc_head + c * (int)sizeof(Vec));
                y[u] = *reinterpret_cast<const Vec*>(vc + h * a.vc_head + c * (int)sizeof(Vec));
                if constexpr (Q) {
                    const int64_t at = ((from * a.heads + h) << a.page_shift) + in;
                    ke[u] = a.k_exp[at];
                    ve[u] = a.v_exp[at];
                }
            }
        }
        auto value = [](const Vec& w, uint32_t e) {
            if constexpr (Q) {
                const float s = kv::scale_of(e);
                uint32_t r[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float2 f = kv::unpack2<true>(kv::half2_of((uint16_t)((i < 2 ? w.x : w.y) >> (i & 1 ? 16 : 0))));
                    r[i] = kv::pack2<H>(f.x * s, f.y * s);
                }
                return make_uint4(r[0], r[1], r[2], r[3]);
            } else {
                return w;
            }
        };
#pragma unroll
        for (int u = 0; u < kReadDeep; u++) {
            const int i = i0 + u * lanes, h = i >> a.vec_shift, c = i & mask;
            if (i < vecs) {
                k[h * a.k_head + c] = value(x[u], ke[u]);
                v[h * a.v_head + c] = value(y[u], ve[u]);
            }
        }
    }
}

// Lanes that a token's row is dealt to, as a power of two, and the CTAs of a launch.
int lanes_of(int vecs) {
    int shift = 0;
    while (shift < 5 && (1 << shift) < vecs) shift++;
    return shift;
}
// Few tokens leave most of the GPU idle: their rows are dealt to several warps, while all lanes are at most these (quantised writes of 64 tokens, 8
// heads of 128, one after another: 4.1 us each, 6.1 with one warp to a token; of 4096 tokens 8.2 either way).
constexpr int64_t kFewLanes = 1 << 17;
int lanes_of(int vecs, int64_t T) {
    int shift = lanes_of(vecs);
    while ((1 << shift) < vecs && T << (shift + 1) <= kFewLanes) shift++;
    return shift;
}
unsigned ctas_of(int64_t T, int lanes_shift, int threads) { return (unsigned)(((T << lanes_shift) + threads - 1) / threads); }

__global__ void k_kv_take(int32_t* err) { err[1] = atomicExch(err, 0); }

}  // namespace

cudaError_t launch_kv_take(int32_t* err, cudaStream_t s) {
    k_kv_take<<<1, 1, 0, s>>>(err);
    return cudaGetLastError();
}

cudaError_t kv_plan_prepare() {
    return cudaFuncSetAttribute(k_kv_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * 4 * kKvMaxRequests);
}

cudaError_t launch_kv_plan(const PlanArgs& a, int sms, cudaStream_t s) {
    const int64_t items = (int64_t)a.T + 4 * (int64_t)a.B;
    int64_t ctas = (items + kPlanItems - 1) / kPlanItems;
    ctas = ctas < 1 ? 1 : ctas > sms ? sms : ctas;
    k_kv_plan<<<(int)ctas, kPlanThreads, 3 * 4 * (size_t)a.B, s>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_kv_append(const AppendArgs& a, cudaStream_t s) {
    const int shift = lanes_of(a.heads << a.vec_shift);
    k_kv_append<<<ctas_of(a.T, shift, kAppendThreads), kAppendThreads, 0, s>>>(a, shift);
    return cudaGetLastError();
}

cudaError_t launch_kv_append8(const Append8Args& a, cudaStream_t s) {
    const int shift = lanes_of(a.heads << a.part_shift, a.T);
    if (a.half) k_kv_append8<true><<<ctas_of(a.T, shift, kAppend8Threads), kAppend8Threads, 0, s>>>(a, shift);
    else k_kv_append8<false><<<ctas_of(a.T, shift, kAppend8Threads), kAppend8Threads, 0, s>>>(a, shift);
    return cudaGetLastError();
}

cudaError_t launch_kv_read(const ReadArgs& a, cudaStream_t s) {
    const int shift = lanes_of(a.heads << a.vec_shift);
    const unsigned ctas = ctas_of(a.T, shift, kReadThreads);
    if (!a.k_exp) k_kv_read<true, false><<<ctas, kReadThreads, 0, s>>>(a, shift);
    else if (a.half) k_kv_read<true, true><<<ctas, kReadThreads, 0, s>>>(a, shift);
    else k_kv_read<false, true><<<ctas, kReadThreads, 0, s>>>(a, shift);
    return cudaGetLastError();
}

}  // namespace kvdro
