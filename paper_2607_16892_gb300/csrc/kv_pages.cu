// Pages for requests (kvdro_kv_plan) and the write into them (kvdro_kv_append).
#include "kv.cuh"

namespace kvdro {

namespace {

constexpr int kPlanThreads = 512;
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

__device__ __forceinline__ Ask ask(const PlanArgs& a, int b) {
    const int32_t cached = a.cached[b], n = a.new_len[b], held = a.held[b];
    const int64_t cap = (int64_t)a.max_pages << a.page_shift;
    Ask r{n > 0 ? n : 0, 0, 0, 0, true, false};
    r.bad = held < 0 || held > a.max_pages || cached < 0 || (n >= 0 && (int64_t)cached > ((int64_t)held << a.page_shift));
    if (r.bad) {
        r.fits = false;
        return r;
    }
    if (n < 0) {
        r.back = held;
        return r;
    }
    const int64_t total = (int64_t)cached + n;
    r.fits = total <= cap;
    if (!r.fits) return r;
    r.kv_len = (int32_t)total;
    if (n > 0) {
        int64_t want = total;
        if (a.reserve) {
            const int64_t res = min((int64_t)a.reserve[b], cap);
            want = res > want ? res : want;
        }
        const int32_t pages = (int32_t)((want + (1 << a.page_shift) - 1) >> a.page_shift);
        r.need = max(0, pages - held);
    }
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

struct Sums {
    int64_t q, need, back;
};

// Every CTA scans all requests (16 bytes each, out of L2 after the first) and keeps the prefix sums in shared
// memory; then the CTAs share the tokens and the pages, each found by a binary search there.  One launch, and no
// CTA waits for another: nothing that a CTA writes is read by any (a new token's page is looked up in the ring, not
// in the table that another CTA may not have written yet).
__global__ void __launch_bounds__(kPlanThreads) k_kv_plan(PlanArgs a) {
    extern __shared__ int32_t sm[];
    int32_t* s_q = sm;             // [B] first token
    int32_t* s_need = sm + a.B;    // [B] pages taken before this request
    int32_t* s_back = sm + 2 * a.B;  // [B] pages returned before this request
    __shared__ Sums s_warp[kPlanThreads / 32];
    __shared__ int32_t s_taken;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool first_cta = blockIdx.x == 0;

    int32_t head = a.pool[0], n_free = a.pool[1];
    const bool pool_bad = head < 0 || head >= a.n_pages || n_free < 0 || n_free > a.n_pages;
    if (pool_bad) head = n_free = 0;
    bool bad = pool_bad;
    const int32_t room = pool_bad ? 0 : a.n_pages - n_free;  // returned pages that the ring can hold

    const int per = (a.B + kPlanThreads - 1) / kPlanThreads, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
    Sums mine{0, 0, 0};
    for (int b = b0; b < b1; b++) {
        const Ask r = ask(a, b);
        mine.q += r.q_len;
        mine.need += r.need;
        mine.back += r.back;
    }
    Sums incl = mine;
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t q = __shfl_up_sync(~0u, incl.q, o), n = __shfl_up_sync(~0u, incl.need, o),
                      k = __shfl_up_sync(~0u, incl.back, o);
        if (lane >= o) {
            incl.q += q;
            incl.need += n;
            incl.back += k;
        }
    }
    if (lane == 31) s_warp[warp] = incl;
    if (tid == 0) s_taken = 0;
    __syncthreads();
    Sums base{0, 0, 0}, all{0, 0, 0};
    for (int w = 0; w < kPlanThreads / 32; w++) {
        if (w == warp) base = all;
        all.q += s_warp[w].q;
        all.need += s_warp[w].need;
        all.back += s_warp[w].back;
    }
    Sums at{base.q + incl.q - mine.q, base.need + incl.need - mine.need, base.back + incl.back - mine.back};

    // Pages are taken in the order of b while they last: the first request that does not fit ends it.
    int32_t taken = 0;
    for (int b = b0; b < b1; b++) {
        const Ask r = ask(a, b);
        if (r.need > 0 && at.need + r.need <= n_free) taken = (int32_t)(at.need + r.need);
        const bool refused = !r.fits || (r.need > 0 && at.need + r.need > n_free);
        // A refused request is marked by its sign; its place among the pages does not matter, but ascends.
        const int32_t need_at = (int32_t)min(at.need, (int64_t)n_free);
        s_q[b] = (int32_t)min(at.q, (int64_t)0x7fffffff);
        s_need[b] = need_at;
        s_back[b] = (int32_t)min(at.back, (int64_t)0x7fffffff) | (refused ? (int32_t)0x80000000 : 0);
        if (first_cta) {
            a.q_off[b] = s_q[b];
            a.kv_len[b] = refused ? 0 : r.kv_len;
            a.held_out[b] = r.back ? 0 : a.held[b] + (refused ? 0 : r.need);
            if (r.bad) bad = true;
        }
        at.q += r.q_len;
        at.need += r.need;
        at.back += r.back;
    }
    if (taken) atomicMax(&s_taken, taken);
    __syncthreads();
    taken = s_taken;
    const int64_t back = min(all.back, (int64_t)room);
    if (first_cta && tid == 0) {
        a.q_off[a.B] = (int32_t)min(all.q, (int64_t)0x7fffffff);
        if (all.back > room || all.q > a.T) bad = true;
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
        a.ring[to] = a.table[(int64_t)lo * a.max_pages + (i - (s_back[lo] & 0x7fffffff))];
    }
    const int64_t tokens = min(all.q, (int64_t)a.T);
    for (int t = id; t < a.T; t += step) {
        int32_t slot = -1, pos = -1;
        if (t < tokens) {
            const int b = find(s_q, a.B, t);
            if (s_back[b] >= 0) {
                pos = a.cached[b] + (t - s_q[b]);
                const int32_t j = pos >> a.page_shift, held = a.held[b];
                const int32_t page = j < held ? a.table[(int64_t)b * a.max_pages + j]
                                              : a.ring[ring_at((int64_t)head + s_need[b] + (j - held))];
                if ((uint32_t)page < (uint32_t)a.n_pages) slot = (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
                else bad = true;
            }
        }
        a.slot[t] = slot;
        if (a.pos) a.pos[t] = pos;
    }
    if (bad) atomicOr(a.err, kKvErrRange);
}

// A copy with a lookup: bound by the bytes read and written.  A token's row is dealt to 2^lanes_shift lanes, 16 bytes
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

}  // namespace

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
    const int vecs = a.heads << a.vec_shift;
    int shift = 0;
    while (shift < 5 && (1 << shift) < vecs) shift++;
    const int64_t threads = (int64_t)a.T << shift;
    k_kv_append<<<(unsigned)((threads + kAppendThreads - 1) / kAppendThreads), kAppendThreads, 0, s>>>(a, shift);
    return cudaGetLastError();
}

}  // namespace kvdro
