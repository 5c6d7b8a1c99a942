// Attention of chunks of new tokens over pages, on the tcgen05 tensor cores.
//
// A tile is 256 rows (tokens times the heads that share a key head) in two halves of 128, a block 128 positions.  Per block and
// half: S = Q K^T (128 x 128 into tensor memory), weights P = 2^(S - m) by four warps, a row per thread, back into
// tensor memory over S, and O += P V.  Both halves use the same K and V out of a ring of shared-memory stages; while the
// four warps of one half exponentiate, the tensor cores work for the other, in the fixed order
//     S0(0) S1(0) | PV0(0) S0(1) PV1(0) S1(1) | PV0(1) S0(2) ...
// which keeps the halves out of step.  (With a warp of its own to issue each half's products they fell into step and waited
// for the same things: 1760 us for the case below.)  The maximum m that weights refer to is raised only when a row's
// true maximum passes it by 2^8, so that O is rescaled in a few blocks at most; sums are exact in any case, for l and O
// refer to the same m.  The line of all blocks is dealt to one CTA per SM (kv_device.cuh); pieces of tiles that
// cross CTAs go through global memory and a second small kernel joins them in a fixed order.
//
// Roles: warps 0-3 and 4-7 the halves' weights, Q and results; 8 issues the products; 9 the copies; 10 and 11 look
// through V of blocks that some row does not see whole: a weight of 0 times infinity or NaN is not 0, so such elements are
// replaced by 0 there, and the rows that do see them get them added at the end.
//
// Bound by the tensor cores where contexts are long.  A block of both halves takes about 3000 cycles: 16 S products of 70 cycles
// and 16 PV products of 81 by themselves (64 at peak), 90 to 100 each beside the copies into shared memory and the weights' traffic
// in tensor memory.  Measured (bf16, 32 heads of 128 over 8 key heads): 4096 tokens at the end of 32768, 2.06 TFLOP in
// 1370 us over ten calls = 1.50 PFLOP/s, 1500 over 400 calls, which heat the GPU = 1.37 (0.80 and 0.73 of the measured 1.89 of
// a burst; 0.81 of the sustained 1.69); 512 tokens over 4099 45 us,
// of which 4 are the search of the line, 6 the join and 3 the launch.
#include "kv_device.cuh"

namespace kvdro {

namespace {

using namespace kv;

constexpr int kHalfRows = 128, kRows = 2 * kHalfRows, kKeys = 128;
constexpr int kThreads = 384;
constexpr int kNotes = 16;  // blocks that the copies are ahead of the weights, at most (a power of two)
constexpr int kOver = 2;   // a tile's fixed cost, in blocks (1 / 2 / 3: mixed batch 148 / 132 / 132 us, capped prompts 95 / 96.5 / 99)

template <int D>
struct Shape {
    static constexpr int kTile = kKeys * D * 2;  // bytes of K or V of a block, and of half a tile of Q
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr int kSmem = 2 * kTile + kStages * kTile + 1024;
    static constexpr int kPieceFloats = kRows * (D + 2);
};

using ChunkLine = Line<kRows, kKeys, kKeys, kOver>;

struct Shared {
    uint64_t kv_full[10], kv_empty[10], v_clean[10];
    uint64_t s_full[2], p_full[2][2], o_full[2], q_full[2], done;
    Stretch<kThreads> part;
    unsigned long long limit;  // of a wait, in ns
    int dead;
    uint32_t tmem;
    uint32_t skip[kNotes];  // by block: 16-slot slices whose page number is none
    int2 odd[2][kNotes];    // by looking warp and piece: first and last block with elements replaced, first > last if none
};

// ------------------------------------------------------------------ tcgen05
__device__ __forceinline__ void tc_alloc(uint32_t at) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(at) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tc_free(uint32_t tmem) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Loads are done; `r` is what one brought, so that nothing is computed from it before.
template <int N, int M>
__device__ __forceinline__ void tc_wait_ld(uint32_t (&r)[N][M]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int n = 0; n < N; n++)
#pragma unroll
        for (int i = 0; i < M; i++) asm volatile("" : "+r"(r[n][i]));
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// d (+)= a b: A in shared memory, or in tensor memory.
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void tc_mma_t(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
// 32 columns of this thread's lane.
__device__ __forceinline__ void tc_load32(uint32_t (&r)[32], uint32_t at) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
}
__device__ __forceinline__ void tc_load16(uint32_t (&r)[16], uint32_t at) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at));
}
__device__ __forceinline__ void tc_store32(uint32_t at, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tc_store16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

// Matrix descriptors of tiles of rows of 128 bytes in the 128-byte swizzle, in units of 16 bytes.  Contiguous along the
// summed dimension (Q, K): groups of 8 rows 1024 bytes apart.  Contiguous along the other (V: rows are positions, summed
// over): groups of 8 positions 1024 bytes apart, chunks of 64 columns one half of the tile apart.
__device__ __forceinline__ uint64_t descriptor(uint32_t addr, uint32_t lead, uint32_t stride) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
template <bool H, int N, bool T>
__device__ __forceinline__ constexpr uint32_t instruction() {  // 128 x N, FP32 sums; T: B contiguous along N
    return 1u << 4 | (H ? 0u : 1u) << 7 | (H ? 0u : 1u) << 10 | (T ? 1u : 0u) << 16 | (uint32_t)(N / 8) << 17 | (128u / 16) << 24;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r, x = *reinterpret_cast<uint64_t*>(&a), y = *reinterpret_cast<uint64_t*>(&b), z = *reinterpret_cast<uint64_t*>(&c);
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t r, x = *reinterpret_cast<uint64_t*>(&a), y = *reinterpret_cast<uint64_t*>(&b);
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return *reinterpret_cast<float2*>(&r);
}

// A bounded wait.  Once one ran out in the CTA (`dead`), every wait ends at once and the roles run on to their ends without
// waiting, over values that mean nothing: no role branches on it, so that warps stay whole; the copies stop.
__device__ __forceinline__ void wait(uint64_t& bar, uint32_t parity, Shared& sh) {
    if (!mbar_try(smem_u32(&bar), parity)) mbar_wait_slow(smem_u32(&bar), parity, sh.limit, &sh.dead);
}

// What the roles, each walking the pieces for itself, ask about one.
struct Pieces : Walk<ChunkLine> {
    using Walk<ChunkLine>::Walk;
    // Rows of a half, and its blocks in the piece: [x, y), empty if no row sees any.
    __device__ __forceinline__ int half_rows(int i) const {
        return min(kHalfRows, at.r.rows - at.rt * kRows - i * kHalfRows);
    }
    __device__ __forceinline__ int2 half_blocks(int i) const {
        const int rows = half_rows(i);
        if (rows <= 0) return make_int2(0, 0);
        const int first = at.rt * kRows + i * kHalfRows;
        const int hi = line.seen(at.r, line.token(first + rows - 1)).y, lo = min(line.seen(at.r, line.token(first)).x, hi);
        const int b0 = max(p0, (lo - at.t.lo) / kKeys), b1 = min(p1, (hi - at.t.lo + kKeys - 1) / kKeys);
        return make_int2(b0, max(b0, b1));
    }
    // Positions that every row of the tile sees.
    __device__ __forceinline__ int2 all_see() const {
        const int first = at.rt * kRows, last = min(first + kRows, at.r.rows) - 1;
        return make_int2(line.seen(at.r, line.token(last)).x, line.seen(at.r, line.token(first)).y);
    }
    __device__ __forceinline__ bool edge(int blk, int2 all) const {
        const int j0 = at.t.lo + blk * kKeys;
        return j0 < all.x || j0 + kKeys > all.y;
    }
};

// Q of a half into shared memory, by its four warps: rows of 16-byte chunks, sixteen (or eight) lanes to a row; arrives at
// `bar` (128 arrivals) once it is there, while the threads go on.  Rows beyond the half's are zero; a negative scale turns Q's
// sign, so that the largest score is the largest product: by ordinary stores, each thread's made known to the tensor cores' proxy
// and released by its arrival (the arrival of asynchronous copies would order none of them).
template <int D>
__device__ __forceinline__ void load_q(const AttendArgs& a, const Pieces& w, int half, uint32_t to, int tid, uint32_t bar) {
    constexpr int C = D / 8, kAtOnce = kHalfRows / C;
    const int rows = w.half_rows(half), c = tid % C, row0 = w.at.rt * kRows + half * kHalfRows;
    const uint32_t at = to + (c >> 3) * (kHalfRows * 128);
    const uint16_t* const q = a.q + (int64_t)w.at.r.q0 * a.q_tok + (int64_t)w.at.h * a.group * a.q_head + c * 8;
#pragma unroll 4
    for (int r = tid / C; r < kHalfRows; r += kAtOnce) {
        const int row = row0 + min(r, rows - 1), tok = w.line.token(row), g = row - tok * a.group;
        const uint16_t* const from = q + (int64_t)tok * a.q_tok + (int64_t)g * a.q_head;
        const uint32_t dst = at + r * 128 + (((c & 7) ^ (r & 7)) << 4);
        if (a.scale >= 0.f) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(from), "r"(r < rows ? 16 : 0) : "memory");
        } else {
            uint4 x = *reinterpret_cast<const uint4*>(from);
            if (r >= rows) x = make_uint4(0, 0, 0, 0);
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(x.x ^ 0x80008000u), "r"(x.y ^ 0x80008000u),
                         "r"(x.z ^ 0x80008000u), "r"(x.w ^ 0x80008000u)
                         : "memory");
        }
    }
    if (a.scale >= 0.f) {
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
    } else {
        fence_proxy_async();
        mbar_arrive(bar);
    }
}

// 16-bit results of 32 columns, 32 or 16 bytes a store.
__device__ __forceinline__ void store_row(uint16_t* to, const uint32_t (&x)[16], bool wide) {
    if (wide) {
#pragma unroll
        for (int i = 0; i < 16; i += 8)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + 2 * i), "r"(x[i]), "r"(x[i + 1]),
                         "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
                         : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4*>(to + 2 * i) = make_uint4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    }
}

// Two scores through the cap, in units of log2: cap2 (1 - 2 / (1 + 2^y)), the two reciprocals from one.  Beyond 2^60 the
// quotient is far below half a unit in the last place of 1; NaN stays NaN (and spreads to both).
__device__ __forceinline__ void cap_pair(uint32_t& x0, uint32_t& x1, float mul, float cap2) {
    float2 y = fma2(make_float2(__uint_as_float(x0), __uint_as_float(x1)), make_float2(mul, mul), make_float2(0.f, 0.f));
    asm("min.NaN.f32 %0, %0, 0f42700000;" : "+f"(y.x));
    asm("min.NaN.f32 %0, %0, 0f42700000;" : "+f"(y.y));
    const float2 a = add2(make_float2(exp2_fast(y.x), exp2_fast(y.y)), make_float2(1.f, 1.f));
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a.x * a.y));
    y = fma2(make_float2(r * a.y, r * a.x), make_float2(-2.f * cap2, -2.f * cap2), make_float2(cap2, cap2));
    x0 = __float_as_uint(y.x);
    x1 = __float_as_uint(y.y);
}

template <bool H, int D, bool CAP>
__global__ void __launch_bounds__(kThreads, 1)
    k_kv_chunk(const AttendArgs a, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
    extern __shared__ __align__(16) char s_raw[];  // 64-bit words of the search first
    __shared__ Shared sh;
    using Sh = Shape<D>;
    constexpr int kTile = Sh::kTile, kStages = Sh::kStages;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_u32(s_raw), smem = (raw + 1023) & ~1023u;
    char* const smem_ptr = s_raw + (smem - raw);
    const uint32_t q_at = smem, kv_at = smem + 2 * kTile;
    ChunkLine line(a);

    if (tid == 0) {
        for (int i = 0; i < kStages; i++) {
            mbar_init(smem_u32(&sh.kv_full[i]), 1);
            mbar_init(smem_u32(&sh.kv_empty[i]), 3);
            mbar_init(smem_u32(&sh.v_clean[i]), 64);
        }
        for (int i = 0; i < 2; i++) {
            mbar_init(smem_u32(&sh.s_full[i]), 1);
            mbar_init(smem_u32(&sh.p_full[i][0]), 4);
            mbar_init(smem_u32(&sh.p_full[i][1]), 4);
            mbar_init(smem_u32(&sh.o_full[i]), 1);
            mbar_init(smem_u32(&sh.q_full[i]), 128);
        }
        mbar_init(smem_u32(&sh.done), 1);
        sh.dead = 0;
        sh.limit = a.wait_ns;
        fence_mbar_init();
    }
    if (warp == 8) tc_alloc(smem_u32(&sh.tmem));

    if (tid == 0) a.joins[blockIdx.x].last = -1;
    sh.part.find(line, s_raw);
    clear_rest<D, kThreads>(line);
    fence_proxy_async();  // the tiles' memory served as scratch
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;

    bool range = false;
    if (!sh.part.empty()) {
        if (warp < 8) {
            // ---------------------------------------------------------- weights and results of a half
            const int half = warp >> 2, row_in = tid & 127;
            const uint32_t lanes = (uint32_t)(warp & 3) << 21;
            const uint32_t s_at = tmem + half * 128 + lanes, o_at = tmem + 256 + half * D + lanes;
            const float cap2 = a.cap * kLog2e, scale = fmaxf(fabsf(a.scale), 0x1p-100f);
            const float mul_in = CAP ? 2.f * kLog2e * scale / a.cap : kLog2e * scale, mul = CAP ? 1.f : mul_in;
            const bool wide = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(2 * a.out_tok) | (uintptr_t)(2 * a.out_head)) & 31) == 0;
            uint32_t n_s = 0, n_o = 0;  // products awaited so far
            int note = 0;               // blocks of the stretch before this piece
            Pieces w(line, sh.part);
            bool loaded = false;
            while (w.more) {
                const int rows = w.half_rows(half);
                const int2 blocks = w.half_blocks(half);
                if (!loaded && blocks.x < blocks.y) load_q<D>(a, w, half, q_at + half * kTile, row_in, smem_u32(&sh.q_full[half]));
                loaded = false;
                const int row = w.at.rt * kRows + half * kHalfRows + row_in, tok = line.token(row);
                const bool valid = row_in < rows;
                const int2 see = valid ? line.seen(w.at.r, tok) : make_int2(0, 0x7fffffff);
                // Blocks inside [whole_lo, whole_hi) are seen whole by every row of the warp.
                const int whole_lo = __reduce_max_sync(~0u, see.x), whole_hi = __reduce_min_sync(~0u, see.y);
                float m = -INFINITY, l = 0.f;  // m in units of log2
                for (int blk = blocks.x; blk < blocks.y; blk++) {
                    wait(sh.s_full[half], n_s & 1, sh);
                    __syncwarp();
                    n_s++;
                    tc_fence_after();
                    const int j0 = w.at.t.lo + blk * kKeys;
                    const uint32_t skip = sh.skip[(note + blk - w.p0) & (kNotes - 1)];
                    const bool masked = j0 < whole_lo || j0 + kKeys > whole_hi || skip;
                    // What the row sees of the block's positions 32 i .. 32 i + 31.
                    auto keeps = [&](int i) {
                        const int x = min(max(see.x - j0 - 32 * i, 0), 32), y = min(max(see.y - j0 - 32 * i, 0), 32);
                        return (y == 32 ? ~0u : (1u << y) - 1u) & (x == 32 ? 0u : ~0u << x) & (skip >> (2 * i) & 1 ? 0xffff0000u : ~0u) &
                               (skip >> (2 * i + 1) & 1 ? 0xffffu : ~0u);
                    };
                    auto put = [](auto& x, uint32_t keep, uint32_t v) {
#pragma unroll
                        for (int c = 0; c < (int)(sizeof(x) / 4); c++)
                            if (!(keep >> c & 1)) x[c] = v;
                    };
                    float tops[4];
                    uint32_t s[1][32];
                    if (CAP) {  // 32 positions at a time, and back.  Rolled: unrolled, the loop leaves the instruction cache
                        tops[0] = tops[1] = tops[2] = tops[3] = -INFINITY;
#pragma unroll 1
                        for (int i = 0; i < 4; i++) {
                            tc_load32(s[0], s_at + 32 * i);
                            const uint32_t keep = masked ? keeps(i) : ~0u;
                            tc_wait_ld(s);
                            if (masked) put(s[0], keep, 0u);  // a NaN that the row does not see would spread
#pragma unroll
                            for (int c = 0; c < 32; c += 2) cap_pair(s[0][c], s[0][c + 1], mul_in, cap2);
                            if (masked) put(s[0], keep, 0xff800000u);
#pragma unroll
                            for (int c = 0; c < 32; c += 2)
                                tops[c >> 1 & 3] = max3(tops[c >> 1 & 3], __uint_as_float(s[0][c]), __uint_as_float(s[0][c + 1]));
                            tc_store32(s_at + 32 * i, s[0]);
                        }
                        tc_wait_st();
                    } else {
                        tops[0] = tops[1] = tops[2] = tops[3] = -INFINITY;
                        // S is read twice, 32 positions at a time: held whole (128 values a thread) and unrolled, the loop left the
                        // instruction cache and the mixed batch took 128 us instead of 122.
#pragma unroll 2
                        for (int i = 0; i < 4; i++) {
                            tc_load32(s[0], s_at + 32 * i);
                            tc_wait_ld(s);
                            if (masked) put(s[0], keeps(i), 0xff800000u);
#pragma unroll
                            for (int c = 0; c < 32; c += 2)
                                tops[c >> 1 & 3] = max3(tops[c >> 1 & 3], __uint_as_float(s[0][c]), __uint_as_float(s[0][c + 1]));
                        }
                    }
                    const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * mul;
                    // Raise the maximum that the weights refer to, and rescale what is summed: rarely.
                    const bool raise = raises<H>(top, m);
                    if (__any_sync(~0u, raise)) {
                        const float to = raise ? top : m, keep = raise ? exp2_fast(m - to) : 1.f;
                        m = to;
                        l *= keep;
                        if (blk > blocks.x) {
                            wait(sh.o_full[half], (n_o - 1) & 1, sh);
                            __syncwarp();
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[1][16];
                                tc_load16(o[0], o_at + c);
                                tc_wait_ld(o);
#pragma unroll
                                for (int i = 0; i < 16; i++) o[0][i] = __float_as_uint(__uint_as_float(o[0][i]) * keep);
                                tc_store16(o_at + c, o[0]);
                            }
                        }
                    }
                    const float shift = (m == -INFINITY ? 0.f : m) - kLift<H>;
                    float2 sum[4] = {};
#pragma unroll 2
                    for (int i = 0; i < 4; i++) {
                        float2 y[16];
                        uint32_t p[16];
                        uint32_t(&x)[32] = s[0];
                        tc_load32(x, s_at + 32 * i);
                        tc_wait_ld(s);
                        if (!CAP && masked) put(x, keeps(i), 0xff800000u);
#pragma unroll
                        for (int c = 0; c < 16; c++) {
                            y[c] = fma2(make_float2(__uint_as_float(x[2 * c]), __uint_as_float(x[2 * c + 1])), make_float2(mul, mul),
                                        make_float2(-shift, -shift));
                            y[c] = make_float2(exp2_fast(y[c].x), exp2_fast(y[c].y));
                        }
#pragma unroll
                        for (int c = 0; c < 16; c++) {
                            sum[c & 3] = add2(sum[c & 3], y[c]);
                            p[c] = pack2<H>(y[c].x, y[c].y);
                        }
                        tc_store16(s_at + 16 * i, p);
                        if (i & 1) {  // half of the positions: their product can start
                            tc_wait_st();
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(smem_u32(&sh.p_full[half][i >> 1]));
                            __syncwarp();
                        }
                    }
                    sum[0] = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
                    l += sum[0].x + sum[0].y;
                    n_o++;
                }
                // The next piece's Q while the last product runs.
                const Pieces cur = w;
                note += cur.p1 - cur.p0;
                w.next();
                if (w.more && blocks.x < blocks.y) {
                    const int2 nb = w.half_blocks(half);
                    if (nb.x < nb.y) {
                        load_q<D>(a, w, half, q_at + half * kTile, row_in, smem_u32(&sh.q_full[half]));
                        loaded = true;
                    }
                }
                const bool some = blocks.x < blocks.y;
                if (some) {
                    wait(sh.o_full[half], (n_o - 1) & 1, sh);
                    __syncwarp();
                    tc_fence_after();
                }
                if (rows <= 0) continue;
                const int cta = blockIdx.x, g = row - tok * a.group, h = cur.at.h * a.group + g;
                const int64_t t = cur.at.r.q0 + tok;
                const bool whole = cur.whole(sh.part), begins = cur.begins(sh.part);
                const float inv = l == 0.f ? 0.f : 1.f / l;
                float* const piece = a.pieces + (int64_t)(2 * cta + begins) * Sh::kPieceFloats;
                const int prow = half * kHalfRows + row_in;
                int2 odd = make_int2(1, 0);
                const int2 all = cur.all_see();
                if (some && (cur.edge(cur.p0, all) || cur.edge(cur.p1 - 1, all))) {  // else nobody looked
                    const int2 x = sh.odd[0][cur.piece & (kNotes - 1)], y = sh.odd[1][cur.piece & (kNotes - 1)];
                    odd = make_int2(min(x.x, y.x), max(x.y, y.y));
                }
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    __syncwarp();  // lanes came through loops of their own; the load takes a whole warp
                    uint32_t got[1][32];
                    uint32_t(&o)[32] = got[0];
                    if (some) {
                        tc_load32(o, o_at + c);
                        tc_wait_ld(got);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; i++) o[i] = 0u;
                    }
                    if (valid && odd.x <= odd.y) {  // what was replaced by 0, for the rows that see it
                        const int j1 = min(see.y, cur.at.t.lo + (odd.y + 1) * kKeys);
                        for (int j = max(see.x, cur.at.t.lo + odd.x * kKeys); j < j1; j++) {
                            const int page = a.table[(int64_t)cur.at.b * a.max_pages + (j >> a.page_shift)];
                            if ((uint32_t)page >= (uint32_t)a.n_pages) continue;
                            const uint16_t* v = a.v + page * a.v_page + (j & ((1 << a.page_shift) - 1)) * a.v_slot + cur.at.h * a.v_head + c;
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const uint32_t x = *reinterpret_cast<const uint32_t*>(v + i);
                                if (!any_nonfinite<H>(x)) continue;
                                const float2 f = unpack2<H>(x);
                                if (!isfinite(f.x)) o[i] = __float_as_uint(__uint_as_float(o[i]) + f.x);
                                if (!isfinite(f.y)) o[i + 1] = __float_as_uint(__uint_as_float(o[i + 1]) + f.y);
                            }
                        }
                    }
                    if (valid && whole) {
                        uint32_t x[16];
#pragma unroll
                        for (int i = 0; i < 16; i++) x[i] = pack2<H>(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
                        store_row(a.out + t * a.out_tok + h * a.out_head + c, x, wide);
                    } else if (valid) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            reinterpret_cast<uint4*>(piece)[(c + i) / 4 * kRows + prow] = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    }
                }
                if (valid) {
                    if (whole) {
                        if (a.lse) a.lse[t * a.heads + h] = log_sum<H>(m, l);
                    } else {
                        reinterpret_cast<float2*>(piece + kRows * D)[prow] = make_float2(m, l);
                    }
                }
                if (!whole && begins && row_in == 0 && half == 0) {
                    Join& j = a.joins[cta];
                    j.q0 = cur.at.r.q0;
                    j.h = cur.at.h;
                    j.row0 = cur.at.rt * kRows;
                    j.rows = min(kRows, cur.at.r.rows - j.row0);
                    j.last = (int)divide(cur.at.start + cur.at.t.blocks - 1, sh.part.share);
                }
                __syncwarp();
                tc_fence_before();
            }
            // Q that nobody waited for, once a wait ran out, must land before the CTA's memory is given away.
            asm volatile("cp.async.wait_all;" ::: "memory");
        } else {
            Pieces w(line, sh.part);
            int stage = 0;
            uint32_t round = 0;  // of the ring
            auto advance = [&] {
                if (++stage == kStages) {
                    stage = 0;
                    round ^= 1;
                }
            };
            if (warp == 8) {
                // ------------------------------------------------------ products
                // The whole warp takes part and one elected lane issues: descriptors and addresses stay in uniform registers
                // (issued by a lane in a branch of its own, a product of 64 cycles took 90 to issue).
                constexpr uint32_t kIdS = instruction<H, 128, false>(), kIdO = instruction<H, D, true>();
                const uint32_t tm = __shfl_sync(~0u, tmem, 0);
                uint32_t n_p[2] = {0, 0}, n_q[2] = {0, 0}, clean = 0;
                bool act_prev[2] = {false, false}, first_prev[2] = {false, false}, any_prev = false;
                int v_prev = 0;
                // O += P V of the block before, half i, as its weights come in two parts; `last`: V's stage is free after it.
                auto issue_o = [&](int i, bool last) {
                    const uint64_t vd = descriptor(__shfl_sync(~0u, kv_at + v_prev * kTile, 0), kKeys * 128, 1024);
                    const bool add = __shfl_sync(~0u, !first_prev[i], 0);
                    const uint32_t free = smem_u32(&sh.kv_empty[v_prev]);
#pragma unroll
                    for (int part = 0; part < 2; part++) {
                        if (act_prev[i]) {
                            wait(sh.p_full[i][part], n_p[i] & 1, sh);
                            tc_fence_after();
                        }
                        __syncwarp();
                        if (elect_one()) {
                            if (act_prev[i]) {
#pragma unroll
                                for (int k = 4 * part; k < 4 * part + 4; k++)
                                    tc_mma_t(tm + 256 + i * D, tm + i * 128 + k * 8, vd + k * 128, kIdO, k > 0 || add);
                                if (part == 1) tc_commit(smem_u32(&sh.o_full[i]));
                            }
                            if (part == 1 && last) tc_commit(free);
                        }
                        __syncwarp();
                    }
                    n_p[i] += act_prev[i];
                };
                while (w.more) {
                    int2 hb[2] = {w.half_blocks(0), w.half_blocks(1)};
                    const int2 all = w.all_see();
                    for (int blk = w.p0; blk < w.p1; blk++) {
                        const uint32_t k_at = kv_at + stage * kTile, k_free = smem_u32(&sh.kv_empty[stage]);
                        uint64_t& k_full = sh.kv_full[stage];
                        const uint32_t k_round = round;
                        advance();
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            if (any_prev) issue_o(i, i == 1);
                            const bool act = blk >= hb[i].x && blk < hb[i].y;
                            if (i == 0) wait(k_full, k_round, sh);
                            if (act && blk == hb[i].x) {
                                wait(sh.q_full[i], n_q[i]++ & 1, sh);
                                fence_proxy_async();  // Q came by ordinary copies
                            }
                            tc_fence_after();
                            const uint64_t qd = descriptor(__shfl_sync(~0u, q_at + i * kTile, 0), 16, 1024);
                            const uint64_t kd = descriptor(__shfl_sync(~0u, k_at, 0), 16, 1024);
                            if (elect_one()) {
                                if (act) {
#pragma unroll
                                    for (int k = 0; k < D / 16; k++) {
                                        const uint32_t off = ((k >> 2) * (kKeys * 128) + (k & 3) * 32) >> 4;
                                        tc_mma(tm + i * 128, qd + off, kd + off, kIdS, k > 0);
                                    }
                                    tc_commit(smem_u32(&sh.s_full[i]));
                                }
                                if (i == 1) tc_commit(k_free);
                            }
                            __syncwarp();
                            act_prev[i] = act;
                            first_prev[i] = blk == hb[i].x;
                        }
                        // V of this block, while S is computed.
                        v_prev = stage;
                        any_prev = true;
                        wait(sh.kv_full[stage], round, sh);
                        if (w.edge(blk, all)) {
                            wait(sh.v_clean[stage], clean >> stage & 1, sh);
                            clean ^= 1u << stage;
                        }
                        advance();
                    }
                    w.next();
                }
                issue_o(0, false);
                issue_o(1, true);
                // Everything issued is done before tensor memory is given back.
                __syncwarp();
                if (elect_one()) tc_commit(smem_u32(&sh.done));
                __syncwarp();
                if (!mbar_try(smem_u32(&sh.done), 0) && !mbar_wait_slow(smem_u32(&sh.done), 0, a.wait_ns, nullptr)) sh.dead = 1;
                __syncwarp();
            } else if (warp == 9) {
                // ------------------------------------------------------ copies
                bool ok = true;
                uint32_t turns = 0;
                int note = 0;
                const int n = kKeys >> a.page_shift;
                while (w.more && ok) {
                    const int seen_lo = line.seen(w.at.r, line.token(w.at.rt * kRows)).x;
                    for (int blk = w.p0; blk < w.p1 && ok; blk++, note++) {
                        const int j = w.at.t.lo + blk * kKeys + (lane << a.page_shift);
                        int page = a.n_pages;  // past the last page: zeros
                        bool none = false;
                        if (lane < n && j < w.at.t.hi && j + (1 << a.page_shift) > seen_lo) {  // else no row's business
                            page = a.table[(int64_t)w.at.b * a.max_pages + (j >> a.page_shift)];
                            if ((uint32_t)page >= (uint32_t)a.n_pages) {
                                page = a.n_pages;
                                none = true;
                                range = true;
                            }
                        }
                        const uint32_t nones = __ballot_sync(~0u, none);
                        uint32_t skip = 0;
                        if (nones) {
                            for (int i = 0; i < kKeys / 16; i++)
                                if (nones >> (16 * i >> a.page_shift) & 1) skip |= 1u << i;
                        }
                        if (lane == 0) sh.skip[note & (kNotes - 1)] = skip;
                        __syncwarp();
                        for (int v = 0; v < 2; v++) {
                            if (turns >= (uint32_t)kStages) wait(sh.kv_empty[stage], round ^ 1, sh);
                            ok = __all_sync(~0u, *(volatile int*)&sh.dead == 0);
                            if (!ok) break;
                            const uint32_t bar = smem_u32(&sh.kv_full[stage]), to = kv_at + stage * kTile + (lane << a.page_shift) * 128;
                            const bool skip_it = a.skip == note;  // a test's wait that runs out
                            if (lane == 0 && !skip_it) mbar_expect(bar, kTile);
                            __syncwarp();
                            if (lane < n && !skip_it) {
#pragma unroll
                                for (int d = 0; d < D / 64; d++)
                                    load_box(to + d * (kKeys * 128), v ? &vmap : &kmap, d * 64, 0, w.at.h, page, bar);
                            }
                            turns++;
                            advance();
                        }
                    }
                    w.next();
                }
                if (!ok) {  // what is in flight must land before the CTA's memory is given away
                    const uint32_t left = turns < (uint32_t)kStages ? turns : kStages;
                    for (uint32_t i = 0; i < left; i++) {
                        stage = stage == 0 ? kStages - 1 : stage - 1;
                        if (stage == kStages - 1) round ^= 1;
                        const uint32_t bar = smem_u32(&sh.kv_full[stage]);
                        if (!mbar_try(bar, round)) mbar_wait_slow(bar, round, a.wait_ns, nullptr);
                    }
                }
            } else {
                // ------------------------------------------------------ V that not every row sees
                const int part = warp - 10;
                while (w.more) {
                    const int2 all = w.all_see();
                    const int seen_lo = line.seen(w.at.r, line.token(w.at.rt * kRows)).x;
                    int2 odd = make_int2(0x7fffffff, -1);
                    if (lane == 0) sh.odd[part][w.piece & (kNotes - 1)] = odd;
                    for (int blk = w.p0; blk < w.p1; blk++) {
                        for (int v = 0; v < 2; v++) {
                            wait(sh.kv_full[stage], round, sh);
                            __syncwarp();
                            if (v && w.edge(blk, all)) {
                                uint4* const at = reinterpret_cast<uint4*>(smem_ptr + 2 * kTile + stage * kTile + part * (kTile / 2));
                                const int j0 = w.at.t.lo + blk * kKeys + (D == 64 ? part * (kKeys / 2) : 0);
                                bool found = false;
#pragma unroll 4
                                for (int i = lane; i < kTile / 32; i += 32) {
                                    uint4 x = at[i];
                                    uint32_t* const e = reinterpret_cast<uint32_t*>(&x);
                                    if (any_nonfinite<H>(x.x) || any_nonfinite<H>(x.y) || any_nonfinite<H>(x.z) || any_nonfinite<H>(x.w)) {
                                        const int j = j0 + (i >> 3);
                                        found |= j >= seen_lo && j < w.at.t.hi;
                                        for (int k = 0; k < 4; k++) {
                                            const float2 f = unpack2<H>(e[k]);
                                            e[k] &= (isfinite(f.x) ? 0xffffu : 0u) | (isfinite(f.y) ? 0xffff0000u : 0u);
                                        }
                                        at[i] = x;
                                    }
                                }
                                if (__any_sync(~0u, found)) {
                                    odd = make_int2(min(odd.x, blk), blk);
                                    if (lane == 0) sh.odd[part][w.piece & (kNotes - 1)] = odd;
                                }
                                fence_proxy_async();
                                __syncwarp();
                                mbar_arrive(smem_u32(&sh.v_clean[stage]));
                            }
                            __syncwarp();
                            if (lane == 0) mbar_arrive(smem_u32(&sh.kv_empty[stage]));
                            advance();
                        }
                    }
                    w.next();
                }
            }
        }
    }
    if (__any_sync(~0u, range || line.bad) && lane == 0) atomicOr(a.err, kKvErrRange);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (tid == 0 && sh.dead) atomicOr(a.err, kKvErrTimeout);
    if (warp == 8) tc_free(tmem);
    asm volatile("griddepcontrol.wait;" ::: "memory");  // a launch for few rows before this one, which ran beside it, is done
}

// Joins the pieces of tiles that cross CTAs: block (c, g) the rows 32 g .. 32 g + 31 of the tile whose first piece is the
// last of CTA c; eight threads a row's sums, lanes along the rows as the pieces are laid out.  Bound by the latency of its
// dependent reads (what to join, the pieces), so many threads read little each, four pieces at a time.
constexpr int kJoinThreads = 256, kJoinRows = 32, kJoinAtOnce = 4;

template <bool H, int D>
__global__ void __launch_bounds__(kJoinThreads) k_kv_join(const AttendArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Join j = a.joins[blockIdx.x];
    const int row_in = blockIdx.y * kJoinRows + (threadIdx.x & 31), part = threadIdx.x >> 5;
    if (j.last < 0 || row_in >= j.rows) return;
    constexpr int kFloats = Shape<D>::kPieceFloats, N = D * 8 / kJoinThreads;  // 16-byte vectors of a part
    float m = -INFINITY, l = 0.f;
    float4 o[N];
#pragma unroll
    for (int i = 0; i < N; i++) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = blockIdx.x; c0 <= j.last; c0 += kJoinAtOnce) {
        float2 ml[kJoinAtOnce];
        float4 x[kJoinAtOnce][N];
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; k++) {
            const int c = min(c0 + k, j.last);
            const float* const piece = a.pieces + (int64_t)(2 * c + (c == (int)blockIdx.x)) * kFloats;
            ml[k] = reinterpret_cast<const float2*>(piece + kRows * D)[row_in];
            if (c0 + k > j.last) ml[k] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int i = 0; i < N; i++) x[k][i] = reinterpret_cast<const float4*>(piece)[(part * N + i) * kRows + row_in];
        }
        float to = m;
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; k++) to = fmaxf(to, ml[k].x);
        const float shift = to == -INFINITY ? 0.f : to, keep = exp2_fast(m - shift);
        m = to;
        l *= keep;
#pragma unroll
        for (int i = 0; i < N; i++) o[i] = make_float4(o[i].x * keep, o[i].y * keep, o[i].z * keep, o[i].w * keep);
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; k++) {
            if (c0 + k > j.last) break;
            const float f = exp2_fast(ml[k].x - shift);
            l += ml[k].y * f;
#pragma unroll
            for (int i = 0; i < N; i++)
                o[i] = make_float4(fmaf(x[k][i].x, f, o[i].x), fmaf(x[k][i].y, f, o[i].y), fmaf(x[k][i].z, f, o[i].z), fmaf(x[k][i].w, f, o[i].w));
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const ChunkLine line(a);
    const int row = j.row0 + row_in, tok = line.token(row), h = j.h * a.group + row - tok * a.group;
    const int64_t t = j.q0 + tok;
    uint2* const out = reinterpret_cast<uint2*>(a.out + t * a.out_tok + h * a.out_head + part * (4 * N));
#pragma unroll
    for (int i = 0; i < N; i++) out[i] = make_uint2(pack2<H>(o[i].x * inv, o[i].y * inv), pack2<H>(o[i].z * inv, o[i].w * inv));
    if (a.lse && part == 0) a.lse[t * a.heads + h] = log_sum<H>(m, l);
}

template <bool H, int D>
cudaError_t prepare() {
    const cudaError_t e = cudaFuncSetAttribute(k_kv_chunk<H, D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D>::kSmem);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(k_kv_chunk<H, D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D>::kSmem);
}

template <bool H, int D>
cudaError_t launch(const AttendArgs& a, const KvMaps& maps, bool after_few, int sms, cudaStream_t s) {
    cudaLaunchAttribute early[1];  // starts while the launch before ends
    early[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(sms);
    c.blockDim = dim3(kThreads);
    c.dynamicSmemBytes = Shape<D>::kSmem;
    c.stream = s;
    c.attrs = early;
    c.numAttrs = after_few ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&c, a.cap > 0.f ? k_kv_chunk<H, D, true> : k_kv_chunk<H, D, false>, a, maps.k, maps.v);
    if (e != cudaSuccess) return e;
    c.gridDim = dim3(sms, kRows / kJoinRows);
    c.blockDim = dim3(kJoinThreads);
    c.dynamicSmemBytes = 0;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, k_kv_join<H, D>, a);
}

}  // namespace

size_t kv_chunk_piece_bytes(int sms) { return (size_t)sms * 2 * Shape<128>::kPieceFloats * sizeof(float); }

cudaError_t kv_chunk_prepare() {
    cudaError_t e;
    if ((e = prepare<false, 64>()) != cudaSuccess || (e = prepare<true, 64>()) != cudaSuccess ||
        (e = prepare<false, 128>()) != cudaSuccess)
        return e;
    return prepare<true, 128>();
}

cudaError_t launch_kv_chunk(const AttendArgs& a, const KvMaps& maps, bool after_few, int sms, cudaStream_t s) {
    if (a.half) return a.head_dim == 128 ? launch<true, 128>(a, maps, after_few, sms, s) : launch<true, 64>(a, maps, after_few, sms, s);
    return a.head_dim == 128 ? launch<false, 128>(a, maps, after_few, sms, s) : launch<false, 64>(a, maps, after_few, sms, s);
}

}  // namespace kvdro
