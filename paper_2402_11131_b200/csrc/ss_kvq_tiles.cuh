// Attention over a 4-bit prefix for blocks of more rows than a warp can hold, on tcgen05.  Included by ss_attention_kvq.cu.
//
// S^T = K Q^T and O^T = V^T P^T with 128 keys (dimensions) as the 128 lanes of TMEM and the N <= 64 query rows as columns: what
// grows with the rows is the cheap side, and codes go from registers to TMEM as A operands, never through shared memory.
//   K: the thread of a key turns the key's codes into bf16 c - z, exactly (128 + c by a mask and an or, less 128 + z), one TMEM lane; the key's
//      scale multiplies the lane's scores.
//   V: transposing loads (ldmatrix, 16 keys by 16 bytes) give a thread four keys' codes of two dimensions; a TMEM lane is a dimension.
//      The scale is part of the weight that meets it.
// Lane 32 w + x of V^T and O^T (w < D / 32) holds, for x < 16, the low codes of byte 16 w + x of a row, else the high codes of
// byte 16 w + x - 16.
//
// 28 warps: 0..3 copy the codes of K and V and turn K's into operands, 4..7 V's, 8..23 softmax (four groups of four, each a quarter of
// the rows, thread = key), 24 issues the MMAs, 25..27 prepare: they walk the list of units one ahead of the others, who find a
// unit's query rows and what else they need to know of it in shared memory.  Two buffers each for K, V, S, P and the query rows, so that
// the roles work on different tiles and units.
//
// What bounds it: each role's chain of latencies per tile (loads, conversion, TMEM round trip, hand-over), some 1800 to 2300 cycles of 128 keys
// by 64 rows whatever the role, where the MMAs need 300 and the exponentials 512: 16 users with 512 to 4096 keys 103 us for 27.5 of HBM.
// On the way there: one softmax group per 32 rows 143 us, four 130; weights without a vote on the references 118 (a sum per tile
// decides) against 112; a unit's start counted in the deal of work 112 for 131; own warps for what comes before a unit 107.
// Registers (72 each, all there are) decide too: what is called seldom is out of line where the loops around it then spill less (rows and
// the wait for a unit: 104, inline 121; not the join: 125).
// Rounding: keys and values are whole numbers from -15 to 15 in bf16, exactly; queries enter as they are; a weight p s_v is rounded once to
// bf16 (2^-8 of itself), as the bf16 attention rounds p.  Sums of q (c - z) are as large as the score's own terms, so a score is off by
// some d / 16 steps of 2^-24 of sum |q k|.  (As sums of q (128 + c) less (128 + z) sum q, which saves a subtraction per two codes, scores of queries
// with a mean and keys with a large channel were off by 3 10^-3; in time the subtractions and the additional step of the product are the same.)
#pragma once
#include "ss_tcgen05.cuh"

namespace ss {

// A unit's start and end take as long as some four tiles.
constexpr int kTileStart = 4;
constexpr int kTileOfKeys = 128, kTileGroups = 4, kTileSoftmax = 128 * kTileGroups, kTilePrepare = 96, kTileThreads = 256 + kTileSoftmax + 32 + kTilePrepare;
constexpr int kTileWarpsOfUnit = (kTileThreads - kTilePrepare) / 32;             // that use a unit's plan

template <int D, int N>
struct TileGeo {
    static constexpr int kRowsOfGroup = N / kTileGroups;          // rows of a softmax group
    static constexpr int kPitch = D == 128 ? 64 : D == 80 ? 48 : 32;         // bytes of a key's codes in shared memory (16-byte aligned)
    static constexpr int kCopy = D == 80 ? 8 : 16, kPer = D / 2 / kCopy;     // asynchronous copies per key
    static constexpr int kWords = D / 8;
    static constexpr int kQuads = (D + 31) / 32;                  // warps that have V lanes
    static constexpr int kCodes = kTileOfKeys * kPitch;
    static constexpr int kStages = 4, kParams = 8;
    static constexpr int kBoxes = D > 64 ? 2 : 1, kBox = N * 128;
    static constexpr int kRowOfV = 64 * kQuads;                   // bytes of a bf16 row in lane order
    static constexpr int kP = kTileOfKeys * 128;
    static constexpr int oP = 0, oQ = oP + 2 * kP, kRowsOfUnit = kBoxes * kBox, oK = oQ + 2 * kRowsOfUnit, oV = oK + kStages * kCodes;
    static constexpr int oRows = oV + kStages * kCodes;           // 64 rows of bf16 values in the order of the lanes
    static constexpr int oKParams = oRows + 64 * kRowOfV, oVParams = oKParams + kParams * kTileOfKeys * 4;
    static constexpr int kBytes = oVParams + kParams * kTileOfKeys * 4;
    static constexpr uint32_t kTmemK = 0, kTmemV = 128, kTmemS = 256, kTmemO = 256 + 2 * N;          // K and V: 64 columns a buffer
    // bf16 operands, fp32 sums, 128 lanes, N columns; P^T is MN-major
    static constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(N >> 3) << 17) | ((128u >> 4) << 24);
    static constexpr uint32_t kIdescPV = kIdescS | (1u << 16);
};

// What the roles have to know of a unit
struct TileUnit {
    int L, T, prefix, from, to;                      // of the sequence; tiles of cached slots, and those of this piece
    int head, real, row0, rows, b;                   // real: there is such a head; rows: of the block
    int whole, first, last, second, me, member, team;            // see Pieces
    int done;                                        // no unit: the list is at its end
    long long start;
    Extra extra;
    long long out[64];                               // where a row's output goes (element offset)
    unsigned long long see[64];                      // per node: the rows that see it
};

// Asynchronous copies of a tile's codes by 128 threads, 16 (8) bytes each, from a pointer that walks along with the tiles.  Slots behind
// the last one are read as the last one again (their weights are zero).
template <int D, int N>
struct TileLoader {
    using G = TileGeo<D, N>;
    static constexpr bool kEven = 128 % G::kPer == 0;
    long long at;                                    // of the next tile: the thread's first copy (80: key 0), in either array of codes
    int left;                                        // slots from there on
    __device__ __forceinline__ TileLoader(const KvqArgs& a, const TileUnit& u, int tile, int t) {
        const long long slot = u.start + static_cast<long long>(tile) * kTileOfKeys + (kEven ? t / G::kPer : 0);
        at = slot * a.slot_stride + u.head * a.head_stride + (kEven ? t % G::kPer * G::kCopy : 0);
        left = u.L - tile * kTileOfKeys;
    }
    __device__ __forceinline__ uint32_t place(int row, int column) const {
        return row * G::kPitch + (D == 128 ? column ^ ((row >> 1) & 3) : D == 64 ? column ^ ((row >> 2) & 1) : column) * G::kCopy;
    }
    __device__ __forceinline__ void next(const KvqArgs& a, uint32_t k_stage, uint32_t v_stage, int t) {
        if (kEven && left >= kTileOfKeys) {
            // (the swizzle is the same for all of the thread's rows: they are a multiple of 8 apart)
            const uint32_t dst = place(t / G::kPer, t % G::kPer);
            #pragma unroll
            for (int i = 0; i < G::kPer; ++i) copy_async<G::kCopy>(k_stage + dst + i * (128 / G::kPer) * G::kPitch, a.k_codes + at + i * (128 / G::kPer) * a.slot_stride);
            #pragma unroll
            for (int i = 0; i < G::kPer; ++i) copy_async<G::kCopy>(v_stage + dst + i * (128 / G::kPer) * G::kPitch, a.v_codes + at + i * (128 / G::kPer) * a.slot_stride);
        } else {
            const int last = left - 1;
            #pragma unroll 1
            for (int i = 0; i < G::kPer; ++i) {
                const int item = i * 128 + t, row = item / G::kPer, column = item - row * G::kPer;
                const long long from = at + (kEven ? (min(row, last) - t / G::kPer) * a.slot_stride : min(row, last) * a.slot_stride + column * G::kCopy);
                copy_async<G::kCopy>(k_stage + place(row, column), a.k_codes + from);
                copy_async<G::kCopy>(v_stage + place(row, column), a.v_codes + from);
            }
        }
        at += kTileOfKeys * a.slot_stride;
        left -= kTileOfKeys;
    }
};

struct alignas(8) TileWaits {
    int abort;                                       // a wait has run out
    int limit;                                       // bound of waits for data, in units of 1024 cycles
};

template <int C>
struct TileCtrl {
    unsigned long long k_full[2], s_full[2], s_free[2], v_full[2], p_full[2], pv_done[2], o_free, drain;
    unsigned long long codes_full[4], codes_free[4];              // V's codes
    unsigned long long plan_full[2], rows_full[2], plan_free[2];
    unsigned long long vote[kTileGroups][2];                      // the warps of a group have looked at their scores
    TileUnit unit[2];
    float neg_ref[64];
    int tile_max[kTileGroups][4][C];
    float sums[kTileGroups][4][C];
    int hot[kTileGroups][2];                                      // a reference has to go up
    uint32_t tmem;
    int joined, any;
    TileWaits waits;
};

// Two kinds of waits.
// Waits for data (codes, operands, products, buffers) end at their bound, and at once when one of them has ended so: from then on the CTA goes
// through its tiles without them, on whatever the buffers hold, and nothing of that is used.  The bound is the caller's (workspace word
// 1), but for the softmax warps a second: they wait for products alone, for whose buffers the others wait as well, and have no registers for
// more (with the caller's bound there, spills in their loop: 16 users 119 for 103 us).
// Waits for the other warps' steps, which decide where a warp goes next (units' plans, a group's vote), are never left early: plans are not
// overwritten under their readers, warps that meet at barriers take the same branches, and addresses are those of the plan.  They end all the
// same: they wait for arrivals alone, which come as soon as the other warps' waits for data have ended.  That may take as long as the longest
// unit (2^24 tiles of some 2000 cycles, 3.4 10^10 cycles), so their bound is 1.3 10^11.
__device__ __forceinline__ uint32_t kilocycles() { return static_cast<uint32_t>(clock64() >> 10); }
static __device__ __noinline__ void wait_for_warps_slow(uint32_t bar, uint32_t parity, volatile TileWaits* w) {
    const uint32_t t0 = kilocycles();
    while (!mbar_try(bar, parity)) {
        if (kilocycles() - t0 > static_cast<uint32_t>(64 * kWaitCycles >> 10)) {
            w->abort = 1;
            return;
        }
    }
}
static __device__ __noinline__ void wait_for_data_slow(uint32_t bar, uint32_t parity, volatile TileWaits* w) {
    const uint32_t t0 = kilocycles();
    while (!mbar_try(bar, parity)) {
        if (w->abort) return;
        if (kilocycles() - t0 > static_cast<uint32_t>(w->limit)) {
            w->abort = 1;
            return;
        }
    }
}
static __device__ __noinline__ void wait_for_product_slow(uint32_t bar, uint32_t parity, volatile int* abort) {
    const uint32_t t0 = static_cast<uint32_t>(clock());
    while (!mbar_try(bar, parity)) {
        if (*abort) return;
        if (static_cast<uint32_t>(clock()) - t0 > static_cast<uint32_t>(kWaitCycles)) {
            *abort = 1;
            return;
        }
    }
}

template <int C>
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[C]) {
    static_assert(C == 8 || C == 16, "columns");
    if constexpr (C == 16) tmem_ld16<0>(addr, r);
    else
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr) : "memory");
}
// 8 or 32 columns
template <int C, int M>
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[M]) {
    static_assert(C == 8 || (C == 32 && M == 32), "columns");
    if constexpr (C == 32) tmem_st32(addr, r);
    else
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
                     ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(addr) : "memory");
}
// 16 lanes by 32 columns: r[2 k + e] is column 4 k + lane % 4 of TMEM lane lane / 4 + 8 e
__device__ __forceinline__ void tmem_store_lanes16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::SS_W16(r, 0), "r"(addr) : "memory");
}
// STEPS (1 or 4) steps of 16 with A in TMEM (8 columns a step), by the warp's elected lane; B K-major (32 bytes a step)
template <int STEPS>
__device__ __forceinline__ void tile_mma(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    const uint32_t blo = static_cast<uint32_t>(b), bhi = static_cast<uint32_t>(b >> 32);
    if constexpr (STEPS == 1)
        asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 b;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 b, {%2, %3};\n\t"
                     "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}" ::"r"(d), "r"(a), "r"(blo), "r"(bhi), "r"(idesc), "r"(acc) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, e, t;\n\t.reg .b32 x, y;\n\t.reg .b64 b;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %5, 0;\n\tsetp.eq.u32 t, 0, 0;\n\t"
                     "mov.b64 b, {%2, %3};\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t"
                     SS_MMA_NEXT_TS("8", "2") SS_MMA_NEXT_TS("16", "4") SS_MMA_NEXT_TS("24", "6") "}"
                     ::"r"(d), "r"(a), "r"(blo), "r"(bhi), "r"(idesc), "r"(acc) : "memory");
}
// bytes of 16 rows (an address each, lanes 0..15) transposed: lane holds bytes 4 (lane % 4) .. of column lane / 4 (r0) and 8 further (r1)
__device__ __forceinline__ void load_transposed_bytes(uint32_t addr, uint32_t& r0, uint32_t& r1) {
    asm volatile("ldmatrix.sync.aligned.m16n16.x1.trans.shared.b8 {%0, %1}, [%2];" : "=r"(r0), "=r"(r1) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load_transposed_halves(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// codes to bf16: 128 + c, which 128 + z is taken from
__device__ __forceinline__ uint32_t code_plus_128(uint32_t x) {
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(r) : "r"(x));     // (x & mask) | two bf16 of 128
    return r;
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// floats in the order of integers
__device__ __forceinline__ int ordered(float x) {
    const int i = __float_as_int(x);
    return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }

// The keys behind the prefix of a unit
__device__ __forceinline__ Extra extra_of(const KvqArgs& a, const Seq& s, int row0, int block) {
    Extra x;
    x.T = s.T, x.gamma = max(a.gamma, 1), x.row0 = row0, x.rows = s.rows, x.t0 = 0, x.count = s.T;
    const int last = min(row0 + block, s.rows) - 1;
    if (last >= s.T) {                               // the block has stream rows: the streams of their nodes
        x.t0 = row0 < s.T ? 0 : (row0 - s.T) / a.gamma;
        x.count = s.T + ((last - s.T) / a.gamma - x.t0 + 1) * a.gamma;
    }
    return x;
}

// Key e behind the prefix on its way to L2
__device__ __forceinline__ void prefetch_extra(const KvqArgs& a, const Extra& x, int D, int b, int h, int e, const __nv_bfloat16* tree, const __nv_bfloat16* spec) {
    if (e >= x.count) return;
    const __nv_bfloat16* const src = (e < x.T ? tree : spec) + extra_offset(a, x, D, b, h, e);
    prefetch_l2(src);
    if (D > 64) prefetch_l2(src + D - 8);
}

// A unit's query rows as THREADS threads put them into shared memory at `rows_at`, where their outputs go, and which rows see which node.
// BATCH: loads of a thread on their way at once
template <int D, int N, int THREADS, int BATCH>
static __device__ __noinline__ void prepare_rows(const KvqArgs& a, TileUnit& u, uint32_t rows_at, int t) {
    using G = TileGeo<D, N>;
    constexpr int kItems = (N * (D / 8) + THREADS - 1) / THREADS;
    const int rows = u.rows, T = u.T, row0 = u.row0, h = u.head, b = u.b, lane = t & 31;
    // the rows that see a node: every warp takes its share of the nodes
    unsigned long long see[2] = {};
    #pragma unroll
    for (int half = 0; half < (N + 31) / 32; ++half) {
        const int n = 32 * half + lane;
        if (n < rows) see[half] = a.trees[b].anc_mask[row_of(row0 + n, T, a.gamma).t];
    }
    #pragma unroll 1
    for (int i = 0; i < kItems; i += BATCH) {
        uint4 v[BATCH];
        #pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            const int item = (i + q) * THREADS + t, r = item / (D / 8), at = item - r * (D / 8), row = row0 + r;
            v[q] = make_uint4(0u, 0u, 0u, 0u);
            if (r < rows) v[q] = *reinterpret_cast<const uint4*>((row < T ? a.q_main : a.q_spec) + row_offset(a, D, b, h, row, T) + 8 * at);
        }
        #pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            const int item = (i + q) * THREADS + t, r = item / (D / 8), at = item - r * (D / 8);
            if (item >= N * (D / 8)) break;
            st_shared_v4(rows_at + (at >> 3) * G::kBox + r * 128 + (((at & 7) ^ (r & 7)) << 4), v[q].x, v[q].y, v[q].z, v[q].w);
        }
    }
    for (int e = t >> 5; e < T; e += THREADS / 32) {
        const uint32_t lo = __ballot_sync(0xffffffffu, see[0] >> e & 1ull), hi = N > 32 ? __ballot_sync(0xffffffffu, see[1] >> e & 1ull) : 0u;
        if (lane == 0) u.see[e] = static_cast<unsigned long long>(hi) << 32 | lo;
    }
    if (t < N) u.out[t] = t < rows ? row_offset(a, D, b, h, row0 + t, T) : 0;
}

template <int D, int N>
__global__ void __launch_bounds__(kTileThreads, 1) msa_attention_kvq_tiles_kernel(const __grid_constant__ KvqArgs a) {
    using G = TileGeo<D, N>;
    constexpr int C = G::kRowsOfGroup;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(16) TileCtrl<C> c;
    const int tid = threadIdx.x, lane = tid & 31, warp = static_cast<int>(uniform(tid >> 5)), quad = warp & 3;
    const uint32_t smem = smem_u32(smem_raw);
    constexpr int kMmaWarp = kTileWarpsOfUnit - 1, kPlanWarp = kMmaWarp + 1;
    if (tid == 0) {
        c.waits.abort = 0, c.waits.limit = static_cast<int>(kWaitCycles >> 10);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&c.k_full[i]), 128), mbar_init(smem_u32(&c.v_full[i]), 128);
            mbar_init(smem_u32(&c.s_free[i]), kTileSoftmax), mbar_init(smem_u32(&c.p_full[i]), kTileSoftmax);
            mbar_init(smem_u32(&c.s_full[i]), 2), mbar_init(smem_u32(&c.pv_done[i]), 1);
            mbar_init(smem_u32(&c.plan_full[i]), 1), mbar_init(smem_u32(&c.rows_full[i]), 1), mbar_init(smem_u32(&c.plan_free[i]), kTileWarpsOfUnit);
        }
        for (int i = 0; i < G::kStages; ++i) mbar_init(smem_u32(&c.codes_full[i]), 128), mbar_init(smem_u32(&c.codes_free[i]), 128);
        for (int i = 0; i < 2 * kTileGroups; ++i) mbar_init(smem_u32(&c.vote[i >> 1][i & 1]), 4), c.hot[i >> 1][i & 1] = 0;
        mbar_init(smem_u32(&c.o_free), kTileSoftmax), mbar_init(smem_u32(&c.drain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&c.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    wait_for_previous_kernel();
    release_next_kernel();
    if (tid == 0) {
        const int lim = reinterpret_cast<const volatile int*>(a.ws)[1];
        if (lim > 0) c.waits.limit = lim;
    }
    Line<N, kTileOfKeys, 0, kTileStart> line;                    // (the planning warp's)
    const auto make_plan = [&](TileUnit& u, bool more) {         // of the unit that the line is at
        if (lane != 0) return;
        u.done = !more;
        if (!more) return;
        const Seq& s = line.s;
        const Pieces share(line);
        u.L = s.L, u.T = s.T, u.prefix = prefix_chunks<kTileOfKeys>(s.L), u.from = line.from, u.to = line.to, u.start = s.start;
        u.head = min(line.head0, a.n_heads - 1), u.real = line.head0 < a.n_heads, u.row0 = line.row0, u.rows = min(N, s.rows - line.row0), u.b = line.b;
        u.whole = line.whole(), u.first = share.first, u.last = share.last, u.second = share.second;
        u.me = line.me, u.member = line.member, u.team = line.team_log2;
        u.extra = extra_of(a, s, line.row0, N);
    };
    if (warp == kPlanWarp) {
        const bool any = line.begin(a, lane);
        if (lane == 0) c.any = any;
        if (any) make_plan(c.unit[0], line.next(a));
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (c.any == 0) {
        if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(c.tmem));
        return;
    }
    const uint32_t tmem = uniform(c.tmem), lanes = static_cast<uint32_t>(32 * quad) << 16;
    const auto wait = [&](unsigned long long& bar, uint32_t parity) {
        if (!mbar_try(smem_u32(&bar), parity)) wait_for_data_slow(smem_u32(&bar), parity, &c.waits);
    };
    const auto wait_for_product = [&](unsigned long long& bar, uint32_t parity) {
        if (!mbar_try(smem_u32(&bar), parity)) wait_for_product_slow(smem_u32(&bar), parity, &c.waits.abort);
    };
    const auto wait_for_warps = [&](unsigned long long& bar, uint32_t parity) {
        if (!mbar_try(smem_u32(&bar), parity)) wait_for_warps_slow(smem_u32(&bar), parity, &c.waits);
    };
    // units one after another: the plan of unit n, and back to the planning warp when a warp is done with it
    const auto plan_of = [&](uint32_t n) -> const TileUnit& {
        wait_for_warps(c.plan_full[n & 1], (n >> 1) & 1);
        return c.unit[n & 1];
    };
    const auto plan_used = [&](uint32_t n) {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&c.plan_free[n & 1]));
    };
    uint32_t tau = 0;                                // tiles so far, over all units: buffer tau & 1, phase (tau >> 1) & 1

    if (warp < 4) {
        // ---- K ------------------------------------------------------------------------------
        const int key = tid;
        uint32_t unit = 0, copied = 0;               // units; tiles of codes copied or on their way
        for (;; ++unit) {
            const TileUnit& u = plan_of(unit);
            if (u.done) break;
            const int from = u.from, to = u.to, held = min(to, u.prefix);
            const bool real = u.real;
            const uint32_t tau0 = tau, copied0 = copied;
            TileLoader<D, N> loader(a, u, from, tid);
            const uint32_t* words = a.k_params + (u.start + static_cast<long long>(from) * kTileOfKeys) * a.p_slot + u.head * a.p_head;
            const long long v_words = a.v_params - a.k_params;
            named_barrier(1, 128);                   // (the ring's last stage has been read by all)
            const auto load = [&](int k) {           // codes, scales and zero points of tile k
                if (k < held) {
                    const uint32_t n = copied0 + (k - from), stage = n % G::kStages;
                    if (n >= G::kStages) wait(c.codes_free[stage], ((n - G::kStages) / G::kStages) & 1);
                    loader.next(a, smem + G::oK + stage * G::kCodes, smem + G::oV + stage * G::kCodes, tid);
                    const long long p = (static_cast<long long>(k - from) * kTileOfKeys + min(key, u.L - 1 - k * kTileOfKeys)) * a.p_slot;
                    const uint32_t dst = (((tau0 + (k - from)) % G::kParams) * kTileOfKeys + key) * 4;
                    copy_async<4>(smem + G::oKParams + dst, words + p);
                    copy_async<4>(smem + G::oVParams + dst, words + v_words + p);
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(&c.codes_full[stage])) : "memory");
                }
                copy_commit();
            };
            #pragma unroll 1
            for (int i = 0; i < G::kStages - 1; ++i) load(from + i);
            #pragma unroll 1
            for (int k = from; k < to; ++k, ++tau) {
                uint32_t w[G::kWords];
                uint32_t z = 0u;
                const uint32_t params = ((tau % G::kParams) * kTileOfKeys + key) * 4;
                if (k < held) {
                    copy_wait<G::kStages - 2>();
                    named_barrier(1, 128);
                    load(k + G::kStages - 1);
                    const uint32_t row = smem + G::oK + (copied % G::kStages) * G::kCodes + key * G::kPitch;
                    ++copied;
                    #pragma unroll
                    for (int i = 0; i < G::kWords / 4; ++i) {
                        const uint4 v = lds128(row + 16 * (D == 128 ? i ^ ((key >> 1) & 3) : D == 64 ? i ^ ((key >> 2) & 1) : i));
                        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
                    }
                    if constexpr (D == 80) {
                        const uint2 v = lds64(row + 32);
                        w[8] = v.x, w[9] = v.y;
                    }
                    z = code_plus_128(__byte_perm(lds32(smem + G::oKParams + params), 0u, 0x3232));
                }
                if (tau >= 2) wait(c.s_full[tau & 1], ((tau - 2) >> 1) & 1);
                tc_fence_after();
                const uint32_t dst = tmem + G::kTmemK + (tau & 1) * 64 + lanes;
                if (k < held) {
                    #pragma unroll
                    for (int i = 0; i < G::kWords; i += 8) {
                        uint32_t r[32];
                        #pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            if (i + q < G::kWords) {
                                #pragma unroll
                                for (int n = 0; n < 4; ++n) r[4 * q + n] = sub_bf16x2(code_plus_128(w[i + q] >> (4 * n)), z);
                            }
                        }
                        if (i + 8 <= G::kWords) tmem_store<32>(dst + 4 * i, r);
                        else tmem_store<8>(dst + 4 * i, r);       // (80: the last two words)
                    }
                } else {
                    const __nv_bfloat16* src = nullptr;
                    if (real) {
                        const int e = (k - u.prefix) * kTileOfKeys + key;
                        if (e < u.extra.count) src = (e < u.T ? a.k_tree : a.k_spec) + extra_offset(a, u.extra, D, u.b, u.head, e);
                    }
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(smem + G::oKParams + params), "r"(0x3f80u) : "memory");      // scales of 1
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(smem + G::oVParams + params), "r"(0x3f80u) : "memory");
                    #pragma unroll
                    for (int i = 0; i < G::kWords; i += 8) {
                        uint32_t r[32];
                        #pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            uint4 v = {};
                            if (src && i + q < G::kWords) v = *reinterpret_cast<const uint4*>(src + 8 * (i + q));
                            r[4 * q] = v.x, r[4 * q + 1] = v.y, r[4 * q + 2] = v.z, r[4 * q + 3] = v.w;
                        }
                        if (i + 8 <= G::kWords) tmem_store<32>(dst + 4 * i, r);
                        else tmem_store<8>(dst + 4 * i, r);
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(smem_u32(&c.k_full[tau & 1]));
            }
            plan_used(unit);
        }
        copy_wait<0>();
    } else if (warp < 8) {
        // ---- V ------------------------------------------------------------------------------
        const int t = tid - 128;
        const bool mine = quad < G::kQuads;
        // keys in the order in which the columns of V^T follow one another: transposed byte 4 q + e of 16 keys goes to column q (e < 2) or
        // 4 + q, which hold keys 2 q, 2 q + 1 and 8 + 2 q, 8 + 2 q + 1
        const int from16 = (lane & 3) < 2 ? 2 * ((lane & 15) >> 2) + (lane & 3) : 8 + 2 * ((lane & 15) >> 2) + (lane & 3) - 2;
        uint32_t unit = 0, used = 0;                 // units; tiles of codes used
        for (;; ++unit) {
            const TileUnit& u = plan_of(unit);
            if (u.done) break;
            const int from = u.from, to = u.to, held = min(to, u.prefix);
            #pragma unroll 1
            for (int k = from; k < to; ++k, ++tau) {
                const uint32_t dst = tmem + G::kTmemV + (tau & 1) * 64 + lanes;
                if (k < held) {
                    const uint32_t st = used % G::kStages;
                    wait(c.codes_full[st], (used / G::kStages) & 1);
                    ++used;
                    if (tau >= 2) wait(c.pv_done[tau & 1], ((tau - 2) >> 1) & 1);
                    tc_fence_after();
                    if (mine) {
                        const uint32_t codes = smem + G::oV + st * G::kCodes, words = smem + G::oVParams + (tau % G::kParams) * kTileOfKeys * 4 + 8 * (lane & 3);
                        #pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t lo[16], hi[16];
                            #pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int key0 = 64 * half + 16 * i, row = key0 + from16;
                                const int place = D == 128 ? quad ^ ((row >> 1) & 3) : D == 64 ? quad ^ ((row >> 2) & 1) : quad;
                                uint32_t r0, r1;
                                load_transposed_bytes(codes + row * G::kPitch + place * 16, r0, r1);
                                const uint2 p0 = lds64(words + 4 * key0), p1 = lds64(words + 4 * key0 + 32);
                                const uint32_t z0 = code_plus_128(__byte_perm(p0.x, p0.y, 0x7632)), z1 = code_plus_128(__byte_perm(p1.x, p1.y, 0x7632));
                                // a byte's low or high code beside 0x43: 128 + c in bf16
                                const auto pair = [](uint32_t x, uint32_t sel) { return __byte_perm(x & 0x0f0f0f0fu, 0x43434343u, sel); };
                                lo[4 * i] = sub_bf16x2(pair(r0, 0x4140), z0), lo[4 * i + 1] = sub_bf16x2(pair(r1, 0x4140), z0);
                                lo[4 * i + 2] = sub_bf16x2(pair(r0, 0x4342), z1), lo[4 * i + 3] = sub_bf16x2(pair(r1, 0x4342), z1);
                                hi[4 * i] = sub_bf16x2(pair(r0 >> 4, 0x4140), z0), hi[4 * i + 1] = sub_bf16x2(pair(r1 >> 4, 0x4140), z0);
                                hi[4 * i + 2] = sub_bf16x2(pair(r0 >> 4, 0x4342), z1), hi[4 * i + 3] = sub_bf16x2(pair(r1 >> 4, 0x4342), z1);
                            }
                            tmem_store_lanes16(dst + 32 * half, lo);
                            tmem_store_lanes16(dst + 32 * half + (16u << 16), hi);
                        }
                    }
                    mbar_arrive(smem_u32(&c.codes_free[st]));
                } else {
                    // bf16 rows in the order of the lanes: of 8 values the low codes' would be 0, 4, 1, 5, the high codes' 2, 6, 3, 7.  64 keys at
                    // a time; a row's words are shared by two threads.
                    const int r = t >> 1;
                    const bool both = (k - u.prefix) * kTileOfKeys + 64 < u.extra.count;      // (else the tile's upper half is empty)
                    uint4 v[2 * G::kQuads];
                    const auto fetch = [&](int half) {
                        const int e = (k - u.prefix) * kTileOfKeys + 64 * half + r;
                        const __nv_bfloat16* src = nullptr;
                        if (u.real && e < u.extra.count) src = (e < u.T ? a.v_tree : a.v_spec) + extra_offset(a, u.extra, D, u.b, u.head, e);
                        #pragma unroll
                        for (int i = 0; i < 2 * G::kQuads; ++i) {
                            const int word = 2 * i + (t & 1);
                            v[i] = make_uint4(0u, 0u, 0u, 0u);
                            if (src && word < G::kWords) v[i] = *reinterpret_cast<const uint4*>(src + 8 * word);
                        }
                    };
                    fetch(0);
                    if (tau >= 2) wait(c.pv_done[tau & 1], ((tau - 2) >> 1) & 1);
                    tc_fence_after();
                    #pragma unroll 1
                    for (int half = 0; half < 2; ++half) {
                        if (half > 0 && !both) {     // the weights there are zero; the values must be numbers
                            if (mine) {
                                uint32_t none[16];
                                #pragma unroll
                                for (int i = 0; i < 16; ++i) none[i] = 0u;
                                tmem_store_lanes16(dst + 32, none);
                                tmem_store_lanes16(dst + 32 + (16u << 16), none);
                            }
                            break;
                        }
                        if (half > 0) fetch(1);
                        named_barrier(2, 128);       // (what lay there has been read)
                        const uint32_t row = smem + G::oRows + r * G::kRowOfV;
                        #pragma unroll
                        for (int i = 0; i < 2 * G::kQuads; ++i) {
                            // bytes: 64 to a quad, low ones first, 8 to a word; 16-byte places swizzled by the key
                            const int word = 2 * i + (t & 1), at = 64 * (word >> 2) + 8 * (word & 3);
                            const uint32_t lo = row + (((at >> 4) ^ (r & 3)) << 4) + (at & 15), hi = row + ((((at + 32) >> 4) ^ (r & 3)) << 4) + (at & 15);
                            st_shared_v2(lo, __byte_perm(v[i].x, v[i].z, 0x5410), __byte_perm(v[i].x, v[i].z, 0x7632));
                            st_shared_v2(hi, __byte_perm(v[i].y, v[i].w, 0x5410), __byte_perm(v[i].y, v[i].w, 0x7632));
                        }
                        named_barrier(2, 128);
                        if (mine) {
                            #pragma unroll
                            for (int high = 0; high < 2; ++high) {
                                uint32_t q16[16];
                                #pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const int kk = 16 * i + 8 * (lane >> 4) + (lane & 7);          // matrices: dims 0..7, 8..15 of 8 keys, then of 8 more
                                    const int at = 64 * quad + 32 * high + 16 * ((lane >> 3) & 1);
                                    uint32_t q[4];
                                    load_transposed_halves(smem + G::oRows + kk * G::kRowOfV + (((at >> 4) ^ (kk & 3)) << 4), q);
                                    q16[4 * i] = q[0], q16[4 * i + 1] = q[1], q16[4 * i + 2] = q[2], q16[4 * i + 3] = q[3];
                                }
                                tmem_store_lanes16(dst + 32 * half + (high ? 16u << 16 : 0u), q16);
                            }
                        }
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(smem_u32(&c.v_full[tau & 1]));
            }
            plan_used(unit);
        }
    } else if (warp < kMmaWarp) {
        // ---- softmax ------------------------------------------------------------------------
        const int group = (warp - 8) >> 2, key = 32 * quad + lane, bar = 3 + group;
        constexpr uint32_t all = (1u << C) - 1u;
        uint32_t unit = 0;
        int* const counters = reinterpret_cast<int*>(a.ws + kWsHeaderBytes);
        float* const partial = reinterpret_cast<float*>(a.ws + kWsHeaderBytes + kCounterBytes);
        constexpr int kPartial = N * (D + 4);
        const uint32_t weights = smem + G::oP + key * 128;        // the key's row of P^T
        // TMEM lane to dimension
        const int byte = 16 * quad + (lane & 15), dim = 8 * (byte >> 2) + ((byte & 1) << 2) + ((byte >> 1) & 1) + ((lane >> 4) << 1);
        if (!plan_of(0).done) {
            prepare_rows<D, N, kTileSoftmax, 2>(a, c.unit[0], smem + G::oQ, tid - 256);
            fence_async_smem();
            named_barrier(3 + kTileGroups, kTileSoftmax);
            if (tid == 256) mbar_arrive(smem_u32(&c.rows_full[0]));
        }
        for (;; ++unit) {
            const TileUnit& u = plan_of(unit);
            if (u.done) break;
            const int L = u.L, P = u.prefix, from = u.from, to = u.to;
            if (quad == 0 && lane < C) c.neg_ref[group * C + lane] = 0.f;
            named_barrier(bar, 128);
            float l[C];
            #pragma unroll
            for (int i = 0; i < C; ++i) l[i] = 0.f;
            uint32_t seen = 0u;                      // rows that have seen a key (the same in all warps of the group)
            #pragma unroll 1
            for (int k = from; k < to; ++k, ++tau) {
                const uint32_t parity = (tau >> 1) & 1;
                wait_for_product(c.s_full[tau & 1], parity);
                tc_fence_after();
                const uint32_t params = ((tau % G::kParams) * kTileOfKeys + key) * 4;
                const float sk = scale_of(lds32(smem + G::oKParams + params)) * a.scale, sv = scale_of(lds32(smem + G::oVParams + params));
                // rows that see the key: all of them if it is a cached one; else those of its node's descendants; of a stream key, from its
                // own row to its node's last
                uint32_t vis = all;
                if (k < P) {
                    if ((k + 1) * kTileOfKeys > L && k * kTileOfKeys + key >= L) vis = 0u;
                } else {
                    const int e = (k - P) * kTileOfKeys + key;
                    vis = 0u;
                    if (e < u.T) {
                        vis = static_cast<uint32_t>(u.see[e] >> (group * C)) & all;
                    } else if (e < u.extra.count) {
                        const int own = e - u.T + u.extra.t0 * u.extra.gamma, first = u.T + own - u.row0 - group * C, last = first + u.extra.gamma - 1 - own % u.extra.gamma;
                        if (first < C && last >= 0) vis = (0xffffffffu >> (31 - min(last, 31))) & (0xffffffffu << max(first, 0));
                    }
                }
                const bool masked = (k + 1) * kTileOfKeys > L;
                float d[C];
                // scores above their references, in log2 units; -inf where the row does not see the key
                const auto scores = [&]() {
                    uint32_t raw[C];
                    tmem_load<C>(tmem + G::kTmemS + (tau & 1) * N + group * C + lanes, raw);
                    tmem_wait_ld();
                    const unsigned long long sk2 = pack_f32x2(sk, sk);
                    #pragma unroll
                    for (int i = 0; i < C; i += 4) {
                        const float4 r = *reinterpret_cast<const float4*>(&c.neg_ref[group * C + i]);
                        unpack_f32x2(fma_f32x2(sk2, pack_f32x2(__uint_as_float(raw[i]), __uint_as_float(raw[i + 1])), pack_f32x2(r.x, r.y)), d[i], d[i + 1]);
                        unpack_f32x2(fma_f32x2(sk2, pack_f32x2(__uint_as_float(raw[i + 2]), __uint_as_float(raw[i + 3])), pack_f32x2(r.z, r.w)), d[i + 2], d[i + 3]);
                    }
                    if (masked) {
                        #pragma unroll
                        for (int i = 0; i < C; ++i)
                            if (!(vis >> i & 1u)) d[i] = -INFINITY;
                    }
                };
                scores();
                float top[4] = {d[0], d[1], d[2], d[3]};
                #pragma unroll
                for (int i = 4; i < C; ++i) top[i & 3] = fmaxf(top[i & 3], d[i]);
                // does a row of the group need a higher reference?  While the four warps' answers come in, the weights are computed as if not.
                const bool hot = __any_sync(0xffffffffu, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) > 8.f) || k == from || (k >= P && seen != all);
                if (lane == 0) {
                    if (hot) *const_cast<volatile int*>(&c.hot[group][tau & 1]) = 1;
                    mbar_arrive(smem_u32(&c.vote[group][tau & 1]));
                }
                #pragma unroll
                for (int i = 0; i < C; ++i) d[i] = exp2_approx(d[i]);
                wait_for_warps(c.vote[group][tau & 1], parity);
                if (*const_cast<volatile int*>(&c.hot[group][tau & 1])) {
                    // references go up to the maxima (a row's first one: to its maximum, whatever it is)
                    scores();
                    int own = 0;
                    #pragma unroll
                    for (int i = 0; i < C; ++i) {
                        const int m = __reduce_max_sync(0xffffffffu, ordered(d[i]));
                        if (lane == i) own = m;
                    }
                    if (lane < C) c.tile_max[group][quad][lane] = own;
                    named_barrier(bar, 128);
                    c.hot[group][tau & 1] = 0;
                    float by = 0.f, f = 1.f;
                    bool any = false;
                    if (lane < C) {
                        const float m = from_ordered(max(max(c.tile_max[group][0][lane], c.tile_max[group][1][lane]), max(c.tile_max[group][2][lane], c.tile_max[group][3][lane])));
                        any = m > -INFINITY;
                        if (seen >> lane & 1u) by = fmaxf(m, 0.f), f = exp2_approx(-by);
                        else if (any) by = m;
                        if (quad == 0) c.neg_ref[group * C + lane] -= by;
                    }
                    seen |= __ballot_sync(0xffffffffu, any);
                    #pragma unroll
                    for (int i = 0; i < C; ++i) {
                        d[i] = exp2_approx(d[i] - __shfl_sync(0xffffffffu, by, i));
                        l[i] *= __shfl_sync(0xffffffffu, f, i);
                    }
                    if (k > from) {                  // and O with them: the products so far are complete, this tile's waits for our weights
                        wait_for_product(c.pv_done[(tau - 1) & 1], ((tau - 1) >> 1) & 1);
                        tc_fence_after();
                        #pragma unroll
                        for (int i = 0; i < C; i += 8) {
                            uint32_t o[8];
                            tmem_load<8>(tmem + G::kTmemO + group * C + i + lanes, o);
                            tmem_wait_ld();
                            #pragma unroll
                            for (int q = 0; q < 8; ++q) o[q] = __float_as_uint(__uint_as_float(o[q]) * __shfl_sync(0xffffffffu, f, i + q));
                            tmem_store<8>(tmem + G::kTmemO + group * C + i + lanes, o);
                        }
                        tmem_wait_st();
                        tc_fence_before();
                    }
                    named_barrier(bar, 128);
                }
                tc_fence_before();
                mbar_arrive(smem_u32(&c.s_free[tau & 1]));
                // (this tile's S was committed behind the product of two tiles ago: its weights' place is free)
                const unsigned long long sv2 = pack_f32x2(sv, sv);
                #pragma unroll
                for (int i = 0; i < C; i += 8) {
                    uint32_t y[4];
                    #pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const unsigned long long e = pack_f32x2(d[i + 2 * q], d[i + 2 * q + 1]);
                        unpack_f32x2(add_f32x2(pack_f32x2(l[i + 2 * q], l[i + 2 * q + 1]), e), l[i + 2 * q], l[i + 2 * q + 1]);
                        float u, v;
                        unpack_f32x2(fma_f32x2(e, sv2, 0ull), u, v);
                        y[q] = pack2_bf16(u, v);
                    }
                    st_shared_v4(weights + (tau & 1) * G::kP + ((((i >> 3) + group * (C / 8)) ^ (key & 7)) << 4), y[0], y[1], y[2], y[3]);
                }
                fence_async_smem();
                mbar_arrive(smem_u32(&c.p_full[tau & 1]));
            }
            // ---- the unit's end: sums over the keys, O
            wait_for_product(c.pv_done[(tau - 1) & 1], ((tau - 1) >> 1) & 1);
            tc_fence_after();
            #pragma unroll
            for (int w = 16; w >= C; w >>= 1) {      // (fewer rows than lanes: whole sums first)
                #pragma unroll
                for (int i = 0; i < C; ++i) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
            }
            #pragma unroll
            for (int w = C / 2; w > 0; w >>= 1) {    // lane i ends with row i
                #pragma unroll
                for (int i = 0; i < w; ++i) {
                    const bool up = lane & w;
                    const float give = up ? l[i] : l[i + w], keep = up ? l[i + w] : l[i];
                    l[i] = keep + __shfl_xor_sync(0xffffffffu, give, w);
                }
            }
            if (lane < C) c.sums[group][quad][lane] = l[0];
            uint32_t raw[C];
            tmem_load<C>(tmem + G::kTmemO + group * C + lanes, raw);
            named_barrier(bar, 128);
            const int at = lane & (C - 1);
            const float sum = (c.sums[group][0][at] + c.sums[group][1][at]) + (c.sums[group][2][at] + c.sums[group][3][at]);
            const float ref = -c.neg_ref[group * C + at];
            tmem_wait_ld();
            tc_fence_before();
            mbar_arrive(smem_u32(&c.o_free));
            // Nothing that was computed from a wait that ran out is written or passed on.  Whoever left one early had set or seen `abort` before it came
            // to the barrier that lies between its results and their use: so it is looked at behind that barrier.
            const auto good = [&] { return *const_cast<volatile int*>(&c.waits.abort) == 0; };
            const int rows = u.real ? u.rows : 0, mains = u.T - u.row0;       // rows, and how many of them are main-stream ones
            if (u.whole) {
                const float f = 1.f / sum;
                if (quad == 0 && lane < C && group * C + lane < rows && good()) {
                    const int n = group * C + lane;
                    float* lse = n < mains ? a.lse_main : a.lse_spec;
                    if (lse != nullptr) lse[u.out[n] / D] = (ref + log2f(sum)) * 0.6931471805599453f;
                }
                // to rows of dimensions, by way of the group's part of the first buffer of P: a TMEM lane's rows lie where a key's weights do
                #pragma unroll
                for (int i = 0; i < C; i += 8) {
                    uint32_t y[4];
                    #pragma unroll
                    for (int q = 0; q < 4; ++q)
                        y[q] = pack2_bf16(__uint_as_float(raw[i + 2 * q]) * __shfl_sync(0xffffffffu, f, i + 2 * q),
                                          __uint_as_float(raw[i + 2 * q + 1]) * __shfl_sync(0xffffffffu, f, i + 2 * q + 1));
                    st_shared_v4(weights + ((((i >> 3) + group * (C / 8)) ^ (key & 7)) << 4), y[0], y[1], y[2], y[3]);
                }
                named_barrier(bar, 128);
                const bool ok = good();
                // matrices of 8 dimensions (a word's) by 8 rows, transposed: a lane gets two dimensions of a row
                #pragma unroll 1
                for (int m0 = 4 * quad; m0 < D / 8 * (C / 8); m0 += 16) {
                    const int m = m0 + (lane >> 3), word = m / (C / 8), eight = m - word * (C / 8), dd = lane & 7;
                    const int from_lane = 32 * (word >> 2) + 4 * (word & 3) + ((dd >> 2) & 1) + 2 * (dd & 1) + 8 * (dd & 2);
                    uint32_t q[4];
                    load_transposed_halves(smem + G::oP + from_lane * 128 + (((eight + group * (C / 8)) ^ (from_lane & 7)) << 4), q);
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int mi = m0 + i, wi = mi / (C / 8), n = group * C + 8 * (mi - wi * (C / 8)) + (lane >> 2);
                        if (n < rows && wi < D / 8 && ok)        // (80: ten words of eight rows are no multiple of four matrices)
                            *reinterpret_cast<uint32_t*>((n < mains ? a.o_main : a.o_spec) + u.out[n] + 8 * wi + 2 * (lane & 3)) = q[i];
                    }
                }
                named_barrier(bar, 128);             // (the next unit's weights go there)
            } else {
                float* const mine = partial + (2ll * blockIdx.x + (u.me == u.first ? u.second : 0)) * kPartial;
                if (quad == 0 && lane < C)
                    __stcg(reinterpret_cast<float2*>(mine + (group * C + lane) * (D + 4) + D), make_float2(seen >> lane & 1u ? ref : kNoRef, sum));
                if (dim < D) {
                    #pragma unroll
                    for (int i = 0; i < C; ++i) __stcg(mine + (group * C + i) * (D + 4) + dim, __uint_as_float(raw[i]));
                }
                named_barrier(3 + kTileGroups, kTileSoftmax);
                if (tid == 256) {
                    // (a piece that is no good is not counted: its unit is never joined)
                    c.joined = good() && last_piece(counters + (u.first << u.team) + u.member, u.last - u.first + 1);
                }
                named_barrier(3 + kTileGroups, kTileSoftmax);
                if (c.joined) {
                    // 8 values of a row at a time, up to four partial rows on their way
                    const int n = u.last - u.first + 1, items = rows * (D / 8);
                    const float* const p0 = partial + (2ll * ((u.first << u.team) + u.member) + u.second) * kPartial;
                    const long long on = (2ll << u.team) * kPartial;         // between teams' places
                    const float* const p1 = p0 - u.second * kPartial + on;
                    #pragma unroll 1
                    for (int item = tid - 256; item < items; item += kTileSoftmax) {
                        const int r = item / (D / 8), d0 = (item - r * (D / 8)) * 8;
                        float m = kNoRef, sm = 0.f, o[8] = {};
                        #pragma unroll 1
                        for (int i = 0; i < n; i += 4) {
                            float2 st[4];
                            float4 u[4], v[4];
                            #pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const int k = min(i + q, n - 1);
                                const float* src = (k == 0 ? p0 : p1 + (k - 1) * on) + r * (D + 4);
                                st[q] = __ldcg(reinterpret_cast<const float2*>(src + D));
                                u[q] = __ldcg(reinterpret_cast<const float4*>(src + d0)), v[q] = __ldcg(reinterpret_cast<const float4*>(src + d0) + 1);
                            }
                            #pragma unroll
                            for (int q = 0; q < 4; ++q)
                                if (i + q < n) join_row(o, m, sm, st[q], u[q], v[q]);
                        }
                        store_row<D>(a, r < mains, u.out[r], d0, o, m, sm);
                    }
                }
            }
            plan_used(unit);
        }
    } else if (warp == kMmaWarp) {
        // ---- MMAs ---------------------------------------------------------------------------
        const uint32_t base = uniform(smem);
        const uint64_t dq = desc_k_major(base + G::oQ), dp = desc_mn_major(base + G::oP, 0);
        uint32_t unit = 0;
        const auto product = [&](uint32_t t, bool first) {       // O^T (+)= V^T P^T of tile t
            if (first && unit > 0) wait(c.o_free, (unit - 1) & 1);
            wait(c.v_full[t & 1], (t >> 1) & 1);
            wait(c.p_full[t & 1], (t >> 1) & 1);
            tc_fence_after();
            const uint64_t b = dp + (t & 1) * (G::kP >> 4);
            const uint32_t va = tmem + G::kTmemV + (t & 1) * 64;
            tc_mma_ts_steps(tmem + G::kTmemO, va, b, G::kIdescPV, first ? 0u : 1u);
            tc_mma_ts_steps(tmem + G::kTmemO, va + 32, b + 4 * 128, G::kIdescPV, 1u);
            tc_commit_e(smem_u32(&c.pv_done[t & 1]));
        };
        for (;; ++unit) {
            const TileUnit& u = plan_of(unit);
            if (u.done) break;
            const uint32_t tiles = uniform(static_cast<uint32_t>(u.to - u.from));
            const uint64_t rows = (unit & 1) * (G::kRowsOfUnit >> 4);
            wait(c.rows_full[unit & 1], (unit >> 1) & 1);
            #pragma unroll 1
            for (uint32_t i = 0; i < tiles; ++i, ++tau) {
                wait(c.k_full[tau & 1], (tau >> 1) & 1);
                if (tau >= 2) wait(c.s_free[tau & 1], ((tau - 2) >> 1) & 1);
                tc_fence_after();
                const uint32_t ka = tmem + G::kTmemK + (tau & 1) * 64, sd = tmem + G::kTmemS + (tau & 1) * N;
                tile_mma<4>(sd, ka, dq + rows, G::kIdescS, 0u);
                if constexpr (D == 128) tile_mma<4>(sd, ka + 32, dq + rows + (G::kBox >> 4), G::kIdescS, 1u);
                if constexpr (D == 80) tile_mma<1>(sd, ka + 32, dq + rows + (G::kBox >> 4), G::kIdescS, 1u);
                tc_commit_e(smem_u32(&c.s_full[tau & 1]));
                if (lane == 0) mbar_arrive(smem_u32(&c.s_full[tau & 1]));            // (passes on what the K warps have written: the keys' scales)
                if (i > 0) product(tau - 1, i == 1);
            }
            product(tau - 1, tiles == 1);
            plan_used(unit);
        }
        tc_commit_e(smem_u32(&c.drain));
        mbar_drain(smem_u32(&c.drain), 0);           // (nothing is in flight when TMEM goes back)
    } else {
        // ---- preparing ----------------------------------------------------------------------
        const int t = tid - 32 * kPlanWarp, place = warp - kPlanWarp;
        for (uint32_t unit = 0;; ++unit) {
            TileUnit& u = c.unit[unit & 1];
            const uint32_t rows_at = smem + G::oQ + (unit & 1) * G::kRowsOfUnit;
            if (place == 0) {
                if (unit > 0) {                      // (the first unit's plan is there)
                    const bool more = line.next(a);
                    // (a unit's rows are free when all are done with the plan: its last S is complete then)
                    if (unit >= 2) wait_for_warps(c.plan_free[unit & 1], ((unit - 2) >> 1) & 1);
                    make_plan(u, more);
                }
            }
            named_barrier(4 + kTileGroups, kTilePrepare);
            if (t == 0) mbar_arrive(smem_u32(&c.plan_full[unit & 1]));
            if (u.done) break;
            // what lies behind the prefix comes to L2 meanwhile
            if (u.to > u.prefix) {
                for (int e = t; e < kTileOfKeys; e += kTilePrepare) {
                    prefetch_extra(a, u.extra, D, u.b, u.head, e, a.k_tree, a.k_spec);
                    prefetch_extra(a, u.extra, D, u.b, u.head, e, a.v_tree, a.v_spec);
                }
            }
            if (unit == 0) continue;                 // (the softmax warps, idle then, fetch the first unit's rows in a third of the time)
            prepare_rows<D, N, kTilePrepare, 6>(a, u, rows_at, t);
            fence_async_smem();
            named_barrier(4 + kTileGroups, kTilePrepare);
            if (t == 0) mbar_arrive(smem_u32(&c.rows_full[unit & 1]));           // (the query rows, and with them `out` and `see`)
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    if (tid == 0 && c.waits.abort != 0) set_status(a.ws, SS_ERR_DEVICE_TIMEOUT);
}

}  // namespace ss
