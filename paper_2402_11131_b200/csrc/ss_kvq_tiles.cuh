// Attention over a 4-bit prefix for blocks of more rows than a warp can hold, on tcgen05.  Included by ss_attention_kvq.cu.
//
// S^T = K Q^T and O^T = V^T P^T with 128 keys (dimensions) as the 128 lanes of TMEM and the N <= 64 query rows as columns: what
// grows with the rows is the cheap side, and codes go from registers to TMEM as A operands, never through shared memory.
//   K: the thread of a key turns the key's codes into bf16 c - z (exact), one TMEM lane; its scale multiplies the lane's scores.
//   V: transposing loads (ldmatrix, 16 keys by 16 bytes) give a thread four keys' codes of two dimensions; a TMEM lane is a dimension.
//      The scale is part of the weight that meets it.
// Lane 32 w + x of V^T and O^T (w < D / 32) holds, for x < 16, the low codes of byte 16 w + x of a row, else the high codes of
// byte 16 w + x - 16.
//
// 25 warps: 0..3 K, 4..7 V, 8..23 softmax (four groups of four, each a quarter of the rows, thread = key), 24 issues the MMAs.  Two
// buffers each for K, V, S and P, so that the five work on different tiles.  Nothing but the order of tiles is shared: every role
// walks the same list of units.
#pragma once
#include "ss_tcgen05.cuh"

namespace ss {

// A unit's start and end take as long as some five tiles.
constexpr int kTileStart = 5;
constexpr int kTileOfKeys = 128, kTileGroups = 4, kTileSoftmax = 128 * kTileGroups, kTileThreads = 256 + kTileSoftmax + 32;

template <int D, int N>
struct TileGeo {
    static constexpr int kRowsOfGroup = N / kTileGroups;          // rows of a softmax group
    static constexpr int kPitch = D == 128 ? 64 : D == 80 ? 48 : 32;         // bytes of a key's codes in shared memory (16-byte aligned)
    static constexpr int kCopy = D == 80 ? 8 : 16, kPer = D / 2 / kCopy;     // asynchronous copies per key
    static constexpr int kWords = D / 8;
    static constexpr int kColumns = D / 2;                        // TMEM columns of a K tile
    static constexpr int kQuads = (D + 31) / 32;                  // warps that have V lanes
    static constexpr int kCodes = kTileOfKeys * kPitch;
    static constexpr int kStages = 3, kParams = 8;
    static constexpr int kBoxes = D > 64 ? 2 : 1, kBox = N * 128;
    static constexpr int kRowOfV = 64 * kQuads;                   // bytes of a bf16 row in lane order
    static constexpr int kP = kTileOfKeys * 128;
    static constexpr int oP = 0, oQ = oP + 2 * kP, oK = oQ + kBoxes * kBox, oV = oK + kStages * kCodes;
    static constexpr int oKParams = oV + kStages * kCodes, oVParams = oKParams + kParams * kTileOfKeys * 8;
    static constexpr int kBytes = oVParams + kStages * kTileOfKeys * 4;
    static_assert(64 * kRowOfV <= kStages * kCodes, "half a tile of bf16 values takes the place of the ring");
    static constexpr uint32_t kTmemK = 0, kTmemV = 128, kTmemS = 256, kTmemO = 256 + 2 * N;
    static constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(N >> 3) << 17) | ((128u >> 4) << 24);
    static constexpr uint32_t kIdescS = kIdesc, kIdescPV = kIdesc | (1u << 16);
};

// A role's place in the list of units: the role's first thread goes on, the others read.  In shared memory, since it is used between
// units only and would cost every thread some 40 registers.
template <int N>
struct TileWalk {
    Line<N, kTileOfKeys, 0, kTileStart> line;
    int more;
};

// Asynchronous copies of a tile's codes by 128 threads, 16 (8) bytes each, from a pointer that walks along with the tiles.  Slots behind
// the last one are read as the last one again (their weights are zero).
template <int D, int N>
struct TileLoader {
    using G = TileGeo<D, N>;
    static constexpr bool kEven = 128 % G::kPer == 0;
    const unsigned char* at;                         // of the next tile: the thread's first copy (80: key 0)
    int left;                                        // slots from there on
    __device__ __forceinline__ TileLoader(const KvqArgs& a, const Seq& s, int h, int tile, int t, const unsigned char* codes) {
        const long long slot = s.start + static_cast<long long>(tile) * kTileOfKeys + (kEven ? t / G::kPer : 0);
        at = codes + slot * a.slot_stride + h * a.head_stride + (kEven ? t % G::kPer * G::kCopy : 0);
        left = s.L - tile * kTileOfKeys;
    }
    __device__ __forceinline__ uint32_t place(int row, int column) const {
        return row * G::kPitch + (D == 128 ? column ^ ((row >> 1) & 3) : D == 64 ? column ^ ((row >> 2) & 1) : column) * G::kCopy;
    }
    __device__ __forceinline__ void next(const KvqArgs& a, uint32_t stage, int t) {
        if (kEven && left >= kTileOfKeys) {
            // (the swizzle is the same for all of the thread's rows: they are a multiple of 8 apart)
            const uint32_t dst = stage + place(t / G::kPer, t % G::kPer);
            #pragma unroll
            for (int i = 0; i < G::kPer; ++i)
                copy_async<G::kCopy>(dst + i * (128 / G::kPer) * G::kPitch, at + i * (128 / G::kPer) * a.slot_stride);
        } else {
            const int last = left - 1;
            #pragma unroll 1
            for (int i = 0; i < G::kPer; ++i) {
                const int item = i * 128 + t, row = item / G::kPer, column = item - row * G::kPer;
                copy_async<G::kCopy>(stage + place(row, column), at + (kEven ? (min(row, last) - t / G::kPer) * a.slot_stride : min(row, last) * a.slot_stride + column * G::kCopy));
            }
        }
        at += kTileOfKeys * a.slot_stride;
        left -= kTileOfKeys;
    }
};

template <int C>
struct TileCtrl {
    unsigned long long k_full[2], s_full[2], s_free[2], v_full[2], p_full[2], pv_done[2], o_free, drain;
    uint32_t see[kTileGroups][64];                                          // per group and node: the rows that see it
    long long out[64];                                            // where a row's output goes (element offset)
    float neg_ref[64];
    int tile_max[kTileGroups][4][C];
    float sums[kTileGroups][4][C];
    unsigned long long vote[kTileGroups][2];                      // the warps of a group have looked at their scores; a reference has to go up
    int hot[kTileGroups][2];
    int first[kTileGroups], last[kTileGroups], second[kTileGroups];          // the unit's pieces
    uint32_t tmem;
    int abort, joined;
};

__device__ __forceinline__ void tile_wait(uint32_t bar, uint32_t parity, int* abort, int* status) {
    if (!mbar_try(bar, parity)) mbar_wait_slow(bar, parity, abort, status);
}
// 128 threads agree on "any"
__device__ __forceinline__ bool any_of_group(int id, bool x) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbar.red.or.pred q, %1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(id), "r"(static_cast<uint32_t>(x)) : "memory");
    return r != 0u;
}
template <int C>
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[C]) {
    if constexpr (C == 32) tmem_ld32<0>(addr, r);
    else if constexpr (C == 16) tmem_ld16<0>(addr, r);
    else
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr) : "memory");
}
template <int C, int O, int M>
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[M]) {
    if constexpr (C == 32)
        asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                     "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::SS_W16(r, O), SS_W16(r, O + 16), "r"(addr) : "memory");
    else if constexpr (C == 16) tmem_st16<O>(addr, r);
    else
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
                     ::"r"(r[O]), "r"(r[O + 1]), "r"(r[O + 2]), "r"(r[O + 3]), "r"(r[O + 4]), "r"(r[O + 5]), "r"(r[O + 6]), "r"(r[O + 7]), "r"(addr) : "memory");
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

template <int D, int N>
__global__ void __launch_bounds__(kTileThreads, 1) msa_attention_kvq_tiles_kernel(const __grid_constant__ KvqArgs a) {
    using G = TileGeo<D, N>;
    constexpr int C = G::kRowsOfGroup;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(16) TileCtrl<C> c;
    __shared__ __align__(16) TileWalk<N> walks[3 + kTileGroups];    // K, V, softmax groups, MMAs
    const int tid = threadIdx.x, lane = tid & 31, warp = static_cast<int>(uniform(tid >> 5)), quad = warp & 3;
    const uint32_t smem = smem_u32(smem_raw);
    int* const status = reinterpret_cast<int*>(a.ws);
    if (tid == 0) {
        c.abort = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&c.k_full[i]), 128), mbar_init(smem_u32(&c.v_full[i]), 128);
            mbar_init(smem_u32(&c.s_free[i]), kTileSoftmax), mbar_init(smem_u32(&c.p_full[i]), kTileSoftmax);
            mbar_init(smem_u32(&c.s_full[i]), 2), mbar_init(smem_u32(&c.pv_done[i]), 1);
        }
        for (int i = 0; i < 2 * kTileGroups; ++i) mbar_init(smem_u32(&c.vote[i >> 1][i & 1]), 4), c.hot[i >> 1][i & 1] = 0;
        mbar_init(smem_u32(&c.o_free), kTileSoftmax), mbar_init(smem_u32(&c.drain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    wait_for_previous_kernel();
    release_next_kernel();
    if (warp < 3 + kTileGroups) {
        Line<N, kTileOfKeys, 0, kTileStart> line;
        const bool any = line.begin(a, lane);
        if (lane == 0) walks[warp].line = line, walks[warp].more = any;
    }
    __syncthreads();
    if (walks[0].more == 0) return;
    constexpr int kMmaWarp = kTileThreads / 32 - 1;
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&c.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(c.tmem), lanes = static_cast<uint32_t>(32 * quad) << 16;
    // (a wait that runs out leaves the roles in step: everyone goes through the same tiles without waiting, and no output is written)
    const auto wait = [&](unsigned long long& bar, uint32_t parity) { tile_wait(smem_u32(&bar), parity, &c.abort, status); };
    // on to the next unit, all `threads` threads of a role together; id: their barrier
    const auto next_unit = [&](TileWalk<N>& w, bool leader, int id, int threads) {
        if (threads > 32) named_barrier(id, threads); else __syncwarp();
        if (leader) w.more = w.line.next(a);
        if (threads > 32) named_barrier(id, threads); else __syncwarp();
        return w.more != 0;
    };
    uint32_t tau = 0;                                // tiles so far, over all units: buffer tau & 1, phase (tau >> 1) & 1

    if (warp < 4) {
        // ---- K ------------------------------------------------------------------------------
        const int key = tid;
        const Line<N, kTileOfKeys, 0, kTileStart>& line = walks[0].line;
        while (next_unit(walks[0], tid == 0, 1, 128)) {
            const Seq s = line.s;
            const int P = prefix_chunks<kTileOfKeys>(s.L), from = line.from, to = line.to, held = min(to, P), h = min(line.head0, a.n_heads - 1);
            const bool real = line.head0 < a.n_heads;
            // (the ring's last stage has been read by all)
            const uint32_t tau0 = tau;
            TileLoader<D, N> loader(a, s, h, from, tid, a.k_codes);
            const long long words = (s.start + static_cast<long long>(from) * kTileOfKeys) * a.p_slot + h * a.p_head;
            const auto load = [&](int k) {           // codes, scales and zero points of tile k
                if (k < held) {
                    loader.next(a, smem + G::oK + ((k - from) % G::kStages) * G::kCodes, tid);
                    const long long p = words + (static_cast<long long>(k - from) * kTileOfKeys + min(key, s.L - 1 - k * kTileOfKeys)) * a.p_slot;
                    const uint32_t dst = smem + G::oKParams + (((tau0 + (k - from)) % G::kParams) * kTileOfKeys + key) * 8;
                    copy_async<4>(dst, a.k_params + p);
                    copy_async<4>(dst + 4, a.v_params + p);
                }
                copy_commit();
            };
            #pragma unroll 1
            for (int i = 0; i < G::kStages - 1; ++i) load(from + i);
            // what lies behind the prefix comes to L2 meanwhile
            if (to > P && real) prefetch_extra(a, extra_of(a, s, line.row0, N), D, line.b, h, key, a.k_tree, a.k_spec);
            // query rows, 16 bytes at a time (all of a thread's on their way at once), swizzled
            {
                constexpr int kItems = N * (D / 8) / 128;
                uint4 v[kItems];
                #pragma unroll
                for (int i = 0; i < kItems; ++i) {
                    const int item = i * 128 + tid, r = item / (D / 8), at = item - r * (D / 8);
                    v[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (real && line.row0 + r < s.rows) {
                        const int row = line.row0 + r;
                        v[i] = *reinterpret_cast<const uint4*>((row < s.T ? a.q_main : a.q_spec) + row_offset(a, D, line.b, h, row, s.T) + 8 * at);
                    }
                }
                // the rows of the unit before have been read once its last S is complete
                if (tau > 0) wait(c.s_full[(tau - 1) & 1], ((tau - 1) >> 1) & 1);
                #pragma unroll
                for (int i = 0; i < kItems; ++i) {
                    const int item = i * 128 + tid, r = item / (D / 8), at = item - r * (D / 8);
                    st_shared_v4(smem + G::oQ + (at >> 3) * G::kBox + r * 128 + (((at & 7) ^ (r & 7)) << 4), v[i].x, v[i].y, v[i].z, v[i].w);
                }
            }
            fence_async_smem();
            #pragma unroll 1
            for (int k = from; k < to; ++k, ++tau) {
                uint32_t w[G::kWords];
                uint32_t z = 0u;
                const uint32_t params = smem + G::oKParams + ((tau % G::kParams) * kTileOfKeys + key) * 8;
                if (k < held) {
                    copy_wait<G::kStages - 2>();
                    named_barrier(1, 128);
                    load(k + G::kStages - 1);
                    const uint32_t row = smem + G::oK + ((k - from) % G::kStages) * G::kCodes + key * G::kPitch;
                    #pragma unroll
                    for (int i = 0; i < G::kWords / 4; ++i) {
                        const uint4 v = lds128(row + 16 * (D == 128 ? i ^ ((key >> 1) & 3) : D == 64 ? i ^ ((key >> 2) & 1) : i));
                        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
                    }
                    if constexpr (D == 80) {
                        const uint2 v = lds64(row + 32);
                        w[8] = v.x, w[9] = v.y;
                    }
                    z = code_plus_128(__byte_perm(lds32(params), 0u, 0x3232));
                } else {
                    asm volatile("st.shared.v2.u32 [%0], {%1, %1};" ::"r"(params), "r"(0x3f80u) : "memory");      // scales of 1
                }
                if (tau >= 2) wait(c.s_full[tau & 1], ((tau - 2) >> 1) & 1);
                tc_fence_after();
                const uint32_t dst = tmem + G::kTmemK + (tau & 1) * 64 + lanes;
                const __nv_bfloat16* src = nullptr;
                if (k >= held && real) {
                    const Extra x = extra_of(a, s, line.row0, N);
                    const int e = (k - P) * kTileOfKeys + key;
                    if (e < x.count) src = (e < x.T ? a.k_tree : a.k_spec) + extra_offset(a, x, D, line.b, h, e);
                }
                #pragma unroll
                for (int i = 0; i < G::kWords; i += 8) {
                    uint32_t r[32];
                    #pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        if (i + q < G::kWords) {
                            if (k < held) {
                                #pragma unroll
                                for (int n = 0; n < 4; ++n) r[4 * q + n] = sub_bf16x2(code_plus_128(w[i + q] >> (4 * n)), z);
                            } else {
                                uint4 v = {};
                                if (src) v = *reinterpret_cast<const uint4*>(src + 8 * (i + q));
                                r[4 * q] = v.x, r[4 * q + 1] = v.y, r[4 * q + 2] = v.z, r[4 * q + 3] = v.w;
                            }
                        }
                    }
                    if (i + 8 <= G::kWords) tmem_store<32, 0>(dst + 4 * i, r);
                    else tmem_store<8, 0>(dst + 4 * i, r);           // (80: the last two words)
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(smem_u32(&c.k_full[tau & 1]));
            }
            copy_wait<0>();
        }
    } else if (warp < 8) {
        // ---- V ------------------------------------------------------------------------------
        const int t = tid - 128;
        const bool mine = quad < G::kQuads;
        // keys in the order in which the columns of V^T follow one another: transposed byte 4 q + e of 16 keys goes to column q (e < 2) or
        // 4 + q, which hold keys 2 q, 2 q + 1 and 8 + 2 q, 8 + 2 q + 1
        const int from16 = (lane & 3) < 2 ? 2 * ((lane & 15) >> 2) + (lane & 3) : 8 + 2 * ((lane & 15) >> 2) + (lane & 3) - 2;
        const Line<N, kTileOfKeys, 0, kTileStart>& line = walks[1].line;
        while (next_unit(walks[1], t == 0, 2, 128)) {            // (the ring's last stage has been read by all)
            const Seq s = line.s;
            const int P = prefix_chunks<kTileOfKeys>(s.L), from = line.from, to = line.to, held = min(to, P), h = min(line.head0, a.n_heads - 1);
            const bool real = line.head0 < a.n_heads;
            TileLoader<D, N> loader(a, s, h, from, t, a.v_codes);
            const long long words = (s.start + static_cast<long long>(from) * kTileOfKeys) * a.p_slot + h * a.p_head;
            const auto load = [&](int k) {
                if (k < held) {
                    const int st = (k - from) % G::kStages;
                    loader.next(a, smem + G::oV + st * G::kCodes, t);
                    copy_async<4>(smem + G::oVParams + (st * kTileOfKeys + t) * 4,
                                  a.v_params + words + (static_cast<long long>(k - from) * kTileOfKeys + min(t, s.L - 1 - k * kTileOfKeys)) * a.p_slot);
                }
                copy_commit();
            };
            #pragma unroll 1
            for (int i = 0; i < G::kStages - 1; ++i) load(from + i);
            if (to > P && real) prefetch_extra(a, extra_of(a, s, line.row0, N), D, line.b, h, t, a.v_tree, a.v_spec);
            #pragma unroll 1
            for (int k = from; k < to; ++k, ++tau) {
                const int st = (k - from) % G::kStages;
                const uint32_t dst = tmem + G::kTmemV + (tau & 1) * 64 + lanes;
                if (k < held) {
                    copy_wait<G::kStages - 2>();
                    named_barrier(2, 128);
                    load(k + G::kStages - 1);
                    if (tau >= 2) wait(c.pv_done[tau & 1], ((tau - 2) >> 1) & 1);
                    tc_fence_after();
                    if (mine) {
                        const uint32_t codes = smem + G::oV + st * G::kCodes, words = smem + G::oVParams + st * kTileOfKeys * 4 + 8 * (lane & 3);
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
                } else {
                    // bf16 rows in the order of the lanes: of 8 values the low codes' would be 0, 4, 1, 5, the high codes' 2, 6, 3, 7.  64 keys at
                    // a time, in the ring's place; a row's words are shared by two threads.
                    const Extra x = extra_of(a, s, line.row0, N);
                    const int r = t >> 1;
                    const bool both = (k - P) * kTileOfKeys + 64 < x.count;      // (else the tile's upper half is empty)
                    uint4 v[2 * G::kQuads];
                    const auto fetch = [&](int half) {
                        const int e = (k - P) * kTileOfKeys + 64 * half + r;
                        const __nv_bfloat16* src = nullptr;
                        if (real && e < x.count) src = (e < x.T ? a.v_tree : a.v_spec) + extra_offset(a, x, D, line.b, h, e);
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
                        const uint32_t row = smem + G::oV + r * G::kRowOfV;
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
                                    load_transposed_halves(smem + G::oV + kk * G::kRowOfV + (((at >> 4) ^ (kk & 3)) << 4), q);
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
            copy_wait<0>();
        }
    } else if (warp < kMmaWarp) {
        // ---- softmax ------------------------------------------------------------------------
        const int group = (warp - 8) >> 2, key = 32 * quad + lane, bar = 3 + group;
        constexpr uint32_t all = C == 32 ? 0xffffffffu : (1u << C) - 1u;
        uint32_t unit = 0;
        int* const counters = reinterpret_cast<int*>(a.ws + kWsHeaderBytes);
        float* const partial = reinterpret_cast<float*>(a.ws + kWsHeaderBytes + (4ull * gridDim.x + 255) / 256 * 256);
        constexpr int kPartial = N * (D + 4);
        const uint32_t weights = smem + G::oP + key * 128;        // the key's row of P^T
        // TMEM lane to dimension
        const int byte = 16 * quad + (lane & 15), dim = 8 * (byte >> 2) + ((byte & 1) << 2) + ((byte >> 1) & 1) + ((lane >> 4) << 1);
        const Line<N, kTileOfKeys, 0, kTileStart>& line = walks[2 + group].line;
        while (next_unit(walks[2 + group], key == 0, bar, 128)) {
            const Seq& s = line.s;
            const int L = s.L, P = prefix_chunks<kTileOfKeys>(L), from = line.from, to = line.to;
            const Extra x = extra_of(a, s, line.row0, N);
            {
                const int n = group * C + lane, r = line.row0 + n;
                unsigned long long see = 0;
                long long out = 0;
                if (lane < C && r < s.rows && line.head0 < a.n_heads) {
                    see = a.trees[line.b].anc_mask[row_of(r, s.T, a.gamma).t];
                    out = row_offset(a, D, line.b, line.head0, r, s.T);
                }
                uint32_t own = 0u;
                #pragma unroll
                for (int i = 0; i < 16; ++i) {       // nodes 16 quad ..
                    const uint32_t rows = __ballot_sync(0xffffffffu, see >> (16 * quad + i) & 1ull);
                    if (lane == i) own = rows;
                }
                if (lane < 16) c.see[group][16 * quad + lane] = own;
                if (quad == 0 && lane < C) c.out[n] = out, c.neg_ref[n] = 0.f;
                if (key == 96) {
                    const Pieces share(line);
                    c.first[group] = share.first, c.last[group] = share.last, c.second[group] = share.second;
                }
            }
            named_barrier(bar, 128);
            float l[C];
            #pragma unroll
            for (int i = 0; i < C; ++i) l[i] = 0.f;
            uint32_t seen = 0u;                      // rows that have seen a key (the same in all warps of the group)
            #pragma unroll 1
            for (int k = from; k < to; ++k, ++tau) {
                const uint32_t parity = (tau >> 1) & 1;
                wait(c.s_full[tau & 1], parity);
                tc_fence_after();
                const uint2 params = lds64(smem + G::oKParams + ((tau % G::kParams) * kTileOfKeys + key) * 8);
                const float sk = scale_of(params.x) * a.scale, sv = scale_of(params.y);
                // rows that see the key: all of them if it is a cached one; else those of its node's descendants; of a stream key, from its
                // own row to its node's last
                uint32_t vis = all;
                if (k < P) {
                    if (k * kTileOfKeys + key >= L) vis = 0u;
                } else {
                    const int e = (k - P) * kTileOfKeys + key;
                    vis = 0u;
                    if (e < x.T) {
                        vis = c.see[group][e];
                    } else if (e < x.count) {
                        const int own = e - x.T + x.t0 * x.gamma, first = x.T + own - x.row0 - group * C, last = first + x.gamma - 1 - own % x.gamma;
                        if (first < C && last >= 0) vis = (0xffffffffu >> (31 - min(last, 31))) & (0xffffffffu << max(first, 0));
                    }
                }
                const bool masked = __any_sync(0xffffffffu, (vis & all) != all);
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
                wait(c.vote[group][tau & 1], parity);
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
                        wait(c.pv_done[(tau - 1) & 1], ((tau - 1) >> 1) & 1);
                        tc_fence_after();
                        #pragma unroll
                        for (int i = 0; i < C; i += 8) {
                            uint32_t o[8];
                            tmem_load<8>(tmem + G::kTmemO + group * C + i + lanes, o);
                            tmem_wait_ld();
                            #pragma unroll
                            for (int q = 0; q < 8; ++q) o[q] = __float_as_uint(__uint_as_float(o[q]) * __shfl_sync(0xffffffffu, f, i + q));
                            tmem_store<8, 0>(tmem + G::kTmemO + group * C + i + lanes, o);
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
            wait(c.pv_done[(tau - 1) & 1], ((tau - 1) >> 1) & 1);
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
            const bool ok = *const_cast<volatile int*>(&c.abort) == 0;
            const int rows = line.head0 < a.n_heads ? min(N, s.rows - line.row0) : 0;
            if (line.whole()) {
                const float f = 1.f / sum;
                if (quad == 0 && lane < C && ok && group * C + lane < rows) {
                    const int n = group * C + lane;
                    float* lse = line.row0 + n < s.T ? a.lse_main : a.lse_spec;
                    if (lse != nullptr) lse[c.out[n] / D] = (ref + log2f(sum)) * 0.6931471805599453f;
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
                        if (n < rows && ok)
                            *reinterpret_cast<uint32_t*>((line.row0 + n < s.T ? a.o_main : a.o_spec) + c.out[n] + 8 * wi + 2 * (lane & 3)) = q[i];
                    }
                }
                named_barrier(bar, 128);             // (the next unit's weights go there)
            } else {
                float* const mine = partial + (2ll * ((line.me << line.team_log2) + line.member) + (line.me == c.first[group] ? c.second[group] : 0)) * kPartial;
                if (quad == 0 && lane < C)
                    __stcg(reinterpret_cast<float2*>(mine + (group * C + lane) * (D + 4) + D), make_float2(seen >> lane & 1u ? ref : kNoRef, sum));
                if (dim < D) {
                    #pragma unroll
                    for (int i = 0; i < C; ++i) __stcg(mine + (group * C + i) * (D + 4) + dim, __uint_as_float(raw[i]));
                }
                named_barrier(3 + kTileGroups, kTileSoftmax);
                if (tid == 256) {
                    c.joined = last_piece(counters + (c.first[0] << line.team_log2) + line.member, c.last[0] - c.first[0] + 1);
                }
                named_barrier(3 + kTileGroups, kTileSoftmax);
                if (c.joined) {
                    // 8 values of a row at a time, up to four partial rows on their way
                    const int first = c.first[group], n = c.last[group] - first + 1, items = rows * (D / 8);
                    const float* const p0 = partial + (2ll * ((first << line.team_log2) + line.member) + c.second[group]) * kPartial;
                    const long long on = (2ll << line.team_log2) * kPartial;                 // between teams' places
                    const float* const p1 = p0 - c.second[group] * kPartial + on;
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
                        if (ok) store_row<D>(a, line.row0 + r < s.T, c.out[r], d0, o, m, sm);
                    }
                    named_barrier(3 + kTileGroups, kTileSoftmax);           // (all groups read all rows' places)
                }
            }
            ++unit;
        }
    } else {
        // ---- MMAs ---------------------------------------------------------------------------
        const uint32_t base = uniform(smem);
        const uint64_t dq = desc_k_major(base + G::oQ), dp = desc_mn_major(base + G::oP, 0);
        const Line<N, kTileOfKeys, 0, kTileStart>& line = walks[2 + kTileGroups].line;
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
        while (next_unit(walks[2 + kTileGroups], lane == 0, 0, 32)) {
            const uint32_t tiles = uniform(static_cast<uint32_t>(line.to - line.from));
            #pragma unroll 1
            for (uint32_t i = 0; i < tiles; ++i, ++tau) {
                wait(c.k_full[tau & 1], (tau >> 1) & 1);
                if (tau >= 2) wait(c.s_free[tau & 1], ((tau - 2) >> 1) & 1);
                tc_fence_after();
                const uint32_t ka = tmem + G::kTmemK + (tau & 1) * 64, sd = tmem + G::kTmemS + (tau & 1) * N;
                tile_mma<4>(sd, ka, dq, G::kIdescS, 0u);
                if constexpr (D == 128) tile_mma<4>(sd, ka + 32, dq + (G::kBox >> 4), G::kIdescS, 1u);
                if constexpr (D == 80) tile_mma<1>(sd, ka + 32, dq + (G::kBox >> 4), G::kIdescS, 1u);
                tc_commit_e(smem_u32(&c.s_full[tau & 1]));
                if (lane == 0) mbar_arrive(smem_u32(&c.s_full[tau & 1]));            // (passes on what the K warps have written: the keys' scales)
                if (i > 0) product(tau - 1, i == 1);
            }
            product(tau - 1, tiles == 1);
            ++unit;
        }
        tc_commit_e(smem_u32(&c.drain));
        mbar_drain(smem_u32(&c.drain), 0);           // (nothing is in flight when TMEM goes back)
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

}  // namespace ss
