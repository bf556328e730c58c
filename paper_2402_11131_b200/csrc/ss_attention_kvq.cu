// Tree-masked multi-stream attention over a prefix held in 4 bits (Eq. 1, Eq. 2; format: ss_msa.h).
#include <cuda_bf16.h>
#include <cfloat>

#include "ss_common.cuh"

namespace ss {

struct alignas(16) KvqArgs {
    const unsigned char *k_codes, *v_codes;          // of this layer
    const uint32_t *k_params, *v_params;
    long long slot_stride, head_stride, p_slot, p_head, total_slots;
    const __nv_bfloat16 *q_main, *q_spec, *k_tree, *v_tree, *k_spec, *v_spec;
    __nv_bfloat16 *o_main, *o_spec;
    float *lse_main, *lse_spec;
    const int64_t* kv_start;
    const int32_t* kv_len;
    const int32_t* kv_capacity;
    const ss_tree_desc* trees;
    unsigned char* ws;
    float scale;                                     // sm_scale * log2(e)
    int batch, n_heads, gamma, max_nodes;
};

// ---- work ---------------------------------------------------------------------------------------
// A unit is a block of query rows of some neighbouring heads of one sequence.  Its keys are cut in chunks of 32: the cached slots, then
// the tree's nodes and the stream keys of the block's own nodes.  A team of CTAs takes a unit together: each of its CTAs has HW
// heads, whose chunks go to its warps, warps / HW chunks of each at a time, a step.  All units' steps, in order of sequence, heads
// and block, are one line that is cut into equal pieces, one per team: a team takes the end of a unit, whole units, and the beginning of
// another.  So every CTA reads the same amount, whatever the lengths (which only the device knows).
// Why neighbouring heads at the same time: with slots as the outer dimension of the cache a head's row of a slot is 64 bytes, and CTAs
// that read single heads at unrelated slots keep DRAM at 2.5 TB/s (64 users, 267638 keys of 128: 485 us; four heads per CTA 265 us).
constexpr int kChunk = 32;
constexpr int kWarps = 4, kWarpsLog2 = 2, kThreads = 32 * kWarps;
constexpr int kStepsForHeads = 6;
constexpr int kMostKeys = 0x7fff0000;                // (places of chunks asked for ahead stay below 2^31)

struct Seq {
    int L, T, rows, blocks, chunks;                  // rows and blocks of rows per head, chunks of each: cached ones and those behind
    long long start;
};

template <int CHUNK>
__device__ __forceinline__ int prefix_chunks(int L) { return (L + CHUNK - 1) / CHUNK; }

// Most keys behind the prefix that a block of `block` rows sees: all nodes, and the streams of the nodes its rows belong to
template <int CHUNK>
__host__ __device__ __forceinline__ int extra_chunks(int T, int gamma, int block) {
    int stream = 0;
    if (gamma > 0) {
        const int nodes = (block + gamma - 2) / gamma + 1;
        stream = (nodes < T ? nodes : T) * gamma;
    }
    return (T + stream + CHUNK - 1) / CHUNK;
}

// One sequence as the call gives it.  A sequence that cannot be run has no blocks.
template <int ROWS, int CHUNK>
__device__ __forceinline__ Seq load_seq(const KvqArgs& a, int b) {
    Seq s;
    s.L = a.kv_len[b];
    s.start = a.kv_start[b];
    s.T = min(a.trees[b].n_nodes, a.max_nodes);
    const bool fits = s.L >= 0 && s.L <= kMostKeys && s.start >= 0 && s.start <= a.total_slots - s.L && (a.kv_capacity == nullptr || s.L <= a.kv_capacity[b]);
    if (!fits) set_status(a.ws, SS_ERR_CAPACITY);
    if (!fits || s.T < 1) s.T = s.rows = s.blocks = s.chunks = 0;
    else {
        s.rows = s.T * (1 + a.gamma);
        s.blocks = (s.rows + ROWS - 1) / ROWS;
        s.chunks = prefix_chunks<CHUNK>(s.L) + extra_chunks<CHUNK>(s.T, a.gamma, ROWS);
    }
    return s;
}

// Heads per CTA and CTAs per team (log2 of both), for `chunks` chunks and `blocks` blocks of one head.  Where every CTA has some steps a
// unit has as many as 32 heads, as long as at most an eighth of the places have none; a CTA has as many of them as it has warps (there is
// nothing to join then), as long as a unit is not cut in more than some ten pieces.  With only a few steps, one head's keys over
// all warps leave fewer partial results to join.
struct Shape {
    int heads, team;
};
template <int WARPS_LOG2>
__device__ __forceinline__ Shape shape_of(const KvqArgs& a, long long chunks, long long blocks) {
    Shape s{0, 0};
    if (chunks * a.n_heads < (static_cast<long long>(kStepsForHeads) << WARPS_LOG2) * gridDim.x) return s;
    const auto fits = [&](int lg) { return 8 * ((a.n_heads + (1 << lg) - 1) >> lg << lg) <= 9 * a.n_heads; };
    while (s.heads < WARPS_LOG2 && fits(s.heads + 1) && 10 * blocks * (a.n_heads >> (s.heads + 1)) >= gridDim.x) ++s.heads;
    while (s.team < 3 && fits(s.heads + s.team + 1)) ++s.team;
    return s;
}

// Sum over a warp of numbers from 0 to 2^42
__device__ __forceinline__ long long warp_sum(long long x) {
    const uint32_t lo = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(x) & 0xffffu), hi = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(x >> 16));
    return (static_cast<long long>(hi) << 16) + lo;
}
__device__ __forceinline__ long long divide(long long a, long long b) {
    return (a >> 32) == 0 && (b >> 32) == 0 ? static_cast<long long>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}

// Row r of a unit's sequence: its node and stream (-1: main stream)
struct Row {
    int t, j;
};
__device__ __forceinline__ Row row_of(int r, int T, int gamma) {
    if (r < T) return Row{r, -1};
    const int s = r - T, t = s / gamma;
    return Row{t, s - t * gamma};
}

// Element offset of row r's vector in the main-stream tensors (r < T) or in the streams' (rows there follow one another as they do here)
__device__ __forceinline__ long long row_offset(const KvqArgs& a, int hd, int b, int h, int r, int T) {
    const int nodes = b * a.max_nodes;               // (at most 65535 sequences' worth, see the entry point)
    return ((r < T ? static_cast<long long>(nodes) + r : static_cast<long long>(nodes) * a.gamma + (r - T)) * a.n_heads + h) * hd;
}

constexpr float kNoRef = -FLT_MAX / 2;               // reference of a partial result that has seen no key

// ---- small helpers ------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t r;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 r;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a));
    return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a));
    return r;
}
__device__ __forceinline__ float exp2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Codes as fp16 operands: a code in the last four mantissa bits of a half word is the subnormal number c 2^-24, one in the four bits above
// them 16 c 2^-24, exactly, and MMAs take subnormal numbers at full value.  So a mask is all it takes, and a shift by 8 for the other two
// codes of a half word; the powers of two are dealt with where sums end.  V's zero points are too: the weights' sums of codes are at most
// some 15 / |c - z| larger than those of values.  Not so K's: they are subtracted here, exactly again, so that scores are sums of q (c - z), no
// larger than the score's own terms.  (With zero points applied to the sums of q, scores of queries with a mean and keys with a large
// channel were off by up to 4 10^-4.  The subtractions cost 1.5 to 2 %: 100,000 keys and 5 rows 93.2 -> 94.6 us, 16 users' tokens 42.7 -> 43.5;
// nothing that shows where memory bounds: 64 users.)
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return w & 0x000f000fu; }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return w & 0x00f000f0u; }
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t less_16_times(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("{.reg .b32 m;\n\tmov.b32 m, 0xcc00cc00;\n\tfma.rn.f16x2 %0, %1, m, %2;}" : "=r"(r) : "r"(b), "r"(a));      // (-16 twice)
    return r;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t times16_bf16x2(uint32_t x) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0x41804180u));
    return r;
}
__device__ __forceinline__ uint32_t zero_pair(uint32_t a, uint32_t b) { return low_codes(__byte_perm(a, b, 0x7632)); }     // of two keys
__device__ __forceinline__ float scale_of(uint32_t word) { return __uint_as_float(word << 16); }
__device__ __forceinline__ uint32_t zero_of(uint32_t word) { return __byte_perm(word, 0u, 0x3232); }                            // twice
constexpr float kCode = 5.9604644775390625e-08f;                 // 2^-24: what a code counts in an MMA

// Pieces of a lone sequence's unit.  What joining p pieces takes grows with p, what the steps of one take falls as 1 / p: the best p grows
// as the root of the steps.  (Two heads of 64 with 20,000 keys, one row: 14.6 us; in as many pieces as there are CTAs 22.7, with twice the
// root as the limit 0.8 more.)  Two steps are not worth a join at all (7.6 against 8.5 us).
// Not the fewest pieces for their longest one: 2048 keys are 17 steps in 12 pieces of one or two, which nine would be as well (8 rows: 13.4 us;
// by the kernel for 16, whose grid allows nine, 11.6).  And equal pieces for all units leave CTAs over: 28 of 444 with 32 heads, 20 of 148 on tcgen05.
__device__ __forceinline__ int most_pieces(int steps) { return steps < 3 ? 1 : static_cast<int>(3.f * sqrtf(static_cast<float>(steps))); }

// The line of steps as one CTA sees it (every thread, or one warp of a role, works it out for itself)
// START: what a unit costs before its first step, in steps, for the sake of an even deal.
template <int ROWS, int CHUNK, int WARPS_LOG2, int START>
struct Line {
    int heads_log2, team_log2, steps_log2;           // heads and chunks per step of a CTA, CTAs of a team
    int groups, me, member;                          // of heads; this CTA's team and its place there
    int pieces, whole_steps;
    long long total, share, rest;
    long long pos, end, base;                        // the piece's next step and its end; first step of sequence b
    int b, steps, units, unit, start;                // sequence; its units and their steps; the next unit; steps that stand for a unit's start
    Seq s;
    // the unit at hand
    long long unit0;                                 // its first step's place in the line
    int from, to, head0, row0;                       // steps of it, its first head for this CTA and its first row

    __device__ __forceinline__ int steps_of(const Seq& q) const { return (q.chunks + (1 << steps_log2) - 1) >> steps_log2; }
    __device__ __forceinline__ long long line_of(const Seq& q) const { return static_cast<long long>(q.blocks > 0 ? steps_of(q) + start : 0) * q.blocks * groups; }
    // first step of team i's piece
    __device__ __forceinline__ long long cut(int i) const {
        const int u = pieces > 0 ? i / pieces : 0, k = i - u * pieces;
        return static_cast<long long>(u) * whole_steps + k * share + min(static_cast<long long>(k), rest);
    }
    // false: nothing for this CTA.  All lanes of a warp come here.
    __device__ __forceinline__ bool begin(const KvqArgs& a, int lane) {
        const bool lone = a.batch == 1;              // (every lane has it: no sums, no searches)
        long long chunks = 0, blocks = 0;            // of all sequences, for one head
        Seq mine;                                    // the lane's sequence of the first 32
        if (lone) {
            mine = load_seq<ROWS, CHUNK>(a, 0);
            chunks = static_cast<long long>(mine.chunks) * mine.blocks, blocks = mine.blocks;
        }
        #pragma unroll 1
        for (int b0 = 0; b0 < (lone ? 0 : a.batch); b0 += 32) {
            const Seq q = b0 + lane < a.batch ? load_seq<ROWS, CHUNK>(a, b0 + lane) : Seq{};
            if (b0 == 0) mine = q;
            chunks += warp_sum(static_cast<long long>(q.chunks) * q.blocks);
            blocks += warp_sum(q.blocks);
        }
        const Shape shape = shape_of<WARPS_LOG2>(a, chunks, blocks);
        heads_log2 = shape.heads, team_log2 = shape.team, steps_log2 = WARPS_LOG2 - shape.heads;
        groups = (a.n_heads + (1 << (heads_log2 + team_log2)) - 1) >> (heads_log2 + team_log2);
        start = lone ? 0 : START;
        total = lone ? line_of(mine) : 0;
        #pragma unroll 1
        for (int b0 = 0; b0 < (lone ? 0 : a.batch); b0 += 32)
            total += warp_sum(b0 + lane < a.batch ? line_of(b0 == 0 ? mine : load_seq<ROWS, CHUNK>(a, b0 + lane)) : 0);
        long long teams = min(static_cast<long long>(gridDim.x >> team_log2), total);
        // one sequence with fewer units than teams: every unit in the same number of pieces, so that all heads' pieces read the same slots
        // at the same time
        pieces = whole_steps = 0;
        if (lone && total > 0) {
            const int n = mine.blocks * groups;
            whole_steps = steps_of(mine);
            pieces = static_cast<int>(static_cast<uint32_t>(teams) / static_cast<uint32_t>(n));
            if (pieces > 0) pieces = min(pieces, most_pieces(whole_steps)), teams = static_cast<long long>(pieces) * n;
        }
        me = static_cast<int>(blockIdx.x) >> team_log2, member = static_cast<int>(blockIdx.x) - (me << team_log2);
        if (me >= teams) return false;
        share = pieces > 0 ? whole_steps / pieces : divide(total, teams);
        rest = (pieces > 0 ? whole_steps : total) - share * (pieces > 0 ? pieces : teams);
        pos = cut(me), end = cut(me + 1);
        // the sequence that holds the piece's first step
        base = 0, b = 0;
        #pragma unroll 1
        for (int b0 = 0; b0 < (lone ? 0 : a.batch); b0 += 32) {
            const long long own = b0 + lane < a.batch ? line_of(b0 == 0 ? mine : load_seq<ROWS, CHUNK>(a, b0 + lane)) : 0;
            long long upto = own;
            #pragma unroll
            for (int x = 1; x < 32; x <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, upto, x);
                if (lane >= x) upto += y;
            }
            const unsigned here = __ballot_sync(0xffffffffu, base + upto > pos);
            if (here) {
                const int l = __ffs(here) - 1;
                b = b0 + l;
                base += __shfl_sync(0xffffffffu, upto - own, l);
                break;
            }
            base += __shfl_sync(0xffffffffu, upto, 31);
        }
        if (lone) {
            s = mine;
        } else if (b < 32) {                         // (a lane has it)
            s.L = __shfl_sync(0xffffffffu, mine.L, b), s.T = __shfl_sync(0xffffffffu, mine.T, b), s.rows = __shfl_sync(0xffffffffu, mine.rows, b);
            s.blocks = __shfl_sync(0xffffffffu, mine.blocks, b), s.chunks = __shfl_sync(0xffffffffu, mine.chunks, b), s.start = __shfl_sync(0xffffffffu, mine.start, b);
        } else {
            s = load_seq<ROWS, CHUNK>(a, b);
        }
        steps = steps_of(s), units = s.blocks * groups;
        unit = static_cast<int>(divide(pos - base, steps + start));
        return true;
    }
    // the unit at hand, or false at the end of the piece
    __device__ __forceinline__ bool next(const KvqArgs& a) {
        if (pos >= end) return false;
        while (unit >= units) {                      // on to the next sequence that has units
            base += static_cast<long long>(units) * (steps + start);
            s = load_seq<ROWS, CHUNK>(a, ++b);
            steps = steps_of(s), units = s.blocks * groups, unit = 0;
        }
        unit0 = base + static_cast<long long>(unit) * (steps + start) + start;
        from = static_cast<int>(max(pos - unit0, 0ll)), to = static_cast<int>(min(end - unit0, static_cast<long long>(steps)));
        if (to <= from) return false;                // (the piece ends before the unit's first step)
        const int group = static_cast<int>(static_cast<uint32_t>(unit) / static_cast<uint32_t>(s.blocks));
        row0 = (unit - group * s.blocks) * ROWS;
        head0 = ((group << team_log2) + member) << heads_log2;
        pos = unit0 + to;
        ++unit;                                      // (only if it is done: else pos is the end)
        return true;
    }
    __device__ __forceinline__ bool whole() const { return from == 0 && to == steps; }
};

// The CTAs that have a piece of a unit, and where their partial results lie: two places per CTA, for its first unit and its last one
struct Pieces {
    int first, last, second;                         // teams; 1 if the first one has begun another unit before
    template <typename L>
    __device__ __forceinline__ explicit Pieces(const L& line) : first(line.me), last(line.me) {
        long long at = line.unit0;
        if (line.pieces > 0) {
            first -= first % line.pieces, last = first + line.pieces - 1;
        } else if (!line.whole()) {
            #pragma unroll 1
            for (at = line.cut(first); at > line.unit0; at = line.cut(--first)) {}
            #pragma unroll 1
            while (line.cut(last + 1) < line.unit0 + line.steps) ++last;
        }
        second = at < line.unit0 - line.start ? 1 : 0;
    }
    template <typename L>
    __device__ __forceinline__ long long place(const L& line, int i) const { return 2ll * ((i << line.team_log2) + line.member) + (i == first ? second : 0); }
};

// Eight values, from d0 on, of the output of a row that lies at element `off`, and its log-sum-exp: o / l
template <int D>
__device__ __forceinline__ void store_row(const KvqArgs& a, bool main, long long off, int d0, const float (&o)[8], float m, float l) {
    const float f = 1.f / l;
    uint4 v;
    v.x = pack2_bf16(o[0] * f, o[1] * f), v.y = pack2_bf16(o[2] * f, o[3] * f);
    v.z = pack2_bf16(o[4] * f, o[5] * f), v.w = pack2_bf16(o[6] * f, o[7] * f);
    *reinterpret_cast<uint4*>((main ? a.o_main : a.o_spec) + off + d0) = v;
    float* lse = main ? a.lse_main : a.lse_spec;
    if (d0 == 0 && lse != nullptr) lse[off / D] = (m + log2f(l)) * 0.6931471805599453f;
}

// A workspace: the header, the counters (one per CTA, zero between calls), the partial rows.  The counters' room does not depend on
// the call: calls of other shapes on the same workspace leave their partial rows elsewhere.
constexpr int kCounterBytes = 4096;

// One more piece of a unit is in the workspace: true for the last of `n`, who joins them and leaves the counter at zero.  Called by one
// thread behind a barrier of those that wrote: the operation releases their partial rows and acquires the others'.
__device__ __forceinline__ bool last_piece(int* counter, int n) {
    int before;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
    if (before != n - 1) return false;
    *counter = 0;
    return true;
}

// One more partial row into (o, m, l)
__device__ __forceinline__ void join_row(float (&o)[8], float& m, float& l, const float2& st, const float4& u, const float4& v) {
    const float now = fmaxf(m, st.x), f = exp2_approx(m - now), e = exp2_approx(st.x - now);
    m = now, l = l * f + st.y * e;
    o[0] = o[0] * f + u.x * e, o[1] = o[1] * f + u.y * e, o[2] = o[2] * f + u.z * e, o[3] = o[3] * f + u.w * e;
    o[4] = o[4] * f + v.x * e, o[5] = o[5] * f + v.y * e, o[6] = o[6] * f + v.z * e, o[7] = o[7] * f + v.w * e;
}

// ---- the kernel ---------------------------------------------------------------------------------
// S^T = K Q^T and O^T = V^T P^T on mma.sync m16n8k16 with the keys (the dimensions) as the 16 rows of A and NG groups of 8 query
// rows as N: a CTA of 4 warps, each with an online softmax of its own over its chunks of the CTA's piece of a unit, its codes on their way
// through a ring of its own in shared memory.
// What bounds it: with one row the bytes (64 users with up to 8191 keys: 224 to 231 us for 178 of HBM), from some eight rows on, and in long
// sequences, the instructions that make fragments of codes and weights of scores, which is why codes are taken as they lie
// (below: a mask, no conversion) and why keys are the wide side of the products.  Short calls are a chain of latencies: lengths, codes,
// a few steps, partial rows and their join.
//
// Fragments, for lane 4 g + c.  Which key is row g of A, and which dimensions are the columns that c holds, is free as long as both
// operands agree; the choice here lets a lane read runs of codes and turn them into fragments in place:
//   K: lane (g, c) holds dimensions c * D/4 .. of keys key(g) and key(g) + 8 of 16, key(g) = 4 (g & 1) + g / 2
//   V: lane (g, c) holds dimensions g * D/8 .. of keys c, 4 + c, 8 + c, 12 + c: these are what P^T's rows 2c, 2c + 1, 2c + 8 and
//      2c + 9 are under key()
// D = 80 is 64 + 16: the last 16 dimensions are one more step (K) and one more tile (V) in the order of the fragments themselves.
template <int D>
struct KvqGeometry {
    static constexpr int kMain = D == 128 ? 128 : 64;            // dimensions dealt out in runs; the rest (16 of 80) apart
    static constexpr int kRowBytes = D / 2;
    static constexpr int kWordsK = kMain / 32;                   // words of 8 codes per lane and key
    static constexpr int kWordsV = kMain / 64;
    static constexpr int kTiles = D / 16;
    static constexpr int kCopy = D == 80 ? 8 : 16;               // bytes per asynchronous copy
    static constexpr int kCodeBytes = kChunk * kRowBytes;
    static constexpr int kStageBytes = 2 * kCodeBytes + 2 * kChunk * 4;
    static constexpr int kStages = 4;
    static constexpr int kRingBytes = kStages * kStageBytes;
};

template <int D, int NG>
struct KvqSmem {
    using G = KvqGeometry<D>;
    static constexpr int kRows = 8 * NG;
    static constexpr int kPad = D + 4;                           // floats per row of a warp's partial result
    static constexpr int kRing = kWarps * G::kRingBytes;
    static constexpr int kJoin = kWarps * kRows * kPad * 4;
    static constexpr int kBytes = (kRing > kJoin ? kRing : kJoin) + kWarps * kRows * 8;
};

// floats of a CTA's partial result in the workspace: per head and row D sums, the reference and the sum of weights
__host__ __device__ constexpr int partial_floats(int D, int rows) { return kWarps * rows * (D + 4); }

// One warp's share.
// Queries enter as fp16: x = q 2^-e, the row's largest |x| in [2^14, 2^15).  A bf16 has 8 significant bits, so x is exact down to 2^-28 of
// the row's largest element (dimensions that meet codes counting 16 times as much are taken as x / 16), and off by at most 2^-36 of
// that below.
// Weights enter as fp16: p s_v 2^(6 - r), r the exponent of the largest V scale so far.  p is at most 2^8, so nothing overflows; a weight
// keeps 11 bits down to 2^-20 of what the reference would weigh, and is off by at most 2^-31 2^r below.
// o: sums of V's codes (tiles of odd number: 16 times that); zo: the same sum of zero points, which is what is to be subtracted.
template <int D, int NG>
struct WarpState {
    float o[D / 16][NG][4], zo[NG][4];
    float ref[NG][2], sum[NG][2];
    uint32_t q[D / 16][NG][2];
    float factor[NG][2];                             // of the lane's two rows: 2^24 2^e scale
    float weight;                                    // 2^(6 - r)
    float limit;                                     // V scales from here on raise r; 0: none seen yet
};

// Moves the references by `by` (log2 units): up, or, a row's first one, to wherever its maximum lies.  That may be far down, where
// 2^-by is no number any more; there is nothing to scale then.
template <int D, int NG>
__device__ __forceinline__ void move_refs(WarpState<D, NG>& w, const float (&by)[NG][2]) {
    #pragma unroll
    for (int n = 0; n < NG; ++n) {
        #pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float f = exp2_approx(-fmaxf(by[n][e], 0.f));
            w.ref[n][e] += by[n][e];
            w.sum[n][e] *= f;
            w.zo[n][e] *= f;
            #pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                w.o[k][n][e] *= f;
                w.o[k][n][2 + e] *= f;
            }
        }
    }
}

// Raises r to the exponent of a V scale
template <int D, int NG>
__device__ __forceinline__ void raise_scale(WarpState<D, NG>& w, float scale) {
    const uint32_t r = min(max(__float_as_uint(scale) >> 23, 32u), 252u);       // (2^125: the largest scale there is)
    const float now = __uint_as_float((254u + 6u - r) << 23), f = now * __uint_as_float((254u << 23) - __float_as_uint(w.weight));   // (powers of two)
    w.weight = now;
    w.limit = __uint_as_float((r + 1u) << 23);
    #pragma unroll
    for (int n = 0; n < NG; ++n) {
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
            w.zo[n][i] *= f;
            #pragma unroll
            for (int k = 0; k < D / 16; ++k) w.o[k][n][i] *= f;
        }
    }
}

// Scores above their references (d, log2 units; -inf: not seen) of H tiles of 16 keys: where one is more than 8 above, references are
// raised to the maxima and d lowered by as much.  A row that has seen no key so far takes the maximum whatever it is: so the first chunk
// always comes here, by its V scales (no limit holds yet; nor does one for NaN) or, `first`, because it is not a cached one.  `top`: the
// largest V scale.
template <int D, int NG, int H>
__device__ __forceinline__ void keep_in_range(WarpState<D, NG>& w, float (&d)[H][NG][4], float top, bool first) {
    float most = d[0][0][0];
    #pragma unroll
    for (int j = 0; j < H; ++j) {
        #pragma unroll
        for (int n = 0; n < NG; ++n) most = fmaxf(fmaxf(fmaxf(most, d[j][n][0]), fmaxf(d[j][n][1], d[j][n][2])), d[j][n][3]);
    }
    if (__any_sync(0xffffffffu, most > 8.f || !(top < w.limit) || first)) {
        float by[NG][2];
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            #pragma unroll
            for (int e = 0; e < 2; ++e) {
                float m = -INFINITY, seen = w.sum[n][e];
                #pragma unroll
                for (int j = 0; j < H; ++j) m = fmaxf(m, fmaxf(d[j][n][e], d[j][n][2 + e]));
                #pragma unroll
                for (int x = 4; x < 32; x <<= 1) {
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
                    seen += __shfl_xor_sync(0xffffffffu, seen, x);
                }
                m = seen == 0.f ? (m == -INFINITY ? 0.f : m) : fmaxf(m, 0.f);
                by[n][e] = m;
                #pragma unroll
                for (int j = 0; j < H; ++j) d[j][n][e] -= m, d[j][n][2 + e] -= m;
            }
        }
        move_refs<D, NG>(w, by);
        #pragma unroll
        for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        if (top >= w.limit) raise_scale<D, NG>(w, top);
    }
}

__device__ __forceinline__ int key_of(int g) { return 4 * (g & 1) + (g >> 1); }

// One chunk of 32 cached slots, of which the first `valid` count: lane offsets kl (codes of K), vl (of V), pl (words of its keys), zl
template <int D, int NG>
__device__ __forceinline__ void prefix_chunk(WarpState<D, NG>& w, uint32_t stage, int valid, uint32_t kl, uint32_t vl, uint32_t pl, uint32_t zl, int g, int c) {
    using G = KvqGeometry<D>;
    constexpr uint32_t kWordsOfV = 4 * kChunk;
    uint32_t pa[2], pb[2];
    float d[2][NG][4];
    // Scores: sums of x (c - z)
    #pragma unroll
    for (int j = 0; j < 2; ++j) {
        pa[j] = lds32(stage + pl + 64 * j), pb[j] = lds32(stage + pl + 64 * j + 32);
        #pragma unroll
        for (int n = 0; n < NG; ++n) d[j][n][0] = d[j][n][1] = d[j][n][2] = d[j][n][3] = 0.f;
        const uint32_t za = zero_of(pa[j]), zb = zero_of(pb[j]);
        const uint32_t row = stage + kl + j * 16 * G::kRowBytes;
        uint32_t wa[4], wb[4];
        if constexpr (G::kWordsK == 4) {
            const uint4 x = lds128(row), y = lds128(row + 8 * G::kRowBytes);
            wa[0] = x.x, wa[1] = x.y, wa[2] = x.z, wa[3] = x.w;
            wb[0] = y.x, wb[1] = y.y, wb[2] = y.z, wb[3] = y.w;
        } else {
            const uint2 x = lds64(row), y = lds64(row + 8 * G::kRowBytes);
            wa[0] = x.x, wa[1] = x.y, wb[0] = y.x, wb[1] = y.y;
        }
        #pragma unroll
        for (int i = 0; i < G::kWordsK; ++i) {
            #pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint32_t u = wa[i] >> (8 * s), v = wb[i] >> (8 * s);
                const uint32_t a0 = sub_f16x2(low_codes(u), za), a1 = sub_f16x2(low_codes(v), zb);
                const uint32_t a2 = less_16_times(high_codes(u), za), a3 = less_16_times(high_codes(v), zb);
                #pragma unroll
                for (int n = 0; n < NG; ++n) mma_f16(d[j][n], a0, a1, a2, a3, w.q[2 * i + s][n][0], w.q[2 * i + s][n][1]);
            }
        }
        if constexpr (D == 80) {
            const uint32_t tail = stage + kl - c * (4 * G::kWordsK) + j * 16 * G::kRowBytes + 32;
            const uint2 x = lds64(tail), y = lds64(tail + 8 * G::kRowBytes);
            const uint32_t a0 = sub_f16x2(low_codes(x.x >> (4 * c)), za), a1 = sub_f16x2(low_codes(y.x >> (4 * c)), zb);
            const uint32_t a2 = sub_f16x2(low_codes(x.y >> (4 * c)), za), a3 = sub_f16x2(low_codes(y.y >> (4 * c)), zb);
            #pragma unroll
            for (int n = 0; n < NG; ++n) mma_f16(d[j][n], a0, a1, a2, a3, w.q[4][n][0], w.q[4][n][1]);
        }
    }
    #pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float sa = scale_of(pa[j]), sb = scale_of(pb[j]);
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            #pragma unroll
            for (int i = 0; i < 4; ++i) {
                d[j][n][i] = fmaf(d[j][n][i] * (i < 2 ? sa : sb), w.factor[n][i & 1], -w.ref[n][i & 1]);
            }
        }
        pa[j] = lds32(stage + pl + kWordsOfV + 64 * j), pb[j] = lds32(stage + pl + kWordsOfV + 64 * j + 32);
    }
    if (valid < kChunk) {
        #pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = 16 * j + key_of(g);
            #pragma unroll
            for (int n = 0; n < NG; ++n) {
                #pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (key + (i < 2 ? 0 : 8) >= valid) d[j][n][i] = -INFINITY;
            }
        }
    }
    keep_in_range<D, NG, 2>(w, d, fmaxf(fmaxf(scale_of(pa[0]), scale_of(pb[0])), fmaxf(scale_of(pa[1]), scale_of(pb[1]))), false);
    #pragma unroll
    for (int j = 0; j < 2; ++j) {
        uint32_t p[NG][2];
        const float sa = scale_of(pa[j]) * w.weight, sb = scale_of(pb[j]) * w.weight;
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            const float x0 = exp2_approx(d[j][n][0]), x1 = exp2_approx(d[j][n][1]), x2 = exp2_approx(d[j][n][2]), x3 = exp2_approx(d[j][n][3]);
            w.sum[n][0] += x0 + x2;
            w.sum[n][1] += x1 + x3;
            p[n][0] = transpose_8x8(pack2_f16(x0 * sa, x1 * sa));
            p[n][1] = transpose_8x8(pack2_f16(x2 * sb, x3 * sb));
        }
        // O^T += V^T P^T
        const uint32_t pz = stage + zl + 64 * j;
        const uint32_t z01 = zero_pair(lds32(pz), lds32(pz + 16)), z23 = zero_pair(lds32(pz + 32), lds32(pz + 48));
        #pragma unroll
        for (int n = 0; n < NG; ++n) mma_f16(w.zo[n], z01, z01, z23, z23, p[n][0], p[n][1]);
        const uint32_t row = stage + vl + j * 16 * G::kRowBytes;
        uint32_t v[4][2];
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (G::kWordsV == 2) {
                const uint2 x = lds64(row + 4 * k * G::kRowBytes);
                v[k][0] = x.x, v[k][1] = x.y;
            } else {
                v[k][0] = lds32(row + 4 * k * G::kRowBytes);
            }
        }
        #pragma unroll
        for (int i = 0; i < G::kWordsV; ++i) {
            const uint32_t l01 = __byte_perm(v[0][i], v[1][i], 0x5410), h01 = __byte_perm(v[0][i], v[1][i], 0x7632);
            const uint32_t l23 = __byte_perm(v[2][i], v[3][i], 0x5410), h23 = __byte_perm(v[2][i], v[3][i], 0x7632);
            #pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int sh = 8 * (s >> 1);
                const auto codes = [&](uint32_t x) { return s & 1 ? high_codes(x >> sh) : low_codes(x >> sh); };
                const uint32_t a0 = codes(l01), a1 = codes(h01), a2 = codes(l23), a3 = codes(h23);
                #pragma unroll
                for (int n = 0; n < NG; ++n) mma_f16(w.o[4 * i + s][n], a0, a1, a2, a3, p[n][0], p[n][1]);
            }
        }
        if constexpr (D == 80) {
            // the last 16 dimensions: rows g and g + 8 of the tile are dimensions 64 + g and 72 + g
            const int sh = 4 * (g >> 1) + 16 * (g & 1);
            uint2 x[4];
            #pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = lds64(row - g * (4 * G::kWordsV) + 32 + 4 * k * G::kRowBytes);
            const uint32_t a0 = low_codes((x[0].x >> sh & 0xfu) | (x[1].x >> sh) << 16), a1 = low_codes((x[0].y >> sh & 0xfu) | (x[1].y >> sh) << 16);
            const uint32_t a2 = low_codes((x[2].x >> sh & 0xfu) | (x[3].x >> sh) << 16), a3 = low_codes((x[2].y >> sh & 0xfu) | (x[3].y >> sh) << 16);
            #pragma unroll
            for (int n = 0; n < NG; ++n) mma_f16(w.o[4][n], a0, a1, a2, a3, p[n][0], p[n][1]);
        }
    }
}

// The keys behind the prefix of a block: nodes 0 .. T - 1, then the streams of nodes t0 ..
struct Extra {
    int T, gamma, t0, count;                         // count: nodes and stream keys
    int row0, rows;                                  // of the block; rows of the sequence
};

// Row r of a head's query rows, or null behind the last one
template <int D>
__device__ __forceinline__ const __nv_bfloat16* query_row(const KvqArgs& a, int T, int rows, int b, int h, int r) {
    if (r >= rows || h >= a.n_heads) return nullptr;
    return (r < T ? a.q_main : a.q_spec) + row_offset(a, D, b, h, r, T);
}

// Where key e lies in k_tree / v_tree or k_spec / v_spec (elements)
__device__ __forceinline__ long long extra_offset(const KvqArgs& a, const Extra& x, int D, int b, int h, int e) {
    return row_offset(a, D, b, h, e < x.T ? e : e + x.t0 * x.gamma, x.T);
}

// Scores above their references of 16 keys behind the prefix, from `first` on; what a row does not see is -inf
template <int D, int NG>
__device__ __forceinline__ void extra_scores(const WarpState<D, NG>& w, float (&acc)[NG][4], const KvqArgs& a, const Extra& x, int b, int h, int first, int g, int c) {
    using G = KvqGeometry<D>;
    const int ea = first + key_of(g), eb = ea + 8;
    const __nv_bfloat16* ka = (ea < x.T ? a.k_tree : a.k_spec) + (ea < x.count ? extra_offset(a, x, D, b, h, ea) : 0);
    const __nv_bfloat16* kb = (eb < x.T ? a.k_tree : a.k_spec) + (eb < x.count ? extra_offset(a, x, D, b, h, eb) : 0);
    const __nv_bfloat16* q[NG];                      // the rows of B: row g of every group
    #pragma unroll
    for (int n = 0; n < NG; ++n) q[n] = query_row<D>(a, x.T, x.rows, b, h, x.row0 + 8 * n + g);
    #pragma unroll
    for (int n = 0; n < NG; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
    #pragma unroll
    for (int i = 0; i < G::kWordsK; ++i) {
        uint4 u = {}, v = {};
        if (ea < x.count) u = *reinterpret_cast<const uint4*>(ka + c * (8 * G::kWordsK) + 8 * i);
        if (eb < x.count) v = *reinterpret_cast<const uint4*>(kb + c * (8 * G::kWordsK) + 8 * i);
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            uint4 r = {};
            if (q[n]) r = *reinterpret_cast<const uint4*>(q[n] + c * (8 * G::kWordsK) + 8 * i);
            mma_bf16(acc[n], u.x, v.x, u.y, v.y, r.x, r.y);
            mma_bf16(acc[n], u.z, v.z, u.w, v.w, r.z, r.w);
        }
    }
    if constexpr (D == 80) {
        uint32_t u[4] = {};
        if (ea < x.count) u[0] = *reinterpret_cast<const uint32_t*>(ka + 64 + 2 * c), u[2] = *reinterpret_cast<const uint32_t*>(ka + 72 + 2 * c);
        if (eb < x.count) u[1] = *reinterpret_cast<const uint32_t*>(kb + 64 + 2 * c), u[3] = *reinterpret_cast<const uint32_t*>(kb + 72 + 2 * c);
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            uint32_t r0 = 0u, r1 = 0u;
            if (q[n]) r0 = *reinterpret_cast<const uint32_t*>(q[n] + 64 + 2 * c), r1 = *reinterpret_cast<const uint32_t*>(q[n] + 72 + 2 * c);
            mma_bf16(acc[n], u[0], u[1], u[2], u[3], r0, r1);
        }
    }
    #pragma unroll
    for (int n = 0; n < NG; ++n) {
        #pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = x.row0 + 8 * n + 2 * c + e;
            unsigned long long see = 0;
            int lo = 0, hi = 0;                      // stream keys the row sees
            if (r < x.rows) {
                const Row q = row_of(r, x.T, x.gamma);
                see = a.trees[b].anc_mask[q.t];
                lo = x.T + (q.t - x.t0) * x.gamma;
                hi = q.j < 0 ? lo : lo + q.j + 1;
            }
            const bool sa = ea < x.T ? (see >> ea & 1ull) : (ea >= lo && ea < hi);
            const bool sb = eb < x.T ? (see >> eb & 1ull) : (eb >= lo && eb < hi);
            acc[n][e] = sa ? fmaf(acc[n][e], a.scale, -w.ref[n][e]) : -INFINITY;
            acc[n][2 + e] = sb ? fmaf(acc[n][2 + e], a.scale, -w.ref[n][e]) : -INFINITY;
        }
    }
}

// O^T += V^T P^T of 16 keys behind the prefix
template <int D, int NG>
__device__ __forceinline__ void extra_values(WarpState<D, NG>& w, const uint32_t (&p)[NG][2], const KvqArgs& a, const Extra& x, int b, int h, int first, int g, int c) {
    using G = KvqGeometry<D>;
    const __nv_bfloat16* vk[4];
    bool there[4];
    #pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int e = first + c + 4 * k;
        there[k] = e < x.count;
        vk[k] = (e < x.T ? a.v_tree : a.v_spec) + (there[k] ? extra_offset(a, x, D, b, h, e) : 0);
    }
    #pragma unroll
    for (int i = 0; i < G::kWordsV; ++i) {
        uint4 v[4] = {};
        #pragma unroll
        for (int k = 0; k < 4; ++k)
            if (there[k]) v[k] = *reinterpret_cast<const uint4*>(vk[k] + g * (8 * G::kWordsV) + 8 * i);
        const uint32_t v0[4] = {v[0].x, v[0].y, v[0].z, v[0].w}, v1[4] = {v[1].x, v[1].y, v[1].z, v[1].w};
        const uint32_t v2[4] = {v[2].x, v[2].y, v[2].z, v[2].w}, v3[4] = {v[3].x, v[3].y, v[3].z, v[3].w};
        #pragma unroll
        for (int s = 0; s < 4; ++s) {
            uint32_t a0 = __byte_perm(v0[s], v1[s], 0x5410), a1 = __byte_perm(v0[s], v1[s], 0x7632);
            uint32_t a2 = __byte_perm(v2[s], v3[s], 0x5410), a3 = __byte_perm(v2[s], v3[s], 0x7632);
            if (s & 1) a0 = times16_bf16x2(a0), a1 = times16_bf16x2(a1), a2 = times16_bf16x2(a2), a3 = times16_bf16x2(a3);
            #pragma unroll
            for (int n = 0; n < NG; ++n) mma_bf16(w.o[4 * i + s][n], a0, a1, a2, a3, p[n][0], p[n][1]);
        }
    }
    if constexpr (D == 80) {
        uint32_t lo[4] = {}, hi[4] = {};
        #pragma unroll
        for (int k = 0; k < 4; ++k)
            if (there[k]) {
                lo[k] = reinterpret_cast<const unsigned short*>(vk[k])[64 + g];
                hi[k] = reinterpret_cast<const unsigned short*>(vk[k])[72 + g];
            }
        #pragma unroll
        for (int n = 0; n < NG; ++n)
            mma_bf16(w.o[4][n], lo[0] | lo[1] << 16, hi[0] | hi[1] << 16, lo[2] | lo[3] << 16, hi[2] | hi[3] << 16, p[n][0], p[n][1]);
    }
}

// Asynchronous copies of chunks' codes, scales and zero points into the stages of a warp's ring.  A lane copies the same column of
// every (32 / lanes per row)-th row, from pointers that walk along with the warp's chunks; slots behind the last one are read as the
// last one again (their weights are zero).
template <int D>
struct ChunkLoader {
    using G = KvqGeometry<D>;
    static constexpr int kPer = G::kRowBytes / G::kCopy;         // copies per row and per lane: 4, 5 or 2
    static constexpr bool kEven = 32 % kPer == 0;
    const unsigned char *k, *v;                                  // of the next chunk: the lane's first copy (80: key 0)
    const uint32_t *kp, *vp;                                     // the lane's key
    long long on, pon, row;                                      // bytes and words to the warp's next chunk; bytes to the lane's next row
    int left, step;                                              // slots from the next chunk on; slots between this warp's chunks

    __device__ __forceinline__ ChunkLoader(const KvqArgs& a, const Seq& s, int h, int chunk, int stride, int lane) {
        const long long slot = s.start + static_cast<long long>(chunk) * kChunk;
        const long long off = (slot + (kEven ? lane / kPer : 0)) * a.slot_stride + h * a.head_stride + (kEven ? lane % kPer * G::kCopy : 0);
        const long long poff = (slot + lane) * a.p_slot + h * a.p_head;
        k = a.k_codes + off, v = a.v_codes + off;
        kp = a.k_params + poff, vp = a.v_params + poff;
        left = s.L - chunk * kChunk;
        step = stride * kChunk;
        on = step * a.slot_stride, pon = step * a.p_slot, row = (32 / kPer) * a.slot_stride;
    }
    // the next chunk of this warp, if it is among the cached ones
    __device__ __forceinline__ void next(const KvqArgs& a, uint32_t stage, int lane, bool wanted) {
        if (wanted) {
            const uint32_t dst = stage + lane * G::kCopy, pdst = stage + 2 * G::kCodeBytes + 4 * lane;
            if (kEven && left >= kChunk) {
                #pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    copy_async<G::kCopy>(dst + i * 32 * G::kCopy, k + i * row);
                    copy_async<G::kCopy>(dst + i * 32 * G::kCopy + G::kCodeBytes, v + i * row);
                }
                copy_async<4>(pdst, kp);
                copy_async<4>(pdst + 4 * kChunk, vp);
            } else {
                const int last = left - 1;
                #pragma unroll 1
                for (int i = 0; i < kPer; ++i) {
                    const int item = i * 32 + lane, key = item / kPer;
                    const long long off = kEven ? (min(key, last) - lane / kPer) * a.slot_stride : min(key, last) * a.slot_stride + (item - key * kPer) * G::kCopy;
                    copy_async<G::kCopy>(dst + i * 32 * G::kCopy, k + off);
                    copy_async<G::kCopy>(dst + i * 32 * G::kCopy + G::kCodeBytes, v + off);
                }
                const long long poff = (min(lane, last) - lane) * a.p_slot;
                copy_async<4>(pdst, kp + poff);
                copy_async<4>(pdst + 4 * kChunk, vp + poff);
            }
            k += on, v += on, kp += pon, vp += pon;
            left -= step;
        }
        copy_commit();
    }
};

// Dimensions that lane (g, c) holds in tile k of O^T: rows g (returned) and g + 8 (the next dimension; 8 further in the last tile of 80)
template <int D>
__device__ __forceinline__ int tile_dim(int k, int g) {
    using G = KvqGeometry<D>;
    return k < 4 * G::kWordsV ? g * (8 * G::kWordsV) + 2 * k : G::kMain + g;
}

template <int D, int NG>
__global__ void __launch_bounds__(kThreads, NG == 1 ? 3 : 2) msa_attention_kvq_rows_kernel(const __grid_constant__ KvqArgs a) {
    using G = KvqGeometry<D>;
    using S = KvqSmem<D, NG>;
    constexpr int ROWS = 8 * NG, PAD = S::kPad;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int joined;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const uint32_t ring = smem_addr(smem) + warp * G::kRingBytes;
    float* const parts = reinterpret_cast<float*>(smem);                                      // [warp][row][PAD], in the rings' place
    float2* const stats = reinterpret_cast<float2*>(smem + S::kBytes - kWarps * ROWS * 8);   // [warp][row]: reference, sum
    const uint32_t kl = key_of(g) * G::kRowBytes + c * (4 * G::kWordsK), vl = G::kCodeBytes + c * G::kRowBytes + g * (4 * G::kWordsV);
    const uint32_t pl = 2 * G::kCodeBytes + 4 * key_of(g), zl = 2 * G::kCodeBytes + 4 * kChunk + 4 * c;
    wait_for_previous_kernel();
    release_next_kernel();

    Line<ROWS, kChunk, kWarpsLog2, 0> line;
    if (!line.begin(a, lane)) return;
    const int HW = 1 << line.heads_log2, KS = 1 << line.steps_log2;
    int* const counters = reinterpret_cast<int*>(a.ws + kWsHeaderBytes);
    float* const partial = reinterpret_cast<float*>(a.ws + kWsHeaderBytes + kCounterBytes);
    const int my_head = warp & (HW - 1), slice = warp >> line.heads_log2;

    while (line.next(a)) {
        const Seq& s = line.s;
        const int b = line.b, from = line.from, to = line.to, row0 = line.row0, h0 = line.head0, h = h0 + my_head;
        const int P = prefix_chunks<kChunk>(s.L), stop = h < a.n_heads ? min(to * KS, s.chunks) : 0;       // (a warp without a head has no chunks)

        WarpState<D, NG> w;
        #pragma unroll
        for (int k = 0; k < G::kTiles; ++k) {
            #pragma unroll
            for (int n = 0; n < NG; ++n) {
                #pragma unroll
                for (int i = 0; i < 4; ++i) w.o[k][n][i] = 0.f;
            }
        }
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            w.ref[n][0] = w.ref[n][1] = 0.f;
            w.sum[n][0] = w.sum[n][1] = 0.f;
            w.zo[n][0] = w.zo[n][1] = w.zo[n][2] = w.zo[n][3] = 0.f;
        }
        w.weight = 64.f, w.limit = 0.f;
        const int held = min(stop, P);               // chunks of cached slots end here
        ChunkLoader<D> loader(a, s, min(h, a.n_heads - 1), from * KS + slice, KS, lane);
        int fetch = from * KS + slice;
        #pragma unroll 1
        for (int i = 0; i < G::kStages - 1; ++i, fetch += KS) loader.next(a, ring + i * G::kStageBytes, lane, fetch < held);
        // query rows: row g of every group, the dimensions that c holds
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            const __nv_bfloat16* q = query_row<D>(a, s.T, s.rows, b, h, row0 + 8 * n + g);
            uint32_t v[D / 16][2] = {};
            if (q) {
                #pragma unroll
                for (int i = 0; i < G::kWordsK; ++i) {
                    const uint4 u = *reinterpret_cast<const uint4*>(q + c * (8 * G::kWordsK) + 8 * i);
                    v[2 * i][0] = u.x, v[2 * i][1] = u.y, v[2 * i + 1][0] = u.z, v[2 * i + 1][1] = u.w;
                }
                if constexpr (D == 80) v[4][0] = *reinterpret_cast<const uint32_t*>(q + 64 + 2 * c), v[4][1] = *reinterpret_cast<const uint32_t*>(q + 72 + 2 * c);
            }
            uint32_t top = 0u;                       // two largest magnitudes (as patterns of bf16 they are in order)
            #pragma unroll
            for (int i = 0; i < D / 16; ++i) top = __vmaxu2(top, __vmaxu2(v[i][0] & 0x7fff7fffu, v[i][1] & 0x7fff7fffu));
            top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // 2^e with the largest |q| 2^-e in [2^14, 2^15), kept where 2^e and 2^-e are normal numbers
            const uint32_t eb = min(max(max(top & 0xffffu, top >> 16) >> 7, 24u), 247u) - 14u;
            const float up = __uint_as_float(eb << 23), down = __uint_as_float((254u - eb) << 23);
            #pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                #pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float x = __uint_as_float(v[i][k] << 16) * down, y = __uint_as_float(v[i][k] & 0xffff0000u) * down;
                    const float f = k && i < 2 * G::kWordsK ? 0.0625f : 1.f;         // (these meet high codes)
                    w.q[i][n][k] = pack2_f16(x * f, y * f);
                }
            }
            // a row's factor goes to the lanes that hold its scores: rows 2c and 2c + 1 of the group
            #pragma unroll
            for (int e = 0; e < 2; ++e) w.factor[n][e] = __shfl_sync(0xffffffffu, up, 4 * (2 * c + e)) * (a.scale * (1.f / kCode));
        }
        uint32_t stage = ring;
        int k = from * KS + slice;
        #pragma unroll 1
        for (; k < held; k += KS) {
            copy_wait<G::kStages - 2>();
            __syncwarp();
            loader.next(a, stage == ring ? stage + (G::kStages - 1) * G::kStageBytes : stage - G::kStageBytes, lane, fetch < held);
            fetch += KS;
            prefix_chunk<D, NG>(w, stage, s.L - k * kChunk, kl, vl, pl, zl, g, c);
            stage = stage == ring + (G::kStages - 1) * G::kStageBytes ? ring : stage + G::kStageBytes;
        }
        if (k < stop) {
            Extra x;
            x.T = s.T, x.gamma = max(a.gamma, 1), x.row0 = row0, x.rows = s.rows, x.t0 = 0, x.count = s.T;
            const int last = min(row0 + ROWS, s.rows) - 1;
            if (last >= s.T) {                       // the block has stream rows: the streams of their nodes
                x.t0 = row0 < s.T ? 0 : (row0 - s.T) / a.gamma;
                x.count = s.T + ((last - s.T) / a.gamma - x.t0 + 1) * a.gamma;
            }
            if (w.weight > 64.f) raise_scale<D, NG>(w, 1.f);             // (V in bf16 may be large: r is at least 0)
            #pragma unroll 1
            for (; k < stop; k += KS) {
                #pragma unroll 1
                for (int j = 0; j < kChunk; j += 16) {
                    const int first = (k - P) * kChunk + j;
                    if (first >= x.count) break;
                    float d[1][NG][4];
                    uint32_t p[NG][2];
                    extra_scores<D, NG>(w, d[0], a, x, b, h, first, g, c);
                    keep_in_range<D, NG, 1>(w, d, -1.f, true);
                    const float f = w.weight * kCode;                    // (a weight meets values here, not codes)
                    #pragma unroll
                    for (int n = 0; n < NG; ++n) {
                        const float x0 = exp2_approx(d[0][n][0]), x1 = exp2_approx(d[0][n][1]), x2 = exp2_approx(d[0][n][2]), x3 = exp2_approx(d[0][n][3]);
                        w.sum[n][0] += x0 + x2;
                        w.sum[n][1] += x1 + x3;
                        p[n][0] = transpose_8x8(pack2_bf16(x0 * f, x1 * f));
                        p[n][1] = transpose_8x8(pack2_bf16(x2 * f, x3 * f));
                    }
                    extra_values<D, NG>(w, p, a, x, b, h, first, g, c);
                }
            }
        }
        copy_wait<0>();
        __syncthreads();                             // all rings are at rest: their place is taken by the warps' partial results

        // the warps' references and sums, then their rows
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            #pragma unroll
            for (int e = 0; e < 2; ++e) {
                #pragma unroll
                for (int x = 4; x < 32; x <<= 1) w.sum[n][e] += __shfl_xor_sync(0xffffffffu, w.sum[n][e], x);
                if (g == 0) stats[warp * ROWS + 8 * n + 2 * c + e] = make_float2(w.sum[n][e] == 0.f ? kNoRef : w.ref[n][e], w.sum[n][e]);
            }
        }
        const float unweigh = __uint_as_float((254u << 23) - __float_as_uint(w.weight));     // (a power of two; 2^24 apart from it, or it may pass fp32)
        #pragma unroll
        for (int k = 0; k < G::kTiles; ++k) {
            const int dim = tile_dim<D>(k, g);
            const float f = k < 4 * G::kWordsV && (k & 1) ? 0.0625f : 1.f;
            #pragma unroll
            for (int n = 0; n < NG; ++n) {
                #pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float* dst = parts + (warp * ROWS + 8 * n + 2 * c + e) * PAD + dim;
                    const float x = fmaf(w.o[k][n][e], f, -w.zo[n][e]) * (1.f / kCode) * unweigh, y = fmaf(w.o[k][n][2 + e], f, -w.zo[n][e]) * (1.f / kCode) * unweigh;
                    if (k < 4 * G::kWordsV) *reinterpret_cast<float2*>(dst) = make_float2(x, y);
                    else dst[0] = x, dst[8] = y;
                }
            }
        }
        __syncthreads();

        // whole unit: output.  A piece of one: partial rows to the workspace; the last CTA of the unit joins them.
        const bool whole = line.whole();
        const Pieces share(line);
        const auto place = [&](int i) { return partial + share.place(line, i) * partial_floats(D, ROWS); };
        const int rows = min(ROWS, s.rows - row0), items = max(0, min(HW, a.n_heads - h0)) * rows * (D / 8);
        #pragma unroll 1
        for (int item = tid; item < items; item += kThreads) {
            const int hr = item / (D / 8), d0 = (item - hr * (D / 8)) * 8, hd = hr / rows, r = hr - hd * rows;
            float m = kNoRef, l = 0.f, o[8] = {};
            #pragma unroll 1
            for (int i = hd; i < kWarps; i += HW) {
                const float* src = parts + (i * ROWS + r) * PAD + d0;
                join_row(o, m, l, stats[i * ROWS + r], *reinterpret_cast<const float4*>(src), *reinterpret_cast<const float4*>(src + 4));
            }
            if (whole) {
                store_row<D>(a, row0 + r < s.T, row_offset(a, D, b, h0 + hd, row0 + r, s.T), d0, o, m, l);
            } else {
                float* dst = place(line.me) + hr * (D + 4) + d0;
                __stcg(reinterpret_cast<float4*>(dst), make_float4(o[0], o[1], o[2], o[3]));
                __stcg(reinterpret_cast<float4*>(dst) + 1, make_float4(o[4], o[5], o[6], o[7]));
                if (d0 == 0) __stcg(reinterpret_cast<float2*>(dst + D), make_float2(m, l));
            }
        }
        if (!whole) {
            __syncthreads();
            if (tid == 0) {
                joined = last_piece(counters + (share.first << line.team_log2) + line.member, share.last - share.first + 1);
            }
            __syncthreads();
            if (joined) {
                constexpr int kJoinAhead = 6;        // partial rows that a thread has on their way (12 pieces of 8 rows: 13.4 us, 8 14.0, 4 13.2; 37 of one: 14.6, 14.1, 15.4)
                #pragma unroll 1
                for (int item = tid; item < items; item += kThreads) {
                    const int hr = item / (D / 8), d0 = (item - hr * (D / 8)) * 8, hd = hr / rows, r = hr - hd * rows;
                    float m = kNoRef, l = 0.f, o[8] = {};
                    #pragma unroll 1
                    for (int i = share.first; i <= share.last; i += kJoinAhead) {
                        float2 st[kJoinAhead];
                        float4 u[kJoinAhead], v[kJoinAhead];
                        #pragma unroll
                        for (int k = 0; k < kJoinAhead; ++k) {
                            const float* src = place(min(i + k, share.last)) + hr * (D + 4);
                            st[k] = __ldcg(reinterpret_cast<const float2*>(src + D));
                            u[k] = __ldcg(reinterpret_cast<const float4*>(src + d0)), v[k] = __ldcg(reinterpret_cast<const float4*>(src + d0) + 1);
                        }
                        #pragma unroll
                        for (int k = 0; k < kJoinAhead; ++k)
                            if (i + k <= share.last) join_row(o, m, l, st[k], u[k], v[k]);
                    }
                    store_row<D>(a, row0 + r < s.T, row_offset(a, D, b, h0 + hd, row0 + r, s.T), d0, o, m, l);
                }
            }
        }
        __syncthreads();                             // the partial results' place goes back to the rings
    }
}

}  // namespace ss

#include "ss_kvq_tiles.cuh"

namespace ss {

// ---- host ---------------------------------------------------------------------------------------
static int q_rows(const ss_kvq_attn_params& p) { return p.max_nodes * (1 + p.gamma); }

// Which kernel takes a call: `tile` > 0: blocks of so many rows on tcgen05, else groups of 8 rows on register-level MMAs
struct KvqPlan {
    int tile, groups, block, ctas;
};
static KvqPlan kvq_plan(const ss_kvq_attn_params& p) {
    const int rows = q_rows(p);
    // Up to 8 rows the rows are one group: three CTAs per SM, and nothing is spent on the second group's padding (16 users with 512 to 4096
    // keys, a row each: 43 us, with two groups 52; 32 heads of 50,000 keys, 8 rows: 57 and 65; 512 keys 9.8 and 10.0; 2048 keys 13.4 and
    // 11.6, the other way round for want of fewer pieces, see most_pieces).  From 17 rows on tcgen05 is faster at all lengths (32 rows: 16 users
    // 84 us, by two groups of 16 rows 124; 50,000 keys 103 and 126; 512 keys 12.1 and 14.8); up to 16 it is slower where it counts (12 rows: 16
    // users 83 and 63 us; 50,000 keys 101 and 68; 512 keys 11.5 and 11.9: only the device knows the lengths).  32 rows in the kernel for 64
    // cost a sixth (100 us).
    KvqPlan k{0, rows <= 8 ? 1 : 2, 0, 0};
    if (rows > 16) k.tile = rows <= 32 ? 32 : 64;
    k.block = k.tile > 0 ? k.tile : 8 * k.groups;
    k.ctas = std::min(sm_count() * (k.tile > 0 ? 1 : k.groups == 1 ? 3 : 2), kCounterBytes / 4);
    return k;
}

static size_t kvq_workspace(const ss_kvq_attn_params& p) {
    const KvqPlan k = kvq_plan(p);
    const size_t ctas = static_cast<size_t>(k.ctas), d = static_cast<size_t>(p.cache.head_dim);
    const size_t floats = k.tile > 0 ? k.tile * (d + 4) : static_cast<size_t>(partial_floats(p.cache.head_dim, k.block));
    return kWsHeaderBytes + kCounterBytes + 2 * ctas * floats * sizeof(float);
}

template <typename Kernel>
static int32_t launch_kvq_kernel(Kernel kernel, int bytes, int threads, const KvqArgs& args, int ctas, cudaStream_t stream) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return SS_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(ctas));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = static_cast<size_t>(bytes);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args) == cudaSuccess ? SS_OK : SS_ERR_CUDA;
}

template <int D>
static int32_t launch_kvq(const KvqPlan& k, const KvqArgs& args, int ctas, cudaStream_t stream) {
    if (k.tile == 32) return launch_kvq_kernel(msa_attention_kvq_tiles_kernel<D, 32>, TileGeo<D, 32>::kBytes, kTileThreads, args, ctas, stream);
    if (k.tile == 64) return launch_kvq_kernel(msa_attention_kvq_tiles_kernel<D, 64>, TileGeo<D, 64>::kBytes, kTileThreads, args, ctas, stream);
    return k.groups == 1 ? launch_kvq_kernel(msa_attention_kvq_rows_kernel<D, 1>, KvqSmem<D, 1>::kBytes, kThreads, args, ctas, stream)
                         : launch_kvq_kernel(msa_attention_kvq_rows_kernel<D, 2>, KvqSmem<D, 2>::kBytes, kThreads, args, ctas, stream);
}

static int32_t kvq_check_shapes(const ss_kvq_attn_params* p) {
    if (!p) return SS_ERR_INVALID_ARG;
    const ss_kvq_cache& c = p->cache;
    if (p->batch < 1 || p->batch > 65535 || c.n_heads < 1 || p->max_nodes < 1 || p->gamma < 0) return SS_ERR_INVALID_ARG;
    if (c.head_dim != 64 && c.head_dim != 80 && c.head_dim != 128) return SS_ERR_UNSUPPORTED;
    if (p->max_nodes > SS_MAX_NODES || p->gamma > SS_MAX_GAMMA) return SS_ERR_UNSUPPORTED;
    return SS_OK;
}

}  // namespace ss

extern "C" size_t ss_msa_attention_kvq_workspace_bytes(const ss_kvq_attn_params* p) {
    return ss::kvq_check_shapes(p) == SS_OK ? ss::kvq_workspace(*p) : 0;
}

extern "C" int32_t ss_msa_attention_kvq(const ss_kvq_attn_params* p, void* stream) {
    using namespace ss;
    int32_t st = kvq_check_shapes(p);
    if (st != SS_OK) return st;
    const ss_kvq_cache& c = p->cache;
    st = kvq_check_cache(c);
    if (st != SS_OK) return st;
    if (p->layer < 0 || p->layer >= c.n_layers) return SS_ERR_INVALID_ARG;
    if (!p->q_main || !p->o_main || !p->k_tree || !p->v_tree || !p->kv_start || !p->kv_len || !p->trees || !p->workspace) return SS_ERR_INVALID_ARG;
    if (p->gamma > 0 && (!p->q_spec || !p->k_spec || !p->v_spec || !p->o_spec)) return SS_ERR_INVALID_ARG;
    for (const void* q : {p->q_main, static_cast<const void*>(p->o_main), p->k_tree, p->v_tree, static_cast<const void*>(p->workspace)})
        if (!aligned16(q)) return SS_ERR_INVALID_ARG;
    if (p->gamma > 0)
        for (const void* q : {p->q_spec, p->k_spec, p->v_spec, static_cast<const void*>(p->o_spec)})
            if (!aligned16(q)) return SS_ERR_INVALID_ARG;
    if (!(p->sm_scale == p->sm_scale) || p->sm_scale - p->sm_scale != 0.f) return SS_ERR_INVALID_ARG;
    if (p->workspace_bytes < kvq_workspace(*p)) return SS_ERR_WORKSPACE;
    const long long layer = p->layer;
    KvqArgs a;
    a.k_codes = static_cast<const unsigned char*>(c.k_codes) + layer * c.layer_stride;
    a.v_codes = static_cast<const unsigned char*>(c.v_codes) + layer * c.layer_stride;
    a.k_params = c.k_params + layer * c.param_layer_stride;
    a.v_params = c.v_params + layer * c.param_layer_stride;
    a.slot_stride = c.slot_stride, a.head_stride = c.head_stride, a.p_slot = c.param_slot_stride, a.p_head = c.param_head_stride;
    a.total_slots = c.total_slots;
    const auto bf = [](const void* x) { return static_cast<const __nv_bfloat16*>(x); };
    a.q_main = bf(p->q_main), a.q_spec = bf(p->q_spec), a.k_tree = bf(p->k_tree), a.v_tree = bf(p->v_tree);
    a.k_spec = bf(p->k_spec), a.v_spec = bf(p->v_spec);
    a.o_main = static_cast<__nv_bfloat16*>(p->o_main), a.o_spec = static_cast<__nv_bfloat16*>(p->o_spec);
    a.lse_main = p->lse_main, a.lse_spec = p->lse_spec;
    a.kv_start = p->kv_start, a.kv_len = p->kv_len, a.kv_capacity = p->kv_capacity, a.trees = p->trees;
    a.ws = static_cast<unsigned char*>(p->workspace);
    a.scale = p->sm_scale * 1.4426950408889634f;
    a.batch = p->batch, a.n_heads = c.n_heads, a.gamma = p->gamma, a.max_nodes = p->max_nodes;
    // no more CTAs than the slab can give steps for
    const KvqPlan k = kvq_plan(*p);
    const int blocks = (q_rows(*p) + k.block - 1) / k.block, chunk = k.tile > 0 ? kTileOfKeys : kChunk;
    const int extra = k.tile > 0 ? extra_chunks<kTileOfKeys>(p->max_nodes, p->gamma, k.block) : extra_chunks<kChunk>(p->max_nodes, p->gamma, k.block);
    const long long chunks = static_cast<long long>(c.n_heads) * blocks * ((c.total_slots + chunk - 1) / chunk + p->batch * (1ll + extra));
    const int ctas = static_cast<int>(std::min<long long>(k.ctas, chunks));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return c.head_dim == 128 ? launch_kvq<128>(k, a, ctas, s) : c.head_dim == 80 ? launch_kvq<80>(k, a, ctas, s) : launch_kvq<64>(k, a, ctas, s);
}
