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
// A unit is a block of query rows of one head of one sequence; its keys are cut in chunks of 32: the cached slots, then the tree's
// nodes and the stream keys of the block's own nodes.  All units' chunks, in order of sequence, head and block, are one line that
// is cut into equal pieces, one per CTA: a CTA takes the end of a unit, whole units, and the beginning of another.  So every CTA
// reads the same amount, whatever the lengths (which only the device knows).
constexpr int kChunk = 32;

struct Seq {
    int L, T, rows, blocks, chunks;                  // chunks of one unit: cached ones and those behind
    long long start;
};

__device__ __forceinline__ int prefix_chunks(int L) { return (L + kChunk - 1) / kChunk; }

// Most keys behind the prefix that a block of `block` rows sees: all nodes, and the streams of the nodes its rows belong to
__host__ __device__ __forceinline__ int extra_chunks(int T, int gamma, int block) {
    int stream = 0;
    if (gamma > 0) {
        const int nodes = (block + gamma - 2) / gamma + 1;
        stream = (nodes < T ? nodes : T) * gamma;
    }
    return (T + stream + kChunk - 1) / kChunk;
}

// One sequence as the call gives it.  A sequence that cannot be run has no units.
template <int ROWS>
__device__ __forceinline__ Seq load_seq(const KvqArgs& a, int b) {
    Seq s;
    s.L = a.kv_len[b];
    s.start = a.kv_start[b];
    s.T = min(a.trees[b].n_nodes, a.max_nodes);
    const bool fits = s.L >= 0 && s.start >= 0 && s.start + s.L <= a.total_slots && (a.kv_capacity == nullptr || s.L <= a.kv_capacity[b]);
    if (!fits) set_status(a.ws, SS_ERR_CAPACITY);
    if (!fits || s.T < 1) s.T = s.rows = s.blocks = s.chunks = 0;
    else {
        s.rows = s.T * (1 + a.gamma);
        s.blocks = (s.rows + ROWS - 1) / ROWS;
        s.chunks = prefix_chunks(s.L) + extra_chunks(s.T, a.gamma, ROWS);
    }
    return s;
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

// Element offset of a row's vector in a main-stream or stream tensor
__device__ __forceinline__ long long row_offset(const KvqArgs& a, int hd, int b, int h, const Row& r) {
    const long long node = static_cast<long long>(b) * a.max_nodes + r.t;
    return ((r.j < 0 ? node : node * a.gamma + r.j) * a.n_heads + h) * hd;
}

// ---- small helpers ------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool real) {
    const int n = real ? BYTES : 0;                  // (nothing is read where n is 0: the destination is filled with zeros)
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(n) : "memory");
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

// Codes to bf16.  0x4300 is 128 in bf16, whose last mantissa bit is worth 1: a code or'd into it is 128 + c, and 128 + z subtracted
// from that leaves c - z, exactly.
__device__ __forceinline__ uint32_t with_magic(uint32_t x) {
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(r) : "r"(x));     // (x & mask) | magic
    return r;
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t zero_pair(uint32_t word) { return with_magic(__byte_perm(word, 0u, 0x3232)); }          // one key's
__device__ __forceinline__ uint32_t zero_pair(uint32_t a, uint32_t b) { return with_magic(__byte_perm(a, b, 0x7632)); }     // two keys'
__device__ __forceinline__ float scale_of(uint32_t word) { return __uint_as_float(word << 16); }

// ---- the kernel ---------------------------------------------------------------------------------
// S^T = K Q^T and O^T = V^T P^T on mma.sync m16n8k16 with the keys (the dimensions) as the 16 rows of A and NG groups of 8 query
// rows as N: a CTA of 8 warps, each with an online softmax of its own over every eighth chunk of the CTA's piece of a unit.
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
    static constexpr int kSteps = D / 16, kTiles = D / 16;
    static constexpr int kCopy = D == 80 ? 8 : 16;               // bytes per asynchronous copy
    static constexpr int kCodeBytes = kChunk * kRowBytes;
    static constexpr int kStageBytes = 2 * kCodeBytes + 2 * kChunk * 4;
    static constexpr int kStages = 3, kWarps = 8;
    static constexpr int kRingBytes = kStages * kStageBytes;
};

template <int D, int NG>
struct KvqSmem {
    using G = KvqGeometry<D>;
    static constexpr int kRows = 8 * NG;
    static constexpr int kPad = D + 4;                           // floats per row of a warp's partial result
    static constexpr int kRing = G::kWarps * G::kRingBytes;
    static constexpr int kJoin = G::kWarps * kRows * kPad * 4;
    static constexpr int kBytes = (kRing > kJoin ? kRing : kJoin) + G::kWarps * kRows * 8;
};

// floats of a CTA's partial result in the workspace: per row D sums, the reference and the sum of weights
__host__ __device__ constexpr int partial_floats(int D, int rows) { return rows * (D + 4); }

template <int D, int NG>
struct WarpState {
    float o[D / 16][NG][4];
    float ref[NG][2], sum[NG][2];
    uint32_t q[D / 16][NG][2];
};

// Raises the references to the maxima of the scores t (rare: only when one exceeds its reference by more than 2^8)
template <int D, int NG>
__device__ __forceinline__ void raise_refs(WarpState<D, NG>& w, const float (&t)[2][NG][4]) {
    #pragma unroll
    for (int n = 0; n < NG; ++n) {
        #pragma unroll
        for (int e = 0; e < 2; ++e) {
            float m = fmaxf(fmaxf(t[0][n][e], t[0][n][2 + e]), fmaxf(t[1][n][e], t[1][n][2 + e]));
            #pragma unroll
            for (int x = 4; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
            const float old = w.ref[n][e], now = fmaxf(old, m), f = exp2_approx(old - now);
            w.ref[n][e] = now;
            w.sum[n][e] *= f;
            #pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                w.o[k][n][e] *= f;
                w.o[k][n][2 + e] *= f;
            }
        }
    }
}

constexpr float kNoRef = -FLT_MAX / 2;               // below every score that counts; masked scores are -inf

// Scores t (log2 units, masked ones -inf) of two tiles of 16 keys to P^T fragments; sv: V scales of the lane's keys
template <int D, int NG>
__device__ __forceinline__ void softmax_chunk(WarpState<D, NG>& w, const float (&t)[2][NG][4], const float (&sv)[2][2], uint32_t (&p)[2][NG][2]) {
    bool high = false;
    #pragma unroll
    for (int n = 0; n < NG; ++n) {
        #pragma unroll
        for (int e = 0; e < 2; ++e)
            high |= fmaxf(fmaxf(t[0][n][e], t[0][n][2 + e]), fmaxf(t[1][n][e], t[1][n][2 + e])) > w.ref[n][e] + 8.f;
    }
    if (__any_sync(0xffffffffu, high)) raise_refs<D, NG>(w, t);
    #pragma unroll
    for (int j = 0; j < 2; ++j) {
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            float x[4];
            #pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = exp2_approx(t[j][n][i] - w.ref[n][i & 1]);
            w.sum[n][0] += x[0] + x[2];
            w.sum[n][1] += x[1] + x[3];
            // (a weight of zero stays zero whatever the scale: what is masked may have any)
            #pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = x[i] == 0.f ? 0.f : x[i] * sv[j][i >> 1];
            p[j][n][0] = transpose_8x8(pack2_bf16(x[0], x[1]));
            p[j][n][1] = transpose_8x8(pack2_bf16(x[2], x[3]));
        }
    }
}

__device__ __forceinline__ int key_of(int g) { return 4 * (g & 1) + (g >> 1); }

// One chunk of 32 cached slots, of which the first `valid` count
template <int D, int NG>
__device__ __forceinline__ void prefix_chunk(WarpState<D, NG>& w, uint32_t stage, int valid, float scale, int g, int c) {
    using G = KvqGeometry<D>;
    const uint32_t ks = stage, vs = stage + G::kCodeBytes, kp = stage + 2 * G::kCodeBytes, vp = kp + 4 * kChunk;
    float t[2][NG][4], sv[2][2];
    #pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int key = 16 * j + key_of(g);
        const uint32_t pa = lds32(kp + 4 * key), pb = lds32(kp + 4 * key + 32);
        sv[j][0] = scale_of(lds32(vp + 4 * key));
        sv[j][1] = scale_of(lds32(vp + 4 * key + 32));
        const uint32_t za = zero_pair(pa), zb = zero_pair(pb);
        uint32_t wa[4], wb[4];
        const uint32_t row = ks + key * G::kRowBytes + c * (4 * G::kWordsK);
        if constexpr (G::kWordsK == 4) {
            const uint4 x = lds128(row), y = lds128(row + 8 * G::kRowBytes);
            wa[0] = x.x, wa[1] = x.y, wa[2] = x.z, wa[3] = x.w;
            wb[0] = y.x, wb[1] = y.y, wb[2] = y.z, wb[3] = y.w;
        } else {
            const uint2 x = lds64(row), y = lds64(row + 8 * G::kRowBytes);
            wa[0] = x.x, wa[1] = x.y, wb[0] = y.x, wb[1] = y.y;
        }
        float acc[NG][4] = {};
        #pragma unroll
        for (int i = 0; i < G::kWordsK; ++i) {
            #pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint32_t a0 = sub_bf16x2(with_magic(wa[i] >> (8 * s)), za), a2 = sub_bf16x2(with_magic(wa[i] >> (8 * s + 4)), za);
                const uint32_t a1 = sub_bf16x2(with_magic(wb[i] >> (8 * s)), zb), a3 = sub_bf16x2(with_magic(wb[i] >> (8 * s + 4)), zb);
                #pragma unroll
                for (int n = 0; n < NG; ++n) mma_bf16(acc[n], a0, a1, a2, a3, w.q[2 * i + s][n][0], w.q[2 * i + s][n][1]);
            }
        }
        if constexpr (D == 80) {
            const uint32_t tail = ks + key * G::kRowBytes + 32;
            const uint2 x = lds64(tail), y = lds64(tail + 8 * G::kRowBytes);
            const uint32_t a0 = sub_bf16x2(with_magic(x.x >> (4 * c)), za), a2 = sub_bf16x2(with_magic(x.y >> (4 * c)), za);
            const uint32_t a1 = sub_bf16x2(with_magic(y.x >> (4 * c)), zb), a3 = sub_bf16x2(with_magic(y.y >> (4 * c)), zb);
            #pragma unroll
            for (int n = 0; n < NG; ++n) mma_bf16(acc[n], a0, a1, a2, a3, w.q[4][n][0], w.q[4][n][1]);
        }
        const float sa = scale_of(pa) * scale, sb = scale_of(pb) * scale;
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            #pragma unroll
            for (int i = 0; i < 4; ++i) t[j][n][i] = acc[n][i] * (i < 2 ? sa : sb);
        }
    }
    if (valid < kChunk) {
        #pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = 16 * j + key_of(g);
            #pragma unroll
            for (int n = 0; n < NG; ++n) {
                #pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (key + (i < 2 ? 0 : 8) >= valid) t[j][n][i] = -INFINITY;
            }
        }
    }
    uint32_t p[2][NG][2];
    softmax_chunk<D, NG>(w, t, sv, p);
    #pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t pz = vp + 4 * (16 * j + c);
        const uint32_t z01 = zero_pair(lds32(pz), lds32(pz + 16)), z23 = zero_pair(lds32(pz + 32), lds32(pz + 48));
        const uint32_t row = vs + (16 * j + c) * G::kRowBytes + g * (4 * G::kWordsV);
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
                const uint32_t a0 = sub_bf16x2(with_magic(l01 >> (4 * s)), z01), a1 = sub_bf16x2(with_magic(h01 >> (4 * s)), z01);
                const uint32_t a2 = sub_bf16x2(with_magic(l23 >> (4 * s)), z23), a3 = sub_bf16x2(with_magic(h23 >> (4 * s)), z23);
                #pragma unroll
                for (int n = 0; n < NG; ++n) mma_bf16(w.o[4 * i + s][n], a0, a1, a2, a3, p[j][n][0], p[j][n][1]);
            }
        }
        if constexpr (D == 80) {
            // the last 16 dimensions: rows g and g + 8 of the tile are dimensions 64 + g and 72 + g
            const int sh = 4 * (g >> 1) + 16 * (g & 1);
            uint2 x[4];
            #pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = lds64(vs + (16 * j + c + 4 * k) * G::kRowBytes + 32);
            const uint32_t a0 = sub_bf16x2(with_magic((x[0].x >> sh & 0xfu) | (x[1].x >> sh) << 16), z01);
            const uint32_t a1 = sub_bf16x2(with_magic((x[0].y >> sh & 0xfu) | (x[1].y >> sh) << 16), z01);
            const uint32_t a2 = sub_bf16x2(with_magic((x[2].x >> sh & 0xfu) | (x[3].x >> sh) << 16), z23);
            const uint32_t a3 = sub_bf16x2(with_magic((x[2].y >> sh & 0xfu) | (x[3].y >> sh) << 16), z23);
            #pragma unroll
            for (int n = 0; n < NG; ++n) mma_bf16(w.o[4][n], a0, a1, a2, a3, p[j][n][0], p[j][n][1]);
        }
    }
}

// The keys behind the prefix of a block: nodes 0 .. T - 1, then the streams of nodes t0 ..
struct Extra {
    int T, gamma, t0, count;                         // count: nodes and stream keys
    int row0, rows;                                  // of the block; rows of the sequence
};

__device__ __forceinline__ const __nv_bfloat16* extra_key(const KvqArgs& a, const Extra& x, int D, int b, int h, int e, bool value) {
    if (e < x.T) return (value ? a.v_tree : a.k_tree) + row_offset(a, D, b, h, Row{e, -1});
    const int s = e - x.T;
    return (value ? a.v_spec : a.k_spec) + row_offset(a, D, b, h, Row{x.t0 + s / x.gamma, s % x.gamma});
}

// One chunk of 32 keys behind the prefix, from `first` on
template <int D, int NG>
__device__ __forceinline__ void extra_chunk(WarpState<D, NG>& w, const KvqArgs& a, const Extra& x, int b, int h, int first, int g, int c) {
    using G = KvqGeometry<D>;
    float t[2][NG][4];
    const float one[2][2] = {{1.f, 1.f}, {1.f, 1.f}};
    #pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int ea = first + 16 * j + key_of(g), eb = ea + 8;
        const __nv_bfloat16* ka = ea < x.count ? extra_key(a, x, D, b, h, ea, false) : nullptr;
        const __nv_bfloat16* kb = eb < x.count ? extra_key(a, x, D, b, h, eb, false) : nullptr;
        float acc[NG][4] = {};
        #pragma unroll
        for (int i = 0; i < G::kWordsK; ++i) {
            uint4 u = {}, v = {};
            if (ka) u = *reinterpret_cast<const uint4*>(ka + c * (8 * G::kWordsK) + 8 * i);
            if (kb) v = *reinterpret_cast<const uint4*>(kb + c * (8 * G::kWordsK) + 8 * i);
            #pragma unroll
            for (int n = 0; n < NG; ++n) {
                mma_bf16(acc[n], u.x, v.x, u.y, v.y, w.q[2 * i][n][0], w.q[2 * i][n][1]);
                mma_bf16(acc[n], u.z, v.z, u.w, v.w, w.q[2 * i + 1][n][0], w.q[2 * i + 1][n][1]);
            }
        }
        if constexpr (D == 80) {
            uint32_t u[4] = {};
            if (ka) u[0] = *reinterpret_cast<const uint32_t*>(ka + 64 + 2 * c), u[2] = *reinterpret_cast<const uint32_t*>(ka + 72 + 2 * c);
            if (kb) u[1] = *reinterpret_cast<const uint32_t*>(kb + 64 + 2 * c), u[3] = *reinterpret_cast<const uint32_t*>(kb + 72 + 2 * c);
            #pragma unroll
            for (int n = 0; n < NG; ++n) mma_bf16(acc[n], u[0], u[1], u[2], u[3], w.q[4][n][0], w.q[4][n][1]);
        }
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            #pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = x.row0 + 8 * n + 2 * c + e;
                unsigned long long see = 0;
                int lo = 0, hi = 0;                  // stream keys the row sees
                if (r < x.rows) {
                    const Row q = row_of(r, x.T, x.gamma);
                    see = a.trees[b].anc_mask[q.t];
                    lo = x.T + (q.t - x.t0) * x.gamma;
                    hi = q.j < 0 ? lo : lo + q.j + 1;
                }
                const bool sa = ea < x.T ? (see >> ea & 1ull) : (ea >= lo && ea < hi);
                const bool sb = eb < x.T ? (see >> eb & 1ull) : (eb >= lo && eb < hi);
                t[j][n][e] = sa ? acc[n][e] * a.scale : -INFINITY;
                t[j][n][2 + e] = sb ? acc[n][2 + e] * a.scale : -INFINITY;
            }
        }
    }
    uint32_t p[2][NG][2];
    softmax_chunk<D, NG>(w, t, one, p);
    #pragma unroll
    for (int j = 0; j < 2; ++j) {
        const __nv_bfloat16* vk[4];
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int e = first + 16 * j + c + 4 * k;
            vk[k] = e < x.count ? extra_key(a, x, D, b, h, e, true) : nullptr;
        }
        #pragma unroll
        for (int i = 0; i < G::kWordsV; ++i) {
            uint4 v[4] = {};
            #pragma unroll
            for (int k = 0; k < 4; ++k)
                if (vk[k]) v[k] = *reinterpret_cast<const uint4*>(vk[k] + g * (8 * G::kWordsV) + 8 * i);
            const uint32_t v0[4] = {v[0].x, v[0].y, v[0].z, v[0].w}, v1[4] = {v[1].x, v[1].y, v[1].z, v[1].w};
            const uint32_t v2[4] = {v[2].x, v[2].y, v[2].z, v[2].w}, v3[4] = {v[3].x, v[3].y, v[3].z, v[3].w};
            #pragma unroll
            for (int s = 0; s < 4; ++s) {
                const uint32_t a0 = __byte_perm(v0[s], v1[s], 0x5410), a1 = __byte_perm(v0[s], v1[s], 0x7632);
                const uint32_t a2 = __byte_perm(v2[s], v3[s], 0x5410), a3 = __byte_perm(v2[s], v3[s], 0x7632);
                #pragma unroll
                for (int n = 0; n < NG; ++n) mma_bf16(w.o[4 * i + s][n], a0, a1, a2, a3, p[j][n][0], p[j][n][1]);
            }
        }
        if constexpr (D == 80) {
            uint32_t lo[4] = {}, hi[4] = {};
            #pragma unroll
            for (int k = 0; k < 4; ++k)
                if (vk[k]) {
                    lo[k] = reinterpret_cast<const unsigned short*>(vk[k])[64 + g];
                    hi[k] = reinterpret_cast<const unsigned short*>(vk[k])[72 + g];
                }
            #pragma unroll
            for (int n = 0; n < NG; ++n)
                mma_bf16(w.o[4][n], lo[0] | lo[1] << 16, hi[0] | hi[1] << 16, lo[2] | lo[3] << 16, hi[2] | hi[3] << 16, p[j][n][0], p[j][n][1]);
        }
    }
}

// Asynchronous copies of a chunk's codes, scales and zero points into a stage of the warp's ring.  Slots behind `last` read as zero.
template <int D>
__device__ __forceinline__ void load_chunk(const KvqArgs& a, const Seq& s, int h, int chunk, uint32_t stage, int lane) {
    using G = KvqGeometry<D>;
    constexpr int kPer = G::kRowBytes / G::kCopy;
    const int key0 = chunk * kChunk;
    const long long slot = s.start + key0;
    #pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int item = i * 32 + lane, key = item / kPer, at = item - key * kPer;
        const bool real = key0 + key < s.L;
        const long long off = real ? (slot + key) * a.slot_stride + h * a.head_stride + at * G::kCopy : 0;
        copy_async<G::kCopy>(stage + key * G::kRowBytes + at * G::kCopy, a.k_codes + off, real);
        copy_async<G::kCopy>(stage + G::kCodeBytes + key * G::kRowBytes + at * G::kCopy, a.v_codes + off, real);
    }
    const bool real = key0 + lane < s.L;
    const long long off = real ? (slot + lane) * a.p_slot + h * a.p_head : 0;
    copy_async<4>(stage + 2 * G::kCodeBytes + 4 * lane, a.k_params + off, real);
    copy_async<4>(stage + 2 * G::kCodeBytes + 4 * kChunk + 4 * lane, a.v_params + off, real);
}

// Dimensions that lane (g, c) holds in tile k of O^T: rows g (returned) and g + 8 (the next dimension; 8 further in the last tile of 80)
template <int D>
__device__ __forceinline__ int tile_dim(int k, int g) {
    using G = KvqGeometry<D>;
    return k < 4 * G::kWordsV ? g * (8 * G::kWordsV) + 2 * k : G::kMain + g;
}

template <int D, int NG>
__global__ void __launch_bounds__(256, NG == 1 ? 2 : 1) msa_attention_kvq_rows_kernel(const __grid_constant__ KvqArgs a) {
    using G = KvqGeometry<D>;
    using S = KvqSmem<D, NG>;
    constexpr int ROWS = 8 * NG, PAD = S::kPad;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int joined;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const uint32_t ring = smem_addr(smem) + warp * G::kRingBytes;
    float* const parts = reinterpret_cast<float*>(smem);                                      // [warp][row][PAD], in the rings' place
    float2* const stats = reinterpret_cast<float2*>(smem + S::kBytes - G::kWarps * ROWS * 8);   // [warp][row]: reference, sum
    wait_for_previous_kernel();
    release_next_kernel();

    // how long the line is, and this CTA's piece of it
    long long total = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
        long long mine = 0;
        if (b0 + lane < a.batch) {
            const Seq s = load_seq<ROWS>(a, b0 + lane);
            mine = static_cast<long long>(s.chunks) * s.blocks * a.n_heads;
        }
        #pragma unroll
        for (int x = 16; x > 0; x >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, x);
        total += mine;
    }
    const long long ctas = min(static_cast<long long>(gridDim.x), (total + G::kWarps - 1) / G::kWarps);
    if (static_cast<long long>(blockIdx.x) >= ctas) return;
    const auto cut = [&](long long i) { return total * i / ctas; };
    const auto owner = [&](long long pos) {                       // the CTA whose piece holds position pos
        long long i = pos * ctas / total;
        while (cut(i + 1) <= pos) ++i;
        while (cut(i) > pos) --i;
        return i;
    };
    long long pos = cut(blockIdx.x);
    const long long end = cut(blockIdx.x + 1ll);
    // the sequence that holds the piece's first chunk
    long long base = 0;
    int b = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
        long long mine = 0;
        if (b0 + lane < a.batch) {
            const Seq s = load_seq<ROWS>(a, b0 + lane);
            mine = static_cast<long long>(s.chunks) * s.blocks * a.n_heads;
        }
        long long upto = mine;
        #pragma unroll
        for (int x = 1; x < 32; x <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, x);
            if (lane >= x) upto += y;
        }
        const unsigned here = __ballot_sync(0xffffffffu, base + upto > pos);
        if (here) {
            const int l = __ffs(here) - 1;
            b = b0 + l;
            base += __shfl_sync(0xffffffffu, upto - mine, l);
            break;
        }
        base += __shfl_sync(0xffffffffu, upto, 31);
    }
    Seq s = load_seq<ROWS>(a, b);
    int* const counters = reinterpret_cast<int*>(a.ws + kWsHeaderBytes);
    float* const partial = reinterpret_cast<float*>(a.ws + kWsHeaderBytes + (4ull * gridDim.x + 255) / 256 * 256);

    while (pos < end) {
        while (pos >= base + static_cast<long long>(s.chunks) * s.blocks * a.n_heads) {
            base += static_cast<long long>(s.chunks) * s.blocks * a.n_heads;
            s = load_seq<ROWS>(a, ++b);
        }
        const int unit = static_cast<int>((pos - base) / s.chunks);
        const long long unit0 = base + static_cast<long long>(unit) * s.chunks;
        const int from = static_cast<int>(pos - unit0), to = static_cast<int>(min(end - unit0, static_cast<long long>(s.chunks)));
        const int h = unit / s.blocks, row0 = (unit - h * s.blocks) * ROWS;
        const int P = prefix_chunks(s.L);

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
            w.ref[n][0] = w.ref[n][1] = kNoRef;
            w.sum[n][0] = w.sum[n][1] = 0.f;
        }
        int fetch = from + warp;
        #pragma unroll
        for (int i = 0; i < G::kStages - 1; ++i, fetch += G::kWarps) {
            if (fetch < min(to, P)) load_chunk<D>(a, s, h, fetch, ring + i * G::kStageBytes, lane);
            copy_commit();
        }
        // query rows: row g of every group, the dimensions that c holds
        #pragma unroll
        for (int n = 0; n < NG; ++n) {
            const int r = row0 + 8 * n + g;
            const __nv_bfloat16* q = nullptr;
            if (r < s.rows) {
                const Row x = row_of(r, s.T, a.gamma);
                q = (x.j < 0 ? a.q_main : a.q_spec) + row_offset(a, D, b, h, x);
            }
            #pragma unroll
            for (int i = 0; i < G::kWordsK; ++i) {
                uint4 v = {};
                if (q) v = *reinterpret_cast<const uint4*>(q + c * (8 * G::kWordsK) + 8 * i);
                w.q[2 * i][n][0] = v.x, w.q[2 * i][n][1] = v.y, w.q[2 * i + 1][n][0] = v.z, w.q[2 * i + 1][n][1] = v.w;
            }
            if constexpr (D == 80) {
                w.q[4][n][0] = q ? *reinterpret_cast<const uint32_t*>(q + 64 + 2 * c) : 0u;
                w.q[4][n][1] = q ? *reinterpret_cast<const uint32_t*>(q + 72 + 2 * c) : 0u;
            }
        }
        int stage = 0;
        for (int k = from + warp; k < to; k += G::kWarps) {
            copy_wait<G::kStages - 2>();
            __syncwarp();
            {
                int slot = stage + G::kStages - 1;
                if (slot >= G::kStages) slot -= G::kStages;
                if (fetch < min(to, P)) load_chunk<D>(a, s, h, fetch, ring + slot * G::kStageBytes, lane);
                copy_commit();
                fetch += G::kWarps;
            }
            if (k < P) {
                prefix_chunk<D, NG>(w, ring + stage * G::kStageBytes, min(kChunk, s.L - k * kChunk), a.scale, g, c);
            } else {
                Extra x;
                x.T = s.T, x.gamma = max(a.gamma, 1), x.row0 = row0, x.rows = s.rows, x.t0 = 0, x.count = s.T;
                const int last = min(row0 + ROWS, s.rows) - 1;
                if (last >= s.T) {                   // the block has stream rows: the streams of their nodes
                    x.t0 = row0 < s.T ? 0 : (row0 - s.T) / a.gamma;
                    x.count = s.T + ((last - s.T) / a.gamma - x.t0 + 1) * a.gamma;
                }
                if ((k - P) * kChunk < x.count) extra_chunk<D, NG>(w, a, x, b, h, (k - P) * kChunk, g, c);
            }
            if (++stage == G::kStages) stage = 0;
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
                if (g == 0) stats[warp * ROWS + 8 * n + 2 * c + e] = make_float2(w.ref[n][e], w.sum[n][e]);
            }
        }
        #pragma unroll
        for (int k = 0; k < G::kTiles; ++k) {
            const int dim = tile_dim<D>(k, g);
            #pragma unroll
            for (int n = 0; n < NG; ++n) {
                #pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float* dst = parts + (warp * ROWS + 8 * n + 2 * c + e) * PAD + dim;
                    if (k < 4 * G::kWordsV) *reinterpret_cast<float2*>(dst) = make_float2(w.o[k][n][e], w.o[k][n][2 + e]);
                    else dst[0] = w.o[k][n][e], dst[8] = w.o[k][n][2 + e];
                }
            }
        }
        __syncthreads();

        // whole unit: output.  A piece of one: partial rows to the workspace; the last CTA of the unit joins them.
        const bool whole = from == 0 && to == s.chunks;
        const long long i0 = whole ? 0 : owner(unit0), i1 = whole ? 0 : owner(unit0 + s.chunks - 1);
        // (a CTA's first unit and its last one: two places per CTA)
        const auto place = [&](long long i) { return partial + (2 * i + (i == i0 && cut(i) < unit0 ? 1 : 0)) * partial_floats(D, ROWS); };
        float* const mine = place(blockIdx.x);
        constexpr int kItems = ROWS * (D / 8);
        const auto store_row = [&](int r, int d0, const float (&o)[8], float m, float l) {
            if (row0 + r >= s.rows) return;
            const Row x = row_of(row0 + r, s.T, a.gamma);
            const long long off = row_offset(a, D, b, h, x);
            const float f = 1.f / l;
            uint4 v;
            v.x = pack2_bf16(o[0] * f, o[1] * f), v.y = pack2_bf16(o[2] * f, o[3] * f);
            v.z = pack2_bf16(o[4] * f, o[5] * f), v.w = pack2_bf16(o[6] * f, o[7] * f);
            *reinterpret_cast<uint4*>((x.j < 0 ? a.o_main : a.o_spec) + off + d0) = v;
            float* lse = x.j < 0 ? a.lse_main : a.lse_spec;
            if (d0 == 0 && lse != nullptr) lse[off / D] = (m + log2f(l)) * 0.6931471805599453f;
        };
        for (int item = tid; item < kItems; item += 256) {
            const int r = item / (D / 8), d0 = (item - r * (D / 8)) * 8;
            float m = kNoRef, l = 0.f, o[8] = {};
            #pragma unroll
            for (int i = 0; i < G::kWarps; ++i) m = fmaxf(m, stats[i * ROWS + r].x);
            #pragma unroll
            for (int i = 0; i < G::kWarps; ++i) {
                const float2 st = stats[i * ROWS + r];
                const float f = exp2_approx(st.x - m);
                l += st.y * f;
                const float* src = parts + (i * ROWS + r) * PAD + d0;
                const float4 u = *reinterpret_cast<const float4*>(src), v = *reinterpret_cast<const float4*>(src + 4);
                o[0] += u.x * f, o[1] += u.y * f, o[2] += u.z * f, o[3] += u.w * f;
                o[4] += v.x * f, o[5] += v.y * f, o[6] += v.z * f, o[7] += v.w * f;
            }
            if (whole) {
                store_row(r, d0, o, m, l);
            } else {
                float* dst = mine + r * D + d0;
                __stcg(reinterpret_cast<float4*>(dst), make_float4(o[0], o[1], o[2], o[3]));
                __stcg(reinterpret_cast<float4*>(dst) + 1, make_float4(o[4], o[5], o[6], o[7]));
                if (d0 == 0) __stcg(reinterpret_cast<float2*>(mine + ROWS * D) + r, make_float2(m, l));
            }
        }
        if (!whole) {
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const int n = static_cast<int>(i1 - i0 + 1);
                const int before = atomicAdd(counters + i0, 1);
                joined = before == n - 1;
                if (joined) counters[i0] = 0;
                __threadfence();
            }
            __syncthreads();
            if (joined) {
                for (int item = tid; item < kItems; item += 256) {
                    const int r = item / (D / 8), d0 = (item - r * (D / 8)) * 8;
                    float m = kNoRef, l = 0.f, o[8] = {};
                    for (long long i = i0; i <= i1; ++i) m = fmaxf(m, __ldcg(reinterpret_cast<const float2*>(place(i) + ROWS * D) + r).x);
                    for (long long i = i0; i <= i1; ++i) {
                        const float* src = place(i);
                        const float2 st = __ldcg(reinterpret_cast<const float2*>(src + ROWS * D) + r);
                        const float f = exp2_approx(st.x - m);
                        l += st.y * f;
                        const float4 u = __ldcg(reinterpret_cast<const float4*>(src + r * D + d0)), v = __ldcg(reinterpret_cast<const float4*>(src + r * D + d0) + 1);
                        o[0] += u.x * f, o[1] += u.y * f, o[2] += u.z * f, o[3] += u.w * f;
                        o[4] += v.x * f, o[5] += v.y * f, o[6] += v.z * f, o[7] += v.w * f;
                    }
                    store_row(r, d0, o, m, l);
                }
            }
        }
        __syncthreads();                             // the partial results' place goes back to the rings
        pos = unit0 + to;
    }
}

// ---- host ---------------------------------------------------------------------------------------
static int q_rows(const ss_kvq_attn_params& p) { return p.max_nodes * (1 + p.gamma); }
static int group_count(const ss_kvq_attn_params& p) { return q_rows(p) <= 8 ? 1 : 2; }
static int most_ctas(const ss_kvq_attn_params& p) { return sm_count() * (group_count(p) == 1 ? 2 : 1); }

static size_t kvq_workspace(const ss_kvq_attn_params& p) {
    const size_t ctas = static_cast<size_t>(most_ctas(p));
    return kWsHeaderBytes + (4 * ctas + 255) / 256 * 256 + 2 * ctas * partial_floats(p.cache.head_dim, 8 * group_count(p)) * sizeof(float);
}

template <int D, int NG>
static int32_t launch_kvq_rows(const KvqArgs& args, int ctas, cudaStream_t stream) {
    const auto kernel = msa_attention_kvq_rows_kernel<D, NG>;
    constexpr int bytes = KvqSmem<D, NG>::kBytes;
    static bool set[64] = {};                        // (per device; setting it twice does no harm)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SS_ERR_CUDA;
    if (dev < 0 || dev >= 64 || !set[dev]) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return SS_ERR_CUDA;
        if (dev >= 0 && dev < 64) set[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(ctas));
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args) == cudaSuccess ? SS_OK : SS_ERR_CUDA;
}

template <int D>
static int32_t launch_kvq(const ss_kvq_attn_params& p, const KvqArgs& args, int ctas, cudaStream_t stream) {
    return group_count(p) == 1 ? launch_kvq_rows<D, 1>(args, ctas, stream) : launch_kvq_rows<D, 2>(args, ctas, stream);
}

static int32_t kvq_check_shapes(const ss_kvq_attn_params* p) {
    if (!p) return SS_ERR_INVALID_ARG;
    const ss_kvq_cache& c = p->cache;
    if (p->batch < 1 || c.n_heads < 1 || p->max_nodes < 1 || p->gamma < 0) return SS_ERR_INVALID_ARG;
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
    // no more CTAs than the slab can give chunks for (eight to a CTA)
    const int block = 8 * group_count(*p), blocks = (q_rows(*p) + block - 1) / block;
    const long long chunks = static_cast<long long>(c.n_heads) * blocks *
                             ((c.total_slots + kChunk - 1) / kChunk + p->batch * (1ll + extra_chunks(p->max_nodes, p->gamma, block)));
    const int ctas = static_cast<int>(std::min<long long>(most_ctas(*p), (chunks + 7) / 8));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return c.head_dim == 128 ? launch_kvq<128>(*p, a, ctas, s) : c.head_dim == 80 ? launch_kvq<80>(*p, a, ctas, s) : launch_kvq<64>(*p, a, ctas, s);
}
