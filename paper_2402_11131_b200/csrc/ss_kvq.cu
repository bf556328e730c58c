// Rows into and out of a cache held in 4 bits (format and layout: ss_msa.h).  Compiled without fast-math: scales and codes are
// defined bit by bit.
//
// Both kernels stream: HBM bounds them, with the instructions per value (12 of a write, 73 % of the issue slots) close behind.  Four
// users' prompts into eight layers, 8240 rows of 32 x 128 each: written in 243 us (1.31 GB, 5.4 TB/s), read back in 222 (1.31 GB, 5.9 TB/s).
// One layer of 2048 slots is read in 7.9 us, 4 of them the launch and one trip to memory.  A thread holds 16 values, 8 at dimension 8 at and 8 at D / 2 + 8 at: a row of a head is 4, 5
// or 8 neighbouring lanes that read (or write) runs of 16 bytes next to each other, and find the row's extremes with three exchanges.
//
// The arithmetic of the scale.  s is the smallest bf16 with 15 s >= hi - lo.  15 s is an fp32 number, so that is 15 s >= t with t the
// sum rounded up to fp32.  (Everything is divided by 16 first, exactly, so that hi - lo does not overflow.)  t * (1 + 2^-22) 16 / 15
// cut to bf16 is that s or the bf16 below: it is not below the quotient's cut, and above it only where the bf16 above is s.
// The arithmetic of the codes.  x and s have 8 significant bits, so x / s either lies exactly between two whole numbers or is at
// least 2^-13 of itself away from there (the midpoints are (2k + 1) / 2 with 2k + 1 <= 31, and 255 * 31 < 2^13).  x * (1 / s) with
// 1 / s enlarged by 2^-16 is off by less than that and on the far side of the midpoint where the quotient is exactly one, so that
// one fused multiply-add with 1.5 * 2^23 + z, whose sum has no fraction bits left, rounds as if the quotient were exact; the sum's low
// 16 bits are round(x / s) + z, clamped two at a time.
#include <cuda_bf16.h>

#include <climits>

#include "ss_common.cuh"

namespace ss {

constexpr int kKvqThreads = 256;
constexpr int kKvqCtas = 4;                         // resident on an SM: 64 registers a thread
constexpr float kRoundMagic = 12582912.f;          // 1.5 * 2^23

struct KvqGeo {
    unsigned char *k_codes, *v_codes;
    uint32_t *k_params, *v_params;
    long long layer_stride, slot_stride, head_stride, p_layer, p_slot, p_head, total_slots;
    unsigned char *k_rows, *v_rows;                 // bf16; strides in bytes
    long long r_layer, r_batch, r_row, r_head;
    int n_heads, max_rows, layers;
};

// Two at a time; NaN where one of the operands is
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

__device__ __forceinline__ float rcp_approx(float x) {
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// A row of D values over D / 16 neighbouring lanes, 16 values each: returns the row's word of scale and zero point and this lane's
// two words of codes.  All 32 lanes take part; `base` is the first lane of the row, `at` this lane's place in it.
template <int D>
__device__ __forceinline__ uint32_t quantise_row(const uint4 (&x)[2], int base, int at, uint32_t (&codes)[2]) {
    constexpr int G = D / 16;
    const uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    // largest and smallest value, with zero among them
    uint32_t hi2 = 0u, lo2 = 0u;
    #pragma unroll
    for (int i = 0; i < 8; ++i) hi2 = max_bf16x2(hi2, w[i]), lo2 = min_bf16x2(lo2, w[i]);
    uint32_t ext = max_bf16x2(__byte_perm(hi2, lo2, 0x5410) & 0x7fff7fffu, __byte_perm(hi2, lo2, 0x7632) & 0x7fff7fffu);   // low half: hi, high half: -lo
    #pragma unroll
    for (int step = 0; step < 3; ++step) {
        const int shift = step == 0 ? 1 : step == 1 ? 2 : (G == 8 ? 4 : 1);     // (after 1 + 2 + 1 a lane has seen all of 4 or 5)
        int from = at + shift;
        if (from >= G) from -= G;
        ext = max_bf16x2(ext, __shfl_sync(0xffffffffu, ext, base + from));
    }
    const float hi = __uint_as_float(ext << 16), nlo = __uint_as_float(ext & 0xffff0000u);
    const bool bad = !(hi < INFINITY && nlo < INFINITY);          // an infinity or a NaN in the row
    const float t = __fadd_ru(hi * 0.0625f, nlo * 0.0625f);
    uint32_t sb = __float_as_uint(__fmul_rn(t, 1.06666692f)) >> 16;
    if (__uint_as_float(sb << 16) * 0.9375f < t) ++sb;
    sb = max(sb, 0x0380u);                                        // 2^-120
    const float s = __uint_as_float(sb << 16);
    const float inv = __fmul_rn(rcp_approx(s), 1.0000152587890625f);
    const uint32_t z = bad ? 0u : (__float_as_uint(__fmaf_rn(nlo, inv, kRoundMagic)) & 0xfu);   // (at most 15: nlo <= 15 s)
    const float from = kRoundMagic + static_cast<float>(z);
    #pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t v = 0u;
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t a = __float_as_uint(__fmaf_rn(__uint_as_float(w[4 * h + i] << 16), inv, from));
            const uint32_t b = __float_as_uint(__fmaf_rn(__uint_as_float(w[4 * h + i] & 0xffff0000u), inv, from));
            v |= __vimin_s16x2_relu(__byte_perm(a, b, 0x5410), 0x000f000fu) << (4 * i);
        }
        codes[h] = bad ? 0u : v;
    }
    return (bad ? 0x7fffu : sb) | (z << 16);
}

// The sequence's run of rows: from slot `*slot0`, `*n` of them (0: nothing to do).  Returns false where they do not fit.
__device__ __forceinline__ bool write_run(const KvqGeo& g, const int64_t* kv_start, const int32_t* kv_len_in, const int32_t* n_rows,
                                          const int32_t* path, const int32_t* kv_capacity, int b, long long* slot0, int* n, int* L) {
    const int limit = path != nullptr ? SS_PATH_STRIDE : g.max_rows;
    *L = kv_len_in[b];
    *n = n_rows != nullptr ? max(0, min(n_rows[b], limit)) : min(g.max_rows, limit);
    const long long start = kv_start[b];             // (anything: no sum of it before it is known to be near the slab)
    const bool fits = *L >= 0 && *n <= INT_MAX - *L && start >= -static_cast<long long>(*L) && start <= g.total_slots - *L - *n &&
                      (kv_capacity == nullptr || *L + *n <= kv_capacity[b]);
    *slot0 = fits ? start + *L : 0;
    return fits;
}

// A warp's unit of work is a few neighbouring slots of one head, D / 16 lanes for each: a head's scales lie slot after slot, and
// written head after head they would cost a sector per word.
template <int D>
struct Unit {
    static constexpr int G = D / 16, SLOTS = 32 / G, WARPS = kKvqThreads / 32;
};

// Units in order from unit `first` on, `by` apart: divisions at the start only.  (r: blocks of slots.  There are at most 2^30 slots and
// steps of some 2^17 units: no overflow.)
struct Walk {
    int r, h, dr, dh, n_heads;
    __device__ __forceinline__ Walk(int heads, int first, int by) : n_heads(heads) {
        r = first / heads, h = first - r * heads;
        dr = by / heads, dh = by - dr * heads;
    }
    // true: on to other slots
    __device__ __forceinline__ bool step() {
        r += dr, h += dh;
        const bool on = h >= n_heads;
        if (on) h -= n_heads, ++r;
        return on;
    }
};

// Where a lane's row of the unit lies, for strides of a slot and of a head: sums along the walk, not products
struct Trail {
    long long at, by, wrap;
    __device__ __forceinline__ Trail(const Walk& w, int slots, int sub, long long slot_stride, long long head_stride)
        : at((static_cast<long long>(w.r) * slots + sub) * slot_stride + w.h * head_stride), by(static_cast<long long>(w.dr) * slots * slot_stride + w.dh * head_stride),
          wrap(slots * slot_stride - w.n_heads * head_stride) {}
    __device__ __forceinline__ void step(bool on) {
        at += by;
        if (on) at += wrap;
    }
};

template <int D>
__global__ void __launch_bounds__(kKvqThreads, kKvqCtas)
kvq_write_kernel(const __grid_constant__ KvqGeo g, const int64_t* __restrict__ kv_start, const int32_t* __restrict__ kv_len_in,
                 const int32_t* __restrict__ n_rows, const int32_t* __restrict__ path, const int32_t* __restrict__ kv_capacity,
                 int32_t* __restrict__ kv_len_out, void* __restrict__ status) {
    using U = Unit<D>;
    constexpr int G = U::G;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = min(lane / G, U::SLOTS - 1), base = sub * G, at = lane < U::SLOTS * G ? lane - base : 0;
    const bool mine = lane < U::SLOTS * G;
    const int layer = blockIdx.y >> 1, b = blockIdx.z;
    const bool is_v = blockIdx.y & 1;
    wait_for_previous_kernel();
    release_next_kernel();
    long long slot0;
    int n, L;
    const bool fits = write_run(g, kv_start, kv_len_in, n_rows, path, kv_capacity, b, &slot0, &n, &L);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
        if (!fits && status != nullptr) set_status(status, SS_ERR_CAPACITY);
        if (kv_len_out != nullptr) kv_len_out[b] = fits ? L + n : L;
    }
    if (!fits) return;
    const int* const nodes = path == nullptr ? nullptr : path + static_cast<long long>(b) * SS_PATH_STRIDE;
    const unsigned char* rows = (is_v ? g.v_rows : g.k_rows) + layer * g.r_layer + b * g.r_batch + 16 * at;
    unsigned char* codes = (is_v ? g.v_codes : g.k_codes) + layer * g.layer_stride + slot0 * g.slot_stride + 4 * at;
    uint32_t* params = (is_v ? g.v_params : g.k_params) + layer * g.p_layer + slot0 * g.p_slot;
    Walk unit(g.n_heads, blockIdx.x * U::WARPS + warp, gridDim.x * U::WARPS);
    Trail row_at(unit, U::SLOTS, sub, g.r_row, g.r_head), code_at(unit, U::SLOTS, sub, g.slot_stride, g.head_stride), word_at(unit, U::SLOTS, sub, g.p_slot, g.p_head);
    // (lanes without a row have its last contents: a row's lanes have one or none together)
    const auto fetch = [&](uint4 (&x)[2]) {
        const int r = unit.r * U::SLOTS + sub;
        bool live = mine && r < n;
        const unsigned char* src = rows + row_at.at;
        if (nodes == nullptr) {
            live = live && r < g.max_rows;
        } else if (live) {
            const int node = nodes[r];
            live = node >= 0 && node < g.max_rows;
            src = rows + node * g.r_row + unit.h * g.r_head;
        }
        if (live) x[0] = __ldcs(reinterpret_cast<const uint4*>(src)), x[1] = __ldcs(reinterpret_cast<const uint4*>(src) + G);
        return live;
    };
    const auto store = [&](const uint4 (&x)[2], bool live, unsigned char* to, uint32_t* word_to) {
        uint32_t c[2];
        const uint32_t word = quantise_row<D>(x, base, at, c);
        if (live) {
            reinterpret_cast<uint32_t*>(to)[0] = c[0], reinterpret_cast<uint32_t*>(to)[G] = c[1];
            if (at == 0) *word_to = word;
        }
    };
    // two units' rows in turn: the next ones are on their way while these are turned into codes
    uint4 x[2] = {}, y[2] = {};
    bool live = fetch(x);
    while (unit.r * U::SLOTS < n) {
        unsigned char* to = codes + code_at.at;
        uint32_t* word_to = params + word_at.at;
        const auto step = [&] {
            const bool on = unit.step();
            row_at.step(on), code_at.step(on), word_at.step(on);
        };
        step();
        const bool more = fetch(y);
        store(x, live, to, word_to);
        if (unit.r * U::SLOTS >= n) break;
        to = codes + code_at.at, word_to = params + word_at.at;
        step();
        live = fetch(x);
        store(y, more, to, word_to);
    }
}

// Where kv_len_out overlaps an array that every CTA reads, the lengths are updated by a second, stream-ordered launch.
__global__ void kvq_len_kernel(const __grid_constant__ KvqGeo g, const int64_t* kv_start, const int32_t* kv_len_in,
                               const int32_t* n_rows, const int32_t* path, const int32_t* kv_capacity, int32_t* kv_len_out, int batch) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    wait_for_previous_kernel();
    long long slot0;
    int n = 0, L = 0;
    const bool fits = b < batch && write_run(g, kv_start, kv_len_in, n_rows, path, kv_capacity, b, &slot0, &n, &L);
    __syncthreads();                     // (one CTA: all inputs are read before the first length is written)
    if (b < batch) kv_len_out[b] = fits ? L + n : L;
}

__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <int D>
__global__ void __launch_bounds__(kKvqThreads, kKvqCtas)
kvq_read_kernel(const __grid_constant__ KvqGeo g, const int64_t* __restrict__ kv_start, const int32_t* __restrict__ first,
                const int32_t* __restrict__ n_rows) {
    using U = Unit<D>;
    constexpr int G = U::G, AHEAD = D == 80 ? 3 : 4;  // units on their way at a time (as many as 64 registers hold)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = min(lane / G, U::SLOTS - 1), at = lane - sub * G;
    const bool mine = lane < U::SLOTS * G;
    wait_for_previous_kernel();
    release_next_kernel();
    const int layer = blockIdx.y >> 1, b = blockIdx.z;
    const bool is_v = blockIdx.y & 1;
    const int n = n_rows != nullptr ? min(n_rows[b], g.max_rows) : g.max_rows;
    // (a start so far outside that no row's slot is in the slab may be nearer: no sum overflows)
    const long long slot0 = min(max(static_cast<long long>(kv_start[b]), -(1ll << 32)), g.total_slots + (1ll << 31)) + (first != nullptr ? first[b] : 0);
    const unsigned char* codes = (is_v ? g.v_codes : g.k_codes) + layer * g.layer_stride + 4 * at;
    const uint32_t* params = (is_v ? g.v_params : g.k_params) + layer * g.p_layer;
    unsigned char* rows = (is_v ? g.v_rows : g.k_rows) + layer * g.r_layer + b * g.r_batch + 16 * at;
    codes += slot0 * g.slot_stride, params += slot0 * g.p_slot;
    // rows whose slots lie in the slab
    const int lo = static_cast<int>(min(max(-slot0, 0ll), static_cast<long long>(max(n, 0)))), hi = static_cast<int>(max(min(g.total_slots - slot0, static_cast<long long>(n)), 0ll));
    Walk unit(g.n_heads, blockIdx.x * U::WARPS + warp, gridDim.x * U::WARPS);
    Trail row_at(unit, U::SLOTS, sub, g.r_row, g.r_head), code_at(unit, U::SLOTS, sub, g.slot_stride, g.head_stride), word_at(unit, U::SLOTS, sub, g.p_slot, g.p_head);
    while (unit.r * U::SLOTS < hi) {
        uint32_t c[AHEAD][2], p[AHEAD];
        unsigned char* to[AHEAD];                     // null: nothing to do
        #pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int r = unit.r * U::SLOTS + sub;
            const bool live = mine && r >= lo && r < hi;
            to[k] = live ? rows + row_at.at : nullptr;
            if (live) {
                const uint32_t* const from = reinterpret_cast<const uint32_t*>(codes + code_at.at);
                c[k][0] = __ldcs(from), c[k][1] = __ldcs(from + G);
                p[k] = params[word_at.at];
            }
            const bool on = unit.step();
            row_at.step(on), code_at.step(on), word_at.step(on);
        }
        #pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (to[k] == nullptr) continue;
            // c - z from bf16 128 + c and 128 + z, exactly; times s, rounded once
            const uint32_t s = __byte_perm(p[k], 0u, 0x1010), z = __byte_perm(p[k], 0u, 0x3232) | 0x43004300u;
            #pragma unroll
            for (int w = 0; w < 2; ++w) {
                uint32_t out[4];
                #pragma unroll
                for (int j = 0; j < 4; ++j) out[j] = mul_bf16x2(sub_bf16x2((c[k][w] >> (4 * j) & 0x000f000fu) | 0x43004300u, z), s);
                __stcs(reinterpret_cast<uint4*>(to[k]) + w * G, make_uint4(out[0], out[1], out[2], out[3]));
            }
        }
    }
}

static int32_t make_geo(const ss_kvq_rows* rows, const ss_kvq_cache* cache, KvqGeo* g) {
    if (!rows || !cache || (rows->max_rows > 0 && (!rows->k || !rows->v))) return SS_ERR_INVALID_ARG;
    const int32_t st = kvq_check_cache(*cache);
    if (st != SS_OK) return st;
    if (rows->batch < 1 || rows->batch > 65535 || rows->max_rows < 0 || rows->max_rows > 1 << 30 || cache->n_layers > 32767) return SS_ERR_INVALID_ARG;
    if ((rows->layer_stride | rows->batch_stride | rows->row_stride | rows->head_stride) & 7) return SS_ERR_UNSUPPORTED;
    if (!aligned16(rows->k) || !aligned16(rows->v)) return SS_ERR_INVALID_ARG;
    *g = KvqGeo{static_cast<unsigned char*>(cache->k_codes), static_cast<unsigned char*>(cache->v_codes), cache->k_params, cache->v_params,
                cache->layer_stride, cache->slot_stride, cache->head_stride, cache->param_layer_stride, cache->param_slot_stride,
                cache->param_head_stride, cache->total_slots, static_cast<unsigned char*>(rows->k), static_cast<unsigned char*>(rows->v),
                2 * rows->layer_stride, 2 * rows->batch_stride, 2 * rows->row_stride, 2 * rows->head_stride, cache->n_heads, rows->max_rows,
                cache->n_layers};
    return SS_OK;
}

// CTAs along x, for the longest run (the lengths are on the device).  The start of a CTA costs as much as several steps, so it gets
// eight of them before there are more (a user's accepted path into 32 layers and back 6.4 us; before, with one step each 10.7, two 8.2, eight 6.8);
// and where runs are long there are up to 32 CTAs per SM, eight times what is resident, so that the shorter runs' end early (the
// prompts of four users and back: up to 8 579 us, up to 32 480).  Sharing the sum of the runs out evenly was slower, whether each CTA
// took a stretch (550) or all went side by side (740): finding one's place and starting anew in every run costs more than it evens out.
static dim3 grid_for(const KvqGeo& g, int batch, long long max_rows, int head_dim) {
    const long long slots = head_dim == 128 ? Unit<128>::SLOTS : head_dim == 80 ? Unit<80>::SLOTS : Unit<64>::SLOTS, warps = kKvqThreads / 32;
    const long long chunks = ((max_rows + slots - 1) / slots * g.n_heads + warps - 1) / warps, planes = 2ll * g.layers * batch;
    const long long most = 32ll * sm_count() / planes;
    return dim3(static_cast<unsigned>(std::max(1ll, std::min((chunks + 7) / 8, most))), static_cast<unsigned>(2 * g.layers), static_cast<unsigned>(batch));
}

}  // namespace ss

extern "C" int32_t ss_kvq_write(const ss_kvq_rows* rows, const ss_kvq_cache* cache, const int64_t* kv_start, const int32_t* kv_len_in,
                                const int32_t* n_rows, const int32_t* path, const int32_t* kv_capacity, int32_t* kv_len_out,
                                void* status, void* stream) {
    ss::KvqGeo g;
    const int32_t st = ss::make_geo(rows, cache, &g);
    if (st != SS_OK) return st;
    if (!kv_start || !kv_len_in) return SS_ERR_INVALID_ARG;
    const size_t n = static_cast<size_t>(rows->batch);
    const auto overlaps_out = [&](const void* p, size_t bytes) {
        const uintptr_t out = reinterpret_cast<uintptr_t>(kv_len_out), in = reinterpret_cast<uintptr_t>(p);
        return p != nullptr && out < in + bytes && in < out + 4 * n;
    };
    const bool overlap = kv_len_out != nullptr && (overlaps_out(kv_len_in, 4 * n) || overlaps_out(n_rows, 4 * n) || overlaps_out(kv_start, 8 * n) ||
                                                   overlaps_out(path, 4 * n * SS_PATH_STRIDE) || overlaps_out(kv_capacity, 4 * n));
    if (overlap && rows->batch > 1024) return SS_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const auto kernel = cache->head_dim == 128 ? ss::kvq_write_kernel<128> : cache->head_dim == 80 ? ss::kvq_write_kernel<80> : ss::kvq_write_kernel<64>;
    const long long most = path != nullptr ? std::min<long long>(rows->max_rows, SS_PATH_STRIDE) : rows->max_rows;
    if (ss::launch_after_previous(kernel, ss::grid_for(g, rows->batch, most, cache->head_dim), dim3(ss::kKvqThreads), s, g, kv_start, kv_len_in,
                                  n_rows, path, kv_capacity, overlap ? nullptr : kv_len_out, status) != cudaSuccess)
        return SS_ERR_CUDA;
    if (!overlap) return SS_OK;
    return ss::launch_after_previous(ss::kvq_len_kernel, dim3(1), dim3((rows->batch + 31) / 32 * 32), s, g, kv_start, kv_len_in, n_rows,
                                     path, kv_capacity, kv_len_out, static_cast<int>(rows->batch)) == cudaSuccess ? SS_OK : SS_ERR_CUDA;
}

extern "C" int32_t ss_kvq_read(const ss_kvq_cache* cache, const ss_kvq_rows* rows, const int64_t* kv_start, const int32_t* first,
                               const int32_t* n_rows, void* stream) {
    ss::KvqGeo g;
    const int32_t st = ss::make_geo(rows, cache, &g);
    if (st != SS_OK) return st;
    if (!kv_start) return SS_ERR_INVALID_ARG;
    if (rows->max_rows == 0) return SS_OK;
    const auto kernel = cache->head_dim == 128 ? ss::kvq_read_kernel<128> : cache->head_dim == 80 ? ss::kvq_read_kernel<80> : ss::kvq_read_kernel<64>;
    return ss::launch_after_previous(kernel, ss::grid_for(g, rows->batch, rows->max_rows, cache->head_dim), dim3(ss::kKvqThreads),
                                     static_cast<cudaStream_t>(stream), g, kv_start, first, n_rows) == cudaSuccess
               ? SS_OK : SS_ERR_CUDA;
}
