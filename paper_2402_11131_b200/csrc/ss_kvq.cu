// Rows into and out of a cache held in 4 bits (format and layout: ss_msa.h).  Compiled without fast-math: scales and codes are
// defined bit by bit.
//
// Both kernels stream: HBM bounds them.  A thread holds 16 values (32 bytes of bf16, 8 bytes of codes), so a row of a head is
// 4, 5 or 8 neighbouring lanes, which find the row's extremes with three exchanges.
//
// The arithmetic of the scale.  s is the smallest bf16 with 15 s >= hi - lo.  Directed rounding composes: a sum rounded up to
// fp32, its quotient rounded up to fp32 and that rounded up to bf16 is the exact quotient rounded up to bf16, because 15 s is
// itself an fp32 number.  (Everything is divided by 16 first, exactly, so that hi - lo does not overflow.)
// The arithmetic of the codes.  x and s have 8 significant bits, so x / s either lies exactly between two whole numbers or is at
// least 2^-13 of itself away from there (the midpoints are (2k + 1) / 2 with 2k + 1 <= 31, and 255 * 31 < 2^13).  x * (1 / s) with
// 1 / s enlarged by 2^-16 is off by less than that and on the far side of the midpoint where the quotient is exactly one, so that
// one fused multiply-add with 1.5 * 2^23, whose sum has no fraction bits left, rounds as if the quotient were exact.
#include <cuda_bf16.h>

#include "ss_common.cuh"

namespace ss {

constexpr int kKvqThreads = 256;
constexpr float kRoundMagic = 12582912.f;          // 1.5 * 2^23

struct KvqGeo {
    unsigned char *k_codes, *v_codes;
    uint32_t *k_params, *v_params;
    long long layer_stride, slot_stride, head_stride, p_layer, p_slot, p_head, total_slots;
    unsigned char *k_rows, *v_rows;                 // bf16; strides in bytes
    long long r_layer, r_batch, r_row, r_head;
    int n_heads, max_rows, layers;
};

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// x / s rounded to the nearest whole number, from the middle away from zero, as the low bits of the result (inv: 1 / s enlarged)
__device__ __forceinline__ uint32_t rounded_bits(float x, float inv) { return __float_as_uint(__fmaf_rn(x, inv, kRoundMagic)); }

// A row of D values over D / 16 neighbouring lanes, 16 values each: returns the row's word of scale and zero point and this lane's
// 16 codes.  All 32 lanes take part; `base` is the first lane of the row, `at` this lane's place in it.
template <int D>
__device__ __forceinline__ uint32_t quantise_row(const uint4 (&x)[2], int base, int at, uint2* codes) {
    constexpr int G = D / 16;
    const uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    // largest value and largest negated value, with zero among them; bits of the largest magnitude
    uint32_t hi2 = 0u, lo2 = 0u, mag = 0u;
    #pragma unroll
    for (int i = 0; i < 8; ++i) {
        hi2 = max_bf16x2(hi2, w[i]);
        lo2 = max_bf16x2(lo2, w[i] ^ 0x80008000u);
        mag = __vmaxu2(mag, w[i] & 0x7fff7fffu);
    }
    uint32_t ext = max_bf16x2(__byte_perm(hi2, lo2, 0x5410), __byte_perm(hi2, lo2, 0x7632));    // low half: hi, high half: -lo
    mag = max(mag & 0xffffu, mag >> 16);
    #pragma unroll
    for (int step = 0; step < 3; ++step) {
        const int shift = step == 0 ? 1 : step == 1 ? 2 : (G == 8 ? 4 : 1);     // (after 1 + 2 + 1 a lane has seen all of 4 or 5)
        int from = at + shift;
        if (from >= G) from -= G;
        ext = max_bf16x2(ext, __shfl_sync(0xffffffffu, ext, base + from));
        mag = max(mag, __shfl_sync(0xffffffffu, mag, base + from));
    }
    const float hi = __uint_as_float(ext << 16), nlo = __uint_as_float(ext & 0xffff0000u);
    const float up = __fdiv_ru(__fadd_ru(hi * 0.0625f, nlo * 0.0625f), 0.9375f);
    uint32_t sb = (__float_as_uint(up) + 0xffffu) >> 16;          // (up is not negative)
    sb = max(sb, 0x0380u);                                        // 2^-120
    const float s = __uint_as_float(sb << 16);
    const float inv = __fmul_rn(__frcp_rn(s), 1.0000152587890625f);
    const bool bad = mag >= 0x7f80u;                              // an infinity or a NaN in the row
    const uint32_t z = bad ? 0u : (rounded_bits(nlo, inv) & 0xfu);   // (at most 15: nlo <= 15 s)
    // rounded(x / s) + z in the low bits of 1.5 * 2^23 + .., clamped as an fp32 number
    const float zf = static_cast<float>(z), top = kRoundMagic + 15.f;
    uint32_t c[16];
    #pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = __uint_as_float(rounded_bits(__uint_as_float(w[i] << 16), inv)) + zf;
        const float b = __uint_as_float(rounded_bits(__uint_as_float(w[i] & 0xffff0000u), inv)) + zf;
        c[2 * i] = __float_as_uint(fminf(fmaxf(a, kRoundMagic), top)) & 0xfu;
        c[2 * i + 1] = __float_as_uint(fminf(fmaxf(b, kRoundMagic), top)) & 0xfu;
    }
    uint32_t out[2];
    #pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t v = 0u;
        #pragma unroll
        for (int i = 0; i < 4; ++i) v |= (c[8 * h + 2 * i] << (4 * i)) | (c[8 * h + 2 * i + 1] << (16 + 4 * i));
        out[h] = bad ? 0u : v;
    }
    *codes = make_uint2(out[0], out[1]);
    return (bad ? 0x7fffu : sb) | (z << 16);
}

// The sequence's run of rows: from slot `*slot0`, `*n` of them (0: nothing to do).  Returns false where they do not fit.
__device__ __forceinline__ bool write_run(const KvqGeo& g, const int64_t* kv_start, const int32_t* kv_len_in, const int32_t* n_rows,
                                          const int32_t* path, const int32_t* kv_capacity, int b, long long* slot0, int* n, int* L) {
    const int limit = path != nullptr ? SS_PATH_STRIDE : g.max_rows;
    *L = kv_len_in[b];
    *n = n_rows != nullptr ? max(0, min(n_rows[b], limit)) : min(g.max_rows, limit);
    *slot0 = kv_start[b] + *L;
    const bool fits = *L >= 0 && *slot0 >= 0 && *slot0 + *n <= g.total_slots &&
                      (kv_capacity == nullptr || static_cast<long long>(*L) + *n <= kv_capacity[b]);
    return fits;
}

template <int D>
__global__ void __launch_bounds__(kKvqThreads)
kvq_write_kernel(const __grid_constant__ KvqGeo g, const int64_t* __restrict__ kv_start, const int32_t* __restrict__ kv_len_in,
                 const int32_t* __restrict__ n_rows, const int32_t* __restrict__ path, const int32_t* __restrict__ kv_capacity,
                 int32_t* __restrict__ kv_len_out, void* __restrict__ status) {
    constexpr int G = D / 16, ROWS = 32 / G, WARPS = kKvqThreads / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = min(lane / G, ROWS - 1), base = sub * G, at = lane < ROWS * G ? lane - base : 0;
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
    const unsigned char* rows = (is_v ? g.v_rows : g.k_rows) + layer * g.r_layer + b * g.r_batch;
    unsigned char* codes = (is_v ? g.v_codes : g.k_codes) + layer * g.layer_stride + slot0 * g.slot_stride;
    uint32_t* params = (is_v ? g.v_params : g.k_params) + layer * g.p_layer + slot0 * g.p_slot;
    const long long items = static_cast<long long>(n) * g.n_heads, step = static_cast<long long>(gridDim.x) * WARPS * ROWS;
    for (long long i0 = (static_cast<long long>(blockIdx.x) * WARPS + warp) * ROWS; i0 < items; i0 += step) {
        const long long i = i0 + sub;
        const int r = static_cast<int>(i / g.n_heads), h = static_cast<int>(i - static_cast<long long>(r) * g.n_heads);
        int src = r;
        if (path != nullptr && i < items) src = path[static_cast<long long>(b) * SS_PATH_STRIDE + r];
        const bool live = i < items && lane < ROWS * G && src >= 0 && src < g.max_rows;
        uint4 x[2] = {};
        if (live) {
            const uint4* p = reinterpret_cast<const uint4*>(rows + src * g.r_row + h * g.r_head) + 2 * at;
            x[0] = __ldcs(p);
            x[1] = __ldcs(p + 1);
        }
        uint2 c;
        const uint32_t word = quantise_row<D>(x, base, at, &c);
        if (live) {
            *reinterpret_cast<uint2*>(codes + r * g.slot_stride + h * g.head_stride + 8 * at) = c;
            if (at == 0) params[r * g.p_slot + h * g.p_head] = word;
        }
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

__device__ __forceinline__ uint32_t pack_values(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

template <int D>
__global__ void __launch_bounds__(kKvqThreads)
kvq_read_kernel(const __grid_constant__ KvqGeo g, const int64_t* __restrict__ kv_start, const int32_t* __restrict__ first,
                const int32_t* __restrict__ n_rows) {
    constexpr int G = D / 16, ROWS = kKvqThreads / G;
    const int sub = threadIdx.x / G, at = threadIdx.x - sub * G;
    const int layer = blockIdx.y >> 1, b = blockIdx.z;
    const bool is_v = blockIdx.y & 1;
    wait_for_previous_kernel();
    release_next_kernel();
    const int n = n_rows != nullptr ? min(n_rows[b], g.max_rows) : g.max_rows;
    const long long slot0 = kv_start[b] + (first != nullptr ? first[b] : 0);
    const unsigned char* codes = (is_v ? g.v_codes : g.k_codes) + layer * g.layer_stride;
    const uint32_t* params = (is_v ? g.v_params : g.k_params) + layer * g.p_layer;
    unsigned char* rows = (is_v ? g.v_rows : g.k_rows) + layer * g.r_layer + b * g.r_batch;
    if (sub >= ROWS) return;
    const long long items = static_cast<long long>(max(n, 0)) * g.n_heads, step = static_cast<long long>(gridDim.x) * ROWS;
    for (long long i = static_cast<long long>(blockIdx.x) * ROWS + sub; i < items; i += step) {
        const int r = static_cast<int>(i / g.n_heads), h = static_cast<int>(i - static_cast<long long>(r) * g.n_heads);
        const long long slot = slot0 + r;
        if (slot < 0 || slot >= g.total_slots) continue;
        const uint2 c = __ldcs(reinterpret_cast<const uint2*>(codes + slot * g.slot_stride + h * g.head_stride + 8 * at));
        const uint32_t p = params[slot * g.p_slot + h * g.p_head];
        const float s = __uint_as_float(p << 16);
        const int z = (p >> 16) & 0xf;
        uint32_t out[8];
        #pragma unroll
        for (int w = 0; w < 2; ++w) {
            const uint32_t v = w ? c.y : c.x;
            #pragma unroll
            for (int j = 0; j < 4; ++j)
                out[4 * w + j] = pack_values(s * static_cast<float>(static_cast<int>((v >> (4 * j)) & 0xf) - z),
                                             s * static_cast<float>(static_cast<int>((v >> (16 + 4 * j)) & 0xf) - z));
        }
        uint4* dst = reinterpret_cast<uint4*>(rows + r * g.r_row + h * g.r_head) + 2 * at;
        __stcs(dst, make_uint4(out[0], out[1], out[2], out[3]));
        __stcs(dst + 1, make_uint4(out[4], out[5], out[6], out[7]));
    }
}

static int32_t make_geo(const ss_kvq_rows* rows, const ss_kvq_cache* cache, KvqGeo* g) {
    if (!rows || !cache || (rows->max_rows > 0 && (!rows->k || !rows->v))) return SS_ERR_INVALID_ARG;
    const int32_t st = kvq_check_cache(*cache);
    if (st != SS_OK) return st;
    if (rows->batch < 1 || rows->batch > 65535 || rows->max_rows < 0 || cache->n_layers > 32767) return SS_ERR_INVALID_ARG;
    if ((rows->layer_stride | rows->batch_stride | rows->row_stride | rows->head_stride) & 7) return SS_ERR_UNSUPPORTED;
    if (!aligned16(rows->k) || !aligned16(rows->v)) return SS_ERR_INVALID_ARG;
    *g = KvqGeo{static_cast<unsigned char*>(cache->k_codes), static_cast<unsigned char*>(cache->v_codes), cache->k_params, cache->v_params,
                cache->layer_stride, cache->slot_stride, cache->head_stride, cache->param_layer_stride, cache->param_slot_stride,
                cache->param_head_stride, cache->total_slots, static_cast<unsigned char*>(rows->k), static_cast<unsigned char*>(rows->v),
                2 * rows->layer_stride, 2 * rows->batch_stride, 2 * rows->row_stride, 2 * rows->head_stride, cache->n_heads, rows->max_rows,
                cache->n_layers};
    return SS_OK;
}

// CTAs along x: enough for the longest run (the lengths are on the device), at most some sixteen CTAs per SM in all
static dim3 grid_for(const KvqGeo& g, int batch, long long max_rows, int per_cta) {
    const long long want = (max_rows * g.n_heads + per_cta - 1) / per_cta, others = 2ll * g.layers * batch;
    const long long most = std::max(1ll, 16ll * sm_count() / others);
    return dim3(static_cast<unsigned>(std::max(1ll, std::min(want, most))), static_cast<unsigned>(2 * g.layers), static_cast<unsigned>(batch));
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
    const int per_cta = ss::kKvqThreads / 32 * (32 / (cache->head_dim / 16));
    const long long most = path != nullptr ? std::min<long long>(rows->max_rows, SS_PATH_STRIDE) : rows->max_rows;
    if (ss::launch_after_previous(kernel, ss::grid_for(g, rows->batch, most, per_cta), dim3(ss::kKvqThreads), s, g, kv_start, kv_len_in,
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
    const int per_cta = ss::kKvqThreads / (cache->head_dim / 16);
    return ss::launch_after_previous(kernel, ss::grid_for(g, rows->batch, rows->max_rows, per_cta), dim3(ss::kKvqThreads),
                                     static_cast<cudaStream_t>(stream), g, kv_start, first, n_rows) == cudaSuccess ? SS_OK : SS_ERR_CUDA;
}
