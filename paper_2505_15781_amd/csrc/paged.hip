// Paged K/V cache: writing rows into its pages, quantised where the cache holds 8 bits, reading them back, and the boundary
// of these and of the attention over it (paged_attn.hip).
//
// Quantising. A row (one position, one K/V head) shares a power-of-two scale 2^e. e4m3 is a floating format, so a power of
// two costs no precision against a scale that brings the largest magnitude to exactly 448: each element is rounded
// once, to 4 significant bits, and x * 2^-e, code * 2^e are exact. In return the scale is 8 bits, scaled elements are exact in bf16
// (attention multiplies them as they are), and what is stored does not depend on how a division rounds. e is the smallest exponent with
// max |x| <= 448 * 2^e, from the bits of the maximum: with max |x| = m 2^E, m in [1, 2), it is E - 8, or E - 7 where m > 1.75.
// At least -110: the smallest code, 2^-9, is then 2^-119, so that every held element is a normal number of fp32 and bf16.
#include "paged.h"

namespace {

constexpr int kLowestExponent = -110, kHighestExponent = 120;

__device__ __forceinline__ int scale_exponent(float amax) {
    const uint32_t bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
    return min(max(e, kLowestExponent), kHighestExponent);
}

// 8 elements of a row whose DH elements lie in DH / 8 neighbouring lanes: writes their codes, and the scale in its first lane.
template <int DH>
__device__ __forceinline__ void store_piece(e4m3_t *row, uint8_t *scale, int piece, f32x8 x) {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = fabsf(x[i]);
        amax = fmaxf(amax, a < INFINITY ? a : 0.f);          // infinities and NaN count for nothing
    }
#pragma unroll
    for (int o = 1; o < DH / 8; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o, 64));
    const int e = scale_exponent(amax);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23), most = e == kHighestExponent ? 240.f : 448.f;
    u32x2 codes;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = fabsf(x[i]);
        x[i] = a < INFINITY ? fminf(fmaxf(x[i] * inv, -most), most) : __uint_as_float(0x7fc00000u);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
        codes[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], w, true);
    }
    *reinterpret_cast<u32x2 *>(row + 8 * piece) = codes;
    if (piece == 0) *scale = (uint8_t)(e + 127);
}
template <int DH>
__device__ __forceinline__ void store_piece(bf16_t *row, uint8_t *, int piece, f32x8 x) { store8(row + 8 * piece, x); }
template <int DH>
__device__ __forceinline__ void store_piece(float *row, uint8_t *, int piece, f32x8 x) { store8(row + 8 * piece, x); }

// One workgroup writes 256 pieces of 8 elements of one row of K and V: piece i is head i / (2 P), K or V, piece i % P of
// its head's P = DH / 8.
template <typename T, typename C, int DH>
__global__ __launch_bounds__(256) void paged_store_kernel(PagedCache c, const T *__restrict__ k_new, const T *__restrict__ v_new,
                                                          int64_t row_stride, const int *__restrict__ positions,
                                                          const int *__restrict__ row_off, int parts) {
    constexpr int P = DH / 8;
    const int r = blockIdx.x / parts, i = (blockIdx.x % parts) * 256 + threadIdx.x;
    const int b = sequence_of_row(row_off, c.batch, r);
    if (b >= c.batch) return;
    const int p = positions[r], page = c.page(b, p);
    if (page < 0 || i >= 2 * P * c.n_kv_heads) return;
    const int head = i / (2 * P), is_v = i / P % 2, piece = i % P;
    const uint32_t at = c.row(page, head, p & (c.page_size() - 1));
    const f32x8 x = load8((is_v ? v_new : k_new) + r * row_stride + head * DH + 8 * piece);
    store_piece<DH>(reinterpret_cast<C *>(is_v ? c.v : c.k) + (size_t)at * DH, (is_v ? c.vs : c.ks) + at, piece, x);
}

template <typename T, typename C, int DH>
__global__ __launch_bounds__(256) void paged_load_kernel(PagedCache c, T *__restrict__ k_out, T *__restrict__ v_out,
                                                         const int *__restrict__ positions, const int *__restrict__ row_off,
                                                         int parts) {
    constexpr int P = DH / 8;
    const int r = blockIdx.x / parts, i = (blockIdx.x % parts) * 256 + threadIdx.x;
    const int b = sequence_of_row(row_off, c.batch, r);
    if (b >= c.batch || i >= 2 * P * c.n_kv_heads) return;
    const int head = i / (2 * P), is_v = i / P % 2, piece = i % P;
    const int p = positions[r], page = c.page(b, p);
    f32x8 x = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (page >= 0) {
        const uint32_t at = c.row(page, head, p & (c.page_size() - 1));
        x = load8(reinterpret_cast<const C *>(is_v ? c.v : c.k) + (size_t)at * DH + 8 * piece);
        if (sizeof(C) == 1) x *= scale_value((is_v ? c.vs : c.ks)[at]);
    }
    store8((is_v ? v_out : k_out) + ((size_t)r * c.n_kv_heads + head) * DH + 8 * piece, x);
}

// Calls f(element type of the rows, of the cache, head_dim) for the combination at hand.
template <typename T> struct Type { typedef T type; };
template <int V> struct Size { static constexpr int value = V; };
template <typename F> int with_types(int dtype, int cache_dtype, int head_dim, F f) {
    auto heads = [&](auto t, auto c) {
        return head_dim == 32 ? f(t, c, Size<32>{}) : head_dim == 64 ? f(t, c, Size<64>{}) : f(t, c, Size<128>{});
    };
    auto caches = [&](auto t) {
        return cache_dtype == DKV_BF16 ? heads(t, Type<bf16_t>{}) : cache_dtype == DKV_FP32 ? heads(t, Type<float>{}) : heads(t, Type<e4m3_t>{});
    };
    return dtype == DKV_BF16 ? caches(Type<bf16_t>{}) : caches(Type<float>{});
}

}  // namespace

int dkv_paged_view(const dkv_paged_cache *c, PagedCache &view) {
    if (!c || !c->k_pages || !c->v_pages || !c->page_table) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    if (c->dtype != DKV_BF16 && c->dtype != DKV_FP32 && c->dtype != DKV_E4M3) { dkv_set_error("unknown cache dtype %d", c->dtype); return DKV_E_INVALID_ARG; }
    if (c->dtype == DKV_E4M3 && (!c->k_scale || !c->v_scale)) { dkv_set_error("an e4m3 cache needs k_scale and v_scale"); return DKV_E_INVALID_ARG; }
    if (c->batch < 1 || c->n_pages < 1 || c->max_pages < 1 || c->n_kv_heads < 1) { dkv_set_error("inconsistent sizes"); return DKV_E_INVALID_ARG; }
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) { dkv_set_error("head_dim %d not supported (32, 64, 128)", c->head_dim); return DKV_E_UNSUPPORTED; }
    if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) {
        dkv_set_error("page_size %d not supported (a power of two, 16 to 65536)", c->page_size); return DKV_E_UNSUPPORTED;
    }
    if ((int64_t)c->max_pages * c->page_size > 1 << 30) { dkv_set_error("the table covers more than 2^30 positions"); return DKV_E_UNSUPPORTED; }
    if ((int64_t)c->n_pages * c->n_kv_heads > (1ll << 32) / c->page_size) { dkv_set_error("more than 2^32 rows of keys in one cache"); return DKV_E_UNSUPPORTED; }
    if ((reinterpret_cast<uintptr_t>(c->k_pages) | reinterpret_cast<uintptr_t>(c->v_pages)) % 16) { dkv_set_error("pages must be 16-byte aligned"); return DKV_E_INVALID_ARG; }
    view = PagedCache{static_cast<unsigned char *>(c->k_pages), static_cast<unsigned char *>(c->v_pages), c->k_scale, c->v_scale,
                      c->page_table, c->seq_len, c->batch, c->n_pages, c->max_pages, __builtin_ctz((unsigned)c->page_size), c->n_kv_heads};
    return DKV_OK;
}

int dkv_paged_check_rows(const dkv_paged_cache &c, const int32_t *row_off, int32_t rows) {
    if (rows < 0) { dkv_set_error("inconsistent sizes"); return DKV_E_INVALID_ARG; }
    if (!row_off && rows != c.batch) { dkv_set_error("without row offsets there is one row per sequence: %d rows, %d sequences", rows, c.batch); return DKV_E_INVALID_ARG; }
    return DKV_OK;
}

namespace {
// what store and load have in common: the checks, and the workgroups of a row
int rows_call(const dkv_paged_cache *cache, PagedCache &view, const void *k, const void *v, const int32_t *positions,
              const int32_t *row_off, int32_t rows, int32_t dtype, int &parts) {
    int rc = dkv_paged_view(cache, view);
    if (rc || (rc = dkv_paged_check_rows(*cache, row_off, rows))) return rc;
    if (dtype != DKV_BF16 && dtype != DKV_FP32) { dkv_set_error("unknown dtype"); return DKV_E_INVALID_ARG; }
    if (rows > 0 && (!k || !v || !positions)) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    const int64_t per_row = (2 * (int64_t)(cache->head_dim / 8) * cache->n_kv_heads + 255) / 256;
    if (per_row * rows >= 1 << 24) { dkv_set_error("%d rows of %d heads are too many for one call", rows, cache->n_kv_heads); return DKV_E_UNSUPPORTED; }
    parts = (int)per_row;
    return DKV_OK;
}
}  // namespace

extern "C" int dkv_paged_store(const dkv_paged_cache *cache, const void *k_new, const void *v_new, int64_t row_stride,
                               const int32_t *positions, const int32_t *row_off, int32_t rows, int32_t dtype, void *stream) {
    PagedCache c;
    int parts;
    const int rc = rows_call(cache, c, k_new, v_new, positions, row_off, rows, dtype, parts);
    if (rc) return rc;
    if (row_stride < (int64_t)cache->n_kv_heads * cache->head_dim) { dkv_set_error("row stride %lld is less than a row", (long long)row_stride); return DKV_E_INVALID_ARG; }
    if (rows == 0) return DKV_OK;
    return with_types(dtype, cache->dtype, cache->head_dim, [&](auto t, auto ct, auto dh) {
        typedef typename decltype(t)::type T;
        typedef typename decltype(ct)::type C;
        hipLaunchKernelGGL((paged_store_kernel<T, C, decltype(dh)::value>), dim3((unsigned)(rows * parts)), dim3(256), 0,
                           static_cast<hipStream_t>(stream), c, (const T *)k_new, (const T *)v_new, row_stride, positions, row_off, parts);
        DKV_LAUNCH_CHECK();
        return DKV_OK;
    });
}

extern "C" int dkv_paged_load(const dkv_paged_cache *cache, void *k_out, void *v_out, const int32_t *positions,
                              const int32_t *row_off, int32_t rows, int32_t dtype, void *stream) {
    PagedCache c;
    int parts;
    const int rc = rows_call(cache, c, k_out, v_out, positions, row_off, rows, dtype, parts);
    if (rc) return rc;
    if (rows == 0) return DKV_OK;
    return with_types(dtype, cache->dtype, cache->head_dim, [&](auto t, auto ct, auto dh) {
        typedef typename decltype(t)::type T;
        typedef typename decltype(ct)::type C;
        hipLaunchKernelGGL((paged_load_kernel<T, C, decltype(dh)::value>), dim3((unsigned)(rows * parts)), dim3(256), 0,
                           static_cast<hipStream_t>(stream), c, (T *)k_out, (T *)v_out, positions, row_off, parts);
        DKV_LAUNCH_CHECK();
        return DKV_OK;
    });
}
