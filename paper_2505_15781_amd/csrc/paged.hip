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

template <typename T> struct Type { typedef T type; };
template <int V> struct Size { static constexpr int value = V; };

constexpr int kLowestExponent = -110, kHighestExponent = 120;

__device__ __forceinline__ int scale_exponent(float amax) {
    const uint32_t bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
    return min(max(e, kLowestExponent), kHighestExponent);
}

// Elements of a lane: 16 bytes of what is written.
template <typename W> constexpr int kPiece = 16 / (int)sizeof(W);
template <int N> using Piece = float __attribute__((ext_vector_type(N)));

__device__ __forceinline__ Piece<4> load_piece(const float *p, Piece<4> *) { return *reinterpret_cast<const f32x4_el *>(p); }
__device__ __forceinline__ Piece<4> load_piece(const bf16_t *p, Piece<4> *) {
    const u32x2 a = *reinterpret_cast<const bf16x4_el *>(p);
    return Piece<4>{__uint_as_float(a.x << 16), __uint_as_float(a.x & 0xffff0000u), __uint_as_float(a.y << 16), __uint_as_float(a.y & 0xffff0000u)};
}
__device__ __forceinline__ Piece<4> load_piece(const e4m3_t *p, Piece<4> *) {
    const uint32_t a = *reinterpret_cast<const uint32_t *>(p);
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(a, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(a, true);
    return Piece<4>{lo[0], lo[1], hi[0], hi[1]};
}
template <typename T> __device__ __forceinline__ Piece<8> load_piece(const T *p, Piece<8> *) { return load8(p); }
template <typename T> __device__ __forceinline__ Piece<16> load_piece(const T *p, Piece<16> *) {
    return __builtin_shufflevector(load8(p), load8(p + 8), 0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15);
}
__device__ __forceinline__ void store_piece(float *p, Piece<4> x) { *reinterpret_cast<f32x4_el *>(p) = x; }
__device__ __forceinline__ void store_piece(bf16_t *p, Piece<8> x) { store8(p, x); }

// Maximum over the 2, 4 or 8 neighbouring lanes that hold a row.
template <int LANES> __device__ __forceinline__ float row_max(float x) {
    auto other = [&](auto control) {
        return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(control)::value, 0xf, 0xf, true));
    };
    x = fmaxf(x, other(Size<0xB1>{}));                               // lane ^ 1
    if (LANES > 2) x = fmaxf(x, other(Size<0x4E>{}));                // lane ^ 2
    if (LANES > 4) x = fmaxf(x, other(Size<0x141>{}));               // mirrored within 8 lanes
    return x;
}

// Writes the elements of a lane into the cache (e4m3: with the rest of the row in the lanes beside it).
template <int DH> __device__ __forceinline__ void put(bf16_t *row, uint8_t *, int piece, Piece<8> x) { store_piece(row + 8 * piece, x); }
template <int DH> __device__ __forceinline__ void put(float *row, uint8_t *, int piece, Piece<4> x) { store_piece(row + 4 * piece, x); }
template <int DH> __device__ __forceinline__ void put(e4m3_t *row, uint8_t *scale, int piece, Piece<16> x) {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float a = fabsf(x[i]);
        amax = fmaxf(amax, a < INFINITY ? a : 0.f);          // infinities and NaN count for nothing
    }
    const int e = scale_exponent(row_max<DH / 16>(amax));
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23), most = e == kHighestExponent ? 240.f : 448.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = fabsf(x[i]) < INFINITY ? fminf(fmaxf(x[i] * inv, -most), most) : __uint_as_float(0x7fc00000u);
    u32x4 codes;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
        codes[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], w, true);
    }
    *reinterpret_cast<u32x4 *>(row + 16 * piece) = codes;
    if (piece == 0) *scale = (uint8_t)(e + 127);
}

// Which row a wavefront works on, and where that row's place in the cache is: N pieces of a lane, 64 apart; piece i of a row is head
// i / (2 P), K or V, piece i % P of its head's P.
struct RowWork {
    int r, first;                      // row, piece of this lane
    template <int N> __device__ __forceinline__ static RowWork of_wavefront(Divisor waves) {
        const int id = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        return RowWork{waves.div(id), waves.mod(id) * (64 * N) + (int)(threadIdx.x & 63)};
    }
    // false where the row belongs to no sequence; page: -1 if there is none
    __device__ __forceinline__ bool place(const PagedCache &c, const int *positions, const int *row_off, int rows, int &page, int &slot) const {
        if (r >= rows) return false;
        const int p = positions[r], b = sequence_of_row(row_off, c.batch, r);
        if (b >= c.batch) return false;
        page = c.page(b, p);
        slot = p & (c.page_size() - 1);
        return true;
    }
};

// A lane writes 16 bytes. It loads its elements before the row's place is known: many rows are bound by the traffic, few by the chain
// of offsets, page number and store. 6144 rows of 32 heads of 128 from bf16 into e4m3 31 us (4.8 TB/s; a large copy 4.45), into bf16 39
// (5.1), from fp32 into fp32 71 (5.7), 64 rows 2.8 us. Four pieces of a lane at once gain nothing here and lose up to 45 % with few rows.
template <typename T, typename C, int DH>
__global__ __launch_bounds__(256) void paged_store_kernel(PagedCache c, const T *__restrict__ k_new, const T *__restrict__ v_new,
                                                          int64_t row_stride, const int *__restrict__ positions,
                                                          const int *__restrict__ row_off, int rows, Divisor waves) {
    constexpr int E = kPiece<C>, P = DH / E;
    const RowWork w = RowWork::of_wavefront<1>(waves);
    const int pieces = 2 * P * c.n_kv_heads, i = min(w.first, pieces - 1), head = i / (2 * P), is_v = i / P % 2, piece = i % P;
    const Piece<E> x = load_piece((is_v ? v_new : k_new) + min(w.r, rows - 1) * row_stride + head * DH + E * piece, (Piece<E> *)nullptr);
    int page, slot;
    if (!w.place(c, positions, row_off, rows, page, slot) || page < 0 || w.first >= pieces) return;
    const uint32_t at = c.row(page, head, slot);
    put<DH>(reinterpret_cast<C *>(is_v ? c.v : c.k) + (size_t)at * DH, (is_v ? c.vs : c.ks) + at, piece, x);
}

// A lane writes N times 16 bytes. Its loads are short where the cache is e4m3 (8 bytes for bf16 rows, 4 for fp32), and wait for the
// row's place: with many rows four at once are ahead, 16384 rows of 32 heads 87 us against 105, 64 rows 3.2 against 2.5. They meet at
// 4096 wavefronts of four pieces a lane (32 heads of 128 to bf16: 512 rows 5.6 against 4.9, 1024 rows 7.3 and 7.5, 2048 rows 14.2 and 16.4; 8 heads of 64 to fp32,
// 4096 rows 6.6 and 7.3). From bf16 and fp32 caches one is. 6144 rows from e4m3 to bf16 35 us (4.3 TB/s), from bf16 to bf16 42 (4.8), to fp32 75 (4.0), from fp32
// to fp32 72 (5.6).
template <typename T, typename C, int DH, int N>
__global__ __launch_bounds__(256) void paged_load_kernel(PagedCache c, T *__restrict__ k_out, T *__restrict__ v_out,
                                                         const int *__restrict__ positions, const int *__restrict__ row_off, int rows,
                                                         Divisor waves) {
    constexpr int E = kPiece<T>, P = DH / E;
    const RowWork w = RowWork::of_wavefront<N>(waves);
    int page, slot;
    if (!w.place(c, positions, row_off, rows, page, slot)) return;
    const int pieces = 2 * P * c.n_kv_heads;
    Piece<E> x[N];
    float scale[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int i = min(w.first + 64 * u, pieces - 1), is_v = i / P % 2;
        const uint32_t at = c.row(max(page, 0), i / (2 * P), slot);
        x[u] = load_piece(reinterpret_cast<const C *>(is_v ? c.v : c.k) + (size_t)at * DH + E * (i % P), (Piece<E> *)nullptr);
        scale[u] = 1.f;
        if constexpr (sizeof(C) == 1) scale[u] = scale_value((is_v ? c.vs : c.ks)[at]);
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int i = w.first + 64 * u;
        if (i >= pieces) return;
        if constexpr (sizeof(C) == 1) x[u] *= scale[u];
        if (page < 0) x[u] = 0.f;
        store_piece((i / P % 2 ? v_out : k_out) + ((size_t)w.r * c.n_kv_heads + i / (2 * P)) * DH + E * (i % P), x[u]);
    }
}

// Calls f(element type of the rows, of the cache, head_dim) for the combination at hand.
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
    if ((int64_t)c->n_kv_heads * c->head_dim >= 1ll << 31) { dkv_set_error("rows of 2^31 elements and more are not supported"); return DKV_E_UNSUPPORTED; }
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
// What store and load refuse alike, and their launch: f(workgroups, wavefronts of a row), `n` pieces of 16 bytes of `written` type to a lane.
int rows_call(const dkv_paged_cache *cache, PagedCache &view, const void *k, const void *v, const int32_t *positions,
              const int32_t *row_off, int32_t rows, int32_t dtype) {
    int rc = dkv_paged_view(cache, view);
    if (rc || (rc = dkv_paged_check_rows(*cache, row_off, rows))) return rc;
    if (dtype != DKV_BF16 && dtype != DKV_FP32) { dkv_set_error("unknown dtype"); return DKV_E_INVALID_ARG; }
    if (rows > 0 && (!k || !v || !positions)) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    return DKV_OK;
}
int64_t row_pieces(const dkv_paged_cache &c, int written) {
    return 2 * (int64_t)(c.head_dim * (written == DKV_BF16 ? 2 : written == DKV_FP32 ? 4 : 1) / 16) * c.n_kv_heads;
}
template <typename F> int rows_launch(const dkv_paged_cache &c, int written, int n, int rows, F f) {
    const int64_t waves = (row_pieces(c, written) + 64 * n - 1) / (64 * n), groups = (waves * rows + 3) / 4;
    if (rows >= 1 << 24 || groups >= 1 << 23) { dkv_set_error("%d rows of %d heads are too many for one call", rows, c.n_kv_heads); return DKV_E_UNSUPPORTED; }
    return rows == 0 ? DKV_OK : f((unsigned)groups, Divisor((int)waves));
}
}  // namespace

extern "C" int dkv_paged_store(const dkv_paged_cache *cache, const void *k_new, const void *v_new, int64_t row_stride,
                               const int32_t *positions, const int32_t *row_off, int32_t rows, int32_t dtype, void *stream) {
    PagedCache c;
    const int rc = rows_call(cache, c, k_new, v_new, positions, row_off, rows, dtype);
    if (rc) return rc;
    if (row_stride < (int64_t)cache->n_kv_heads * cache->head_dim) { dkv_set_error("row stride %lld is less than a row", (long long)row_stride); return DKV_E_INVALID_ARG; }
    return rows_launch(*cache, cache->dtype, 1, rows, [&](unsigned groups, Divisor waves) {
        return with_types(dtype, cache->dtype, cache->head_dim, [&](auto t, auto ct, auto dh) {
            typedef typename decltype(t)::type T;
            typedef typename decltype(ct)::type C;
            hipLaunchKernelGGL((paged_store_kernel<T, C, decltype(dh)::value>), dim3(groups), dim3(256), 0,
                               static_cast<hipStream_t>(stream), c, (const T *)k_new, (const T *)v_new, row_stride, positions, row_off, rows, waves);
            DKV_LAUNCH_CHECK();
            return DKV_OK;
        });
    });
}

extern "C" int dkv_paged_load(const dkv_paged_cache *cache, void *k_out, void *v_out, const int32_t *positions,
                              const int32_t *row_off, int32_t rows, int32_t dtype, void *stream) {
    PagedCache c;
    const int rc = rows_call(cache, c, k_out, v_out, positions, row_off, rows, dtype);
    if (rc) return rc;
    const int n = cache->dtype == DKV_E4M3 && rows * ((row_pieces(*cache, dtype) + 255) / 256) >= 4096 ? 4 : 1;
    return rows_launch(*cache, dtype, n, rows, [&](unsigned groups, Divisor waves) {
        return with_types(dtype, cache->dtype, cache->head_dim, [&](auto t, auto ct, auto dh) {
            typedef typename decltype(t)::type T;
            typedef typename decltype(ct)::type C;
            auto launch = [&](auto pieces) {
                hipLaunchKernelGGL((paged_load_kernel<T, C, decltype(dh)::value, decltype(pieces)::value>), dim3(groups), dim3(256), 0,
                                   static_cast<hipStream_t>(stream), c, (T *)k_out, (T *)v_out, positions, row_off, rows, waves);
                DKV_LAUNCH_CHECK();
                return DKV_OK;
            };
            if constexpr (sizeof(C) == 1) return n == 4 ? launch(Size<4>{}) : launch(Size<1>{});
            else return launch(Size<1>{});
        });
    });
}
