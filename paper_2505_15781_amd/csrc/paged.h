// The paged K/V cache as its kernels see it (see dkv_paged_cache in dkv.h), and what they share.
#pragma once
#include "common.h"

struct PagedCache {
    unsigned char *k, *v;             // [n_pages][n_kv_heads][page_size][head_dim]
    uint8_t *ks, *vs;                 // [n_pages][n_kv_heads][page_size], e4m3 only
    const int *table, *seq_len;
    int batch, n_pages, max_pages, page_shift, n_kv_heads;

    __device__ __forceinline__ int page_size() const { return 1 << page_shift; }
    __device__ __forceinline__ int capacity() const { return max_pages << page_shift; }
    // page of a position of sequence b, -1 if there is none
    __device__ __forceinline__ int page(int b, int p) const {
        if ((unsigned)p >= (unsigned)capacity()) return -1;
        const int id = table[(size_t)b * max_pages + (p >> page_shift)];
        return (unsigned)id < (unsigned)n_pages ? id : -1;
    }
    // index of a (page, head, slot) row: times head_dim elements, or itself in the scales. A cache has at most 2^32 rows.
    __device__ __forceinline__ uint32_t row(int page, int head, int slot) const {
        return (((uint32_t)page * n_kv_heads + head) << page_shift) + slot;
    }
    __device__ __forceinline__ int keys(int b) const { return max(0, min(seq_len[b], capacity())); }
};

// Division by a number that the host knows: x / d = x * mul >> (31 + l) for 0 <= x < 2^31, with 2^(l - 1) < d <= 2^l and mul = 2^(31 + l) / d
// rounded up: the excess of mul * d over 2^(31 + l) is less than 2^l, so that x times it stays below 2^(31 + l).
struct Divisor {
    int d;
    uint32_t mul;
    int shift;
    __host__ explicit Divisor(int d_ = 1) : d(d_) {
        int l = 0;
        while ((1ll << l) < d) ++l;
        shift = 31 + l;
        mul = (uint32_t)(((1ull << shift) + d - 1) / d);
    }
    __device__ __forceinline__ int div(int x) const { return (int)((uint64_t)(uint32_t)x * mul >> shift); }
    __device__ __forceinline__ int mod(int x) const { return x - div(x) * d; }
};

typedef uint8_t e4m3_t;      // a code; its row's scale is a biased exponent

// Value of a scale: a normal number for the exponents that a store writes (-110 to 120).
__device__ __forceinline__ float scale_value(uint8_t biased) { return __uint_as_float((uint32_t)biased << 23); }

// Sequence of row r: the number of i with row_off[i + 1] <= r, `batch` for rows behind the last sequence. Called by whole
// wavefronts with r uniform; a lane per sequence, so that batches of up to 64 cost one load instead of a search's chain.
__device__ __forceinline__ int sequence_of_row(const int *row_off, int batch, int r) {
    if (!row_off) return r < batch ? r : batch;
    const int lane = threadIdx.x & 63;
    int b = 0;
    for (int i = 0; i < batch; i += 64) {
        const int n = __popcll(__ballot(i + lane < batch && row_off[min(i + lane, batch - 1) + 1] <= r));
        b += n;
        if (n < 64) break;
    }
    return b;
}

// First row and number of rows of sequence b.
__device__ __forceinline__ void rows_of_sequence(const int *row_off, int b, int &r0, int &n) {
    r0 = row_off ? row_off[b] : b;
    n = row_off ? row_off[b + 1] - r0 : 1;
}

// 8 consecutive elements as floats, at any address that is aligned to an element.
__device__ __forceinline__ f32x8 load8(const float *p) {
    const f32x4 a = *reinterpret_cast<const f32x4_el *>(p), b = *reinterpret_cast<const f32x4_el *>(p + 4);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f32x8 load8(const bf16_t *p) {
    const u32x4 a = *reinterpret_cast<const bf16x8_el *>(p);
    f32x8 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(a[i] << 16);
        x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
    return x;
}
// 8 codes times 1
__device__ __forceinline__ f32x8 load8(const e4m3_t *p) {
    const u32x2 a = *reinterpret_cast<const u32x2 *>(p);
    f32x8 x;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(a[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(a[i], true);
        x[4 * i] = lo[0];
        x[4 * i + 1] = lo[1];
        x[4 * i + 2] = hi[0];
        x[4 * i + 3] = hi[1];
    }
    return x;
}
__device__ __forceinline__ void store8(float *p, f32x8 x) {
    *reinterpret_cast<f32x4_el *>(p) = __builtin_shufflevector(x, x, 0, 1, 2, 3);
    *reinterpret_cast<f32x4_el *>(p + 4) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
}
__device__ __forceinline__ void store8(bf16_t *p, f32x8 x) {
    u32x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (uint32_t)f2bf(x[2 * i]) | ((uint32_t)f2bf(x[2 * i + 1]) << 16);
    *reinterpret_cast<bf16x8_el *>(p) = y;
}

// ---- host side ----
// Checks what every entry point asks of a cache and fills the kernels' view of it; an error code else.
int dkv_paged_view(const dkv_paged_cache *cache, PagedCache &view);
// Rows and row offsets as the entry points take them; `rows` > 0 on success says that there is work.
int dkv_paged_check_rows(const dkv_paged_cache &cache, const int32_t *row_off, int32_t rows);

// What a call of attention is routed to.
struct PagedAttnPlan {
    int nq, q_groups;       // query tiles of 16 rows per workgroup, groups of them
    int wide;               // 0: paged_attn_split; paged_attn_wide: groups of wavefronts in a workgroup
    int blocks;             // blocks of 128 query rows over all K/V heads at most: the workgroups of paged_attn_wide without slices
    int cap;                // slices of the whole batch at most
    int spread;             // log2 of the XCDs that the query groups of one (slice, K/V head) are on
    int least, want;        // see SlicePlan
    bool split;             // whether a sequence can have several slices
};
// What both entry points of the attention refuse, and the plan of what they do not.
int dkv_paged_attn_plan(const dkv_paged_cache *cache, PagedCache &view, PagedAttnPlan &plan, int n_q_heads, int rows, int max_rows_per_seq,
                        int dtype);
