// Attention of new rows over a paged K/V cache.
//
// One wavefront per (row, query head): a lane per key of a chunk of 64 for the scores, a lane per DH / 64 output dims for the
// products with V; one pass with the running maximum and sum of the softmax, fp32 throughout.
#include <math.h>

#include "paged.h"

namespace {

constexpr float kLowest = -3.0e38f;    // start of a running maximum: finite, so that a score of -infinity has probability zero

template <typename T, typename C, int DH>
__global__ __launch_bounds__(256) void paged_attn_simple(PagedCache c, const T *__restrict__ Q, int64_t q_stride,
                                                         const int *__restrict__ row_off, T *__restrict__ out, int rows,
                                                         int max_rows, int Hq, float scale_log2e) {
    constexpr int ND = DH < 64 ? 1 : DH / 64;
    const int lane = threadIdx.x & 63;
    const int64_t pair = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (pair >= (int64_t)rows * Hq) return;
    const int r = (int)(pair / Hq), h = (int)(pair % Hq), b = sequence_of_row(row_off, c.batch, r);
    if (b >= c.batch) return;
    int r0, n;
    rows_of_sequence(row_off, b, r0, n);
    if (r - r0 >= max_rows) return;
    const int kvh = h / (Hq / c.n_kv_heads), len = c.keys(b);
    const T *q = Q + r * q_stride + h * DH;
    const C *K = reinterpret_cast<const C *>(c.k), *V = reinterpret_cast<const C *>(c.v);
    float m = kLowest, l = 0.f, o[ND] = {};
    for (int k0 = 0; k0 < len; k0 += 64) {
        const int p = k0 + lane, page = p < len ? c.page(b, p) : -1;
        const size_t at = c.row(max(page, 0), kvh, p & (c.page_size() - 1));
        float s = -INFINITY;
        if (page >= 0) {
            s = 0.f;
            for (int d = 0; d < DH; d += 8) {
                const f32x8 x = load8(K + at * DH + d), y = load8(q + d);
                for (int i = 0; i < 8; ++i) s = fmaf(x[i], y[i], s);
            }
            s *= scale_log2e;
            if (sizeof(C) == 1) s *= scale_value(c.ks[at]);
        }
        const float mn = fmaxf(m, wave_max(s)), alpha = exp2f(m - mn);
        const float pr = exp2f(s - mn);
        l = l * alpha + wave_sum(pr);
        m = mn;
        for (int i = 0; i < ND; ++i) o[i] *= alpha;
        for (int j = 0; j < min(64, len - k0); ++j) {
            if (__shfl(page, j, 64) < 0) continue;
            const float w = __shfl(pr, j, 64);
            const size_t row = c.row(__shfl(page, j, 64), kvh, (k0 + j) & (c.page_size() - 1));
            for (int i = 0; i < ND; ++i) {
                const int d = lane + 64 * i;
                if (d >= DH) continue;
                float v;
                if constexpr (sizeof(C) == 1) v = __builtin_amdgcn_cvt_f32_fp8(V[row * DH + d], 0) * scale_value(c.vs[row]);
                else v = El<C>::ld(V + row * DH + d);
                o[i] = fmaf(w, v, o[i]);
            }
        }
    }
    for (int i = 0; i < ND; ++i)
        if (lane + 64 * i < DH) El<T>::st(out + (size_t)pair * DH + lane + 64 * i, l == 0.f ? 0.f : o[i] / l);
}

template <typename T, typename C>
int launch_simple(const PagedCache &c, int dh, const void *q, int64_t q_stride, const int *row_off, void *out, int rows, int max_rows,
                  int Hq, hipStream_t s) {
    const float scale_log2e = 1.4426950408889634f / sqrtf((float)dh);
    const unsigned grid = (unsigned)(((int64_t)rows * Hq + 3) / 4);
#define SIMPLE(D)                                                                                                          \
    hipLaunchKernelGGL((paged_attn_simple<T, C, D>), dim3(grid), dim3(256), 0, s, c, (const T *)q, q_stride, row_off, (T *)out, rows, \
                       max_rows, Hq, scale_log2e)
    if (dh == 32) SIMPLE(32);
    else if (dh == 64) SIMPLE(64);
    else SIMPLE(128);
#undef SIMPLE
    DKV_LAUNCH_CHECK();
    return DKV_OK;
}

// What both entry points refuse.
int attn_call(const dkv_paged_cache *cache, PagedCache &view, int32_t n_q_heads, int32_t rows, int32_t max_rows_per_seq, int32_t dtype) {
    const int rc = dkv_paged_view(cache, view);
    if (rc) return rc;
    if (!cache->seq_len) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads || rows < 0 || max_rows_per_seq < 0 || rows > (int64_t)cache->batch * max_rows_per_seq) {
        dkv_set_error("inconsistent sizes"); return DKV_E_INVALID_ARG;
    }
    if (dtype != DKV_BF16 && dtype != DKV_FP32) { dkv_set_error("unknown dtype"); return DKV_E_INVALID_ARG; }
    if (cache->dtype != dtype && cache->dtype != DKV_E4M3) { dkv_set_error("rows of dtype %d do not read a cache of dtype %d", dtype, cache->dtype); return DKV_E_UNSUPPORTED; }
    if ((int64_t)rows * n_q_heads >= 1 << 24) { dkv_set_error("%d rows of %d heads are too many for one call", rows, n_q_heads); return DKV_E_UNSUPPORTED; }
    return DKV_OK;
}

}  // namespace

extern "C" size_t dkv_paged_attn_workspace_bytes(const dkv_paged_cache *cache, int32_t n_q_heads, int32_t rows,
                                                 int32_t max_rows_per_seq, int32_t dtype) {
    PagedCache c;
    return attn_call(cache, c, n_q_heads, rows, max_rows_per_seq, dtype) ? 0 : 256;
}

extern "C" int dkv_paged_attn(const dkv_paged_cache *cache, const void *q, int64_t q_stride, const int32_t *row_off, void *out,
                              int32_t rows, int32_t max_rows_per_seq, int32_t n_q_heads, int32_t dtype, void *workspace,
                              size_t workspace_bytes, void *stream) {
    PagedCache c;
    int rc = attn_call(cache, c, n_q_heads, rows, max_rows_per_seq, dtype);
    if (rc || (rc = dkv_paged_check_rows(*cache, row_off, rows))) return rc;
    if (q_stride < (int64_t)n_q_heads * cache->head_dim) { dkv_set_error("row stride %lld is less than a row", (long long)q_stride); return DKV_E_INVALID_ARG; }
    if (rows == 0) return DKV_OK;
    if (!q || !out) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == DKV_BF16)
        return cache->dtype == DKV_BF16
                   ? launch_simple<bf16_t, bf16_t>(c, cache->head_dim, q, q_stride, row_off, out, rows, max_rows_per_seq, n_q_heads, s)
                   : launch_simple<bf16_t, e4m3_t>(c, cache->head_dim, q, q_stride, row_off, out, rows, max_rows_per_seq, n_q_heads, s);
    return cache->dtype == DKV_FP32
               ? launch_simple<float, float>(c, cache->head_dim, q, q_stride, row_off, out, rows, max_rows_per_seq, n_q_heads, s)
               : launch_simple<float, e4m3_t>(c, cache->head_dim, q, q_stride, row_off, out, rows, max_rows_per_seq, n_q_heads, s);
}
