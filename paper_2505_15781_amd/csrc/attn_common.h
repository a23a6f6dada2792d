// What the attention kernels share: operands that come out of LDS transposed, reductions over the lanes of a query, the step of
// the online softmax.
#pragma once
#include "common.h"

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((address_space(3))) bf16x4 *lds_bf16x4_ptr;

// MFMA operand V^T[dim 16 mt + (lane & 15)][8 keys] from V rows stored as they are in the cache (row = key).
// ds_read_b64_tr_b16 works on blocks of 16 lanes: lane j points at 4 consecutive 16-bit elements, and lane i
// receives element i % 4 of the pieces of lanes i / 4, i / 4 + 4, i / 4 + 8, i / 4 + 12. With lane j pointing
// at dims [16 mt + 4 (j % 4), +4) of key j / 4, lane i gets dim 16 mt + i of four consecutive keys. Two reads
// give the 8 keys of the lane's K group in the order the probabilities come out of the score MFMA:
// keys key0 + 4 g + {0..3} and key0 + 16 + 4 g + {0..3}, g = lane / 16. `vrow0` = address of (key 4 g + j / 4,
// dim 4 (j % 4)) of the tile, precomputed per lane.
__device__ __forceinline__ bf16x8 vt_operand(const unsigned char *vrow0, int mt, int v_stride, int key0) {
    const unsigned char *a = vrow0 + key0 * v_stride + mt * 32;
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(a));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(a + 16 * v_stride));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Reductions over the four lanes that hold one query (lane, lane ^ 16, lane ^ 32, lane ^ 48), every lane getting the
// result: gfx950's row swaps (v_permlane16_swap exchanges the odd 16-lane rows of one register with the even rows of
// another, v_permlane32_swap the upper half of one with the lower half of another; applied to two copies of x they
// leave "my value" and "my partner's value" side by side). Two vector instructions per stage instead of an LDS
// round trip (ds_bpermute) with its index arithmetic, on the path between the two products of every key tile.
__device__ __forceinline__ void swap_rows16(float x, float &u, float &v) {
    const unsigned a = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const unsigned r0 = r[0], r1 = r[1];
    u = __builtin_bit_cast(float, r0);
    v = __builtin_bit_cast(float, r1);
}
__device__ __forceinline__ void swap_rows32(float x, float &u, float &v) {
    const unsigned a = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const unsigned r0 = r[0], r1 = r[1];
    u = __builtin_bit_cast(float, r0);
    v = __builtin_bit_cast(float, r1);
}
__device__ __forceinline__ float query_lanes_max(float x) {
    float u, v;
    swap_rows16(x, u, v);
    x = fmaxf(u, v);
    swap_rows32(x, u, v);
    return fmaxf(u, v);
}
__device__ __forceinline__ float query_lanes_sum(float x) {
    float u, v;
    swap_rows16(x, u, v);
    x = u + v;
    swap_rows32(x, u, v);
    return u + v;
}

// One online-softmax step of a lane over NT sub-tiles of 16 keys (Eq. 4's softmax, streamed): st[jt][i] is the raw
// score of key key_base + 16 jt + i against this lane's query. Updates the running max (log2 domain) and sum,
// rescales the output accumulators, and returns the probabilities as bf16 MFMA operands: operand hh covers
// sub-tiles 2hh and 2hh+1. The running sum is not formed here: the caller multiplies the same operands with a row of
// ones (row_sum_operand) into l_acc, so the matrix pipe adds up exactly the rounded probabilities that enter the
// second product and the vector units are spared sixteen additions per lane and tile; l_acc is only rescaled here.
template <int NT, int NACC>
__device__ __forceinline__ void softmax_step(f32x4 (&st)[NT], float &m_run, f32x4 &l_acc, f32x4 (&acc)[NACC],
                                             bf16x8 (&pb)[NT / 2], int key_base, int L, bool masked,
                                             float scale_log2e) {
    if (masked) {              // wave-uniform: only the last tile of a sequence has keys past the end
#pragma unroll
        for (int jt = 0; jt < NT; ++jt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (key_base + 16 * jt + i >= L) st[jt][i] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int jt = 0; jt < NT; ++jt)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, st[jt][i]);
    mx = query_lanes_max(mx);
    const float m_new = fmaxf(m_run, mx * scale_log2e);
    // Rescale only when some query of the wavefront got a new maximum (rare after the first tiles): for the
    // others the factor would be exactly 1.
    if (__builtin_amdgcn_ballot_w64(m_new > m_run) != 0) {
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        l_acc *= alpha;
#pragma unroll
        for (int mt = 0; mt < NACC; ++mt) acc[mt] *= alpha;
        m_run = m_new;
    }
#pragma unroll
    for (int hh = 0; hh < NT / 2; ++hh) {
        f32x8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            p[e] = __builtin_amdgcn_exp2f(fmaf(st[2 * hh + (e >> 2)][e & 3], scale_log2e, -m_new));
        pb[hh] = __builtin_convertvector(p, bf16x8);
    }
}

// First operand of the product that sums the probabilities of a query: a 16 x 32 tile whose row 0 is all ones (the
// lanes with lane % 16 == 0 hold that row). mfma(row_sum_operand, pb, l_acc) adds the sum over the 32 keys of pb to
// element 0 of l_acc in the lanes below 16 (row 0, column = query); everything else in l_acc stays zero, so the sum
// over a query's four lanes (query_lanes_sum of element 0) is the running sum.
__device__ __forceinline__ bf16x8 row_sum_operand(int lane) {
    const __bf16 one = (lane & 15) == 0 ? (__bf16)1.0f : (__bf16)0.0f;
    return bf16x8{one, one, one, one, one, one, one, one};
}

// 16 bytes with the non-temporal hint (data that this launch reads once)
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load16_nt(const void *p) {
    const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p));
    return make_uint4(v.x, v.y, v.z, v.w);
}
