// Attention over a paged cache for blocks of 128 query rows: 32 query rows per wavefront, 32x32x16 MFMA, head_dim 128.
// Included by paged_attn.hip.
//
// Work item = (sequence, K/V head, block of 128 query rows). The loop is that of attn_wide.h: keys in tiles of 64 through two LDS
// stages, half tiles of 32 keys in a skewed order, a stretch holding the scores of half tile j + 1, the output products of half tile
// j - 1 and the exponentials of half tile j. What differs is where a tile comes from. It is four groups of 16 keys, each on one page;
// their places are found once per tile from page numbers that a lane each holds for the next 1024 keys.
//   bf16: global memory to LDS without registers; keys that are not there (behind the end, no page) come from a row of zeros.
//   e4m3: through registers, a tile ahead, converted with their row's scale (exact) on the way into LDS. K and V are converted
//         once per 128 query rows: 32 of a wavefront's vector instructions per tile, next to some 280 of softmax and rescaling.
#pragma once

typedef __attribute__((address_space(3))) void *lds_ptr_t;
template <int V> struct StageC { static constexpr int value = V; };
constexpr int WIDE_LDS_BYTES = 4 * 64 * 256;         // K0 K1 V0 V1, rows of 256 bytes

// Place of the 16-byte chunk c of row r: c ^ wide_swizzle(r) (see attn_wide.h).
__device__ __forceinline__ int wide_swizzle(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }

__device__ __align__(256) const u32x4 zero_row[16] = {};

// Work item of this workgroup. The blocks of a (sequence, K/V head) pair read the same keys and live on one XCD, pair % 8; workgroups
// are handed out to the blocks that hold rows, pair by pair, so that none without rows stands between others.
__device__ __forceinline__ bool wide_item(const PagedCache &c, const int *row_off, int max_rows, int G, int &pair, int &qb) {
    const int lane = threadIdx.x & 63, slot = blockIdx.x >> 3, pairs = c.batch * c.n_kv_heads;
    int before = 0;
    for (int p0 = blockIdx.x & 7; p0 < pairs; p0 += 512) {
        const int p = p0 + 8 * lane, b = min(p, pairs - 1) / c.n_kv_heads;
        int r0, n;
        rows_of_sequence(row_off, b, r0, n);
        n = p < pairs ? (max(0, min(n, max_rows)) * G + 127) / 128 : 0;
        const int upto = before + wave_prefix(n);
        const unsigned long long behind = __builtin_amdgcn_ballot_w64(upto > slot);
        if (behind) {
            const int at = __builtin_ctzll(behind);
            pair = p0 + 8 * at;
            qb = slot - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(n, at));
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Where a tile of 64 keys is: the rows (see PagedCache::row) of its four groups of 16 keys, and which of them have a page.
struct WideTile {
    size_t row[4];
    int pages;
};

template <typename C>
__global__ __launch_bounds__(256, 2) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_attn_wide(
    PagedCache c, const bf16_t *__restrict__ Q, int64_t q_stride, const int *__restrict__ row_off, bf16_t *__restrict__ out, int rows,
    int max_rows, int Hq, float scale_log2e) {
    constexpr int NW = 4, DH = 128, ROW = DH * 2, KT2 = 64, TILE = KT2 * ROW;     // bytes of an LDS row, of a K or V tile
    constexpr bool E4M3 = sizeof(C) == 1;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = Hq / c.n_kv_heads;
    const int qi = lane & 31, g = lane >> 5, l16 = lane & 15, l4 = lane >> 4;
    const uint32_t lds_base = (uint32_t)(size_t)(lds_ptr_t)smem_raw;
    int pair, qb;
    if (!wide_item(c, row_off, max_rows, G, pair, qb)) return;
    const int kvh = pair % c.n_kv_heads, b = pair / c.n_kv_heads;
    int r0, nrows;
    rows_of_sequence(row_off, b, r0, nrows);
    const int nq = min(nrows, max_rows) * G, mb0 = qb * NW * 32;
    const int L = c.keys(b), n_tiles = max(1, (L + KT2 - 1) / KT2);

    // pages of the 64 groups of 16 keys of a window, a lane each; -1: none, or behind the end
    auto load_pages = [&](int window) {
        const int key = (window * 64 + lane) * 16;
        return key < L ? c.page(b, key) : -1;
    };
    int pages = load_pages(0), pages_ahead = load_pages(1);
    auto find = [&](int t) {                        // tiles in order
        WideTile x;
        x.pages = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int id = __builtin_amdgcn_readlane(pages, (t & 15) * 4 + i);
            x.pages |= (id >= 0) << i;
            x.row[i] = c.row(max(id, 0), kvh, (t * KT2 + 16 * i) & (c.page_size() - 1));
        }
        if ((t & 15) == 15) {
            pages = pages_ahead;
            pages_ahead = load_pages((t >> 4) + 2);
        }
        return x;
    };
    // keys that are there of a tile's group
    auto there = [&](int t, int tile_pages, int i) { return tile_pages >> i & 1 ? L - (t * KT2 + 16 * i) : 0; };

    // bf16. Load i of a wavefront fills rows 16 i + 4 wave + [0, 4) of a tile; lane -> row lane / 16, place lane % 16.
    const uint32_t chunk = (l16 ^ wide_swizzle(4 * wave + l4)) << 4;
    auto fill = [&](const unsigned char *base, const WideTile &x, int t, uint32_t dst) {
        if (x.pages == 15 && (t + 1) * KT2 <= L) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                dma16_at(l4 * ROW + chunk, base + (x.row[i] + 4 * wave) * ROW, lds_base + dst + (16 * i + 4 * wave) * ROW);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned char *p = base + (x.row[i] + 4 * wave + l4) * ROW;
                dma16((4 * wave + l4 < there(t, x.pages, i) ? p : reinterpret_cast<const unsigned char *>(zero_row)) + chunk,
                      lds_base + dst + (16 * i + 4 * wave) * ROW);
            }
        }
    };
    // e4m3. Load i of a wavefront has rows 32 i + 8 wave + [0, 8); lane -> row lane / 8, elements 16 (lane % 8) + [0, 16).
    const int r16 = 8 * (wave & 1) + (lane >> 3);                     // row within the group 2 i + wave / 2
    u32x4 kreg[2], vreg[2];
    uint32_t k_scale[2], v_scale[2];
    auto fetch = [&](u32x4 (&reg)[2], uint32_t (&scale)[2], const unsigned char *base, const uint8_t *scales, const WideTile &x) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const size_t row = wave >> 1 ? x.row[2 * i + 1] : x.row[2 * i];
            reg[i] = *reinterpret_cast<const u32x4 *>(base + row * DH + r16 * DH + 16 * (lane & 7));
            scale[i] = scales[row + r16];
        }
    };
    auto convert = [&](const u32x4 (&reg)[2], const uint32_t (&scale)[2], int tile_pages, int t, uint32_t dst) {
        const bool whole = tile_pages == 15 && (t + 1) * KT2 <= L;    // uniform
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = 32 * i + 8 * wave + (lane >> 3), sw = wide_swizzle(row);
            const float s = __uint_as_float(scale[i] << 23);
            u32x4 y[2];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e >> 1][2 * (e & 1)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(reg[i][e], s, false));
                y[e >> 1][2 * (e & 1) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(reg[i][e], s, true));
            }
            if (!whole && r16 >= there(t, tile_pages, 2 * i + (wave >> 1))) y[0] = y[1] = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<u32x4 *>(smem_raw + dst + row * ROW + (((2 * (lane & 7) + e) ^ sw) << 4)) = y[e];
        }
    };
    // this lane's query row; rows beyond the host's bound have no slot in Q and out
    const int mq = mb0 + wave * 32 + qi, r = r0 + mq / G, h = kvh * G + mq % G;
    const bool q_ok = mq < nq && (unsigned)r < (unsigned)rows;
    bf16x8 qf[DH / 16];
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks)
        qf[ks] = __builtin_bit_cast(bf16x8, (u32x4)*reinterpret_cast<const bf16x8_el *>(Q + (q_ok ? r * q_stride + h * DH : 0) + 8 * g + 16 * ks));
    // pages of the tiles t, t + 1, t + 2 (of the last ones: of some tile), and where tile t + 1 (bf16) or t + 2 (e4m3) is
    int pages_0, pages_1, pages_2;
    WideTile x = find(0), ahead = x;
    pages_0 = pages_1 = pages_2 = x.pages;
    if constexpr (E4M3) {
        fetch(kreg, k_scale, c.k, c.ks, x);
        fetch(vreg, v_scale, c.v, c.vs, x);
        convert(kreg, k_scale, pages_0, 0, 0);
        convert(vreg, v_scale, pages_0, 0, 2 * TILE);
        if (n_tiles > 1) {
            x = find(1);
            pages_1 = x.pages;
            fetch(kreg, k_scale, c.k, c.ks, x);
            fetch(vreg, v_scale, c.v, c.vs, x);
            convert(kreg, k_scale, pages_1, 1, TILE);
        }
        if (n_tiles > 2) {
            x = find(2);
            pages_2 = x.pages;
            fetch(kreg, k_scale, c.k, c.ks, x);
        }
    } else {
        fill(c.k, x, 0, 0);
        fill(c.v, x, 0, 2 * TILE);
        if (n_tiles > 1) {
            x = find(1);
            pages_1 = x.pages;
            fill(c.k, x, 1, TILE);
        }
    }

    // score operands: row lane & 31, chunk 2 ks + g
    const unsigned char *krow = smem_raw + qi * ROW;
    const int kx = (g ^ wide_swizzle(qi)) << 4;
    // output operand: see vt_operand; block lane / 16 = (g, dims + 16 half), key 4 g + j / 4 (+ 8), dims 4 (j % 4)
    const unsigned char *vrow = smem_raw + 2 * TILE + (4 * g + (l16 >> 2)) * ROW + ((l16 & 1) << 3);
    const int vx = ((2 * (l4 & 1) + ((l16 & 3) >> 1)) ^ (((l16 >> 2) << 2) | g)) << 4;       // keys + 8: swizzle ^ 2

    // lowest finite start: scores of -inf then give probabilities of zero, also where a whole half tile is masked
    float m_run = -3.0e38f, alpha = 1.f;
    bool behind = false;
    // sum of exactly the rounded probabilities of the second product: a product with a tile whose row 0 is ones; element 0
    // of the lanes below 32 is the sum of query qi, everything else stays zero
    f32x16 l_acc;
    bf16x8 ones;
#pragma unroll
    for (int v = 0; v < 16; ++v) l_acc[v] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = qi == 0 ? (__bf16)1.0f : (__bf16)0.0f;
    f32x16 acc[DH / 32], stA, stB;               // stA, stB: scores of the first and the second 32 keys of a tile
    bf16x8 pA[2], pB[2];                         // their probabilities
#pragma unroll
    for (int i = 0; i < DH / 32; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][v] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) pB[0][e] = pB[1][e] = (__bf16)0.f;

    auto k_operand = [&](int ks, int stage, int half) {
        return *reinterpret_cast<const bf16x8 *>(krow + (kx ^ (ks << 5)) + stage * TILE + half * 32 * ROW);
    };
    // keys of k step ks in operand order: 16 ks + 4 g + {0..3}, 16 ks + 8 + 4 g + {0..3}: as the scores leave the MFMA
    auto v_operand = [&](int mt, int ks, int stage, int half) {
        const unsigned char *p = vrow + stage * TILE + (2 * half + ks) * 16 * ROW;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(p + (vx ^ (mt << 6))));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(p + 8 * ROW + (vx ^ (mt << 6) ^ 32)));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // One stretch: scores of a half tile (into sn), output products of the half tile before the last (pv), exponentials of
    // the last one (so -> pn). The three are independent of each other.
    auto stretch = [&](f32x16 &sn, int kstage, int khalf, const bf16x8 (&pv)[2], int vstage, int vhalf, const f32x16 &so,
                       bf16x8 (&pn)[2]) {
#pragma unroll
        for (int v = 0; v < 16; ++v) sn[v] = 0.f;
        f32x8 p[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) l_acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones, pv[ks], l_acc, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(i, kstage, khalf), qf[i], sn, 0, 0, 0);
            acc[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(i & 3, i >> 2, vstage, vhalf), pv[i >> 2], acc[i & 3], 0, 0, 0);
#pragma unroll
            for (int e = 2 * i; e < 2 * i + 2; ++e)
                p[e >> 3][e & 7] = __builtin_amdgcn_exp2f(fmaf(so[e], scale_log2e, -m_run));
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) pn[ks] = __builtin_convertvector(p[ks], bf16x8);
        asm volatile("" : "+v"(pn[0]), "+v"(pn[1]));        // here, not behind the branches of maximum()
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
        }
    };
    // Brings the output up to the reference m_run of the exponentials.
    auto rescale = [&]() {
        if (!behind) return;
#pragma unroll
        for (int mt = 0; mt < DH / 32; ++mt) acc[mt] *= alpha;
        l_acc[0] *= alpha;
    };
    // Maximum of half `half` of tile t. The running maximum is the reference of the exponentials, so that the largest
    // probability is exactly 1. The probabilities of the half tile before still wait for their product: the output is
    // rescaled to the new reference only behind that product, at the next call.
    auto maximum = [&](f32x16 &st, int t, int half, int tile_pages) {
        rescale();
        if ((tile_pages >> (2 * half) & 3) != 3 || t * KT2 + 32 * half + 32 > L) {           // uniform
            const int left[2] = {there(t, tile_pages, 2 * half), there(t, tile_pages, 2 * half + 1)};
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (8 * (v >> 2 & 1) + 4 * g + (v & 3) >= left[v >> 3]) st[v] = -INFINITY;
        }
        float mx = st[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) mx = fmaxf(mx, st[v]);
        float u, w;
        swap_rows32(mx, u, w);
        mx = fmaxf(u, w) * scale_log2e;
        const float m_new = fmaxf(m_run, mx);
        behind = __builtin_amdgcn_ballot_w64(m_new > m_run) != 0;       // else the factor is exactly 1 for every query
        alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
    };
    auto tile_barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);      // vmcnt(0), lgkmcnt(0): this wavefront's fills have landed, its LDS accesses are done
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // the first stretch multiplies (zero) probabilities with the second half of V stage 1: no NaN may be there
    for (int i = tid; i < TILE / 32; i += 64 * NW) reinterpret_cast<uint4 *>(smem_raw + 3 * TILE + TILE / 2)[i] = make_uint4(0, 0, 0, 0);
    tile_barrier();
#pragma unroll
    for (int v = 0; v < 16; ++v) stA[v] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) stA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(i, 0, 0), qf[i], stA, 0, 0, 0);
    maximum(stA, 0, 0, pages_0);
    // Tile t, in stage S; the scores of its first half are formed.
    auto step = [&](int t, auto stage) {
        constexpr int S = decltype(stage)::value;
        stretch(stB, S, 1, pB, S ^ 1, 1, stA, pA);
        maximum(stB, t, 1, pages_0);
        // behind the barrier K(t + 1) and V(t) have landed for everybody, and everybody is done with K(t) and V(t - 1)
        tile_barrier();
        if constexpr (E4M3) {
            if (t + 2 < n_tiles) convert(kreg, k_scale, pages_2, t + 2, S * TILE);
            if (t + 1 < n_tiles) convert(vreg, v_scale, pages_1, t + 1, (2 + (S ^ 1)) * TILE);
            pages_0 = pages_1;
            pages_1 = pages_2;
            if (t + 2 < n_tiles) fetch(vreg, v_scale, c.v, c.vs, x);
            if (t + 3 < n_tiles) {
                x = find(t + 3);
                pages_2 = x.pages;
                fetch(kreg, k_scale, c.k, c.ks, x);
            }
        } else {
            if (t + 2 < n_tiles) {
                ahead = find(t + 2);
                pages_2 = ahead.pages;
                fill(c.k, ahead, t + 2, S * TILE);
            }
            if (t + 1 < n_tiles) fill(c.v, x, t + 1, (2 + (S ^ 1)) * TILE);
            x = ahead;
            pages_0 = pages_1;
            pages_1 = pages_2;
        }
        stretch(stA, S ^ 1, 0, pA, S, 0, stB, pB);            // behind the last tile: scores of an old tile, never used
        if (t + 1 < n_tiles) maximum(stA, t + 1, 0, pages_0);
    };
    for (int t = 0; t < n_tiles; t += 2) {
        step(t, StageC<0>{});
        if (t + 1 < n_tiles) step(t + 1, StageC<1>{});
    }
    const int last = (n_tiles - 1) & 1;
    rescale();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) l_acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones, pB[ks], l_acc, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        acc[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(i & 3, i >> 2, last, 1), pB[i >> 2], acc[i & 3], 0, 0, 0);

    float u, w;
    swap_rows32(l_acc[0], u, w);
    const float inv = u + w == 0.f ? 0.f : 1.f / (u + w);
    if (!q_ok) return;
    bf16_t *op = out + ((size_t)r * Hq + h) * DH + 8 * g;
#pragma unroll
    for (int mt = 0; mt < DH / 32; ++mt)
#pragma unroll
        for (int c = 0; c < 4; c += 2) {
            // lane qi holds dims 8 c + {0..3} and 8 c + 8 + {0..3}, lane qi + 32 the other four of each: after the swaps the
            // first has the lower 8 dims, the second the upper 8
            uint32_t y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = 4 * c + (e >> 1) * 4 + (e & 1) * 2;
                y[e] = (uint32_t)f2bf(acc[mt][v] * inv) | ((uint32_t)f2bf(acc[mt][v + 1] * inv) << 16);
            }
            const auto p0 = __builtin_amdgcn_permlane32_swap(y[0], y[2], false, false);
            const auto p1 = __builtin_amdgcn_permlane32_swap(y[1], y[3], false, false);
            *reinterpret_cast<bf16x8_el *>(op + 32 * mt + 8 * c) = u32x4{p0[0], p1[0], p0[1], p1[1]};
        }
}
