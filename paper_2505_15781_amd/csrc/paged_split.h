// Attention over a paged cache for few and middling numbers of rows: the NW wavefronts of a workgroup share the keys.
// Included by paged_attn.hip.
//
// Work item = (sequence, K/V head, group of NQ query tiles of 16 rows, slice of the keys); a query row is a (row, query head of the
// group) pair. The tiles of 32 keys of a slice are dealt to the wavefronts in turn. A wavefront brings its tile into an LDS region of
// its own, the next tile on its way in registers, and keeps an online softmax for its query tiles; the states of the
// wavefronts meet in LDS at the end. With one slice that is the result, else a record (max, sum, unnormalised output) for
// paged_merge.
//
// Slices are made on the device, because only it knows the lengths: all workgroups compute the same slice length from the
// total number of key tiles and the number of slices that the host wants for the whole batch, and find their own by a prefix
// sum over the sequences. So a captured call follows the lengths, and a ragged batch is cut where its keys are.
//
// e4m3 elements are converted on their way into LDS with their row's scale (exact in bf16 and fp32), everything behind is the same
// for all caches. A tile is two halves of 16 keys, each on one page: no load needs a bounds check, a half without a page reads page 0
// and is masked. Masked scores become -infinity and masked V rows zero, whatever they hold.
//
// Bound by the K/V stream where there is much of it: one token of 32 sequences of up to 4096 keys, 32 heads of 128 in e4m3 (558 MB), 95 us, 5.9
// TB/s (a cold read of that size reaches 6.0); two sequences of 131072 keys, 28/4 heads, e4m3 (271 MB), 45 us and 4.5 us
// of paged_merge. 32 query rows of 8 sequences of 1024 keys, 32 heads, bf16 (138 MB) 25 us, 5.5 TB/s. Few keys are a chain of latencies
// (length, page number, first tile, join): 512 keys of 32 heads 7.6 us.
#pragma once

constexpr int PKT = 32;                // keys per tile

// How the keys of a batch are cut: into at most `want` slices for one K/V head and query group over the whole batch (each sequence
// with rows has one at least, and there are fewer sequences than `want`), none shorter than `least` tiles before they are evened
// out within their sequence.
struct SlicePlan {
    int least;
    Divisor want;
    bool split;
};
// Workgroup id -> (slice, K/V head) and query group. The groups of one (slice, K/V head) read the same keys and are on one XCD (id mod 8),
// or in 2^shift parts on as many, where one XCD would get more of them than run at once.
struct GroupMap {
    Divisor groups;                    // of a part
    int shift, q_rows;                 // q_rows: rows of records for each (slice, K/V head)
    __device__ __forceinline__ void find(int id, int &unit, int &group) const {
        const int slot = id >> 3, at = groups.div(slot) * 8 + (id & 7);
        unit = at >> shift;
        group = (at & ((1 << shift) - 1)) * groups.d + groups.mod(slot);
    }
};
struct Slices {
    int first, n;                      // slices of the sequences before, and of this one
    int b, r0, rows, keys;             // the sequence
};

__device__ __forceinline__ int wave_prefix(int x) {        // inclusive: within rows of 16 lanes, then across the rows
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
// x / d rounded up for 0 <= x <= 2^25 and d > 0: a quotient that is off by a few at most, that of what it leaves, and one more or less
__device__ __forceinline__ int ceil_div_fast(int x, int d) {
    const float inv = __builtin_amdgcn_rcpf((float)d);
    int q = (int)((float)x * inv), r = x - q * d;
    const int more = (int)((float)r * inv);
    q += more;
    r -= more * d;
    if (r < 0) --q, r += d;
    return q + (r > 0) + (r > d);
}
// Key tiles of a sequence: at least one where there are rows, which makes the slice that writes their zeros.
__device__ __forceinline__ int key_tiles(int keys, int rows) { return rows > 0 ? max(1, (keys + PKT - 1) / PKT) : 0; }
__device__ __forceinline__ int key_tiles(const PagedCache &c, const int *row_off, int b) {
    return key_tiles(c.keys(b), row_off ? row_off[b + 1] - row_off[b] : 1);
}
// Key tiles of a slice: a want-th of all, or, where rounding up within the sequences makes more than `want` slices of that, a
// (want - k)th for the first k of batch / 2 (what that rounding adds on average), 3 batch / 4 and batch that does not: with the last there are
// no more than want - batch whole slices, and one for each sequence's rest. (Ragged batches, us with only the
// first and the last of these, and as it is: 160 sequences of up to 4096 keys, one K/V head, e4m3 37.9 and 32.1; 12 of up to 18822, 24/8 heads of 64,
// 38.8 and 34; 5 of up to 16792, 91 rows of 16/1 heads 73 and 65.)
// Whole wavefronts; `tiles`: of sequence `lane`.
__device__ __forceinline__ int slice_length(const PagedCache &c, const int *row_off, const SlicePlan &plan, int tiles) {
    const int lane = threadIdx.x & 63;
    auto sum = [&](auto f) {
        int x = f(tiles);
        for (int i = 64 + lane; i < c.batch; i += 64) x += f(key_tiles(c, row_off, i));
        return __builtin_amdgcn_readlane(wave_prefix(x), 63);
    };
    const int total = sum([](int x) { return x; });
    int slice = max(plan.least, plan.want.div(total + plan.want.d - 1));
    for (int quarters = 2; quarters <= 4 && sum([&](int x) { return ceil_div_fast(x, slice); }) > plan.want.d; ++quarters)
        slice = max(plan.least, ceil_div(total, plan.want.d - (c.batch * quarters >> 2)));
    return slice;
}
// Whole wavefronts. Finds slice `at` of the batch; false if there are fewer.
__device__ __forceinline__ bool find_slice(const PagedCache &c, const int *row_off, const SlicePlan &plan, int at, Slices &s) {
    const int lane = threadIdx.x & 63;
    if (!plan.split) {
        if (at >= c.batch) return false;
        s.b = s.first = at;
        s.n = 1;
        rows_of_sequence(row_off, at, s.r0, s.rows);
        s.keys = c.keys(at);
        return true;
    }
    int slice = 0, before = 0;
    for (int i = 0; i < c.batch; i += 64) {
        const int b = min(i + lane, c.batch - 1), keys = c.keys(b);
        int r0, rows;
        rows_of_sequence(row_off, b, r0, rows);
        const int tiles = i + lane < c.batch ? key_tiles(keys, rows) : 0;
        if (i == 0) slice = slice_length(c, row_off, plan, tiles);
        const int n = ceil_div_fast(tiles, slice), upto = before + wave_prefix(n);
        const unsigned long long hit = __builtin_amdgcn_ballot_w64(upto > at);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            s.b = i + l;
            s.n = __builtin_amdgcn_readlane(n, l);
            s.first = __builtin_amdgcn_readlane(upto, l) - s.n;
            s.r0 = __builtin_amdgcn_readlane(r0, l);
            s.rows = __builtin_amdgcn_readlane(rows, l);
            s.keys = __builtin_amdgcn_readlane(keys, l);
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

template <typename T, int DH> struct SplitSmem {
    static constexpr int K_STRIDE = DH * (int)sizeof(T) + 16;                               // bytes per row; the rest spreads
    static constexpr int V_STRIDE = DH * (int)sizeof(T) + (sizeof(T) == 2 ? 32 : 16);       // the reads over the banks
    static constexpr int K_BYTES = PKT * K_STRIDE;
    static constexpr int WAVE_BYTES = PKT * (K_STRIDE + V_STRIDE);
};

// A 16-byte piece of a row as it is stored -> elements of T in LDS.
__device__ __forceinline__ void stage(bf16_t *dst, const bf16_t *, u32x4 x, float) { *reinterpret_cast<u32x4 *>(dst) = x; }
__device__ __forceinline__ void stage(float *dst, const float *, u32x4 x, float) { *reinterpret_cast<u32x4 *>(dst) = x; }
__device__ __forceinline__ void stage(bf16_t *dst, const e4m3_t *, u32x4 x, float scale) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        u32x4 y;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            y[2 * k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * i + k], scale, false));
            y[2 * k + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * i + k], scale, true));
        }
        *reinterpret_cast<u32x4 *>(dst + 8 * i) = y;
    }
}
__device__ __forceinline__ void stage(float *dst, const e4m3_t *, u32x4 x, float scale) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(x[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(x[i], true);
        *reinterpret_cast<f32x4 *>(dst + 4 * i) = f32x4{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale};
    }
}

// softmax_step with probabilities that stay in fp32 (in st), and their sum over this lane's keys in l_acc[0]
template <int NT, int NACC>
__device__ __forceinline__ void softmax_step_f32(f32x4 (&st)[NT], float &m_run, f32x4 &l_acc, f32x4 (&acc)[NACC], float scale_log2e) {
    float mx = -INFINITY;
#pragma unroll
    for (int jt = 0; jt < NT; ++jt)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, st[jt][i]);
    const float m_new = fmaxf(m_run, query_lanes_max(mx) * scale_log2e);
    if (__builtin_amdgcn_ballot_w64(m_new > m_run) != 0) {
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        l_acc[0] *= alpha;
#pragma unroll
        for (int mt = 0; mt < NACC; ++mt) acc[mt] *= alpha;
        m_run = m_new;
    }
#pragma unroll
    for (int jt = 0; jt < NT; ++jt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            st[jt][i] = __builtin_amdgcn_exp2f(fmaf(st[jt][i], scale_log2e, -m_new));
            l_acc[0] += st[jt][i];
        }
}

// T: rows (and LDS), C: cache, ONCE: one query group, so that nobody else reads these keys (non-temporal loads)
template <typename T, typename C, int DH, int NQ, int NW, bool ONCE>
__global__ __launch_bounds__(64 * NW, 8 / NW) void paged_attn_split(PagedCache c, SlicePlan plan, const T *__restrict__ Q, int64_t q_stride,
                                                                    const int *__restrict__ row_off, T *__restrict__ out, int2 *__restrict__ meta,
                                                                    float *__restrict__ part, int rows, int max_rows, GroupMap map, Divisor heads,
                                                                    Divisor G, float scale_log2e) {
    using SM = SplitSmem<T, DH>;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int REC = DH + 4;                       // floats per record: m, l, pad, pad, o[DH]
    static_assert(NQ * 16 * REC * 4 <= SM::WAVE_BYTES, "records fit the wavefront's LDS region");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unsigned char *ksm = smem_raw + wave * SM::WAVE_BYTES, *vsm = ksm + SM::K_BYTES;

    int unit, qg;
    map.find((int)blockIdx.x, unit, qg);
    const int at = heads.div(unit), kvh = heads.mod(unit);
    // Pages of this wavefront's tiles t_begin + wave + NW j: lane i has half i & 1 of tile j0 + i / 2. The entry is read whatever the
    // length is, so that a plan without slices asks for it before it knows the length.
    int entry = -1, entry_ahead = -1;
    auto first_key = [&](int t_begin, int j0) { return (t_begin + wave + NW * (j0 + (lane >> 1))) * PKT + 16 * (lane & 1); };
    auto load_entry = [&](int b, int key) { return key < c.capacity() ? c.table[(size_t)b * c.max_pages + (key >> c.page_shift)] : -1; };
    if (!plan.split && at < c.batch) entry = load_entry(at, first_key(0, 0));
    Slices sl;
    if (!find_slice(c, row_off, plan, at, sl)) return;
    // the same in every lane, which the compiler does not see behind the two ways to a slice
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    const int b = uniform(sl.b), r0 = uniform(sl.r0), len = uniform(sl.keys), first = uniform(sl.first), n_slices = uniform(sl.n);
    const int nq = uniform(min(sl.rows, max_rows)) * G.d, m0 = qg * NQ * 16;      // query rows of this (sequence, K/V head), first one here
    if (m0 >= nq) return;                                             // uniform for the workgroup
    const int tiles = key_tiles(len, 1), per = plan.split ? uniform(ceil_div_fast(tiles, n_slices)) : tiles;
    const int t_begin = (at - first) * per, t_end = min(tiles, t_begin + per);
    if (plan.split && tid == 0 && at == first && kvh == 0 && qg == 0) meta[b] = make_int2(first, n_slices);

    // the page of such an entry; -1: none, or behind the end
    auto page_of = [&](int entry, int j0) { return first_key(t_begin, j0) < len && (unsigned)entry < (unsigned)c.n_pages ? entry : -1; };
    constexpr int ROW = DH * (int)sizeof(C), LPR = ROW / 16, RPI = 64 / LPR, N = PKT / RPI;    // lanes per row, rows per load, loads
    u32x4 kreg[N], vreg[N];
    uint32_t scales = 0;                      // e4m3: lane i has the scale of K row i, or of V row i - 32, as a float
    int pages = -1, seen0 = 0, seen1 = 0;     // seen: keys of each half that are attended to
    auto load_tile = [&](int t, int j) {
        const int id0 = __builtin_amdgcn_readlane(pages, 2 * (j & 31)), id1 = __builtin_amdgcn_readlane(pages, 2 * (j & 31) + 1);
        const int key = t * PKT, slot = key & (c.page_size() - 1), slot1 = (key + 16) & (c.page_size() - 1);
        seen0 = id0 < 0 ? 0 : min(16, len - key);
        seen1 = id1 < 0 ? 0 : min(16, len - key - 16);
        const uint32_t row0 = c.row(max(id0, 0), kvh, slot), row1 = c.row(max(id1, 0), kvh, slot1);
        auto fetch = [&](u32x4 (&reg)[N], const unsigned char *base) {
            const unsigned char *p0 = base + (size_t)row0 * ROW, *p1 = base + (size_t)row1 * ROW;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const unsigned char *p;
                if constexpr (RPI > 16) p = (lane < 32 ? p0 : p1) + (lane / LPR % 16) * ROW + lane % LPR * 16;
                else p = (i * RPI < 16 ? p0 : p1) + i * RPI % 16 * ROW + (lane / LPR) * ROW + lane % LPR * 16;
                reg[i] = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)) : *reinterpret_cast<const u32x4 *>(p);
            }
        };
        fetch(kreg, c.k);
        fetch(vreg, c.v);
        if constexpr (sizeof(C) == 1) scales = (uint32_t)(lane < 32 ? c.ks : c.vs)[(lane & 16 ? row1 : row0) + (lane & 15)] << 23;
    };
    auto store_tile = [&]() {
        const bool masked = seen0 < 16 || seen1 < 16;                 // uniform
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = i * RPI + lane / LPR, el = lane % LPR * (16 / (int)sizeof(C));
            float k_scale = 1.f, v_scale = 1.f;
            if constexpr (sizeof(C) == 1) {
                k_scale = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(row << 2, (int)scales));
                v_scale = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute((32 + row) << 2, (int)scales));
            }
            if (masked && (row & 15) >= (row < 16 ? seen0 : seen1)) {
                vreg[i] = u32x4{0, 0, 0, 0};
                v_scale = 1.f;
            }
            stage(reinterpret_cast<T *>(ksm + row * SM::K_STRIDE) + el, (const C *)nullptr, kreg[i], k_scale);
            stage(reinterpret_cast<T *>(vsm + row * SM::V_STRIDE) + el, (const C *)nullptr, vreg[i], v_scale);
        }
    };

    const int qi = lane & 15, g = lane >> 4;
    float m_run[NQ];
    f32x4 acc[NQ][DH / 16], l_acc[NQ];
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
        m_run[j] = -3.0e38f;            // finite, so that a score of -infinity has probability zero
        l_acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    int t = t_begin + wave, j = 0;
    if (plan.split) entry = load_entry(b, first_key(t_begin, 0));
    entry_ahead = load_entry(b, first_key(t_begin, 32));
    // Query operands. bf16: dims 32 ks + 8 g + [0, 8); fp32: dims 16 ks + 4 g + [0, 4), one of the four for each product
    constexpr int QS = BF ? DH / 32 : DH / 16;
    u32x4 qf[NQ][QS];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int mq = m0 + 16 * n + qi;
        const int r = r0 + G.div(mq);
        const bool ok = mq < nq && (unsigned)r < (unsigned)rows;
        const T *qp = Q + (ok ? r * q_stride + (kvh * G.d + G.mod(mq)) * DH : 0) + (BF ? 8 : 4) * g;
#pragma unroll
        for (int ks = 0; ks < QS; ++ks) {
            const u32x4 x = *reinterpret_cast<const bf16x8_el *>(qp + (BF ? 32 : 16) * ks);
            qf[n][ks] = ok ? x : u32x4{0, 0, 0, 0};
        }
    }
    pages = page_of(entry, 0);
    if (t < t_end) load_tile(t, 0);
    const bf16x8 ones = row_sum_operand(lane);
    const unsigned char *vrow0 = vsm + (4 * g + (qi >> 2)) * SM::V_STRIDE + (qi & 3) * 8;      // bf16: see vt_operand

    for (; t < t_end; t += NW, ++j) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        store_tile();
        const int now0 = seen0, now1 = seen1;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if ((j & 31) == 31) {
            pages = page_of(entry_ahead, j + 1);
            entry_ahead = load_entry(b, first_key(t_begin, j + 33));
        }
        if (t + NW < t_end) load_tile(t + NW, j + 1);

        f32x4 st[NQ][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned char *krow = ksm + (16 * h + qi) * SM::K_STRIDE + g * 16;
#pragma unroll
            for (int n = 0; n < NQ; ++n) st[n][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < QS; ++ks) {
                const u32x4 kf = *reinterpret_cast<const u32x4 *>(krow + ks * 64);
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    if constexpr (BF) {
                        st[n][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[n][ks]),
                                                                           st[n][h], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            st[n][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[e]), __uint_as_float(qf[n][ks][e]), st[n][h], 0, 0, 0);
                    }
                }
            }
        }
        // st[n][h][i] is the score of key 16 h + 4 g + i of this tile against query qi of tile n
        if (now0 < 16 || now1 < 16) {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (4 * g + i >= (h ? now1 : now0)) st[n][h][i] = -INFINITY;
        }
        if constexpr (BF) {
            bf16x8 pb[NQ][1];
#pragma unroll
            for (int n = 0; n < NQ; ++n) softmax_step<2, DH / 16>(st[n], m_run[n], l_acc[n], acc[n], pb[n], 0, 0, false, scale_log2e);
#pragma unroll
            for (int n = 0; n < NQ; ++n) l_acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[n][0], l_acc[n], 0, 0, 0);
#pragma unroll
            for (int mt = 0; mt < DH / 16; ++mt) {
                const bf16x8 av = vt_operand(vrow0, mt, SM::V_STRIDE, 0);
#pragma unroll
                for (int n = 0; n < NQ; ++n) acc[n][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, pb[n][0], acc[n][mt], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int n = 0; n < NQ; ++n) softmax_step_f32<2, DH / 16>(st[n], m_run[n], l_acc[n], acc[n], scale_log2e);
#pragma unroll
            for (int mt = 0; mt < DH / 16; ++mt)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float av = *reinterpret_cast<const float *>(vsm + (16 * h + 4 * g + i) * SM::V_STRIDE + (16 * mt + qi) * 4);
#pragma unroll
                        for (int n = 0; n < NQ; ++n) acc[n][mt] = __builtin_amdgcn_mfma_f32_16x16x4f32(av, st[n][h][i], acc[n][mt], 0, 0, 0);
                    }
        }
    }

    // Each wavefront leaves its state in its own LDS region: record (tile n, query qi) = m, l, -, -, o[DH].
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    float *my_rec = reinterpret_cast<float *>(ksm);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const float l = query_lanes_sum(l_acc[n][0]);
        float *rec = my_rec + (n * 16 + qi) * REC;
        if (g == 0) {
            rec[0] = m_run[n];
            rec[1] = l;
        }
#pragma unroll
        for (int mt = 0; mt < DH / 16; ++mt) *reinterpret_cast<f32x4 *>(rec + 4 + 16 * mt + 4 * g) = acc[n][mt];
    }
    __syncthreads();

    constexpr int CHUNKS = DH / 4;                    // a thread joins 4 output dims of a query row
    for (int idx = tid; idx < NQ * 16 * CHUNKS; idx += 64 * NW) {
        const int qr = idx / CHUNKS, ch = idx % CHUNKS, mq = m0 + qr, r = r0 + G.div(mq);
        if (mq >= nq || (unsigned)r >= (unsigned)rows) continue;
        float mw[NW], M = -3.0e38f, lsum = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            mw[w] = reinterpret_cast<const float *>(smem_raw + w * SM::WAVE_BYTES)[qr * REC];
            M = fmaxf(M, mw[w]);
        }
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float *rec = reinterpret_cast<const float *>(smem_raw + w * SM::WAVE_BYTES) + qr * REC;
            const float wgt = __builtin_amdgcn_exp2f(mw[w] - M);
            lsum += wgt * rec[1];
            o += wgt * *reinterpret_cast<const f32x4 *>(rec + 4 + 4 * ch);
        }
        if (n_slices == 1) {
            store_result(out + (((size_t)r * c.n_kv_heads + kvh) * G.d + G.mod(mq)) * DH + 4 * ch, o, lsum);
        } else {
            float *rec = part + ((int64_t)unit * map.q_rows + mq) * REC;
            if (ch == 0) {
                rec[0] = M;
                rec[1] = lsum;
            }
            *reinterpret_cast<f32x4 *>(rec + 4 + 4 * ch) = o;
        }
    }
}

// Joins the slices of one (row, query head): a workgroup each, so that up to GROUPS records are on their way at once (with a wavefront
// each, 32 slices were 16 memory latencies). Rows of sequences with one slice have their result already.
template <typename T, int DH>
__global__ __launch_bounds__(256) void paged_merge(const int *__restrict__ row_off, int batch, const int2 *__restrict__ meta,
                                                   const float *__restrict__ part, T *__restrict__ out, int rows, int max_rows, Divisor Hq,
                                                   Divisor G, int q_rows) {
    constexpr int REC = DH + 4, CH = DH / 4, GROUPS = 256 / CH;    // CH lanes hold a record's output
    __shared__ f32x4 os[GROUPS][CH];
    __shared__ float2 stats[GROUPS];
    const int tid = threadIdx.x, lane = tid % CH, group = tid / CH, pair = (int)blockIdx.x, r = Hq.div(pair), h = Hq.mod(pair);
    // the row's sequence, its first row and slices: a lane per sequence asks for all three at once
    int in = 0, first = 0, n = 0;
    for (int i = 0; i < batch; i += 64) {
        const int b = min(i + (tid & 63), batch - 1);
        int r0, rows_here;
        rows_of_sequence(row_off, b, r0, rows_here);
        const int2 slices = meta[b];
        const unsigned long long hit = __builtin_amdgcn_ballot_w64(r >= r0 && r < r0 + rows_here && b == i + (tid & 63));
        if (hit) {
            const int l = __builtin_ctzll(hit);
            in = r - __builtin_amdgcn_readlane(r0, l);
            first = __builtin_amdgcn_readlane(slices.x, l);
            n = __builtin_amdgcn_readlane(slices.y, l);
            break;
        }
    }
    if ((unsigned)in >= (unsigned)max_rows || n <= 1) return;      // no sequence, left out, or done
    const int kvh = G.div(h), mq = in * G.d + G.mod(h), heads = G.div(Hq.d);
    const size_t step = (size_t)heads * q_rows * REC;
    const float *rec = part + (((size_t)first * heads + kvh) * q_rows + mq) * REC;
    float m = -3.0e38f, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s = group; s < n; s += 2 * GROUPS) {
        const bool two = s + GROUPS < n;
        const float *x = rec + s * step, *y = two ? x + GROUPS * step : x;
        const float2 xs = *reinterpret_cast<const float2 *>(x), ys = *reinterpret_cast<const float2 *>(y);
        const f32x4 xo = *reinterpret_cast<const f32x4 *>(x + 4 + 4 * lane), yo = *reinterpret_cast<const f32x4 *>(y + 4 + 4 * lane);
        const float top = fmaxf(m, fmaxf(xs.x, ys.x)), w = __builtin_amdgcn_exp2f(m - top), wx = __builtin_amdgcn_exp2f(xs.x - top),
                    wy = two ? __builtin_amdgcn_exp2f(ys.x - top) : 0.f;
        l = w * l + wx * xs.y;
        o = w * o + wx * xo;
        if (two) {
            l += wy * ys.y;
            o += wy * yo;
        }
        m = top;
    }
    os[group][lane] = o;
    if (lane == 0) stats[group] = make_float2(m, l);
    __syncthreads();
    if (group) return;
    float top = m;
    for (int i = 1; i < GROUPS; ++i) top = fmaxf(top, stats[i].x);
    const float w = __builtin_amdgcn_exp2f(m - top);
    l *= w;
    o *= w;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) {
        const float2 x = stats[i];
        const float wi = __builtin_amdgcn_exp2f(x.x - top);
        l += wi * x.y;
        o += wi * os[i][lane];
    }
    store_result(out + (size_t)pair * DH + 4 * lane, o, l);
}
