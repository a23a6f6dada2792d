// Attention over a paged cache for blocks of 128 query rows: 32 query rows per wavefront, 32x32x16 MFMA, head_dim 64 or 128.
// Included by paged_attn.hip.
//
// Work item = (sequence, K/V head, block of 128 query rows). The loop is that of attn_wide.h: keys in tiles of 64 through two LDS
// stages, half tiles of 32 keys in a skewed order, a stretch holding the scores of half tile j + 1, the output products of half tile
// j - 1 and the exponentials of half tile j. What differs is where a tile comes from. It is four groups of 16 keys, each on one page;
// their places are found once per tile from page numbers that a lane each holds for the next 1024 keys.
//   bf16: global memory to LDS without registers; keys that are not there (behind the end, no page) come from a row of zeros.
//   e4m3, e2m1: through registers, a tile ahead, converted with their scale (exact) on the way into LDS. K and V are converted
//         once per 128 query rows: 32 of a wavefront's vector instructions per tile, next to some 200 of the softmax.
//
// 4 sequences of 1536 rows and keys, 32 heads of 128 (155 GFLOP): e4m3 178-188 us by card, 820-870 TFLOP/s, bf16 191-193. A large product would take
// 111 us. Power is part of the rest: with zeros for data the same launches take 160 and 143 us. What the other part is no counters show yet. Softmax,
// products and LDS reads hide behind each other: without its exponentials the e4m3 launch took 5 % less, without the maximum 2 %, without the reads
// of V 4 %. Measured and not kept there: the maximum inside the stretch (193 us), 64 query rows per wavefront (227), e4m3 conversion spread over the
// stretch (no gain; 64 dims 125 -> 150), two groups of wavefronts (187-209), blocks of 256 query rows with eight wavefronts behind one barrier, which
// halves the fills (201 against 183: two workgroups to a compute unit drift apart and fill each other's gaps), LDS reads 9 and 12 ahead instead of 6
// (no change). Over e2m1 171-188 us by card. Not kept there: the conversion between the products of a stretch, from two sets of registers (171 -> 179
// us), or of K where it is used, each wavefront for itself and without LDS (172 -> 177); keys that are not there made zero when they are fetched (178
// -> 181). Two wavefronts of a SIMD take 1.25 us for a tile each, one alone 1.5. Products of K in 4 bits with the queries in two parts of 8 (the same
// matrix time, no conversion) add up to less than fp32: up to 2^-12 of the sum of magnitudes is lost.
#pragma once

typedef __attribute__((address_space(3))) void *lds_ptr_t;
template <int V> struct StageC { static constexpr int value = V; };
template <int DH> constexpr int kWideLds = 4 * 64 * DH * 2;       // K0 K1 V0 V1

// Place of the 16-byte chunk c of row r: c ^ wide_swizzle(r). 16 consecutive rows put a chunk (score operands) into 16 different places of
// 256 bytes, and the 4 chunks of 8 rows that a transposing read takes are spread evenly over them. Rows of 128 bytes lie two to
// 256 bytes; with either length the value of row r + 8 is that of row r with bit 1 turned, of row r + 16 the same.
template <int DH> __device__ __forceinline__ int wide_swizzle(int row) {
    if (DH == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
    return ((row >> 1 & 1) << 2) | ((row >> 2) & 3);
}

__device__ __align__(256) const u32x4 zero_row[16] = {};

// Work item of this workgroup: the sequences in the order of their key tiles, the longest first (64 of them at a time), so that
// compute units that get two workgroups get short ones, and none without rows stands between others (rows behind those of the call
// count for nothing: the host has no workgroups for them). Within a sequence the K/V
// heads go fastest: the blocks of a head, which read the same keys, are on one XCD (id % 8) with 8 heads, on two with 4.
// With two groups of wavefronts a workgroup takes one block of a long sequence, a group each half of its key tiles (parts = 2), or two
// blocks of a short one, a group each: as many sequences are long as `units` workgroups (one per compute unit) have room for.
// (Where blocks are so few that compute units would be idle and the keys many, these are cut into slices as for paged_attn_split instead.)
struct WideItem {
    Slices seq;
    int kvh, qb, parts;                // qb: the first block
};
template <int KS>
__device__ __forceinline__ bool wide_item(const PagedCache &c, const int *row_off, int total_rows, int max_rows, Divisor heads, int G, int units, WideItem &w) {
    const int lane = threadIdx.x & 63, at = heads.div(blockIdx.x);
    w.kvh = heads.mod(blockIdx.x);
    int before = 0;
    for (int i = 0; i < c.batch; i += 64) {
        const int b = min(i + lane, c.batch - 1), keys = c.keys(b);
        int r0, rows;
        rows_of_sequence(row_off, b, r0, rows);
        const int blocks = i + lane < c.batch ? (max(0, min(min(rows, max_rows), total_rows - r0)) * G + 127) / 128 : 0, cost = (keys + 63) / 64;
        int rank = 0;                                      // sequences before this one
        for (int k = 0; k < min(64, c.batch - i); ++k) {
            const int other = __builtin_amdgcn_readlane(cost, k);
            rank += other > cost || (other == cost && k < lane);
        }
        if (i + lane >= c.batch) rank = lane;
        int n = __builtin_amdgcn_ds_permute(rank << 2, blocks);
        const int from = __builtin_amdgcn_ds_permute(rank << 2, lane);
        int parts = 1;
        if constexpr (KS == 2) {
            const int pairs = (n + 1) / 2, one = __builtin_amdgcn_ds_permute(rank << 2, (int)(cost <= 1)) ? pairs : n;
            // workgroups if this sequence and all before it are long
            const int all = __builtin_amdgcn_readlane(wave_prefix(pairs), 63) + wave_prefix(one - pairs);
            parts = c.batch <= 64 && one == n && all <= units ? 2 : 1;
            n = parts == 2 ? n : pairs;
        }
        const int upto = before + wave_prefix(n);
        const unsigned long long behind = __builtin_amdgcn_ballot_w64(upto > at);
        if (behind) {
            const int k = __builtin_ctzll(behind), l = __builtin_amdgcn_readlane(from, k);
            w.parts = __builtin_amdgcn_readlane(parts, k);
            w.qb = (at - (__builtin_amdgcn_readlane(upto, k) - __builtin_amdgcn_readlane(n, k))) * (KS == 2 && w.parts == 1 ? 2 : 1);
            w.seq.b = i + l;
            w.seq.r0 = __builtin_amdgcn_readlane(r0, l);
            w.seq.rows = __builtin_amdgcn_readlane(rows, l);
            w.seq.keys = __builtin_amdgcn_readlane(keys, l);
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Words e and e ^ turn change places.
__device__ __forceinline__ void turn_words(u32x4 &a, int turn) {
    const u32x4 b = turn & 1 ? u32x4{a[1], a[0], a[3], a[2]} : a;
    a = turn & 2 ? u32x4{b[2], b[3], b[0], b[1]} : b;
}

// Where a tile of 64 keys is: the rows (see PagedCache::row) of its four groups of 16 keys, and which of them have a page.
struct WideTile {
    uint32_t row[4];
    int pages;
};

template <typename C, int DH, int KS>
__global__ __launch_bounds__(256 * KS, 2) __attribute__((amdgpu_waves_per_eu(2, DH == 128 ? 2 : 4))) void paged_attn_wide(
    PagedCache c, const bf16_t *__restrict__ Q, int64_t q_stride, const int *__restrict__ row_off, bf16_t *__restrict__ out, int rows,
    int2 *__restrict__ meta, float *__restrict__ partial, SlicePlan plan, int max_rows, GroupMap map, Divisor heads, Divisor G, int units,
    float scale_log2e) {
    constexpr int NW = 4, ROW = DH * 2, KT2 = 64, TILE = KT2 * ROW;     // bytes of an LDS row, of a K or V tile
    constexpr bool CODES = sizeof(C) == 1;                              // e4m3 or e2m1
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_all[];

    // KS groups of four wavefronts, in LDS stages of their own
    const int tid = threadIdx.x & 255, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group_id = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 8);
    unsigned char *smem_raw = smem_all + group_id * kWideLds<DH>;
    const int qi = lane & 31, g = lane >> 5, l16 = lane & 15, l4 = lane >> 4;
    const uint32_t lds_base = (uint32_t)(size_t)(lds_ptr_t)smem_raw;
    // a group works on the tiles t0 + part, t0 + part + parts, ... below t1
    WideItem item;
    int parts = 1, t0 = 0, t1 = INT_MAX, slices = 1;
    int64_t record = 0;                              // first record of this (slice, K/V head)
    constexpr bool CUT = (KS == 2) == (DH == 128);   // whether there are plans with slices
    if (CUT && plan.split) {                     // slices as in paged_attn_split, all groups on one block
        int unit;
        map.find((int)blockIdx.x, unit, item.qb);
        const int at = heads.div(unit);
        item.kvh = heads.mod(unit);
        if (!find_slice(c, row_off, plan, at, item.seq)) return;
        slices = item.seq.n;
        parts = KS;
        const int tiles = (key_tiles(item.seq.keys, 1) + 1) / 2, per = __builtin_amdgcn_readfirstlane(ceil_div_fast(tiles, slices));
        t0 = (at - item.seq.first) * per;
        t1 = t0 + per;
        record = (int64_t)unit * map.q_rows;
        if (threadIdx.x == 0 && at == item.seq.first && item.kvh == 0 && item.qb == 0) meta[item.seq.b] = make_int2(item.seq.first, slices);
    } else {
        if (!wide_item<KS>(c, row_off, rows, max_rows, heads, G.d, units, item)) return;
        if (KS == 2) parts = item.parts;
    }
    // all of it the same in every lane, which the compiler does not see behind the two ways to an item
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    parts = KS == 1 ? 1 : uniform(parts);
    t0 = CUT ? uniform(t0) : 0;
    const int part = parts == 1 ? 0 : group_id, b = uniform(item.seq.b), r0 = uniform(item.seq.r0), kvh = uniform(item.kvh);
    const int keys = uniform(item.seq.keys), tiles = (keys + KT2 - 1) / KT2, end = CUT ? uniform(min(tiles, t1)) : tiles;
    const int L = end < tiles ? end * KT2 : keys;                     // keys from here on are another slice's, or none
    const int n_tiles = (max(1, end - t0) + parts - 1) / parts;
    const int nq = uniform(min(item.seq.rows, max_rows)) * G.d, mb0 = (uniform(item.qb) + (parts == 1 ? group_id : 0)) * NW * 32;
    if (CUT && mb0 >= nq && parts == KS) return;                      // uniform for the workgroup

    // this lane's query row; rows beyond the host's bound have no slot in Q and out
    const int mq = mb0 + wave * 32 + qi, r = r0 + G.div(mq), h = kvh * G.d + G.mod(mq);
    const bool q_ok = mq < nq && (unsigned)r < (unsigned)rows;
    bf16x8 qf[DH / 16];
#pragma unroll
    for (int i = 0; i < DH / 16; ++i)
        qf[i] = __builtin_bit_cast(bf16x8, (u32x4)*reinterpret_cast<const bf16x8_el *>(Q + (q_ok ? r * q_stride + h * DH : 0) + 8 * g + 16 * i));
    // The 64 groups of 16 keys of a window, a lane each: the row of the first key, and (a bit each) whether there is a page.
    auto look_up = [&](int window, uint32_t &row, unsigned long long &pages) {
        const int key = (window * 64 + lane) * 16, id = key < L ? c.page(b, key) : -1;
        row = c.row(max(id, 0), kvh, key & (c.page_size() - 1));
        pages = __builtin_amdgcn_ballot_w64(id >= 0);
    };
    uint32_t group, group_ahead;
    unsigned long long pages, pages_ahead;
    look_up((t0 + part) >> 4, group, pages);
    look_up(((t0 + part) >> 4) + 1, group_ahead, pages_ahead);
    auto find = [&](int step) {                     // steps in order
        const int t = t0 + step * parts + part;
        WideTile x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x.row[i] = __builtin_amdgcn_readlane(group, (t & 15) * 4 + i);
        x.pages = (int)(pages >> ((t & 15) * 4)) & 15;
        if ((t & 15) >= 16 - parts) {
            group = group_ahead;
            pages = pages_ahead;
            look_up((t >> 4) + 2, group_ahead, pages_ahead);
        }
        return x;
    };
    // keys that are there of a tile's group
    auto there = [&](int step, int tile_pages, int i) { return tile_pages >> i & 1 ? L - ((t0 + step * parts + part) * KT2 + 16 * i) : 0; };
    auto whole = [&](int step, int tile_pages) { return tile_pages == 15 && (t0 + step * parts + part + 1) * KT2 <= L; };

    // bf16. Load i of a wavefront fills rows RPL (4 i + wave) + [0, RPL) of a tile; lane -> row lane / LPR, place lane % LPR.
    constexpr int LPR = ROW / 16, RPL = 64 / LPR, LOADS = KT2 / (RPL * NW);
    const int d_row = (RPL * wave + lane / LPR) % 16;                  // row within its group of 16, the same for all loads
    const uint32_t chunk = (lane % LPR ^ wide_swizzle<DH>(d_row)) << 4;
    auto fill = [&](const unsigned char *base, const WideTile &x, int t, uint32_t dst) {
        const bool all = whole(t, x.pages);                           // uniform
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int first = RPL * (NW * i + wave), gr = RPL * NW * i / 16 + RPL * wave / 16;      // first row, its group: uniform
            const uint32_t row = (RPL * NW >= 32 ? (wave >> 1 ? x.row[RPL * NW * i / 16 + 1] : x.row[RPL * NW * i / 16]) : x.row[i]) + first % 16;
            const uint32_t lds = lds_base + dst + first * ROW;
            if (all) {
                dma16_at(lane / LPR * ROW + chunk, base + (size_t)row * ROW, lds);
            } else {
                const unsigned char *p = base + (size_t)(row + lane / LPR) * ROW;
                dma16((d_row < there(t, x.pages, gr) ? p : reinterpret_cast<const unsigned char *>(zero_row)) + chunk, lds);
            }
        }
    };
    // e4m3, e2m1. Load i of a wavefront has rows RPF (4 i + wave) + [0, RPF); lane -> row lane / LPF, elements PER (lane % LPF) + [0, PER).
    constexpr int LPF = kE2M1<C> ? 4 : DH / 16, PER = DH / LPF, RPF = 64 / LPF, FETCHES = KT2 / (RPF * NW);
    constexpr int SCALES = kE2M1<C> ? DH / 32 : 1, BYTES = kRowBytes<C, DH>;
    typedef typename PieceBits<BYTES / LPF>::type Bits;
    const int f_row = (RPF * wave + lane / LPF) % 16;
    auto f_group = [&](const WideTile &x, int i) {
        if constexpr (RPF == 16) {                   // numbers, not places, to choose from: those would put the tile into memory
            const uint32_t r0 = x.row[0], r1 = x.row[1], r2 = x.row[2], r3 = x.row[3], lo = wave & 1 ? r1 : r0, hi = wave & 1 ? r3 : r2;
            return wave & 2 ? hi : lo;
        } else {
            return wave >> 1 ? x.row[2 * i + 1] : x.row[2 * i];
        }
    };
    Bits kreg[FETCHES], vreg[FETCHES];
    uint32_t k_scale[FETCHES], v_scale[FETCHES];
    auto fetch = [&](Bits (&reg)[FETCHES], uint32_t (&scale)[FETCHES], const unsigned char *base, const uint8_t *scales, const WideTile &x) {
#pragma unroll
        for (int i = 0; i < FETCHES; ++i) {
            const size_t row = f_group(x, i);                         // uniform
            reg[i] = *reinterpret_cast<const Bits *>(base + row * BYTES + (uint32_t)(f_row * BYTES + BYTES / LPF * (lane % LPF)));
            scale[i] = (scales + row * SCALES)[(uint32_t)(f_row * SCALES + (kE2M1<C> ? lane % LPF * PER / 32 : 0))];
        }
    };
    // e2m1, 128 dims: a lane writes four chunks in a row, and four neighbouring rows would have theirs on the same banks at a time: each begins
    // with another one
    const int turn = kE2M1<C> && DH == 128 ? lane / LPF & 3 : 0;
    auto convert = [&](const Bits (&reg)[FETCHES], const uint32_t (&scale)[FETCHES], int tile_pages, int t, uint32_t dst) {
        const bool all = whole(t, tile_pages);                        // uniform
#pragma unroll
        for (int i = 0; i < FETCHES; ++i) {
            const int row = RPF * (NW * i + wave) + lane / LPF, sw = wide_swizzle<DH>(row);
            const float s = __uint_as_float(scale[i] << 23);
            u32x4 y[PER / 8];
            if constexpr (kE2M1<C>) {
                Bits a = reg[i];
                if constexpr (DH == 128) turn_words(a, turn);
#pragma unroll
                for (int e = 0; e < PER / 8; ++e) y[e] = bf16_of_e2m1(a[e], s);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e >> 1][2 * (e & 1)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(reg[i][e], s, false));
                    y[e >> 1][2 * (e & 1) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(reg[i][e], s, true));
                }
            }
            if (!all && f_row >= there(t, tile_pages, RPF == 16 ? wave : 2 * i + (wave >> 1))) {
#pragma unroll
                for (int e = 0; e < PER / 8; ++e) y[e] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int e = 0; e < PER / 8; ++e)
                *reinterpret_cast<u32x4 *>(smem_raw + dst + row * ROW + (((PER / 8 * (lane % LPF) + (e ^ turn)) ^ sw) << 4)) = y[e];
        }
    };
    // pages of the tiles t, t + 1, t + 2 (of the last ones: of some tile), and where tile t + 1 (bf16) or t + 2 (codes) is
    int pages_0, pages_1, pages_2;
    WideTile x = find(0), ahead = x;
    pages_0 = pages_1 = pages_2 = x.pages;
    if constexpr (CODES) {                        // all loads at once: K0 V0 K1, and V1 K2 for the loop
        Bits k0[FETCHES], v0[FETCHES], k1[FETCHES];
        uint32_t k0_scale[FETCHES], v0_scale[FETCHES], k1_scale[FETCHES];
        fetch(k0, k0_scale, c.k, c.ks, x);
        fetch(v0, v0_scale, c.v, c.vs, x);
        if (n_tiles > 1) x = find(1);
        pages_1 = x.pages;
        fetch(k1, k1_scale, c.k, c.ks, x);
        fetch(vreg, v_scale, c.v, c.vs, x);
        if (n_tiles > 2) x = find(2);
        pages_2 = x.pages;
        fetch(kreg, k_scale, c.k, c.ks, x);
        convert(k0, k0_scale, pages_0, 0, 0);
        convert(v0, v0_scale, pages_0, 0, 2 * TILE);
        convert(k1, k1_scale, pages_1, 1, TILE);
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
    const int kx = (g ^ wide_swizzle<DH>(qi)) << 4;
    // output operand: see vt_operand; block lane / 16 = (g, dims + 16 half), key 4 g + j / 4 (+ 8), dims 4 (j % 4)
    const unsigned char *vrow = smem_raw + 2 * TILE + (4 * g + (l16 >> 2)) * ROW + ((l16 & 1) << 3);
    const int vx = ((2 * (l4 & 1) + ((l16 & 3) >> 1)) ^ wide_swizzle<DH>(4 * g + (l16 >> 2))) << 4;

    // lowest finite start: scores of -inf then give probabilities of zero, also where a whole half tile is masked
    float m_run = -3.0e38f, alpha = 1.f;
    bool behind = false;
    // Sum of exactly the rounded probabilities that weigh the values, so that a weight is off by at most half a step however few keys share it:
    // with the unrounded ones the largest error of peaked scores is half as large again (0.024 against 0.016; 4 x 32 heads, 1536 rows and keys 184 us
    // against 187). A product with a tile whose row 0 is ones: element 0 of the lanes below 32 is the sum of query qi, everything else stays zero.
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
        // heads of 64, whose exponentials weigh as much as the products: the wavefront in here goes first (e2m1, 4 sequences of 1536 102 -> 98 us;
        // 128 dims: no change)
        if constexpr (DH == 64) __builtin_amdgcn_s_setprio(1);
        f32x8 p[2];
        constexpr int MT = DH / 32, N = DH / 16, PER = 16 / N;        // products of the scores, and of the output; exponentials next to each two
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) l_acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones, pv[ks], l_acc, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(i, kstage, khalf), qf[i], sn, 0, 0, 0);
            acc[i % MT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(i % MT, i / MT, vstage, vhalf), pv[i / MT], acc[i % MT], 0, 0, 0);
#pragma unroll
            for (int e = PER * i; e < PER * (i + 1); ++e) p[e >> 3][e & 7] = __builtin_amdgcn_exp2f(fmaf(so[e], scale_log2e, -m_run));
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) pn[ks] = __builtin_convertvector(p[ks], bf16x8);
        asm volatile("" : "+v"(pn[0]), "+v"(pn[1]));        // here, not behind the branches of maximum()
        if constexpr (DH == 64) __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, PER, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, PER / 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, PER, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, PER / 2, 0);
        }
    };
    // Brings the output up to the reference m_run of the exponentials.
    auto rescale = [&]() {
        if (!behind) return;
#pragma unroll
        for (int mt = 0; mt < DH / 32; ++mt) acc[mt] *= alpha;
        l_acc[0] *= alpha;
    };
    // Maximum of half `half` of tile t. bf16 caches: the running maximum is the reference of the exponentials, so that the largest
    // probability is exactly 1, as in attn_wide.h. e4m3 caches: the reference follows only where the maximum gets more than 2^8 ahead. That saves the
    // rescaling of the output at nearly every half tile (32 queries, each with a new maximum now and then), a third of a wavefront's vector
    // instructions: 4 sequences x 32 heads, 1536 rows and keys 199 -> 187 us. The largest probability is then rounded as all others are (half a step of
    // the value, whatever its size): relative error against float64 of the held values 0.0023 instead of 0.0022, with scores three times as large 0.0020
    // instead of 0.0018, next to the 2^-4 by which e4m3 rounds the elements themselves. A bf16 cache has no such rounding: what is read from it
    // is as exact as what dkv_attn_update reads (the reference that lags: 8 sequences x 32 heads, 512 rows, 1024 keys 98 us instead of 105).
    // The probabilities of the half tile before still wait for their product: the output is rescaled to the new reference
    // only behind that product, at the next call.
    constexpr float LAG = CODES ? 8.f : 0.f;
    auto maximum = [&](f32x16 &st, int t, int half, int tile_pages) {
        rescale();
        if (!whole(t, tile_pages)) {                                   // uniform
            const int left[2] = {there(t, tile_pages, 2 * half), there(t, tile_pages, 2 * half + 1)};
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (8 * (v >> 2 & 1) + 4 * g + (v & 3) >= left[v >> 3]) st[v] = -INFINITY;
        }
        float mx = st[0];                // a NaN goes on: v_maximum3_f32 needs no canonical operands, v_max3_f32 does
#pragma unroll
        for (int v = 1; v < 16; ++v) mx = __builtin_elementwise_maximum(mx, st[v]);
        float u, w;
        swap_rows32(mx, u, w);
        mx = fmaxf(u, w) * scale_log2e;
        behind = __builtin_amdgcn_ballot_w64(mx > m_run + LAG) != 0;
        if (!behind) return;
        const float m_new = fmaxf(m_run, mx);
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
    for (int i = 0; i < DH / 16; ++i) stA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(i, 0, 0), qf[i], stA, 0, 0, 0);
    maximum(stA, 0, 0, pages_0);
    // Tile t, in stage S; the scores of its first half are formed. LIVE: a wavefront with query rows; the others bring their share of the tiles.
    auto step = [&](int t, auto stage, auto alive) {
        constexpr int S = decltype(stage)::value, LIVE = decltype(alive)::value;
        if constexpr (LIVE) {
            stretch(stB, S, 1, pB, S ^ 1, 1, stA, pA);
            maximum(stB, t, 1, pages_0);
        }
        // behind the barrier K(t + 1) and V(t) have landed for everybody, and everybody is done with K(t) and V(t - 1)
        tile_barrier();
        if constexpr (CODES) {
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
        if constexpr (LIVE) {
            stretch(stA, S ^ 1, 0, pA, S, 0, stB, pB);        // behind the last tile: scores of an old tile, never used
            if (t + 1 < n_tiles) maximum(stA, t + 1, 0, pages_0);
        }
    };
    auto all_steps = [&](auto alive) {
        for (int t = 0; t < n_tiles; t += 2) {
            step(t, StageC<0>{}, alive);
            if (t + 1 < n_tiles) step(t + 1, StageC<1>{}, alive);
        }
    };
    if (mb0 + wave * 32 < nq) all_steps(StageC<1>{});
    else all_steps(StageC<0>{});
    const int last = (n_tiles - 1) & 1;
    rescale();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) l_acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones, pB[ks], l_acc, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < DH / 16; ++i)
        acc[i % (DH / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(i % (DH / 32), i / (DH / 32), last, 1), pB[i / (DH / 32)], acc[i % (DH / 32)], 0, 0, 0);

    float u, w;
    swap_rows32(l_acc[0], u, w);
    float sum = u + w;
    if (KS == 2 && parts == 2) {                 // the second group's state goes through LDS to the same lanes of the first
        f32x4 *parked = reinterpret_cast<f32x4 *>(smem_all + kWideLds<DH>);
        float2 *stats = reinterpret_cast<float2 *>(smem_all);
        __syncthreads();
        if (part == 1) {
#pragma unroll
            for (int i = 0; i < DH / 8; ++i) parked[i * 256 + tid] = f32x4{acc[i >> 2][4 * (i & 3)], acc[i >> 2][4 * (i & 3) + 1], acc[i >> 2][4 * (i & 3) + 2], acc[i >> 2][4 * (i & 3) + 3]};
            stats[tid] = make_float2(m_run, sum);
        }
        __syncthreads();
        if (part == 1) return;
        const float2 other = stats[tid];
        const float m = fmaxf(m_run, other.x), mine = __builtin_amdgcn_exp2f(m_run - m), theirs = __builtin_amdgcn_exp2f(other.x - m);
        sum = mine * sum + theirs * other.y;
        m_run = m;
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) {
            const f32x4 x = parked[i * 256 + tid];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i >> 2][4 * (i & 3) + e] = mine * acc[i >> 2][4 * (i & 3) + e] + theirs * x[e];
        }
    }
    if (!q_ok) return;
    if (CUT && slices > 1) {                     // a record for paged_merge: m, l, -, -, o[DH]
        float *rec = partial + (record + mq) * (DH + 4);
        if (g == 0) {
            rec[0] = m_run;
            rec[1] = sum;
        }
#pragma unroll
        for (int i = 0; i < DH / 8; ++i)
            *reinterpret_cast<f32x4 *>(rec + 4 + 32 * (i >> 2) + 8 * (i & 3) + 4 * g) =
                f32x4{acc[i >> 2][4 * (i & 3)], acc[i >> 2][4 * (i & 3) + 1], acc[i >> 2][4 * (i & 3) + 2], acc[i >> 2][4 * (i & 3) + 3]};
        return;
    }
    const float inv = 1.f / sum;
    bf16_t *op = out + ((size_t)r * (c.n_kv_heads * G.d) + h) * DH + 8 * g;
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
                y[e] = (uint32_t)f2bf(result(acc[mt][v], sum, inv)) | ((uint32_t)f2bf(result(acc[mt][v + 1], sum, inv)) << 16);
            }
            const auto p0 = __builtin_amdgcn_permlane32_swap(y[0], y[2], false, false);
            const auto p1 = __builtin_amdgcn_permlane32_swap(y[1], y[3], false, false);
            *reinterpret_cast<bf16x8_el *>(op + 32 * mt + 8 * c) = u32x4{p0[0], p1[0], p0[1], p1[1]};
        }
}
