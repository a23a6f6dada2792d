// Attention of new rows over a paged K/V cache: plans and boundary (kernels in paged_split.h and paged_wide.h).
#include <math.h>

#include <atomic>
#include <initializer_list>

#include "attn_common.h"
#include "paged.h"

namespace {

// An element of a result from its sums. A sum of exponentials of zero (nothing seen, or scores of -infinity only) gives zero, chosen and not
// multiplied: the products of zero probabilities with infinite or NaN values are NaN. `inv`: 1 / l.
__device__ __forceinline__ float result(float o, float l, float inv) { return l == 0.f ? 0.f : o * inv; }
// Four dims of a result.
__device__ __forceinline__ void store_result(float *p, f32x4 o, float l) {
    const float inv = 1.f / l;
    *reinterpret_cast<f32x4_el *>(p) = f32x4{result(o[0], l, inv), result(o[1], l, inv), result(o[2], l, inv), result(o[3], l, inv)};
}
__device__ __forceinline__ void store_result(bf16_t *p, f32x4 o, float l) {
    const float inv = 1.f / l;
    *reinterpret_cast<bf16x4_el *>(p) = u32x2{(uint32_t)f2bf(result(o[0], l, inv)) | ((uint32_t)f2bf(result(o[1], l, inv)) << 16),
                                              (uint32_t)f2bf(result(o[2], l, inv)) | ((uint32_t)f2bf(result(o[3], l, inv)) << 16)};
}

#include "paged_split.h"
#include "paged_wide.h"

// Lets a kernel have its LDS on the current device, once (racing threads only repeat it).
int allow_lds(const void *kernel, int bytes, std::atomic<uint64_t> &devices) {
    int dev = -1;
    DKV_HIP_TRY(hipGetDevice(&dev));
    const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
    if (!(devices.load(std::memory_order_acquire) & bit)) {
        DKV_HIP_TRY(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
        devices.fetch_or(bit, std::memory_order_release);
    }
    return DKV_OK;
}

typedef PagedAttnPlan Plan;

// Slices of paged_attn_split make up to one workgroup for each compute unit. With 128 dims that is all that a unit's LDS holds, and a second round costs
// what the first does (two sequences of 131072 keys: 56 us with 256 workgroups, 67 with 512). Smaller heads would leave room for two and more, which
// is not made use of: nothing gained over bf16 and fp32 caches but for a few calls, 10 to 30 % over e4m3 ones (two sequences of 131072 keys of 28/4 heads, one
// workgroup and two a unit: 64 dims, bf16 47.8 us and 48.7, e4m3 33.1 and 30.5; 32 dims, e4m3 28.1 and 21.9; 16 ragged ones of 4096, 64 dims, bf16 13.2
// and 13.9). A slice has 4 tiles of keys at least: what a compute unit
// reads is bound to some 50 GB/s, so idle units cost more than wavefronts without a tile (28/4 heads, 4 sequences of 2000 keys in
// bf16: 10.5 us with 4 tiles, 11.4 with 8, 17.2 with 32, 22.3 without slices). paged_attn_wide, whose groups take 64 keys at a time: 16
// tiles of 32 (28/4 heads, 64 rows, 4096 keys 23.1 us with 8, 21.9 with 16, 26.7 with 32; 16384 keys 36.8, 35.4, 35.3).
constexpr int kWorkgroups = 256, kLeast = 4, kLeastWide = 16;
// Key tiles of a table (the host does not know the lengths) up to which sequences stay whole: the launch that joins slices costs some 2 us. bf16, 128 dims: 16 tiles 8.6 us whole and 9.0
// in slices, 24 tiles 11.5 and 9.3; 64 dims: 24 tiles 7.3 and 8.1, 47 tiles 10.8 and 9.0. fp32 (four wavefronts, matrix instructions of an
// eighth of the rate): 128 dims, 8 tiles 13.3 and 11.8; 64 dims, 8 tiles 7.4 and 8.4, 16 tiles 12.1 and 8.5; 32 dims, 16 tiles 7.5 and 8.2, 24 9.7 and 8.5.
int whole_tiles(int dtype, int head_dim) { return (dtype == DKV_BF16 ? 2304 : 640) / head_dim; }

// Slices of one K/V head, all sequences together, that run at once: `per_cu` workgroups to a compute unit, `groups` query groups to a slice on
// 2^shift XCDs.
int slices_at_once(int groups, int heads, int shift, int per_cu) { return per_cu * (kWorkgroups / 8) / ceil_div(groups, 1 << shift) * 8 / (heads << shift); }
int best_spread(int groups, int heads, int per_cu) {
    int best = 0;
    for (int shift = 1; shift <= 3 && groups >> shift; ++shift)
        if (slices_at_once(groups, heads, shift, per_cu) > slices_at_once(groups, heads, best, per_cu)) best = shift;
    return best;
}

// Groups of n query rows, each of one (sequence, K/V head), at most: by the longest sequence's rows, or by the rows of all.
int64_t row_groups(const PagedCache &c, int rows, int max_rows, int G, int n) {
    const int64_t by_longest = (int64_t)c.batch * ceil_div(max_rows * G, n), by_all = c.batch + (int64_t)ceil_div(rows * G, n);
    return (by_longest < by_all ? by_longest : by_all) * c.n_kv_heads;
}
// Blocks of 128 query rows, see make_plan: whether there are rows enough, whether groups of 32 are so many or the keys that are cut so long, and
// whether keys are cut. None of them turns back with more rows.
bool rows_for_blocks(int dtype, int head_dim, int query_rows) { return dtype == DKV_BF16 && head_dim >= 64 && query_rows > (head_dim == 128 ? 32 : 64); }
bool blocks_for_rounds(int head_dim, int64_t groups) { return groups > (head_dim == 128 ? kWorkgroups : 3 * kWorkgroups); }
bool blocks_for_keys(int head_dim, int64_t groups, int64_t keys) { return keys * head_dim >= 4096 * 128 && groups * keys >= kWorkgroups * 1536; }
bool keys_to_cut(int head_dim, int64_t keys) { return keys >= (head_dim == 64 ? 4096 : 2048); }
int block_workgroups_per_cu(int head_dim) { return head_dim == 64 ? 3 : 1; }
int split_tiles(int dtype, int tiles) { return dtype == DKV_BF16 && tiles > 1 ? 2 : 1; }

Plan make_plan(const PagedCache &c, int n_q_heads, int rows, int max_rows, int dtype, int head_dim) {
    Plan p;
    max_rows = max_rows < rows ? max_rows : rows;
    const int G = n_q_heads / c.n_kv_heads, heads = c.n_kv_heads;
    const int tiles = ceil_div(max_rows > 0 ? max_rows * G : 1, 16), key_tiles = ceil_div(c.max_pages << c.page_shift, PKT);
    const int64_t keys = (int64_t)key_tiles * PKT;
    p.nq = split_tiles(dtype, tiles);
    p.q_groups = ceil_div(tiles, p.nq);
    p.wide = p.blocks = 0;
    p.spread = best_spread(p.q_groups, heads, 1);
    p.least = kLeast;
    int want = slices_at_once(p.q_groups, heads, p.spread, 1);
    p.split = key_tiles > whole_tiles(dtype, head_dim) && want > c.batch;
    // Blocks of 128 query rows (paged_wide.h) where tiles of 32 would make more than one round of workgroups (128 dims; 28/4 heads, 1024 keys: 1
    // sequence of 300 rows, 264 workgroups, 29 -> 26 us, 4 of 128 rows, 448, 30 -> 27, but 4 of 64 rows, 224, 17 -> 26) or more than three (64
    // dims, 32 heads, 8 ragged sequences of up to 5600 keys: bf16, 80 rows 61 -> 61, 128 rows 81 -> 70, 250 rows, 119 -> 104; e4m3 65 ->
    // 68, 94 -> 77, 144 -> 125; of 700 keys each 24.1 -> 21, 32 -> 22, 59 -> 32). Also where the
    // keys are so many that slices of them keep the compute units busy without those workgroups: 1536 keys each for tiles of 32 (28/4
    // heads, 1 sequence of 128 rows, 4096 keys 30.3 -> 28.9 us, 32768 keys 131 -> 98, but 32 rows, 4096 keys 15.9 -> 21.4, 8192 keys 21.0 -> 23.3),
    // of more than 4096 keys of 128 dims (64 dims, 28/4 heads, 2 sequences of 128 rows: 4096 keys 27.6 -> 34.4 over e4m3, 8192 keys 48.3 -> 46.9, bf16 42.8 -> 44.6).
    // More than 32 query rows to a sequence, which two of the four wavefronts work on (19 sequences of 700 keys, 32/32 heads, 40 rows 73 -> 59 us,
    // 32/8 heads, 10 rows 27.9 -> 25.1); with 64 dims more than 64 (32/32 heads, 64 rows, 12 sequences of 8192 keys 160 -> 198, e4m3 156 -> 245).
    // Two groups of wavefronts to a workgroup where the blocks are few and the keys many enough to share (96 blocks of 1024 keys 28.6 -> 26.0 us,
    // 128 blocks of 256 keys 12.8 -> 13.6), and one round of workgroups holds them two by two (36 sequences
    // of 700 keys, 32/8 heads, 32 rows: 288 blocks, each of a sequence of its own, 43 -> 58). Few are 320 at most, for the longest sequences of ragged batches
    // are then shared and the shorter ones paired (28/4 heads, 129 rows and 1536 keys at most: at most 308 blocks 45.8 -> 42.3, 344 47.2 -> 46.5, 380 50.8 -> 52.9);
    // batches of one length gain up to 256 and lose a little from there (32/32 heads, 1536 keys: 256 blocks 45.9 -> 43.9, 288 60.2 -> 63.4).
    // Their keys are cut where every sequence can have two slices, from 2048 keys of 128 dims on (32/8 heads, 300 rows, 80 blocks: 1300 keys
    // 32.9 us whole and 33.8 in slices, 2700 keys 55.9 and 43.0; 28/4 heads, 4 ragged sequences of 130 rows and 2000 keys at most 43.8 and 35.4),
    // from 4096 of 64 dims (4 sequences of 300 rows, 2700 keys: 32/32 heads 69 and 86, 28/4 heads 69 and 79, 3500 keys 85 and 89).
    // Slices of heads of 64 have one group of wavefronts, and three workgroups a compute unit, which hold more loads on their way than one of
    // two groups (28/4 heads, 130 rows, 100000 keys: e4m3 214 -> 167 us, bf16 155 -> 151; 32/32 heads, 80 rows, 2 sequences of 31000
    // 152 -> 123 and 116 -> 113; the other way 28/4 heads, 17 rows of 2 sequences of 31000 31.1 -> 32.8 and 28.4 -> 28.8).
    // With fewer slices the long sequences of a ragged batch are cut all the same. The host knows the rows, and takes it that keys go with
    // them (a batch of equal rows over ragged lengths is not seen): ragged is a batch with at most 3/4 of the rows that the longest sequence's would make (28/4 heads, 8 sequences of up to 9000 keys and 80 rows, 12
    // slices: 0.6 of them 159 -> 102 us, 0.75 158 -> 130, 1 161 -> 166; 14 of up to 2100, 37 rows, 20 slices: 0.6 45 -> 41, 0.75 46 -> 48, 0.8 46 -> 49), and
    // from four slices for three sequences on (9 sequences, 12 slices 158 -> 133, 10 158 -> 162; of up to 3000 keys, 40 rows, 20 slices for 13 sequences
    // 59 -> 44, 15 59.5 -> 59.5, 16 59.8 -> 63; 16/1 heads, 6000 keys, 64 rows, 32 slices for 24 109 -> 105, 26 109 -> 114). In two rounds of slices batches of one length lose (8 sequences of 5600 keys, 32 heads, 80
    // rows 119 -> 141).
    if (rows_for_blocks(dtype, head_dim, max_rows * G)) {
        const int64_t groups = row_groups(c, rows, max_rows, G, 32), blocks = row_groups(c, rows, max_rows, G, 128);
        const int per_cu = block_workgroups_per_cu(head_dim), q_groups = ceil_div(tiles, 8), spread = best_spread(q_groups, heads, per_cu);
        const int slices = slices_at_once(q_groups, heads, spread, per_cu);
        const int64_t two_by_two = (int64_t)c.batch * heads * ceil_div(max_rows * G, 256), other = (blocks + (int64_t)c.batch * heads) / 2;
        int wide = blocks <= 320 && (two_by_two < other ? two_by_two : other) <= kWorkgroups && key_tiles > 16 ? 2 : 1;
        const bool ragged = 4 * (int64_t)rows <= 3 * (int64_t)c.batch * max_rows;
        const bool cut = (wide == 2 || head_dim == 64) && keys_to_cut(head_dim, keys) &&
                         (slices >= 2 * c.batch || (ragged && 3 * slices >= 4 * c.batch));
        if (cut && head_dim == 64) wide = 1;
        if (blocks_for_rounds(head_dim, groups) || (cut && blocks_for_keys(head_dim, groups, keys))) {
            p.wide = wide;
            p.blocks = (int)blocks;
            p.nq = 8;
            p.q_groups = q_groups;
            p.spread = spread;
            p.least = kLeastWide;
            want = slices;
            p.split = cut;
        }
    }
    // Query groups on one XCD or several (see GroupMap): whatever allows most slices of a K/V head (all sequences together), with all workgroups
    // running at once, 32 to an XCD (28/4 heads, 32 rows, 8192 keys: 7 groups; 9 slices with 35 workgroups on some XCDs 29.6 us, 8 slices
    // with 28 on each 20.5; 300 rows, 16384 keys: 17 blocks, 2 slices on one XCD each 140 us, 3 on two each 105), and without slices
    // the fewest rounds (one K/V head, 33 groups of 6 sequences of 1006 keys: 6 XCDs 29 us, 8 XCDs 15.6; 150 groups of one of 1000 keys 67 and 15.7).
    if (!p.split) {
        auto rounds = [&](int shift) {
            const int64_t fullest = (((int64_t)c.batch * heads << shift) + 7) / 8 * ceil_div(p.q_groups, 1 << shift);
            return (fullest + kWorkgroups / 8 - 1) / (kWorkgroups / 8);
        };
        p.spread = 0;
        for (int shift = 1; shift <= 3 && p.q_groups >> shift; ++shift)
            if (rounds(shift) < rounds(p.spread)) p.spread = shift;
        // in several rounds also where few (sequence, K/V head) pairs of different lengths would leave XCDs behind (one K/V head, 6 ragged
        // sequences of 100 rows and 3700 keys at most: 71 -> 45 us; of one length 62 -> 62)
        if (rounds(p.spread) > 1)
            while (((int64_t)c.batch * heads << p.spread) < kWorkgroups / 8 && p.spread < 3 && p.q_groups >> (p.spread + 1)) ++p.spread;
    }
    p.want = p.split ? want : 1;
    const int64_t most = (int64_t)c.batch * ceil_div(key_tiles, p.least);
    p.cap = !p.split ? c.batch : (int)(most < want ? most : want);      // see slice_length
    return p;
}

// Workspace: (first slice, slices) of each sequence, then the records.
size_t meta_bytes(const PagedCache &c) { return align_up(c.batch * sizeof(int2), 16); }
size_t partial_bytes(const Plan &p, const PagedCache &c, int head_dim) {
    return p.split ? meta_bytes(c) + (size_t)p.cap * c.n_kv_heads * (p.q_groups * p.nq * 16) * (head_dim + 4) * sizeof(float) : 0;
}
// What no plan of this many rows and fewer exceeds, so that one workspace serves an active set that shrinks (fewer rows can have more slices: 28/4
// heads, 8 sequences of 4096 keys, none with 128 rows each, 17 MB with 64, 4 with 8). The slices of a plan times its K/V heads and query groups are
// one round of workgroups at most (slices_at_once), and no sequence has slices of less than `least` tiles.
size_t most_partial_bytes(const PagedCache &c, int n_q_heads, int rows, int max_rows, int dtype, int head_dim) {
    max_rows = max_rows < rows ? max_rows : rows;
    const int G = n_q_heads / c.n_kv_heads, tiles = ceil_div(max_rows > 0 ? max_rows * G : 1, 16), key_tiles = ceil_div(c.max_pages << c.page_shift, PKT);
    if (key_tiles <= whole_tiles(dtype, head_dim)) return 0;
    auto bytes = [&](int nq, int least, int per_cu) {
        int64_t n = 1;
        for (int64_t factor : {(int64_t)c.batch * ceil_div(key_tiles, least), (int64_t)c.n_kv_heads, (int64_t)ceil_div(tiles, nq)}) {
            n *= factor;
            if (n > per_cu * kWorkgroups) n = per_cu * kWorkgroups;
        }
        return meta_bytes(c) + (size_t)n * (nq * 16) * (head_dim + 4) * sizeof(float);
    };
    const size_t split = bytes(split_tiles(dtype, tiles), kLeast, 1);
    const int64_t groups = row_groups(c, rows, max_rows, G, 32), keys = (int64_t)key_tiles * PKT;
    if (!rows_for_blocks(dtype, head_dim, max_rows * G) || !keys_to_cut(head_dim, keys) ||
        !(blocks_for_rounds(head_dim, groups) || blocks_for_keys(head_dim, groups, keys)))
        return split;
    const size_t blocks = bytes(8, kLeastWide, block_workgroups_per_cu(head_dim));
    return blocks > split ? blocks : split;
}
SlicePlan slice_plan(const Plan &p) { return SlicePlan{p.least, Divisor(p.want), p.split}; }
GroupMap group_map(const Plan &p) { return GroupMap{Divisor(ceil_div(p.q_groups, 1 << p.spread)), p.spread, p.q_groups * p.nq * 16}; }
int64_t split_grid(const Plan &p, const PagedCache &c) {
    return (((int64_t)p.cap * c.n_kv_heads << p.spread) + 7) / 8 * 8 * ceil_div(p.q_groups, 1 << p.spread);
}

template <typename T, int DH>
int launch_merge(const PagedCache &c, const Plan &p, const int *row_off, void *out, void *part, int rows, int max_rows, int Hq, hipStream_t s) {
    hipLaunchKernelGGL((paged_merge<T, DH>), dim3((unsigned)(rows * Hq)), dim3(256), 0, s, row_off, c.batch, (const int2 *)part,
                       (const float *)((char *)part + meta_bytes(c)), (T *)out, rows, max_rows, Divisor(Hq), Divisor(Hq / c.n_kv_heads),
                       p.q_groups * p.nq * 16);
    DKV_LAUNCH_CHECK();
    return DKV_OK;
}

template <typename T, typename C, int DH, int NQ, int NW>
int launch_split(const PagedCache &c, const Plan &p, const void *q, int64_t q_stride, const int *row_off, void *out, void *part, int rows,
                 int max_rows, int Hq, hipStream_t s) {
    constexpr int smem = NW * SplitSmem<T, DH>::WAVE_BYTES;
    const float scale_log2e = 1.4426950408889634f / sqrtf((float)DH);
#define SPLIT(ONCE)                                                                                                              \
    do {                                                                                                                         \
        static std::atomic<uint64_t> devices{0};                                                                                 \
        const int rc = allow_lds(reinterpret_cast<const void *>(&paged_attn_split<T, C, DH, NQ, NW, ONCE>), smem, devices);      \
        if (rc) return rc;                                                                                                       \
        hipLaunchKernelGGL((paged_attn_split<T, C, DH, NQ, NW, ONCE>), dim3((unsigned)split_grid(p, c)), dim3(64 * NW), smem, s, c, slice_plan(p), \
                           (const T *)q, q_stride, row_off, (T *)out, (int2 *)part, (float *)((char *)part + meta_bytes(c)), rows, max_rows, \
                           group_map(p), Divisor(c.n_kv_heads), Divisor(Hq / c.n_kv_heads), scale_log2e);                \
    } while (0)
    if (p.q_groups == 1) SPLIT(true);
    else SPLIT(false);
#undef SPLIT
    DKV_LAUNCH_CHECK();
    return p.split ? launch_merge<T, DH>(c, p, row_off, out, part, rows, max_rows, Hq, s) : DKV_OK;
}

template <typename C, int DH, int KS>
int launch_wide(const PagedCache &c, const Plan &p, const void *q, int64_t q_stride, const int *row_off, void *out, void *part, int rows,
                int max_rows, int Hq, hipStream_t s) {
    static std::atomic<uint64_t> devices{0};
    const int rc = allow_lds(reinterpret_cast<const void *>(&paged_attn_wide<C, DH, KS>), KS * kWideLds<DH>, devices);
    if (rc) return rc;
    hipLaunchKernelGGL((paged_attn_wide<C, DH, KS>), dim3((unsigned)(p.split ? split_grid(p, c) : p.blocks)), dim3(256 * KS), KS * kWideLds<DH>, s, c,
                       (const bf16_t *)q, q_stride, row_off, (bf16_t *)out, rows, (int2 *)part, (float *)((char *)part + meta_bytes(c)), slice_plan(p),
                       max_rows, group_map(p), Divisor(c.n_kv_heads), Divisor(Hq / c.n_kv_heads), kWorkgroups / c.n_kv_heads,
                       1.4426950408889634f / sqrtf((float)DH));
    DKV_LAUNCH_CHECK();
    return p.split ? launch_merge<bf16_t, DH>(c, p, row_off, out, part, rows, max_rows, Hq, s) : DKV_OK;
}

template <typename T, typename C, int DH>
int launch_heads(const PagedCache &c, const Plan &p, const void *q, int64_t q_stride, const int *row_off, void *out, void *part, int rows,
                 int max_rows, int Hq, hipStream_t s) {
    if constexpr (sizeof(T) == 4) {
        return launch_split<T, C, DH, 1, 4>(c, p, q, q_stride, row_off, out, part, rows, max_rows, Hq, s);
    } else {
        if constexpr (DH >= 64) {
            if (p.wide == 1) return launch_wide<C, DH, 1>(c, p, q, q_stride, row_off, out, part, rows, max_rows, Hq, s);
            if (p.wide == 2) return launch_wide<C, DH, 2>(c, p, q, q_stride, row_off, out, part, rows, max_rows, Hq, s);
        }
        return p.nq == 1 ? launch_split<T, C, DH, 1, 8>(c, p, q, q_stride, row_off, out, part, rows, max_rows, Hq, s)
                         : launch_split<T, C, DH, 2, 8>(c, p, q, q_stride, row_off, out, part, rows, max_rows, Hq, s);
    }
}

template <typename T, typename C, typename... A> int launch_attn(int head_dim, A... a) {
    return head_dim == 32 ? launch_heads<T, C, 32>(a...) : head_dim == 64 ? launch_heads<T, C, 64>(a...) : launch_heads<T, C, 128>(a...);
}

}  // namespace

int dkv_paged_attn_plan(const dkv_paged_cache *cache, PagedCache &view, PagedAttnPlan &plan, int n_q_heads, int rows, int max_rows_per_seq,
                        int dtype) {
    const int rc = dkv_paged_view(cache, view);
    if (rc) return rc;
    if (!cache->seq_len) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads || rows < 0 || max_rows_per_seq < 0 || rows > (int64_t)cache->batch * max_rows_per_seq) {
        dkv_set_error("inconsistent sizes"); return DKV_E_INVALID_ARG;
    }
    if (dtype != DKV_BF16 && dtype != DKV_FP32) { dkv_set_error("unknown dtype"); return DKV_E_INVALID_ARG; }
    if (cache->dtype != dtype && cache->dtype != DKV_E4M3) { dkv_set_error("rows of dtype %d do not read a cache of dtype %d", dtype, cache->dtype); return DKV_E_UNSUPPORTED; }
    if ((int64_t)rows * n_q_heads < 1 << 24 && (int64_t)cache->batch * cache->n_kv_heads < 1 << 22 &&
        (int64_t)cache->batch * cache->max_pages * cache->page_size <= 1ll << 35) {
        plan = make_plan(view, n_q_heads, rows, max_rows_per_seq, dtype, cache->head_dim);
        if (plan.wide && !plan.split ? plan.blocks < 1 << 23 : split_grid(plan, view) < 1 << 22) return DKV_OK;
    }
    dkv_set_error("%d rows of %d heads in %d sequences are too many for one call", rows, n_q_heads, cache->batch);
    return DKV_E_UNSUPPORTED;
}

extern "C" size_t dkv_paged_attn_workspace_bytes(const dkv_paged_cache *cache, int32_t n_q_heads, int32_t rows,
                                                 int32_t max_rows_per_seq, int32_t dtype) {
    PagedCache c;
    Plan p;
    if (dkv_paged_attn_plan(cache, c, p, n_q_heads, rows, max_rows_per_seq, dtype)) return 0;
    return align_up(most_partial_bytes(c, n_q_heads, rows, max_rows_per_seq, dtype, cache->head_dim) + 256, 256);
}

extern "C" int dkv_paged_attn(const dkv_paged_cache *cache, const void *q, int64_t q_stride, const int32_t *row_off, void *out,
                              int32_t rows, int32_t max_rows_per_seq, int32_t n_q_heads, int32_t dtype, void *workspace,
                              size_t workspace_bytes, void *stream) {
    PagedCache c;
    Plan p;
    int rc = dkv_paged_attn_plan(cache, c, p, n_q_heads, rows, max_rows_per_seq, dtype);
    if (rc || (rc = dkv_paged_check_rows(*cache, row_off, rows))) return rc;
    const int dh = cache->head_dim;
    if (q_stride < (int64_t)n_q_heads * dh) { dkv_set_error("row stride %lld is less than a row", (long long)q_stride); return DKV_E_INVALID_ARG; }
    if (rows == 0) return DKV_OK;
    if (!q || !out) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    const size_t need = partial_bytes(p, c, dh);
    if (need > workspace_bytes || (need && !workspace)) {
        dkv_set_error("workspace has %zu bytes, %zu needed", workspace_bytes, need);
        return DKV_E_WORKSPACE_TOO_SMALL;
    }
    if (need && reinterpret_cast<uintptr_t>(workspace) % 16) { dkv_set_error("workspace must be 16-byte aligned"); return DKV_E_INVALID_ARG; }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int max_rows = max_rows_per_seq < rows ? max_rows_per_seq : rows;
    auto launch = [&](auto f) { return f(dh, c, p, q, q_stride, row_off, out, workspace, rows, max_rows, n_q_heads, s); };
    if (dtype == DKV_BF16)
        return cache->dtype == DKV_BF16 ? launch([](auto... a) { return launch_attn<bf16_t, bf16_t>(a...); })
                                        : launch([](auto... a) { return launch_attn<bf16_t, e4m3_t>(a...); });
    return cache->dtype == DKV_FP32 ? launch([](auto... a) { return launch_attn<float, float>(a...); })
                                    : launch([](auto... a) { return launch_attn<float, e4m3_t>(a...); });
}
