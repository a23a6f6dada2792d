// Page tables that follow the lengths of their sequences (dkv_paged_resize): pages taken from a ring of free ones or given back to it, and
// the new positions listed with their slots.
//
// Everything depends on sums over the sequences before: pages taken, pages given back, new rows. One workgroup forms them (paged_resize_plan, a
// thread per sequence, 1024 at a time), and a launch of many wavefronts writes tables and lists from them (paged_resize_fill). Small calls are
// nothing but latency: there the workgroup goes on with its own wavefronts, in one launch, its sums in LDS. No sum depends on an order, so the
// results do not either.
//
// Entries that give a page back may name none, so these have to be counted before their places in the ring are known: by a launch of its own, a
// wavefront to a sequence (by the one workgroup, a sequence after the other to a wavefront, 512 sequences of 256 pages took 28 us instead of 3 + 3),
// or in the one-launch form by going through all such entries in a row, 4096 at a time.
//
// One launch: 64 sequences, 1000 rows, 4 of them leave 5.8-6.5 us in a trace, the least 4.1: the chain of lengths, barriers, ring or table, stores.
// Three: 512 sequences, 1.9 million rows 16 us (3 + 3 + 9.7; 23 MB written at 2.4 TB/s in the last). There each row of a lane that looked its
// sequence up in memory by itself, with the row before stored between, took 12.4 instead of 9.7.
#include <type_traits>

#include "paged.h"

namespace {

struct Tables {
    int *table, *len, *ring, *ring_at;
    int batch, max_pages, shift;
    uint32_t n_pages;
    __device__ __forceinline__ int pages(int positions) const { return (positions + (1 << shift) - 1) >> shift; }
    __device__ __forceinline__ uint32_t place(uint32_t x) const { return x < n_pages ? x : x - n_pages; }      // of x < 2 n_pages in the ring
    __device__ __forceinline__ bool is_page(int id) const { return (uint32_t)id < n_pages; }
};
struct Lists {
    int *row_off, *positions;
    int64_t *slots;
    int rows;
};
// In the workspace (one launch: in LDS): totals, then arrays of one number for each sequence.
struct Totals {
    uint32_t head, count;        // the free pages of the ring before the call
    int taken, rows;
    uint32_t left;               // see Work::give, all sequences
};
struct Work {
    Totals *totals;
    int *before, *after;         // lengths
    int *take, *row;             // pages taken, new rows of the sequences before
    int *give;                   // pages given back by them (one launch: entries that are cleared, whether they name a page or not)
};

constexpr uint32_t kMost = 0x7fffffff;      // sums end here
__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return min(a + b, kMost); }

// Inclusive sums over a wavefront.
__device__ __forceinline__ uint32_t wave_sums(uint32_t x) {
    auto from = [&](auto control, auto rows, auto zero) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(control)::value, decltype(rows)::value, 0xf, decltype(zero)::value);
    };
    x = add(x, from(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{}, std::true_type{}));
    x = add(x, from(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{}, std::true_type{}));
    x = add(x, from(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{}, std::true_type{}));
    x = add(x, from(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{}, std::true_type{}));
    x = add(x, from(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{}, std::false_type{}));
    x = add(x, from(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{}, std::false_type{}));
    return x;
}

// The number of the lane before, zero in the first.
__device__ __forceinline__ uint32_t lane_before(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x138, 0xf, 0xf, true); }

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// Entries [from, to) of a sequence's row of the table, 256 at a time by a whole wavefront: f(entry, whether it is one, its index).
template <typename F> __device__ __forceinline__ void each_entry(const int *row, int from, int to, F f) {
    const int lane = threadIdx.x & 63;
    for (int j = from; j < to; j += 256) {
        int id[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) id[u] = row[min(j + 64 * u + lane, to - 1)];
#pragma unroll
        for (int u = 0; u < 4; ++u) f(id[u], j + 64 * u + lane < to, j + 64 * u + lane);
    }
}

// The sequences of the items x and y: the last ones with first[b] <= x, and y. Whole wavefronts, x and y uniform; 64 sequences are asked at once, for both.
__device__ __forceinline__ void find(const int *first, int batch, int x, int y, int &bx, int &by) {
    const int lane = threadIdx.x & 63;
    int lo[2] = {0, 0}, n[2] = {batch, batch};
    const int item[2] = {x, y};
    while (n[0] > 1 || n[1] > 1) {
        int at[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) at[i] = first[lo[i] + min(lane * ((n[i] + 63) >> 6), n[i] - 1)];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int step = (n[i] + 63) >> 6, k = __popcll(__ballot(lane * step < n[i] && at[i] <= item[i])) - 1;
            lo[i] += k * step;
            n[i] = min(step, n[i] - k * step);
        }
    }
    bx = __builtin_amdgcn_readfirstlane(lo[0]);
    by = __builtin_amdgcn_readfirstlane(lo[1]);
}
__device__ __forceinline__ int find_between(const int *first, int lo, int hi, int x) {
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Lengths of sequence b before the call and wanted.
__device__ __forceinline__ void lengths_of(const Tables &t, const int *lengths, int b, int &old, int &now) {
    old = min(max(t.len[b], 0), t.max_pages << t.shift);
    now = lengths[b];
    if (now < 0 || now > t.max_pages << t.shift) now = old;
}
__device__ __forceinline__ void move_ring(const Tables &t, const Totals &all, uint32_t given) {
    t.ring_at[0] = (int)t.place(all.head + all.taken);
    t.ring_at[1] = (int)(min(given, t.n_pages - all.count) + (all.count - all.taken));
}
// Pages that a sequence gives back, of its entries [from, to).
__device__ __forceinline__ int count_pages(const Tables &t, int b, int from, int to) {
    int n = 0;
    each_entry(t.table + (size_t)b * t.max_pages, from, to, [&](int id, bool is, int) { n += __popcll(__ballot(is && t.is_page(id))); });
    return n;
}

// COUNTED: w.give has the pages that each sequence gives back (paged_resize_count), otherwise the ring's new place is left to give_entries.
template <bool COUNTED> __device__ __forceinline__ void plan(const Tables &t, const int *lengths, const Lists &l, const Work &w) {
    __shared__ uint32_t sums[3][kWaves];
    __shared__ int most[2];                      // pages and rows of the sequences that fit
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t head = (uint32_t)t.ring_at[0] % t.n_pages;
    const uint32_t count = (uint32_t)min(max(t.ring_at[1], 0), (int)t.n_pages);
    const uint32_t rows_most = (uint32_t)l.rows;
    uint32_t pages_before = 0, rows_before = 0, given_before = 0;
    if (tid < 2) most[tid] = -1;
    for (int base = 0; base < t.batch; base += kThreads) {
        const int b = base + tid;
        const bool here = b < t.batch;
        int old = 0, now = 0;
        if (here) lengths_of(t, lengths, b, old, now);
        const int have = t.pages(old);
        const uint32_t pages = max(t.pages(now) - have, 0), rows = l.row_off ? max(now - old, 0) : 0;
        const uint32_t gives = COUNTED ? (here ? (uint32_t)w.give[b] : 0) : max(have - t.pages(now), 0);
        const uint32_t pages_upto = wave_sums(pages), rows_upto = wave_sums(rows), given_upto = wave_sums(gives);
        if (lane == 63) {
            sums[0][wave] = pages_upto;
            sums[1][wave] = rows_upto;
            sums[2][wave] = given_upto;
        }
        __syncthreads();
        const uint32_t p = wave_sums(lane < kWaves ? sums[0][lane & (kWaves - 1)] : 0), r = wave_sums(lane < kWaves ? sums[1][lane & (kWaves - 1)] : 0),
                       g = wave_sums(lane < kWaves ? sums[2][lane & (kWaves - 1)] : 0);
        auto upto = [&](uint32_t x, int i) { return (uint32_t)__builtin_amdgcn_readlane((int)x, i); };
        const uint32_t pages_first = add(pages_before, wave ? upto(p, wave - 1) : 0), rows_first = add(rows_before, wave ? upto(r, wave - 1) : 0),
                       given_first = add(given_before, wave ? upto(g, wave - 1) : 0);
        pages_before = add(pages_before, upto(p, kWaves - 1));
        rows_before = add(rows_before, upto(r, kWaves - 1));
        given_before = add(given_before, upto(g, kWaves - 1));
        // Sums only grow: from the first sequence that does not fit on none does. That one says what all before it take. (A sum that has reached
        // kMost is more than there are pages and rows.)
        const uint32_t p1 = add(pages_first, pages_upto), r1 = add(rows_first, rows_upto);
        const uint32_t p0 = add(pages_first, lane_before(pages_upto)), r0 = add(rows_first, lane_before(rows_upto));
        const bool fits = p1 <= count && r1 <= rows_most;
        if (here && !fits && p0 <= count && r0 <= rows_most) {
            most[0] = (int)p0;
            most[1] = (int)r0;
        }
        __syncthreads();
        if (here) {
            const int after = now > old && !fits ? old : now;
            t.len[b] = after;
            w.before[b] = old;
            w.after[b] = after;
            w.take[b] = fits ? (int)p0 : most[0];
            w.row[b] = fits ? (int)r0 : most[1];
            w.give[b] = (int)(add(given_first, given_upto) - gives);
            if (l.row_off) l.row_off[b + 1] = fits ? (int)r1 : most[1];
        }
        __syncthreads();
    }
    if (tid == 0) {
        const int taken = most[0] < 0 ? (int)pages_before : most[0], rows = most[0] < 0 ? (int)rows_before : most[1];
        *w.totals = Totals{head, count, taken, rows, given_before};
        if (l.row_off) l.row_off[0] = 0;
        if constexpr (COUNTED) move_ring(t, *w.totals, given_before);
    }
}

// The parts of the work are independent of each other; each for wavefront `wave` of `waves`.
// Without lists of the new positions.
__device__ __forceinline__ void take_pages(const Tables &t, const Work &w, int wave, int waves) {
    const int lane = threadIdx.x & 63;
    const Totals all = *w.totals;
    for (int x = wave * 64; x < all.taken; x += waves * 64) {
        const int mine = x + lane;
        int b0, b1;
        find(w.take, t.batch, x, min(x + 63, all.taken - 1), b0, b1);
        if (mine < all.taken) {
            const int b = find_between(w.take, b0, b1, mine);
            t.table[(size_t)b * t.max_pages + t.pages(w.before[b]) + mine - w.take[b]] = t.ring[t.place(all.head + mine)];
        }
    }
}
// Four rows to a lane (eight: 1.9 million rows 15.2 us instead of 13.6). The first position of a new page is one of them: it writes the table's entry.
__device__ __forceinline__ void list_rows(const Tables &t, const Lists &l, const Work &w, int wave, int waves) {
    constexpr int N = 4;
    const int lane = threadIdx.x & 63;
    const Totals all = *w.totals;
    for (int x = wave * 64 * N; x < all.rows; x += waves * 64 * N) {
        int b0, b1, b[N], old[N], row[N], take[N], p[N], id[N], entry[N];      // entry: of the table, -1 where it is there already
        find(w.row, t.batch, x, min(x + 64 * N - 1, all.rows - 1), b0, b1);
        if (b1 - b0 < 64) {                                // a lane reads what there is of one sequence, for all rows of the wavefront
            const int mine = min(b0 + lane, b1), olds = w.before[mine], rows = w.row[mine], takes = w.take[mine];
#pragma unroll
            for (int u = 0; u < N; ++u) b[u] = 0;
            for (int step = 32; step > 0; step >>= 1) {
                if (step > b1 - b0) continue;              // uniform
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    const int i = b[u] + step, first = __builtin_amdgcn_ds_bpermute(min(i, b1 - b0) << 2, rows);       // by all lanes
                    if (i <= b1 - b0 && first <= x + 64 * u + lane) b[u] = i;
                }
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                old[u] = __builtin_amdgcn_ds_bpermute(b[u] << 2, olds);
                row[u] = __builtin_amdgcn_ds_bpermute(b[u] << 2, rows);
                take[u] = __builtin_amdgcn_ds_bpermute(b[u] << 2, takes);
                b[u] += b0;
            }
        } else {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                b[u] = find_between(w.row, b0, b1, min(x + 64 * u + lane, all.rows - 1));
                old[u] = w.before[b[u]], row[u] = w.row[b[u]], take[u] = w.take[b[u]];
            }
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            p[u] = old[u] + min(x + 64 * u + lane, all.rows - 1) - row[u];
            const int j = p[u] >> t.shift, have = t.pages(old[u]), at = b[u] * t.max_pages + j;
            id[u] = *(j < have ? t.table + at : t.ring + t.place(all.head + take[u] + j - have));
            entry[u] = j >= have && !(p[u] & ((1 << t.shift) - 1)) ? at : -1;
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int r = x + 64 * u + lane;
            if (r >= all.rows) continue;
            if (entry[u] >= 0) t.table[entry[u]] = id[u];
            if (l.positions) l.positions[r] = p[u];
            if (l.slots) l.slots[r] = t.is_page(id[u]) ? ((int64_t)id[u] << t.shift) + (p[u] & ((1 << t.shift) - 1)) : -1;
        }
    }
}
// To the end of the ring, a sequence at a time.
__device__ __forceinline__ void give_pages(const Tables &t, const Work &w, int wave, int waves) {
    const int lane = threadIdx.x & 63;
    const Totals all = *w.totals;
    for (int base = 0; base < t.batch; base += 64 * waves) {
        const int b = base + lane * waves + wave;
        const int need = b < t.batch ? t.pages(w.after[b]) : 0, have = b < t.batch ? t.pages(w.before[b]) : 0;
        unsigned long long left = __ballot(need < have);
        while (left) {
            const int i = __builtin_ctzll(left), seq = base + i * waves + wave;
            left &= left - 1;
            int at = w.give[seq];
            int *row = t.table + (size_t)seq * t.max_pages;
            each_entry(row, __builtin_amdgcn_readlane(need, i), __builtin_amdgcn_readlane(have, i), [&](int id, bool is, int j) {
                const bool page = is && t.is_page(id);
                const unsigned long long pages = __ballot(page);
                const uint32_t n = at + __popcll(pages & ((1ull << lane) - 1));
                if (page && n < t.n_pages - all.count) t.ring[t.place(t.place(all.head + all.count) + n)] = id;
                if (is) row[j] = -1;
                at += __popcll(pages);
            });
        }
    }
}

// The same by a whole workgroup for all entries in a row, where nobody has counted the pages among them: 4 kThreads at a time.
__device__ __forceinline__ void give_entries(const Tables &t, const Work &w) {
    static_assert(4 * kWaves == 64, "a count for each lane");
    __shared__ int counts[4 * kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Totals all = *w.totals;
    uint32_t given = 0;
    for (uint32_t x = 0; x < all.left; x += 4 * kThreads) {
        int *entry[4], id[4];
        unsigned long long pages[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t begin = x + u * kThreads + wave * 64, mine = begin + lane;
            entry[u] = nullptr;
            if (begin < all.left) {                       // uniform
                int b0, b1;
                find(w.give, t.batch, (int)begin, (int)min(begin + 63, all.left - 1), b0, b1);
                const int b = find_between(w.give, b0, b1, (int)min(mine, all.left - 1));
                if (mine < all.left) entry[u] = t.table + (size_t)b * t.max_pages + t.pages(w.after[b]) + ((int)mine - w.give[b]);
            }
            id[u] = entry[u] ? *entry[u] : -1;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            pages[u] = __ballot(t.is_page(id[u]));
            if (lane == 0) counts[u * kWaves + wave] = __popcll(pages[u]);
        }
        __syncthreads();
        const uint32_t upto = wave_sums((uint32_t)counts[lane]);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t before = u * kWaves + wave ? (uint32_t)__builtin_amdgcn_readlane((int)upto, max(u * kWaves + wave - 1, 0)) : 0;
            const uint32_t n = given + before + __popcll(pages[u] & ((1ull << lane) - 1));
            if (t.is_page(id[u]) && n < t.n_pages - all.count) t.ring[t.place(t.place(all.head + all.count) + n)] = id[u];
            if (entry[u]) *entry[u] = -1;
        }
        given += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        __syncthreads();
    }
    if (tid == 0) move_ring(t, all, given);
}

__global__ __launch_bounds__(256) void paged_resize_count(Tables t, const int *lengths, Work w) {
    const int b = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (b >= t.batch) return;
    int old, now;
    lengths_of(t, lengths, b, old, now);
    const int n = count_pages(t, b, t.pages(now), t.pages(old));
    if ((threadIdx.x & 63) == 0) w.give[b] = n;
}
__global__ __launch_bounds__(kThreads) void paged_resize_plan(Tables t, const int *lengths, Lists l, Work w) { plan<true>(t, lengths, l, w); }
__global__ __launch_bounds__(256) void paged_resize_fill(Tables t, Lists l, Work w, int takers) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), block = (int)blockIdx.x;
    if (block >= takers) give_pages(t, w, (block - takers) * 4 + wave, ((int)gridDim.x - takers) * 4);
    else if (l.row_off) list_rows(t, l, w, block * 4 + wave, takers * 4);
    else take_pages(t, w, block * 4 + wave, takers * 4);
}
// Up to kThreads sequences, all in one workgroup.
__global__ __launch_bounds__(kThreads) void paged_resize_small(Tables t, const int *lengths, Lists l) {
    __shared__ int arrays[5][kThreads];
    __shared__ Totals totals;
    const Work w = {&totals, arrays[0], arrays[1], arrays[2], arrays[3], arrays[4]};
    plan<false>(t, lengths, l, w);
    __syncthreads();
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (l.row_off) list_rows(t, l, w, wave, kWaves);
    else take_pages(t, w, wave, kWaves);
    give_entries(t, w);
}

constexpr int kMostSequences = 1 << 20;
constexpr size_t kTotalsBytes = 32;
static_assert(sizeof(Totals) <= kTotalsBytes, "totals lie in front of the arrays");
size_t work_bytes(int batch) { return kTotalsBytes + 5 * sizeof(int) * (size_t)batch; }

}  // namespace

// By what the host knows, rows of the lists and entries of the tables that can move, in one launch and in three, us in a graph:
//   rows: 4096 4.4 and -, 8192 6.3-8.2 and 7-10, 16384 8.8-14.5 and 7.1-9.7, 65536 31-39 and 8.1-9.3.
//   entries without lists, where moving many is what a call is for. 64 sequences that leave: 64 pages each 5.3 and 7.7, 128 8.1 and 7.7, 256 13.4 and
//     8.0; that take them 4.8 and 7.4, 6.7 and 7.4, 10.8 and 7.2. 512 sequences: 4 pages 5.6 and 8.1 (4.4 and 7.6), 16 11.4 and 7.9 (9.8 and 8.2), 256
//     119 and 8.4 (92 and 8.4); 1024 of 2048 pages 2088 and 23.
//   entries with a list of a few rows, a server's step, which seldom moves more than a page for each sequence (4.0 and 7.1, with 512 sequences 6.1 and
//     10.6, however wide the tables) but can give all back: 64 sequences of 1024 pages 46 and 13, of 4096 176 and 28; 512 of 64 32 and 8.6, of 256
//     119 and 8.6; 1024 of 64 69 and 9.4.
// A sequence gives its pages back by one wavefront in the three-launch form, 4 us for 1024 of them and 0.65 in the other (one of 4096 pages 4.4 and 20,
// 16 of 4096 45 and 24): the pages of six sequences do not count.
int dkv_paged_resize_launches(const dkv_paged_tables &c, bool listed, int rows) {
    const int64_t entries = (int64_t)c.batch * c.max_pages, move = (entries < c.n_pages ? entries : c.n_pages) - 6 * (int64_t)c.max_pages;
    return c.batch <= kThreads && (!listed || rows <= 8192) && move <= (listed ? 65536 : 6144) ? 1 : 3;
}

extern "C" size_t dkv_paged_resize_workspace_bytes(int32_t batch) {
    if (batch < 1 || batch > kMostSequences) { dkv_set_error("%d sequences: 1 to %d are expected", batch, kMostSequences); return 0; }
    return work_bytes(batch);
}

extern "C" int dkv_paged_resize(const dkv_paged_tables *tables, const int32_t *lengths, int32_t *row_off, int32_t *positions, int64_t *slots,
                                int32_t rows, void *workspace, size_t workspace_bytes, void *stream) {
    if (!tables || !tables->page_table || !tables->seq_len || !tables->free_pages || !tables->free_at || !lengths) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    const dkv_paged_tables &c = *tables;
    if (c.batch < 1 || c.n_pages < 1 || c.max_pages < 1 || rows < 0) { dkv_set_error("inconsistent sizes"); return DKV_E_INVALID_ARG; }
    if (c.page_size < 16 || c.page_size > 65536 || (c.page_size & (c.page_size - 1))) {
        dkv_set_error("page_size %d not supported (a power of two, 16 to 65536)", c.page_size); return DKV_E_UNSUPPORTED;
    }
    if ((int64_t)c.max_pages * c.page_size > 1 << 30) { dkv_set_error("the table covers more than 2^30 positions"); return DKV_E_UNSUPPORTED; }
    if ((int64_t)c.batch * c.max_pages >= 1ll << 31) { dkv_set_error("tables of 2^31 entries and more are not supported"); return DKV_E_UNSUPPORTED; }
    if (c.n_pages > 1 << 30 || c.batch > kMostSequences || rows > 1 << 30) { dkv_set_error("%d pages, %d sequences or %d rows are too many for one call", c.n_pages, c.batch, rows); return DKV_E_UNSUPPORTED; }
    if ((positions || slots) && !row_off) { dkv_set_error("positions and slots go with row_off"); return DKV_E_INVALID_ARG; }
    if (!workspace || workspace_bytes < work_bytes(c.batch)) {
        dkv_set_error("workspace has %zu bytes, %zu needed", workspace ? workspace_bytes : 0, work_bytes(c.batch));
        return DKV_E_WORKSPACE_TOO_SMALL;
    }
    if (reinterpret_cast<uintptr_t>(workspace) % 16) { dkv_set_error("workspace must be 16-byte aligned"); return DKV_E_INVALID_ARG; }
    const Tables t = {c.page_table, c.seq_len, c.free_pages, c.free_at, c.batch, c.max_pages, __builtin_ctz((unsigned)c.page_size), (uint32_t)c.n_pages};
    const Lists l = {row_off, positions, slots, rows};      // no rows are counted without row_off
    int *arrays = reinterpret_cast<int *>(static_cast<char *>(workspace) + kTotalsBytes);
    const Work w = {static_cast<Totals *>(workspace), arrays, arrays + c.batch, arrays + 2 * (size_t)c.batch, arrays + 3 * (size_t)c.batch, arrays + 4 * (size_t)c.batch};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dkv_paged_resize_launches(c, row_off != nullptr, rows) == 1) {
        hipLaunchKernelGGL(paged_resize_small, dim3(1), dim3(kThreads), 0, s, t, lengths, l);
        DKV_LAUNCH_CHECK();
        return DKV_OK;
    }
    hipLaunchKernelGGL(paged_resize_count, dim3((unsigned)((c.batch + 3) / 4)), dim3(256), 0, s, t, lengths, w);
    DKV_LAUNCH_CHECK();
    hipLaunchKernelGGL(paged_resize_plan, dim3(1), dim3(kThreads), 0, s, t, lengths, l, w);
    DKV_LAUNCH_CHECK();
    // a wavefront for 256 rows or 64 pages that are taken, and for a sequence that gives some, up to what runs at once
    const int64_t pages = (int64_t)c.batch * c.max_pages < c.n_pages ? (int64_t)c.batch * c.max_pages : c.n_pages;
    auto blocks = [](int64_t waves) { return (int)(waves < 8192 ? (waves + 3) / 4 : 2048); };
    const int takers = blocks(row_off ? ((int64_t)rows + 255) / 256 : (pages + 63) / 64);
    hipLaunchKernelGGL(paged_resize_fill, dim3((unsigned)(takers + blocks(c.batch))), dim3(256), 0, s, t, l, w, takers);
    DKV_LAUNCH_CHECK();
    return DKV_OK;
}
