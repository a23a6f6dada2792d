// Page tables that follow the lengths of their sequences (dkv_paged_resize): pages taken from a ring of free ones or given back to it, and
// the new positions listed with their slots.
//
// Everything depends on sums over the sequences before: pages taken, pages given back, new rows. One workgroup forms them (paged_resize_plan, a
// thread per sequence, 1024 at a time), and a launch of many wavefronts writes tables and lists from them (paged_resize_fill). Small calls
// are nothing but latency: there the workgroup goes on with its own wavefronts, in one launch. No sum depends on an order, so the results do not either.
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
// In the workspace: `head`, then arrays of one number for each sequence.
struct Totals {
    uint32_t head, count;        // the free pages of the ring before the call
    int taken, rows;
};
struct Work {
    Totals *totals;
    int *before, *after;         // lengths
    int *take, *give, *row;      // pages taken, pages given back, new rows of the sequences before
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

// The sequence of item x: the last one with first[b] <= x. Whole wavefronts, x uniform; 64 of them are asked at once.
__device__ __forceinline__ int find(const int *first, int n, int x) {
    const int lane = threadIdx.x & 63;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) >> 6;
        const int k = __popcll(__ballot(lane * step < n && first[lo + min(lane * step, n - 1)] <= x)) - 1;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
__device__ __forceinline__ int find_between(const int *first, int lo, int hi, int x) {
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ void plan(const Tables &t, const int *lengths, const Lists &l, const Work &w) {
    __shared__ int from[kThreads], to[kThreads], given[kThreads];
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
        if (here) {
            old = min(max(t.len[b], 0), t.max_pages << t.shift);
            now = lengths[b];
            if (now < 0 || now > t.max_pages << t.shift) now = old;
        }
        const int have = t.pages(old);
        const uint32_t pages = max(t.pages(now) - have, 0), rows = l.row_off ? max(now - old, 0) : 0;
        from[tid] = t.pages(now);
        to[tid] = have;
        given[tid] = 0;
        __syncthreads();
        // pages given back, where entries may be missing: the wavefronts take the sequences in turn
        {
            const int mine = lane * kWaves + wave;
            unsigned long long left = __ballot(from[mine] < to[mine]);
            while (left) {
                const int i = __builtin_ctzll(left) * kWaves + wave;
                left &= left - 1;
                int n = 0;
                each_entry(t.table + (size_t)(base + i) * t.max_pages, from[i], to[i], [&](int id, bool is, int) { n += __popcll(__ballot(is && t.is_page(id))); });
                if (lane == 0) given[i] = n;
            }
        }
        uint32_t pages_upto = wave_sums(pages), rows_upto = wave_sums(rows);
        __syncthreads();
        const uint32_t gives = given[tid];
        uint32_t given_upto = wave_sums(gives);
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
        *w.totals = Totals{head, count, taken, rows};
        if (l.row_off) l.row_off[0] = 0;
        t.ring_at[0] = (int)t.place(head + taken);
        t.ring_at[1] = (int)(min(given_before, t.n_pages - count) + (count - taken));
    }
}

// Wavefront `wave` of `waves`.
__device__ void fill(const Tables &t, const Lists &l, const Work &w, int wave, int waves) {
    const int lane = threadIdx.x & 63;
    const Totals all = *w.totals;
    // pages taken
    for (int x = wave * 64; x < all.taken; x += waves * 64) {
        const int b0 = find(w.take, t.batch, x), b1 = find(w.take, t.batch, min(x + 63, all.taken - 1)), mine = x + lane;
        if (mine < all.taken) {
            const int b = find_between(w.take, b0, b1, mine);
            t.table[(size_t)b * t.max_pages + t.pages(w.before[b]) + mine - w.take[b]] = t.ring[t.place(all.head + mine)];
        }
    }
    // new rows, four to a lane
    for (int x = wave * 256; x < all.rows; x += waves * 256) {
        const int b0 = find(w.row, t.batch, x), b1 = find(w.row, t.batch, min(x + 255, all.rows - 1));
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = x + 64 * u + lane;
            if (r >= all.rows) continue;
            const int b = find_between(w.row, b0, b1, r), old = w.before[b], p = old + r - w.row[b];
            if (l.positions) l.positions[r] = p;
            if (l.slots) {
                const int j = p >> t.shift, have = t.pages(old);
                const int id = j < have ? t.table[(size_t)b * t.max_pages + j] : t.ring[t.place(all.head + w.take[b] + j - have)];
                l.slots[r] = t.is_page(id) ? ((int64_t)id << t.shift) + (p & ((1 << t.shift) - 1)) : -1;
            }
        }
    }
    // pages given back: behind the end of the ring
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

__global__ __launch_bounds__(kThreads) void paged_resize_plan(Tables t, const int *lengths, Lists l, Work w) { plan(t, lengths, l, w); }
__global__ __launch_bounds__(256) void paged_resize_fill(Tables t, Lists l, Work w) {
    fill(t, l, w, (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), (int)gridDim.x * 4);
}
__global__ __launch_bounds__(kThreads) void paged_resize_small(Tables t, const int *lengths, Lists l, Work w) {
    plan(t, lengths, l, w);
    __syncthreads();
    fill(t, l, w, __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), kWaves);
}

constexpr int kMostSequences = 1 << 20;
size_t work_bytes(int batch) { return 16 + 5 * sizeof(int) * (size_t)batch; }

}  // namespace

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
    if (c.n_pages > 1 << 30 || c.batch > kMostSequences || rows > 1 << 30) { dkv_set_error("%d pages, %d sequences or %d rows are too many for one call", c.n_pages, c.batch, rows); return DKV_E_UNSUPPORTED; }
    if ((positions || slots) && !row_off) { dkv_set_error("positions and slots go with row_off"); return DKV_E_INVALID_ARG; }
    if (!workspace || workspace_bytes < work_bytes(c.batch)) {
        dkv_set_error("workspace has %zu bytes, %zu needed", workspace ? workspace_bytes : 0, work_bytes(c.batch));
        return DKV_E_WORKSPACE_TOO_SMALL;
    }
    if (reinterpret_cast<uintptr_t>(workspace) % 16) { dkv_set_error("workspace must be 16-byte aligned"); return DKV_E_INVALID_ARG; }
    const Tables t = {c.page_table, c.seq_len, c.free_pages, c.free_at, c.batch, c.max_pages, __builtin_ctz((unsigned)c.page_size), (uint32_t)c.n_pages};
    const Lists l = {row_off, positions, slots, rows};      // no rows are counted without row_off
    int *arrays = reinterpret_cast<int *>(static_cast<char *>(workspace) + 16);
    const Work w = {static_cast<Totals *>(workspace), arrays, arrays + c.batch, arrays + 2 * (size_t)c.batch, arrays + 3 * (size_t)c.batch, arrays + 4 * (size_t)c.batch};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (c.batch <= kThreads && (!row_off || rows <= 8192)) {
        hipLaunchKernelGGL(paged_resize_small, dim3(1), dim3(kThreads), 0, s, t, lengths, l, w);
        DKV_LAUNCH_CHECK();
        return DKV_OK;
    }
    hipLaunchKernelGGL(paged_resize_plan, dim3(1), dim3(kThreads), 0, s, t, lengths, l, w);
    DKV_LAUNCH_CHECK();
    hipLaunchKernelGGL(paged_resize_fill, dim3(512), dim3(256), 0, s, t, l, w);
    DKV_LAUNCH_CHECK();
    return DKV_OK;
}
