// Rotary positions of rows of queries and keys (dkv_rope): each pair (a, b) of a head becomes c (a cos t - b sin t, b cos t + a sin t) with
// t = position * frequency of the pair.
//
// Bound by the traffic, each element read and written once: the angles must not cost as much as that. A lane has V pairs of one row and
// works through its heads, so their cosines are computed once for all of them. Angles of far positions need more than 32 bits (2^20
// positions at one radian each: an fp32 product is off by 2^-4): position times frequency, in quarter turns, and what is left of it in the
// quarter are formed in 64 bits, sine and cosine of that from their Taylor series in 32.
//
// 6144 rows of 64 heads of 128 in bf16 (201 MB) 35.7 us in place, 39.4 into other memory (5.1 TB/s; a large copy 4.46), 2048 in fp32 21.9 and 25.8;
// 64 rows 3.4 us, the call is 5.5 us of the host. Neighbouring pairs in one piece of 32 bytes a lane, every other 16 to a load, took 30.1 us instead of
// 27.0 (4099 rows of 32 heads in fp32, 64 dims). Part of a head into other memory moves all of it, in place all is read and what turns is written: 64
// and 32 dims of 128 26 and 24 us. Where the pairs of a head are no multiple of 4 (neighbouring ones: of 2) a lane has one pair, and these rows take 41
// to 58.
//
// The results are written into the caches: the next launches of a layer read them. With the non-temporal hint rope alone is faster in some calls
// (6144 rows in bf16 into other memory 39.8 -> 35.3 us, in place 35.7 -> 34.4, but with 28 and 4 heads 17.1 -> 19.2, 32 of 128 dims into other
// memory 41 -> 47), not with its readers: stored into a cache and attended to 242 -> 246, in place 241.5 -> 242.5, 1024 rows 55.2 -> 55.3 and
// 54.7 -> 55.0, 512 rows 47.0 -> 48.0 and 46.9 -> 47.0; with a copy of the results 57 -> 61.
#include <math.h>

#include <type_traits>

#include "paged.h"

namespace {

template <typename T> struct RopeArgs {
    const T *q, *k;
    T *q_out, *k_out;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;
    const int *positions, *row_off;
    int batch, rows, n_q, heads;           // heads: of q and k
    int head_dim, half, lanes;             // half: pairs of a head; lanes (log2) that have a head
    Divisor parts{1};                      // wavefronts of a row
    float scale, way;                      // way: -1 turns back
    double quarters[64];                   // quarter turns of a pair for one position
};

// V elements at any address that is aligned to an element
template <typename T, int V> struct Bits;
template <> struct Bits<bf16_t, 8> { typedef bf16x8_el at; typedef u32x4 type; };
template <> struct Bits<bf16_t, 4> { typedef bf16x4_el at; typedef u32x2 type; };
template <> struct Bits<bf16_t, 1> { typedef bf16_t at; typedef bf16_t type; };
template <> struct Bits<float, 4> { typedef f32x4_el at; typedef f32x4 type; };
template <> struct Bits<float, 1> { typedef float at; typedef float type; };

template <int V> struct Floats { float x[V]; };
__device__ __forceinline__ Floats<1> widen(bf16_t a) { return {bf2f(a)}; }
__device__ __forceinline__ Floats<1> widen(float a) { return {a}; }
__device__ __forceinline__ Floats<4> widen(f32x4 a) { return {a[0], a[1], a[2], a[3]}; }
template <int N> struct Words { uint32_t w[N]; };
template <typename W> __device__ __forceinline__ Floats<(int)sizeof(W) / 2> widen(W a) {         // words of two bf16
    const Words<(int)sizeof(W) / 4> u = __builtin_bit_cast(Words<(int)sizeof(W) / 4>, a);
    Floats<(int)sizeof(W) / 2> y;
#pragma unroll
    for (int i = 0; i < (int)sizeof(W) / 4; ++i) {
        y.x[2 * i] = __uint_as_float(u.w[i] << 16);
        y.x[2 * i + 1] = __uint_as_float(u.w[i] & 0xffff0000u);
    }
    return y;
}
__device__ __forceinline__ void narrow(Floats<1> a, bf16_t &b) { b = f2bf(a.x[0]); }
__device__ __forceinline__ void narrow(Floats<1> a, float &b) { b = a.x[0]; }
__device__ __forceinline__ void narrow(Floats<4> a, f32x4 &b) { b = f32x4{a.x[0], a.x[1], a.x[2], a.x[3]}; }
template <int V, typename W> __device__ __forceinline__ void narrow(Floats<V> a, W &b) {
    Words<V / 2> u;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) u.w[i] = (uint32_t)f2bf(a.x[2 * i]) | ((uint32_t)f2bf(a.x[2 * i + 1]) << 16);
    b = __builtin_bit_cast(W, u);
}

// Cosine and sine of a number of quarter turns. What is left of it is at most half a quarter, where the first terms that are left out are
// below 2^-28.
__device__ __forceinline__ void cos_sin(double quarters, float &c, float &s) {
    const double whole = rint(quarters);
    const float f = (float)((quarters - whole) * 1.5707963267948966), y = f * f;
    const int n = (int)(whole - 4.0 * floor(0.25 * whole));
    const float sn = fmaf(f * y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), f);
    const float cs = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    c = n & 1 ? sn : cs;
    s = n & 1 ? cs : sn;
    if ((n + 1) & 2) c = -c;
    if (n & 2) s = -s;
}

// A wavefront has H times 64 >> lanes heads of a row, a lane two pieces of V elements of each: pieces that hold V pairs (i, i + half), or with PAIRS
// the pieces `piece` and 1 << lanes further on, of V / 2 pairs (2 i, 2 i + 1) each (V = 1: the two elements of a pair). The dims behind the pairs are copied.
template <typename T, int V, bool PAIRS, int H>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs<T> a) {
    typedef Bits<T, V> B;
    constexpr bool WITHIN = PAIRS && V > 1;            // pairs within a piece
    const int id = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = a.parts.div(id), piece = lane & ((1 << a.lanes) - 1), at_once = 64 >> a.lanes;
    const int first = a.parts.mod(id) * H * at_once + (lane >> a.lanes);
    if (r >= a.rows || (a.row_off && r >= a.row_off[a.batch])) return;
    const int ahead = V << a.lanes, behind = 2 * V * piece - 2 * a.half;          // behind: of a piece of pairs (i, i + half) after all of them
    const int lo = WITHIN ? V * piece : PAIRS || behind >= 0 ? 2 * V * piece : V * piece;
    const int hi = WITHIN ? lo + ahead : PAIRS || behind >= 0 ? lo + V : lo + a.half;
    const bool turn_lo = WITHIN ? lo < 2 * a.half : behind < 0, turn_hi = WITHIN ? hi < 2 * a.half : behind < 0;
    typename B::type x[H], y[H];
#pragma unroll
    for (int i = 0; i < H; ++i) {
        const int h = min(first + i * at_once, a.heads - 1);
        const T *p = h < a.n_q ? a.q + r * a.q_stride + h * a.head_dim : a.k + r * a.k_stride + (h - a.n_q) * a.head_dim;
        x[i] = *reinterpret_cast<const typename B::at *>(p + lo);
        y[i] = *reinterpret_cast<const typename B::at *>(p + hi);
    }
    const double position = a.positions[r];
    float c[V], s[V];                                  // WITHIN: of lo's pairs, then of hi's
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int pair = WITHIN ? ((2 * e < V ? lo : hi) >> 1) + e % ((V + 1) / 2) : V * piece + e;
        cos_sin(position * a.quarters[min(pair, a.half - 1)], c[e], s[e]);
        c[e] *= a.scale;
        s[e] *= a.scale * a.way;
    }
#pragma unroll
    for (int i = 0; i < H; ++i) {
        const int h = first + i * at_once;
        if (h >= a.heads) return;
        const bool is_q = h < a.n_q, moves = (is_q ? a.q : a.k) != (is_q ? a.q_out : a.k_out);
        T *p = is_q ? a.q_out + r * a.q_out_stride + h * a.head_dim : a.k_out + r * a.k_out_stride + (h - a.n_q) * a.head_dim;
        const Floats<V> u = widen(x[i]), w = widen(y[i]);
        Floats<V> m, n;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int k = 2 * e % V;                   // WITHIN: pair e is elements k and k + 1 of a piece
            const float p0 = !WITHIN ? u.x[e] : 2 * e < V ? u.x[k] : w.x[k], p1 = !WITHIN ? w.x[e] : 2 * e < V ? u.x[(k + 1) % V] : w.x[(k + 1) % V];
            const float r0 = p0 * c[e] - p1 * s[e], r1 = p1 * c[e] + p0 * s[e];
            (WITHIN && 2 * e >= V ? n : m).x[WITHIN ? k : e] = r0;
            (WITHIN && 2 * e < V ? m : n).x[WITHIN ? (k + 1) % V : e] = r1;
        }
        if (turn_lo) narrow(m, x[i]);
        if (turn_hi) narrow(n, y[i]);
        if (turn_lo || moves) *reinterpret_cast<typename B::at *>(p + lo) = x[i];
        if (turn_hi || moves) *reinterpret_cast<typename B::at *>(p + hi) = y[i];
    }
}

template <typename T, int V> int launch(RopeArgs<T> &a, bool pairs, hipStream_t s) {
    a.lanes = __builtin_ctz((unsigned)(a.head_dim / (2 * V)));
    const int n = dkv_rope_lane_heads(sizeof(T) == 2 ? DKV_BF16 : DKV_FP32, V, a.head_dim, a.heads, a.rows);
    if (!n) { dkv_set_error("%d rows of %d heads are too many for one call", a.rows, a.heads); return DKV_E_UNSUPPORTED; }
    const int parts = ceil_div(a.heads, n * (64 >> a.lanes));
    a.parts = Divisor(parts);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)(((int64_t)parts * a.rows + 3) / 4)), dim3(256), 0, s, a);
        DKV_LAUNCH_CHECK();
        return DKV_OK;
    };
    if (pairs) return n == 4 ? go(rope_kernel<T, V, true, 4>) : go(rope_kernel<T, V, true, 1>);
    return n == 4 ? go(rope_kernel<T, V, false, 4>) : go(rope_kernel<T, V, false, 1>);
}

bool rope_ok(const dkv_rope_desc &d) {
    if (d.head_dim != 32 && d.head_dim != 64 && d.head_dim != 128) { dkv_set_error("head_dim %d not supported (32, 64, 128)", d.head_dim); return false; }
    if (d.rot_dim < 2 || d.rot_dim > d.head_dim || d.rot_dim % 2) { dkv_set_error("rot_dim %d: an even number of 2 to head_dim is expected", d.rot_dim); return false; }
    return true;
}

}  // namespace

// Four heads at once, so that a lane's cosines cost less (us with one head and with four):
//   bf16 in pieces of 4 and 8, from 1024 wavefronts on: 32 and 32 heads of 128 in place 256 rows 4.2 and 4.4, 512 rows 6.1 and 5.2, 2048 rows 15.9 and
//     12.0, 6144 rows 39.4 and 35.7; 28 and 4: 512 rows 4.2 and 4.4, 1024 rows 6.1 and 5.2
//   one pair to a lane, from 2048 on: bf16, 32 and 32 heads 128 rows 3.6 and 3.5, 2048 rows 26 and 15; 28 and 4: 128 rows 3.1 and 3.2; fp32, 32 and 32:
//     2048 rows 24 and 15
//   fp32 in pieces of 4 does not: 32 and 32 heads of 128 in place 1024 rows 12.7 and 12.0, 6144 rows 71 and 76; neighbouring pairs into other memory
//     512 rows 7.3 and 8.2, 1024 rows 12.0 and 12.1, 6144 rows 69 and 75
// and only where one wavefront has not all heads anyway (8 and 2 heads of 64 in bf16, 6144 rows 6.6 and 7.3). Also where workgroups would be too many.
int dkv_rope_lane_heads(int dtype, int v, int head_dim, int heads, int rows) {
    const int at_once = 64 / (head_dim / (2 * v));
    const int64_t ones = (int64_t)ceil_div(heads, at_once) * rows, fours = (int64_t)ceil_div(heads, 4 * at_once) * rows, most = 4ll << 23;      // wavefronts
    if (fours > most - 4) return 0;
    const bool gains = heads > at_once && (v == 1 ? fours >= 2048 : dtype == DKV_BF16 && fours >= 1024);
    return gains || ones > most - 4 ? 4 : 1;
}

extern "C" int dkv_rope_init(dkv_rope_desc *rope, int32_t head_dim, int32_t rot_dim, int32_t interleaved, double theta, int32_t scaling,
                             double factor, double original, double slow, double fast) {
    if (!rope) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    dkv_rope_desc d = {head_dim, rot_dim, interleaved != 0, 1.f, {0.0}};
    if (!rope_ok(d)) return DKV_E_UNSUPPORTED;
    auto positive = [](double x) { return x > 0.0 && x < 1e300; };        // a NaN is not
    if (!positive(theta)) { dkv_set_error("theta has to be positive and finite"); return DKV_E_INVALID_ARG; }
    if (scaling < DKV_ROPE_NONE || scaling > DKV_ROPE_PARTS) { dkv_set_error("unknown scaling %d", scaling); return DKV_E_INVALID_ARG; }
    if (scaling != DKV_ROPE_NONE && !positive(factor)) { dkv_set_error("the factor has to be positive and finite"); return DKV_E_INVALID_ARG; }
    if (scaling == DKV_ROPE_BASE && rot_dim == 2) { dkv_set_error("a single pair has no base to scale"); return DKV_E_INVALID_ARG; }
    if (scaling == DKV_ROPE_PARTS && !(positive(original) && slow >= 0.0 && fast > slow && fast < 1e300)) {
        dkv_set_error("scaling by parts needs original > 0 and 0 <= slow < fast"); return DKV_E_INVALID_ARG;
    }
    const double base = scaling == DKV_ROPE_BASE ? theta * pow(factor, rot_dim / (rot_dim - 2.0)) : theta;
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / rot_dim);
        if (scaling == DKV_ROPE_LINEAR) f /= factor;
        if (scaling == DKV_ROPE_PARTS) {
            double stay = (original * f / 6.283185307179586 - slow) / (fast - slow);
            stay = stay < 0.0 ? 0.0 : stay > 1.0 ? 1.0 : stay;
            f = f * stay + f / factor * (1.0 - stay);
        }
        d.freq[i] = f;
    }
    if (scaling == DKV_ROPE_PARTS) d.scale = (float)(0.1 * log(factor) + 1.0);
    *rope = d;
    return DKV_OK;
}

extern "C" int dkv_rope(const dkv_rope_desc *rope, const void *q, int64_t q_stride, void *q_out, int64_t q_out_stride, int32_t n_q_heads,
                        const void *k, int64_t k_stride, void *k_out, int64_t k_out_stride, int32_t n_k_heads, const int32_t *positions,
                        const int32_t *row_off, int32_t batch, int32_t rows, int32_t dtype, int32_t inverse, void *stream) {
    if (!rope) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    if (!rope_ok(*rope)) return DKV_E_UNSUPPORTED;
    if (dtype != DKV_BF16 && dtype != DKV_FP32) { dkv_set_error("unknown dtype"); return DKV_E_INVALID_ARG; }
    if (rows < 0 || n_q_heads < 0 || n_k_heads < 0 || (row_off && batch < 1)) { dkv_set_error("inconsistent sizes"); return DKV_E_INVALID_ARG; }
    if (rows >= 1 << 24 || ((int64_t)n_q_heads + n_k_heads) * rope->head_dim >= 1ll << 31) {
        dkv_set_error("%d rows of %d and %d heads are too many for one call", rows, n_q_heads, n_k_heads); return DKV_E_UNSUPPORTED;
    }
    auto strides = [&](const void *x, int64_t in, const void *y, int64_t out, int32_t heads) {
        if (heads > 0 && rows > 0 && (!x || !y)) { dkv_set_error("null argument"); return false; }
        const int64_t row = (int64_t)heads * rope->head_dim;
        if (in < row || out < row) { dkv_set_error("row stride %lld is less than a row", (long long)(in < out ? in : out)); return false; }
        if (x && x == y && in != out) { dkv_set_error("rows that are rotated in place have one stride"); return false; }
        return true;
    };
    if (!strides(q, q_stride, q_out, q_out_stride, n_q_heads) || !strides(k, k_stride, k_out, k_out_stride, n_k_heads)) return DKV_E_INVALID_ARG;
    if (rows == 0 || n_q_heads + n_k_heads == 0) return DKV_OK;
    if (!positions) { dkv_set_error("null argument"); return DKV_E_INVALID_ARG; }
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto call = [&](auto *type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        RopeArgs<T> a = {};
        a.q = static_cast<const T *>(q), a.k = static_cast<const T *>(k);
        a.q_out = static_cast<T *>(q_out), a.k_out = static_cast<T *>(k_out);
        a.q_stride = q_stride, a.k_stride = k_stride, a.q_out_stride = q_out_stride, a.k_out_stride = k_out_stride;
        a.positions = positions, a.row_off = row_off, a.batch = batch, a.rows = rows, a.n_q = n_q_heads, a.heads = n_q_heads + n_k_heads;
        a.head_dim = rope->head_dim, a.half = rope->rot_dim / 2;
        a.scale = rope->scale, a.way = inverse ? -1.f : 1.f;
        for (int i = 0; i < a.half; ++i) a.quarters[i] = rope->freq[i] * 0.6366197723675814;      // 2 / pi
        const bool pairs = rope->interleaved != 0;
        const int piece = pairs ? 2 * a.half : a.half;             // what pieces have to fit
        if constexpr (sizeof(T) == 2)
            return piece % 8 == 0 ? launch<T, 8>(a, pairs, s) : piece % 4 == 0 ? launch<T, 4>(a, pairs, s) : launch<T, 1>(a, pairs, s);
        else return piece % 4 == 0 ? launch<T, 4>(a, pairs, s) : launch<T, 1>(a, pairs, s);
    };
    return dtype == DKV_BF16 ? call((bf16_t *)nullptr) : call((float *)nullptr);
}
