// Orthogonal updates: X_0 = G / |G|, X_k+1 = (a + b A + c A A) X_k with A = X_k X_k^T, for each matrix of a list (its transpose where it has more rows than
// columns).  An odd polynomial of X acts on its singular values alone, and the usual coefficients bring them all near 1.
//
// A step is three products: A = X X^T and B = b A + c A A, which are symmetric (the tiles above the diagonal are computed and written twice), and
// a X + B X.  The steps stretch small singular values by a each, up to a^5 = 485 times in all, and with them what a rounding of X put there: X is
// therefore held in two fp16 parts (22 bits).  The diagonals of A and B, which are large against the rest, are kept in fp32 beside them and enter the
// next result element by element: X' = (a + diag B) X + (B - diag B) X.  Only what is left goes through the matrix units, in two parts and three
// products, at the precision of fp32 for all types.  (One part would do for bf16 matrices of noise: 5e-4 of the norm beside the 1.7e-3 of the result's own rounding, in half the
// time.  But where elements share a few sizes, as in a matrix of ones and signs, their roundings do not average out, and the result is off by 1.2e-2.)
// Powers of two bring the entries into the range of fp16: X holds at most |X| <= 1.3 (for coefficients that keep it there), entries of the size 1/sqrt(n).
#include "products.h"

namespace mlip {
namespace {

constexpr int kThreads = 256;
constexpr int kList = 24;                  // matrices of a launch
constexpr int kNormBlocks = 256;           // partial sums of a matrix
constexpr float kGramScale = 256.f;

using P = _Float16;

struct Item {
    const void *src;
    void *dst;
    int64_t src_rs, src_cs, dst_rs, dst_cs;   // of the matrix with m <= n
    int64_t x[2], low[2], gram, poly, diag;   // places in scratch memory, in elements of 16 bits: X's high and low parts, now and next; A, B, their diagonals
    int32_t m, n, m_p, n_p, m_ld, n_ld, dtype;  // sizes, filled up with zeros to, rows apart
    float x_scale;
};
struct List {
    int32_t count;
    uint32_t first[kList + 1];   // first block of every item
    Item item[kList];
};
static_assert(sizeof(List) <= 3960, "arguments of a launch");

// The item of a block, and the block's number among the item's
__device__ inline int item_of(const List &l, uint32_t block, uint32_t &at)
{
    int i = 0;
    while (i + 1 < l.count && l.first[i + 1] <= block) ++i;
    at = block - l.first[i];
    return i;
}

template <class Fn> __device__ inline void device_elem(int32_t dtype, Fn &&f)
{
    if (dtype == MLIP_DTYPE_F32) f(float{});
    else if (dtype == MLIP_DTYPE_BF16) f(__bf16{});
    else f(_Float16{});
}

// ---------------------------------------------------------------- norm and layout

__device__ inline double block_sum(double v)
{
    __shared__ double red[kThreads / 64];
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) v += red[w];
    return v;
}

// squares of item i to part[i * kNormBlocks + block], in kNormBlocks blocks each: rows (or columns, whichever lie close together) in pieces of eight elements
__global__ __launch_bounds__(kThreads) void k_squares(List l, double *part)
{
    const Item &it = l.item[blockIdx.y];
    double sum = 0.0;
    device_elem(it.dtype, [&](auto e) {
        using E = decltype(e);
        const E *src = static_cast<const E *>(it.src);
        const bool by_row = it.src_cs <= it.src_rs;
        const int64_t is = by_row ? it.src_cs : it.src_rs, os = by_row ? it.src_rs : it.src_cs;
        const int in = by_row ? it.n : it.m, out = by_row ? it.m : it.n, pieces = (in + 7) / 8;
        const int64_t total = (int64_t)pieces * out;
#pragma unroll 4
        for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < total; k += (int64_t)kNormBlocks * kThreads) {
            const int o = (int)((uint32_t)k / (uint32_t)pieces), i = (int)((uint32_t)k % (uint32_t)pieces) * 8;
            const E *p = src + o * os + i * is;
            if (is == 1 && i + 8 <= in) {
                const Cols<E, 8> w = *reinterpret_cast<const Far<E, 8> *>(p);
#pragma unroll
                for (int t = 0; t < 8; ++t) sum = fma((double)(float)w[t], (double)(float)w[t], sum);
            } else
                for (int t = 0; t < 8 && i + t < in; ++t) sum = fma((double)(float)p[t * is], (double)(float)p[t * is], sum);
        }
    });
    sum = block_sum(sum);
    if (threadIdx.x == 0) part[blockIdx.y * kNormBlocks + blockIdx.x] = sum;
}

// What X_0 is G times, x_scale included; NaN for a matrix with an infinity or NaN (squares of fp32 values do not overflow)
__device__ inline double start_scale(double squares, double eps, float x_scale)
{
    if (!(squares < __builtin_inf())) return __builtin_nan("");
    const double norm = sqrt(squares), by = norm > eps ? norm : eps;
    return by == 0.0 ? (double)x_scale : (double)x_scale / by;   // (zeros stay zeros)
}

// X_0 in parts: tiles of 64 rows and 64 columns, zeros up to n_p.  Loads and stores go along what lies close together, eight elements a thread.
__global__ __launch_bounds__(kThreads) void k_start(List l, const double *part, double eps, P *ws)
{
    __shared__ float tile[64][65];
    uint32_t at;
    const int i = item_of(l, blockIdx.x, at);
    const Item &it = l.item[i];
    const double scale = start_scale(block_sum(threadIdx.x < kNormBlocks ? part[i * kNormBlocks + threadIdx.x] : 0.0), eps, it.x_scale);
    const int tiles = it.n_p / 64, m = it.m, n = it.n, r0 = at / tiles * 64, c0 = at % tiles * 64;
    const bool by_row = it.src_cs <= it.src_rs;
    const int64_t in = by_row ? it.src_cs : it.src_rs, out = by_row ? it.src_rs : it.src_cs;   // strides along the inner and the outer loop
    device_elem(it.dtype, [&](auto e) {
        using E = decltype(e);
        const E *src = static_cast<const E *>(it.src) + r0 * it.src_rs + c0 * it.src_cs;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int piece = threadIdx.x + k * kThreads, o = piece / 8, i0 = piece % 8 * 8;
            const int most = by_row ? n - c0 : m - r0;
            float v[8] = {};
            if (o < (by_row ? m - r0 : n - c0)) {
                if (in == 1 && i0 + 8 <= most) {
                    const Cols<E, 8> w = *reinterpret_cast<const Far<E, 8> *>(src + o * out + i0);
#pragma unroll
                    for (int t = 0; t < 8; ++t) v[t] = (float)w[t];
                } else
#pragma unroll
                    for (int t = 0; t < 8; ++t) v[t] = i0 + t < most ? (float)src[o * out + (i0 + t) * in] : 0.f;
            }
#pragma unroll
            for (int t = 0; t < 8; ++t) (by_row ? tile[o][i0 + t] : tile[i0 + t][o]) = (float)(v[t] * scale);
        }
    });
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int piece = threadIdx.x + k * kThreads, r = piece / 8, c = piece % 8 * 8;
        if (r0 + r >= m) continue;
        Half8<P> hi, lo;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            P v[2];
            split(tile[r][c + t], v);
            hi[t] = v[0];
            lo[t] = v[1];
        }
        const int64_t to = (int64_t)(r0 + r) * it.n_ld + c0 + c;
        *reinterpret_cast<Half8<P> *>(ws + it.x[0] + to) = hi;
        *reinterpret_cast<Half8<P> *>(ws + it.low[0] + to) = lo;
    }
}

// ---------------------------------------------------------------- products

struct NoEach { template <class F> __device__ inline void operator()(F &) const {} };

// A tile's product over k in [0, k1), in runs that are summed by themselves first: what one fp32 sum loses grows with its terms, and where they are alike (a matrix of ones) it
// loses the same way every time (1 x 2^20: 4.4e-3 of the result in one run, 2e-5 so)
constexpr int64_t kRun = 4096;
template <class M> __device__ inline void product(const Panel &a, const Panel &b, int64_t m0, int64_t n0, int64_t k1, typename M::Lds &lds, f32x16 (&sum)[2][2])
{
    for (int64_t k = 0; k < k1; k += kRun) {
        f32x16 acc[2][2] = {};
        M::run(a, b, m0, n0, k, k + kRun < k1 ? k + kRun : k1, lds, acc, NoEach{});
        __syncthreads();   // nobody reads the tiles any more
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) sum[i][j] += acc[i][j];
    }
}

// X, or A - diag A, or B - diag B
__device__ inline Panel x_panel(const Item &it, const P *ws, int which) { return {ws + it.x[which], it.n_ld, it.low[which] - it.x[which], it.m, it.n_p}; }
__device__ inline Panel square_panel(const Item &it, const P *ws, int64_t at) { return {ws + at, it.m_ld, (int64_t)it.m * it.m_ld, it.m, it.m_p}; }

__device__ inline float both(P hi, P lo) { return (float)hi + (float)lo; }

// Four values split in two
__device__ inline void split4(const float (&v)[4], Half4<P> &hi, Half4<P> &lo)
{
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        P s[2];
        split(v[t], s);
        hi[t] = s[0];
        lo[t] = s[1];
    }
}

// Tile (i, j) with j >= i of number t: rows of the triangle of `tiles` tiles a side one after another
__device__ inline void triangle(int t, int tiles, int &i, int &j)
{
    i = 0;
    while (t >= tiles - i) t -= tiles - i++;
    j = i + t;
}

// SQUARE: B = b A + c A A; else A = X X^T.  Off the diagonal with D = diag A, R = A - D:  A A = R R + (D_i + D_j) R_ij, on it D_i^2 + (R R)_ii.
// Twelve matrices of 1024 x 4096: A 201 us (0.86 PF), B 63.
template <bool SQUARE> __global__ __launch_bounds__(kThreads) void k_symmetric(List l, P *ws, int which, float b, float c)
{
    using M = Product<P, 2, 2, true, true, 128, 128, 64, 64>;
    __shared__ typename M::Lds lds;
    uint32_t at;
    const Item &it = l.item[item_of(l, (uint32_t)xcd_order(blockIdx.x, gridDim.x), at)];
    int ti, tj;
    triangle((int)at, (it.m + 127) / 128, ti, tj);
    const Panel from = SQUARE ? square_panel(it, ws, it.gram) : x_panel(it, ws, which);
    f32x16 acc[2][2] = {};
    product<M>(from, from, tj * 128, ti * 128, SQUARE ? it.m_p : it.n_p, lds, acc);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = it.m, m_p = it.m_p, ld = it.m_ld, row0 = ti * 128 + wave % 2 * 64, col0 = tj * 128 + wave / 2 * 64;
    const Turned turned{reinterpret_cast<float *>(&lds) + wave * 4096};
    turned.put(acc);
    const int64_t part = (int64_t)m * ld;
    P *to = ws + (SQUARE ? it.poly : it.gram);
    const P *gram = ws + it.gram;
    float *diag = reinterpret_cast<float *>(ws + it.diag);   // of A, then of B
    const float scale = SQUARE ? c / kGramScale : kGramScale / (it.x_scale * it.x_scale);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int r = lane / 8 + 8 * k, row = row0 + r, col = col0 + lane % 8 * 8;
        if (row >= m || col >= m_p) continue;
        const int64_t here = (int64_t)row * ld + col;
        float y[8];
        turned.get(y, r, lane % 8 * 8);
#pragma unroll
        for (int t = 0; t < 8; ++t) y[t] *= scale;
        float dr = 0.f;
        if constexpr (SQUARE) {
            const Half8<P> gh = *reinterpret_cast<const Half8<P> *>(gram + here), gl = *reinterpret_cast<const Half8<P> *>(gram + part + here);
            float dc[8];
            load_cols<float>(dc, diag, 1, col, m);
            dr = diag[row];
#pragma unroll
            for (int t = 0; t < 8; ++t) y[t] = fmaf(fmaf(c, dr + dc[t], b), both(gh[t], gl[t]), y[t]);
        }
        if (row >= col && row < col + 8) {
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (col + t == row) {
                    const float d = y[t] * (1.f / kGramScale);
                    diag[SQUARE ? m + row : row] = SQUARE ? fmaf(dr, fmaf(c, dr, b), d) : d;
                    y[t] = 0.f;
                }
        }
        if (col + 8 > m)
#pragma unroll
            for (int t = 0; t < 8; ++t) y[t] = col + t < m ? y[t] : 0.f;
        Half8<P> v[2];
        split_cols<P>(y, v);
#pragma unroll
        for (int p = 0; p < 2; ++p) *reinterpret_cast<Half8<P> *>(to + p * part + here) = v[p];
        if (tj > ti) turned.set(y, r, lane % 8 * 8);
    }
    if (tj == ti) return;
    turned.fence();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int r = lane / 8 + 8 * k, row = col0 + r, col = row0 + lane % 8 * 8;   // (columns of the tile above the diagonal are whole: col + 8 <= m)
        if (row >= m) continue;
        float y[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) y[t] = turned.one(lane % 8 * 8 + t, r);
        Half8<P> v[2];
        split_cols<P>(y, v);
#pragma unroll
        for (int p = 0; p < 2; ++p) *reinterpret_cast<Half8<P> *>(to + p * part + (int64_t)row * ld + col) = v[p];
    }
}

// X' = (a + diag B) X + (B - diag B) X; the last one to where it belongs, times `scale`.  Columns of X are the first operand, its rows the second.
// Twelve matrices of 1024 x 4096: 387 us (0.80 PF), of which both parts of X read and written (400 MB) are 80.  (In tiles of 256 the whole call takes 2.99 ms for 3.08, but lists of
// fewer or smaller ones leave compute units idle: two of 1024 x 1024 766 us for 552, 24 of 512 x 512 520 for 420.)
template <bool LAST> __global__ __launch_bounds__(Middle::kThreads) void k_apply(List l, P *ws, int which, float a, float scale)
{
    using B = Middle;
    using M = typename B::template Of<P, 2, 2, false, true>;
    __shared__ typename M::Lds lds;
    uint32_t at;
    const Item &it = l.item[item_of(l, (uint32_t)xcd_order(blockIdx.x, gridDim.x), at)];
    const int tiles = (it.m + B::kRows - 1) / B::kRows, m0 = at % tiles * B::kRows, n0 = at / tiles * B::kCols;   // (tiles of the same columns one after another)
    f32x16 acc[2][2] = {};
    product<M>(x_panel(it, ws, which), square_panel(it, ws, it.poly), n0, m0, it.m_p, lds, acc);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane % 8 * 8;
    const Turned turned{reinterpret_cast<float *>(&lds) + wave * 4096};
    const P *old = ws + it.x[which], *old_low = ws + it.low[which];
    P *to = ws + it.x[which ^ 1], *to_low = ws + it.low[which ^ 1];
    const float *diag = reinterpret_cast<const float *>(ws + it.diag) + it.m;
    turned.put(acc);
    const int col = n0 + B::first(wave) + c;
    if (col >= it.n_p) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int r = lane / 8 + 8 * k, row = m0 + B::second(wave) + r;
        if (row >= it.m) continue;
        const int64_t here = (int64_t)row * it.n_ld + col;
        const Half8<P> hi = *reinterpret_cast<const Half8<P> *>(old + here), lo = *reinterpret_cast<const Half8<P> *>(old_low + here);
        const float f = a + diag[row];
        float y[8];
        turned.get(y, r, c);
#pragma unroll
        for (int t = 0; t < 8; ++t) y[t] = fmaf(f, both(hi[t], lo[t]), y[t] * (1.f / kGramScale));
        if constexpr (LAST) {
            device_elem(it.dtype, [&](auto e) {
                using E = decltype(e);
                E *dst = static_cast<E *>(it.dst) + row * it.dst_rs;
                const float s = scale / it.x_scale;
#pragma unroll
                for (int t = 0; t < 8; ++t) y[t] *= s;
                if (it.dst_cs == 1) store_cols<E>(y, dst, col, it.n);
                else
#pragma unroll
                    for (int t = 0; t < 8; ++t)
                        if (col + t < it.n) dst[(col + t) * it.dst_cs] = to_elem<E>(y[t]);
            });
        } else {
            Half8<P> v[2];
            split_cols<P>(y, v);
            *reinterpret_cast<Half8<P> *>(to + here) = v[0];
            *reinterpret_cast<Half8<P> *>(to_low + here) = v[1];
        }
    }
}

// no steps: the matrix divided by its norm
__global__ __launch_bounds__(kThreads) void k_normed(List l, const double *part, double eps, float scale)
{
    const Item &it = l.item[blockIdx.y];
    const double f = start_scale(block_sum(threadIdx.x < kNormBlocks ? part[blockIdx.y * kNormBlocks + threadIdx.x] : 0.0), eps, scale);
    device_elem(it.dtype, [&](auto e) {
        using E = decltype(e);
        const int64_t total = (int64_t)it.m * it.n;
        for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < total; k += (int64_t)gridDim.x * kThreads) {
            const int64_t r = k / it.n, c = k % it.n;
            static_cast<E *>(it.dst)[r * it.dst_rs + c * it.dst_cs] = to_elem<E>((float)((double)(float)static_cast<const E *>(it.src)[r * it.src_rs + c * it.src_cs] * f));
        }
    });
}

// ---------------------------------------------------------------- matrices that fit a compute unit

// All steps of one matrix in one block of eight wavefronts, X and A (then B) in two parts each in LDS, rows 16 bytes longer than a multiple of 32 elements.  A
// wavefront has up to two 32 x 32 squares of A or B and four of X.  Bound by latency: five steps of 64 x 128 31 us (253 by the launches below for the same list).
constexpr int kSmallThreads = 512, kSmallWaves = kSmallThreads / 64;
constexpr int kSmallHalves = 36 << 10, kSmallMost = 76 << 10;   // elements in LDS: 72 KB, so that two blocks share a compute unit, or 152

inline int64_t small_elems(int64_t m, int64_t n)
{
    const int64_t mp = pad_to(m, 32), np = pad_to(n, 32);
    return mp <= 128 && mp / 32 * (np / 32) <= 32 ? 2 * mp * (np + 8 + mp + 8) : (int64_t)1 << 40;
}

__device__ inline Half8<P> along(const P *p, int ld, int row, int k) { const int lane = threadIdx.x & 63; return *reinterpret_cast<const Half8<P> *>(p + (row + (lane & 31)) * ld + k + (lane >> 5) * 8); }
__device__ inline Half8<P> across(const P *p, int ld, int col, int k)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
    const P *q = p + (k + (g >> 1) * 8 + (i >> 2)) * ld + col + (g & 1) * 16 + (i & 3) * 4;
    return __builtin_shufflevector(read_turned(q), read_turned(q + 4 * ld), 0, 1, 2, 3, 4, 5, 6, 7);
}

template <int ELEMS> __global__ __launch_bounds__(kSmallThreads) void k_small(List l, double eps, int steps, float a, float b, float c, float scale)
{
    __shared__ alignas(16) P lds[ELEMS];
    __shared__ alignas(16) float diag[2][128];
    __shared__ double red[kSmallWaves];
    const Item &it = l.item[blockIdx.x];
    const int m = it.m, n = it.n, mp = (m + 31) / 32 * 32, np = (n + 31) / 32 * 32, xs = np + 8, as = mp + 8, mb = mp / 32, nb = np / 32;
    P *x[2] = {lds, lds + mp * xs}, *q[2] = {lds + 2 * mp * xs, lds + 2 * mp * xs + mp * as};
    const int wave = threadIdx.x >> 6;
    for (int k = threadIdx.x; k < mp * xs / 4; k += kSmallThreads) *reinterpret_cast<Half8<P> *>(lds + 8 * k) = Half8<P>{};   // what the matrix does not fill stays zero
    device_elem(it.dtype, [&](auto e) {
        using E = decltype(e);
        const E *src = static_cast<const E *>(it.src);
        // eight neighbours at a time, along rows or columns
        const bool by_row = it.src_cs <= it.src_rs;
        const unsigned inner = by_row ? n : m, outer = by_row ? m : n, pieces = (inner + 7) / 8, total = pieces * outer;
        const int64_t is = by_row ? it.src_cs : it.src_rs, os = by_row ? it.src_rs : it.src_cs;
        auto load = [&](unsigned k, float (&v)[8]) {
            const unsigned o = k / pieces, i = k % pieces * 8;
            load_cols(v, src + o * os, is, i, inner);
        };
        double sum = 0.0;
#pragma unroll 2
        for (unsigned k = threadIdx.x; k < total; k += kSmallThreads) {
            float v[8];
            load(k, v);
#pragma unroll
            for (int t = 0; t < 8; ++t) sum = fma((double)v[t], (double)v[t], sum);
        }
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        if ((threadIdx.x & 63) == 0) red[wave] = sum;
        __syncthreads();
        sum = 0.0;
        for (int w = 0; w < kSmallWaves; ++w) sum += red[w];
        const double f = start_scale(sum, eps, it.x_scale);
#pragma unroll 2
        for (unsigned k = threadIdx.x; k < total; k += kSmallThreads) {
            const int o = k / pieces, i = k % pieces * 8;
            float v[8];
            load(k, v);
            const int at = by_row ? o * xs + i : i * xs + o, step = by_row ? 1 : xs;
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (i + t < (int)inner) {
                    P w[2];
                    split((float)(v[t] * f), w);
                    x[0][at + t * step] = w[0];
                    x[1][at + t * step] = w[1];
                }
        }
    });
    const float from_gram = kGramScale / (it.x_scale * it.x_scale);
    for (int step = 0; step < steps; ++step) {
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; ++s) {   // A
            const int sq = wave + s * kSmallWaves, i0 = sq / mb * 32, j0 = sq % mb * 32;
            if (sq >= mb * mb) break;
            f32x16 acc = {}, cross = {};   // (two sums, so that a product does not wait for the one before)
#pragma unroll 4
            for (int k = 0; k < np; k += 16) {
                const Half8<P> u0 = along(x[0], xs, i0, k), u1 = along(x[1], xs, i0, k), v0 = along(x[0], xs, j0, k), v1 = along(x[1], xs, j0, k);
                cross = mfma<P>(u1, v0, cross);
                acc = mfma<P>(u0, v0, acc);
                cross = mfma<P>(u0, v1, cross);
            }
            acc += cross;
            const int row = j0 + acc_col();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float y[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    y[t] = acc[4 * g + t] * from_gram;
                    if (i0 + acc_row(4 * g + t) == row) {
                        diag[0][row] = y[t] * (1.f / kGramScale);
                        y[t] = 0.f;
                    }
                }
                Half4<P> v[2];
                split4(y, v[0], v[1]);
#pragma unroll
                for (int p = 0; p < 2; ++p) *reinterpret_cast<Half4<P> *>(q[p] + row * as + i0 + acc_row(4 * g)) = v[p];
            }
        }
        __syncthreads();
        f32x16 poly[2] = {};
#pragma unroll
        for (int s = 0; s < 2; ++s) {   // B
            const int sq = wave + s * kSmallWaves, i0 = sq / mb * 32, j0 = sq % mb * 32;
            if (sq >= mb * mb) break;
            f32x16 cross = {};
#pragma unroll 2
            for (int k = 0; k < mp; k += 16) {
                const Half8<P> u0 = along(q[0], as, i0, k), u1 = along(q[1], as, i0, k), v0 = along(q[0], as, j0, k), v1 = along(q[1], as, j0, k);
                cross = mfma<P>(u1, v0, cross);
                poly[s] = mfma<P>(u0, v0, poly[s]);
                cross = mfma<P>(u0, v1, cross);
            }
            poly[s] += cross;
            const int row = j0 + acc_col();
            const float dr = diag[0][row];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = i0 + acc_row(4 * g);
                const Half4<P> gh = *reinterpret_cast<const Half4<P> *>(q[0] + row * as + col), gl = *reinterpret_cast<const Half4<P> *>(q[1] + row * as + col);
                const Cols<float, 4> dc = *reinterpret_cast<const Cols<float, 4> *>(diag[0] + col);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    float y = fmaf(fmaf(c, dr + dc[t], b), both(gh[t], gl[t]), poly[s][4 * g + t] * (c / kGramScale));
                    if (col + t == row) {
                        diag[1][row] = fmaf(dr, fmaf(c, dr, b), y * (1.f / kGramScale));
                        y = 0.f;
                    }
                    poly[s][4 * g + t] = y;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int sq = wave + s * kSmallWaves, i0 = sq / mb * 32, j0 = sq % mb * 32;
            if (sq >= mb * mb) break;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float y[4] = {poly[s][4 * g], poly[s][4 * g + 1], poly[s][4 * g + 2], poly[s][4 * g + 3]};
                Half4<P> v[2];
                split4(y, v[0], v[1]);
#pragma unroll
                for (int p = 0; p < 2; ++p) *reinterpret_cast<Half4<P> *>(q[p] + (j0 + acc_col()) * as + i0 + acc_row(4 * g)) = v[p];
            }
        }
        __syncthreads();
        f32x16 next[4] = {};
#pragma unroll
        for (int s = 0; s < 4; ++s) {   // X: columns i0, rows j0
            const int sq = wave + s * kSmallWaves, i0 = sq / mb * 32, j0 = sq % mb * 32;
            if (sq >= mb * nb) break;
            f32x16 cross = {};
#pragma unroll 2
            for (int k = 0; k < mp; k += 16) {
                const Half8<P> u0 = across(x[0], xs, i0, k), u1 = across(x[1], xs, i0, k), v0 = along(q[0], as, j0, k), v1 = along(q[1], as, j0, k);
                cross = mfma<P>(u1, v0, cross);
                next[s] = mfma<P>(u0, v0, next[s]);
                cross = mfma<P>(u0, v1, cross);
            }
            next[s] += cross;
            const int row = j0 + acc_col();
            const float f = a + diag[1][row];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int at = row * xs + i0 + acc_row(4 * g);
                const Half4<P> hi = *reinterpret_cast<const Half4<P> *>(x[0] + at), lo = *reinterpret_cast<const Half4<P> *>(x[1] + at);
#pragma unroll
                for (int t = 0; t < 4; ++t) next[s][4 * g + t] = fmaf(f, both(hi[t], lo[t]), next[s][4 * g + t] * (1.f / kGramScale));
            }
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int sq = wave + s * kSmallWaves, i0 = sq / mb * 32, j0 = sq % mb * 32, row = j0 + acc_col();
            if (sq >= mb * nb) break;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float y[4] = {next[s][4 * g], next[s][4 * g + 1], next[s][4 * g + 2], next[s][4 * g + 3]};
                Half4<P> v[2];
                split4(y, v[0], v[1]);
#pragma unroll
                for (int p = 0; p < 2; ++p) *reinterpret_cast<Half4<P> *>(x[p] + row * xs + i0 + acc_row(4 * g)) = v[p];
            }
        }
    }
    __syncthreads();
    device_elem(it.dtype, [&](auto e) {   // (X has 22 bits: fp32 results too)
        using E = decltype(e);
        const bool by_row = it.dst_cs <= it.dst_rs;
        const unsigned inner = by_row ? n : m, outer = by_row ? m : n, pieces = (inner + 7) / 8, total = pieces * outer;
        const int64_t is = by_row ? it.dst_cs : it.dst_rs, os = by_row ? it.dst_rs : it.dst_cs;
        const float to = scale / it.x_scale;
#pragma unroll 2
        for (unsigned k = threadIdx.x; k < total; k += kSmallThreads) {
            const int o = k / pieces, i = k % pieces * 8, at = by_row ? o * xs + i : i * xs + o, step = by_row ? 1 : xs;
            E *dst = static_cast<E *>(it.dst) + o * os;
            float v[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int from = i + t < (int)inner ? at + t * step : at;
                v[t] = both(x[0][from], x[1][from]) * to;
            }
            if (is == 1) store_cols<E>(v, dst, i, inner);
            else
#pragma unroll
                for (int t = 0; t < 8; ++t)
                    if (i + t < (int)inner) dst[(i + t) * is] = to_elem<E>(v[t]);
        }
    });
}

// ---------------------------------------------------------------- a call's launches

constexpr int64_t kHead = kList * kNormBlocks * 8;   // bytes of the norms' partial sums
constexpr int64_t kMostBytes = (int64_t)1 << 31;    // of a group's scratch memory, where it has more than one matrix

// How a matrix is taken: in one block (of the smaller or the larger amount of LDS), or by products in tiles
enum { W_SMALL, W_MEDIUM, W_TILES, W_COUNT };
int way_of(const mlip_matrix_t &x)
{
    const int64_t elems = x.rows < x.cols ? small_elems(x.rows, x.cols) : small_elems(x.cols, x.rows);
    return elems <= kSmallHalves ? W_SMALL : elems <= kSmallMost ? W_MEDIUM : W_TILES;
}

struct Group {
    List l;
    int64_t bytes;
    int32_t next;
};

// The next matrices of the list, from `at` on, that go one way
Group group_of(const mlip_matrix_t *list, int32_t count, int32_t at, int way, bool no_steps)
{
    Group g{};
    int64_t used = kHead;
    for (; at < count && g.l.count < kList; ++at) {
        const mlip_matrix_t &x = list[at];
        if (x.rows == 0 || x.cols == 0 || way_of(x) != way) continue;
        Item it{};
        const bool tall = x.rows > x.cols;
        it.src = x.src;
        it.dst = x.dst;
        it.m = (int32_t)(tall ? x.cols : x.rows);
        it.n = (int32_t)(tall ? x.rows : x.cols);
        it.src_rs = tall ? x.src_col_stride : x.src_row_stride;
        it.src_cs = tall ? x.src_row_stride : x.src_col_stride;
        it.dst_rs = tall ? x.dst_col_stride : x.dst_row_stride;
        it.dst_cs = tall ? x.dst_row_stride : x.dst_col_stride;
        it.dtype = x.dtype;
        it.m_p = (int32_t)pad_to(it.m, kPadK);
        it.n_p = (int32_t)pad_to(it.n, kPadK);
        it.m_ld = (int32_t)pad_odd(it.m);
        it.n_ld = (int32_t)pad_odd(it.n);
        int e = 4;
        while ((int64_t)1 << (2 * (e - 4)) < it.n) ++e;
        it.x_scale = (float)(1 << e);
        int64_t place = used;
        auto take = [&](int64_t bytes) { const int64_t here = place / 2; place += pad_to(bytes, 256); return here; };
        if (way == W_TILES && !no_steps) {
            const int64_t all = (int64_t)it.m * it.n_ld * 2, square = (int64_t)it.m * it.m_ld * 2;
            it.x[0] = take(all);
            it.low[0] = take(all);
            it.x[1] = take(all);
            it.low[1] = take(all);
            it.gram = take(2 * square);
            it.poly = take(2 * square);
            it.diag = take((int64_t)it.m * 8);
        }
        if (g.l.count && place > kMostBytes) break;
        used = place;
        g.l.item[g.l.count++] = it;
    }
    g.bytes = used;
    g.next = at;
    return g;
}

template <class Fn> unsigned number_blocks(List &l, Fn &&blocks_of)
{
    uint32_t at = 0;
    for (int i = 0; i < l.count; ++i) {
        l.first[i] = at;
        at += (uint32_t)blocks_of(l.item[i]);
    }
    l.first[l.count] = at;
    return at;
}

void steps_of(List &l, P *ws, int32_t steps, float a, float b, float c, float scale, hipStream_t stream)
{
    for (int s = 0; s < steps; ++s) {
        const int now = s & 1;
        unsigned blocks = number_blocks(l, [](const Item &it) { const int64_t t = (it.m + 127) / 128; return t * (t + 1) / 2; });
        k_symmetric<false><<<blocks, kThreads, 0, stream>>>(l, ws, now, 0.f, 0.f);
        k_symmetric<true><<<blocks, kThreads, 0, stream>>>(l, ws, now, b, c);
        blocks = number_blocks(l, [](const Item &it) { return (int64_t)((it.m + Middle::kRows - 1) / Middle::kRows) * ((it.n_p + Middle::kCols - 1) / Middle::kCols); });
        (s + 1 == steps ? k_apply<true> : k_apply<false>)<<<blocks, Middle::kThreads, 0, stream>>>(l, ws, now, a, scale);
    }
}

}  // namespace

size_t ortho_workspace(const mlip_matrix_t *list, int32_t count)
{
    int64_t most = kHead;
    for (int way = 0; way < W_COUNT; ++way)
        for (int32_t at = 0; at < count;) {
            const Group g = group_of(list, count, at, way, false);
            at = g.next;
            if (g.bytes > most) most = g.bytes;
        }
    return (size_t)most;
}

int ortho_impl(const mlip_matrix_t *list, int32_t count, int32_t steps, const double coef[3], double eps, float scale, void *workspace, hipStream_t stream)
{
    double *norms = static_cast<double *>(workspace);
    P *ws = static_cast<P *>(workspace);
    const float a = (float)coef[0], b = (float)coef[1], c = (float)coef[2];
    for (int way = 0; way < W_COUNT; ++way)
        for (int32_t at = 0; at < count;) {
            Group g = group_of(list, count, at, way, steps == 0);
            at = g.next;
            List &l = g.l;
            if (!l.count) continue;
            if (way != W_TILES && steps) {
                (way == W_SMALL ? k_small<kSmallHalves> : k_small<kSmallMost>)<<<l.count, kSmallThreads, 0, stream>>>(l, eps, steps, a, b, c, scale);
                MLIP_HIP(hipGetLastError());
                continue;
            }
            k_squares<<<dim3(kNormBlocks, l.count), kThreads, 0, stream>>>(l, norms);
            if (!steps) {
                k_normed<<<dim3(256, l.count), kThreads, 0, stream>>>(l, norms, eps, scale);
            } else {
                const unsigned blocks = number_blocks(l, [](const Item &it) { return (int64_t)((it.m + 63) / 64) * (it.n_p / 64); });
                k_start<<<blocks, kThreads, 0, stream>>>(l, norms, eps, ws);
                steps_of(l, ws, steps, a, b, c, scale, stream);
            }
            MLIP_HIP(hipGetLastError());
        }
    return MLIP_OK;
}

}  // namespace mlip
