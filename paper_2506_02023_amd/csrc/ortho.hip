// Orthogonal updates: X_0 = G / |G|, X_k+1 = (a + b A + c A A) X_k with A = X_k X_k^T, for each matrix of a list (its transpose where it has more rows than
// columns).  An odd polynomial of X acts on its singular values alone, and the usual coefficients bring them all near 1.
//
// A step is three products: A = X X^T and B = b A + c A A, which are symmetric (the tiles above the diagonal are computed and written twice), and
// a X + B X.  The steps stretch small singular values by a each, up to a^5 = 485 times in all, and with them what a rounding of X put there: X, A and
// B are therefore held in two fp16 parts each (22 bits) and the products taken as three, at the precision of fp32 and at 16/3 of its matrix rate.
// Powers of two bring the entries into the range of fp16: X holds at most |X| <= 1.3 (for coefficients that keep it there), entries of the size 1/sqrt(n).
#include "products.h"

namespace mlip {
namespace {

constexpr int kThreads = 256;
constexpr int kList = 24;                  // matrices of a launch
constexpr int kNormBlocks = 64;            // partial sums of a matrix
constexpr float kGramScale = 256.f;

using P = _Float16;
constexpr int kParts = 2;

struct Item {
    const void *src;
    void *dst;
    int64_t src_rs, src_cs, dst_rs, dst_cs;   // of the matrix with m <= n
    int64_t x[2], gram, poly;                 // places in scratch memory, in elements of 16 bits
    int32_t m, n, m_p, n_p, dtype;
    float x_scale;
};
struct List {
    int32_t count;
    uint32_t first[kList + 1];   // first block of every item
    Item item[kList];
};
static_assert(sizeof(List) <= 3800, "arguments of a launch");

// The item of a block, and the block's number among the item's
__device__ inline const Item &item_of(const List &l, uint32_t block, uint32_t &at)
{
    int i = 0;
    while (i + 1 < l.count && l.first[i + 1] <= block) ++i;
    at = block - l.first[i];
    return l.item[i];
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

// squares of item i to part[i * kNormBlocks + block], in kNormBlocks blocks each
__global__ __launch_bounds__(kThreads) void k_squares(List l, double *part)
{
    const Item &it = l.item[blockIdx.y];
    double sum = 0.0;
    device_elem(it.dtype, [&](auto e) {
        const decltype(e) *src = static_cast<const decltype(e) *>(it.src);
        const bool by_row = it.src_cs <= it.src_rs;   // the inner loop along what lies close together
        const int64_t in = by_row ? it.n : it.m, out = by_row ? it.m : it.n, is = by_row ? it.src_cs : it.src_rs, os = by_row ? it.src_rs : it.src_cs;
        const int64_t total = in * out;
        for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < total; k += (int64_t)kNormBlocks * kThreads) {
            const double x = (double)(float)src[k / in * os + k % in * is];
            sum = fma(x, x, sum);
        }
    });
    sum = block_sum(sum);
    if (threadIdx.x == 0) part[blockIdx.y * kNormBlocks + blockIdx.x] = sum;
}

// X_0 in parts: tiles of 64 rows and 64 columns, zeros up to n_p
__global__ __launch_bounds__(kThreads) void k_start(List l, const double *part, double eps, P *ws)
{
    __shared__ float tile[64][65];
    uint32_t at;
    const Item &it = item_of(l, blockIdx.x, at);
    const double squares = block_sum(threadIdx.x < kNormBlocks ? part[(&it - l.item) * kNormBlocks + threadIdx.x] : 0.0);
    const double norm = sqrt(squares);
    const double scale = (double)it.x_scale / (norm > eps || norm != norm ? norm : eps);
    const int tiles = it.n_p / 64;
    const int64_t r0 = at / tiles * 64, c0 = at % tiles * 64;
    const bool by_row = it.src_cs <= it.src_rs;
    const int p = threadIdx.x & 63, q = threadIdx.x >> 6;
    device_elem(it.dtype, [&](auto e) {
        const decltype(e) *src = static_cast<const decltype(e) *>(it.src);
        for (int i = q; i < 64; i += 4) {
            const int r = by_row ? i : p, c = by_row ? p : i;
            tile[r][c] = r0 + r < it.m && c0 + c < it.n ? (float)((double)(float)src[(r0 + r) * it.src_rs + (c0 + c) * it.src_cs] * scale) : 0.f;
        }
    });
    __syncthreads();
    for (int i = q; i < 64 && r0 + i < it.m; i += 4) {
        P v[kParts];
        split(tile[i][p], v);
        P *to = ws + it.x[0] + (r0 + i) * it.n_p + c0 + p;
        for (int k = 0; k < kParts; ++k) to[(int64_t)k * it.m * it.n_p] = v[k];
    }
}

// ---------------------------------------------------------------- products

struct NoEach { template <class F> __device__ inline void operator()(F &) const {} };

__device__ inline Panel x_panel(const Item &it, const P *ws, int which)
{
    return {ws + it.x[which], it.n_p, (int64_t)it.m * it.n_p, it.m, it.n_p};
}
__device__ inline Panel square_panel(const Item &it, const P *ws, int64_t at) { return {ws + at, it.m_p, (int64_t)it.m * it.m_p, it.m, it.m_p}; }

__device__ inline float both(const P *p, int64_t part) { return (float)p[0] + (float)p[part]; }

// Tile (i, j) with j >= i of number t: rows of the triangle of `tiles` tiles a side one after another
__device__ inline void triangle(int t, int tiles, int &i, int &j)
{
    i = 0;
    while (t >= tiles - i) t -= tiles - i++;
    j = i + t;
}

// SQUARE: poly = b gram + c gram gram; else gram = X X^T
template <bool SQUARE> __global__ __launch_bounds__(kThreads) void k_symmetric(List l, P *ws, int which, float b, float c)
{
    using M = Product<P, kParts, true, true, 128, 128, 64, 64>;
    __shared__ M::Lds lds;
    uint32_t at;
    const Item &it = item_of(l, blockIdx.x, at);
    int ti, tj;
    triangle((int)at, (it.m + 127) / 128, ti, tj);
    const Panel from = SQUARE ? square_panel(it, ws, it.gram) : x_panel(it, ws, which);
    f32x16 acc[2][2] = {};
    M::run(from, from, ti * 128, tj * 128, 0, SQUARE ? it.m_p : it.n_p, lds, acc, NoEach{});
    const int wave = threadIdx.x >> 6, row0 = ti * 128 + wave / 2 * 64, col0 = tj * 128 + wave % 2 * 64 + acc_col();
    P *to = ws + (SQUARE ? it.poly : it.gram);
    const int64_t part = (int64_t)it.m * it.m_p;
    const float scale = SQUARE ? c / kGramScale : kGramScale / (it.x_scale * it.x_scale);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = row0 + 32 * i + acc_row(r), col = col0 + 32 * j;
                if (row >= it.m || col >= it.m_p) continue;
                float y = acc[i][j][r] * scale;
                if (SQUARE && col < it.m) y = fmaf(b, both(ws + it.gram + (int64_t)row * it.m_p + col, part), y);
                if (col >= it.m) y = 0.f;
                P v[kParts];
                split(y, v);
                for (int p = 0; p < kParts; ++p) {
                    to[p * part + (int64_t)row * it.m_p + col] = v[p];
                    if (tj > ti && col < it.m) to[p * part + (int64_t)col * it.m_p + row] = v[p];
                }
            }
}

// X' = a X + poly X; the last one to where it belongs, times `scale`
template <bool LAST> __global__ __launch_bounds__(kThreads) void k_apply(List l, P *ws, int which, float a, float scale)
{
    using M = Product<P, kParts, true, false, 128, 128, 64, 64>;
    __shared__ M::Lds lds;
    uint32_t at;
    const Item &it = item_of(l, blockIdx.x, at);
    const int tiles = (it.n_p + 127) / 128, m0 = at / tiles * 128, n0 = at % tiles * 128;
    f32x16 acc[2][2] = {};
    M::run(square_panel(it, ws, it.poly), x_panel(it, ws, which), m0, n0, 0, it.m_p, lds, acc, NoEach{});
    const int wave = threadIdx.x >> 6, row0 = m0 + wave / 2 * 64, col0 = n0 + wave % 2 * 64 + acc_col();
    const int64_t part = (int64_t)it.m * it.n_p;
    const P *old = ws + it.x[which];
    P *to = ws + it.x[which ^ 1];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = row0 + 32 * i + acc_row(r), col = col0 + 32 * j;
                if (row >= it.m || col >= (LAST ? it.n : it.n_p)) continue;
                const int64_t here = (int64_t)row * it.n_p + col;
                const float y = fmaf(a, both(old + here, part), acc[i][j][r] * (1.f / kGramScale));
                if constexpr (LAST) {
                    device_elem(it.dtype, [&](auto e) {
                        static_cast<decltype(e) *>(it.dst)[row * it.dst_rs + col * it.dst_cs] = to_elem<decltype(e)>(y * (scale / it.x_scale));
                    });
                } else {
                    P v[kParts];
                    split(y, v);
                    for (int p = 0; p < kParts; ++p) to[p * part + here] = v[p];
                }
            }
}

// no steps: the matrix divided by its norm
__global__ __launch_bounds__(kThreads) void k_normed(List l, const double *part, double eps, float scale)
{
    const Item &it = l.item[blockIdx.y];
    const double norm = sqrt(block_sum(threadIdx.x < kNormBlocks ? part[blockIdx.y * kNormBlocks + threadIdx.x] : 0.0));
    const double f = (double)scale / (norm > eps || norm != norm ? norm : eps);
    device_elem(it.dtype, [&](auto e) {
        using E = decltype(e);
        const int64_t total = (int64_t)it.m * it.n;
        for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < total; k += (int64_t)gridDim.x * kThreads) {
            const int64_t r = k / it.n, c = k % it.n;
            static_cast<E *>(it.dst)[r * it.dst_rs + c * it.dst_cs] = to_elem<E>((float)((double)(float)static_cast<const E *>(it.src)[r * it.src_rs + c * it.src_cs] * f));
        }
    });
}

// ---------------------------------------------------------------- a call's launches

constexpr int64_t kHead = kList * kNormBlocks * 8;   // bytes of the norms' partial sums

struct Group {
    List l;
    int64_t bytes;
    int32_t next;
};
constexpr int64_t kMostBytes = (int64_t)1 << 31;    // of a group's scratch memory, where it has more than one matrix

Group group_of(const mlip_matrix_t *list, int32_t count, int32_t at)
{
    Group g{};
    int64_t used = kHead;
    for (; at < count && g.l.count < kList; ++at) {
        const mlip_matrix_t &x = list[at];
        if (x.rows == 0 || x.cols == 0) continue;
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
        int e = 4;
        while ((int64_t)1 << (2 * (e - 4)) < it.n) ++e;
        it.x_scale = (float)(1 << e);
        int64_t place = used;
        auto take = [&](int64_t elems) { const int64_t here = place / 2; place += pad_to(elems * kParts * 2, 256); return here; };
        it.x[0] = take((int64_t)it.m * it.n_p);
        it.x[1] = take((int64_t)it.m * it.n_p);
        it.gram = take((int64_t)it.m * it.m_p);
        it.poly = take((int64_t)it.m * it.m_p);
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

}  // namespace

size_t ortho_workspace(const mlip_matrix_t *list, int32_t count)
{
    int64_t most = kHead;
    for (int32_t at = 0; at < count;) {
        const Group g = group_of(list, count, at);
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
    for (int32_t at = 0; at < count;) {
        Group g = group_of(list, count, at);
        at = g.next;
        List &l = g.l;
        if (!l.count) continue;
        k_squares<<<dim3(kNormBlocks, l.count), kThreads, 0, stream>>>(l, norms);
        if (!steps) {
            k_normed<<<dim3(256, l.count), kThreads, 0, stream>>>(l, norms, eps, scale);
            MLIP_HIP(hipGetLastError());
            continue;
        }
        unsigned blocks = number_blocks(l, [](const Item &it) { return (int64_t)((it.m + 63) / 64) * (it.n_p / 64); });
        k_start<<<blocks, kThreads, 0, stream>>>(l, norms, eps, ws);
        for (int s = 0; s < steps; ++s) {
            blocks = number_blocks(l, [](const Item &it) { const int64_t t = (it.m + 127) / 128; return t * (t + 1) / 2; });
            k_symmetric<false><<<blocks, kThreads, 0, stream>>>(l, ws, s & 1, 0.f, 0.f);
            k_symmetric<true><<<blocks, kThreads, 0, stream>>>(l, ws, s & 1, b, c);
            blocks = number_blocks(l, [](const Item &it) { return (int64_t)((it.m + 127) / 128) * ((it.n_p + 127) / 128); });
            (s + 1 == steps ? k_apply<true> : k_apply<false>)<<<blocks, kThreads, 0, stream>>>(l, ws, s & 1, a, scale);
        }
        MLIP_HIP(hipGetLastError());
    }
    return MLIP_OK;
}

}  // namespace mlip
