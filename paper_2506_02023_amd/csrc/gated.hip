// Gated projections: h = phi(x Wg + bg, x Wv + bv), and their gradient.
//
// With g = x Wg + bg, v = x Wv + bv and the incoming gradient H of h:
//   G = H phi_g(g, v), V = H phi_v(g, v);  dx = G Wg^T + V Wv^T;  dWg = x^T G, dWv = x^T V;  dbg, dbv = column sums of G, V.
// The gradient computes g and v again: 4 n d f of its 12 n d f operations, in place of 2 n f values that a forward pass would have to keep and
// both to move, which costs more where d is small, as it is here.
//
// Both matrices are laid out as one of 2 f columns, 32 of Wg and 32 of Wv in turn, so that a lane has g and v of the same feature in two
// registers; G and V lie the same way.  Rows go through in chunks whose G and V stay in the caches between the kernel that makes them and
// the two products that read them.
#include "products.h"

namespace mlip {
namespace {

// The types of a call: E of its arrays, T of the parts
template <class T_, int PARTS_, class E_> struct Kind {
    using T = T_;
    using E = E_;
    static constexpr int kParts = PARTS_;
};
template <class Fn> int with_kind(int32_t dtype, Fn &&f)
{
    if (dtype == MLIP_DTYPE_F32) return f(Kind<__bf16, 3, float>{});
    if (dtype == MLIP_DTYPE_BF16) return f(Kind<__bf16, 1, __bf16>{});
    return f(Kind<_Float16, 1, _Float16>{});
}
int parts_of(int32_t dtype) { return dtype == MLIP_DTYPE_F32 ? 3 : 1; }

// Column c of the 2 f: the feature, and whether of v
__host__ __device__ inline int64_t feature_of(int64_t c) { return c / 64 * 32 + c % 32; }
__host__ __device__ inline bool is_value(int64_t c) { return c & 32; }

// ---------------------------------------------------------------- layouts

constexpr int kPackThreads = 256;

// dst [rows][cols_p] in parts from src at (r, c) -> r rs + c cs, zeros from cols on; eight columns a thread
template <class K> __global__ __launch_bounds__(kPackThreads) void k_pack_rows(const typename K::E *src, int64_t rs, int64_t cs, int64_t rows, int64_t cols, int64_t cols_p,
                                                                             typename K::T *dst, int64_t part)
{
    const int64_t per_row = cols_p / 8, at = (int64_t)blockIdx.x * kPackThreads + threadIdx.x, r = at / per_row, c = at % per_row * 8;
    if (r >= rows) return;
    Half8<typename K::T> out[K::kParts];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        typename K::T v[K::kParts];
        if constexpr (K::kParts == 1) v[0] = c + k < cols ? src[r * rs + (c + k) * cs] : (typename K::E)0.f;
        else split(c + k < cols ? (float)src[r * rs + (c + k) * cs] : 0.f, v);
#pragma unroll
        for (int p = 0; p < K::kParts; ++p) out[p][k] = v[p];
    }
#pragma unroll
    for (int p = 0; p < K::kParts; ++p) *reinterpret_cast<Half8<typename K::T> *>(dst + p * part + r * cols_p + c) = out[p];
}

// A matrix of the weights' 32 x 32 squares: `across` [2 f][d_p] for g and v, `down` [d][2 f] for dx (either may be missing)
template <class K> struct Weights {
    const typename K::E *wg, *wv;
    int64_t g_rs, g_cs, v_rs, v_cs, d, f, d_p, f2;
    typename K::T *across, *down;
    int64_t across_part, down_part;
};
template <class K> __global__ __launch_bounds__(kPackThreads) void k_pack_weights(Weights<K> w)
{
    __shared__ float tile[32][33];
    const int64_t c0 = (int64_t)blockIdx.x * 32, d0 = (int64_t)blockIdx.y * 32;
    const bool value = is_value(c0);
    const typename K::E *src = value ? w.wv : w.wg;
    const int64_t rs = value ? w.v_rs : w.g_rs, cs = value ? w.v_cs : w.g_cs, f0 = feature_of(c0);
    const int a = threadIdx.x & 31, b = threadIdx.x >> 5;
    const bool by_row = cs <= rs;   // a along the columns of src, else along its rows
    for (int i = b; i < 32; i += 8) {
        const int dd = by_row ? i : a, ff = by_row ? a : i;
        tile[dd][ff] = d0 + dd < w.d && f0 + ff < w.f ? (float)src[(d0 + dd) * rs + (f0 + ff) * cs] : 0.f;
    }
    __syncthreads();
    for (int i = b; i < 32; i += 8) {
        typename K::T v[K::kParts];
        split(tile[a][i], v);
        for (int p = 0; p < K::kParts; ++p) w.across[p * w.across_part + (c0 + i) * w.d_p + d0 + a] = v[p];
        if (w.down && d0 + i < w.d) {
            split(tile[i][a], v);
            for (int p = 0; p < K::kParts; ++p) w.down[p * w.down_part + (d0 + i) * w.f2 + c0 + a] = v[p];
        }
    }
}

// ---------------------------------------------------------------- phi

__device__ inline float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __expf(-x)); }

struct Phi { float h, g, v; };   // phi, its derivatives

template <int ACT> __device__ inline Phi phi(float g, float v)
{
    if constexpr (ACT == MLIP_GATE_GELU) {
        const float c = 0.5f + 0.5f * erff(g * 0.70710678f);
        return {g * c * v, (c + g * __expf(-0.5f * g * g) * 0.39894228f) * v, g * c};
    }
    const float s = sigmoid(g);
    if constexpr (ACT == MLIP_GATE_SILU) return {g * s * v, s * (1.f + g * (1.f - s)) * v, g * s};
    if constexpr (ACT == MLIP_GATE_SIGMOID) return {s * v, s * (1.f - s) * v, s};
    const float t = sigmoid(v), b = v * t;
    return {s * b, s * (1.f - s) * b, s * t * (1.f + v * (1.f - t))};
}

template <class Fn> __device__ inline void with_act(int act, Fn &&f)
{
    if (act == MLIP_GATE_SILU) f(std::integral_constant<int, MLIP_GATE_SILU>{});
    else if (act == MLIP_GATE_GELU) f(std::integral_constant<int, MLIP_GATE_GELU>{});
    else if (act == MLIP_GATE_SIGMOID) f(std::integral_constant<int, MLIP_GATE_SIGMOID>{});
    else f(std::integral_constant<int, MLIP_GATE_SILU_SIGMOID>{});
}

// ---------------------------------------------------------------- products

struct NoEach { template <class F> __device__ inline void operator()(F &) const {} };

template <class K> struct GateArgs {
    Panel x, w;              // rows of the chunk; [2 f][d_p]
    int64_t d_p, f, n_tiles;
    int act;
    const typename K::E *bg, *bv;
    // forward: out [rows][f]; backward: the gradient of h, and where G and V go, [rows][2 f] in parts
    typename K::E *out;
    int64_t out_rs;
    const typename K::E *bar;
    int64_t bar_rs, bar_cs;
    typename K::T *gv;
    int64_t gv_ld, gv_part;
};

// Four elements from column c of a row on, zeros from `cols` on
template <class E> __device__ inline void load4(float (&v)[4], const E *row, int64_t cs, int64_t c, int64_t cols)
{
    if (cs == 1 && c + 4 <= cols) {
        const Cols<E, 4> w = *reinterpret_cast<const Far<E, 4> *>(row + c);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (float)w[k];
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = c + k < cols ? (float)row[(c + k) * cs] : 0.f;
}
template <class E> __device__ inline void store4(const float (&v)[4], E *row, int64_t c, int64_t cols)
{
    if (c + 4 <= cols) {
        Cols<E, 4> w;
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = to_elem<E>(v[k]);
        *reinterpret_cast<Far<E, 4> *>(row + c) = w;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (c + k < cols) row[c + k] = to_elem<E>(v[k]);
}

// The weights are the products' first operand and the rows their second, so that a lane has four neighbouring features of one row in a row of
// registers, and loads and stores them as one access.
template <class K, bool BACK> __global__ __launch_bounds__(256) void k_gates(GateArgs<K> a)
{
    using P = Product<typename K::T, K::kParts, true, true, 128, 128, 64, 64>;
    __shared__ typename P::Lds lds;
    const int64_t tile = xcd_order(blockIdx.x, gridDim.x), m0 = tile / a.n_tiles * 128, n0 = tile % a.n_tiles * 128;
    f32x16 acc[2][2] = {};
    P::run(a.w, a.x, n0, m0, 0, a.d_p, lds, acc, NoEach{});
    const int wave = threadIdx.x >> 6;
    const int64_t col0 = n0 + wave / 2 * 64, f0 = col0 / 2 + acc_row(0);
    if (col0 >= a.w.rows) return;
    float bg[4][4] = {}, bv[4][4] = {};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (a.bg) load4(bg[q], a.bg, 1, f0 + 8 * q, a.f);
        if (a.bv) load4(bv[q], a.bv, 1, f0 + 8 * q, a.f);
    }
    with_act(a.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t row = m0 + wave % 2 * 64 + 32 * j + acc_col();
            if (row >= a.x.rows) continue;
            float bar[4][4];
            if constexpr (BACK)
#pragma unroll
                for (int q = 0; q < 4; ++q) load4(bar[q], a.bar + row * a.bar_rs, a.bar_cs, f0 + 8 * q, a.f);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t f = f0 + 8 * q;
                float h[4];
                Half4<typename K::T> g[K::kParts], v[K::kParts];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const Phi y = phi<decltype(act)::value>(acc[0][j][4 * q + t] + bg[q][t], acc[1][j][4 * q + t] + bv[q][t]);
                    if constexpr (!BACK) h[t] = y.h;
                    else {
                        typename K::T gs[K::kParts], vs[K::kParts];
                        split(f + t < a.f ? bar[q][t] * y.g : 0.f, gs);
                        split(f + t < a.f ? bar[q][t] * y.v : 0.f, vs);
#pragma unroll
                        for (int p = 0; p < K::kParts; ++p) {
                            g[p][t] = gs[p];
                            v[p][t] = vs[p];
                        }
                    }
                }
                if constexpr (!BACK) store4(h, a.out + row * a.out_rs, f, a.f);
                else {
                    typename K::T *to = a.gv + row * a.gv_ld + col0 + acc_row(4 * q);
#pragma unroll
                    for (int p = 0; p < K::kParts; ++p) {
                        *reinterpret_cast<Half4<typename K::T> *>(to + p * a.gv_part) = g[p];
                        *reinterpret_cast<Half4<typename K::T> *>(to + p * a.gv_part + 32) = v[p];
                    }
                }
            }
        }
    });
}

// dx = [G V] [Wg Wv]^T
template <class K> struct RowBarArgs {
    Panel gv, w;             // [rows][2 f], [d][2 f]
    int64_t n_tiles;
    typename K::E *out;
    int64_t out_rs;
};
template <class K, int BM, int BN> __global__ __launch_bounds__(256) void k_row_bars(RowBarArgs<K> a)
{
    using P = Product<typename K::T, K::kParts, true, true, BN, BM, 64, 64>;   // (d first, rows second, as above)
    __shared__ typename P::Lds lds;
    const int64_t tile = xcd_order(blockIdx.x, gridDim.x), m0 = tile / a.n_tiles * BM, n0 = tile % a.n_tiles * BN;
    f32x16 acc[2][2] = {};
    P::run(a.w, a.gv, n0, m0, 0, a.gv.cols, lds, acc, NoEach{});
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t row = m0 + wave % (BM / 64) * 64 + 32 * j + acc_col();
        if (row >= a.gv.rows) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                store4(v, a.out + row * a.out_rs, n0 + wave / (BM / 64) * 64 + 32 * i + acc_row(4 * q), a.w.rows);
            }
    }
}

// The chunk's share of [dWg dWv]^T = [G V]^T x, [2 f][d], its rows in `splits` runs; and of the biases' gradients, the column sums of G and V
template <class K> struct WeightSumArgs {
    Panel gv, x;             // [rows][2 f], [rows][d]
    int64_t d, m_tiles, n_tiles, run;   // rows of a run, a multiple of a step
    float *part, *bias;      // [splits][2 f][d], [splits][2 f]
    bool add;
};
template <class K, int BM, int BN> __global__ __launch_bounds__(256) void k_weight_sums(WeightSumArgs<K> a)
{
    using P = Product<typename K::T, K::kParts, false, false, BM, BN, 64, 64>;
    __shared__ typename P::Lds lds;
    const int64_t at = xcd_order(blockIdx.x, gridDim.x), tiles = a.m_tiles * a.n_tiles, s = at / tiles, tile = at % tiles;
    const int64_t m0 = tile / a.n_tiles * BM, n0 = tile % a.n_tiles * BN;
    const int64_t k0 = s * a.run, k1 = k0 + a.run < a.gv.rows ? k0 + a.run : a.gv.rows;
    const int wave = threadIdx.x >> 6, wn = wave % (BN / 64) * 64;
    const bool sums = a.bias && n0 + wn == 0;
    f32x16 acc[2][2] = {}, ones[2] = {};
    P::run(a.gv, a.x, m0, n0, k0, k1, lds, acc, [&](auto &fa) {
        if (!sums) return;
        Half8<typename K::T> one;
#pragma unroll
        for (int k = 0; k < 8; ++k) one[k] = (typename K::T)1.f;
#pragma unroll
        for (int p = K::kParts - 1; p >= 0; --p)
#pragma unroll
            for (int i = 0; i < 2; ++i) ones[i] = mfma<typename K::T>(fa[i][p], one, ones[i]);
    });
    const int64_t row0 = m0 + wave / (BN / 64) * 64, col0 = n0 + wn + acc_col();
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int64_t row = row0 + 32 * i + acc_row(r);
            if (row >= a.gv.cols) continue;
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (col0 + 32 * j < a.d) {
                    float *to = a.part + (s * a.gv.cols + row) * a.d + col0 + 32 * j;
                    *to = a.add ? *to + acc[i][j][r] : acc[i][j][r];
                }
            if (sums && acc_col() == 0) {
                float *to = a.bias + s * a.gv.cols + row;
                *to = a.add ? *to + ones[i][r] : ones[i][r];
            }
        }
}

// The runs' shares added up, in their order
template <class K> struct JoinArgs {
    const float *part, *bias;
    int64_t splits, d, f, f2;
    typename K::E *dwg, *dwv, *dbg, *dbv;
    int64_t g_rs, g_cs, v_rs, v_cs;
};
template <class K> __global__ __launch_bounds__(kPackThreads) void k_join(JoinArgs<K> a)
{
    __shared__ float tile[32][33];
    const int64_t c0 = (int64_t)blockIdx.x * 32, d0 = (int64_t)blockIdx.y * 32, f0 = feature_of(c0);
    const bool value = is_value(c0);
    typename K::E *dw = value ? a.dwv : a.dwg, *db = value ? a.dbv : a.dbg;
    const int64_t rs = value ? a.v_rs : a.g_rs, cs = value ? a.v_cs : a.g_cs;
    const int p = threadIdx.x & 31, q = threadIdx.x >> 5;
    if (dw) {
        for (int i = q; i < 32; i += 8) {
            float sum = 0.f;
            if (d0 + p < a.d)
                in_steps<4>(0, a.splits, 1, [&](int64_t s) { return a.part[(s * a.f2 + c0 + i) * a.d + d0 + p]; }, [&](float x) { sum += x; });
            tile[i][p] = sum;   // [feature][d]
        }
        __syncthreads();
        const bool by_row = cs <= rs;
        for (int i = q; i < 32; i += 8) {
            const int dd = by_row ? i : p, ff = by_row ? p : i;
            if (d0 + dd < a.d && f0 + ff < a.f) dw[(d0 + dd) * rs + (f0 + ff) * cs] = to_elem<typename K::E>(tile[ff][dd]);
        }
    }
    if (db && d0 == 0 && q == 0 && f0 + p < a.f) {
        float sum = 0.f;
        for (int64_t s = 0; s < a.splits; ++s) sum += a.bias[s * a.f2 + c0 + p];
        db[f0 + p] = to_elem<typename K::E>(sum);
    }
}

// ---------------------------------------------------------------- a call's sizes and scratch memory

constexpr int64_t kChunkBytes = 96 << 20;     // of x's parts, G and V of a chunk
constexpr int64_t kMostTiles = 1 << 23;       // blocks of a launch

struct Plan {
    int parts;
    bool pack_x;
    int64_t d_p, f2, chunk;                    // columns of the laid out x and weights, rows of a chunk
    int64_t splits, run;
    size_t across, down, xs, gv, part, bias, bytes;   // offsets
};

// x is read where it lies if its rows are whole lines of pieces and steps
bool reads_x(const GatedArgs &a)
{
    return a.dtype != MLIP_DTYPE_F32 && a.d % kPadK == 0 && a.x_cs == 1 && a.x_rs % 8 == 0 && a.x_rs >= a.d && a.x_rs <= (1 << 21) &&
           reinterpret_cast<uintptr_t>(a.x) % 16 == 0;
}

Plan plan_of(const GatedArgs &a, bool grad)
{
    Plan p{};
    p.parts = parts_of(a.dtype);
    p.pack_x = !reads_x(a);
    p.d_p = pad_to(a.d, kPadK);
    p.f2 = 2 * pad_to(a.f, 32);
    // (scratch memory does not depend on where x lies: a size asked for once holds for all)
    const int64_t row_bytes = ((grad ? p.f2 : 0) + p.d_p) * p.parts * 2;
    p.chunk = pad_to(kChunkBytes / row_bytes + 1, 1024);
    const int64_t most = kMostTiles / ((p.f2 > p.d_p ? p.f2 : p.d_p) / 64 + 1) * 64 / 1024 * 1024;
    if (p.chunk > most) p.chunk = most;
    const int64_t all = pad_to(a.n > 0 ? a.n : 1, 128);
    if (p.chunk > all) p.chunk = all;
    size_t at = 0;
    auto take = [&](int64_t bytes) { const size_t here = at; at += (size_t)pad_to(bytes, 256); return here; };
    p.across = take(p.f2 * p.d_p * p.parts * 2);
    p.xs = take(p.chunk * p.d_p * p.parts * 2);
    if (grad) {
        p.down = take(a.d * p.f2 * p.parts * 2);
        p.gv = take(p.chunk * p.f2 * p.parts * 2);
        const int64_t tiles = a.d <= 64 ? (p.f2 + 255) / 256 : (p.f2 + 127) / 128 * ((a.d + 127) / 128);
        int64_t splits = 512 / tiles, most_splits = (p.chunk + 511) / 512;
        if (splits > most_splits) splits = most_splits;
        if (splits < 1) splits = 1;
        p.run = pad_to((p.chunk + splits - 1) / splits, 64);
        p.splits = (p.chunk + p.run - 1) / p.run;
        p.part = take(p.splits * p.f2 * a.d * 4);
        p.bias = take(p.splits * p.f2 * 4);
    }
    p.bytes = at;
    return p;
}

template <class K> int launch(const GatedArgs &a, const GatedGrad *g)
{
    using E = typename K::E;
    using T = typename K::T;
    const Plan p = plan_of(a, g != nullptr);
    char *ws = static_cast<char *>(a.workspace);
    T *across = reinterpret_cast<T *>(ws + p.across), *down = g ? reinterpret_cast<T *>(ws + p.down) : nullptr, *xs = reinterpret_cast<T *>(ws + p.xs);
    T *gv = g ? reinterpret_cast<T *>(ws + p.gv) : nullptr;
    const bool rows = !g || g->dx, weights = g && (g->dwg || g->dwv || g->dbg || g->dbv);
    const Weights<K> w = {static_cast<const E *>(a.wg), static_cast<const E *>(a.wv), a.wg_rs, a.wg_cs, a.wv_rs, a.wv_cs, a.d, a.f, p.d_p, p.f2,
                          across, rows ? down : nullptr, p.f2 * p.d_p, a.d * p.f2};
    if (a.n > 0) k_pack_weights<K><<<dim3((unsigned)(p.f2 / 32), (unsigned)(p.d_p / 32)), kPackThreads, 0, a.stream>>>(w);
    const Panel across_panel = {across, p.d_p, p.f2 * p.d_p, p.f2, p.d_p}, down_panel = {down, p.f2, a.d * p.f2, a.d, p.f2};
    int64_t first = 0;
    do {
        const int64_t n = a.n - first < p.chunk ? a.n - first : p.chunk;
        if (n <= 0 && a.n > 0) break;
        const E *x = static_cast<const E *>(a.x) + first * a.x_rs;
        Panel xp = {x, a.x_rs, 0, n, a.d};
        if (p.pack_x && n > 0) {
            const int64_t threads = n * (p.d_p / 8);
            k_pack_rows<K><<<(unsigned)((threads + kPackThreads - 1) / kPackThreads), kPackThreads, 0, a.stream>>>(x, a.x_rs, a.x_cs, n, a.d, p.d_p, xs, p.chunk * p.d_p);
            xp = {xs, p.d_p, p.chunk * p.d_p, n, p.d_p};
        }
        if (n > 0) {
            const int64_t n_tiles = (p.f2 + 127) / 128;
            GateArgs<K> ga = {xp, across_panel, p.d_p, a.f, n_tiles, a.act, static_cast<const E *>(a.bg), static_cast<const E *>(a.bv)};
            const unsigned blocks = (unsigned)((n + 127) / 128 * n_tiles);
            if (!g) {
                ga.out = static_cast<E *>(a.out) + first * a.out_rs;
                ga.out_rs = a.out_rs;
                k_gates<K, false><<<blocks, 256, 0, a.stream>>>(ga);
            } else {
                ga.bar = static_cast<const E *>(g->bar) + first * g->bar_rs;
                ga.bar_rs = g->bar_rs;
                ga.bar_cs = g->bar_cs;
                ga.gv = gv;
                ga.gv_ld = p.f2;
                ga.gv_part = p.chunk * p.f2;
                k_gates<K, true><<<blocks, 256, 0, a.stream>>>(ga);
            }
        }
        if (g) {
            const Panel gp = {gv, p.f2, p.chunk * p.f2, n, p.f2};
            if (g->dx && n > 0) {
                const bool narrow = a.d <= 64;
                const int64_t bm = narrow ? 256 : 128, bn = narrow ? 64 : 128, n_tiles = (a.d + bn - 1) / bn;
                const RowBarArgs<K> ra = {gp, down_panel, n_tiles, static_cast<E *>(g->dx) + first * g->dx_rs, g->dx_rs};
                (narrow ? k_row_bars<K, 256, 64> : k_row_bars<K, 128, 128>)<<<(unsigned)((n + bm - 1) / bm * n_tiles), 256, 0, a.stream>>>(ra);
            }
            if (weights) {
                const bool narrow = a.d <= 64;
                const int64_t bm = narrow ? 256 : 128, bn = narrow ? 64 : 128, m_tiles = (p.f2 + bm - 1) / bm, n_tiles = (a.d + bn - 1) / bn;
                const WeightSumArgs<K> wa = {gp, xp, a.d, m_tiles, n_tiles, p.run, reinterpret_cast<float *>(ws + p.part),
                                             g->dbg || g->dbv ? reinterpret_cast<float *>(ws + p.bias) : nullptr, first > 0};
                (narrow ? k_weight_sums<K, 256, 64> : k_weight_sums<K, 128, 128>)<<<(unsigned)(m_tiles * n_tiles * p.splits), 256, 0, a.stream>>>(wa);
            }
        }
        first += p.chunk;
    } while (first < a.n);
    if (weights) {
        const JoinArgs<K> ja = {reinterpret_cast<float *>(ws + p.part), reinterpret_cast<float *>(ws + p.bias), p.splits, a.d, a.f, p.f2, static_cast<E *>(g->dwg),
                                static_cast<E *>(g->dwv), static_cast<E *>(g->dbg), static_cast<E *>(g->dbv), g->dwg_rs, g->dwg_cs, g->dwv_rs, g->dwv_cs};
        k_join<K><<<dim3((unsigned)(p.f2 / 32), (unsigned)((a.d + 31) / 32)), kPackThreads, 0, a.stream>>>(ja);
    }
    MLIP_HIP(hipGetLastError());
    return MLIP_OK;
}

}  // namespace

size_t gated_workspace(const GatedArgs &a, bool grad) { return plan_of(a, grad).bytes; }

int gated_impl(const GatedArgs &a)
{
    if (a.n == 0) return MLIP_OK;
    return with_kind(a.dtype, [&](auto kind) { return launch<decltype(kind)>(a, nullptr); });
}

int gated_grad_impl(const GatedArgs &a, const GatedGrad &g)
{
    return with_kind(a.dtype, [&](auto kind) { return launch<decltype(kind)>(a, &g); });
}

}  // namespace mlip
