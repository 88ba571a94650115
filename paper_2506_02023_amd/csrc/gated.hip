// Gated projections: h = phi(x Wg + bg, x Wv + bv), and their gradient.
//
// With g = x Wg + bg, v = x Wv + bv and the incoming gradient H of h:
//   G = H phi_g(g, v), V = H phi_v(g, v);  dx = G Wg^T + V Wv^T;  dWg = x^T G, dWv = x^T V;  dbg, dbv = column sums of G, V.
// The gradient computes g and v again: 4 n d f of its 12 n d f operations, in place of 2 n f values that a forward pass would have to keep until then.
//
// Both matrices are laid out as one of 2 f columns, 32 of Wg and 32 of Wv in turn, so that a lane has g and v of the same feature in two
// registers; G and V lie the same way.  Rows go through in chunks that take up to 4 GB of scratch memory; the kernel that makes G and V writes them there, and the two products each
// read them again.  Where d is small that is what takes the time: 1,000,188 x 64 x 128 bf16 809 us, of which the call's own bytes would take 100.
#include "products.h"

namespace mlip {
namespace {

// The types of a call: E of its arrays, T of the parts; parts of g's and v's factors, or of G and V, and of what those are multiplied with
template <class T_, int PARTS_, class E_, int FACTORS_ = PARTS_> struct Kind {
    using T = T_;
    using E = E_;
    static constexpr int kParts = PARTS_, kFactors = FACTORS_, kWide = 16 / sizeof(E_);   // kWide: elements of a lane's load or store
};
using Brain = Kind<__bf16, 1, __bf16>;
using Half = Kind<_Float16, 1, _Float16>;
// Gradients of 16-bit arrays: G and V go in two bf16 parts (16 bits, the range of fp32).  Rounded to the arrays' type they would lose what sums over many terms of both signs leave (bf16:
// up to a tenth of such a result in 30,000 drawn calls; 2.35e-3 of the norm usually, of which a result's own rounding is 1.66e-3), and of fp16 what lies outside of its range, as they may on
// both sides.  x and the weights beside them are bf16, or exactly two bf16 parts: two products, or three, for one.  (32,768 x 1024 x 4096 bf16: 2.74 ms, 1.77 rounded to
// bf16; fp16 3.54, 1.85 rounded to fp16; 1,000,188 x 64 x 128: 809 and 520 us, fp16 930 and 516.)
using BrainBack = Kind<__bf16, 2, __bf16, 1>;
using HalfBack = Kind<__bf16, 2, _Float16>;
template <bool BACK, class Fn> int with_kind(int32_t dtype, Fn &&f)
{
    if (dtype == MLIP_DTYPE_F32) return f(Kind<__bf16, 3, float>{});
    if (dtype == MLIP_DTYPE_BF16) return f(std::conditional_t<BACK, BrainBack, Brain>{});
    return f(std::conditional_t<BACK, HalfBack, Half>{});
}
// g and v of fp32 arrays: two fp16 parts (22 bits) and three products, half the matrix time, where that is what bounds (wide rows of the forward call) or registers are
// short (rows of up to 128 features).  Every row of x and column of the weights is brought by a power of two to a largest value in [2^13, 2^14).  A value then has its 22 bits
// down to 2^-3; what is below is off by up to 2^-25.  That is nothing beside a sum of large terms, but it is all there is of a sum whose row is large where the column is small
// and the other way round.  So values of 2^7 and more are counted: of a column all but t (an eighth) shall be that large, of a row t and an eighth of those that are not zero.
// Then an eighth of the row's terms at least are 2^14 and more, and what is lost, twice 2^-25 2^14 a term at most, is below 2^-21 of the terms' sizes.  The results of a row or
// column that falls short are computed again by the fp32 matrix instruction.  (32,768 x 512 x 1365: 343 us, with three bf16 parts 635; 300,000 x 128 x 256: 236 and
// 361; the gradient's g and v of 202,612 x 128 x 341: 458 and 588.)
using Scaled = Kind<_Float16, 2, float>;
// In what g and v are computed, by tiles and by k_gates_narrow
template <class K> using InTiles = std::conditional_t<std::is_same_v<K, HalfBack>, Half, std::conditional_t<std::is_same_v<K, BrainBack>, Brain, K>>;
template <class K> using Inner = std::conditional_t<K::kParts == 3, Scaled, InTiles<K>>;

// Column c of the 2 f: the feature, and whether of v
__host__ __device__ inline int64_t feature_of(int64_t c) { return c / 64 * 32 + c % 32; }
__host__ __device__ inline bool is_value(int64_t c) { return c & 32; }

// ---------------------------------------------------------------- layouts

constexpr int kPackThreads = 256;
constexpr int64_t kNarrow = 128;              // d up to which rows stay in registers

// dst [rows][cols_p] in parts from src at (r, c) -> r rs + c cs, zeros from cols on; eight columns a thread
template <class K> __global__ __launch_bounds__(kPackThreads) void k_pack_rows(const typename K::E *src, int64_t rs, int64_t cs, int64_t rows, int64_t cols, int64_t cols_p,
                                                                             typename K::T *dst, int64_t ld, int64_t part)
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
    for (int p = 0; p < K::kParts; ++p) *reinterpret_cast<Half8<typename K::T> *>(dst + p * part + r * ld + c) = out[p];
}

// A matrix of the weights' 32 x 32 squares: `across` [2 f][d_p] for g and v, `down` [d][2 f] for dx (either may be missing)
template <class K> struct Weights {
    const typename K::E *wg, *wv;
    int64_t g_rs, g_cs, v_rs, v_cs, d, f, d_ld, f2_ld;
    typename InTiles<K>::T *across;
    typename K::T *down;
    int64_t across_part, down_part;
    const float *scale;      // of the columns, or NULL
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
        typename InTiles<K>::T u[InTiles<K>::kParts];
        typename K::T v[K::kFactors];
        split(w.scale ? tile[a][i] * w.scale[c0 + i] : tile[a][i], u);
        for (int p = 0; p < InTiles<K>::kParts; ++p) w.across[p * w.across_part + (c0 + i) * w.d_ld + d0 + a] = u[p];
        if (w.down && d0 + i < w.d) {
            split(tile[i][a], v);
            for (int p = 0; p < K::kFactors; ++p) w.down[p * w.down_part + (d0 + i) * w.f2_ld + c0 + a] = v[p];
        }
    }
}

// The power of two that brings a largest value to [2^13, 2^14), as its exponent (0 for none, and for one that is not finite)
constexpr int kMostExponent = 110;
__device__ inline int scale_for(float largest)
{
    const int e = largest > 0.f && largest < __builtin_inff() ? 13 - ilogbf(largest) : 0;
    return e > kMostExponent ? kMostExponent : e;
}
// Scaled values of a row or column of the weights, counted
constexpr float kLarge = 128.f;
struct Counts {
    int large = 0, there = 0;
    __device__ inline void add(float scaled)
    {
        large += fabsf(scaled) >= kLarge;
        there += scaled != 0.f;
    }
    __device__ inline void join(int lane_step)   // with those of lane ^ lane_step
    {
        large += __shfl_xor(large, lane_step);
        there += __shfl_xor(there, lane_step);
    }
};
// Whether the d values of a row (or column) fall short; `largest` before they were scaled.  (Not if one is infinite: their results are NaN either way.)
__device__ inline bool cannot_be_scaled(float largest, int e) { return e == kMostExponent && ldexpf(largest, e) < 8192.f; }
__device__ inline int spared(int d) { return d / 8 + 1 < d / 4 ? d / 8 + 1 : d / 4; }
__device__ inline bool row_falls_short(float largest, int e, Counts n, int d)
{
    return largest > 0.f && largest < __builtin_inff() && (8 * (n.large - spared(d)) < n.there || cannot_be_scaled(largest, e));
}
__device__ inline bool column_falls_short(float largest, int e, Counts n, int d)
{
    return largest > 0.f && largest < __builtin_inff() && (d - n.large > spared(d) || cannot_be_scaled(largest, e));
}

// fp32 weights as the caller has them
struct Plain {
    const float *wg, *wv;
    int64_t g_rs, g_cs, v_rs, v_cs;
    int32_t d, f;
};

// g and v of 32 features from f0 on and of a lane's row (32 of them) by the fp32 matrix instruction, in the same order whatever the strides
__device__ inline void plain_products(const Plain &w, const float *row, int64_t x_cs, int64_t f0, f32x16 &g, f32x16 &v)
{
    const int k_lane = (threadIdx.x & 63) >> 5 << 2;
    const int64_t f = f0 + (threadIdx.x & 31), f_within = f < w.f ? f : w.f - 1;
    const float *wg = w.wg + f_within * w.g_cs, *wv = w.wv + f_within * w.v_cs;
    g = v = f32x16{};
#pragma unroll 2
    for (int k0 = 0; k0 < w.d; k0 += 8) {
        float x[4], a[4], b[4];
        load_cols(x, row, x_cs, k0 + k_lane, w.d);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t k = k0 + k_lane + t, within = k < w.d ? k : w.d - 1;
            a[t] = wg[within * w.g_rs];
            b[t] = wv[within * w.v_rs];
            if (k >= w.d || f >= w.f) a[t] = b[t] = 0.f;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            g = __builtin_amdgcn_mfma_f32_32x32x2f32(a[t], x[t], g, 0, 0, 0);
            v = __builtin_amdgcn_mfma_f32_32x32x2f32(b[t], x[t], v, 0, 0, 0);
        }
    }
}

// Scales of 32 columns of the weights, and whether they fall short
constexpr int kScaleThreads = 1024;
__global__ __launch_bounds__(kScaleThreads) void k_column_scales(Weights<Scaled> w, float *scale, float *exponent, int32_t *short_of)
{
    __shared__ float most[kScaleThreads];
    __shared__ int counts[kScaleThreads];   // of large ones
    const int64_t c = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31), f = feature_of(c);
    const bool value = is_value(c);
    const float *src = value ? w.wv : w.wg;
    const int64_t rs = value ? w.v_rs : w.g_rs, cs = value ? w.v_cs : w.g_cs;
    constexpr int kHeld = 16, kStep = kScaleThreads / 32;   // values that a thread keeps from the first look to the second: columns of up to 512
    const int first = threadIdx.x >> 5;
    float held[kHeld], m = 0.f;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) held[k] = f < w.f && first + k * kStep < w.d ? src[(first + k * kStep) * rs + f * cs] : 0.f;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) m = fmaxf(m, fabsf(held[k]));
    if (f < w.f) in_steps<8>(first + kHeld * kStep, w.d, kStep, [&](int64_t d) { return src[d * rs + f * cs]; }, [&](float x) { m = fmaxf(m, fabsf(x)); });
    most[threadIdx.x] = m;
    __syncthreads();
    for (int k = threadIdx.x & 31; k < kScaleThreads; k += 32) m = fmaxf(m, most[k]);
    const int e = scale_for(m);
    const float by = ldexpf(1.f, e);
    Counts n;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) n.add(held[k] * by);
    if (f < w.f) in_steps<8>(first + kHeld * kStep, w.d, kStep, [&](int64_t d) { return src[d * rs + f * cs]; }, [&](float x) { n.add(x * by); });
    counts[threadIdx.x] = n.large;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    for (int k = 32; k < kScaleThreads; k += 32) n.large += counts[threadIdx.x + k];
    scale[c] = by;
    exponent[c] = (float)e;
    short_of[c] = column_falls_short(m, e, n, (int)w.d);
}

// The weights for k_gates_narrow in fp32, all of up to 128 rows of 32 columns in a block: `across` scaled and in two fp16 parts, the scales' exponents, which columns fall short,
// and `down` as k_pack_weights makes it
template <class K> __global__ __launch_bounds__(kPackThreads) void k_pack_scaled_weights(Weights<K> w, int64_t d_p, _Float16 *across, float *exponent, int32_t *short_of)
{
    __shared__ float tile[kNarrow][33], most[kPackThreads / 32][32];
    const int64_t c0 = (int64_t)blockIdx.x * 32, f0 = feature_of(c0);
    const bool value = is_value(c0);
    const typename K::E *src = value ? w.wv : w.wg;
    const int64_t rs = value ? w.v_rs : w.g_rs, cs = value ? w.v_cs : w.g_cs;
    const int a = threadIdx.x & 31, b = threadIdx.x >> 5;
    const bool by_row = cs <= rs;
#pragma unroll
    for (int k = 0; k < kNarrow / 32; ++k) {
        if (k * 32 >= d_p) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = b + 8 * j, dd = k * 32 + (by_row ? i : a), ff = by_row ? a : i;
            tile[dd][ff] = dd < w.d && f0 + ff < w.f ? (float)src[dd * rs + (f0 + ff) * cs] : 0.f;
        }
    }
    __syncthreads();
    float m = 0.f;
    for (int dd = b; dd < d_p; dd += 8) m = fmaxf(m, fabsf(tile[dd][a]));
    most[b][a] = m;
    __syncthreads();
    for (int j = 0; j < 4; ++j) {
        const int i = b + 8 * j;   // column
        m = 0.f;
        for (int k = 0; k < kPackThreads / 32; ++k) m = fmaxf(m, most[k][i]);
        const int e = scale_for(m);
        Counts n;
        for (int64_t dd = a; dd < d_p; dd += 32) {
            const float x = tile[dd][i] * ldexpf(1.f, e);
            _Float16 v[2];
            n.add(x);
            split(x, v);
            for (int p = 0; p < 2; ++p) across[p * w.across_part + (c0 + i) * w.d_ld + dd] = v[p];
        }
        for (int k = 16; k; k >>= 1) n.join(k);
        if (a == 0) {
            exponent[c0 + i] = (float)e;
            short_of[c0 + i] = m == __builtin_inff() ? -1 : column_falls_short(m, e, n, (int)w.d);
        }
    }
    if (!w.down) return;
    for (int64_t dd = b; dd < w.d; dd += 8) {
        typename K::T v[K::kParts];
        split(tile[dd][a], v);
        for (int p = 0; p < K::kParts; ++p) w.down[p * w.down_part + dd * w.f2_ld + c0 + a] = v[p];
    }
}

// Rows of x scaled and in parts, a wavefront each; zeros from `cols` on
__global__ __launch_bounds__(kPackThreads) void k_pack_scaled_rows(const float *src, int64_t rs, int64_t cs, int64_t rows, int64_t cols, int64_t cols_p, _Float16 *dst, int64_t ld, int64_t part,
                                                                   float *exponent, int32_t *short_of)
{
    const int64_t r = (int64_t)blockIdx.x * (kPackThreads / 64) + (threadIdx.x >> 6);
    if (r >= rows) return;
    const int lane = threadIdx.x & 63;
    const float *row = src + r * rs;
    constexpr int kHeld = 4;   // pieces of four columns that a lane keeps from the first look to the second: rows of up to 1024
    float v[kHeld][4], m = 0.f;
    auto look = [&](float (&x)[4], int64_t c) {
        load_cols(x, row, cs, c, cols);
#pragma unroll
        for (int t = 0; t < 4; ++t) m = fmaxf(m, fabsf(x[t]));
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k) look(v[k], (k * 64 + lane) * 4);
    for (int64_t c = (kHeld * 64 + lane) * 4; c < cols; c += 256) {
        float x[4];
        look(x, c);
    }
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    const int e = scale_for(m);
    const float scale = ldexpf(1.f, e);
    Counts n;
    auto put = [&](float (&x)[4], int64_t c) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            x[t] *= scale;
            n.add(x[t]);
        }
        Cols<_Float16, 4> p[2];
        split_cols<_Float16>(x, p);
        *reinterpret_cast<Cols<_Float16, 4> *>(dst + r * ld + c) = p[0];
        *reinterpret_cast<Cols<_Float16, 4> *>(dst + part + r * ld + c) = p[1];
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if ((k * 64 + lane) * 4 < cols_p) put(v[k], (k * 64 + lane) * 4);
    for (int64_t c = (kHeld * 64 + lane) * 4; c < cols_p; c += 256) {
        float x[4];
        load_cols(x, row, cs, c, cols);
        put(x, c);
    }
    for (int d = 32; d; d >>= 1) n.join(d);
    if (lane == 0) {
        exponent[r] = (float)e;
        short_of[r] = row_falls_short(m, e, n, (int)cols);
    }
}

// ---------------------------------------------------------------- phi

__device__ inline float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __expf(-x)); }
// sigmoid(x) and 1 - sigmoid(x), the latter to its own size's precision
struct Sigmoid { float s, rest; };
__device__ inline Sigmoid sigmoid_both(float x)
{
    const float e = __expf(-fabsf(x)), r = __builtin_amdgcn_rcpf(1.f + e), q = e * r;
    return x < 0.f ? Sigmoid{q, r} : Sigmoid{r, q};
}

// Phi(x), the normal distribution function, given e = exp(-x^2 / 2): Phi(-|x|) is e times a function that falls like 1 / |x|, here a polynomial in u = 1 / (1 + 0.35 |x|) of
// least relative error for |x| <= 14.5 (2^-25, in fp32 2^-21.5; 1 + erf would cancel in the tail; 1,000,188 x 64 -> 128 bf16 142 us, with erf 170, with erfc 198)
__device__ inline float normal(float x, float e)
{
    constexpr float c[9] = {0.139621302f, 0.139863521f, 0.119821288f, 0.105552502f, -0.0232123528f, 0.159319699f, -0.25583899f, 0.144030914f, -0.0291578863f};
    const float u = __builtin_amdgcn_rcpf(fmaf(0.35f, fabsf(x), 1.f));
    float q = c[8];
#pragma unroll
    for (int k = 7; k >= 0; --k) q = fmaf(q, u, c[k]);
    q *= u * e;
    return x < 0.f ? q : 1.f - q;
}

struct Phi { float h, g, v; };   // phi, its derivatives (BACK)

template <int ACT, bool BACK> __device__ inline Phi phi(float g, float v)
{
    if constexpr (ACT == MLIP_GATE_GELU) {
        const float e = __expf(-0.5f * g * g), c = normal(g, e);
        return {g * c * v, (c + g * e * 0.39894228f) * v, g * c};
    }
    Sigmoid s{}, t{};
    if constexpr (BACK) s = sigmoid_both(g);
    else s.s = sigmoid(g);
    if constexpr (ACT == MLIP_GATE_SILU) return {g * s.s * v, s.s * (1.f + g * s.rest) * v, g * s.s};
    if constexpr (ACT == MLIP_GATE_SIGMOID) return {s.s * v, s.s * s.rest * v, s.s};
    if constexpr (BACK) t = sigmoid_both(v);
    else t.s = sigmoid(v);
    const float b = v * t.s;
    return {s.s * b, s.s * s.rest * b, s.s * t.s * (1.f + v * t.rest)};
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
    // Scaled: the exponents of the scales to take off again, which rows and columns fall short, x and the weights as the caller has them
    const float *x_exponent, *w_exponent;
    const int32_t *x_short, *w_short;
    const float *x_plain;
    int64_t x_rs, x_cs;
    Plain plain;
};

// The weights are the products' first operand and the rows their second; a lane ends with neighbouring features of a row.  Bound by the matrix units, the activations behind
// them: 32,768 x 1024 x 4096 bf16, backward, 799 us (0.69 PF; with one part of G and V 706, and 1250 in tiles of 128 with four features a store).
template <class K, class B, bool BACK> __global__ __launch_bounds__(B::kThreads) void k_gates(GateArgs<K> a)
{
    using T = typename K::T;
    using P = typename B::template Of<typename InTiles<K>::T, InTiles<K>::kParts, InTiles<K>::kParts, true, true>;
    __shared__ typename P::Lds lds;
    const int64_t tile = xcd_order(blockIdx.x, gridDim.x), m0 = tile / a.n_tiles * B::kRows, n0 = tile % a.n_tiles * B::kCols;
    f32x16 acc[B::kPer / 32][2] = {};
    P::run(a.w, a.x, n0, m0, 0, a.d_p, lds, acc, NoEach{});
    __syncthreads();
    constexpr int W = K::kWide, lanes = 32 / W;   // of a row
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane % lanes * W;
    const Turned turned{reinterpret_cast<float *>(&lds) + wave * 4096};
    auto finish = [&](f32x16 (*part)[2], int64_t col0) {   // 64 columns of a wavefront
        const int64_t f = col0 / 2 + c;
        if (col0 >= a.w.rows) return;
        if constexpr (std::is_same_v<K, Scaled>) {
            const uint64_t columns = __ballot(a.w_short[col0 + lane]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                int64_t row = m0 + B::second(wave) + 32 * j + (lane & 31);
                if (row >= a.x.rows) row = a.x.rows - 1;
                const bool short_row = a.x_short[row];
                if (!__ballot(short_row) && !columns) continue;
                const float ex = a.x_exponent[row];
                f32x16 g, v;
                plain_products(a.plain, a.x_plain + row * a.x_rs, a.x_cs, col0 / 2, g, v);
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const int q = acc_row(k);
                    if (!short_row && !(columns >> q & 0x100000001)) continue;
                    // (brought to the others' scale; NaN, of an infinity in the row or column, stays)
                    if (part[0][j][k] == part[0][j][k]) part[0][j][k] = ldexpf(g[k], (int)(ex + a.w_exponent[col0 + q]));
                    if (part[1][j][k] == part[1][j][k]) part[1][j][k] = ldexpf(v[k], (int)(ex + a.w_exponent[col0 + 32 + q]));
                }
            }
        }
        turned.put(part);
        float bg[W] = {}, bv[W] = {};
        if (a.bg) load_cols(bg, a.bg, 1, f, a.f);
        if (a.bv) load_cols(bv, a.bv, 1, f, a.f);
        float eg[W], ev[W];
        if constexpr (std::is_same_v<K, Scaled>) {
            load_cols(eg, a.w_exponent, 1, col0 + c, a.w.rows);
            load_cols(ev, a.w_exponent, 1, col0 + 32 + c, a.w.rows);
        }
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < lanes; ++k) {
                const int r = lane / lanes + 64 / lanes * k;
                const int64_t row = m0 + B::second(wave) + r;
                if (row >= a.x.rows) continue;
                float g[W], v[W], bar[W];
                turned.get(g, r, c);
                turned.get(v, r, 32 + c);
                if constexpr (std::is_same_v<K, Scaled>) {
                    const float ex = a.x_exponent[row];
#pragma unroll
                    for (int t = 0; t < W; ++t) {
                        g[t] = ldexpf(g[t], -(int)(ex + eg[t]));
                        v[t] = ldexpf(v[t], -(int)(ex + ev[t]));
                    }
                }
                if constexpr (BACK) load_cols(bar, a.bar + row * a.bar_rs, a.bar_cs, f, a.f);
#pragma unroll
                for (int t = 0; t < W; ++t) {
                    const Phi y = phi<decltype(act)::value, BACK>(g[t] + bg[t], v[t] + bv[t]);
                    if constexpr (!BACK) g[t] = y.h;
                    else {
                        g[t] = f + t < a.f ? bar[t] * y.g : 0.f;
                        v[t] = f + t < a.f ? bar[t] * y.v : 0.f;
                    }
                }
                if constexpr (!BACK) store_cols(g, a.out + row * a.out_rs, f, a.f);
                else {
                    Cols<T, W> gp[K::kParts], vp[K::kParts];
                    split_cols<T>(g, gp);
                    split_cols<T>(v, vp);
                    T *to = a.gv + row * a.gv_ld + col0 + c;
#pragma unroll
                    for (int p = 0; p < K::kParts; ++p) {
                        *reinterpret_cast<Cols<T, W> *>(to + p * a.gv_part) = gp[p];
                        *reinterpret_cast<Cols<T, W> *>(to + p * a.gv_part + 32) = vp[p];
                    }
                }
            }
        });
    };
    finish(&acc[0], n0 + B::first(wave));
    if constexpr (B::kPer == 128) finish(&acc[2], n0 + B::first(wave) + 64);
}

// Rows of up to 128 features (STRIDED: which, or those of the gradient, do not lie one after another; the same bits): a block keeps the weights of PAIRS times 32 + 32 columns in LDS, in the order in which the lanes take them, and its
// wavefronts go over the rows, 32 at a time and without a barrier, each with its rows in registers (fp32 split there).  Such calls are bound by memory: rows come and go
// once for each such group of columns (from the L2 for all but the first), and nothing but the weights is laid out before.  1,000,188 x 64 -> 128 bf16: 124 us (3.1 TB/s; 189 by k_gates,
// whose blocks have one step of products each).
template <class K, int STEPS> struct NarrowShape {
    static constexpr int kDp = STEPS * 16, kPairs = (Inner<K>::kParts == 1 ? 256 : 128) / kDp, kFrags = kPairs * 2 * STEPS * Inner<K>::kParts;   // 32 KB of weights
    static constexpr int kStage = 32 * 72;   // elements of 16 bits for a wavefront's results on their way out: 32 rows of 64 and 8 (or of 32 and 4 fp32)
};
template <class K> struct NarrowArgs {
    GateArgs<K> a;           // (x: rows of the chunk as the caller has them)
    int64_t x_cs, groups, tiles;   // groups of columns; runs of 32 rows
    int32_t blocks, pairs;   // of a group; pairs of 32 columns in a group, NarrowShape's or, where that leaves compute units idle, one
};

// What a wavefront has to compute again of its rows and group of columns, stored over what it has stored before.  (Not in the kernel's loop, which has no registers to spare for
// it.  What has an infinity in its row or column has become NaN and stays so: `lost` features.)  1,000,188 x 64 -> 128 with four of five features zero: 1.05 ms, 0.24 with none.
template <class K, int STEPS, bool BACK>
__device__ inline void gates_again(const NarrowArgs<K> &na, const uint32_t *short_of, const uint32_t *lost, const float (*bias)[NarrowShape<K, STEPS>::kPairs * 32], int pairs, int64_t col_first,
                                   int64_t first_tile, int64_t stride)
{
    const GateArgs<K> &a = na.a;
    const Plain &w = a.plain;
    const int lane = threadIdx.x & 63, half = lane >> 5, d = w.d;
    __threadfence();   // (the earlier stores are other lanes')
    for (int64_t tile = first_tile; tile < na.tiles; tile += stride) {
        const int64_t mine = tile * 32 + (lane & 31), row = mine < a.x.rows ? mine : a.x.rows - 1;
        float x[STEPS][8], m = 0.f;
#pragma unroll
        for (int kk = 0; kk < STEPS; ++kk) load_cols(x[kk], static_cast<const float *>(a.x.p) + row * a.x.ld, na.x_cs, kk * 16 + half * 8, d);
#pragma unroll
        for (int kk = 0; kk < STEPS; ++kk)
#pragma unroll
            for (int k = 0; k < 8; ++k) m = fmaxf(m, fabsf(x[kk][k]));
        m = fmaxf(m, __shfl_xor(m, 32));
        const int e = scale_for(m);
        const float scale = ldexpf(1.f, e);
        Counts n;
#pragma unroll
        for (int kk = 0; kk < STEPS; ++kk)
#pragma unroll
            for (int k = 0; k < 8; ++k) n.add(x[kk][k] * scale);
        n.join(32);
        const bool short_row = row_falls_short(m, e, n, d), rows = __ballot(short_row) != 0, leave = mine >= a.x.rows || m == __builtin_inff();
        for (int pair = 0; pair < pairs; ++pair) {
            const int64_t col0 = col_first + pair * 64, f0 = col0 / 2, f_mine = f0 + (lane & 31);
            if (col0 >= a.w.rows) break;
            if (!rows && !short_of[pair]) continue;
            const int64_t f = f_mine < w.f ? f_mine : w.f - 1;
            f32x16 g = {}, v = {};
#pragma unroll
            for (int kk = 0; kk < STEPS; ++kk) {
                float ag[8], av[8];
                int from = half * 8;
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("" : "+v"(from));   // (else all addresses are worked out before the loops, for registers that there are not)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int at = kk * 16 + from + k, within = at < d ? at : d - 1;
                    ag[k] = w.wg[within * w.g_rs + f * w.g_cs];
                    av[k] = w.wv[within * w.v_rs + f * w.v_cs];
                    if (at >= d || f_mine >= w.f) ag[k] = av[k] = 0.f;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    g = __builtin_amdgcn_mfma_f32_32x32x2f32(ag[k], x[kk][k], g, 0, 0, 0);
                    v = __builtin_amdgcn_mfma_f32_32x32x2f32(av[k], x[kk][k], v, 0, 0, 0);
                }
            }
            const uint32_t mask = (leave ? 0 : short_row ? ~0u : short_of[pair]) & ~lost[pair];   // of the row's features
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = acc_row(4 * q);
                    float bar[4];
                    if constexpr (BACK) load_cols(bar, a.bar + row * a.bar_rs, a.bar_cs, f0 + c, a.f);
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const Phi y = phi<decltype(act)::value, BACK>(g[4 * q + t] + bias[0][pair * 32 + c + t], v[4 * q + t] + bias[1][pair * 32 + c + t]);
                        if (!(mask >> (c + t) & 1) || f0 + c + t >= a.f) continue;
                        if constexpr (!BACK) a.out[row * a.out_rs + f0 + c + t] = y.h;
                        else {
                            typename K::T gp[K::kParts], vp[K::kParts];
                            split(bar[t] * y.g, gp);
                            split(bar[t] * y.v, vp);
#pragma unroll
                            for (int p = 0; p < K::kParts; ++p) {
                                typename K::T *to = a.gv + p * a.gv_part + row * a.gv_ld + col0 + c + t;
                                to[0] = gp[p];
                                to[32] = vp[p];
                            }
                        }
                    }
                }
            });
        }
    }
}

template <class K, int STEPS, bool BACK, bool STRIDED> __global__ __launch_bounds__(256, K::kParts == 1 && !BACK ? 3 : 2) void k_gates_narrow(NarrowArgs<K> na)
{
    using T = typename K::T;
    using E = typename K::E;
    using C = typename Inner<K>::T;
    using S = NarrowShape<K, STEPS>;
    constexpr int PARTS = Inner<K>::kParts;
    constexpr bool SCALED = std::is_same_v<Inner<K>, Scaled>;
    __shared__ alignas(16) C weights[S::kFrags * 512];
    __shared__ alignas(16) float exponents[2][SCALED ? S::kPairs * 32 : 4];
    __shared__ alignas(16) T stage_[4 * S::kStage];
    __shared__ alignas(16) float bias[2][S::kPairs * 32];
    __shared__ uint32_t short_of[SCALED ? S::kPairs : 1], lost[SCALED ? S::kPairs : 1];   // features whose columns fall short, or hold an infinity, a bit each
    const GateArgs<K> &a = na.a;
    const int64_t at = xcd_order(blockIdx.x, gridDim.x);
    const int pairs = S::kPairs == 1 ? 1 : na.pairs;
    const int64_t group = at % na.groups, col_first = group * pairs * 64;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5, d = (int)a.x.cols;
    const C *across = static_cast<const C *>(a.w.p);
#pragma unroll 4
    for (int k = threadIdx.x; k < pairs * (2 * STEPS * PARTS * 64); k += 256) {
        const int l = k & 63, f = k >> 6, p = f % PARTS, kk = f / PARTS % STEPS, c = f / PARTS / STEPS;
        const int64_t col = col_first + c * 32 + (l & 31);
        Half8<C> w = {};
        if (col < a.w.rows && kk * 16 < a.w.cols) w = *reinterpret_cast<const Half8<C> *>(across + p * a.w.part + col * a.w.ld + kk * 16 + (l >> 5) * 8);
        *reinterpret_cast<Half8<C> *>(weights + k * 8) = w;
    }
    for (int k = threadIdx.x; k < pairs * 32; k += 256) {
        const int64_t f = col_first / 2 + k;
        bias[0][k] = a.bg && f < a.f ? (float)a.bg[f] : 0.f;
        bias[1][k] = a.bv && f < a.f ? (float)a.bv[f] : 0.f;
        if constexpr (SCALED) {
            const int64_t col = col_first + k / 32 * 64 + k % 32;
            exponents[0][k] = col < a.w.rows ? a.w_exponent[col] : 0.f;
            exponents[1][k] = col < a.w.rows ? a.w_exponent[col + 32] : 0.f;
            const int32_t sg = col < a.w.rows ? a.w_short[col] : 0, sv = col < a.w.rows ? a.w_short[col + 32] : 0;
            const uint64_t some = __ballot(sg > 0 || sv > 0), none = __ballot(sg < 0 || sv < 0);
            if (k % 32 == 0) {
                short_of[k / 32] = (uint32_t)(some >> (lane & 32));
                lost[k / 32] = (uint32_t)(none >> (lane & 32));
            }
        }
    }
    __syncthreads();
    T *stage = stage_ + wave * S::kStage;
    const E *x = static_cast<const E *>(a.x.p);
    auto fence = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    bool again = false;   // whether there may be something that falls short
    const int64_t first_tile = at / na.groups * 4 + wave, stride = (int64_t)na.blocks * 4;
    for (int64_t tile = first_tile; tile < na.tiles; tile += stride) {
        const int64_t row0 = tile * 32, mine = row0 + (lane & 31), row = mine < a.x.rows ? mine : a.x.rows - 1;
        Half8<C> fx[STEPS][PARTS];
        float ex = 0.f;
        if constexpr (!SCALED) {
#pragma unroll
            for (int kk = 0; kk < STEPS; ++kk) {
                const int c = kk * 16 + half * 8;
                const E *p = x + row * a.x.ld;
                if (!STRIDED && c + 8 <= d) fx[kk][0] = *reinterpret_cast<const Far<E, 8> *>(p + c);
                else
#pragma unroll
                    for (int k = 0; k < 8; ++k) fx[kk][0][k] = c + k < d ? p[(c + k) * (STRIDED ? na.x_cs : 1)] : (E)0.f;
            }
        } else {   // (the two halves of the wavefront have half of a row's features each)
            float v[STEPS][8], m = 0.f;
#pragma unroll
            for (int kk = 0; kk < STEPS; ++kk) load_cols(v[kk], x + row * a.x.ld, STRIDED ? na.x_cs : 1, kk * 16 + half * 8, d);
#pragma unroll
            for (int kk = 0; kk < STEPS; ++kk)
#pragma unroll
                for (int k = 0; k < 8; ++k) m = fmaxf(m, fabsf(v[kk][k]));
            m = fmaxf(m, __shfl_xor(m, 32));
            const int e = scale_for(m);
            const float scale = ldexpf(1.f, e);
            ex = (float)e;
            Counts n;
            n.there = d;   // (at most: gates_again looks closer)
#pragma unroll
            for (int kk = 0; kk < STEPS; ++kk) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[kk][k] *= scale;
                    n.large += fabsf(v[kk][k]) >= kLarge;
                }
                split_cols<C>(v[kk], fx[kk]);
            }
            n.large += __shfl_xor(n.large, 32);
            again |= __ballot(row_falls_short(m, e, n, d)) != 0;
        }
#pragma unroll 1
        for (int pair = 0; pair < pairs; ++pair) {
            const int64_t col0 = col_first + pair * 64, f0 = col0 / 2;
            if (col0 >= a.w.rows) break;
            float bar[4][4];
            if constexpr (BACK)
#pragma unroll
                for (int q = 0; q < 4; ++q) load_cols(bar[q], a.bar + row * a.bar_rs, STRIDED ? a.bar_cs : 1, f0 + acc_row(4 * q), a.f);
            f32x16 g = {}, v = {};
#pragma unroll
            for (int kk = 0; kk < STEPS; ++kk) {
                Half8<C> wg[PARTS], wv[PARTS];
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    wg[p] = *reinterpret_cast<const Half8<C> *>(weights + (((pair * 2 * STEPS + kk) * PARTS + p) * 64 + lane) * 8);
                    wv[p] = *reinterpret_cast<const Half8<C> *>(weights + ((((pair * 2 + 1) * STEPS + kk) * PARTS + p) * 64 + lane) * 8);
                }
                for_products<PARTS, PARTS>([&](int p, int q) {
                    g = mfma<C>(wg[p], fx[kk][q], g);
                    v = mfma<C>(wv[p], fx[kk][q], v);
                });
                if (kk % 2) __builtin_amdgcn_sched_barrier(0);   // (else all fragments are fetched at once, into registers that there are not)
            }
            // bias, phi: registers 4 q + t have feature f0 + acc_row(4 q) + t of the lane's row
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t f = f0 + acc_row(4 * q);
                    const int c = pair * 32 + acc_row(4 * q);
                    const Cols<float, 4> bg = *reinterpret_cast<const Cols<float, 4> *>(bias[0] + c), bv = *reinterpret_cast<const Cols<float, 4> *>(bias[1] + c);
                    if constexpr (SCALED) {
                        const Cols<float, 4> eg = *reinterpret_cast<const Cols<float, 4> *>(exponents[0] + c), ev = *reinterpret_cast<const Cols<float, 4> *>(exponents[1] + c);
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            g[4 * q + t] = ldexpf(g[4 * q + t], -(int)(ex + eg[t]));
                            v[4 * q + t] = ldexpf(v[4 * q + t], -(int)(ex + ev[t]));
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const Phi y = phi<decltype(act)::value, BACK>(g[4 * q + t] + bg[t], v[4 * q + t] + bv[t]);
                        if constexpr (!BACK) g[4 * q + t] = y.h;
                        else {
                            g[4 * q + t] = f + t < a.f ? bar[q][t] * y.g : 0.f;
                            v[4 * q + t] = f + t < a.f ? bar[q][t] * y.v : 0.f;
                        }
                    }
                }
            });
            if constexpr (!BACK) {
                constexpr int W = K::kWide, lanes = 32 / W, ld = 32 + W;   // of a row in the stage
                E *st = reinterpret_cast<E *>(stage);
                fence();
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    Cols<E, 4> h;
#pragma unroll
                    for (int t = 0; t < 4; ++t) h[t] = to_elem<E>(g[4 * q + t]);
                    *reinterpret_cast<Cols<E, 4> *>(st + (lane & 31) * ld + acc_row(4 * q)) = h;
                }
                fence();
#pragma unroll
                for (int k = 0; k < lanes / 2; ++k) {
                    const int r = lane / lanes + 64 / lanes * k, c = lane % lanes * W;
                    if (row0 + r >= a.x.rows) continue;
                    const Cols<E, W> h = *reinterpret_cast<const Cols<E, W> *>(st + r * ld + c);
                    E *to = a.out + (row0 + r) * a.out_rs + f0;
                    if (f0 + c + W <= a.f) *reinterpret_cast<Far<E, W> *>(to + c) = h;
                    else
#pragma unroll
                        for (int t = 0; t < W; ++t)
                            if (f0 + c + t < a.f) to[c + t] = h[t];
                }
            } else {
#pragma unroll
                for (int p = 0; p < K::kParts; ++p) {
                    fence();
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        Half4<T> gp, vp;
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            gp[t] = to_elem<T>(g[4 * q + t]);
                            vp[t] = to_elem<T>(v[4 * q + t]);
                            if (p + 1 < K::kParts) {
                                g[4 * q + t] -= (float)gp[t];
                                v[4 * q + t] -= (float)vp[t];
                            }
                        }
                        *reinterpret_cast<Half4<T> *>(stage + (lane & 31) * 72 + acc_row(4 * q)) = gp;
                        *reinterpret_cast<Half4<T> *>(stage + (lane & 31) * 72 + 32 + acc_row(4 * q)) = vp;
                    }
                    fence();
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = lane / 8 + 8 * k, c = lane % 8 * 8;
                        if (row0 + r < a.x.rows)
                            *reinterpret_cast<Half8<T> *>(a.gv + p * a.gv_part + (row0 + r) * a.gv_ld + col0 + c) = *reinterpret_cast<const Half8<T> *>(stage + r * 72 + c);
                    }
                }
            }
        }
    }
    if constexpr (SCALED) {
        for (int pair = 0; pair < pairs; ++pair) again |= short_of[pair] != 0;
        if (again) gates_again<K, STEPS, BACK>(na, short_of, lost, bias, pairs, col_first, first_tile, stride);
    }
}

// dx = [G V] [Wg Wv]^T.  32,768 x 8192 in two parts by 1024 in one: 931 us (1.18 PF); 202,612 x 704 by 128 of three parts: 320 us (0.68 PF)
template <class K> struct RowBarArgs {
    Panel gv, w;             // [rows][2 f], [d][2 f]
    int64_t n_tiles;
    typename K::E *out;
    int64_t out_rs;
};
template <class K, class B> using RowBars = typename B::template Of<typename K::T, K::kFactors, K::kParts, true, true>;   // (d first, rows second)
template <class K, class B> __device__ inline void row_bars(const RowBarArgs<K> &a, int64_t tile, typename RowBars<K, B>::Lds &lds)
{
    using P = RowBars<K, B>;
    const int64_t m0 = tile / a.n_tiles * B::kRows, n0 = tile % a.n_tiles * B::kCols;
    f32x16 acc[B::kPer / 32][2] = {};
    P::run(a.w, a.gv, n0, m0, 0, a.gv.cols, lds, acc, NoEach{});
    __syncthreads();
    constexpr int W = K::kWide, lanes = 64 / W;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane % lanes * W;
    const Turned turned{reinterpret_cast<float *>(&lds) + wave * 4096};
#pragma unroll
    for (int i = 0; i < B::kPer / 64; ++i) {
        turned.put(&acc[2 * i]);
#pragma unroll
        for (int k = 0; k < lanes; ++k) {
            const int r = lane / lanes + 64 / lanes * k;
            const int64_t row = m0 + B::second(wave) + r;
            if (row >= a.gv.rows) continue;
            float v[W];
            turned.get(v, r, c);
            store_cols(v, a.out + row * a.out_rs, n0 + B::first(wave) + 64 * i + c, a.w.rows);
        }
    }
}

// The chunk's share of [dWg dWv]^T = [G V]^T x, [2 f][d], its rows in `splits` runs; and of the biases' gradients, the column sums of G and V.
// 32,768 x 8192 in two parts by 1024 in one: 1115 us (0.99 PF); 202,612 x 704 by 128 of three parts: 316 us
template <class K> struct WeightSumArgs {
    Panel gv, x;             // [rows][2 f], [rows][d]
    int64_t d, m_tiles, n_tiles, run;   // rows of a run, a multiple of a step
    float *part, *bias;      // [splits][2 f][d], [splits][2 f]
    bool add;
};
template <class K, class B> using WeightSums = typename B::template Of<typename K::T, K::kFactors, K::kParts, false, false>;   // (d first, the 2 f columns second)
template <class K, class B> __device__ inline void weight_sums(const WeightSumArgs<K> &a, int64_t at, typename WeightSums<K, B>::Lds &lds)
{
    using P = WeightSums<K, B>;
    const int64_t tiles = a.m_tiles * a.n_tiles, s = at / tiles, tile = at % tiles;
    const int64_t m0 = tile / a.n_tiles * B::kRows, n0 = tile % a.n_tiles * B::kCols;
    const int64_t k0 = s * a.run, k1 = k0 + a.run < a.gv.rows ? k0 + a.run : a.gv.rows;
    const int wave = threadIdx.x >> 6;
    const bool sums = a.bias && n0 + B::first(wave) == 0;
    f32x16 acc[B::kPer / 32][2] = {}, ones[2] = {};
    P::run(a.x, a.gv, n0, m0, k0, k1, lds, acc, [&](auto &fb) {
        if (!sums) return;
        Half8<typename K::T> one;
#pragma unroll
        for (int k = 0; k < 8; ++k) one[k] = (typename K::T)1.f;
#pragma unroll
        for (int p = K::kParts - 1; p >= 0; --p)
#pragma unroll
            for (int j = 0; j < 2; ++j) ones[j] = mfma<typename K::T>(one, fb[j][p], ones[j]);
    });
    __syncthreads();
    constexpr int lanes = 16;
    const int lane = threadIdx.x & 63, c = lane % lanes * 4;
    const int64_t row0 = m0 + B::second(wave);
    const Turned turned{reinterpret_cast<float *>(&lds) + wave * 4096};
#pragma unroll
    for (int i = 0; i < B::kPer / 64; ++i) {
        turned.put(&acc[2 * i]);
#pragma unroll
        for (int k = 0; k < lanes; ++k) {
            const int r = lane / lanes + 64 / lanes * k;
            const int64_t row = row0 + r, col = n0 + B::first(wave) + 64 * i + c;
            if (row >= a.gv.cols) continue;
            float v[4], old[4] = {};
            turned.get(v, r, c);
            float *to = a.part + (s * a.gv.cols + row) * a.d;
            if (a.add) load_cols(old, to, 1, col, a.d);
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] += old[t];
            store_cols(v, to, col, a.d);
        }
    }
    if (sums && lane < 32) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t row = row0 + 32 * j + lane;
            float *to = a.bias + s * a.gv.cols + row;
            if (row < a.gv.cols) *to = a.add ? *to + ones[j][0] : ones[j][0];
        }
    }
}

template <class K, class B> __global__ __launch_bounds__(B::kThreads) void k_row_bars(RowBarArgs<K> a)
{
    __shared__ typename RowBars<K, B>::Lds lds;
    row_bars<K, B>(a, xcd_order(blockIdx.x, gridDim.x), lds);
}
template <class K, class B> __global__ __launch_bounds__(B::kThreads) void k_weight_sums(WeightSumArgs<K> a)
{
    __shared__ typename WeightSums<K, B>::Lds lds;
    weight_sums<K, B>(a, xcd_order(blockIdx.x, gridDim.x), lds);
}
// Both at once, where neither fills the chip
template <class K, class B> __global__ __launch_bounds__(B::kThreads) void k_row_bars_and_weight_sums(RowBarArgs<K> r, WeightSumArgs<K> w, unsigned of_rows)
{
    __shared__ union Both {
        typename RowBars<K, B>::Lds r;
        typename WeightSums<K, B>::Lds w;
        __device__ Both() {}
    } lds;
    if (blockIdx.x < of_rows) row_bars<K, B>(r, blockIdx.x, lds.r);
    else weight_sums<K, B>(w, blockIdx.x - of_rows, lds.w);
}

// The runs' shares added up, in their order
template <class K> struct JoinArgs {
    const float *part, *bias;
    int64_t splits, d, f, f2;
    typename K::E *dwg, *dwv, *dbg, *dbv;
    int64_t g_rs, g_cs, v_rs, v_cs;
};
// RUNS: of splits that a block's threads take side by side and then join in order: four for 32 splits and more (512 splits of 256 x 64: 19 us, 57 one after another), else one
template <class K, int RUNS> __global__ __launch_bounds__(256 * RUNS) void k_join(JoinArgs<K> a)
{
    __shared__ float tile[RUNS][8][33], sums[RUNS][8];
    const int64_t c0 = (int64_t)blockIdx.x * 8, d0 = (int64_t)blockIdx.y * 32, f0 = feature_of(c0);
    const bool value = is_value(c0);
    typename K::E *dw = value ? a.dwv : a.dwg, *db = value ? a.dbv : a.dbg;
    const int64_t rs = value ? a.v_rs : a.g_rs, cs = value ? a.v_cs : a.g_cs;
    const int run = threadIdx.x >> 8, t = threadIdx.x & 255, p = t & 31, q = t >> 5;
    const int64_t each = (a.splits + RUNS - 1) / RUNS, from = run * each, end = from + each < a.splits ? from + each : a.splits;
    float sum = 0.f;
    if (dw && d0 + p < a.d) in_steps<8>(from, end, 1, [&](int64_t s) { return a.part[(s * a.f2 + c0 + q) * a.d + d0 + p]; }, [&](float x) { sum += x; });
    tile[run][q][p] = sum;   // [feature][d]
    const bool bias = db && d0 == 0;
    if (bias && t < 8) {
        sum = 0.f;
        in_steps<8>(from, end, 1, [&](int64_t s) { return a.bias[s * a.f2 + c0 + t]; }, [&](float x) { sum += x; });
        sums[run][t] = sum;
    }
    __syncthreads();
    if (run) return;
    const bool by_row = cs <= rs;
    const int dd = by_row ? t >> 3 : p, ff = by_row ? t & 7 : q;
    if (dw && d0 + dd < a.d && f0 + ff < a.f) {
        sum = tile[0][ff][dd];
        for (int k = 1; k < RUNS; ++k) sum += tile[k][ff][dd];
        dw[(d0 + dd) * rs + (f0 + ff) * cs] = to_elem<typename K::E>(sum);
    }
    if (bias && t < 8 && f0 + t < a.f) {
        sum = sums[0][t];
        for (int k = 1; k < RUNS; ++k) sum += sums[k][t];
        db[f0 + t] = to_elem<typename K::E>(sum);
    }
}

// ---------------------------------------------------------------- a call's sizes and scratch memory

constexpr int64_t kChunkBytes = (int64_t)4 << 30;     // of x's parts, G and V of a chunk
constexpr int64_t kMostTiles = 1 << 23;       // blocks of a launch
constexpr int64_t kFull = 256;                // blocks that leave no compute unit idle
constexpr int64_t kNarrowBlocks = 1024;       // blocks of such a launch

struct Plan {
    int parts;                                 // of G, V and what they are multiplied with (without a gradient: of g's and v's factors)
    bool pack_x;
    int64_t d_p, f2, gv_ld, d_ld, chunk;       // columns of the laid out x and weights and where their rows lie, rows of a chunk
    int64_t splits, run;
    size_t across, down, x_tiles, xs, gv, part, bias, x_exponent, w_scale, bytes;   // offsets (x_exponent: and which rows fall short; w_scale: scales, exponents, which columns do)
};

// Whether a call goes by Scaled: large enough for its one more launch and the counts to pay (us, and by three bf16 parts: 3000 x 256 x 256 28 and 26, 4000 x 256 x 512 30 and 30,
// 2000 x 512 x 1024 42 and 44, 1024 x 1024 x 4096 111 and 135, 32,768 x 512 x 1365 343 and 635)
bool by_scale(const GatedArgs &a, bool grad) { return a.dtype == MLIP_DTYPE_F32 && !grad && a.d > kNarrow && (double)a.n * (double)a.d * (double)a.f >= 5e8; }

// x is read where it lies if its rows are whole lines of pieces and steps
bool reads_x(const GatedArgs &a)
{
    return a.dtype != MLIP_DTYPE_F32 && a.d % kPadK == 0 && a.x_cs == 1 && a.x_rs % 8 == 0 && a.x_rs >= a.d && a.x_rs <= (1 << 21) &&
           reinterpret_cast<uintptr_t>(a.x) % 16 == 0;
}

// f(Block{}) for a product of `cols` columns (of the first operand) and `rows` rows (of the second).  Large tiles if there are enough for half the compute units, or K is
// split for more (1500 x 300 x 700 in fp32: 44 us by 36 large tiles, 30 by 144).
template <class K, class Fn> void with_tile(int64_t cols, int64_t rows, bool split, Fn &&f)
{
    if (K::kParts <= 2 && cols >= 512 && rows >= 512 && (split || (double)cols * (double)rows >= 128.0 * 65536.0)) f(std::conditional_t<K::kParts <= 2, Large, Middle>{});
    else if (cols <= 64) f(Narrow{});
    else f(Middle{});
}

Plan plan_of(const GatedArgs &a, bool grad)
{
    Plan p{};
    const bool f32 = a.dtype == MLIP_DTYPE_F32, apart = a.dtype == MLIP_DTYPE_F16 && grad;
    const int factors = by_scale(a, grad) ? Scaled::kParts : f32 ? 3 : apart ? 2 : 1, tiles_parts = apart ? 1 : factors;   // parts of x and weights, and of those that make g and v
    p.parts = f32 || !grad ? factors : 2;
    p.pack_x = !reads_x(a);
    p.d_p = pad_to(a.d, kPadK);
    p.f2 = 2 * pad_to(a.f, 32);
    p.gv_ld = pad_odd(p.f2);
    p.d_ld = pad_odd(p.d_p);
    // (scratch memory does not depend on where x lies: a size asked for once holds for all)
    const int64_t row_bytes = ((grad ? p.gv_ld : 0) * p.parts + p.d_ld * factors) * 2;
    p.chunk = pad_to(kChunkBytes / row_bytes + 1, 1024);
    const int64_t most = kMostTiles / ((p.f2 > p.d_p ? p.f2 : p.d_p) / 64 + 1) * 64 / 1024 * 1024;
    if (p.chunk > most) p.chunk = most;
    const int64_t all = pad_to(a.n > 0 ? a.n : 1, 128);
    if (p.chunk > all) p.chunk = all;
    size_t at = 0;
    auto take = [&](int64_t bytes) { const size_t here = at; at += (size_t)pad_to(bytes, 256); return here; };
    p.across = take(p.f2 * p.d_ld * tiles_parts * 2);
    if (apart && a.d > kNarrow) p.x_tiles = take(p.chunk * p.d_ld * 2);
    if (grad || a.d > kNarrow) p.xs = take(p.chunk * p.d_ld * factors * 2);
    if (by_scale(a, grad)) p.x_exponent = take(2 * p.chunk * 4);
    if (a.dtype == MLIP_DTYPE_F32) p.w_scale = take(3 * p.f2 * 4);
    if (grad) {
        p.down = take(a.d * p.gv_ld * factors * 2);
        p.gv = take(p.chunk * p.gv_ld * p.parts * 2);
        const int64_t tiles = p.parts <= 2 && a.d >= 512 && p.f2 >= 512 ? (p.f2 + 255) / 256 * ((a.d + 255) / 256) : a.d <= 64 ? (p.f2 + 255) / 256 : (p.f2 + 127) / 128 * ((a.d + 127) / 128);
        const int64_t blocks = p.parts <= 2 && a.d >= 512 && p.f2 >= 512 ? 256 : 512;   // one or two to a compute unit
        int64_t splits = blocks / tiles, most_splits = (p.chunk + 127) / 128;
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

Plain plain_of(const GatedArgs &a)
{
    return {static_cast<const float *>(a.wg), static_cast<const float *>(a.wv), a.wg_rs, a.wg_cs, a.wv_rs, a.wv_cs, (int32_t)a.d, (int32_t)a.f};
}

// g: of a gradient (BACK)
template <class K, bool BACK> int launch(const GatedArgs &a, const GatedGrad *g)
{
    using E = typename K::E;
    using T = typename K::T;
    const Plan p = plan_of(a, BACK);
    char *ws = static_cast<char *>(a.workspace);
    using Tiles = InTiles<K>;
    constexpr bool apart = !std::is_same_v<T, typename Tiles::T>;   // whether the products with G and V have x in other parts than those that make g and v
    typename Tiles::T *across = reinterpret_cast<typename Tiles::T *>(ws + p.across), *x_tiles = reinterpret_cast<typename Tiles::T *>(ws + (apart ? p.x_tiles : p.xs));
    T *down = reinterpret_cast<T *>(ws + p.down), *xs = reinterpret_cast<T *>(ws + p.xs), *gv = reinterpret_cast<T *>(ws + p.gv);
    const bool in_registers = a.d <= kNarrow, strided = a.x_cs != 1 || (BACK && g->bar_cs != 1);
    const bool weights = BACK && (g->dwg || g->dwv || g->dbg || g->dbv);
    const Weights<K> w = {static_cast<const E *>(a.wg), static_cast<const E *>(a.wv), a.wg_rs, a.wg_cs, a.wv_rs, a.wv_cs, a.d, a.f, p.d_ld, p.gv_ld,
                          across, BACK && g->dx ? down : nullptr, p.f2 * p.d_ld, a.d * p.gv_ld};
    float *w_exponent = reinterpret_cast<float *>(ws + p.w_scale);
    int32_t *w_short = reinterpret_cast<int32_t *>(w_exponent + p.f2);
    if (a.n > 0 && in_registers && K::kParts == 3) {
        if constexpr (K::kParts == 3)
            k_pack_scaled_weights<K><<<(unsigned)(p.f2 / 32), kPackThreads, 0, a.stream>>>(w, p.d_p, reinterpret_cast<_Float16 *>(across), w_exponent, w_short);
    } else if (a.n > 0) k_pack_weights<K><<<dim3((unsigned)(p.f2 / 32), (unsigned)(p.d_p / 32)), kPackThreads, 0, a.stream>>>(w);
    const Panel across_panel = {across, p.d_ld, p.f2 * p.d_ld, p.f2, p.d_p}, down_panel = {down, p.gv_ld, a.d * p.gv_ld, a.d, p.f2};
    int64_t first = 0;
    do {
        const int64_t n = a.n - first < p.chunk ? a.n - first : p.chunk;
        if (n <= 0 && a.n > 0) break;
        const E *x = static_cast<const E *>(a.x) + first * a.x_rs;
        Panel xp = {x, a.x_rs, 0, n, a.d}, xw = xp;
        const unsigned pack_blocks = (unsigned)((n * (p.d_p / 8) + kPackThreads - 1) / kPackThreads);
        if (p.pack_x && n > 0 && (!in_registers || (weights && !apart))) {
            k_pack_rows<Tiles><<<pack_blocks, kPackThreads, 0, a.stream>>>(x, a.x_rs, a.x_cs, n, a.d, p.d_p, x_tiles, p.d_ld, p.chunk * p.d_ld);
            xp = xw = {x_tiles, p.d_ld, p.chunk * p.d_ld, n, p.d_p};
        }
        if (apart && n > 0 && weights) {
            k_pack_rows<K><<<pack_blocks, kPackThreads, 0, a.stream>>>(x, a.x_rs, a.x_cs, n, a.d, p.d_p, xs, p.d_ld, p.chunk * p.d_ld);
            xw = {xs, p.d_ld, p.chunk * p.d_ld, n, p.d_p};
        }
        if (n > 0) {
            GateArgs<K> ga = {xp, across_panel, p.d_p, a.f, 0, a.act, static_cast<const E *>(a.bg), static_cast<const E *>(a.bv)};
            if constexpr (!BACK) {
                ga.out = static_cast<E *>(a.out) + first * a.out_rs;
                ga.out_rs = a.out_rs;
            } else {
                ga.bar = static_cast<const E *>(g->bar) + first * g->bar_rs;
                ga.bar_rs = g->bar_rs;
                ga.bar_cs = g->bar_cs;
                ga.gv = gv;
                ga.gv_ld = p.gv_ld;
                ga.gv_part = p.chunk * p.gv_ld;
            }
            auto narrow = [&](auto steps) {
                constexpr int STEPS = decltype(steps)::value;
                const int64_t tiles = (n + 31) / 32, all = p.f2 / 64, pairs = (tiles + 3) / 4 * all < kFull ? 1 : NarrowShape<K, STEPS>::kPairs;
                NarrowArgs<K> na = {ga, a.x_cs, (all + pairs - 1) / pairs, tiles, 0, (int32_t)pairs};
                na.a.x = {x, a.x_rs, 0, n, a.d};
                na.a.w_exponent = w_exponent;
                na.a.w_short = w_short;
                na.a.plain = plain_of(a);
                const int64_t most = kNarrowBlocks / na.groups > 0 ? kNarrowBlocks / na.groups : 1, blocks = (na.tiles + 3) / 4;
                na.blocks = (int32_t)(blocks < most ? blocks : most);
                (strided ? k_gates_narrow<K, STEPS, BACK, true> : k_gates_narrow<K, STEPS, BACK, false>)<<<(unsigned)(na.blocks * na.groups), 256, 0, a.stream>>>(na);
            };
            if (in_registers && a.d <= 64) narrow(std::integral_constant<int, 4>{});
            else if (in_registers) narrow(std::integral_constant<int, 8>{});
            else with_tile<Tiles>(p.f2, n, false, [&](auto block) {
                using B = decltype(block);
                ga.n_tiles = (p.f2 + B::kCols - 1) / B::kCols;
                const unsigned blocks = (unsigned)((n + B::kRows - 1) / B::kRows * ga.n_tiles);
                k_gates<K, B, BACK><<<blocks, B::kThreads, 0, a.stream>>>(ga);
            });
        }
        if constexpr (BACK) {
            const Panel gp = {gv, p.gv_ld, p.chunk * p.gv_ld, n, p.f2};
            auto row_args = [&](auto block) {
                using B = decltype(block);
                return RowBarArgs<K>{gp, down_panel, (a.d + B::kCols - 1) / B::kCols, static_cast<E *>(g->dx) + first * g->dx_rs, g->dx_rs};
            };
            auto row_blocks = [&](auto block) {
                using B = decltype(block);
                return (n + B::kRows - 1) / B::kRows * ((a.d + B::kCols - 1) / B::kCols);
            };
            auto weight_args = [&](auto block) {
                using B = decltype(block);
                return WeightSumArgs<K>{gp, xw, a.d, (p.f2 + B::kRows - 1) / B::kRows, (a.d + B::kCols - 1) / B::kCols, p.run, reinterpret_cast<float *>(ws + p.part),
                                        g->dbg || g->dbv ? reinterpret_cast<float *>(ws + p.bias) : nullptr, first > 0};
            };
            bool together = false;
            if (g->dx && n > 0 && weights)
                with_tile<K>(a.d, n < p.f2 ? n : p.f2, false, [&](auto block) {
                    using B = decltype(block);
                    const WeightSumArgs<K> wa = weight_args(block);
                    const int64_t rb = row_blocks(block), wb = wa.m_tiles * wa.n_tiles * p.splits;
                    together = rb < kFull && wb < kFull && B::kThreads == 256;
                    if constexpr (B::kThreads == 256) {
                        if (together) k_row_bars_and_weight_sums<K, B><<<(unsigned)(rb + wb), B::kThreads, 0, a.stream>>>(row_args(block), wa, (unsigned)rb);
                    }
                });
            if (g->dx && n > 0 && !together)
                with_tile<K>(a.d, n, false, [&](auto block) {
                    k_row_bars<K, decltype(block)><<<(unsigned)row_blocks(block), decltype(block)::kThreads, 0, a.stream>>>(row_args(block));
                });
            if (weights && !together)
                with_tile<K>(a.d, p.f2, true, [&](auto block) {
                    const WeightSumArgs<K> wa = weight_args(block);
                    k_weight_sums<K, decltype(block)><<<(unsigned)(wa.m_tiles * wa.n_tiles * p.splits), decltype(block)::kThreads, 0, a.stream>>>(wa);
                });
        }
        first += p.chunk;
    } while (first < a.n);
    if constexpr (BACK) if (weights) {
        const JoinArgs<K> ja = {reinterpret_cast<float *>(ws + p.part), reinterpret_cast<float *>(ws + p.bias), p.splits, a.d, a.f, p.f2, static_cast<E *>(g->dwg),
                                static_cast<E *>(g->dwv), static_cast<E *>(g->dbg), static_cast<E *>(g->dbv), g->dwg_rs, g->dwg_cs, g->dwv_rs, g->dwv_cs};
        const dim3 blocks((unsigned)(p.f2 / 8), (unsigned)((a.d + 31) / 32));
        if (p.splits >= 32) k_join<K, 4><<<blocks, 1024, 0, a.stream>>>(ja);
        else k_join<K, 1><<<blocks, 256, 0, a.stream>>>(ja);
    }
    MLIP_HIP(hipGetLastError());
    return MLIP_OK;
}

int launch_scaled(const GatedArgs &a)
{
    const Plan p = plan_of(a, false);
    char *ws = static_cast<char *>(a.workspace);
    _Float16 *across = reinterpret_cast<_Float16 *>(ws + p.across), *xs = reinterpret_cast<_Float16 *>(ws + p.xs);
    float *x_exponent = reinterpret_cast<float *>(ws + p.x_exponent), *w_scale = reinterpret_cast<float *>(ws + p.w_scale), *w_exponent = w_scale + p.f2;
    int32_t *x_short = reinterpret_cast<int32_t *>(x_exponent + p.chunk), *w_short = reinterpret_cast<int32_t *>(w_exponent + p.f2);
    const Weights<Scaled> w = {static_cast<const float *>(a.wg), static_cast<const float *>(a.wv), a.wg_rs, a.wg_cs, a.wv_rs, a.wv_cs, a.d, a.f, p.d_ld, p.gv_ld,
                               across, nullptr, p.f2 * p.d_ld, 0, w_scale};
    k_column_scales<<<(unsigned)(p.f2 / 32), kScaleThreads, 0, a.stream>>>(w, w_scale, w_exponent, w_short);
    k_pack_weights<Scaled><<<dim3((unsigned)(p.f2 / 32), (unsigned)(p.d_p / 32)), kPackThreads, 0, a.stream>>>(w);
    for (int64_t first = 0; first < a.n; first += p.chunk) {
        const int64_t n = a.n - first < p.chunk ? a.n - first : p.chunk;
        k_pack_scaled_rows<<<(unsigned)((n + kPackThreads / 64 - 1) / (kPackThreads / 64)), kPackThreads, 0, a.stream>>>(
            static_cast<const float *>(a.x) + first * a.x_rs, a.x_rs, a.x_cs, n, a.d, p.d_p, xs, p.d_ld, p.chunk * p.d_ld, x_exponent, x_short);
        GateArgs<Scaled> ga = {{xs, p.d_ld, p.chunk * p.d_ld, n, p.d_p}, {across, p.d_ld, p.f2 * p.d_ld, p.f2, p.d_p}, p.d_p, a.f, 0, a.act,
                               static_cast<const float *>(a.bg), static_cast<const float *>(a.bv)};
        ga.out = static_cast<float *>(a.out) + first * a.out_rs;
        ga.out_rs = a.out_rs;
        ga.x_exponent = x_exponent;
        ga.w_exponent = w_exponent;
        ga.x_short = x_short;
        ga.w_short = w_short;
        ga.x_plain = static_cast<const float *>(a.x) + first * a.x_rs;
        ga.x_rs = a.x_rs;
        ga.x_cs = a.x_cs;
        ga.plain = plain_of(a);
        with_tile<Scaled>(p.f2, n, false, [&](auto block) {
            using B = decltype(block);
            ga.n_tiles = (p.f2 + B::kCols - 1) / B::kCols;
            k_gates<Scaled, B, false><<<(unsigned)((n + B::kRows - 1) / B::kRows * ga.n_tiles), B::kThreads, 0, a.stream>>>(ga);
        });
    }
    MLIP_HIP(hipGetLastError());
    return MLIP_OK;
}

}  // namespace

size_t gated_workspace(const GatedArgs &a, bool grad) { return plan_of(a, grad).bytes; }

int gated_impl(const GatedArgs &a)
{
    if (a.n == 0) return MLIP_OK;
    if (by_scale(a, false)) return launch_scaled(a);
    return with_kind<false>(a.dtype, [&](auto kind) { return launch<decltype(kind), false>(a, nullptr); });
}

int gated_grad_impl(const GatedArgs &a, const GatedGrad &g)
{
    return with_kind<true>(a.dtype, [&](auto kind) { return launch<decltype(kind), true>(a, &g); });
}

}  // namespace mlip
