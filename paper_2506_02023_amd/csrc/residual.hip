// A block's norms, gate and residual sum, and their gradient:  y = x + factor gate scale post(z),  n = pre(y).
//
// With N(t) = that w + b, that = (t - m) r, r = 1 / sqrt(mean of (t - m)^2 + eps), m the row's mean (layer) or 0 (rms), D the whole gradient of y and
// t = factor gate scale, p = post(z):
//   D = dy + r_y (B - yhat mean(B yhat) - mean(B)),  B = dn w_pre      (the last mean for layer only)
//   dx = D;  P = t D;  dz = r_z (C - zhat mean(C zhat) - mean(C)),  C = P w_post
//   dgate = factor scale p D, summed as the gate is spread;  dscale = sum over rows of factor gate p D
//   dw_post = sum P zhat, db_post = sum P, dw_pre = sum dn yhat, db_pre = sum dn   (over rows)
//
// Bound by memory: every row is read once and stays in registers, four columns of it in a lane (rows of up to 256 columns in part of a
// wavefront, wider ones in a block of their own), and all is fp32.  Wider rows have 128 registers a lane, because a block may have 1024 threads: the fp32 gradient spills 14 of them up
// to 4096 columns, all types 26 to 123 beyond (eight columns a lane; 16,384 x 8192 bf16: 697 us, its gradient 1.83 ms, floors 263 and 421).  The gradient starts from x and z again, so the forward pass keeps nothing.  Up to 4096 columns the
// next row is requested before the present one is worked on.
// 1,000,188 x 64 bf16 with both norms: 125 us (4.1 TB/s; 8 columns a lane 157), its gradient with 128 columns 433 us (4.7 TB/s; 8 columns a lane, each row loaded when its turn comes, 728).
// Sums over rows: each lane over the rows it meets, the lanes of a block joined in registers and LDS, the blocks in a second launch, all in a fixed order.
#include <type_traits>

#include "elem.h"

namespace mlip {
namespace {

constexpr int kThreads = 256;
constexpr int kMostThreads = 1024;
constexpr int kSums = 6;   // dscale, dw_post, db_post, dw_pre, db_pre, dgate of columns
enum { S_SCALE, S_POST_W, S_POST_B, S_PRE_W, S_PRE_B, S_GATE };

struct Input { const void *p; int64_t rs, cs; };
struct Back {
    Input dy, dn;
    void *dx, *dz, *dgate;
    int64_t dx_rs, dz_rs, dgate_rs;
    void *sum[kSums];     // final outputs
    float *part;          // [blocks][kSums][width] where there are several blocks
};
struct Args {
    Input x, z, gate;
    const void *scale, *post_w, *post_b, *pre_w, *pre_b;
    void *y, *norm;
    int64_t y_rs, norm_rs, n;
    int32_t width, gate_kind, params_f32;
    bool layer, post, pre;
    float eps, factor;
};

template <class E> using Four = Cols<E, 4>;

template <class E> __device__ inline Four<E> load4(const void *base, int64_t cs, int64_t at, int c, int width)
{
    const E *p = static_cast<const E *>(base) + at;
    Four<E> w = {};
    if (cs == 1 && c + 4 <= width) w = *reinterpret_cast<const Far<E, 4> *>(p + c);
    else
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k < width) w[k] = p[(c + k) * cs];
    return w;
}
template <class E> __device__ inline Four<E> narrow(const float (&v)[4])
{
    if constexpr (std::is_same_v<E, __bf16>) return __builtin_convertvector(Four<float>{v[0], v[1], v[2], v[3]}, Four<__bf16>);
    Four<E> w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = to_elem<E>(v[k]);
    return w;
}
template <class E> __device__ inline void store4(Four<E> w, void *base, int64_t at, int c, int width)
{
    E *p = static_cast<E *>(base) + at;
    if (c + 4 <= width) {
        *reinterpret_cast<Far<E, 4> *>(p + c) = w;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (c + k < width) p[c + k] = w[k];
}
// Four columns of a row of 4 or more, without a branch: past the end of the row the last four stand in, from which widen() takes those that belong, and zeros
template <class E> __device__ inline Four<E> load4_within(const void *base, int64_t at, int c, int width)
{
    return *reinterpret_cast<const Far<E, 4> *>(static_cast<const E *>(base) + at + (c + 4 <= width ? c : width - 4));
}
// beyond: columns by which the load stands further left than its place; fix: whether any lane of the wavefront has such a load
template <class E> __device__ inline void widen(float (&v)[4], Four<E> w, int beyond = 0, bool fix = false)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = (float)w[k];
    if (fix) {
        const float u[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = beyond == 0 ? u[k] : 0.f;
#pragma unroll
            for (int s = 1; s + k < 4; ++s) v[k] = beyond == s ? u[k + s] : v[k];
        }
    }
}
// A parameter's columns; `none` where there is no such parameter
template <class E> __device__ inline void param4(float (&v)[4], const void *p, bool f32, int c, int width, float none)
{
    if (!p) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = none;
    } else if (f32) widen<float>(v, load4<float>(p, 1, 0, c, width));
    else widen<E>(v, load4<E>(p, 1, 0, c, width));
}

// Lanes of a row: G of a wavefront, or (0) all of the block; N vectors of 4 columns each
template <int G_, int N_> struct Shape {
    static constexpr int G = G_, N = N_;
    static constexpr bool kWide = G == 0;
    static constexpr int kBlock = kWide ? kMostThreads : kThreads;   // at most
    static __device__ inline int lanes() { return kWide ? (int)blockDim.x : G; }
    static __device__ inline int lane() { return kWide ? (int)threadIdx.x : (int)threadIdx.x % (kWide ? 1 : G); }
    static constexpr int kRows = kWide ? 1 : kThreads / (kWide ? 1 : G);
};

// Sum over G neighbouring lanes, for all of them
template <int G> __device__ inline float lanes_sum(float v)
{
    auto moved = [](float x, auto way) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(way)::value, 0xf, 0xf, true)); };
    if constexpr (G >= 2) v += moved(v, std::integral_constant<int, 0xb1>{});    // neighbours in pairs,
    if constexpr (G >= 4) v += moved(v, std::integral_constant<int, 0x4e>{});    // pairs in fours,
    if constexpr (G >= 8) v += moved(v, std::integral_constant<int, 0x141>{});   // halves of eight mirrored,
    if constexpr (G >= 16) v += moved(v, std::integral_constant<int, 0x140>{});  // and of sixteen
    if constexpr (G >= 32) v += __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401f));   // lane ^ 16
    if constexpr (G >= 64) v += __shfl_xor(v, 32);
    return v;
}

// Columns of a row that wavefront w of its block has
template <class S> __device__ inline float row_cols(int w, int width)
{
    int cols = 0;
#pragma unroll
    for (int i = 0; i < S::N; ++i) {
        const int from = (i * S::lanes() + w * 64) * 4, left = width - from;
        cols += left < 0 ? 0 : left < 256 ? left : 256;
    }
    return (float)cols;
}

// What the wavefronts of a row exchange: two values of each, in the half of the memory that was not used last
struct Exchange {
    float (*at)[2][kMostThreads / 64];   // [2]
    int turn;
    __device__ inline void put(float a, float b)
    {
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
            at[turn][0][threadIdx.x >> 6] = a;
            at[turn][1][threadIdx.x >> 6] = b;
        }
        // a barrier for what lies in LDS alone: loads and stores of rows go on
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    }
};

// Sums of a and b over the lanes of a row
template <class S> __device__ inline void row_sum(float &a, float &b, Exchange &x)
{
    a = lanes_sum<S::kWide ? 64 : S::G>(a);
    b = lanes_sum<S::kWide ? 64 : S::G>(b);
    if constexpr (S::kWide) {
        x.put(a, b);
        a = b = 0.f;
        for (int w = 0; w < (int)blockDim.x / 64; ++w) {
            a += x.at[x.turn][0][w];
            b += x.at[x.turn][1][w];
        }
    }
}
template <class S> __device__ inline float row_sum(float a, Exchange &x)
{
    float none = 0.f;
    if constexpr (!S::kWide) return lanes_sum<S::G>(a);
    row_sum<S>(a, none, x);
    return a;
}

// t becomes that; returns r.  Over several wavefronts the squares are summed about each wavefront's own mean, and the means' about the row's, so that one exchange
// will do: mine = columns of this wavefront.
template <class S> __device__ inline float normalise(float (&t)[S::N][4], const Args &a, float inv, bool ragged, float mine, Exchange &x)
{
    constexpr int G = S::kWide ? 64 : S::G;
    const int c0 = S::lane() * 4, step = S::lanes() * 4;
    float sum = 0.f, mean = 0.f, sq = 0.f;
    if (a.layer) {
#pragma unroll
        for (int i = 0; i < S::N; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum += t[i][k];
        sum = lanes_sum<G>(sum);
        mean = S::kWide ? sum / fmaxf(mine, 1.f) : sum * inv;
#pragma unroll
        for (int i = 0; i < S::N; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) t[i][k] -= mean;
        if (ragged)
#pragma unroll
            for (int i = 0; i < S::N; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) t[i][k] = c0 + i * step + k < a.width ? t[i][k] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < S::N; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) sq = fmaf(t[i][k], t[i][k], sq);
    sq = lanes_sum<G>(sq);
    if constexpr (S::kWide) {
        x.put(sq, sum);
        const int waves = blockDim.x / 64;
        float all = 0.f;
        sq = 0.f;
        for (int w = 0; w < waves; ++w) {
            sq += x.at[x.turn][0][w];
            all += x.at[x.turn][1][w];
        }
        if (a.layer) {
            all *= inv;   // the row's mean
            for (int w = 0; w < waves; ++w) {
                const float cols = row_cols<S>(w, a.width), d = x.at[x.turn][1][w] / fmaxf(cols, 1.f) - all;
                sq = fmaf(cols * d, d, sq);
            }
            const float shift = mean - all;
#pragma unroll
            for (int i = 0; i < S::N; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) t[i][k] = !ragged || c0 + i * step + k < a.width ? t[i][k] + shift : 0.f;
        }
    }
    const float r = 1.f / sqrtf(fmaf(sq, inv, a.eps));
#pragma unroll
    for (int i = 0; i < S::N; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) t[i][k] *= r;
    return r;
}

// bar, the gradient of that, becomes the gradient of t
template <class S> __device__ inline void normalise_back(float (&bar)[S::N][4], const float (&hat)[S::N][4], float r, const Args &a, float inv, bool ragged, Exchange &x)
{
    const int c0 = S::lane() * 4, step = S::lanes() * 4;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < S::N; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) s1 = fmaf(bar[i][k], hat[i][k], s1);
    if (a.layer) {
#pragma unroll
        for (int i = 0; i < S::N; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) s0 += bar[i][k];
        row_sum<S>(s0, s1, x);
    } else s1 = row_sum<S>(s1, x);
    const float mean = s0 * inv, along = s1 * inv;
#pragma unroll
    for (int i = 0; i < S::N; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) bar[i][k] = r * (bar[i][k] - fmaf(hat[i][k], along, mean));   // (a row of equal gradients comes out as zeros)
    if (ragged)
#pragma unroll
        for (int i = 0; i < S::N; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) bar[i][k] = c0 + i * step + k < a.width ? bar[i][k] : 0.f;
}

// PLAIN: rows of four columns or more, the columns one after another in all inputs
template <class E, class S, bool BACK, bool PLAIN> __global__ __launch_bounds__(S::kBlock, S::kWide ? 4 : 1) void k_residual(Args a, Back b)
{
    constexpr int N = S::N;
    __shared__ float between[2][2][kMostThreads / 64];
    __shared__ float sums[BACK && !S::kWide ? kThreads / 64 : 1][BACK && !S::kWide ? S::G * 4 : 1];
    Exchange ex{between, 0};
    const int c0 = S::lane() * 4, step = S::lanes() * 4;
    const float inv = 1.f / (float)a.width, mine = S::kWide ? row_cols<S>(threadIdx.x >> 6, a.width) : 0.f;
    const bool ragged = a.width != N * step;
    auto col = [&](int i) { return c0 + i * step; };
    const bool gate_cols = a.gate_kind == MLIP_RESIDUAL_GATE_COL, gate_full = a.gate_kind == MLIP_RESIDUAL_GATE_FULL, gate_row = a.gate_kind == MLIP_RESIDUAL_GATE_ROW;

    // the parameters' columns stay in registers where a lane has four, and come from the caches where it has more.
    struct Params { float scale[4], gate[4], post_w[4], post_b[4], pre_w[4], pre_b[4]; };
    auto params_of = [&](Params &p, int i) {
        param4<E>(p.scale, a.scale, a.params_f32, col(i), a.width, 1.f);
        param4<E>(p.gate, gate_cols ? a.gate.p : nullptr, false, col(i), a.width, 1.f);
        param4<E>(p.post_w, a.post_w, a.params_f32, col(i), a.width, 1.f);
        param4<E>(p.post_b, a.post_b, a.params_f32, col(i), a.width, 0.f);
        param4<E>(p.pre_w, a.pre_w, a.params_f32, col(i), a.width, 1.f);
        param4<E>(p.pre_b, a.pre_b, a.params_f32, col(i), a.width, 0.f);
    };
    Params held;
    if constexpr (N == 1) params_of(held, 0);

    struct Raw { Four<E> x[N], z[N], gate[N], dy[N], dn[N]; E g; };
    int beyond[N];
    bool fix[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        beyond[i] = PLAIN && col(i) + 4 > a.width ? col(i) + 4 - a.width : 0;
        fix[i] = __ballot(beyond[i] != 0) != 0;
    }
    auto load = [&](Raw &w, int64_t r0) {
        int64_t row = r0 + (S::kWide ? 0 : threadIdx.x / (S::kWide ? 1 : S::G));
        if (row >= a.n) row = a.n - 1;
        auto take = [&](Four<E> (&to)[N], const Input &from) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (PLAIN) to[i] = load4_within<E>(from.p, row * from.rs, col(i), a.width);
                else to[i] = load4<E>(from.p, from.cs, row * from.rs, col(i), a.width);
            }
        };
        take(w.x, a.x);
        if (a.z.p) take(w.z, a.z);
        if (gate_full) take(w.gate, a.gate);
        if constexpr (BACK) {
#pragma unroll
            for (int i = 0; i < N; ++i) w.dy[i] = w.dn[i] = Four<E>{};
            if (b.dy.p) take(w.dy, b.dy);
            if (b.dn.p) take(w.dn, b.dn);
        }
        if (gate_row) w.g = static_cast<const E *>(a.gate.p)[row * a.gate.rs];
    };

    // A row's results are stored when the next row has come: a wait for loads is one for all stores made before them, which take longest.
    struct Done { Four<E> first[N], second[N], gate[N]; } done;   // y and norm, or dx, dz and dgate
    int64_t done_row = -1;
    auto store = [&] {
        if (done_row < 0) return;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (BACK) {
                if (b.dx) store4<E>(done.first[i], b.dx, done_row * b.dx_rs, col(i), a.width);
                if (b.dz) store4<E>(done.second[i], b.dz, done_row * b.dz_rs, col(i), a.width);
                if (gate_full && b.dgate) store4<E>(done.gate[i], b.dgate, done_row * b.dgate_rs, col(i), a.width);
            } else {
                if (a.y) store4<E>(done.first[i], a.y, done_row * a.y_rs, col(i), a.width);
                if (a.pre) store4<E>(done.second[i], a.norm, done_row * a.norm_rs, col(i), a.width);
            }
        }
    };

    float sum[BACK ? kSums : 1][N][4] = {};
    const int64_t stride = (int64_t)gridDim.x * S::kRows;
    Raw next;
    int64_t r0 = (int64_t)blockIdx.x * S::kRows;
    if (N == 1 && r0 < a.n) load(next, r0);
    // (all lanes of a block make the same number of rounds: rows of several wavefronts meet at barriers)
    for (; r0 < a.n; r0 += stride) {
        const int64_t row = r0 + (S::kWide ? 0 : threadIdx.x / (S::kWide ? 1 : S::G));
        const bool there = row < a.n;
        float y[N][4], zh[N][4], gate[N][4], dy[N][4], dn[N][4];
        if (N > 1) load(next, r0);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            widen<E>(y[i], next.x[i], beyond[i], fix[i]);
            if (a.z.p) widen<E>(zh[i], next.z[i], beyond[i], fix[i]);
            if (gate_full) widen<E>(gate[i], next.gate[i], beyond[i], fix[i]);
            else {
                const float g = gate_row ? (float)next.g : 1.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) gate[i][k] = g;
            }
            if constexpr (BACK) {
                widen<E>(dy[i], next.dy[i], beyond[i], fix[i]);
                widen<E>(dn[i], next.dn[i], beyond[i], fix[i]);
            }
        }
        store();
        done_row = there ? row : -1;
        if (N == 1 && r0 + stride < a.n) load(next, r0 + stride);
        float rz = 1.f;
        if (a.z.p) {
            if (a.post) rz = normalise<S>(zh, a, inv, ragged, mine, ex);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (N > 1) params_of(held, i);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    gate[i][k] *= held.gate[k] * a.factor;   // (from here on with the factor)
                    y[i][k] = fmaf(gate[i][k] * held.scale[k], fmaf(zh[i][k], held.post_w[k], held.post_b[k]), y[i][k]);
                }
            }
        }
        if constexpr (!BACK) {
#pragma unroll
            for (int i = 0; i < N; ++i) done.first[i] = narrow<E>(y[i]);
            if (!a.pre) continue;
            normalise<S>(y, a, inv, ragged, mine, ex);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (N > 1) params_of(held, i);
#pragma unroll
                for (int k = 0; k < 4; ++k) y[i][k] = fmaf(y[i][k], held.pre_w[k], held.pre_b[k]);
                done.second[i] = narrow<E>(y[i]);
            }
        } else {
            if (a.pre) {
                const float ry = normalise<S>(y, a, inv, ragged, mine, ex);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (there && b.sum[S_PRE_W])
#pragma unroll
                        for (int k = 0; k < 4; ++k) sum[S_PRE_W][i][k] = fmaf(dn[i][k], y[i][k], sum[S_PRE_W][i][k]);
                    if (there && b.sum[S_PRE_B])
#pragma unroll
                        for (int k = 0; k < 4; ++k) sum[S_PRE_B][i][k] += dn[i][k];
                    if constexpr (N > 1) params_of(held, i);
#pragma unroll
                    for (int k = 0; k < 4; ++k) dn[i][k] *= held.pre_w[k];
                }
                normalise_back<S>(dn, y, ry, a, inv, ragged, ex);
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) dy[i][k] += dn[i][k];
            }
#pragma unroll
            for (int i = 0; i < N; ++i) done.first[i] = narrow<E>(dy[i]);
            if (!a.z.p) continue;
            float gate_sum = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (N > 1) params_of(held, i);
                float pd[4], bar[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    pd[k] = fmaf(zh[i][k], held.post_w[k], held.post_b[k]) * dy[i][k];
                    bar[k] = dy[i][k] * gate[i][k] * held.scale[k];
                }
                if (there && b.sum[S_SCALE])
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[S_SCALE][i][k] = fmaf(pd[k], gate[i][k], sum[S_SCALE][i][k]);
                if (there && b.sum[S_POST_W])
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[S_POST_W][i][k] = fmaf(bar[k], zh[i][k], sum[S_POST_W][i][k]);
                if (there && b.sum[S_POST_B])
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[S_POST_B][i][k] += bar[k];
                if (a.gate_kind != MLIP_RESIDUAL_GATE_NONE) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        pd[k] *= held.scale[k] * a.factor;
                        gate_sum += pd[k];
                    }
                    if (there && b.sum[S_GATE])
#pragma unroll
                        for (int k = 0; k < 4; ++k) sum[S_GATE][i][k] += pd[k];
                    done.gate[i] = narrow<E>(pd);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) dy[i][k] = a.post ? bar[k] * held.post_w[k] : bar[k];
            }
            if (gate_row && b.dgate) {
                gate_sum = row_sum<S>(gate_sum, ex);
                if (there && S::lane() == 0) static_cast<E *>(b.dgate)[row * b.dgate_rs] = to_elem<E>(gate_sum);
            }
            if (a.post && b.dz) normalise_back<S>(dy, zh, rz, a, inv, ragged, ex);
#pragma unroll
            for (int i = 0; i < N; ++i) done.second[i] = narrow<E>(dy[i]);
        }
    }
    store();
    if constexpr (BACK) {
#pragma unroll
        for (int s = 0; s < kSums; ++s) {
            if (!b.sum[s]) continue;
            const bool f32 = b.part || (a.params_f32 && s != S_GATE);
            void *to = b.part ? static_cast<void *>(b.part + ((int64_t)blockIdx.x * kSums + s) * a.width) : b.sum[s];
            if constexpr (S::kWide) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (f32) store4<float>(narrow<float>(sum[s][i]), to, 0, col(i), a.width);
                    else store4<E>(narrow<E>(sum[s][i]), to, 0, col(i), a.width);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float v = sum[s][0][k];
#pragma unroll
                    for (int d = S::G; d < 64; d <<= 1) v += __shfl_xor(v, d);
                    if ((int)(threadIdx.x & 63) < S::G) sums[threadIdx.x >> 6][c0 + k] = v;
                }
                __syncthreads();
                for (int c = threadIdx.x; c < a.width; c += kThreads) {
                    float v = 0.f;
                    for (int w = 0; w < kThreads / 64; ++w) v += sums[w][c];
                    if (f32) static_cast<float *>(to)[c] = v;
                    else static_cast<E *>(to)[c] = to_elem<E>(v);
                }
                __syncthreads();
            }
        }
    }
}

// The blocks' sums added up, in their order: 32 columns a block, eight runs of blocks each
template <class E> __global__ __launch_bounds__(kThreads) void k_residual_join(Back b, int32_t blocks, int32_t width, bool params_f32)
{
    __shared__ float run[8][32];
    const int s = blockIdx.y, c = blockIdx.x * 32 + (threadIdx.x & 31), q = threadIdx.x >> 5;
    if (!b.sum[s]) return;
    float sum = 0.f;
    if (c < width) in_steps<8>(q, blocks, 8, [&](int64_t k) { return b.part[(k * kSums + s) * width + c]; }, [&](float x) { sum += x; });
    run[q][threadIdx.x & 31] = sum;
    __syncthreads();
    if (q || c >= width) return;
    for (int k = 1; k < 8; ++k) sum += run[k][threadIdx.x];
    if (params_f32 && s != S_GATE) static_cast<float *>(b.sum[s])[c] = sum;
    else static_cast<E *>(b.sum[s])[c] = to_elem<E>(sum);
}

// f(Shape{}, threads of a block)
template <class Fn> void with_shape(int64_t width, Fn &&f)
{
    if (width <= 8) f(Shape<2, 1>{}, kThreads);
    else if (width <= 16) f(Shape<4, 1>{}, kThreads);
    else if (width <= 32) f(Shape<8, 1>{}, kThreads);
    else if (width <= 64) f(Shape<16, 1>{}, kThreads);
    else if (width <= 128) f(Shape<32, 1>{}, kThreads);
    else if (width <= 256) f(Shape<64, 1>{}, kThreads);
    else if (width <= 4096) f(Shape<0, 1>{}, (int)(width + 255) / 256 * 64);   // wavefronts of 256 columns, or of 512
    else f(Shape<0, 2>{}, (int)(width + 511) / 512 * 64);
}

// Blocks of the gradient: a block's sums take as much as a few rows
int64_t back_blocks(int64_t n, int64_t width)
{
    int64_t blocks = 0;
    with_shape(width, [&](auto s, int threads) {
        const int64_t rounds = (n + decltype(s)::kRows - 1) / decltype(s)::kRows;
        const int64_t most = 256 * (1024 / threads);   // sixteen wavefronts to a compute unit
        blocks = rounds <= 8 ? 1 : (rounds + 3) / 4;   // (one block needs no second launch)
        if (blocks > most) blocks = most;
    });
    return blocks < 1 ? 1 : blocks;
}

template <bool BACK> int run(const ResidualArgs &a, const Back &b0, int64_t blocks)
{
    auto along = [](const Input &m) { return !m.p || m.cs == 1; };
    const bool plain = a.width >= 4 && a.x_cs == 1 && (!a.z || a.z_cs == 1) && (a.gate_kind != MLIP_RESIDUAL_GATE_FULL || a.gate_cs == 1) && along(b0.dy) && along(b0.dn);
    Args d{{a.x, a.x_rs, a.x_cs}, {a.z, a.z_rs, a.z_cs}, {a.gate, a.gate_rs, a.gate_cs}, a.scale, a.post_w, a.post_b, a.pre_w, a.pre_b, a.y, a.norm, a.y_rs, a.norm_rs, a.n,
           (int32_t)a.width, a.gate_kind, a.param_dtype == MLIP_DTYPE_F32, a.kind == MLIP_NORM_LAYER, a.post, a.pre, a.eps, a.factor};
    with_elem(a.dtype, [&](auto e) {
        using E = decltype(e);
        with_shape(a.width, [&](auto s, int threads) {
            using S = decltype(s);
            (plain ? k_residual<E, S, BACK, true> : k_residual<E, S, BACK, false>)<<<(unsigned)blocks, threads, 0, a.stream>>>(d, b0);
        });
        if (BACK && b0.part)
            k_residual_join<E><<<dim3((unsigned)((a.width + 31) / 32), kSums), kThreads, 0, a.stream>>>(b0, (int32_t)blocks, (int32_t)a.width, d.params_f32);
    });
    MLIP_HIP(hipGetLastError());
    return MLIP_OK;
}

}  // namespace

size_t residual_grad_workspace(int64_t n, int64_t width)
{
    const int64_t blocks = back_blocks(n, width);
    return blocks > 1 ? (size_t)(blocks * kSums * width) * sizeof(float) : 0;
}

int residual_impl(const ResidualArgs &a)
{
    if (a.n == 0) return MLIP_OK;
    int64_t blocks = 0;
    with_shape(a.width, [&](auto s, int) { blocks = (a.n + decltype(s)::kRows - 1) / decltype(s)::kRows; });
    const int64_t most = 2048;
    return run<false>(a, Back{}, blocks < most ? blocks : most);
}

int residual_grad_impl(const ResidualArgs &a, const ResidualGrad &g)
{
    const int64_t blocks = back_blocks(a.n, a.width);
    Back b{{g.dy, g.dy_rs, g.dy_cs}, {g.dn, g.dn_rs, g.dn_cs}, g.dx, g.dz, a.gate_kind == MLIP_RESIDUAL_GATE_COL ? nullptr : g.dgate, g.dx_rs, g.dz_rs, g.dgate_rs,
           {g.dscale, g.dpost_w, g.dpost_b, g.dpre_w, g.dpre_b, a.gate_kind == MLIP_RESIDUAL_GATE_COL ? g.dgate : nullptr}, nullptr};
    bool any = false;
    for (void *s : b.sum) any |= s != nullptr;
    if (any && blocks > 1) b.part = static_cast<float *>(g.workspace);
    if (a.n == 0 && !any) return MLIP_OK;
    ResidualArgs used = a;
    used.pre = a.pre && g.dn;   // a norm that nobody used: nothing comes back through it, not even where it is NaN
    return run<true>(used, b, blocks);
}

}  // namespace mlip
