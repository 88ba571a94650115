// A block's norms, gate and residual sum, and their gradient:  y = x + factor gate scale post(z),  n = pre(y).
//
// With N(t) = that w + b, that = (t - m) r, r = 1 / sqrt(mean of (t - m)^2 + eps), m the row's mean (layer) or 0 (rms), D the whole gradient of y and
// t = factor gate scale, p = post(z):
//   D = dy + r_y (B - yhat mean(B yhat) - mean(B)),  B = dn w_pre      (the last mean for layer only)
//   dx = D;  P = t D;  dz = r_z (C - zhat mean(C zhat) - mean(C)),  C = P w_post
//   dgate = factor scale p D, summed as the gate is spread;  dscale = sum over rows of factor gate p D
//   dw_post = sum P zhat, db_post = sum P, dw_pre = sum dn yhat, db_pre = sum dn   (over rows)
//
// Bound by memory: every row is read once and stays in registers, 8 columns of a row in each of G lanes (rows of up to 512 columns in
// part of a wavefront, wider ones in several), and all is fp32.  The gradient starts from x and z again, so the forward pass keeps nothing.
// Sums over rows: each lane over the rows it meets, the lanes of a block joined in registers and LDS, the blocks in a second launch, all in a fixed order.
#include "elem.h"

namespace mlip {
namespace {

constexpr int kThreads = 256;
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

template <class E> __device__ inline void load8(float (&v)[8], const void *base, int64_t cs, int64_t at, int c, int width)
{
    const E *p = static_cast<const E *>(base) + at;
    if (cs == 1 && c + 8 <= width) {
        const Cols<E, 8> w = *reinterpret_cast<const Far<E, 8> *>(p + c);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (float)w[k];
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = c + k < width ? (float)p[(c + k) * cs] : 0.f;
}
template <class E> __device__ inline void store8(const float (&v)[8], void *base, int64_t at, int c, int width)
{
    E *p = static_cast<E *>(base) + at;
    if (c + 8 <= width) {
        Cols<E, 8> w;
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = to_elem<E>(v[k]);
        *reinterpret_cast<Far<E, 8> *>(p + c) = w;
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (c + k < width) p[c + k] = to_elem<E>(v[k]);
}
// A parameter's columns; `none` where there is no such parameter
template <class E> __device__ inline void param8(float (&v)[8], const void *p, bool f32, int c, int width, float none)
{
    if (!p) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = none;
    } else if (f32) load8<float>(v, p, 1, 0, c, width);
    else load8<E>(v, p, 1, 0, c, width);
}

// Lanes of a row: G, in one wavefront or several; N vectors of 8 columns each
template <int G_, int N_> struct Shape {
    static constexpr int G = G_, N = N_, kBlock = G > kThreads ? G : kThreads, kRows = kBlock / G;
    static constexpr int kWaves = kBlock / 64;
};

template <class S> struct Red { float v[2][2][S::kWaves]; };

// Sums of a and b over the lanes of a row; turn: which half of the scratch memory, the other one than the last time
template <class S> __device__ inline void row_sum(float &a, float &b, Red<S> &red, int &turn)
{
    constexpr int in_wave = S::G < 64 ? S::G : 64;
#pragma unroll
    for (int d = in_wave / 2; d; d >>= 1) {
        a += __shfl_xor(a, d);
        b += __shfl_xor(b, d);
    }
    if constexpr (S::G > 64) {
        const int wave = threadIdx.x >> 6, first = threadIdx.x / S::G * (S::G / 64);
        if ((threadIdx.x & 63) == 0) {
            red.v[turn][0][wave] = a;
            red.v[turn][1][wave] = b;
        }
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int w = 0; w < S::G / 64; ++w) {
            a += red.v[turn][0][first + w];
            b += red.v[turn][1][first + w];
        }
        turn ^= 1;
    }
}

// t becomes that; returns r
template <class S> __device__ inline float normalise(float (&t)[S::N][8], const Args &a, int c0, float inv, Red<S> &red, int &turn)
{
    float none = 0.f;
    if (a.layer) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < S::N; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += t[i][k];
        row_sum<S>(sum, none, red, turn);
        const float mean = sum * inv;
#pragma unroll
        for (int i = 0; i < S::N; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) t[i][k] = c0 + i * S::G * 8 + k < a.width ? t[i][k] - mean : 0.f;
    }
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < S::N; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) sq = fmaf(t[i][k], t[i][k], sq);
    row_sum<S>(sq, none, red, turn);
    const float r = 1.f / sqrtf(fmaf(sq, inv, a.eps));
#pragma unroll
    for (int i = 0; i < S::N; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) t[i][k] *= r;
    return r;
}

// bar, the gradient of that, becomes the gradient of t
template <class S> __device__ inline void normalise_back(float (&bar)[S::N][8], const float (&hat)[S::N][8], float r, const Args &a, int c0, float inv, Red<S> &red, int &turn)
{
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < S::N; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            s0 += bar[i][k];
            s1 = fmaf(bar[i][k], hat[i][k], s1);
        }
    row_sum<S>(s0, s1, red, turn);
    const float mean = a.layer ? s0 * inv : 0.f, along = s1 * inv;
#pragma unroll
    for (int i = 0; i < S::N; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) bar[i][k] = c0 + i * S::G * 8 + k < a.width ? r * (bar[i][k] - fmaf(hat[i][k], along, mean)) : 0.f;
}

template <class E, class S, bool BACK> __global__ __launch_bounds__(S::kBlock) void k_residual(Args a, Back b)
{
    __shared__ Red<S> red;
    __shared__ float sums[BACK && S::kRows > 1 ? S::kWaves : 1][BACK && S::kRows > 1 ? S::G * 8 * S::N : 1];
    int turn = 0;
    const int lane = threadIdx.x % S::G, c0 = lane * 8;
    const float inv = 1.f / (float)a.width;
    auto col = [&](int i) { return c0 + i * S::G * 8; };
    float scale[S::N][8], post_w[S::N][8], post_b[S::N][8], pre_w[S::N][8], pre_b[S::N][8], gate_c[S::N][8];
#pragma unroll
    for (int i = 0; i < S::N; ++i) {
        param8<E>(scale[i], a.scale, a.params_f32, col(i), a.width, 1.f);
        param8<E>(post_w[i], a.post_w, a.params_f32, col(i), a.width, 1.f);
        param8<E>(post_b[i], a.post_b, a.params_f32, col(i), a.width, 0.f);
        param8<E>(pre_w[i], a.pre_w, a.params_f32, col(i), a.width, 1.f);
        param8<E>(pre_b[i], a.pre_b, a.params_f32, col(i), a.width, 0.f);
        param8<E>(gate_c[i], a.gate_kind == MLIP_RESIDUAL_GATE_COL ? a.gate.p : nullptr, false, col(i), a.width, 1.f);
#pragma unroll
        for (int k = 0; k < 8; ++k) scale[i][k] *= a.factor;
    }
    float sum[BACK ? kSums : 1][S::N][8] = {};
    // (all lanes of a block make the same number of rounds: rows of several wavefronts meet at barriers)
    for (int64_t r0 = (int64_t)blockIdx.x * S::kRows; r0 < a.n; r0 += (int64_t)gridDim.x * S::kRows) {
        const int64_t row_at = r0 + threadIdx.x / S::G;
        const bool there = row_at < a.n;
        const int64_t row = there ? row_at : a.n - 1;
        float y[S::N][8], zh[S::N][8], gate[S::N][8], dy[S::N][8], dn[S::N][8];
#pragma unroll
        for (int i = 0; i < S::N; ++i) {
            load8<E>(y[i], a.x.p, a.x.cs, row * a.x.rs, col(i), a.width);
            if (a.z.p) load8<E>(zh[i], a.z.p, a.z.cs, row * a.z.rs, col(i), a.width);
            if (a.gate_kind == MLIP_RESIDUAL_GATE_FULL) load8<E>(gate[i], a.gate.p, a.gate.cs, row * a.gate.rs, col(i), a.width);
            else {
                const float g = a.gate_kind == MLIP_RESIDUAL_GATE_ROW ? (float)static_cast<const E *>(a.gate.p)[row * a.gate.rs] : 1.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) gate[i][k] = gate_c[i][k] * g;
            }
            if constexpr (BACK) {
#pragma unroll
                for (int k = 0; k < 8; ++k) dy[i][k] = dn[i][k] = 0.f;
                if (b.dy.p) load8<E>(dy[i], b.dy.p, b.dy.cs, row * b.dy.rs, col(i), a.width);
                if (b.dn.p) load8<E>(dn[i], b.dn.p, b.dn.cs, row * b.dn.rs, col(i), a.width);
            }
        }
        float rz = 1.f;
        if (a.z.p) {
            if (a.post) rz = normalise<S>(zh, a, c0, inv, red, turn);
#pragma unroll
            for (int i = 0; i < S::N; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) y[i][k] = fmaf(gate[i][k] * scale[i][k], fmaf(zh[i][k], post_w[i][k], post_b[i][k]), y[i][k]);
        }
        if constexpr (!BACK) {
            if (a.y && there)
#pragma unroll
                for (int i = 0; i < S::N; ++i) store8<E>(y[i], a.y, row * a.y_rs, col(i), a.width);
            if (!a.pre) continue;
            normalise<S>(y, a, c0, inv, red, turn);
            if (there)
#pragma unroll
                for (int i = 0; i < S::N; ++i) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[i][k] = fmaf(y[i][k], pre_w[i][k], pre_b[i][k]);
                    store8<E>(y[i], a.norm, row * a.norm_rs, col(i), a.width);
                }
        } else {
            if (a.pre) {
                const float ry = normalise<S>(y, a, c0, inv, red, turn);
#pragma unroll
                for (int i = 0; i < S::N; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (there) {
                            sum[S_PRE_W][i][k] = fmaf(dn[i][k], y[i][k], sum[S_PRE_W][i][k]);
                            sum[S_PRE_B][i][k] += dn[i][k];
                        }
                        dn[i][k] *= pre_w[i][k];
                    }
                normalise_back<S>(dn, y, ry, a, c0, inv, red, turn);
#pragma unroll
                for (int i = 0; i < S::N; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) dy[i][k] += dn[i][k];
            }
            if (b.dx && there)
#pragma unroll
                for (int i = 0; i < S::N; ++i) store8<E>(dy[i], b.dx, row * b.dx_rs, col(i), a.width);
            if (!a.z.p) continue;
            float gate_sum = 0.f, none = 0.f;
#pragma unroll
            for (int i = 0; i < S::N; ++i) {
                float dgate[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float pd = fmaf(zh[i][k], post_w[i][k], post_b[i][k]) * dy[i][k];
                    dgate[k] = pd * scale[i][k];
                    if (col(i) + k >= a.width) dgate[k] = 0.f;
                    const float bar = dy[i][k] * gate[i][k] * scale[i][k];
                    if (there) {
                        sum[S_SCALE][i][k] = fmaf(pd * a.factor, gate[i][k], sum[S_SCALE][i][k]);
                        sum[S_GATE][i][k] += dgate[k];
                        sum[S_POST_W][i][k] = fmaf(bar, zh[i][k], sum[S_POST_W][i][k]);
                        sum[S_POST_B][i][k] += bar;
                    }
                    gate_sum += dgate[k];
                    dy[i][k] = a.post ? bar * post_w[i][k] : bar;
                }
                if (b.dgate && a.gate_kind == MLIP_RESIDUAL_GATE_FULL && there) store8<E>(dgate, b.dgate, row * b.dgate_rs, col(i), a.width);
            }
            if (a.gate_kind == MLIP_RESIDUAL_GATE_ROW && b.dgate) {
                row_sum<S>(gate_sum, none, red, turn);
                if (there && lane == 0) static_cast<E *>(b.dgate)[row * b.dgate_rs] = to_elem<E>(gate_sum);
            }
            if (a.post) normalise_back<S>(dy, zh, rz, a, c0, inv, red, turn);
            if (b.dz && there)
#pragma unroll
                for (int i = 0; i < S::N; ++i) store8<E>(dy[i], b.dz, row * b.dz_rs, col(i), a.width);
        }
    }
    if constexpr (BACK) {
#pragma unroll
        for (int s = 0; s < kSums; ++s) {
            if (!b.sum[s]) continue;
            const bool f32 = b.part || (a.params_f32 && s != S_GATE);
            void *to = b.part ? static_cast<void *>(b.part + ((int64_t)blockIdx.x * kSums + s) * a.width) : b.sum[s];
            if constexpr (S::kRows == 1) {
#pragma unroll
                for (int i = 0; i < S::N; ++i) {
                    if (f32) store8<float>(sum[s][i], to, 0, col(i), a.width);
                    else store8<E>(sum[s][i], to, 0, col(i), a.width);
                }
            } else {
                constexpr int in_wave = S::G < 64 ? S::G : 64, step = S::G > 64 ? S::G / 64 : 1;
#pragma unroll
                for (int i = 0; i < S::N; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        float v = sum[s][i][k];
#pragma unroll
                        for (int d = in_wave; d < 64; d <<= 1) v += __shfl_xor(v, d);
                        if ((int)(threadIdx.x & 63) < in_wave) sums[threadIdx.x >> 6][col(i) + k] = v;
                    }
                __syncthreads();
                for (int c = threadIdx.x; c < a.width; c += S::kBlock) {
                    float v = 0.f;
                    for (int w = S::G > 64 ? c / 8 % S::G / 64 : 0; w < S::kWaves; w += step) v += sums[w][c];
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

template <class Fn> void with_shape(int64_t width, Fn &&f)
{
    if (width <= 8) f(Shape<1, 1>{});
    else if (width <= 16) f(Shape<2, 1>{});
    else if (width <= 32) f(Shape<4, 1>{});
    else if (width <= 64) f(Shape<8, 1>{});
    else if (width <= 128) f(Shape<16, 1>{});
    else if (width <= 256) f(Shape<32, 1>{});
    else if (width <= 512) f(Shape<64, 1>{});
    else if (width <= 1024) f(Shape<128, 1>{});
    else if (width <= 2048) f(Shape<256, 1>{});
    else if (width <= 4096) f(Shape<256, 2>{});
    else f(Shape<512, 2>{});
}

// Blocks of the gradient: a block's sums take as much as a few dozen rows
int64_t back_blocks(int64_t n, int64_t width)
{
    int64_t blocks = 0;
    with_shape(width, [&](auto s) {
        using S = decltype(s);
        const int64_t rounds = (n + S::kRows - 1) / S::kRows;
        const int64_t most = 1024;
        blocks = (rounds + 3) / 4;
        if (blocks > most) blocks = most;
    });
    return blocks < 1 ? 1 : blocks;
}

template <bool BACK> int run(const ResidualArgs &a, const Back &b0, int64_t blocks)
{
    Args d{{a.x, a.x_rs, a.x_cs}, {a.z, a.z_rs, a.z_cs}, {a.gate, a.gate_rs, a.gate_cs}, a.scale, a.post_w, a.post_b, a.pre_w, a.pre_b, a.y, a.norm, a.y_rs, a.norm_rs, a.n,
           (int32_t)a.width, a.gate_kind, a.param_dtype == MLIP_DTYPE_F32, a.kind == MLIP_NORM_LAYER, a.post, a.pre, a.eps, a.factor};
    with_elem(a.dtype, [&](auto e) {
        using E = decltype(e);
        with_shape(a.width, [&](auto s) {
            using S = decltype(s);
            k_residual<E, S, BACK><<<(unsigned)blocks, S::kBlock, 0, a.stream>>>(d, b0);
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
    with_shape(a.width, [&](auto s) { blocks = (a.n + decltype(s)::kRows - 1) / decltype(s)::kRows; });
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
    return run<true>(a, b, blocks);
}

}  // namespace mlip
