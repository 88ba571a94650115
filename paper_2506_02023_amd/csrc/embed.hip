// Per-species parameter tables: row lookup with scaling, and its gradient.
#include "elem.h"

namespace mlip {

// out[i][f] = scale * table[id_i][f], a thread per element.
template <class T, class O, class Id>
__global__ __launch_bounds__(256) void k_embed(const T *table, int64_t n_rows, int64_t width, int64_t rs, int64_t cs, const Id *ids,
                                               int64_t n, float scale, O *out, int64_t os)
{
    const int64_t total = n * width, step = (int64_t)gridDim.x * 256;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += step) {
        const int64_t i = e / width, f = e - i * width, id = ids[i];
        float v = 0.f;
        if (id >= n_rows) v = __builtin_nanf("");
        else if (id >= 0) v = scale * (float)table[id * rs + f * cs];
        out[i * os + f] = to_elem<O>(v);
    }
}

int embed_impl(const EmbedArgs &a)
{
    if (a.n == 0) return MLIP_OK;
    const int64_t blocks = (a.n * a.width + 255) / 256;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536));
    with_elem(a.in_dtype, [&](auto t) {
        with_elem(a.out_dtype, [&](auto o) {
            with_ids(a.id_bits, [&](auto id) {
                using T = decltype(t);
                using O = decltype(o);
                using Id = decltype(id);
                k_embed<T, O, Id><<<grid, 256, 0, a.stream>>>(static_cast<const T *>(a.in), a.n_rows, a.width, a.rs, a.cs,
                                                              static_cast<const Id *>(a.ids), a.n, a.scale,
                                                              static_cast<O *>(a.out), a.os);
            });
        });
    });
    MLIP_HIP(hipGetLastError());
    return MLIP_OK;
}

// out[r][f] = scale * sum over id_i == r of grad[i][f]: a wavefront for 64 columns of one row, which goes over all ids and adds
// up the rows it finds, in their order.
template <class T, class Id>
__global__ __launch_bounds__(64) void k_embed_grad(const T *grad, int64_t rs, int64_t cs, const Id *ids, int64_t n, int64_t width,
                                                   float scale, int accumulate, void *out, int out_dtype, int64_t os)
{
    const int lane = threadIdx.x;
    const int64_t r = blockIdx.x;
    for (int64_t f0 = 0; f0 < width; f0 += 64) {
        const int64_t f = f0 + lane;
        double sum = 0.0;
        for (int64_t i0 = 0; i0 < n; i0 += 64) {
            const bool mine = i0 + lane < n && (int64_t)ids[i0 + lane] == r;
            for (uint64_t left = __ballot(mine); left; left &= left - 1) {
                const int64_t i = i0 + __ffsll((unsigned long long)left) - 1;
                if (f < width) sum += (double)(float)grad[i * rs + f * cs];
            }
        }
        if (f >= width) continue;
        sum *= (double)scale;
        const int64_t at = r * os + f;
        if (out_dtype == MLIP_DTYPE_F32) {
            float *o = static_cast<float *>(out) + at;
            *o = (float)(accumulate ? sum + (double)*o : sum);
        } else if (out_dtype == MLIP_DTYPE_BF16) {
            __bf16 *o = static_cast<__bf16 *>(out) + at;
            *o = (__bf16)(float)(accumulate ? sum + (double)(float)*o : sum);
        } else {
            _Float16 *o = static_cast<_Float16 *>(out) + at;
            *o = (_Float16)(float)(accumulate ? sum + (double)(float)*o : sum);
        }
    }
}

size_t embed_grad_workspace(int64_t, int64_t, int64_t) { return 0; }

int embed_grad_impl(const EmbedArgs &a)
{
    with_elem(a.in_dtype, [&](auto t) {
        with_ids(a.id_bits, [&](auto id) {
            using T = decltype(t);
            using Id = decltype(id);
            k_embed_grad<T, Id><<<dim3((unsigned)a.n_rows), 64, 0, a.stream>>>(static_cast<const T *>(a.in), a.rs, a.cs,
                                                                               static_cast<const Id *>(a.ids), a.n, a.width, a.scale,
                                                                               a.accumulate, a.out, a.out_dtype, a.os);
        });
    });
    MLIP_HIP(hipGetLastError());
    return MLIP_OK;
}

}  // namespace mlip
