// Global norm of a list of tensors, and clipping by it.
#include <type_traits>

#include "elem.h"

namespace mlip {

// Tensors of one launch, by value in its arguments (4 KB at most): a list of any length takes no upload and can be captured.
constexpr int kListMax = 128, kBlocksMax = 1024, kTile = 4096;   // tensors of a launch, blocks of a launch, elements of a tile
struct TensorChunk {
    const void *src[kListMax];
    void *dst[kListMax];
    int64_t n[kListMax];
    int32_t first[kListMax + 1];   // first tile of every tensor, tiles of all
    uint8_t dtype[kListMax];
    int32_t count;
};

struct NormOut { float norm, coef; };

__device__ inline double block_sum(double v, double *red)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (unsigned w = 0; w < blockDim.x / 64; ++w) v += red[w];
    __syncthreads();
    return v;
}

// f(T *src, T *dst, elements) for every tile of the block
template <class Fn> __device__ inline void for_tiles(const TensorChunk &c, Fn &&f)
{
    const int tiles = c.first[c.count];
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        int t = 0;
        while (c.first[t + 1] <= tile) ++t;
        const int64_t at = (int64_t)(tile - c.first[t]) * kTile;
        const int len = (int)(c.n[t] - at < kTile ? c.n[t] - at : kTile);
        if (c.dtype[t] == MLIP_DTYPE_F32) f(static_cast<const float *>(c.src[t]) + at, static_cast<float *>(c.dst[t]) + at, len);
        else if (c.dtype[t] == MLIP_DTYPE_BF16) f(static_cast<const __bf16 *>(c.src[t]) + at, static_cast<__bf16 *>(c.dst[t]) + at, len);
        else f(static_cast<const _Float16 *>(c.src[t]) + at, static_cast<_Float16 *>(c.dst[t]) + at, len);
    }
}

__global__ __launch_bounds__(256) void k_square_sums(TensorChunk c, double *part)
{
    __shared__ double red[4];
    double sum = 0.0;
    for_tiles(c, [&](const auto *src, auto *, int len) {
        for (int k = threadIdx.x; k < len; k += 256) {
            const double x = (double)(float)src[k];
            sum += x * x;
        }
    });
    sum = block_sum(sum, red);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void k_norm_join(const double *part, int count, float max_norm, float *norm, float *coef)
{
    __shared__ double red[4];
    double sum = 0.0;
    for (int k = threadIdx.x; k < count; k += 256) sum += part[k];
    sum = block_sum(sum, red);
    if (threadIdx.x) return;
    const double n = sqrt(sum);
    *norm = (float)n;
    *coef = (n > (double)max_norm && n < (double)__builtin_inff()) ? (float)((double)max_norm / n) : 1.f;
}

__global__ __launch_bounds__(256) void k_clip(TensorChunk c, const float *coef)
{
    const float s = *coef;
    for_tiles(c, [&](const auto *src, auto *dst, int len) {
        if (s == 1.f && src == dst) return;
        for (int k = threadIdx.x; k < len; k += 256) dst[k] = to_elem<std::remove_reference_t<decltype(*dst)>>((float)src[k] * s);
    });
}

size_t grad_workspace(int32_t count) { return 256 + (size_t)(count / kListMax + 1) * kBlocksMax * sizeof(double); }

// the next tensors of the list as a launch takes them, from tensor `at` on; tensors without elements are left out
static int fill(TensorChunk &c, const mlip_tensor_t *list, int32_t count, int32_t at)
{
    c.count = 0;
    int64_t tiles = 0;
    for (; at < count && c.count < kListMax; ++at) {
        const int64_t more = (list[at].n + kTile - 1) / kTile;
        if (!more) continue;
        if (tiles + more > 0x7fffff00) break;
        c.src[c.count] = list[at].src;
        c.dst[c.count] = list[at].dst;
        c.n[c.count] = list[at].n;
        c.dtype[c.count] = (uint8_t)list[at].dtype;
        c.first[c.count++] = (int32_t)tiles;
        tiles += more;
    }
    c.first[c.count] = (int32_t)tiles;
    return at;
}

static unsigned blocks_of(const TensorChunk &c) { return (unsigned)(c.first[c.count] < kBlocksMax ? c.first[c.count] : kBlocksMax); }

int grad_norm_impl(const mlip_tensor_t *list, int32_t count, bool clip, float max_norm, float *norm, void *workspace, hipStream_t stream)
{
    TensorChunk c;
    float *coef = static_cast<float *>(workspace);
    double *part = reinterpret_cast<double *>(static_cast<char *>(workspace) + 256);
    int parts = 0;
    for (int32_t at = 0; at < count;) {
        at = fill(c, list, count, at);
        if (!c.count) continue;
        k_square_sums<<<blocks_of(c), 256, 0, stream>>>(c, part + parts);
        parts += (int)blocks_of(c);
    }
    k_norm_join<<<1, 256, 0, stream>>>(part, parts, max_norm, norm, coef);
    for (int32_t at = 0; clip && at < count;) {
        at = fill(c, list, count, at);
        if (c.count) k_clip<<<blocks_of(c), 256, 0, stream>>>(c, coef);
    }
    MLIP_HIP(hipGetLastError());
    return MLIP_OK;
}

}  // namespace mlip
