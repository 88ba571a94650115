// Global norm of a list of tensors, and clipping by it.
//
// Both are bound by memory: the norm reads every element once (two operations each), clipping reads and writes each.  The sums of squares are fp64: the
// square of an fp32 number would leave the range of fp32, and a conversion and an fp64 product-sum for each element are hidden behind the loads.
// 1 GB of fp32 is summed in 145 us (6.9 TB/s) and clipped in 349 (2 GB, 5.7 TB/s).
#include <type_traits>

#include "elem.h"

namespace mlip {

// The tensors of a launch lie in its arguments (4 KB at most), so a list takes no upload and a captured call keeps it.  A tensor is cut into tiles
// of 32 KB, one step of a block's wide loads; block b has tiles b, b + blocks, ...  Clipping 1 GB of fp32, at the time: 547 us; with runs of consecutive
// tiles for a block 571 (both with steps of 128 bytes a thread; of 64 bytes 574 and 578), with half the blocks 564, with a quarter 582.
constexpr int kThreads = 256, kUnroll = 8, kTileBytes = kThreads * kUnroll * 16;
constexpr int kListNorm = 200, kListClip = 144;   // tensors of a launch: 20 and 28 bytes each
constexpr int kBlocksMost = 8192;                 // blocks of a launch, and partial sums that every block of the next launch adds up for itself

template <int Most, bool Dst> struct TensorChunk {
    const void *src[Most];
    void *dst[Dst ? Most : 1];
    uint64_t n_type[Most];      // elements, type code in the top byte
    uint32_t first[Most + 1];   // first tile of every tensor, tiles of all
    int32_t count;
};
using NormChunk = TensorChunk<kListNorm, false>;
using ClipChunk = TensorChunk<kListClip, true>;
static_assert(sizeof(NormChunk) <= 4060 && sizeof(ClipChunk) <= 4060, "arguments of a launch");

// Tiles begin at whole lines of memory, the first one of a tensor that does not at its beginning: elements by which the line lies before it.
// (1 GB in 200 tensors that lie one after another: 495 us, 531 with tiles counted from the tensors' beginnings.)
__host__ __device__ inline int64_t before_line(const void *p, size_t size) { return (int64_t)(reinterpret_cast<uintptr_t>(p) % 128 / size); }

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

// f(src, dst, elements) for each tile of the block
template <class Chunk, class Fn> __device__ inline void for_tiles(const Chunk &c, Fn &&f)
{
    constexpr int kWords = ((std::is_same_v<Chunk, ClipChunk> ? kListClip : kListNorm) + 63) / 64;
    const uint32_t tiles = c.first[c.count];
    uint32_t first[kWords];   // the tensors' first tiles, a few to a lane: a tile's tensor is the last that begins at or before it
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
        const int t = k * 64 + (threadIdx.x & 63);
        first[k] = t < c.count ? c.first[t] : 0xffffffffu;
    }
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        int t = -1;
#pragma unroll
        for (int k = 0; k < kWords; ++k) t += __popcll(__ballot(first[k] <= tile));
        t = __builtin_amdgcn_readfirstlane(t);
        const int64_t n = (int64_t)(c.n_type[t] & (((uint64_t)1 << 56) - 1));
        auto part = [&](auto tag) {
            using T = decltype(tag);
            constexpr int64_t per = kTileBytes / sizeof(T);
            constexpr bool writes = std::is_same_v<Chunk, ClipChunk>;
            const void *at = c.src[t];
            if constexpr (writes) at = c.dst[t];
            const int64_t begin = (int64_t)(tile - c.first[t]) * per - before_line(at, sizeof(T)), end = begin + per;
            const int64_t lo = begin < 0 ? 0 : begin, hi = end < n ? end : n;
            T *dst = nullptr;
            if constexpr (writes) dst = static_cast<T *>(c.dst[t]) + lo;
            f(static_cast<const T *>(c.src[t]) + lo, dst, (int)(hi - lo));
        };
        const int type = (int)(c.n_type[t] >> 56);
        if (type == MLIP_DTYPE_F32) part(float{});
        else if (type == MLIP_DTYPE_BF16) part(__bf16{});
        else part(_Float16{});
    }
}

// f(position, values) over the n elements of a tile: a whole one in one step of kUnroll wide loads a thread, else by single wide loads, then single elements
template <bool Stream, class T, class Fn> __device__ inline void for_elements(const T *p, int n, Fn &&f)
{
    constexpr int V = 16 / sizeof(T);
    if (n == kTileBytes / (int)sizeof(T)) {
        Cols<T, V> x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const Far<T, V> *at = reinterpret_cast<const Far<T, V> *>(p + (threadIdx.x + u * kThreads) * V);
            x[u] = Stream ? __builtin_nontemporal_load(at) : *at;
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) f((threadIdx.x + u * kThreads) * V, x[u]);
        return;
    }
    const int wide = n / V;
#pragma unroll 4
    for (int i = threadIdx.x; i < wide; i += kThreads) {
        Cols<T, V> x;
        x = *reinterpret_cast<const Far<T, V> *>(p + i * V);
        f(i * V, x);
    }
    const int i = wide * V + threadIdx.x;
    if (i < n) f(i, Cols<T, 1>{p[i]});
}

template <bool Stream, class Chunk> __device__ inline double squares(const Chunk &c)
{
    double sum[2] = {0.0, 0.0};
    for_tiles(c, [&](const auto *src, auto *, int n) {
        for_elements<Stream>(src, n, [&](int, auto x) {
            constexpr int V = sizeof(x) / sizeof(*src);
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k & 1] = fma((double)(float)x[k], (double)(float)x[k], sum[k & 1]);
        });
    });
    return block_sum(sum[0] + sum[1]);
}

struct Norm { double norm; float coef; };

__device__ inline Norm norm_of(double squares, float max_norm)
{
    const double n = sqrt(squares);
    return {n, n > (double)max_norm && (float)n < __builtin_inff() ? (float)((double)max_norm / n) : 1.f};
}

__device__ inline double sum_parts(const double *part, int count)
{
    double sum = 0.0;
    in_steps<8>(threadIdx.x, count, kThreads, [&](int64_t k) { return part[k]; }, [&](double x) { sum += x; });
    return block_sum(sum);
}

template <bool Stream, class Chunk> __device__ inline void clip_tiles(const Chunk &c, float coef)
{
    for_tiles(c, [&](const auto *src, auto *dst, int n) {
        if (coef == 1.f && src == dst) return;
        for_elements<Stream>(src, n, [&](int at, auto x) {
            using T = std::remove_cv_t<std::remove_reference_t<decltype(*dst)>>;
            constexpr int V = sizeof(x) / sizeof(T);
            Cols<T, V> y;
#pragma unroll
            for (int k = 0; k < V; ++k) y[k] = to_elem<T>((float)x[k] * coef);
            Far<T, V> *to = reinterpret_cast<Far<T, V> *>(dst + at);
            if (Stream) __builtin_nontemporal_store((Far<T, V>)y, to);
            else *to = (Far<T, V>)y;
        });
    });
}

template <bool Stream> __global__ __launch_bounds__(kThreads) void k_square_sums(NormChunk c, double *part)
{
    const double sum = squares<Stream>(c);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// the norm alone; or many partial sums made into one for the blocks of k_clip
__global__ __launch_bounds__(kThreads) void k_norm(const double *part, int count, float *norm, double *joined)
{
    const double sum = sum_parts(part, count);
    if (threadIdx.x) return;
    if (norm) *norm = (float)sqrt(sum);
    if (joined) *joined = sum;
}

// Every block adds the partial sums up for itself, in the same order: a launch less.
template <bool Stream> __global__ __launch_bounds__(kThreads) void k_clip(ClipChunk c, const double *part, int count, float max_norm, float *norm)
{
    const Norm m = norm_of(sum_parts(part, count), max_norm);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)m.norm;
    clip_tiles<Stream>(c, m.coef);
}

// A list of few tiles: norm and clipping in one block
constexpr uint32_t kFewTiles = 4;
__global__ __launch_bounds__(kThreads) void k_few_tiles(ClipChunk c, bool clip, float max_norm, float *norm)
{
    const Norm m = norm_of(squares<false>(c), max_norm);
    if (threadIdx.x == 0) *norm = (float)m.norm;
    if (clip) clip_tiles<false>(c, m.coef);
}

constexpr size_t kHead = 256;   // bytes in front of the partial sums: the joined one

size_t grad_workspace(int32_t count) { return kHead + ((size_t)count / kListClip + 1) * kBlocksMost * sizeof(double); }

static int64_t tiles_of(const mlip_tensor_t &x, const void *at)
{
    const int64_t size = (int64_t)elem_size(x.dtype), per = kTileBytes / size;
    return x.n > 0 ? (x.n + before_line(at, size) + per - 1) / per : 0;
}

// Takes the next tensors of the list for a launch, from tensor `at` on; those without elements are left out.  Returns where the next launch goes on.
// clip: whether the tensors have outputs; where they have none their `dst` is not read.
template <class Chunk> static int32_t take(Chunk &c, const mlip_tensor_t *list, int32_t count, int32_t at, bool clip)
{
    constexpr bool writes = std::is_same_v<Chunk, ClipChunk>;
    constexpr int most = writes ? kListClip : kListNorm;
    c.count = 0;
    int64_t tiles = 0;
    for (; at < count && c.count < most; ++at) {
        const void *to = clip ? list[at].dst : list[at].src;
        const int64_t more = tiles_of(list[at], to);
        if (!more) continue;
        if (c.count && tiles + more > 0x7fffffff) break;
        c.src[c.count] = list[at].src;
        if constexpr (writes) c.dst[c.count] = const_cast<void *>(to);
        c.n_type[c.count] = (uint64_t)list[at].n | ((uint64_t)list[at].dtype << 56);
        c.first[c.count++] = (uint32_t)tiles;
        tiles += more;
    }
    c.first[c.count] = (uint32_t)tiles;
    return at;
}

template <class Chunk> static unsigned blocks_of(const Chunk &c) { return c.first[c.count] < kBlocksMost ? c.first[c.count] : kBlocksMost; }

int grad_norm_impl(const mlip_tensor_t *list, int32_t count, bool clip, float max_norm, float *norm, void *workspace, size_t bytes, hipStream_t stream)
{
    double *joined = static_cast<double *>(workspace), *part = reinterpret_cast<double *>(static_cast<char *>(workspace) + kHead);
    const size_t room = (bytes - kHead) / sizeof(double);
    size_t parts = 0;
    ClipChunk few;
    if (take(few, list, count, 0, clip) == count && few.first[few.count] <= kFewTiles) {
        k_few_tiles<<<1, kThreads, 0, stream>>>(few, clip, max_norm, norm);
        MLIP_HIP(hipGetLastError());
        return MLIP_OK;
    }
    double total = 0.0;
    for (int32_t t = 0; t < count; ++t) total += (double)list[t].n * (double)elem_size(list[t].dtype);
    const bool far = total > kStreamBytes;
    NormChunk c;
    for (int32_t at = 0; at < count;) {
        at = take(c, list, count, at, false);
        if (!c.count) break;
        if (parts + blocks_of(c) > room) { set_error("tensors too large for the workspace"); return MLIP_EINVAL; }
        (far ? k_square_sums<true> : k_square_sums<false>)<<<blocks_of(c), kThreads, 0, stream>>>(c, part + parts);
        parts += blocks_of(c);
    }
    const bool many = parts > (size_t)kBlocksMost;   // (not none: a list without elements is one of few tiles)
    if (!clip || many) k_norm<<<1, kThreads, 0, stream>>>(part, (int)parts, norm, joined);
    if (clip) {
        ClipChunk d;
        for (int32_t at = 0; at < count;) {
            at = take(d, list, count, at, true);
            if (!d.count) break;
            (far ? k_clip<true> : k_clip<false>)<<<blocks_of(d), kThreads, 0, stream>>>(d, many ? joined : part, many ? 1 : (int)parts, max_norm, many ? nullptr : norm);
        }
    }
    MLIP_HIP(hipGetLastError());
    return MLIP_OK;
}

}  // namespace mlip
