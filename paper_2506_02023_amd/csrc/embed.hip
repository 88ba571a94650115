// Per-species parameter tables: row lookup with scaling, and its gradient.
#include <type_traits>

#include "elem.h"

namespace mlip {

// x / d for 0 <= x < 2^31 as a product and a shift: m = floor(2^(31 + l) / d) + 1 with 2^l >= d errs by less than 2^-31 / d relative
struct Div31 {
    uint32_t m;
    int shift;
    explicit Div31(uint32_t d)
    {
        int l = 0;
        while (((uint64_t)1 << l) < d) ++l;
        m = (uint32_t)(((uint64_t)1 << (31 + l)) / d + 1);
        shift = 31 + l;
    }
    __device__ uint32_t operator()(uint32_t x) const { return (uint32_t)(((uint64_t)x * m) >> shift); }
};

// A row is worked on in lots of V columns, one wide access each at whatever alignment (rows of odd widths begin anywhere).  The last lot of a row ends
// with the row: it begins up to V - 1 columns inside the one before it, and computes those columns too.  V = 1 where the
// columns of the input do not lie one after another or where there are fewer than a wide access has.
template <int V> struct Lot {
    int64_t f;   // first column
    int skip;    // columns that the lot before has
    __device__ Lot(int64_t number, int64_t width)
    {
        const int64_t want = number * V, most = width - V;
        f = want < most ? want : most;
        skip = (int)(want - f);
    }
    // the lots of a row in memory that begin at multiples of V elements there, but for the row's first and last
    template <class O> __device__ Lot(int64_t number, int64_t width, const O *row)
    {
        const int64_t want = number * V - (int64_t)(reinterpret_cast<uintptr_t>(row) / sizeof(O) % V), most = width - V;
        f = want < 0 ? 0 : want < most ? want : most;
        skip = 0;
    }
};
inline int64_t lots_of(int64_t width, int V) { return (width + V - 1) / V; }

// Stream: past the caches, for what is read once and is larger than they are
template <int V, bool Stream = false, class T> __device__ inline void load_cols(float (&v)[V], const T *p)
{
    const Far<T, V> *at = reinterpret_cast<const Far<T, V> *>(p);
    const Cols<T, V> x = Stream ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = (float)x[k];
}

template <class T, int V> __device__ inline Cols<T, V> to_cols(const float (&v)[V])
{
    Cols<T, V> x;
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] = to_elem<T>(v[k]);
    return x;
}

// Stores a whole lot: where lots overlap, both write the same bits.
template <int V, class T> __device__ inline void store_cols(T *p, const float (&v)[V])
{
    *reinterpret_cast<Far<T, V> *>(p) = to_cols<T>(v);
}

// The same past the caches, for what is larger than they are.
template <int V, class T> __device__ inline void stream_cols(T *p, const float (&v)[V])
{
    __builtin_nontemporal_store((Far<T, V>)to_cols<T>(v), reinterpret_cast<Far<T, V> *>(p));
}

// ---- lookup: out[i][f] = scale * table[id_i][f].  A thread has a lot of columns of a row, and kEmbedUnroll of them at a time, a grid's size
// apart.  Writing bounds it: a million rows of 64 fp32 take 43 us, 6.0 TB/s.  Results that the caches do not hold are stored past them if their rows begin at
// whole lots (a million rows of 64: 43.6 us a call, 45.4 through the caches); stored so, lots that share a line of memory cost more than they save, and the lots are
// shifted to where memory has whole ones (1,546,331 fp32 rows of 59: 80 us shifted, 82 from the row's beginning on, 90 so and past the caches).

enum { kPlain, kStreamed, kShifted };
constexpr int kEmbedUnroll = 4;

template <class T, class O, class Id, int V, int Way>
__global__ __launch_bounds__(256) void k_embed(const T *table, int64_t n_rows, int64_t width, int64_t rs, int64_t cs, const Id *ids,
                                               uint32_t items, uint32_t per_row, Div31 div, float scale, O *out, int64_t os)
{
    constexpr int U = kEmbedUnroll;
    const uint32_t step = gridDim.x * 256;
    for (uint32_t e0 = blockIdx.x * 256 + threadIdx.x; e0 < items; e0 += step * U) {
        O *to[U];
        int64_t id[U];
        float v[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t e = e0 + u * step < items ? e0 + u * step : e0;   // past the end: the first once more, not stored
            const uint32_t row = div(e);
            id[u] = ids[row];
            to[u] = out + row * os;
            const int64_t f = Way == kShifted ? Lot<V>(e - row * per_row, width, to[u]).f : Lot<V>(e - row * per_row, width).f;
            to[u] += f;
            load_cols<V>(v[u], table + (id[u] >= 0 && id[u] < n_rows ? id[u] : 0) * rs + (V == 1 ? f * cs : f));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u > 0 && e0 + u * step >= items) break;
#pragma unroll
            for (int k = 0; k < V; ++k) v[u][k] = id[u] < 0 ? 0.f : id[u] < n_rows ? v[u][k] * scale : __builtin_nanf("");
            if (Way == kStreamed) stream_cols<V>(to[u], v[u]);
            else store_cols<V>(to[u], v[u]);
        }
    }
}

int embed_impl(const EmbedArgs &a)
{
    if (a.n == 0) return MLIP_OK;
    with_elem(a.in_dtype, [&](auto t) {
        with_elem(a.out_dtype, [&](auto o) {
            with_ids(a.id_bits, [&](auto id) {
                using T = decltype(t);
                using O = decltype(o);
                using Id = decltype(id);
                constexpr int V = sizeof(T) == 2 || sizeof(O) == 2 ? 8 : 4;   // 16 bytes of the smaller type
                const bool wide = (a.cs == 1 || a.width == 1) && a.width >= V;
                const bool large = (double)a.n * (double)a.width * sizeof(O) > kStreamBytes;
                const bool even = reinterpret_cast<uintptr_t>(a.out) % (V * sizeof(O)) == 0 && a.os % V == 0;
                const int64_t per_row = !wide ? a.width : lots_of(large && !even ? a.width + V - 1 : a.width, V);
                const int64_t most = ((int64_t)1 << 30) / per_row;   // rows of a launch: items are numbered in 31 bits
                const Div31 div((uint32_t)per_row);
                for (int64_t i0 = 0; i0 < a.n; i0 += most) {
                    const int64_t rows = a.n - i0 < most ? a.n - i0 : most, items = rows * per_row;
                    const int64_t blocks = (items + 256 * kEmbedUnroll - 1) / (256 * kEmbedUnroll);
                    auto launch = [&](auto kernel) {
                        kernel<<<(unsigned)(blocks < 16384 ? blocks : 16384), 256, 0, a.stream>>>(
                            static_cast<const T *>(a.in), a.n_rows, a.width, a.rs, a.cs, static_cast<const Id *>(a.ids) + i0, (uint32_t)items,
                            (uint32_t)per_row, div, a.scale, static_cast<O *>(a.out) + i0 * a.os, a.os);
                    };
                    if (!wide) launch(k_embed<T, O, Id, 1, kPlain>);
                    else if (!large) launch(k_embed<T, O, Id, V, kPlain>);
                    else even ? launch(k_embed<T, O, Id, V, kStreamed>) : launch(k_embed<T, O, Id, V, kShifted>);
                }
            });
        });
    });
    MLIP_HIP(hipGetLastError());
    return MLIP_OK;
}

// ---- gradient: out[r][f] = scale * sum over id_i == r of grad[i][f]

// the output matrix, whatever its type
struct GradOut {
    void *p;
    int dtype;
    int64_t os;
    float scale;
    int accumulate;
    // writes the finished sums of a lot of columns of a row
    template <int V> __device__ void put(int64_t r, int64_t f, int skip, const double (&sum)[V]) const
    {
        if (dtype == MLIP_DTYPE_F32) put_as<float>(r, f, skip, sum);
        else if (dtype == MLIP_DTYPE_BF16) put_as<__bf16>(r, f, skip, sum);
        else put_as<_Float16>(r, f, skip, sum);
    }
    template <class O, int V, class S> __device__ void put_as(int64_t r, int64_t f, int skip, const S (&sum)[V]) const
    {   // (fp32 sums: their fp32 product with the scale is what the fp64 product rounds to)
        O *o = static_cast<O *>(p) + r * os + f;
        float v[V];
        if (accumulate) {   // a column that another lot has too is that lot's to add to
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k >= skip) o[k] = to_elem<O>((float)((double)sum[k] * (double)scale + (double)(float)o[k]));
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = (float)(sum[k] * (S)scale);
            store_cols<V>(o, v);
        }
    }
};

// Few rows: every wavefront keeps a table of all rows in LDS, 64 floats to a row, one for each lane: lane l owns column l % tile of the
// wavefront's rows l / tile, l / tile + slots, ...  A lane adds its values to its own float of the row, so nothing collides and the order of
// the additions is the order of the atoms.  A block then joins the lanes that own the same column (fp64, rounded to fp32: one more fp32 addition to
// the bound) and its wavefronts' tables (the same), k_few_join the blocks.  Ids without a row go to one row more, which is not read.
// Reading the gradients bounds it: a million rows of 64 into 8 take 48 us, 5.4 TB/s, and the join 4.5; with LDS additions without return in place of
// read, add and write (220 clocks a wavefront each) 361 us against 134 at the time.  Small and narrow calls are bound by the latency of the few steps.
constexpr int kFewLds = 65536, kFewWaves = 16;
constexpr int few_unroll(bool one) { return one ? 16 : 8; }   // rows of a lane in flight, as the registers of 8 wavefronts a SIMD hold

// One: one row a step (wider than 32 columns), whose id is the same for the wavefront's lanes; Near: the lanes' elements of a step lie within 4 GB.
template <class T, class Id, bool One, bool Near, bool Stream>
__global__ __launch_bounds__(1024, 8) void k_few_rows(const T *grad, int64_t rs, int64_t cs, const Id *ids, int64_t n, int n_rows, int64_t width,
                                                      int tile, int slots, int waves, int64_t rows_per_wave, int chunks, bool grouped, int64_t block0,
                                                      float *part, GradOut out)
{
    extern __shared__ float tables[];
    // Blocks go to the eight XCDs in turn.  Grouped: the tiles of a chunk of rows are consecutive on one of them, whose L2 has the lines that the tiles
    // share (300,000 fp32 rows of 257 into 8: 66 us, 79 chunk by chunk).  Tiles of whole lines share none (100,000 rows of 512 into 64: 55 us either way).
    const int tiles = (int)((width + tile - 1) / tile);
    const uint32_t b = (uint32_t)block0 + blockIdx.x;   // (2^32 blocks have more parts than memory holds)
    const int chunk = (int)(grouped ? (b >> 3) / tiles * 8 + (b & 7) : b % chunks), tile_at = (int)(grouped ? (b >> 3) % tiles : b / chunks);
    if (chunk >= chunks) return;
    constexpr int U = few_unroll(One);
    if (One) slots = 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), size = (n_rows + 1) * 64;
    float *mine = tables + wave * size;
    for (int k = threadIdx.x; k < waves * size; k += blockDim.x) tables[k] = 0.f;
    __syncthreads();
    const int64_t f0 = (int64_t)tile_at * tile;
    const int cols = (int)(width - f0 < tile ? width - f0 : tile), slot = One ? 0 : lane / tile, col = lane - slot * tile;
    const int64_t r0 = ((int64_t)chunk * waves + wave) * rows_per_wave, r1 = n - r0 < rows_per_wave ? n : r0 + rows_per_wave;
    if (wave < waves && slot < slots && col < cols) {
        using Offset = std::conditional_t<Near, uint32_t, int64_t>;
        const Offset mine_at = (Offset)(slot * rs + col * cs);
        // a step: U rows of the lane, all loaded before the first is added; past the end the last row stands in, and goes nowhere
        auto step = [&](int64_t r, auto whole) {
            Id id[U];
            float v[U];
            const T *g = grad + r * rs + f0 * cs;
            const Id *p = ids + r;
            const int left = (int)(r1 - r);   // rows, of all slots together
            if (!decltype(whole)::value && slot >= left) return;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                int k = u * slots;
                if (!decltype(whole)::value && k + slot >= left) k = 0;
                id[u] = p[(uint32_t)(k + slot)];
                v[u] = (float)(Stream ? __builtin_nontemporal_load(g + k * rs + mine_at) : (g + k * rs)[mine_at]);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool there = decltype(whole)::value || u * slots + slot < left;
                const int at = id[u] >= 0 && id[u] < n_rows && there ? (int)id[u] : n_rows;
                mine[at * 64 + lane] += v[u];
            }
        };
        int64_t r = r0;
        for (; r + slots * U <= r1; r += slots * U) step(r, std::true_type{});
        if (r < r1) step(r, std::false_type{});
    }
    __syncthreads();
    if (!One) {   // each table's slots into its first
        for (int e = threadIdx.x; e < waves * n_rows * cols; e += blockDim.x) {
            const int row = e / cols, w = row / n_rows;
            float *at = tables + w * size + (row - w * n_rows) * 64 + (e - row * cols);
            double sum = 0.0;
#pragma unroll 8
            for (int k = 0; k < slots; ++k) sum += (double)at[k * tile];
            at[0] = (float)sum;
        }
        __syncthreads();
    }
    for (int e = threadIdx.x; e < n_rows * cols; e += blockDim.x) {
        const int r = e / cols, c = e - r * cols;
        double sum[1] = {0.0};
#pragma unroll 4
        for (int w = 0; w < waves; ++w) sum[0] += (double)tables[w * size + r * 64 + c];
        if (part) part[((int64_t)chunk * n_rows + r) * width + f0 + c] = (float)sum[0];
        else out.put<1>(r, f0 + c, 0, sum);
    }
}

// sum over the blocks of k_few_rows: a block has 16 elements, whose parts 64 groups of 16 lanes share
__global__ __launch_bounds__(1024) void k_few_join(const float *part, int parts, int64_t elements, int64_t width, int64_t block0, GradOut out)
{
    __shared__ double red[16][16];
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int64_t e = (block0 + blockIdx.x) * 16 + lane;
    double sum[1] = {0.0};
    if (e < elements) {
        in_steps<8>(group, parts, 64, [&](int64_t p) { return part[p * elements + e]; }, [&](float x) { sum[0] += (double)x; });
    }
    sum[0] += __shfl_xor(sum[0], 16);
    sum[0] += __shfl_xor(sum[0], 32);
    if ((group & 3) == 0) red[group >> 2][lane] = sum[0];
    __syncthreads();
    if (group || e >= elements) return;
#pragma unroll
    for (int g = 1; g < 16; ++g) sum[0] += red[g][lane];
    out.put<1>(e / width, e % width, 0, sum);
}

struct FewPlan {
    int tiles, tile, slots, waves, threads, blocks;   // waves: wavefronts with a table; all threads clear and join the tables
    int64_t rows_per_wave;
    FewPlan(int64_t n, int64_t n_rows, int64_t width)
    {
        tiles = (int)((width + 63) / 64);
        tile = (int)((width + tiles - 1) / tiles);
        slots = 64 / tile;
        waves = (int)(kFewLds / ((n_rows + 1) * 256));
        waves = waves < 1 ? 1 : waves > kFewWaves ? kFewWaves : waves;
        threads = 64 * (waves < 8 ? 8 : waves);
        // wavefronts: as many as have a step of rows in flight, at most the blocks that are resident together (two a compute unit where several rows lie
        // in one load and more blocks only are more to join: a million rows of 2 into 89 15 us, 18; of 64 into 89 81, 68), but no more than
        // MLIP_EMBED_GRAD_RUN rows a lane; where one block does with four steps, one block (and no second launch to join)
        const int64_t step = (int64_t)slots * few_unroll(slots == 1);
        const int lds = waves * (int)(n_rows + 1) * 256, fit = 163840 / lds < 2048 / threads ? 163840 / lds : 2048 / threads;
        const int resident = 256 * (slots > 1 && fit > 2 ? 2 : fit);
        const int64_t most = tiles * 8 <= resident ? resident / tiles / 8 * 8 : tiles <= resident ? resident / tiles : 1;   // (as many for each XCD)
        int64_t b = (n + step * waves - 1) / (step * waves);
        b = b <= 4 ? 1 : b > most ? most : b;
        int64_t r = ((n + b * waves - 1) / (b * waves) + step - 1) / step * step;
        const int64_t run = MLIP_EMBED_GRAD_RUN - 16;   // (room for the two roundings to fp32 on the way to the blocks' join)
        if (r > slots * run) r = slots * run;
        rows_per_wave = r > 0 ? r : step;
        b = (n + rows_per_wave * waves - 1) / (rows_per_wave * waves);
        blocks = (int)(b < 1 ? 1 : b);
    }
};

// Which way a table takes.  The tables' LDS leaves the fewer wavefronts to load the more rows there are, so rows that fill a wavefront (33 columns and more) pass
// to the sort at 80; of narrow ones several lie in one wavefront's load, and the sort's cost by atom is paid back later; where there is little to load the sort's
// launches count for more.  Measured, us a call by LDS tables and by sorting: a million rows of 64 into 64 58 and 76, into 119 83 and 74; 20,000
// rows of 64 into 64 15 and 19, into 89 23 and 18; 100,000 of 512 into 64 53 and 57, into 89 64 and 56; 300,000 rows of 16 into 119 21 and 28, into 200
// 27.5 and 28.5, into 255 31 and 28.5; a million rows of 2 into 255 20 and 48; 4000 rows of 64 into 119 14 and 19, into 160 19 and 18.  Between 4096 and some
// 100,000 atoms sorting is the better way for 89 rows of 64, beyond it the LDS tables would be (100,000: 23.6 and 24.4; a million: 67 and 75): the rule has no such
// second limit.
static bool takes_few(int64_t n, int64_t n_rows, int64_t width)
{
    const int64_t slots = width < 64 ? 64 / width : 1, most = 32 + 48 * slots + (n <= 4096 ? 64 : 0);
    return n_rows <= (most < kFewLds / 256 - 1 ? most : kFewLds / 256 - 1);
}

// Many rows: the ids are sorted (stable, by digits of at most 8 bits, places of the atoms along with them), so that every row's atoms lie one
// after another in their order; spans of the sorted list are summed, whatever rows they hold, and a row that spans share is joined.  An item is 8 bytes, so
// the sort's kernels are bound by latency (4 and 6 to 9 us a pass at 131,072 to 300,000 items), the sums by memory: 131,072 bf16 rows of 1024 into
// 50,021 are read in 83 us along with the writing of the rows that lie in one span, 4.5 TB/s (without those writes 5.0), the rest written in 24.
constexpr int kSortThreads = 1024, kSortTile = 2048, kSortBlocks = 256, kRadix = 256;

struct Pair { uint32_t key, at; };

struct SortPlan {
    int passes, bits, blocks;
    int64_t range;   // items of a block, a multiple of kSortTile
    SortPlan(int64_t n, int64_t n_rows)
    {
        int total = 0;
        while (((int64_t)1 << total) <= n_rows) ++total;   // keys 0 .. n_rows
        passes = (total + 7) / 8;
        bits = (total + passes - 1) / passes;
        const int64_t per = (n + kSortBlocks - 1) / kSortBlocks;
        range = (per + kSortTile - 1) / kSortTile * kSortTile;
        if (range < kSortTile) range = kSortTile;
        blocks = (int)((n + range - 1) / range);
    }
};

template <class Id> __device__ inline Pair item_of(const Id *ids, int64_t i, int64_t n_rows)
{
    const int64_t id = ids[i];
    return {id >= 0 && id < n_rows ? (uint32_t)id : (uint32_t)n_rows, (uint32_t)i};
}
__device__ inline Pair item_of(const Pair *list, int64_t i, int64_t) { return list[i]; }

// how often each digit comes up in a block's range; on the first pass also clears the ends of the rows' spans
template <class In>
__global__ __launch_bounds__(kSortThreads) void k_digit_counts(const In *in, int64_t n, int64_t n_rows, int64_t range, int shift, int bits,
                                                               uint32_t *counts, uint32_t *row_end)
{
    __shared__ uint32_t count[kRadix];
    const uint32_t mask = (1u << bits) - 1;
    if (threadIdx.x < kRadix) count[threadIdx.x] = 0;
    if (row_end)
        for (int64_t r = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; r < n_rows; r += (int64_t)gridDim.x * kSortThreads) row_end[r] = 0;
    __syncthreads();
    const int64_t end = n - range * blockIdx.x < range ? n : range * (blockIdx.x + 1);
    for (int64_t i = range * blockIdx.x + threadIdx.x; i < end; i += kSortThreads)
        atomicAdd(&count[(item_of(in, i, n_rows).key >> shift) & mask], 1u);
    __syncthreads();
    if (threadIdx.x < kRadix) counts[(int64_t)blockIdx.x * kRadix + threadIdx.x] = count[threadIdx.x];
}

constexpr int kSortWaves = kSortThreads / 64, kSortRounds = kSortTile / kSortThreads;

// place of a thread's j-th item in a tile: a wavefront has consecutive items, 64 in a round
__device__ inline int tile_place(int j) { return (threadIdx.x >> 6) * (64 * kSortRounds) + j * 64 + (threadIdx.x & 63); }

// Ranks of a tile's `there` items among those of the same digit and wavefront; before[w][d] is left with the number of wavefront w's items of digit d.
__device__ inline void tile_ranks(const Pair (&item)[kSortRounds], int there, int shift, int bits, uint32_t (&before)[kSortWaves][kRadix],
                                  uint32_t (&rank)[kSortRounds])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();
    for (int k = threadIdx.x; k < kSortWaves * kRadix; k += kSortThreads) (&before[0][0])[k] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j) {
        const uint32_t d = (item[j].key >> shift) & ((1u << bits) - 1);
        const bool mine = tile_place(j) < there;
        uint64_t same = __ballot(mine);
#pragma unroll
        for (int b = 0; b < 8; ++b) {   // bits that a shorter digit lacks are zero in all
            const uint64_t set = __ballot((d >> b) & 1);
            same &= (d >> b) & 1 ? set : ~set;
        }
        const uint32_t lower = (uint32_t)__popcll(same & (((uint64_t)1 << lane) - 1));
        rank[j] = before[wave][d] + lower;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // all lanes have read before the first of each digit writes
        if (mine && lower == 0) before[wave][d] = rank[j] + (uint32_t)__popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
}

// sum over the digits below thread t's digit t (t < kRadix; all threads call)
__device__ inline uint32_t digits_below(uint32_t own, uint32_t (&sums)[kRadix / 64])
{
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    uint32_t scan = own;
    if (t < kRadix) {
        for (int k = 1; k < 64; k <<= 1) {
            const uint32_t up = __shfl_up(scan, k);
            if (lane >= k) scan += up;
        }
        if (lane == 63) sums[wave] = scan;
    }
    __syncthreads();
    if (t < kRadix)
        for (int w = 0; w < wave; ++w) scan += sums[w];
    return scan - own;
}

// one pass of the sort: a block takes its range tile by tile
template <class In>
__global__ __launch_bounds__(kSortThreads) void k_digit_scatter(const In *in, int64_t n, int64_t n_rows, int64_t range, int shift, int bits,
                                                                const uint32_t *counts, Pair *sorted)
{
    __shared__ uint32_t before[kSortWaves][kRadix];
    __shared__ uint32_t base[kRadix];             // where the digit's next item of this block goes
    __shared__ uint32_t sums[kRadix / 64];
    const int t = threadIdx.x, wave = t >> 6;
    const uint32_t mask = (1u << bits) - 1;
    const int64_t end = n - range * blockIdx.x < range ? n : range * (blockIdx.x + 1);
    Pair item[kSortRounds];   // of the tile under way; the first one's are on their way while the counts are added up
    auto load = [&](int64_t i0) {
#pragma unroll
        for (int j = 0; j < kSortRounds; ++j) {
            const int64_t i = i0 + tile_place(j);
            item[j] = item_of(in, i < end ? i : end - 1, n_rows);
        }
    };
    load(range * blockIdx.x);
    {   // base: items of lower digits anywhere, and of this digit in the blocks before
        constexpr int kShares = kSortThreads / kRadix;
        const int d = t & (kRadix - 1), share = t / kRadix;
        uint32_t all = 0, earlier = 0;
#pragma unroll 16
        for (int b = share; b < (int)gridDim.x; b += kShares) {
            const uint32_t c = counts[(int64_t)b * kRadix + d];
            all += c;
            earlier += b < (int)blockIdx.x ? c : 0;
        }
        before[share][d] = all;
        before[share + kShares][d] = earlier;
        __syncthreads();
        all = earlier = 0;
        if (t < kRadix) {
            for (int k = 0; k < kShares; ++k) {
                all += before[k][t];
                earlier += before[k + kShares][t];
            }
        }
        const uint32_t below = digits_below(all, sums);
        if (t < kRadix) base[t] = below + earlier;
    }
    for (int64_t i0 = range * blockIdx.x; i0 < end; i0 += kSortTile) {
        if (i0 > range * blockIdx.x) load(i0);
        const int there = end - i0 < kSortTile ? (int)(end - i0) : kSortTile;
        uint32_t rank[kSortRounds];
        tile_ranks(item, there, shift, bits, before, rank);
        if (t < kRadix) {
            uint32_t at = base[t];
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = before[w][t];
                before[w][t] = at;
                at += c;
            }
            base[t] = at;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kSortRounds; ++j)
            if (tile_place(j) < there) sorted[before[wave][(item[j].key >> shift) & mask] + rank[j]] = item[j];
    }
}

// All passes over a list of one tile, in the first block's LDS; the others clear the ends of the rows' spans.
template <class Id>
__global__ __launch_bounds__(kSortThreads) void k_sort_tile(const Id *ids, int n, int64_t n_rows, int passes, int bits, Pair *sorted, uint32_t *row_end)
{
    __shared__ uint32_t before[kSortWaves][kRadix];
    __shared__ uint32_t sums[kRadix / 64];
    __shared__ Pair list[kSortTile];
    const int t = threadIdx.x, wave = t >> 6;
    if (blockIdx.x > 0) {
        for (int64_t r = (int64_t)(blockIdx.x - 1) * kSortThreads + t; r < n_rows; r += (int64_t)(gridDim.x - 1) * kSortThreads) row_end[r] = 0;
        return;
    }
    Pair item[kSortRounds];
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j) item[j] = item_of(ids, tile_place(j) < n ? tile_place(j) : n - 1, n_rows);
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * bits;
        uint32_t rank[kSortRounds], all = 0;
        tile_ranks(item, n, shift, bits, before, rank);
        if (t < kRadix)
            for (int w = 0; w < kSortWaves; ++w) all += before[w][t];
        uint32_t at = digits_below(all, sums);
        if (t < kRadix) {
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = before[w][t];
                before[w][t] = at;
                at += c;
            }
        }
        __syncthreads();
        Pair *to = pass + 1 < passes ? list : sorted;
#pragma unroll
        for (int j = 0; j < kSortRounds; ++j)
            if (tile_place(j) < n) to[before[wave][(item[j].key >> shift) & ((1u << bits) - 1)] + rank[j]] = item[j];
        if (pass + 1 == passes) break;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kSortRounds; ++j) item[j] = list[tile_place(j) < n ? tile_place(j) : 0];
    }
}

// Sums over spans of `span` items of the sorted list, a group of `lanes` lanes (V columns each) to a span; Wave: a whole wavefront, whose items are then
// scalars to it, which leaves the vector unit the additions alone.  A row that lies within the span is
// written; what a span holds of a row that began before it goes to edge[span][0], of one that goes on behind it to edge[span][1].
template <class T, class O, int V, bool Stream, bool Wave>
__global__ __launch_bounds__(256) void k_span_sums(const Pair *sorted, const T *grad, int64_t rs, int64_t cs, int64_t n, int64_t n_rows,
                                                   int64_t width, int lanes, int span, uint32_t *row_begin, uint32_t *row_end, float *edge,
                                                   GradOut out)
{
    constexpr int U = 8;
    if (Wave) lanes = 64;
    const int group = Wave ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : threadIdx.x / lanes;
    const int64_t s = (int64_t)blockIdx.x * (256 / lanes) + group, p0 = s * span;
    const int64_t number = (int64_t)blockIdx.y * lanes + threadIdx.x % lanes;
    if (group >= 256 / lanes || p0 >= n || number * V >= width) return;
    const Lot<V> lot(number, width);
    const int64_t p1 = n - p0 < span ? n : p0 + span;
    uint32_t key = sorted[p0].key;
    if (key >= n_rows) return;   // ids without a row are the last ones
    bool from_before = p0 > 0 && sorted[p0 - 1].key == key;
    const T *mine = grad + (V == 1 ? lot.f * cs : lot.f);
    float sum[V];
#pragma unroll
    for (int k = 0; k < V; ++k) sum[k] = 0.f;
    auto finish = [&](int64_t end, bool goes_on) {   // the row `key` up to `end`, as far as this span has it
        if (from_before || goes_on) {
            store_cols<V>(edge + (s * 2 + (from_before ? 0 : 1)) * width + lot.f, sum);
        } else {
            out.put_as<O>(key, lot.f, lot.skip, sum);
        }
        if (number == 0 && !goes_on) row_end[key] = (uint32_t)end;
    };
    if (number == 0 && !from_before) row_begin[key] = (uint32_t)p0;
    // places past the span's end are its last one; the items of a step are loaded while the one before is under way
    Pair next[U];
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = sorted[p0 + u < p1 ? p0 + u : p1 - 1];
    for (int64_t p = p0; p < p1; p += U) {
        Pair item[U];
        float v[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) item[u] = next[u];
#pragma unroll
        for (int u = 0; u < U; ++u) load_cols<V, Stream>(v[u], mine + item[u].at * rs);   // of ids without a row too: their atoms are there
        if (p + U < p1) {
#pragma unroll
            for (int u = 0; u < U; ++u) next[u] = sorted[p + U + u < p1 ? p + U + u : p1 - 1];
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u >= p1) break;
            if (item[u].key != key) {
                finish(p + u, false);
                key = item[u].key;
                if (key >= n_rows) return;
                from_before = false;
                if (number == 0) row_begin[key] = (uint32_t)(p + u);
#pragma unroll
                for (int k = 0; k < V; ++k) sum[k] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k] += v[u][k];
        }
    }
    finish(p1, p1 < n && sorted[p1].key == key);
}

// Rows that no id names, and rows that spans share.  A thread has V columns of a row and adds up what at most kJoinSerial spans hold of it;
// a row of more spans is the work of one of the first `heavy` blocks (64 such lots of columns at most): block b looks at span b * kJoinSerial, and if the row
// that runs into this span from before is such a row, and no earlier block sees it, shares the row's spans out over its threads.  heavy0: of them, those
// of the launches before.
constexpr int kJoinSerial = 8, kJoinUnroll = 2;   // the second: rows looked up at a time

template <class O, int V>
__global__ __launch_bounds__(256) void k_row_join(const Pair *sorted, const uint32_t *row_begin, const uint32_t *row_end, const float *edge,
                                                  int shift, uint32_t heavy0, uint32_t heavy, uint32_t items, uint32_t per_row, Div31 div, int64_t row0,
                                                  int64_t n_rows, int64_t width, GradOut out)
{
    __shared__ double red[256][V];
    auto add = [&](double (&sum)[V], int64_t s, int64_t first, int64_t f) {
        float v[V];
        load_cols<V>(v, edge + (s * 2 + (s == first ? 1 : 0)) * width + f);
#pragma unroll
        for (int k = 0; k < V; ++k) sum[k] += (double)v[k];
    };
    if (blockIdx.x < heavy) {
        const uint32_t tiles = (per_row + 63) / 64, heavy_at = heavy0 + blockIdx.x;   // (2^32 of them have more parts than memory holds)
        const int lanes = per_row < 64 ? per_row : 64, groups = 256 / lanes;
        const int64_t at = ((int64_t)(heavy_at / tiles) + 1) * kJoinSerial;
        const uint32_t r = sorted[at << shift].key;
        if (r >= n_rows) return;
        const int64_t first = row_begin[r] >> shift, last = (row_end[r] - 1) >> shift;
        if (last - first < kJoinSerial || first >= at || first < at - kJoinSerial) return;
        const int group = threadIdx.x / lanes;
        const int64_t number = (int64_t)(heavy_at % tiles) * lanes + threadIdx.x % lanes;
        const bool mine = group < groups && number < per_row;
        const Lot<V> lot(number, width);
        double sum[V];
#pragma unroll
        for (int k = 0; k < V; ++k) sum[k] = 0.0;
        if (mine) {
#pragma unroll 8
            for (int64_t s = first + group; s <= last; s += groups) add(sum, s, first, lot.f);
        }
#pragma unroll
        for (int k = 0; k < V; ++k) red[threadIdx.x][k] = sum[k];
        __syncthreads();
        if (!mine || group > 0) return;
        for (int g = 1; g < groups; ++g) {
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k] += red[g * lanes + threadIdx.x][k];
        }
        out.put_as<O>(r, lot.f, lot.skip, sum);
        return;
    }
    constexpr int U = kJoinUnroll;
    const uint32_t step = (gridDim.x - heavy) * 256;
    for (uint32_t e0 = (blockIdx.x - heavy) * 256 + threadIdx.x; e0 < items; e0 += step * U) {
        uint32_t row[U], end[U], begin[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = div(e0 + u * step < items ? e0 + u * step : e0);
            end[u] = row_end[row0 + row[u]];
            begin[u] = row_begin[row0 + row[u]];   // anything where the row has no end
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t e = e0 + u * step;
            if (u > 0 && e >= items) break;
            const int64_t first = begin[u] >> shift, last = (end[u] - 1) >> shift;
            if (end[u] > 0 && (first == last || last - first >= kJoinSerial)) continue;
            const Lot<V> lot(e - row[u] * per_row, width);
            double sum[V];
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k] = 0.0;
            if (end[u] > 0) {
#pragma unroll 4
                for (int64_t s = first; s <= last; ++s) add(sum, s, first, lot.f);
            }
            out.put_as<O>(row0 + row[u], lot.f, lot.skip, sum);
        }
    }
}

// the parts of the workspace of the sorted way
struct SortSpace {
    size_t pairs[2], counts, row_begin, row_end, edge, bytes;
    int span;
    SortSpace(int64_t n, int64_t n_rows, int64_t width)
    {
        // spans as long as 2048 wavefronts still come of them, up to 64 items
        const int64_t lots = (width + 3) / 4;
        span = 64;
        while (span > 8 && n / span * lots < 2048 * 64) span /= 2;
        size_t at = 0;
        auto take = [&](size_t size) { const size_t here = at; at += (size + 255) & ~(size_t)255; return here; };
        for (size_t &p : pairs) p = take((size_t)n * sizeof(Pair));
        counts = take((size_t)kSortBlocks * kRadix * 4);
        row_begin = take((size_t)n_rows * 4);
        row_end = take((size_t)n_rows * 4);
        edge = take((size_t)((n + span - 1) / span) * 2 * (size_t)width * 4);
        bytes = at;
    }
};

size_t embed_grad_workspace(int64_t n, int64_t n_rows, int64_t width)
{
    if (takes_few(n, n_rows, width)) {
        const FewPlan p(n, n_rows, width);
        return p.blocks > 1 ? (size_t)p.blocks * (size_t)n_rows * (size_t)width * 4 : 0;
    }
    return SortSpace(n, n_rows, width).bytes;
}

// whether the gradients' rows begin at whole lines of memory
static bool whole_lines(const EmbedArgs &a)
{
    return reinterpret_cast<uintptr_t>(a.in) % 128 == 0 && a.rs * (int64_t)elem_size(a.in_dtype) % 128 == 0;
}

// Whether they are read past the caches: where there are more than the caches hold and rows share no lines.  (Lines that rows or tiles of
// columns share are better kept: a million bf16 rows of 77 into 8 58 us a call, 61 past the caches; of 800,000 fp32 rows of 64 43 and 38.)
static bool streams(const EmbedArgs &a)
{
    return (double)a.n * (double)a.width * (double)elem_size(a.in_dtype) > kStreamBytes && whole_lines(a);
}

static int few_rows(const EmbedArgs &a, const GradOut &out)
{
    const FewPlan p(a.n, a.n_rows, a.width);
    float *part = p.blocks > 1 ? static_cast<float *>(a.workspace) : nullptr;
    const bool stream = streams(a), grouped = p.blocks >= 8 && p.tiles > 1 && !(whole_lines(a) && p.tile * elem_size(a.in_dtype) % 128 == 0);
    const bool near = ((double)p.slots * (double)a.rs + (double)p.tile * (double)a.cs) * 4.0 < 4e9;
    with_elem(a.in_dtype, [&](auto t) {
        with_ids(a.id_bits, [&](auto id) {
            using T = decltype(t);
            using Id = decltype(id);
            auto launch = [&](auto kernel) {
                launch_blocks((int64_t)(grouped ? (p.blocks + 7) / 8 * 8 : p.blocks) * p.tiles, p.threads, [&](int64_t block0, unsigned blocks) {
                    kernel<<<blocks, p.threads, (size_t)p.waves * (a.n_rows + 1) * 256, a.stream>>>(
                        static_cast<const T *>(a.in), a.rs, a.cs, static_cast<const Id *>(a.ids), a.n, (int)a.n_rows, a.width, p.tile, p.slots,
                        p.waves, p.rows_per_wave, p.blocks, grouped, block0, part, out);
                });
            };
            auto pick = [&](auto one, auto close) {
                stream ? launch(k_few_rows<T, Id, one.value, close.value, true>) : launch(k_few_rows<T, Id, one.value, close.value, false>);
            };
            if (p.slots == 1) near ? pick(std::true_type{}, std::true_type{}) : pick(std::true_type{}, std::false_type{});
            else near ? pick(std::false_type{}, std::true_type{}) : pick(std::false_type{}, std::false_type{});
        });
    });
    MLIP_HIP(hipGetLastError());
    if (part) {
        const int64_t elements = a.n_rows * a.width;
        launch_blocks((elements + 15) / 16, 1024, [&](int64_t block0, unsigned blocks) {
            k_few_join<<<blocks, 1024, 0, a.stream>>>(part, p.blocks, elements, a.width, block0, out);
        });
        MLIP_HIP(hipGetLastError());
    }
    return MLIP_OK;
}

static int many_rows(const EmbedArgs &a, const GradOut &out)
{
    const SortSpace w(a.n, a.n_rows, a.width);
    const SortPlan p(a.n, a.n_rows);
    char *base = static_cast<char *>(a.workspace);
    auto u32 = [&](size_t at) { return reinterpret_cast<uint32_t *>(base + at); };
    Pair *list[2] = {reinterpret_cast<Pair *>(base + w.pairs[0]), reinterpret_cast<Pair *>(base + w.pairs[1])};
    uint32_t *counts = u32(w.counts), *row_begin = u32(w.row_begin), *row_end = u32(w.row_end);
    float *edge = reinterpret_cast<float *>(base + w.edge);
    const bool one_tile = a.n > 0 && a.n <= kSortTile;
    const Pair *sorted = one_tile ? list[0] : list[(p.passes - 1) & 1];
    with_ids(a.id_bits, [&](auto id) {
        using Id = decltype(id);
        const Id *ids = static_cast<const Id *>(a.ids);
        if (one_tile) {
            const int64_t clear = (a.n_rows + kSortThreads * 8 - 1) / (kSortThreads * 8);
            k_sort_tile<<<(unsigned)(1 + (clear < 256 ? clear : 256)), kSortThreads, 0, a.stream>>>(ids, (int)a.n, a.n_rows, p.passes, p.bits, list[0],
                                                                                               row_end);
            return;
        }
        const int64_t clear = (a.n_rows + kSortThreads * 8 - 1) / (kSortThreads * 8);   // blocks past the list's only clear
        const int blocks = clear > kSortBlocks ? kSortBlocks : clear > p.blocks ? (int)clear : p.blocks;
        k_digit_counts<<<blocks, kSortThreads, 0, a.stream>>>(ids, a.n, a.n_rows, p.range, 0, p.bits, counts, row_end);
        if (a.n > 0) k_digit_scatter<<<p.blocks, kSortThreads, 0, a.stream>>>(ids, a.n, a.n_rows, p.range, 0, p.bits, counts, list[0]);
    });
    for (int k = 1; k < p.passes && a.n > kSortTile; ++k) {
        const Pair *in = list[(k - 1) & 1];
        k_digit_counts<<<p.blocks, kSortThreads, 0, a.stream>>>(in, a.n, a.n_rows, p.range, k * p.bits, p.bits, counts, (uint32_t *)nullptr);
        k_digit_scatter<<<p.blocks, kSortThreads, 0, a.stream>>>(in, a.n, a.n_rows, p.range, k * p.bits, p.bits, counts, list[k & 1]);
    }
    MLIP_HIP(hipGetLastError());
    if (a.n > 0) {
        with_elem(a.in_dtype, [&](auto t) {
            using T = decltype(t);
            const int64_t spans = (a.n + w.span - 1) / w.span;
            const bool stream = streams(a);
            with_elem(a.out_dtype, [&](auto o) {
                using O = decltype(o);
                constexpr int V = 16 / sizeof(T);
                const bool wide = (a.cs == 1 || a.width == 1) && a.width >= V;
                const int64_t per_row = wide ? lots_of(a.width, V) : a.width;
                const int lanes = (int)(per_row < 64 ? per_row : 64);
                const int64_t groups = 256 / lanes;
                // (2^31 items in spans of 64, four spans or more to a block of 256 threads: not half of what one launch has)
                const dim3 grid((unsigned)((spans + groups - 1) / groups), (unsigned)((per_row + lanes - 1) / lanes));
                auto launch = [&](auto kernel) {
                    kernel<<<grid, 256, 0, a.stream>>>(sorted, static_cast<const T *>(a.in), a.rs, a.cs, a.n, a.n_rows, a.width, lanes, w.span,
                                                       row_begin, row_end, edge, out);
                };
                if (!wide) launch(k_span_sums<T, O, 1, false, false>);
                else if (lanes < 64) stream ? launch(k_span_sums<T, O, V, true, false>) : launch(k_span_sums<T, O, V, false, false>);
                else stream ? launch(k_span_sums<T, O, V, true, true>) : launch(k_span_sums<T, O, V, false, true>);
            });
        });
        MLIP_HIP(hipGetLastError());
    }
    const bool wide = a.width >= 4;
    const int64_t per_row = wide ? lots_of(a.width, 4) : a.width, most = ((int64_t)1 << 30) / per_row;
    const Div31 div((uint32_t)per_row);
    for (int64_t r0 = 0; r0 < a.n_rows; r0 += most) {
        const int64_t rows = a.n_rows - r0 < most ? a.n_rows - r0 : most, items = rows * per_row, blocks = (items + 256 * kJoinUnroll - 1) / (256 * kJoinUnroll);
        // spans kJoinSerial, 2 kJoinSerial, ... that there are, each for every 64 lots of columns; once
        const int64_t heavy = r0 == 0 && a.n > 0 ? ((a.n + w.span - 1) / w.span - 1) / kJoinSerial * ((per_row + 63) / 64) : 0;
        const int64_t light = blocks < 16384 ? blocks : 16384;
        auto launch = [&](auto kernel) {
            const int64_t most = most_blocks(256) - light;
            for (int64_t h = 0; h == 0 || h < heavy; h += most) {
                const int64_t some = heavy - h < most ? heavy - h : most;
                kernel<<<(unsigned)(some + (h + some == heavy ? light : 0)), 256, 0, a.stream>>>(
                    sorted, row_begin, row_end, edge, __builtin_ctz((unsigned)w.span), (uint32_t)h, (uint32_t)some, (uint32_t)items, (uint32_t)per_row, div, r0,
                    a.n_rows, a.width, out);
            }
        };
        with_elem(a.out_dtype, [&](auto o) {
            using O = decltype(o);
            wide ? launch(k_row_join<O, 4>) : launch(k_row_join<O, 1>);
        });
    }
    MLIP_HIP(hipGetLastError());
    return MLIP_OK;
}

int embed_grad_impl(const EmbedArgs &a)
{
    const GradOut out = {a.out, a.out_dtype, a.os, a.scale, a.accumulate};
    return takes_few(a.n, a.n_rows, a.width) ? few_rows(a, out) : many_rows(a, out);
}

}  // namespace mlip
