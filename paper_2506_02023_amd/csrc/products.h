// Matrix products of 16-bit parts on the matrix units, for the operators that train node networks: a block's tile of
// C = A B^T with A and B as panels of parts, handed to an epilogue in registers.
//
// An operand of a type of 16 bits is one part, itself (or, fp16 beside bf16, two bf16 parts, exact).  fp32 operands are three bf16 parts (hi + mid + lo, exact), of whose products the six down to 2^-24 are
// taken: 2.7 times the rate of the fp32 matrix instructions at their precision.  Values near 1 can be two fp16 parts (22 bits), three products.
// Sums are fp32.
#pragma once

#include <type_traits>

#include "elem.h"

namespace mlip {

// An operand: `parts` matrices of rows x cols elements of 16 bits, `part` elements apart, rows `ld` apart, all aligned to 16 bytes.  Along the summed
// dimension "K", a panel with K in its columns holds zeros up to a multiple of kStepK; one with K in its rows ends where it ends.
struct Panel {
    const void *p;
    int64_t ld, part, rows, cols;
};

#ifdef __HIPCC__
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void LdsVoid;

template <class T> using Half8 = Cols<T, 8>;
template <class T> using Half4 = Cols<T, 4>;

template <class T> __device__ inline f32x16 mfma(Half8<T> a, Half8<T> b, f32x16 c)
{
    if constexpr (std::is_same_v<T, __bf16>) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Four elements of a column of 16 lanes' 16 x 4 block of rows, per lane
template <class T> __device__ inline Half4<T> read_turned(const T *lds)
{
    typedef __attribute__((address_space(3))) Half4<__bf16> Lds4;
    return __builtin_bit_cast(Half4<T>, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((Lds4 *)lds));
}

// An fp32 value as PARTS parts of T, each the rest of the ones before rounded to nearest
template <class T, int PARTS> __device__ inline void split(float v, T (&part)[PARTS])
{
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        part[p] = to_elem<T>(v);
        v -= (float)part[p];
    }
}
#endif

// Elements of K that one step takes: 64 of one part, 32 of several (LDS), 16 of several where both panels have K in their rows and the tiles are of 128, so that two blocks share a
// compute unit (202,612 rows of 128 x 704 of three parts: 507 us in steps of 32, 312 here; panels with K in their columns would be read in quarters of lines; tiles of 256 have one
// to themselves either way: 32,768 x 1024 x 4096 bf16 2.97 ms in steps of 16, 2.74 in 32)
template <int PARTS, bool KC, int LEAST> constexpr int kStepK = PARTS == 1 ? 64 : KC || LEAST != 128 ? 32 : 16;
// Columns that a panel with K in its columns is filled up to: a multiple of both
constexpr int64_t kPadK = 64;
inline int64_t pad_to(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
// The same with an odd number of memory lines, so that the rows of a tile do not all lie in the same memory channels
inline int64_t pad_odd(int64_t n) { return pad_to(n, 64) | 64; }

#ifdef __HIPCC__
// A tile of a panel in LDS: PARTS times ROWS rows of m (or n) by KT of k.  KC: the panel has k in its columns, the tile is [ROWS][KT];
// else [KT][ROWS].  Pieces of 16 bytes come straight from memory, 64 of a wavefront one after another; which piece lies where within a row is
// turned with the row so that the reads of fragments below meet all banks.
template <class T, int PARTS, bool KC, int ROWS, int KT, int THREADS> struct Tile {
    static constexpr int kRow = KC ? KT : ROWS, kPieces = kRow / 8, kPart = ROWS * KT, kElems = PARTS * kPart;
    static constexpr int kLoads = PARTS * kPart / 8 / THREADS;
    static_assert(kPart / 8 % THREADS == 0 && (kPieces == 2 || kPieces == 4 || kPieces == 8 || kPieces % 16 == 0), "whole rounds of loads");

    static __device__ inline int turn(int row)
    {
        if constexpr (KC) return kPieces == 8 ? (row >> 1) & 7 : kPieces == 4 ? (row >> 2) & 3 : (row >> 3) & 1;
        else return kPieces == 8 ? ((row >> 1) & 1) * 4 : (row & 3) * 4;
    }

    // Requests the tile whose first row of the operand is `at` and whose first k is `k` (uniform over the block)
    static __device__ inline void load(const Panel &a, int64_t at, int64_t k, T *lds)
    {
        const int64_t r0 = KC ? at : k, c0 = KC ? k : at;
        const int64_t left = r0 < a.rows && c0 < a.cols ? ((a.rows - 1 - r0) * a.ld + a.cols - c0) * 2 : 0;
        const int records = (int)(left < 0x7ffffff0 ? left : 0x7ffffff0);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)(static_cast<const T *>(a.p) + p * a.part + r0 * a.ld + c0), 0, records, 0x00020000);
#pragma unroll
            for (int i = 0; i < kLoads / PARTS; ++i) {
                const int q = i * THREADS + threadIdx.x, row = q / kPieces, piece = q % kPieces ^ turn(row);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsVoid *)(lds + p * kPart + (i * THREADS + wave * 64) * 8), 16, (row * (int)a.ld + piece * 8) * 2, 0, 0, 0);
            }
        }
    }

    // The fragment of a lane for 32 rows from `at` and 16 k from 16 kk: row lane % 32, k = 8 (lane / 32) + 0 .. 7
    static __device__ inline Half8<T> frag(const T *lds, int p, int at, int kk)
    {
        const int lane = threadIdx.x & 63;
        if constexpr (KC) {
            const int row = at + (lane & 31), piece = kk * 2 + (lane >> 5);
            return *reinterpret_cast<const Half8<T> *>(lds + p * kPart + (row * kPieces + (piece ^ turn(row))) * 8);
        } else {
            const int g = lane >> 4, i = lane & 15, k = kk * 16 + (g >> 1) * 8 + (i >> 2), piece = at / 8 + (g & 1) * 2 + ((i & 3) >> 1);
            const T *q = lds + p * kPart + (k * kPieces + (piece ^ turn(k))) * 8 + (i & 1) * 4;
            const Half4<T> lo = read_turned(q), hi = read_turned(q + 4 * kPieces * 8);   // (k + 4 has k's turn)
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// The pairs of parts of A and B whose products are taken, large ones last (they are added to what is there)
template <int PA, int PB, class Fn> __device__ inline void for_products(Fn &&f)
{
    if constexpr (PA == 3 && PB == 3) { f(2, 0); f(0, 2); f(1, 1); }
    if constexpr (PA >= 2) f(1, 0);
    if constexpr (PB >= 2) f(0, 1);
    f(0, 0);
}

// acc[i][j] += rows 32 i .. of A times rows 32 j .. of B, of a wavefront's WM x WN part of the block's BM x BN tile, summed over k in [k0, k1).
// each(fragments of B): called in every step, for sums along K.
template <class T, int PA, int PB, bool AKC, bool BKC, int BM, int BN, int WM, int WN> struct Product {
    static constexpr int kWaves = (BM / WM) * (BN / WN), kThreads = kWaves * 64, KT = kStepK<(PA > PB ? PA : PB), AKC || BKC, (BM < BN ? BM : BN)>;
    using TA = Tile<T, PA, AKC, BM, KT, kThreads>;
    using TB = Tile<T, PB, BKC, BN, KT, kThreads>;
    static constexpr int kStage = TA::kElems + TB::kElems;
    static constexpr int kTurned = kWaves * 64 * 64 * 2;   // what Turned takes of it afterwards
    struct alignas(16) Lds { T e[2 * kStage > kTurned ? 2 * kStage : kTurned]; };

    template <class Each>
    static __device__ inline void run(const Panel &a, const Panel &b, int64_t m0, int64_t n0, int64_t k0, int64_t k1, Lds &lds, f32x16 (&acc)[WM / 32][WN / 32],
                                      Each &&each)
    {
        const int wave = threadIdx.x >> 6, wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
        int at = 0;
        if (k0 < k1) {
            TA::load(a, m0, k0, lds.e);
            TB::load(b, n0, k0, lds.e + TA::kElems);
        }
        for (int64_t k = k0; k < k1; k += KT, at ^= 1) {
            __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): loads to LDS are loads, for which a barrier by itself does not wait
            __syncthreads();   // this step's tiles are there, and all are done with the other ones
            T *la = lds.e + at * kStage, *lb = la + TA::kElems;
            if (k + KT < k1) {
                TA::load(a, m0, k + KT, lds.e + (at ^ 1) * kStage);
                TB::load(b, n0, k + KT, lds.e + (at ^ 1) * kStage + TA::kElems);
            }
#pragma unroll
            for (int kk = 0; kk < KT / 16; ++kk) {
                Half8<T> fa[WM / 32][PA], fb[WN / 32][PB];
#pragma unroll
                for (int p = 0; p < PA; ++p)
#pragma unroll
                    for (int i = 0; i < WM / 32; ++i) fa[i][p] = TA::frag(la, p, wm + 32 * i, kk);
#pragma unroll
                for (int p = 0; p < PB; ++p)
#pragma unroll
                    for (int j = 0; j < WN / 32; ++j) fb[j][p] = TB::frag(lb, p, wn + 32 * j, kk);
                for_products<PA, PB>([&](int p, int q) {
#pragma unroll
                    for (int i = 0; i < WM / 32; ++i)
#pragma unroll
                        for (int j = 0; j < WN / 32; ++j) acc[i][j] = mfma<T>(fa[i][p], fb[j][q], acc[i][j]);
                });
                each(fb);
            }
        }
    }
};

// A block's tile: 128 x 128 in four wavefronts (64 x 256 where there are no more columns), or 256 x 256 in eight of 128 x 64 each.  The larger one brings half the bytes from the caches for the same
// products, the smaller one shares a compute unit with another block and leaves no one idle where there are few.
template <int COLS, int ROWS> struct Block {   // of the first operand and of the second
    static constexpr int kCols = COLS, kRows = ROWS, kPer = COLS == 256 ? 128 : 64, kThreads = COLS / kPer * (ROWS / 64) * 64;   // kPer x 64: a wavefront's share
    template <class T, int PA, int PB, bool AKC, bool BKC> using Of = Product<T, PA, PB, AKC, BKC, COLS, ROWS, kPer, 64>;
    static __device__ inline int first(int wave) { return wave / (ROWS / 64) * kPer; }
    static __device__ inline int second(int wave) { return wave % (ROWS / 64) * 64; }
};
using Narrow = Block<64, 256>;
using Middle = Block<128, 128>;
using Large = Block<256, 256>;

// Row and column of register r of a 32 x 32 result: the row of A and, in the lane, of B
__device__ inline int acc_row(int r) { return 8 * (r >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (r & 3); }
__device__ inline int acc_col() { return threadIdx.x & 31; }

// A wavefront's 64 x 64 result, turned around in 16 KB of LDS of its own so that memory is met in whole lines: lanes take four or eight neighbouring elements along the
// first operand's rows ("columns" here) of one of the second's ("rows").  The caller has made sure that nobody reads what lay in the LDS before.  Four
// columns together are a piece; which piece lies where is turned with the row so that writes and reads meet all banks.
struct Turned {
    float *at;
    __device__ inline float *piece(int row, int p) const { return at + row * 64 + ((p ^ (row & 15)) << 2); }
    __device__ inline void fence() const
    {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");   // a wavefront's LDS operations are done in order: this only keeps the compiler from moving them
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    __device__ inline void put(const f32x16 (*acc)[2]) const
    {
        fence();
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<Cols<float, 4> *>(piece(32 * j + acc_col(), (32 * i + acc_row(4 * q)) / 4)) =
                        Cols<float, 4>{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        fence();
    }
    template <int W> __device__ inline void get(float (&v)[W], int row, int col) const
    {
#pragma unroll
        for (int p = 0; p < W / 4; ++p) {
            const Cols<float, 4> w = *reinterpret_cast<const Cols<float, 4> *>(piece(row, col / 4 + p));
#pragma unroll
            for (int k = 0; k < 4; ++k) v[4 * p + k] = w[k];
        }
    }
    __device__ inline void set(const float (&v)[8], int row, int col) const
    {
        *reinterpret_cast<Cols<float, 4> *>(piece(row, col / 4)) = Cols<float, 4>{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<Cols<float, 4> *>(piece(row, col / 4 + 1)) = Cols<float, 4>{v[4], v[5], v[6], v[7]};
    }
    __device__ inline float one(int row, int col) const { return piece(row, col >> 2)[col & 3]; }
};

// W elements from column c of a row on, zeros from `cols` on; and stored, those before `cols`
template <class E, int W> __device__ inline void load_cols(float (&v)[W], const E *row, int64_t cs, int64_t c, int64_t cols)
{
    if (cs == 1 && c + W <= cols) {
        const Cols<E, W> w = *reinterpret_cast<const Far<E, W> *>(row + c);
#pragma unroll
        for (int k = 0; k < W; ++k) v[k] = (float)w[k];
        return;
    }
#pragma unroll
    for (int k = 0; k < W; ++k) v[k] = c + k < cols ? (float)row[(c + k) * cs] : 0.f;
}
template <class E, int W> __device__ inline void store_cols(const float (&v)[W], E *row, int64_t c, int64_t cols)
{
    if (c + W <= cols) {
        Cols<E, W> w;
#pragma unroll
        for (int k = 0; k < W; ++k) w[k] = to_elem<E>(v[k]);
        *reinterpret_cast<Far<E, W> *>(row + c) = w;
        return;
    }
#pragma unroll
    for (int k = 0; k < W; ++k)
        if (c + k < cols) row[c + k] = to_elem<E>(v[k]);
}
template <class T, int PARTS, int W> __device__ inline void split_cols(const float (&v)[W], Cols<T, W> (&part)[PARTS])
{
#pragma unroll
    for (int k = 0; k < W; ++k) {
        T s[PARTS];
        split(v[k], s);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) part[p][k] = s[p];
    }
}

// Block b of `blocks` takes place (b % 8) * (blocks / 8) + b / 8 of the order, as far as that divides: the blocks that an XCD gets lie one after another, so
// that its L2 holds what neighbours share.
__device__ inline int64_t xcd_order(int64_t b, int64_t blocks)
{
    const int64_t each = blocks / 8, whole = each * 8;
    return b < whole ? b % 8 * each + b / 8 : b;
}
#endif

}  // namespace mlip
