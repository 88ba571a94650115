// Element types of the parameter tables and gradients: a call's type codes become template arguments.
#pragma once

#include "mlip_internal.h"

namespace mlip {

inline size_t elem_size(int32_t dtype) { return dtype == MLIP_DTYPE_F32 ? 4 : 2; }
inline bool elem_known(int32_t dtype) { return dtype >= MLIP_DTYPE_F32 && dtype <= MLIP_DTYPE_F16; }

// f(T{}) with the element type of a (checked) type code
template <class Fn> inline void with_elem(int32_t dtype, Fn &&f)
{
    if (dtype == MLIP_DTYPE_F32) f(float{});
    else if (dtype == MLIP_DTYPE_BF16) f(__bf16{});
    else f(_Float16{});
}

// f(Id{}) with the type of the ids
template <class Fn> inline void with_ids(int32_t id_bits, Fn &&f)
{
    if (id_bits == 32) f(int32_t{});
    else f(int64_t{});
}

// What is larger than this is read or written past the caches where it is touched once: they could not keep it for anyone.  Measured, us a call past
// the caches and through them (fp32, rows of 64): clipping 32 MB 22 and 19, 96 MB 51 and 55, 256 MB 128 and 146; lookup of 32 MB 9.6 and 9.0, 64 MB 12.3 and
// 12.5, 256 MB 43.6 and 45.4; gradient into few rows of 32 MB 16 and 15, 96 MB 21.6 and 22, 256 MB 50 and 54, into many of 64 MB 51 and 47, 128 MB 66.5 and 69.5.
constexpr double kStreamBytes = 100e6;

// Blocks that a launch has at most, a multiple of eight so that the XCDs' turn goes on from launch to launch: HIP takes a grid's threads modulo 2^32, with
// no error, and leaves the other blocks out.
inline int64_t most_blocks(int threads) { return 0xffffffffll / threads / 8 * 8; }

// launch(first block, blocks) for `blocks` blocks, in as many launches as that takes
template <class Fn> inline void launch_blocks(int64_t blocks, int threads, Fn &&launch)
{
    const int64_t most = most_blocks(threads);
    for (int64_t b = 0; b < blocks; b += most) launch(b, (unsigned)(blocks - b < most ? blocks - b : most));
}

// V elements, as one access has them
template <class T, int V> using Cols = T __attribute__((ext_vector_type(V)));
template <class T, int V> struct FarT { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };
template <class T, int V> using Far = typename FarT<T, V>::type;   // the same at the alignment of an element

#ifdef __HIPCC__
// An fp32 value rounded to an element's type.  The value is made opaque on its way to fp16: the compiler would otherwise take the
// product that it may be and this rounding as one mixed-precision instruction, which rounds once where two roundings are documented.
template <class T> __device__ inline T to_elem(float v)
{
    if constexpr (sizeof(T) == 2) asm("" : "+v"(v));
    return (T)v;
}
// add(load(k)) for k = from, from + step, ... below end, in this order, U loads at a time (the last ones too: past the end the first one of the step
// stands in, which is not added)
template <int U, class Load, class Add> __device__ inline void in_steps(int64_t from, int64_t end, int64_t step, Load &&load, Add &&add)
{
    for (int64_t k = from; k < end; k += step * U) {
        decltype(load(k)) x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load(k + u * step < end ? k + u * step : k);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (k + u * step < end) add(x[u]);
    }
}
#endif

}  // namespace mlip
