// Element types of the parameter tables and gradients: a call's type codes become template arguments.
#pragma once

#include "mlip_internal.h"

namespace mlip {

template <int DT> struct ElemT;
template <> struct ElemT<MLIP_DTYPE_F32> { using type = float; };
template <> struct ElemT<MLIP_DTYPE_BF16> { using type = __bf16; };
template <> struct ElemT<MLIP_DTYPE_F16> { using type = _Float16; };

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

// V elements, as one access has them
template <class T, int V> using Cols = T __attribute__((ext_vector_type(V)));

#ifdef __HIPCC__
// An fp32 value rounded to an element's type.  The value is made opaque on its way to fp16: the compiler would otherwise take the
// product that it may be and this rounding as one mixed-precision instruction, which rounds once where two roundings are documented.
template <class T> __device__ inline T to_elem(float v)
{
    if constexpr (sizeof(T) == 2) asm("" : "+v"(v));
    return (T)v;
}
#endif

}  // namespace mlip
