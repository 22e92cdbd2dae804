// Element types of the operators on lists of tensors and on embeddings: runs of elements as fp32 values, at any address that the
// element itself may have.  Vector accesses wider than the element's own alignment are split by nothing on gfx950: the same
// instruction serves an aligned and an unaligned address.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qadam_internal.h"

namespace qadam {

typedef float f4 __attribute__((ext_vector_type(4)));

// Addresses that a kernel reads from a table are global ones: said here, else the compiler takes the instructions that find out.
#define QADAM_GLOBAL __attribute__((address_space(1)))
template <typename T>
__device__ __forceinline__ QADAM_GLOBAL T* global(T* p) { return (QADAM_GLOBAL T*)p; }

template <int TYPE> struct Element;
template <> struct Element<QADAM_F32> { typedef float T; };
template <> struct Element<QADAM_BF16> { typedef __bf16 T; };
template <> struct Element<QADAM_F16> { typedef _Float16 T; };
template <> struct Element<QADAM_CODES8> { typedef int8_t T; };
template <> struct Element<QADAM_CODES16> { typedef int16_t T; };

template <int TYPE, int N>
struct Run {
    typedef typename Element<TYPE>::T T;
    typedef T V __attribute__((ext_vector_type(N)));
    typedef V U __attribute__((aligned(sizeof(T))));
    typedef float F __attribute__((ext_vector_type(N)));
};

// N elements at p, read past the caches (ONCE) or through them
template <int TYPE, int N, bool ONCE = true>
__device__ __forceinline__ typename Run<TYPE, N>::V load_raw(const void* p)
{
    const auto* q = (const QADAM_GLOBAL typename Run<TYPE, N>::U*)p;
    if constexpr (ONCE) return __builtin_nontemporal_load(q);
    else return *q;
}

template <int TYPE, int N>
__device__ __forceinline__ typename Run<TYPE, N>::F to_float(typename Run<TYPE, N>::V v)
{
    return __builtin_convertvector(v, typename Run<TYPE, N>::F);
}

// rounding to bfloat16 and half is to nearest, ties to even
template <int TYPE, int N, bool ONCE = true>
__device__ __forceinline__ void store_run(void* p, typename Run<TYPE, N>::F x)
{
    const auto v = __builtin_convertvector(x, typename Run<TYPE, N>::V);
    auto* q = (QADAM_GLOBAL typename Run<TYPE, N>::U*)p;
    if constexpr (ONCE) __builtin_nontemporal_store(v, q);
    else *q = v;
}

inline __host__ __device__ int element_size(int type)
{
    return type == QADAM_F32 ? 4 : type == QADAM_CODES8 ? 1 : 2;
}

// one element of a type known at run time
__device__ __forceinline__ float load_one(const void* p, int type, int64_t i)
{
    if (type == QADAM_F32) return global(static_cast<const float*>(p))[i];
    if (type == QADAM_BF16) return (float)global(static_cast<const __bf16*>(p))[i];
    return (float)global(static_cast<const _Float16*>(p))[i];
}

}  // namespace qadam
