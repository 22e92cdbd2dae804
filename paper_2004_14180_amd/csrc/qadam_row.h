// Rows of elements in runs per lane, and sums over the lanes of a wavefront or a workgroup.
#pragma once

#include "qadam_elements.h"

namespace qadam {

constexpr int kRowRun = 8;
typedef float f8 __attribute__((ext_vector_type(8)));

// `n` elements at p, at most kRowRun of them; zeros behind them
template <int TYPE, bool ONCE = true>
__device__ __forceinline__ typename Run<TYPE, kRowRun>::V load_part(const void* p, int n)
{
    if (n >= kRowRun) return load_raw<TYPE, kRowRun, ONCE>(p);
    typename Run<TYPE, kRowRun>::V v = 0;
    const auto* q = (const QADAM_GLOBAL typename Element<TYPE>::T*)p;
#pragma unroll
    for (int k = 0; k < kRowRun - 1; ++k)
        if (k < n) v[k] = q[k];
    return v;
}

// The run at `at` < dim of a row of `dim` elements, not yet put in its place: where the row ends within it, its last kRowRun elements, in one
// load that nothing waits for before the run is used, as a wave does for loads of single elements under conditions.  REPEAT: `at` may be
// behind the row, and what `loaded` gives behind the row's end are elements of the row, where there are zeros else.
template <int TYPE, bool REPEAT = false>
__device__ __forceinline__ typename Run<TYPE, kRowRun>::V load_ahead(const typename Element<TYPE>::T* row, int at, int dim)
{
    if (dim < kRowRun) {
        typename Run<TYPE, kRowRun>::V v = load_part<TYPE, false>(row, dim);
        if constexpr (REPEAT) {
#pragma unroll
            for (int k = 1; k < kRowRun; ++k) v[k] = k < dim ? v[k] : v[0];
        }
        return v;
    }
    return load_raw<TYPE, kRowRun, false>(row + (at + kRowRun <= dim ? at : dim - kRowRun));
}

// ... and its elements in their place
template <int TYPE, bool REPEAT = false>
__device__ __forceinline__ f8 loaded(typename Run<TYPE, kRowRun>::V v, int at, int dim)
{
    typedef typename Element<TYPE>::T T;
    if (at < dim && at + kRowRun > dim && dim >= kRowRun) {
        const int by = at + kRowRun - dim;
#pragma unroll
        for (int b = kRowRun / 2; b > 0; b /= 2)
            if (by & b) {
#pragma unroll
                for (int k = 0; k < kRowRun; ++k) v[k] = k + b < kRowRun ? v[k + b < kRowRun ? k + b : 0] : REPEAT ? v[k] : (T)0;
            }
    }
    return to_float<TYPE, kRowRun>(v);
}

template <int TYPE, bool ONCE = true>
__device__ __forceinline__ void store_part(void* p, f8 x, int n)
{
    if (n >= kRowRun) return store_run<TYPE, kRowRun, ONCE>(p, x);
    auto* q = (QADAM_GLOBAL typename Element<TYPE>::T*)p;
#pragma unroll
    for (int k = 0; k < kRowRun - 1; ++k)
        if (k < n) q[k] = (typename Element<TYPE>::T)x[k];
}

// ... of elements whose type is known at run time
__device__ __forceinline__ f8 load_part(const void* base, int type, int64_t at, int n)
{
    if (type == QADAM_F32) return load_part<QADAM_F32, false>(static_cast<const float*>(base) + at, n);
    if (type == QADAM_BF16) return to_float<QADAM_BF16, kRowRun>(load_part<QADAM_BF16, false>(static_cast<const __bf16*>(base) + at, n));
    return to_float<QADAM_F16, kRowRun>(load_part<QADAM_F16, false>(static_cast<const _Float16*>(base) + at, n));
}

__device__ __forceinline__ void store_part(void* base, int type, int64_t at, f8 x, int n)
{
    if (type == QADAM_F32) store_part<QADAM_F32>(static_cast<float*>(base) + at, x, n);
    else if (type == QADAM_BF16) store_part<QADAM_BF16>(static_cast<__bf16*>(base) + at, x, n);
    else store_part<QADAM_F16>(static_cast<_Float16*>(base) + at, x, n);
}

// Value of another lane of the wavefront, by the pattern CTRL of a data-parallel move; lanes outside the rows of 16 in ROWS get 0.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float moved(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
}

// Sum over a wavefront, the same in all lanes, always in the same order: pairs, quads, 8, 16, then the rows of 16.
__device__ __forceinline__ float wave_sum(float x)
{
    x += moved<0xb1>(x);            // lanes 1 0 3 2
    x += moved<0x4e>(x);            // lanes 2 3 0 1
    x += moved<0x141>(x);           // mirrored within 8
    x += moved<0x140>(x);           // mirrored within 16
    x += moved<0x142, 0xa>(x);      // lane 15 of each row of 16 into the next row, rows 1 and 3
    x += moved<0x143, 0xc>(x);      // lane 31 into rows 2 and 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

}  // namespace qadam
