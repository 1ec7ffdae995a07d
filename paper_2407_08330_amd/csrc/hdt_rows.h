// Rows of bf16 or fp32 values eight at a time, and sums over a row.
#pragma once

#include <hip/hip_runtime.h>

#include "hdt_lanes.h"

namespace hdt_rows {

// 8 consecutive elements as they are in memory; `left` of them exist (WHOLE: all).  The address is aligned to an element only.
template <typename T>
struct Vec {
    typedef T V __attribute__((ext_vector_type(8)));
    typedef V Any __attribute__((aligned(sizeof(T))));
};
template <bool WHOLE, typename T>
__device__ __forceinline__ typename Vec<T>::V load8(const T *p, int left)
{
    if (WHOLE || left >= 8) return *reinterpret_cast<const typename Vec<T>::Any *>(p);
    typename Vec<T>::V r;
#pragma unroll
    for (int e = 0; e < 8; e++) r[e] = e < left ? p[e] : (T)0.f;
    return r;
}
struct Eight {
    float x[8];
};
template <bool WHOLE, typename T>
__device__ __forceinline__ void store8(T *p, const Eight &r, int left)
{
    if (WHOLE || left >= 8) {
        typename Vec<T>::V v;
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (T)r.x[e];
        *reinterpret_cast<typename Vec<T>::Any *>(p) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (e < left) p[e] = (T)r.x[e];
}
template <bool WHOLE>
__device__ __forceinline__ Eight load_weight(const void *p, int bf16, int at, int left)
{
    Eight r;
    if (bf16) {
        const auto v = load8<WHOLE>((const __bf16 *)p + at, left);
#pragma unroll
        for (int e = 0; e < 8; e++) r.x[e] = (float)v[e];
    } else {
        const auto v = load8<WHOLE>((const float *)p + at, left);
#pragma unroll
        for (int e = 0; e < 8; e++) r.x[e] = v[e];
    }
    return r;
}

// the sum over the threads of a row: a wave, or (TPR > 64) the whole workgroup
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float *lds)
{
    x = hdt_lanes::wave_sum(x);
    if (TPR > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int i = 0; i < TPR / 64; i++) x += lds[i];
    }
    return x;
}

}  // namespace hdt_rows
