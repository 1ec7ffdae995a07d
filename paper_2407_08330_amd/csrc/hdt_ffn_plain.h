// The products of the gated feed-forward block for every size, type and alignment: tiles of 64 x 64, operands taken element by element.
#pragma once

#include "hdt_ffn.h"

namespace hdt_ffn {

template <typename T>
struct PlainOp;
template <>
struct PlainOp<__bf16> {
    static constexpr int STEP = 16, PAD = 8;
    // row l % 32, k = (l / 32) 8 + 0 .. 7
    static __device__ __forceinline__ f32x16 mma(const __bf16 *a, const __bf16 *b, int lane, f32x16 c)
    {
        const int k = (lane >> 5) * 8;
        return mfma_32x32x16(*reinterpret_cast<const bf16x8 *>(a + k), *reinterpret_cast<const bf16x8 *>(b + k), c);
    }
};
template <>
struct PlainOp<float> {
    static constexpr int STEP = 2, PAD = 2;
    static __device__ __forceinline__ f32x16 mma(const float *a, const float *b, int lane, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x2f32(a[lane >> 5], b[lane >> 5], c, 0, 0, 0);
    }
};

// A workgroup of 2 x 2 waves, a wave 32 x 32 (two sums of them for GATE).  What is beyond m, n or k counts as zero on both sides, so that
// nothing there, NaN or not, is met.  C^T = B A^T: a lane holds one m and rows of n.
template <typename T, int KIND, bool A_SLOW, bool B_SLOW>
__global__ __launch_bounds__(256) void k_ffn_plain(Product p)
{
    using Op = PlainOp<T>;
    constexpr int BK = 32, LD = BK + Op::PAD, NB = KIND == GATE ? 2 : 1;
    __shared__ __attribute__((aligned(16))) T sa[64 * LD], sb[NB][64 * LD];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t tiles_n = (p.n + 63) / 64;
    const int64_t tile = blockIdx.x;
    const int m0 = (int)(tile / tiles_n) * 64, n0 = (int)(tile % tiles_n) * 64;
    f32x16 acc[NB];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[b][e] = 0.f;

    auto stage = [&](T *to, const T *from, int64_t ld, bool slow, int r0, int rows, int k0) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int r = slow ? tid & 63 : (tid >> 5) + 8 * i, k = slow ? (tid >> 6) + 4 * i : tid & 31;
            T v = (T)0.f;
            if (r0 + r < rows && k0 + k < p.k) v = slow ? from[(int64_t)(k0 + k) * ld + r0 + r] : from[(int64_t)(r0 + r) * ld + k0 + k];
            to[r * LD + k] = v;
        }
    };
    for (int range = 0; range < p.ranges; range++)
        for (int k0 = 0; k0 < p.k; k0 += BK) {
            __syncthreads();
            stage(sa, (const T *)p.a[range], p.lda, A_SLOW, m0, p.m, k0);
#pragma unroll
            for (int b = 0; b < NB; b++) stage(sb[b], (const T *)p.b[NB == 2 ? b : range], p.ldb, B_SLOW, n0, p.n, k0);
            __syncthreads();
            const T *pa = sa + ((wave >> 1) * 32 + (lane & 31)) * LD;
#pragma unroll
            for (int k = 0; k < BK; k += Op::STEP)
#pragma unroll
                for (int b = 0; b < NB; b++) acc[b] = Op::mma(sb[b] + ((wave & 1) * 32 + (lane & 31)) * LD + k, pa + k, lane, acc[b]);
        }

    const int m = m0 + (wave >> 1) * 32 + (lane & 31);
    if (m >= p.m) return;
#pragma unroll
    for (int e = 0; e < 16; e++) {
        const int n = n0 + (wave & 1) * 32 + (lane >> 5) * 4 + 8 * (e >> 2) + (e & 3);
        if (n >= p.n) continue;
        const int64_t at = (int64_t)m * p.ldo + n;
        if (KIND == GATE) {
            const float g = acc[0][e], u = acc[NB - 1][e];
            Act f;
            by_act(p.act, [&](auto act) { f = activate<true, decltype(act)::value>(g); });
            if (p.out[0]) {
                ((T *)p.out[0])[at] = (T)(u * f.slope);
                ((T *)p.out[1])[at] = (T)f.value;
            }
            ((T *)p.out[2])[at] = (T)(f.value * u);
        } else if (KIND == DGATE) {
            ((T *)p.out[0])[at] = (T)(acc[0][e] * (float)((const T *)p.by_gate)[at]);
            ((T *)p.out[1])[at] = (T)(acc[0][e] * (float)((const T *)p.by_up)[at]);
        } else {
            ((T *)p.out[0])[at] = (T)acc[0][e];
        }
    }
}

template <typename T, int KIND, bool A_SLOW, bool B_SLOW>
void launch_plain(const Product &p, hipStream_t st)
{
    const int64_t tiles = ((int64_t)p.m + 63) / 64 * (((int64_t)p.n + 63) / 64);
    hipLaunchKernelGGL((k_ffn_plain<T, KIND, A_SLOW, B_SLOW>), dim3((unsigned)tiles), dim3(256), 0, st, p);
}

}  // namespace hdt_ffn
