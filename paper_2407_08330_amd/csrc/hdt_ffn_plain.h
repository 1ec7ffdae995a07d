// The products of the gated feed-forward block in fp32.
#pragma once

#include "hdt_ffn.h"
#include "hdt_ffn_plan.h"

namespace hdt_ffn {

// A group of W x W waves makes a tile, a wave 32 x 32 of it (two sums of them for GATE).  GROUPS of them divide k, 32 at a time, and join at the end
// in a fixed order: where there are few tiles a tile's walk along k is what takes the time.  A tile of k is requested before the one in
// front of it is multiplied.  What is beyond m, n or k counts as zero on both sides, so that nothing there, NaN or not, is met.  C^T = B A^T: a
// lane holds one m and rows of n.
constexpr int kPlainK = 32;
constexpr int kPlainRow = kPlainK + 2;  // floats of a row in LDS
template <int KIND, int W, int GROUPS>
constexpr int plain_lds() { return GROUPS * (KIND == GATE ? 3 : 2) * 32 * W * kPlainRow * (int)sizeof(float); }
struct PlainArgs {
    Product p[3];
    unsigned first[3], tiles;  // first tile of each product; of all
};

template <int KIND, bool A_SLOW, bool B_SLOW, int W, int GROUPS>
__global__ __launch_bounds__(64 * W * W * GROUPS) void k_ffn_plain(PlainArgs a)
{
    constexpr int LD = kPlainRow, NB = KIND == GATE ? 2 : 1, SIDE = 32 * W, THREADS = 64 * W * W, EACH = SIDE * kPlainK / THREADS, TILE = SIDE * LD;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int all = threadIdx.x, group = __builtin_amdgcn_readfirstlane(all / THREADS), tid = all % THREADS, lane = tid & 63, wave = tid >> 6;
    float *const sa = reinterpret_cast<float *>(smem) + group * (1 + NB) * TILE, *const sb = sa + TILE;
    const int which = blockIdx.x >= a.first[2] ? 2 : blockIdx.x >= a.first[1] ? 1 : 0;
    const Product &p = a.p[which];
    const int64_t tiles_n = (p.n + SIDE - 1) / SIDE, tile = blockIdx.x - a.first[which];
    const int m0 = (int)(tile / tiles_n) * SIDE, n0 = (int)(tile % tiles_n) * SIDE;
    f32x16 acc[NB];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[b][e] = 0.f;

    // four values a load, of k or, of operands whose k is slow, of rows (one a load, each with its bounds: 512 x 384 x 1000, forward and backward, 159 us for 126,
    // 98 x 1024 x 3248 318 for 215, 2048 x 768 x 2048 943 for 789)
    typedef float Four __attribute__((ext_vector_type(4)));
    typedef Four FourAnywhere __attribute__((aligned(4)));
    constexpr int LOADS = EACH / 4, KS = kPlainK / 4, RS = SIDE / 4;
    struct Part {
        Four v[LOADS];
    };
    auto row_of = [&](bool slow, int i) { return slow ? tid % RS * 4 : tid / KS + THREADS / KS * i; };
    auto k_of = [&](bool slow, int i) { return slow ? tid / RS + THREADS / RS * i : tid % KS * 4; };
    auto take = [&](Part &to, const float *from, int64_t ld, bool slow, int r0, int rows, int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int r = r0 + row_of(slow, i), k = k0 + k_of(slow, i);
            const int left = slow ? (k < p.k ? rows - r : 0) : p.k - k;
            const float *const at = slow ? from + (int64_t)k * ld + r : from + (int64_t)min(r, rows - 1) * ld + k;  // (copies of the last row are not stored)
            to.v[i] = Four{0.f, 0.f, 0.f, 0.f};
            if (left >= 4)
                to.v[i] = *reinterpret_cast<const FourAnywhere *>(at);
            else if (left > 0) {
                to.v[i][0] = at[0];
                if (left > 1) to.v[i][1] = at[1];
                if (left > 2) to.v[i][2] = at[2];
            }
        }
    };
    auto put = [&](float *to, const Part &from, bool slow) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) to[(row_of(slow, i) + (slow ? e : 0)) * LD + k_of(slow, i) + (slow ? 0 : e)] = from.v[i][e];
    };
    const int per_range = (p.k + kPlainK - 1) / kPlainK, steps = p.ranges * per_range, rounds = (steps + GROUPS - 1) / GROUPS;
    Part va, vb[NB];
    auto request = [&](int t) __attribute__((always_inline)) {
        const int range = t >= per_range, k0 = t < steps ? (t - range * per_range) * kPlainK : p.k;  // (beyond the end: zeros)
        take(va, (const float *)(range ? p.a[1] : p.a[0]), p.lda, A_SLOW, m0, p.m, k0);
#pragma unroll
        for (int b = 0; b < NB; b++) take(vb[b], (const float *)((NB == 2 ? b : range) ? p.b[1] : p.b[0]), p.ldb, B_SLOW, n0, p.n, k0);
    };
    if (rounds > 0) request(group);
    for (int i = 0; i < rounds; i++) {
        __syncthreads();
        put(sa, va, A_SLOW);
#pragma unroll
        for (int b = 0; b < NB; b++) put(sb + b * TILE, vb[b], B_SLOW);
        __syncthreads();
        if (i + 1 < rounds) request((i + 1) * GROUPS + group);
        const float *pa = sa + (wave / W * 32 + (lane & 31)) * LD + (lane >> 5), *pb = sb + (wave % W * 32 + (lane & 31)) * LD + (lane >> 5);
#pragma unroll
        for (int k = 0; k < kPlainK; k += 2)
#pragma unroll
            for (int b = 0; b < NB; b++) acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(pb[b * TILE + k], pa[k], acc[b], 0, 0, 0);
    }
    if (GROUPS > 1) {
        float *const join = reinterpret_cast<float *>(smem);  // [threads][17]: one group's sums at a time
        static_assert(GROUPS == 1 || THREADS * 17 * 4 <= plain_lds<KIND, W, GROUPS>(), "room for a group's sums");
#pragma unroll
        for (int b = 0; b < NB; b++)
            for (int g = 1; g < GROUPS; g++) {
                __syncthreads();
                if (group == g)
#pragma unroll
                    for (int e = 0; e < 16; e++) join[tid * 17 + e] = acc[b][e];
                __syncthreads();
                if (group == 0)
#pragma unroll
                    for (int e = 0; e < 16; e++) acc[b][e] += join[tid * 17 + e];
            }
        if (group > 0) return;
    }

    const int m = m0 + wave / W * 32 + (lane & 31);
    if (m >= p.m) return;
    auto finish = [&](auto act) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 16; e++) {
            const int n = n0 + wave % W * 32 + (lane >> 5) * 4 + 8 * (e >> 2) + (e & 3);
            if (n >= p.n) continue;
            const int64_t at = (int64_t)m * p.ldo + n;
            if (KIND == GATE) {
                const float u = acc[NB - 1][e];
                const Act f = activate<true, decltype(act)::value>(acc[0][e]);
                if (p.out[0]) {
                    ((float *)p.out[0])[at] = u * f.slope;
                    ((float *)p.out[1])[at] = f.value;
                }
                ((float *)p.out[2])[at] = f.value * u;
            } else if (KIND == DGATE) {
                ((float *)p.out[0])[at] = acc[0][e] * ((const float *)p.by_gate)[at];
                ((float *)p.out[1])[at] = acc[0][e] * ((const float *)p.by_up)[at];
            } else {
                ((float *)p.out[0])[at] = acc[0][e];
            }
        }
    };
    if constexpr (KIND == GATE)
        by_act(p.act, [&](auto act) __attribute__((always_inline)) { finish(act); });
    else
        finish(Constant<0>());
}

template <int KIND, bool A_SLOW, bool B_SLOW, int W, int GROUPS>
hdt_status_t launch_plain_as(const Product *of, int products, hipStream_t st)
{
    constexpr int SIDE = 32 * W, LDS = plain_lds<KIND, W, GROUPS>();
    PlainArgs a = {};
    for (int i = 0; i < 3; i++) {
        a.first[i] = ~0u;
        if (i >= products) continue;
        a.p[i] = of[i];
        a.first[i] = a.tiles;
        a.tiles += (unsigned)(((int64_t)of[i].m + SIDE - 1) / SIDE * (((int64_t)of[i].n + SIDE - 1) / SIDE));
    }
    const auto kernel = k_ffn_plain<KIND, A_SLOW, B_SLOW, W, GROUPS>;
    if (LDS > 65536) HDT_HIP_TRY(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
    hipLaunchKernelGGL(kernel, dim3(a.tiles), dim3(64 * W * W * GROUPS), LDS, st, a);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

template <int KIND, bool A_SLOW, bool B_SLOW>
hdt_status_t launch_plain(const Product *of, int products, hipStream_t st)
{
    int64_t tiles = 0;
    for (int i = 0; i < products; i++) tiles += plain_tiles({of[i].m, of[i].n});
    switch (plain_form(tiles)) {
    case PlainForm::kSmallDivided: return launch_plain_as<KIND, A_SLOW, B_SLOW, 1, 8>(of, products, st);
    case PlainForm::kDivided: return launch_plain_as<KIND, A_SLOW, B_SLOW, 2, 4>(of, products, st);
    default: return launch_plain_as<KIND, A_SLOW, B_SLOW, 2, 1>(of, products, st);
    }
}

}  // namespace hdt_ffn
