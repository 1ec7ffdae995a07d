// The forward products of the gated feed-forward block for few rows, in bf16: what takes time is reading the weights.
//
// A workgroup makes 16 rows of weights' sums with all rows of x, 16 x 16 blocks of them by matrix instructions: eight columns of the gate and the
// same eight of up, or 16 columns of the last product.  Its waves divide k, 32 at a time, and join in LDS in a fixed order.  Operands go straight
// from memory to registers: a weight is read once, by one wave.  One row of 768 x 2048: 3.7 and 4.5 us, of which the 9.4 MB of weights are 1.8; 32 rows of
// 1024 x 2816: 8.3 and 9.8 (17 MB, and every workgroup reads all of x or H from the L2).
#pragma once

#include "hdt_ffn_tile.h"

namespace hdt_ffn {

// BLOCKS: of 16 rows of x.  GATE: weights p.b[0], p.b[1]; else p.b[0].
template <int KIND, int WAVES, int BLOCKS, bool EVEN>
__global__ __launch_bounds__(WAVES * 64) void k_ffn_few(Product p)
{
    constexpr int COLS = KIND == GATE ? 8 : 16, AHEAD = BLOCKS <= 2 ? 8 : 4;
    __shared__ float lds[WAVES][BLOCKS][16][17];  // [..][row of x][sum]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15;
    const int n0 = blockIdx.x * COLS;
    const int column = min(n0 + (KIND == GATE ? r & 7 : r), p.n - 1);
    const __bf16 *w = (const __bf16 *)(KIND == GATE && r >= 8 ? p.b[1] : p.b[0]) + (int64_t)column * p.ldb;
    const __bf16 *x[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; b++) x[b] = (const __bf16 *)p.a[0] + (int64_t)min(b * 16 + r, p.m - 1) * p.lda;
    f32x4 acc[BLOCKS] = {};
    for (int k0 = wave * 32; k0 < p.k; k0 += WAVES * 32 * AHEAD) {
        bf16x8 wv[AHEAD], xv[AHEAD][BLOCKS];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            const int k = k0 + u * WAVES * 32 + (lane >> 4) * 8, left = p.k - k;
            wv[u] = zero_bf16x8();
#pragma unroll
            for (int b = 0; b < BLOCKS; b++) xv[u][b] = zero_bf16x8();
            if (left > 0) {
                wv[u] = load_chunk<EVEN>(w + k, left);
#pragma unroll
                for (int b = 0; b < BLOCKS; b++) xv[u][b] = load_chunk<EVEN>(x[b] + k, left);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; u++)
#pragma unroll
            for (int b = 0; b < BLOCKS; b++) acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[u], xv[u][b], acc[b], 0, 0, 0);
    }
    // lane: row of x r, sums (lane / 16) 4 + 0 .. 3
#pragma unroll
    for (int b = 0; b < BLOCKS; b++)
#pragma unroll
        for (int e = 0; e < 4; e++) lds[wave][b][r][(lane >> 4) * 4 + e] = acc[b][e];
    __syncthreads();
    for (int i = tid; i < BLOCKS * 16 * COLS; i += WAVES * 64) {
        const int m = i / COLS, c = i % COLS, n = n0 + c;
        if (m >= p.m || n >= p.n) continue;
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < WAVES; v++) {
            s[0] += lds[v][m >> 4][m & 15][c];
            if (KIND == GATE) s[1] += lds[v][m >> 4][m & 15][c + 8];
        }
        const int64_t at = (int64_t)m * p.ldo + n;
        if (KIND == GATE) {
            Act f;
            by_act(p.act, [&](auto act) { f = activate<true, decltype(act)::value>(s[0]); });
            if (p.out[0]) {
                ((__bf16 *)p.out[0])[at] = (__bf16)(s[1] * f.slope);
                ((__bf16 *)p.out[1])[at] = (__bf16)f.value;
            }
            ((__bf16 *)p.out[2])[at] = (__bf16)(f.value * s[1]);
        } else {
            ((__bf16 *)p.out[0])[at] = (__bf16)s[0];
        }
    }
}

// most rows (us with events around each kernel, this way | in tiles: 8 rows of 1024 x 2816 16 | 37, 32 22 | 37, 64 32 | 38; of 768 x 2048 14 | 28, 17 | 28, 22 | 28)
constexpr int kFew = 64;

template <int KIND, bool EVEN>
void launch_few(const Product &p, hipStream_t st)
{
    constexpr int WAVES = KIND == GATE ? 8 : 16;
    const dim3 grid((unsigned)((p.n + (KIND == GATE ? 7 : 15)) / (KIND == GATE ? 8 : 16))), block(WAVES * 64);
    if (p.m <= 16)
        hipLaunchKernelGGL((k_ffn_few<KIND, WAVES, 1, EVEN>), grid, block, 0, st, p);
    else if (p.m <= 32)
        hipLaunchKernelGGL((k_ffn_few<KIND, WAVES, 2, EVEN>), grid, block, 0, st, p);
    else
        hipLaunchKernelGGL((k_ffn_few<KIND, WAVES, 4, EVEN>), grid, block, 0, st, p);
}

}  // namespace hdt_ffn
