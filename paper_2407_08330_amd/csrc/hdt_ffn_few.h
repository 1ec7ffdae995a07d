// The forward products of the gated feed-forward block for few rows, in bf16: reading the weights is what cannot be saved.
//
// A workgroup makes 16 rows of weights' sums with 16, 32 or 64 rows of x, 16 x 16 blocks of them by matrix instructions: eight columns of the gate and the
// same eight of up, or 16 (8) columns of the last product.  Its waves divide k, 64 at a time, and join in LDS in a fixed order.  A load takes 128 bytes of eight
// rows, which LDS of the wave's own turns into the instructions' operands.  (Loaded as the instructions take them, 16 neighbouring lanes meet 16 lines, and a
// compute unit gets 16 bytes a clock: 32 rows of 1024 x 2816 17.0 us for 9.2, 64 rows of 768 x 2048 17.3 for 8.7.)  Kernels: 32 rows of 1024 x 2816 5.6 and 4.7 us
// (17 MB of weights are 3.4), one row of 768 x 2048 3.4 and 3.7 (9.4 MB, 1.8): a load's latency, a join in LDS.
#pragma once

#include "hdt_ffn_tile.h"

namespace hdt_ffn {

// BLOCKS: of 16 rows of x.  GATE: weights p.b[0], p.b[1]; else p.b[0].
template <int KIND, int WAVES, int BLOCKS, int COLS, bool EVEN>
__global__ __launch_bounds__(WAVES * 64) void k_ffn_few(Product p)
{
    constexpr int WEIGHTS = KIND == GATE ? 16 : COLS, ROWS = WEIGHTS + 16 * BLOCKS, LOADS = ROWS / 8, FIRST = WEIGHTS / 8;
    constexpr int CHUNKS = BLOCKS == 1 ? 4 : BLOCKS == 2 ? 3 : 2;  // of 64 of k in flight: as many as registers take
    constexpr int kStage = WAVES * ROWS * 128, kJoin = WAVES * BLOCKS * 16 * 17 * 4;
    __shared__ __attribute__((aligned(16))) char room[kStage > kJoin ? kStage : kJoin];
    float(*lds)[BLOCKS][16][17] = (float(*)[BLOCKS][16][17])room;  // [wave][..][row of x][sum]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15;
    const int n0 = blockIdx.x * COLS, m0 = blockIdx.y * (BLOCKS * 16);
    // load j: 128 bytes of eight rows, of the weights (j < FIRST) or x
    const __bf16 *from[LOADS];
    const int piece = lane & 7;
#pragma unroll
    for (int j = 0; j < LOADS; j++) {
        const int row = (j < FIRST ? j : j - FIRST) * 8 + (lane >> 3);
        if (j < FIRST)
            from[j] = (const __bf16 *)(KIND == GATE && j == 1 ? p.b[1] : p.b[0]) + (int64_t)min(n0 + (KIND == GATE ? row & 7 : row), p.n - 1) * p.ldb;
        else
            from[j] = (const __bf16 *)p.a[0] + (int64_t)min(m0 + row, p.m - 1) * p.lda;
        from[j] += piece * 8;
    }
    char *const mine = room + wave * (ROWS * 128);
    // row i's piece q is at q ^ (i / 2 mod 8): 16 lanes that read a piece of 16 rows, or write two rows, meet every bank once
    char *const put = mine + (lane >> 3) * 128;
    const int turn = lane >> 4;
    f32x4 acc[BLOCKS] = {};
    bf16x8 v[CHUNKS][LOADS];
    auto load = [&](int u, int k) __attribute__((always_inline)) {
        const int left = p.k - k - piece * 8;
#pragma unroll
        for (int j = 0; j < LOADS; j++) {
            v[u][j] = zero_bf16x8();
            if (left > 0) v[u][j] = load_chunk<EVEN>(from[j] + k, left);
        }
    };
    constexpr int STEP = WAVES * 64;
    constexpr bool ROLLING = BLOCKS <= 2;  // a chunk's registers take the next one as soon as it is in LDS (with four blocks that spills)
    if (ROLLING)
#pragma unroll
        for (int u = 0; u < CHUNKS; u++) load(u, wave * 64 + u * STEP);
    for (int k0 = wave * 64; k0 < p.k; k0 += STEP * CHUNKS) {
        if (!ROLLING)
#pragma unroll
            for (int u = 0; u < CHUNKS; u++) load(u, k0 + u * STEP);
#pragma unroll
        for (int u = 0; u < CHUNKS; u++) {
            if (k0 + u * STEP >= p.k) break;
#pragma unroll
            for (int j = 0; j < LOADS; j++) *(bf16x8 *)(put + j * 1024 + (piece ^ ((j < FIRST ? j : j - FIRST) % 2 * 4 + turn)) * 16) = v[u][j];
            if (ROLLING && k0 + (u + CHUNKS) * STEP < p.k) load(u, k0 + (u + CHUNKS) * STEP);
            hdt_lanes::wave_lds_barrier();
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int q = (lane >> 4) + h * 4, i = r & (WEIGHTS - 1);
                const bf16x8 w = *(const bf16x8 *)(mine + i * 128 + (q ^ (i >> 1)) * 16);
                const char *const at = mine + WEIGHTS * 128 + r * 128 + (q ^ (r >> 1)) * 16;
#pragma unroll
                for (int b = 0; b < BLOCKS; b++) acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, *(const bf16x8 *)(at + b * 2048), acc[b], 0, 0, 0);
            }
            hdt_lanes::wave_lds_barrier();
        }
    }
    __syncthreads();  // the room is the join's now
    // lane: row of x r, sums (lane / 16) 4 + 0 .. 3
#pragma unroll
    for (int b = 0; b < BLOCKS; b++)
#pragma unroll
        for (int e = 0; e < 4; e++) lds[wave][b][r][(lane >> 4) * 4 + e] = acc[b][e];
    __syncthreads();
    for (int i = tid; i < BLOCKS * 16 * COLS; i += WAVES * 64) {
        const int m = i / COLS, c = i % COLS, n = n0 + c;
        if (m0 + m >= p.m || n >= p.n) continue;
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < WAVES; v++) {
            s[0] += lds[v][m >> 4][m & 15][c];
            if (KIND == GATE) s[1] += lds[v][m >> 4][m & 15][c + 8];
        }
        const int64_t at = (int64_t)(m0 + m) * p.ldo + n;
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

// Rows a workgroup: 16 where that is not more than a workgroup a compute unit, else 32, else 64 (the last product, 64 rows of 1024 x 2816: 16 rows each, 256
// workgroups, 4.2 us, 64 each 7.4; but 32 rows of 4096 x 11008: 16 each, 512 workgroups, 32 us, 32 each 23).  Up to 16 rows in the last product,
// where these are few workgroups: eight columns each (one row of 768 x 2048 6.4 -> 6.2 in all, but of 4096 x 11008 46 -> 49).
template <int KIND, bool EVEN>
void launch_few(const Product &p, hipStream_t st)
{
    constexpr int WAVES = KIND == GATE ? 8 : 16, COLS = KIND == GATE ? 8 : 16;
    const int groups = (p.m + 15) / 16, across = (p.n + COLS - 1) / COLS, most = std::max(256 / across, 1);
    auto launch = [&](auto kernel, int cols, int blocks) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((p.n + cols - 1) / cols), (unsigned)((groups + blocks - 1) / blocks)), dim3(WAVES * 64), 0, st, p);
    };
    if (KIND != GATE && groups == 1 && p.n <= 2048)
        launch(k_ffn_few<KIND, WAVES, 1, 8, EVEN>, 8, 1);
    else if (groups <= most)
        launch(k_ffn_few<KIND, WAVES, 1, COLS, EVEN>, COLS, 1);
    else if ((groups + 1) / 2 <= most)
        launch(k_ffn_few<KIND, WAVES, 2, COLS, EVEN>, COLS, 2);
    else
        launch(k_ffn_few<KIND, WAVES, 4, COLS, EVEN>, COLS, 4);
}

}  // namespace hdt_ffn
