// The products of the gated feed-forward block in bf16, in large tiles.
//
// A workgroup of WM x WN waves makes a tile of BM x BN of C^T = B A^T, a wave MB x NB blocks of 32 x 32.  64 of k at a time go straight from
// memory to LDS, two stages of them.  A wave holds the operands of 16 of k in registers and those of the next 16 on their way, over the
// barrier between two stages too: the last products of a stage run while the first operands of the next arrive.
//
// C^T rather than C, and the rows of B (n) that an operand holds in the order 0-3, 8-11, 4-7, 12-15: a lane's sums are then eight
// consecutive n at a time of one m, which leave as 16 bytes, and what the epilogue multiplies them with comes as 16 bytes.
//
// LDS tiles.  Rows of "fast" operands: 128 bytes, 64 of k, whose 16-byte chunks are exchanged so that 16 consecutive rows read without a
// conflict (hdt_tile.h has the rule).  Rows of "slow" operands: one k, BM or BN values, read transposed; four consecutive k at the same
// 64 bytes are moved apart.
//
// Rows beyond m or n read the last one there is and are not stored; of k what is beyond the end is written as zeros, on both sides.
#pragma once

#include "hdt_ffn.h"
#include "hdt_tile.h"

namespace hdt_ffn {

using hdt_tile::dma16;
using hdt_tile::lds_addr;
using hdt_tile::wait_vmcnt;
using hdt_tile::wg_barrier;

constexpr int BK = 64;

// One product of a launch: tiles of C beginning at number `first`
struct TileProduct {
    const __bf16 *a[2], *b[2];  // GATE: b of the gate and of up; else the two ranges of k
    __bf16 *out[3];
    const __bf16 *by_gate, *by_up;
    int64_t lda, ldb, ldo;
    int m, n, tiles_m, tiles_n;  // GATE: n and its tiles count pairs of columns
    unsigned first;
};
struct TileArgs {
    TileProduct p[3];
    int products, k, ranges;    // k of a range
    int splits, per;            // the tiles of k are divided into `splits` pieces of `per`
    unsigned tiles;             // of all products
    float *parts;               // [tiles][splits][BM BN] where splits > 1
    hdt_tile::FastDiv chunk, by_split;
    int act, group;             // group: tiles along m that are taken side by side
};

template <int WM_, int WN_, int MB_, int NB_>
struct Shape {
    static constexpr int WM = WM_, WN = WN_, MB = MB_, NB = NB_, NW = WM * WN, THREADS = NW * 64;
    static constexpr int BM = WM * MB * 32, BN = WN * NB * 32;
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, STAGE = A_BYTES + B_BYTES, LDS = 2 * STAGE;
};

// One operand of R rows: how it comes to LDS, and how its blocks of 32 rows are read.  PERMUTED: in the order of the sums' rows.
template <int R, int NW, bool SLOW, bool PERMUTED>
struct Operand {
    static constexpr int CPR = SLOW ? R / 8 : 8;        // chunks of 16 bytes a row in LDS
    static constexpr int LOADS = R * 8 / 64 / NW;       // wave-level loads of a tile, for each wave
    static_assert(R * 8 % (64 * NW) == 0, "tile");

    static __device__ __forceinline__ int swizzle(int row)
    {
        if (!SLOW) return hdt_tile::swz<8>(row);
        return CPR % 16 == 0 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
    }
    // row and chunk (as in memory) of load i of this wave and lane
    static __device__ __forceinline__ void place(int i, int wave, int lane, int *row, int *chunk)
    {
        const int at = (i * NW + wave) * 64 + lane;
        *row = at / CPR;
        *chunk = (at % CPR) ^ swizzle(*row);
    }
    uint32_t off[LOADS];  // bytes from the tile's first row (fast) or column (slow)
    int64_t ld;

    // rows (fast) or columns (slow) first .. of `count`
    __device__ __forceinline__ void init(int64_t ld_, int first, int count, int wave, int lane)
    {
        ld = ld_;
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            int row, chunk;
            place(i, wave, lane, &row, &chunk);
            if (!SLOW)
                off[i] = (uint32_t)(min(first + row, count - 1) - first) * (uint32_t)(ld * 2) + chunk * 16;
            else
                off[i] = (uint32_t)row * (uint32_t)(ld * 2) + (uint32_t)(min(first + chunk * 8, count - 8) - first) * 2;
        }
    }
    // base: of the tile's first row or column, at k0
    __device__ __forceinline__ void request(const __bf16 *base, uint32_t to, int wave) const
    {
#pragma unroll
        for (int i = 0; i < LOADS; i++) dma16(base, off[i], to + (uint32_t)(i * NW + wave) * 1024u);
    }
    // the same with zeros from `left` of k on
    __device__ __forceinline__ void fill(const __bf16 *base, char *to, int left, int wave, int lane) const
    {
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            int row, chunk;
            place(i, wave, lane, &row, &chunk);
            bf16x8 v = zero_bf16x8();
            if ((SLOW ? row : chunk * 8) < left) v = *reinterpret_cast<const bf16x8 *>((const char *)base + off[i]);
            *reinterpret_cast<bf16x8 *>(to + (i * NW + wave) * 1024 + lane * 16) = v;
        }
    }

    // where a lane reads, at the first 16 of k; blocks: of 32 rows from `first` on
    uint32_t at[SLOW ? R / 32 : 1];  // (of which a wave uses its own blocks')
    template <int BLOCKS>
    __device__ __forceinline__ void reader(int first, int lane)
    {
        const int hf = lane >> 5;
        if (!SLOW) {
            const int i = lane & 31, r = PERMUTED ? (i & 0x13) | (i & 4) << 1 | (i & 8) >> 1 : i;
            at[0] = (uint32_t)((first + r) * 128 + ((hf ^ swizzle(r)) * 16));
        } else {
            const int t = lane & 15, piece = t & 3, k = hf * 8 + (t >> 2);
            const int low = 2 * ((lane >> 4) & 1) + (PERMUTED ? piece & 1 : piece >> 1), half = PERMUTED ? piece >> 1 : piece & 1;
#pragma unroll
            for (int b = 0; b < BLOCKS; b++) at[b] = (uint32_t)(k * CPR * 16 + (((first / 8 + b * 4 + low) ^ swizzle(k)) * 16) + half * 8);
        }
    }
    __device__ __forceinline__ bf16x8 read(const char *tile, int block, int step) const
    {
        if (!SLOW) return lds_read_8(tile + ((at[0] ^ (uint32_t)(step * 32)) + block * 4096));
        const char *p = tile + at[block] + step * 16 * CPR * 16;
        return lds_read_tr_8(p, p + 4 * CPR * 16);
    }
};

template <int KIND, typename S, bool A_SLOW, bool B_SLOW>
__global__ __launch_bounds__(S::THREADS, S::THREADS == 512 ? 2 : 2) void k_ffn_tile(TileArgs a)
{
    constexpr int MB = S::MB, NB = S::NB, NW = S::NW;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned item = hdt_tile::logical_block(blockIdx.x, a.chunk);
    if (item >= a.tiles * (unsigned)a.splits) return;
    const unsigned tile = a.splits > 1 ? a.by_split.div(item) : item, piece = item - tile * a.splits;
    int which = 0;
    if (a.products > 1) which = tile >= a.p[2].first ? 2 : tile >= a.p[1].first ? 1 : 0;
    const TileProduct &p = a.p[which];
    // `group` tiles along m, then the next n: what runs at the same time on an XCD shares operands in its L2
    const unsigned local = tile - p.first, wide = (unsigned)(a.group * p.tiles_n), g = local / wide, in = local - g * wide;
    const int rows = min(a.group, p.tiles_m - (int)g * a.group), tn = (int)(in / (unsigned)rows), tm = (int)g * a.group + (int)(in - (unsigned)tn * rows);
    const int m0 = tm * S::BM, n0 = tn * (KIND == GATE ? S::BN / 2 : S::BN);

    const int per_range = (a.k + BK - 1) / BK, whole = a.k / BK, t0 = (int)piece * a.per, t1 = min(t0 + a.per, a.ranges * per_range);
    Operand<S::BM, NW, A_SLOW, false> oa;
    Operand<S::BN, NW, B_SLOW, true> ob;
    oa.init(p.lda, m0, p.m, wave, lane);
    if (KIND != GATE) {
        ob.init(p.ldb, n0, p.n, wave, lane);
    } else {  // blocks of 32 columns of the gate and of up in turn
        ob.ld = p.ldb;
#pragma unroll
        for (int i = 0; i < ob.LOADS; i++) {
            int row, chunk;
            ob.place(i, wave, lane, &row, &chunk);
            const int n = min(n0 + (row >> 6) * 32 + (row & 31), p.n - 1) - n0;
            ob.off[i] = (uint32_t)n * (uint32_t)(p.ldb * 2) + chunk * 16;
        }
    }
    const int wm = wave / S::WN * MB * 32, wn = wave % S::WN * NB * 32;
    oa.template reader<MB>(wm, lane);
    ob.template reader<NB>(wn, lane);

    auto load = [&](int t, int stage) {
        const int range = t >= per_range, kt = t - range * per_range, k0 = kt * BK;
        const __bf16 *pa = (range ? p.a[1] : p.a[0]) + (A_SLOW ? (int64_t)k0 * p.lda + m0 : (int64_t)m0 * p.lda + k0);
        const __bf16 *pb = (range && KIND != GATE ? p.b[1] : p.b[0]) + (B_SLOW ? (int64_t)k0 * p.ldb + n0 : (int64_t)n0 * p.ldb + k0);
        char *to = smem + stage * S::STAGE;
        if (kt < whole) {
            oa.request(pa, lds_addr(to), wave);
            if (KIND != GATE) {
                ob.request(pb, lds_addr(to) + S::A_BYTES, wave);
            } else {
                const int64_t up = (p.b[1] - p.b[0]);
#pragma unroll
                for (int i = 0; i < ob.LOADS; i++) {
                    const int block = ((i * NW + wave) * 8) >> 5;  // (a load's eight rows are of one block)
                    dma16(pb + (block & 1 ? up : 0), ob.off[i], lds_addr(to) + S::A_BYTES + (uint32_t)(i * NW + wave) * 1024u);
                }
            }
        } else {
            const int left = a.k - k0;
            oa.fill(pa, to, left, wave, lane);
            if (KIND != GATE) {
                ob.fill(pb, to + S::A_BYTES, left, wave, lane);
            } else {
                const int64_t up = (p.b[1] - p.b[0]);
#pragma unroll
                for (int i = 0; i < ob.LOADS; i++) {
                    int row, chunk;
                    ob.place(i, wave, lane, &row, &chunk);
                    bf16x8 v = zero_bf16x8();
                    if (chunk * 8 < left) v = *reinterpret_cast<const bf16x8 *>((const char *)(pb + (row >> 5 & 1 ? up : 0)) + ob.off[i]);
                    *reinterpret_cast<bf16x8 *>(to + S::A_BYTES + (i * NW + wave) * 1024 + lane * 16) = v;
                }
            }
        }
    };

    f32x16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
        for (int j = 0; j < NB; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.f;

    struct Frags {
        bf16x8 a[MB], b[NB];
    } f[2];
    auto read = [&](Frags &to, int stage, int step) {
        const char *ta = smem + stage * S::STAGE, *tb = ta + S::A_BYTES;
#pragma unroll
        for (int i = 0; i < MB; i++) to.a[i] = oa.read(ta, i, step);
#pragma unroll
        for (int j = 0; j < NB; j++) to.b[j] = ob.read(tb, j, step);
    };
    auto multiply = [&](const Frags &x) {
#pragma unroll
        for (int i = 0; i < MB; i++)
#pragma unroll
            for (int j = 0; j < NB; j++) acc[i][j] = mfma_32x32x16(x.b[j], x.a[i], acc[i][j]);
    };
    if (t0 < t1) {
        load(t0, 0);
        wait_vmcnt<0>();
        wg_barrier();
        if (t0 + 1 < t1) load(t0 + 1, 1);
        read(f[0], 0, 0);
        int stage = 0;
        for (int t = t0; t < t1; t++, stage ^= 1) {
            read(f[1], stage, 1);
            multiply(f[0]);
            read(f[0], stage, 2);
            multiply(f[1]);
            read(f[1], stage, 3);
            multiply(f[0]);
            if (t + 1 < t1) {
                wait_vmcnt<0>();
                wg_barrier();
                if (t + 2 < t1) load(t + 2, stage);
                read(f[0], stage ^ 1, 0);
            }
            multiply(f[1]);
        }
    }

    // a lane's sums: row m of its block, columns of eight
    const int hf = lane >> 5;
    if (KIND == STORE && a.splits > 1) {
        float *part = a.parts + (size_t)item * S::BM * S::BN;
#pragma unroll
        for (int i = 0; i < MB; i++)
#pragma unroll
            for (int j = 0; j < NB; j++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    typedef __attribute__((ext_vector_type(4))) float f32x4;
                    const f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    *reinterpret_cast<f32x4 *>(part + ((size_t)((i * NB + j) * 4 + q) * S::THREADS + tid) * 4) = v;
                }
        return;
    }
#pragma unroll
    for (int i = 0; i < MB; i++) {
        const int m = m0 + wm + i * 32 + (lane & 31);
        if (m >= p.m) continue;
#pragma unroll
        for (int j = 0; j < (KIND == GATE ? NB / 2 : NB); j++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int n = n0 + (KIND == GATE ? wn / 2 : wn) + j * 32 + h * 16 + hf * 8;
                if (n >= p.n) continue;
                const int64_t at = (int64_t)m * p.ldo + n;
                if (KIND == GATE) {
                    bf16x8 vg, vu, vh;
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const float g = acc[i][2 * j][h * 8 + e], u = acc[i][2 * j + 1][h * 8 + e];
                        if (p.out[0]) {
                            const Act f = activate<true>(g, a.act);
                            vg[e] = (__bf16)(u * f.slope), vu[e] = (__bf16)f.value, vh[e] = (__bf16)(f.value * u);
                        } else {
                            vh[e] = (__bf16)(activate<false>(g, a.act).value * u);
                        }
                    }
                    if (p.out[0]) {
                        *reinterpret_cast<bf16x8 *>(p.out[0] + at) = vg;
                        *reinterpret_cast<bf16x8 *>(p.out[1] + at) = vu;
                    }
                    *reinterpret_cast<bf16x8 *>(p.out[2] + at) = vh;
                } else if (KIND == DGATE) {
                    const bf16x8 pg = *reinterpret_cast<const bf16x8 *>(p.by_gate + at), pu = *reinterpret_cast<const bf16x8 *>(p.by_up + at);
                    bf16x8 vg, vu;
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const float dh = acc[i][j][h * 8 + e];
                        vg[e] = (__bf16)(dh * (float)pg[e]), vu[e] = (__bf16)(dh * (float)pu[e]);
                    }
                    *reinterpret_cast<bf16x8 *>(p.out[0] + at) = vg;
                    *reinterpret_cast<bf16x8 *>(p.out[1] + at) = vu;
                } else {
                    *reinterpret_cast<bf16x8 *>(p.out[0] + at) = pack_bf16x8(acc[i][j], h * 8);
                }
            }
    }
}

// The pieces of k added up in order: a workgroup has one row of blocks of a tile.
template <typename S>
__global__ __launch_bounds__(S::THREADS) void k_ffn_join(TileArgs a)
{
    constexpr int MB = S::MB, NB = S::NB;
    typedef __attribute__((ext_vector_type(4))) float f32x4;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    const unsigned tile = blockIdx.x / MB;
    const int i = blockIdx.x % MB;
    int which = 0;
    if (a.products > 1) which = tile >= a.p[2].first ? 2 : tile >= a.p[1].first ? 1 : 0;
    const TileProduct &p = a.p[which];
    const unsigned local = tile - p.first, wide = (unsigned)(a.group * p.tiles_n), g = local / wide, in = local - g * wide;
    const int rows = min(a.group, p.tiles_m - (int)g * a.group), tn = (int)(in / (unsigned)rows), tm = (int)g * a.group + (int)(in - (unsigned)tn * rows);
    const int m = tm * S::BM + wave / S::WN * MB * 32 + i * 32 + (lane & 31), n0 = tn * S::BN + wave % S::WN * NB * 32;
    const float *part = a.parts + (size_t)tile * a.splits * S::BM * S::BN;
#pragma unroll
    for (int j = 0; j < NB; j++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll 4
            for (int s = 0; s < a.splits; s++) {
                const float *q = part + (size_t)s * S::BM * S::BN + ((size_t)((i * NB + j) * 4 + 2 * h) * S::THREADS + tid) * 4;
                const f32x4 x = *reinterpret_cast<const f32x4 *>(q), y = *reinterpret_cast<const f32x4 *>(q + (size_t)S::THREADS * 4);
#pragma unroll
                for (int e = 0; e < 4; e++) lo[e] += x[e], hi[e] += y[e];
            }
            const int n = n0 + j * 32 + h * 16 + hf * 8;
            if (m >= p.m || n >= p.n) continue;
            bf16x8 v;
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = (__bf16)lo[e], v[4 + e] = (__bf16)hi[e];
            *reinterpret_cast<bf16x8 *>(p.out[0] + (int64_t)m * p.ldo + n) = v;
        }
}

}  // namespace hdt_ffn
