// The products of the gated feed-forward block in bf16, in large tiles.
//
// A workgroup of WM x WN waves makes a tile of BM x BN of C^T = B A^T, a wave MB x NB blocks of 32 x 32.  BK of k at a time go straight from
// memory to LDS: 32 in tiles of 256 x 256, four stages of them, 64 in tiles of 128 x 128, two stages.  A wave holds the operands of 16 of k in registers and those of the next 16 on their way, over the
// barrier between two stages too: the last products of a stage run while the first operands of the next arrive.
//
// C^T rather than C, and the rows of B (n) that an operand holds in the order 0-3, 8-11, 4-7, 12-15: a lane's sums are then eight
// consecutive n at a time of one m, which leave as 16 bytes, and what the epilogue multiplies them with comes as 16 bytes.
//
// What bounds it: the direct loads.  At 32768 x 768 x 2048 the weights' gradients take 300 us (1.03 PFLOP/s) and dX 207 (1.0), without the loads 206
// and 174, with all of them from the L2 265 and 221; the matrix pipe alone would take 155 and 103.  Hence 256 x 256, the most a compute unit's
// registers hold, and tiles that run at the same time at the same place of k (dX 250 -> 203 us, the gradients 352 -> 298).  The loads are
// requested between the products of a step, three stages ahead (all of them behind the barrier, four stages of 32: dX 269 us, now 249 before the
// cuts).  Two workgroups a compute unit with tiles of 256 x 128 take 1.5 times the loads: gate 317-336 us against 306, gradients 394 against 328.
// The forward's gate product takes 217 us where H alone leaves and 293 where its derivatives leave too (402 MB), dG and dU 178 (537 MB in and out): stores and
// what comes from memory at a tile's end find the other waves at the same place, and the tile's walk is only 24 stages long.
//
// LDS tiles.  Rows of "fast" operands: BK of k, 64 or 128 bytes, whose 16-byte chunks are exchanged so that 16 consecutive rows read without a
// conflict (hdt_tile.h has the rule).  Rows of "slow" operands: one k, BM or BN values, read transposed; four consecutive k at the same
// 64 bytes are moved apart.
//
// Rows beyond m or n read the last one there is and are not stored; of k what is beyond the end is written as zeros, on both sides.  Where rows do
// not begin at multiples of 16 bytes (EVEN: they do) tiles come by way of registers, in pieces of any alignment.
#pragma once

#include "hdt_ffn.h"
#include "hdt_ffn_plan.h"
#include "hdt_rows.h"
#include "hdt_tile.h"

namespace hdt_ffn {

typedef __attribute__((ext_vector_type(4))) float f32x4;

using hdt_tile::dma16;
using hdt_tile::lds_addr;
using hdt_tile::wait_vmcnt;
using hdt_tile::wg_barrier;

// Eight values, `left` of which exist.  EVEN: all, at a multiple of 16 bytes; else at any element.  ONCE: what nothing soon to come reads
// again, past the caches: the derivatives that the forward keeps, there and in the backward (H then waits for its product in the last cache: down
// projection of 32768 rows 130 -> 119 us, dG and dU 195 -> 181).
template <bool EVEN, bool ONCE = false>
__device__ __forceinline__ bf16x8 load_chunk(const __bf16 *p, int left)
{
    if (EVEN && ONCE) return __builtin_nontemporal_load(reinterpret_cast<const bf16x8 *>(p));
    if (EVEN) return *reinterpret_cast<const bf16x8 *>(p);
    return hdt_rows::load8<false>(p, left);
}
template <bool EVEN, bool ONCE = false>
__device__ __forceinline__ void store_chunk(__bf16 *p, bf16x8 v, int left)
{
    if (EVEN) {
        if (ONCE)
            __builtin_nontemporal_store(v, reinterpret_cast<bf16x8 *>(p));
        else
            *reinterpret_cast<bf16x8 *>(p) = v;
        return;
    }
    hdt_rows::Eight e;
#pragma unroll
    for (int i = 0; i < 8; i++) e.x[i] = (float)v[i];
    hdt_rows::store8<false>(p, e, left);
}

// a pointer that is the same for the whole wave, in scalar registers
__device__ __forceinline__ const __bf16 *uniform(const __bf16 *p)
{
    const uint64_t u = (uint64_t)(uintptr_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
    return (const __bf16 *)(uintptr_t)((uint64_t)hi << 32 | lo);
}

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
    // The first `direct` tiles have a workgroup each (`spread` of them, a multiple of 8).  Each of the others is cut along k into `pieces` of `per` tiles of
    // k (the last of fewer where that is all), which workgroups make side by side, all tiles' first pieces before the second: what an XCD does at a time is at one place of k, and its
    // tiles share what they read.  What is left of the tiles, `rest` each, one behind the other, is divided among `sharers` further
    // workgroups, `per` each.  Sums that are not all of a tile go to `parts`, and k_ffn_join adds them up.
    unsigned direct, spread, tiles, piece_items, sharers;
    int pieces, per, rest;
    hdt_tile::FastDiv chunk;
    float *parts;               // [pieces][tiles - direct], then [number of a sharer + number of the tile], of [BM BN]
    int act, group;             // group: tiles along m that are taken side by side
};
// item number b of n (a multiple of 8) in an order in which an XCD, which gets every eighth workgroup, has consecutive items
__device__ __forceinline__ unsigned by_xcd(unsigned b, unsigned n) { return (b & 7u) * (n >> 3) + (b >> 3); }
struct TilePlace {
    int which, m, n;  // product, first row, tile of columns
};
template <typename S, bool SEVERAL>
__device__ __forceinline__ TilePlace place_of(const TileArgs &a, unsigned tile)
{
    TilePlace at = {0, 0, 0};
    if (SEVERAL && a.products > 1) at.which = tile >= a.p[2].first ? 2 : tile >= a.p[1].first ? 1 : 0;
    const TileProduct &p = a.p[at.which];
    // `group` tiles along m, then the next n: what runs at the same time on an XCD shares operands in its L2
    const unsigned local = tile - p.first, wide = (unsigned)(a.group * p.tiles_n), g = local / wide, in = local - g * wide;
    const int rows = min(a.group, p.tiles_m - (int)g * a.group);
    at.n = (int)(in / (unsigned)rows);
    at.m = ((int)g * a.group + (int)(in - (unsigned)at.n * rows)) * S::BM;
    return at;
}

// One operand of R rows: how it comes to LDS, and how its blocks of 32 rows are read.  PERMUTED: in the order of the sums' rows.
template <int R, int NW, int BK, bool SLOW, bool PERMUTED, bool EVEN>
struct Operand {
    static constexpr int CPR = (SLOW ? R : BK) / 8;     // chunks of 16 bytes a row in LDS
    static constexpr int LOADS = R * BK / 8 / 64 / NW;  // wave-level loads of a tile, for each wave
    static_assert(R * BK / 8 % (64 * NW) == 0, "tile");

    static __device__ __forceinline__ int swizzle(int row)
    {
        if (!SLOW) return CPR == 8 ? hdt_tile::swz<8>(row) : (row >> 2) & 3;
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
    int columns;          // slow: how many there are from the tile's first on

    // rows (fast) or columns (slow) first .. of `count`
    __device__ __forceinline__ void init(int64_t ld_, int first, int count, int wave, int lane)
    {
        ld = ld_;
        columns = count - first;
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            int row, chunk;
            place(i, wave, lane, &row, &chunk);
            if (!SLOW)
                off[i] = (uint32_t)(min(first + row, count - 1) - first) * (uint32_t)(ld * 2) + chunk * 16;
            else
                off[i] = (uint32_t)row * (uint32_t)(ld * 2) + (uint32_t)(EVEN ? min(first + chunk * 8, count - 8) - first : chunk * 8) * 2;
        }
    }
    // load i of the tile by way of registers, with zeros from `left` of k on.  base: of its first row or column; other: from there to the
    // second weight, whose rows are every second block of 32
    __device__ __forceinline__ bf16x8 take(int i, const __bf16 *base, int64_t other, int left, int wave, int lane) const
    {
        int row, chunk;
        place(i, wave, lane, &row, &chunk);
        const __bf16 *p = (const __bf16 *)((const char *)(base + (row >> 5 & 1 ? other : 0)) + off[i]);
        const int there = SLOW ? (row >= left ? 0 : EVEN ? 8 : columns - chunk * 8) : left - chunk * 8;
        return there > 0 ? load_chunk<EVEN>(p, there) : zero_bf16x8();
    }
    __device__ __forceinline__ void put(int i, bf16x8 v, char *to, int wave, int lane) const
    {
        *reinterpret_cast<bf16x8 *>(to + (i * NW + wave) * 1024 + lane * 16) = v;
    }

    // where a lane reads, at the first 16 of k; blocks: of 32 rows from `first` on
    uint32_t at[SLOW ? R / 32 : 1];  // (of which a wave uses its own blocks')
    template <int BLOCKS>
    __device__ __forceinline__ void reader(int first, int lane)
    {
        const int hf = lane >> 5;
        if (!SLOW) {
            const int i = lane & 31, r = PERMUTED ? (i & 0x13) | (i & 4) << 1 | (i & 8) >> 1 : i;
            at[0] = (uint32_t)((first + r) * (CPR * 16) + ((hf ^ swizzle(r)) * 16));
        } else {
            const int t = lane & 15, piece = t & 3, k = hf * 8 + (t >> 2);
            const int low = 2 * ((lane >> 4) & 1) + (PERMUTED ? piece & 1 : piece >> 1), half = PERMUTED ? piece >> 1 : piece & 1;
#pragma unroll
            for (int b = 0; b < BLOCKS; b++) at[b] = (uint32_t)(k * CPR * 16 + (((first / 8 + b * 4 + low) ^ swizzle(k)) * 16) + half * 8);
        }
    }
    __device__ __forceinline__ bf16x8 read(const char *tile, int block, int step) const
    {
        if (!SLOW) return lds_read_8(tile + ((at[0] ^ (uint32_t)(step * 32)) + block * (32 * CPR * 16)));
        const char *p = tile + at[block] + step * 16 * CPR * 16;
        return lds_read_tr_8(p, p + 4 * CPR * 16);
    }
};

// Where chunk c of row r of a block row of results is, rows of CH chunks of 16 bytes: a chunk of 16 consecutive rows, and the chunks of a row,
// without a conflict.
template <int CH>
__device__ __forceinline__ int result_at(int r, int c)
{
    return (r * CH + (CH % 16 == 0 ? c ^ (r & 15) : CH == 8 ? c ^ hdt_tile::swz<8>(r) : c ^ ((r >> 1) & 7))) * 16;
}

// tiles of k t0 .. t1 - 1 of a tile.  PART: not all of it, and its sums go to `part`
template <int KIND, typename S, bool A_SLOW, bool B_SLOW, bool EVEN, bool PART>
__device__ __forceinline__ void make_tile(const TileArgs &a, char *smem, unsigned tile, int t0, int t1, float *part)
{
    constexpr int MB = S::MB, NB = S::NB, NW = S::NW, BK = S::BK;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const TilePlace at = place_of<S, KIND == STORE>(a, tile);
    const TileProduct &p = a.p[at.which];
    const int m0 = at.m, n0 = at.n * (KIND == GATE ? S::BN / 2 : S::BN);

    const int per_range = (a.k + BK - 1) / BK, whole = a.k / BK;
    Operand<S::BM, NW, BK, A_SLOW, false, EVEN> oa;
    Operand<S::BN, NW, BK, B_SLOW, true, EVEN> ob;
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

    auto is_whole = [&](int t) { return EVEN && (t >= per_range ? t - per_range : t) < whole; };
    struct From {
        const __bf16 *a, *b;
        int left;  // of k
    };
    const int64_t up = KIND == GATE ? p.b[1] - p.b[0] : 0;
    auto from = [&](int t) {
        const int range = t >= per_range, k0 = (t - range * per_range) * BK;
        return From{(range ? p.a[1] : p.a[0]) + (A_SLOW ? (int64_t)k0 * p.lda + m0 : (int64_t)m0 * p.lda + k0),
                    (range && KIND != GATE ? p.b[1] : p.b[0]) + (B_SLOW ? (int64_t)k0 * p.ldb + n0 : (int64_t)n0 * p.ldb + k0), a.k - k0};
    };
    // load number i of a whole tile, of A's and then of B's
    auto request = [&](const From &f, int stage, int i) __attribute__((always_inline)) {
        const uint32_t to = lds_addr(smem) + (uint32_t)(stage * S::STAGE);
        if (i < oa.LOADS) {
            dma16(uniform(f.a), oa.off[i], __builtin_amdgcn_readfirstlane(to + (uint32_t)(i * NW + wave) * 1024u));
        } else {
            const int j = i - oa.LOADS, block = (j * NW + wave) * (512 / BK) >> 5;  // GATE: a load's rows are of one block
            dma16(uniform(f.b + (KIND == GATE && (block & 1) ? up : 0)), ob.off[j],
                  __builtin_amdgcn_readfirstlane(to + S::A_BYTES + (uint32_t)(j * NW + wave) * 1024u));
        }
    };
    // a tile by way of registers: the last of k where it is not whole, and every tile where rows do not begin at multiples of 16 bytes
    bf16x8 held[S::LOADS];
    auto take = [&](const From &f) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < S::LOADS; i++) held[i] = i < oa.LOADS ? oa.take(i, f.a, 0, f.left, wave, lane) : ob.take(i - oa.LOADS, f.b, up, f.left, wave, lane);
    };
    auto put = [&](int stage) __attribute__((always_inline)) {
        char *to = smem + stage * S::STAGE;
#pragma unroll
        for (int i = 0; i < S::LOADS; i++) i < oa.LOADS ? oa.put(i, held[i], to, wave, lane) : ob.put(i - oa.LOADS, held[i], to + S::A_BYTES, wave, lane);
    };
    auto load = [&](int t, int stage) {
        const From f = from(t);
        if (is_whole(t)) {
#pragma unroll
            for (int i = 0; i < S::LOADS; i++) request(f, stage, i);
        } else {
            take(f);
            put(stage);
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
    // the products of one step, rows of blocks one after the other; between them between(i)
    auto multiply = [&](const Frags &x, auto between) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MB; i++) {
#pragma unroll
            for (int j = 0; j < NB; j++) acc[i][j] = mfma_32x32x16(x.b[j], x.a[i], acc[i][j]);
            between(i);
        }
    };
    // a stage is requested STAGES - 1 ahead; before it is read, those behind it may still be on their way
    auto arrived = [&](int t) {  // tile t has, for this wave
        if (!EVEN) return;
        constexpr int MORE = (S::STAGES - 2) * S::LOADS;
        bool direct = t + S::STAGES - 2 < t1;
#pragma unroll
        for (int u = 1; u < S::STAGES - 1; u++) direct = direct && is_whole(t + u);
        if (direct)
            wait_vmcnt<MORE>();
        else
            wait_vmcnt<0>();
    };
    if (t0 < t1) {
#pragma unroll
        for (int u = 0; u < S::STAGES - 1; u++)
            if (t0 + u < t1) load(t0 + u, u);
        arrived(t0);
        wg_barrier();
        read(f[0], 0, 0);
        int stage = 0, before = S::STAGES - 1;
        for (int t = t0; t < t1; t++) {
            const int next = stage + 1 == S::STAGES ? 0 : stage + 1, ahead = t + S::STAGES - 1;
            const From fr = from(min(ahead, t1 - 1));
            const bool direct = ahead < t1 && is_whole(ahead);
            if (ahead < t1 && !direct) {
                take(fr);
                if (EVEN) put(before);
            }
#pragma unroll
            for (int s = 0; s < S::STEPS; s++) {
                if (s + 1 < S::STEPS) {
                    read(f[(s + 1) & 1], stage, s + 1);
                } else if (t + 1 < t1) {
                    if (!EVEN && ahead < t1) put(before);
                    arrived(t + 1);
                    wg_barrier();
                    read(f[0], next, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                multiply(f[s & 1], [&](int i) __attribute__((always_inline)) {
                    if (s == 0 && direct) {
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int q = i * S::LOADS / MB; q < (i + 1) * S::LOADS / MB; q++) request(fr, before, q);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                });
                __builtin_amdgcn_sched_barrier(0);
            }
            before = stage;
            stage = next;
        }
    }

    // a lane's sums: row m of its block, columns of eight
    const int hf = lane >> 5;
    if constexpr (PART) {
#pragma unroll
        for (int i = 0; i < MB; i++)
#pragma unroll
            for (int j = 0; j < NB; j++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    *reinterpret_cast<f32x4 *>(part + ((size_t)((i * NB + j) * 4 + q) * S::THREADS + tid) * 4) = v;
                }
        return;
    }
    // Results leave by LDS, block row by block row of all waves, so that a wave stores whole rows of the tile: by itself it has 32 or 64
    // columns of 32 rows, and as many requests of a piece of a row each (dG and dU 265 -> 204 us).
    wg_barrier();  // (the stages are no longer read)
    constexpr int GROUP = S::WM * 32;  // rows of a block row
    auto row_of = [&](int r, int i) { return m0 + (r >> 5) * MB * 32 + i * 32 + (r & 31); };
    const int my_row = wave / S::WN * 32 + (lane & 31);
    if constexpr (KIND != DGATE) {
        constexpr int OUTS = KIND == GATE ? 3 : 1, COLS = KIND == GATE ? NB / 2 : NB, WIDE = KIND == GATE ? S::BN / 2 : S::BN, CH = WIDE / 8;
        constexpr int BUFFER = GROUP * WIDE * 2;  // of one result
        static_assert(2 * OUTS * BUFFER <= S::LDS, "room for two block rows");
        auto finish = [&](auto act, auto keep) __attribute__((always_inline)) {
            constexpr int FIRST = KIND == GATE && !decltype(keep)::value ? 2 : 0;
#pragma unroll
            for (int i = 0; i < MB; i++) {
                char *buf = smem + (i & 1) * OUTS * BUFFER;
#pragma unroll
                for (int c = 0; c < COLS * 2; c++) {
                    const int j = c >> 1, h = c & 1, to = result_at<CH>(my_row, wave % S::WN * (COLS * 4) + j * 4 + h * 2 + hf);
                    if constexpr (KIND == GATE) {
                        bf16x8 v[3];
#pragma unroll
                        for (int e = 0; e < 8; e++) {
                            const float g = acc[i][2 * j][h * 8 + e], u = acc[i][2 * j + 1][h * 8 + e];
                            const Act f = activate<decltype(keep)::value, decltype(act)::value>(g);
                            v[0][e] = (__bf16)(u * f.slope), v[1][e] = (__bf16)f.value, v[2][e] = (__bf16)(f.value * u);
                        }
#pragma unroll
                        for (int o = FIRST; o < OUTS; o++) *reinterpret_cast<bf16x8 *>(buf + o * BUFFER + to) = v[o];
                    } else {
                        *reinterpret_cast<bf16x8 *>(buf + to) = pack_bf16x8(acc[i][j], h * 8);
                    }
                }
                wg_barrier();
#pragma unroll
                for (int o = FIRST; o < OUTS; o++)
#pragma unroll
                    for (int q = 0; q < GROUP * CH / S::THREADS; q++) {
                        const int r = (q * S::THREADS + tid) / CH, chunk = (q * S::THREADS + tid) % CH, m = row_of(r, i), n = n0 + chunk * 8;
                        const bf16x8 v = *reinterpret_cast<const bf16x8 *>(buf + o * BUFFER + result_at<CH>(r, chunk));
                        __bf16 *const to = p.out[o] + (int64_t)m * p.ldo + n;
                        if (m < p.m && n < p.n) KIND == GATE && o < 2 ? store_chunk<EVEN, true>(to, v, p.n - n) : store_chunk<EVEN>(to, v, p.n - n);
                    }
            }
        };
        if constexpr (KIND == GATE)
            by_act(a.act, [&](auto act) __attribute__((always_inline)) {
                if (p.out[0])
                    finish(act, Constant<1>());
                else
                    finish(act, Constant<0>());
            });
        else
            finish(Constant<0>(), Constant<0>());
    } else {
        // dH goes through LDS in fp32
        constexpr int CH = S::BN / 8, BUFFER = GROUP * S::BN * 4, EACH = GROUP * CH / S::THREADS;
        static_assert(2 * BUFFER <= S::LDS, "room for two block rows");
        struct Factors {
            bf16x8 g[EACH], u[EACH];
        } with, next;
        auto factors = [&](Factors &to, int i) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < EACH; q++) {
                const int r = (q * S::THREADS + tid) / CH, chunk = (q * S::THREADS + tid) % CH;
                const int n = n0 + chunk * 8;
                const int64_t at = (int64_t)min(row_of(r, i), p.m - 1) * p.ldo + (EVEN ? min(n, p.n - 8) : n);
                bf16x8 g = zero_bf16x8(), u = g;
                if (EVEN || n < p.n) g = load_chunk<EVEN, true>(p.by_gate + at, p.n - n), u = load_chunk<EVEN, true>(p.by_up + at, p.n - n);
                to.g[q] = g, to.u[q] = u;
            }
        };
        factors(next, 0);
#pragma unroll
        for (int i = 0; i < MB; i++) {
            char *buf = smem + (i & 1) * BUFFER;
#pragma unroll
            for (int c = 0; c < NB * 4; c++)  // four columns
                *reinterpret_cast<f32x4 *>(buf + result_at<CH * 2>(my_row, wave % S::WN * (NB * 8) + (c >> 2) * 8 + (c >> 1 & 1) * 4 + hf * 2 + (c & 1))) =
                    f32x4{acc[i][c >> 2][(c & 3) * 4], acc[i][c >> 2][(c & 3) * 4 + 1], acc[i][c >> 2][(c & 3) * 4 + 2], acc[i][c >> 2][(c & 3) * 4 + 3]};
            with = next;
            if (i + 1 < MB) factors(next, i + 1);
            wg_barrier();
#pragma unroll
            for (int q = 0; q < EACH; q++) {
                const int r = (q * S::THREADS + tid) / CH, chunk = (q * S::THREADS + tid) % CH, m = row_of(r, i), n = n0 + chunk * 8;
                bf16x8 vg, vu;
#pragma unroll
                for (int half = 0; half < 2; half++) {
                    const f32x4 dh = *reinterpret_cast<const f32x4 *>(buf + result_at<CH * 2>(r, chunk * 2 + half));
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        vg[half * 4 + e] = (__bf16)(dh[e] * (float)with.g[q][half * 4 + e]);
                        vu[half * 4 + e] = (__bf16)(dh[e] * (float)with.u[q][half * 4 + e]);
                    }
                }
                if (m < p.m && n < p.n) {
                    store_chunk<EVEN>(p.out[0] + (int64_t)m * p.ldo + n, vg, p.n - n);
                    store_chunk<EVEN>(p.out[1] + (int64_t)m * p.ldo + n, vu, p.n - n);
                }
            }
        }
    }
}

template <int KIND, typename S, bool A_SLOW, bool B_SLOW, bool EVEN>
__global__ __launch_bounds__(S::THREADS, 2) void k_ffn_tile(TileArgs a)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int k_tiles = a.ranges * ((a.k + S::BK - 1) / S::BK);
    if (KIND != STORE || blockIdx.x < a.spread) {
        const unsigned tile = hdt_tile::logical_block(blockIdx.x, a.chunk);
        if (tile < a.direct) make_tile<KIND, S, A_SLOW, B_SLOW, EVEN, false>(a, smem, tile, 0, k_tiles, nullptr);
        return;
    }
    if constexpr (KIND == STORE) {
        const unsigned cut = a.tiles - a.direct, block = blockIdx.x - a.spread;
        constexpr size_t SIZE = (size_t)S::BM * S::BN;
        if (block < a.piece_items) {
            const unsigned item = by_xcd(block, a.piece_items), piece = item / cut, tile = item - piece * cut;
            if (piece < (unsigned)a.pieces)
                make_tile<KIND, S, A_SLOW, B_SLOW, EVEN, true>(a, smem, a.direct + tile, piece * a.per, min((int)(piece + 1) * a.per, k_tiles), a.parts + item * SIZE);
            return;
        }
        const unsigned me = by_xcd(block - a.piece_items, a.sharers);
        int64_t at = (int64_t)me * a.per;
        const int64_t end = min(at + a.per, (int64_t)cut * a.rest);
        while (at < end) {
            const int64_t tile = at / a.rest;
            const int t0 = (int)(at - tile * a.rest), t1 = (int)min((int64_t)a.rest, t0 + (end - at)), from = a.pieces * a.per;
            wg_barrier();  // (the LDS of the tile before is no longer read)
            make_tile<KIND, S, A_SLOW, B_SLOW, EVEN, true>(a, smem, a.direct + (unsigned)tile, from + t0, from + t1,
                                                           a.parts + ((size_t)a.pieces * cut + me + tile) * SIZE);
            at += t1 - t0;
        }
    }
}

// The parts of the tiles that were cut, added up in the order of k: a workgroup has a block of each of a tile's waves.
template <typename S, bool EVEN>
__global__ __launch_bounds__(S::THREADS) void k_ffn_join(TileArgs a)
{
    constexpr int MB = S::MB, NB = S::NB;
    constexpr size_t SIZE = (size_t)S::BM * S::BN;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    const unsigned tile = blockIdx.x / (MB * NB), cut = a.tiles - a.direct;
    const int i = blockIdx.x / NB % MB, j = blockIdx.x % NB;
    const int64_t first = (int64_t)tile * a.rest / a.per, last = a.rest ? ((int64_t)(tile + 1) * a.rest - 1) / a.per : first - 1;
    const int parts = a.pieces + (int)(last - first + 1);  // two or more
    const TilePlace at = place_of<S, true>(a, a.direct + tile);
    const TileProduct &p = a.p[at.which];
    const int m = at.m + wave / S::WN * MB * 32 + i * 32 + (lane & 31), n0 = at.n * S::BN + wave % S::WN * NB * 32;
    f32x4 sum[4] = {};
#pragma unroll 4
    for (int s = 0; s < parts; s++) {
        const size_t slot = s < a.pieces ? (size_t)s * cut + tile : (size_t)a.pieces * cut + (size_t)(first + s - a.pieces) + tile;
        const float *q = a.parts + slot * SIZE + ((size_t)((i * NB + j) * 4) * S::THREADS + tid) * 4;
        f32x4 x[4];
#pragma unroll
        for (int h = 0; h < 4; h++) x[h] = *reinterpret_cast<const f32x4 *>(q + (size_t)h * S::THREADS * 4);
#pragma unroll
        for (int h = 0; h < 4; h++)
#pragma unroll
            for (int e = 0; e < 4; e++) sum[h][e] += x[h][e];
    }
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int n = n0 + j * 32 + h * 16 + hf * 8;
        if (m >= p.m || n >= p.n) continue;
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (__bf16)sum[2 * h + (e >> 2)][e & 3];
        store_chunk<EVEN>(p.out[0] + (int64_t)m * p.ldo + n, v, p.n - n);
    }
}

}  // namespace hdt_ffn
