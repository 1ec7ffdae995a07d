// Backward pass of self-attention with a relative position bias:
//     D_i = sum_c dO_ic O_ic,  P = exp(S - LSE),  dP = dO V^T,  dS = P o (dP - D),
//     dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO,  dbias[u][h] = sum of dS over the pairs of head h in bucket u.
// No atomics on memory: the results do not depend on the order in which workgroups run.
//
// Three launches.  k_rel_rows: D and the other numbers of a row, and every head's bias by distance.  k_rel_bwd: workgroups of two kinds, a
// tile of query rows that walks the keys (dQ, sums of dS by distance) and a tile of keys that walks the queries of every head that shares
// them (dK, dV), so that each result has one owner; S and dP are computed in both, seven products in place of five, and
// no dQ in fp32 that is added up in memory, in an order that changes.  k_rel_dbias: the sums by distance added up, then by bucket.
//
// P and dS are rounded to bf16 as operands of their products (sums of dS by distance are taken before), and D is made of the rounded O that
// the forward wrote.  Against 64 bits, as shares of a gradient's norm: dv 0.0023, dq and dk 0.0024-0.0028 (the largest at 65 rows), dbias
// 0.0013-0.0036 (the largest both ways, where the errors of D add up in the far buckets), where rounding the result alone gives 0.0017.
//
// What bounds k_rel_bwd: with 128 columns, one wave a SIMD and its chain of LDS reads, products and exponentials: 32 heads x 4096, causal,
// 550-600 us, 0.80-0.87 PFLOP/s in seven products (two waves a SIMD with spilled registers 680-770); with 64 columns, 36 heads x 2047 both
// ways, ragged, 150 us.  Small calls are bound by the life of a workgroup, about 5 us in front of and behind its walk, which is why the
// first loads are single ones, results leave as whole rows and sums leave by distance: 48 heads x 512, 34 -> 25 us.
#include <algorithm>
#include <type_traits>

#include "hdt_rel.h"
#include "hdt_rel_args.h"

namespace {

using namespace hdt_rel;

// Four numbers of every row, four arrays of [batch][heads][n_pad]: n = -LSE / scale, minus infinity for a row without keys (its pairs then
// weigh exp2(-inf) = 0); -D; and n with the bias of far keys behind and ahead, over the scale too: what the contractions of a far block
// start from.  Every head's rows are filled up to whole tiles with rows without keys.
// The last workgroups write every head's bias by distance, which the tiles' workgroups then read at one load's latency instead of two.
constexpr int kRowsU = 2;  // rows a thread has in flight
__host__ __device__ __forceinline__ int table_row(int max_distance, bool causal) { return (table_length(max_distance, causal) + 3) & ~3; }
template <typename T, int D>
__global__ __launch_bounds__(256) void k_rel_rows(RelBwdArgs a, long long rows, unsigned row_groups, bool causal)
{
    if (blockIdx.x >= row_groups) {
        const int h = blockIdx.x - row_groups;
        fill_table(a.tables + (size_t)h * table_row(a.bias.max_distance, causal), a.bias, h, 1, causal, threadIdx.x, 256);
        return;
    }
    constexpr int LANES = D * (int)sizeof(T) / 16, PER = 256 / LANES, V = 16 / (int)sizeof(T);
    typedef typename Op<T>::Frag Frag;
    const int c = threadIdx.x % LANES;
    const long long r0 = (long long)blockIdx.x * (PER * kRowsU) + threadIdx.x / LANES;
    Frag o[kRowsU], g[kRowsU];
    float lse[kRowsU];
    int bh[kRowsU], ri[kRowsU];
#pragma unroll
    for (int u = 0; u < kRowsU; u++) {
        const long long r = min(r0 + u * PER, rows - 1);
        bh[u] = (int)(r / a.n_pad), ri[u] = (int)(r - (long long)bh[u] * a.n_pad);
        const int i = min(ri[u], a.n_q - 1), b = bh[u] / a.heads, h = bh[u] - b * a.heads;
        o[u] = *reinterpret_cast<const Frag *>((const T *)a.o + (size_t)b * a.so.batch + (size_t)h * a.so.head + (size_t)i * a.so.row + V * c);
        g[u] = *reinterpret_cast<const Frag *>((const T *)a.d_o + (size_t)b * a.sdo.batch + (size_t)h * a.sdo.head + (size_t)i * a.sdo.row + V * c);
        lse[u] = a.lse[(size_t)bh[u] * a.n_q + i];
    }
#pragma unroll
    for (int u = 0; u < kRowsU; u++) {
        float d = 0.f;
#pragma unroll
        for (int e = 0; e < V; e++) d = fmaf((float)o[u][e], (float)g[u][e], d);
#pragma unroll
        for (int m = 1; m < LANES; m <<= 1) d += __shfl_xor(d, m);
        const long long r = r0 + u * PER;
        if (c != 0 || r >= rows) continue;
        const int b = bh[u] / a.heads, h = bh[u] - b * a.heads;
        const Sample smp = sample_of(a.lengths, a.starts, b, a.n_q, a.n_kv);
        const bool dead = ri[u] < smp.lo || ri[u] >= smp.hi || minus_infinity(lse[u]);
        const float n = dead ? -INFINITY : -lse[u] * a.bias.inv_scale;
        a.row_scalars[r] = n;
        a.row_scalars[rows + r] = dead ? 0.f : -d;
        a.row_scalars[2 * rows + r] = n + bias_of(a.bias, -a.bias.max_distance, h);
        a.row_scalars[3 * rows + r] = n + bias_of(a.bias, a.bias.max_distance, h);
    }
}

// The sums of a 32 x 32 block's diagonals.  x[v] of lane (column q = 16 a + c, half f) belongs to key r(v) + 4 f, distance r + 4 f - q.
// Shifted down by s = r % 16 lanes within its row of 16, the values of distance 16 (r / 16 - a) + 4 f - c' stand at lane c' for c >= s, and
// those that run out of the row are the ones of distance 16 more, shifted up by 16 - s: so two additions with a shifted operand per
// register, without LDS, give d[j] at lane (a, c', f) = the sum over the block's pairs of distance 16 (j - a) + 4 f - c'.
// (As 16 LDS additions per block the near blocks took four times as long: 512 rows x 48 heads, the dQ kernel 41.0 us.)
template <int V>
__device__ __forceinline__ void add_diagonals(const f32x16 &x, float (&d)[3])
{
    if constexpr (V < 16) {
        constexpr int r = 8 * (V >> 2) + (V & 3), s = r & 15, j = r >> 4;
        const float value = x[V];  // (__builtin_bit_cast of x[V] itself would take the vector's first element)
        const int bits = __builtin_bit_cast(int, value);
        if constexpr (s == 0) {
            d[j] += value;
        } else {
            d[j] += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, bits, 0x100 | s, 0xf, 0xf, true));             // row_shl: lane c' takes c' + s
            d[j + 1] += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, bits, 0x110 | (16 - s), 0xf, 0xf, true));  // row_shr: c' + s - 16
        }
        add_diagonals<V + 1>(x, d);
    }
}

constexpr int kAheadRows = 3, kAheadCols = 2;  // operands on their way from LDS

// KS groups of NW waves take every KS-th tile of the walk, each through a ring of its own, and their sums are added up at the end
template <typename T, int D, int NW_, int KS_>
struct BwdShape {
    static constexpr int NW = NW_, KS = KS_, THREADS = NW * KS * 64, BM = 32 * NW, BN = sizeof(T) == 4 ? 32 : 64;
    static constexpr int RING = 2 * Pair<T, D, BN, NW>::STAGE, SCALARS = 2 * 4 * 256;  // two stages of four arrays of 64 floats
    // 64 rows at a time and constant stages, for more registers: 36 heads x 2047 x 64 213 -> 206 us forward and backward, 32 x 4096 x 128
    // 774 -> 743; with groups, whose walks are short, 50.4 -> 51.8 (48 heads x 512)
    static constexpr bool CONST = sizeof(T) == 2 && (D == 128 || KS == 1);
    static constexpr int KB = BN / 32, J = CONST ? KB : 1;  // blocks of a tile, and how many at a time
};

// bytes of LDS that the joining of the groups leaves in use
template <int NW, int KS, int BLOCKS>
constexpr int kJoined = (KS - 1) * NW * BLOCKS * 16 * 256;

// A wave's accumulators plus those of the same rows' waves in the other groups, in their order; false for those other waves
template <int NW, int KS, int BLOCKS>
__device__ __forceinline__ bool join_groups(char *smem, f32x16 (&acc)[BLOCKS], int grp, int wave, int lane)
{
    if constexpr (KS > 1) {
        float *const at = reinterpret_cast<float *>(smem) + lane;
        __syncthreads();
        if (grp > 0) {
            float *const to = at + ((grp - 1) * NW + wave) * BLOCKS * 16 * 64;
#pragma unroll
            for (int j = 0; j < BLOCKS; j++)
#pragma unroll
                for (int e = 0; e < 16; e++) to[(16 * j + e) * 64] = acc[j][e];
        }
        __syncthreads();
        if (grp > 0) return false;
#pragma unroll
        for (int k = 1; k < KS; k++) {
            const float *const from = at + ((k - 1) * NW + wave) * BLOCKS * 16 * 64;
#pragma unroll
            for (int j = 0; j < BLOCKS; j++)
#pragma unroll
                for (int e = 0; e < 16; e++) acc[j][e] += from[(16 * j + e) * 64];
        }
    }
    return true;
}

// a head's bias by distance into LDS
__device__ __forceinline__ void copy_table(float *lds, const RelBwdArgs &a, int h, int row, int tid, int threads)
{
    for (int x = 4 * tid; x < row; x += 4 * threads) *reinterpret_cast<f32x4 *>(lds + x) = *reinterpret_cast<const f32x4 *>(a.tables + (size_t)h * row + x);
}

// dQ of a tile of query rows, and the sums of its dS by distance
template <typename T, int D, int NW_, int KS_, bool CAUSAL>
__device__ __forceinline__ void dq_role(const RelBwdArgs &a, char *smem, int bh, int I)
{
    using S = BwdShape<T, D, NW_, KS_>;
    using RowsT = Rows<T, D>;
    constexpr int BM = S::BM, BN = S::BN, NW = S::NW, KS = S::KS, KB = S::KB, J = S::J;
    const int M = a.bias.max_distance, len = table_length(M, CAUSAL), line = table_row(M, CAUSAL);
    float *const tab = reinterpret_cast<float *>(smem + KS * S::RING), *const bins = tab + line;

    const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
    const int wave_all = __builtin_amdgcn_readfirstlane(tid >> 6), grp = KS > 1 ? wave_all / NW : 0, wave = wave_all - grp * NW;
    const int b = bh / a.heads, h = bh - b * a.heads;
    const Sample smp = sample_of(a.lengths, a.starts, b, a.n_q, a.n_kv);
    const int r0 = I * BM, first = max(r0, smp.lo), last = min(r0 + BM, smp.hi) - 1;
    const int row = r0 + wave * 32 + (lane & 31);
    const bool real = row >= first && row <= last;
    const int seen = first <= last ? (CAUSAL ? smp.start + last + 1 : smp.length) : 0, tiles = (seen + BN - 1) / BN;

    f32x16 acc[RowsT::BLOCKS];
#pragma unroll
    for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[j][e] = 0.f;
    float behind = 0.f, beyond = 0.f;                       // this lane's sums of dS in the far tiles
    float *const my_bins = bins + (wave_all * 2 + hf) * line;   // one copy for each half-wave: no two lanes of an instruction meet
    for (int x = 4 * tid; x < line * NW * KS * 2; x += 4 * S::THREADS) *reinterpret_cast<f32x4 *>(bins + x) = f32x4{0.f, 0.f, 0.f, 0.f};

    if (tiles > 0) {
        const int rc = min(max(row, first), last), pos = smp.start + rc;
        const int w0 = max(r0 + wave * 32, first), w1 = min(r0 + wave * 32 + 31, last), p0 = smp.start + w0, p1 = smp.start + w1;
        const size_t kvh = (size_t)(h / a.group);
        Pair<T, D, BN, NW> kv;
        kv.init((const T *)a.k + (size_t)b * a.sk.batch + kvh * a.sk.head, a.sk.row, (const T *)a.v + (size_t)b * a.sv.batch + kvh * a.sv.head,
                a.sv.row, smem + grp * S::RING, wave, lane);
        typename RowsT::Frag qf[RowsT::STEPS], dof[RowsT::STEPS];
        const char *qp = (const char *)((const T *)a.q + (size_t)b * a.sq.batch + (size_t)h * a.sq.head + (size_t)rc * a.sq.row);
        const char *dp = (const char *)((const T *)a.d_o + (size_t)b * a.sdo.batch + (size_t)h * a.sdo.head + (size_t)rc * a.sdo.row);
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) {
            qf[st] = *reinterpret_cast<const typename RowsT::Frag *>(qp + (2 * st + hf) * 16);
            dof[st] = *reinterpret_cast<const typename RowsT::Frag *>(dp + (2 * st + hf) * 16);
        }
        const size_t at_row = (size_t)bh * a.n_pad + rc, rows = (size_t)a.batch * a.heads * a.n_pad;
        const float nl = real ? a.row_scalars[at_row] * a.scale_log2 : -INFINITY, nd = a.row_scalars[rows + at_row];
        if (grp < tiles) kv.request(grp * BN, 0, seen - 1, 0);
        copy_table(tab, a, h, line, tid, S::THREADS);
        const float *const my_tab = tab + 4 * hf - pos + M + kPad;
        float *const diagonal = my_bins + 4 * hf - (lane & 31) - (smp.start + r0 + wave * 32) + M + kPad;  // of key 0 and j = 0
        const RowLane rl = row_lane<RowsT::CPR>(lane);
        const TrLane tl = tr_lane<RowsT::CPR>(lane);
        __syncthreads();
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) {
            settle(qf[st]);
            settle(dof[st]);
        }
        settle(nl);
        settle(nd);
        const float c_behind = tab[0] * a.scale_log2, c_ahead = tab[len - 1] * a.scale_log2;
        f32x16 nd16;  // what dP starts from
#pragma unroll
        for (int e = 0; e < 16; e++) nd16[e] = nd;

        auto tile = [&](int round, auto stage) {
            const int ST = stage, t = round * KS + grp;
            wait_vmcnt<0>();
            wg_barrier();
            if (t + KS < tiles) kv.request((t + KS) * BN, 0, seen - 1, 1 - ST);
            const char *sK = smem + grp * S::RING + ST * kv.STAGE, *sV = sK + kv.TILE;
            const Kind kind = kind_of<CAUSAL, BN>(t * BN, p0, p1, M, smp.length);
            if (kind == Kind::SKIP || w0 > w1 || (KS > 1 && t >= tiles)) return;  // (nor has a wave without real rows anything to do)
            const float off = nl + (kind == Kind::FAR_BEHIND ? c_behind : kind == Kind::FAR_AHEAD ? c_ahead : 0.f);
#pragma unroll
            for (int k2 = 0; k2 < KB; k2 += J) {
                const int k0 = t * BN + 32 * k2;
                f32x16 s[J], dp16[J];
                // S^T = K Q^T, then dP^T - D = V dO^T - D
                constexpr int N = J * RowsT::STEPS;
                auto read = [&](int i) { return RowsT::read(i < N ? sK : sV, rl, (k2 + i % J) * 32, i % N / J); };
                auto rows_ahead = ahead<2 * N, kAheadRows, typename RowsT::Frag>(read);
                if (kind == Kind::NEAR) {
#pragma unroll
                    for (int u = 0; u < J; u++)
#pragma unroll
                        for (int e = 0; e < 16; e++) s[u][e] = my_tab[k0 + 32 * u + 8 * (e >> 2) + (e & 3)];
                } else {
#pragma unroll
                    for (int u = 0; u < J; u++)
#pragma unroll
                        for (int e = 0; e < 16; e++) s[u][e] = 0.f;
                }
                rows_ahead.run([&](int i, typename RowsT::Frag f) {
                    if (i < N) s[i % J] = Op<T>::mma(f, qf[i / J], s[i % J]);
                    else dp16[i % J] = Op<T>::mma(f, dof[(i - N) / J], i < N + J ? nd16 : dp16[i % J]);
                });
                auto read_t = [&](int i) { return RowsT::wread(sK, tl, lane, (k2 + i / (RowsT::WSTEPS * RowsT::BLOCKS)) * 32, i % RowsT::BLOCKS, i / RowsT::BLOCKS % RowsT::WSTEPS); };
                auto k_ahead = ahead<J * RowsT::WSTEPS * RowsT::BLOCKS, kAheadCols, typename RowsT::WFrag>(read_t);
                if (!CAUSAL && k0 + 32 * J > smp.length) {
#pragma unroll
                    for (int u = 0; u < J; u++)
#pragma unroll
                        for (int e = 0; e < 16; e++)
                            s[u][e] = k0 + 32 * u + 4 * hf + 8 * (e >> 2) + (e & 3) < smp.length ? s[u][e] : -INFINITY;
                }
#pragma unroll
                for (int u = 0; u < J; u++)
#pragma unroll
                    for (int e = 0; e < 16; e++) s[u][e] = fast_exp2(fmaf(s[u][e], a.scale_log2, off)) * dp16[u][e];  // dS^T
                if (kind == Kind::NEAR) {
#pragma unroll
                    for (int u = 0; u < J; u++) {
                        float d[3] = {0.f, 0.f, 0.f};
                        add_diagonals<0>(s[u], d);
#pragma unroll
                        for (int j = 0; j < 3; j++)
                            __hip_atomic_fetch_add(diagonal + k0 + 32 * u + 16 * j, d[j], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                    }
                } else {
                    float sum = 0.f;
#pragma unroll
                    for (int u = 0; u < J; u++)
#pragma unroll
                        for (int e = 0; e < 16; e++) sum += s[u][e];
                    if (CAUSAL || kind == Kind::FAR_BEHIND) behind += sum;
                    else beyond += sum;
                }
                Weights<T> w[J];
#pragma unroll
                for (int u = 0; u < J; u++) w[u] = Weights<T>(s[u]);
                k_ahead.run([&](int i, typename RowsT::WFrag f) {
                    acc[i % RowsT::BLOCKS] = RowsT::wmma(f, w[i / (RowsT::WSTEPS * RowsT::BLOCKS)], i / RowsT::BLOCKS % RowsT::WSTEPS, acc[i % RowsT::BLOCKS]);
                });
            }
        };
        walk<S::CONST>((tiles + KS - 1) / KS, tile);  // (barriers are the whole workgroup's: every group takes the same number of rounds)
    }
    // the far tiles' sums join the bins at the two ends of the table
    behind = wave_sum(behind);
    if (!CAUSAL) beyond = wave_sum(beyond);
    __syncthreads();
    if (lane == 0) {
        bins[wave_all * 2 * line] += behind;
        if (!CAUSAL) bins[wave_all * 2 * line + len - 1] += beyond;
    }
    __syncthreads();  // (and the ring is free)
    float *const out = a.bins + ((size_t)(h * a.batch + b) * a.tiles_q + I) * line;
    for (int x = 4 * tid; x < line; x += 4 * S::THREADS) {
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < NW * KS * 2; u++) {
            const f32x4 y = *reinterpret_cast<const f32x4 *>(bins + u * line + x);
#pragma unroll
            for (int e = 0; e < 4; e++) sum[e] += y[e];
        }
        *reinterpret_cast<f32x4 *>(out + x) = sum;
    }
    if (!join_groups<NW, KS>(smem, acc, grp, wave, lane)) return;
    const int w0 = r0 + wave * 32;
    store_rows<T, D>(smem + kJoined<NW, KS, RowsT::BLOCKS> + wave * 32 * RowsT::ROWB, opaque(lane), acc, real, a.scale,
                     (T *)a.dq + (size_t)b * a.sdq.batch + (size_t)h * a.sdq.head + (size_t)w0 * a.sdq.row, a.sdq.row, a.n_q - w0);
}

// dK and dV of a tile of keys of one key head: over the query rows of every head that shares it
template <typename T, int D, int NW_, int KS_, bool CAUSAL>
__device__ __forceinline__ void dkv_role(const RelBwdArgs &a, char *smem, int bk, int J0)
{
    using S = BwdShape<T, D, NW_, KS_>;
    using RowsT = Rows<T, D>;
    constexpr int BM = S::BM, BN = S::BN, NW = S::NW, KS = S::KS, KB = S::KB, J = S::J;
    const int M = a.bias.max_distance, line = table_row(M, CAUSAL);
    float *const scal_all = reinterpret_cast<float *>(smem + KS * S::RING), *const tab = scal_all + KS * S::SCALARS / 4;

    const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
    const int wave_all = __builtin_amdgcn_readfirstlane(tid >> 6), grp = KS > 1 ? wave_all / NW : 0, wave = wave_all - grp * NW;
    float *const scal = scal_all + grp * (S::SCALARS / 4);
    const int b = bk / a.kv_heads, kvh = bk - b * a.kv_heads;
    const Sample smp = sample_of(a.lengths, a.starts, b, a.n_q, a.n_kv);
    const int key0 = J0 * BM, kw0 = key0 + wave * 32, key = kw0 + (lane & 31), kc = min(key, smp.length - 1);
    // the query rows that see a key of the tile
    const int from = CAUSAL ? max(smp.lo, key0 - smp.start) : smp.lo, tile0 = from / BN;
    const int tile1 = key0 < smp.length && from < smp.hi ? (smp.hi + BN - 1) / BN : tile0;

    f32x16 dk[RowsT::BLOCKS], dv[RowsT::BLOCKS];
#pragma unroll
    for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) dk[j][e] = dv[j][e] = 0.f;

    if (tile0 < tile1) {
        typename RowsT::Frag kf[RowsT::STEPS], vf[RowsT::STEPS];
        const char *kp = (const char *)((const T *)a.k + (size_t)b * a.sk.batch + (size_t)kvh * a.sk.head + (size_t)kc * a.sk.row);
        const char *vp = (const char *)((const T *)a.v + (size_t)b * a.sv.batch + (size_t)kvh * a.sv.head + (size_t)kc * a.sv.row);
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) {
            kf[st] = *reinterpret_cast<const typename RowsT::Frag *>(kp + (2 * st + hf) * 16);
            vf[st] = *reinterpret_cast<const typename RowsT::Frag *>(vp + (2 * st + hf) * 16);
        }
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) {
            settle(kf[st]);
            settle(vf[st]);
        }
        const RowLane rl = row_lane<RowsT::CPR>(lane);
        const TrLane tl = tr_lane<RowsT::CPR>(lane);
        const size_t rows = (size_t)a.batch * a.heads * a.n_pad;
        for (int h = kvh * a.group; h < (kvh + 1) * a.group; h++) {
            Pair<T, D, BN, NW> qd;
            qd.init((const T *)a.q + (size_t)b * a.sq.batch + (size_t)h * a.sq.head, a.sq.row,
                    (const T *)a.d_o + (size_t)b * a.sdo.batch + (size_t)h * a.sdo.head, a.sdo.row, smem + grp * S::RING, wave, lane);
            const float *rs = a.row_scalars + ((size_t)b * a.heads + h) * a.n_pad;
            auto request = [&](int t, int stage) {
                // (rows that are not real: copies, weighed zero)
                qd.request(t * BN, smp.lo, smp.hi - 1, stage);
                for (int w = wave; w < 4; w += NW)
                    dma4(rs + w * rows + t * BN, (uint32_t)(lane & (BN - 1)) * 4u, __builtin_amdgcn_readfirstlane(lds_addr(scal) + (stage * 4 + w) * 256));
            };
            __syncthreads();  // the head before is done with the table and the ring
            if (tile0 + grp < tile1) request(tile0 + grp, 0);
            copy_table(tab, a, h, line, tid, S::THREADS);
            __syncthreads();
            auto tile = [&](int round, auto stage) {
                const int ST = stage, t = tile0 + round * KS + grp;
                wait_vmcnt<0>();
                wg_barrier();
                if (t + KS < tile1) request(t + KS, 1 - ST);
                const char *sQ = smem + grp * S::RING + ST * qd.STAGE, *sDO = sQ + qd.TILE;
                const int q0 = smp.start + t * BN;  // position of the tile's first row
                // seen from the wave's 32 keys: the kinds of keys kw0 .. kw0 + 31 against positions q0 .. q0 + BN - 1
                const Kind kind = (CAUSAL && kw0 > q0 + BN - 1) || kw0 >= smp.length ? Kind::SKIP
                                  : kw0 + 31 - q0 <= -M                              ? Kind::FAR_BEHIND
                                  : !CAUSAL && kw0 - (q0 + BN - 1) >= M              ? Kind::FAR_AHEAD
                                                                                     : Kind::NEAR;
                if (kind == Kind::SKIP || (KS > 1 && t >= tile1)) return;
                const float *const st4 = scal + ST * 256, *const nd = st4 + 64;
                const float *const nl = kind == Kind::FAR_BEHIND ? st4 + 128 : kind == Kind::FAR_AHEAD ? st4 + 192 : st4;
#pragma unroll
                for (int q2 = 0; q2 < KB; q2 += J) {
                    f32x16 s[J], dp16[J];
                    // S = Q K^T, then dP - D = dO V^T - D
                    constexpr int N = J * RowsT::STEPS;
                    auto read = [&](int i) { return RowsT::read(i < N ? sQ : sDO, rl, (q2 + i % J) * 32, i % N / J); };
                    auto rows_ahead = ahead<2 * N, kAheadRows, typename RowsT::Frag>(read);
#pragma unroll
                    for (int u = 0; u < J; u++)
#pragma unroll
                        for (int q4 = 0; q4 < 4; q4++) {
                            const f32x4 x = *reinterpret_cast<const f32x4 *>(nl + (q2 + u) * 32 + 4 * hf + 8 * q4);
#pragma unroll
                            for (int e = 0; e < 4; e++) s[u][4 * q4 + e] = x[e];
                        }
                    if (kind == Kind::NEAR) {
                        const float *my = tab + key - (q0 + 32 * q2) - 4 * hf + M + kPad - 64;  // (from 64 back: offsets count up)
#pragma unroll
                        for (int u = 0; u < J; u++)
#pragma unroll
                            for (int e = 0; e < 16; e++) s[u][e] += my[64 - (32 * u + 8 * (e >> 2) + (e & 3))];
                    }
#pragma unroll
                    for (int u = 0; u < J; u++)
#pragma unroll
                        for (int q4 = 0; q4 < 4; q4++) {
                            const f32x4 x = *reinterpret_cast<const f32x4 *>(nd + (q2 + u) * 32 + 4 * hf + 8 * q4);
#pragma unroll
                            for (int e = 0; e < 4; e++) dp16[u][4 * q4 + e] = x[e];
                        }
                    rows_ahead.run([&](int i, typename RowsT::Frag f) {
                        if (i < N) s[i % J] = Op<T>::mma(f, kf[i / J], s[i % J]);
                        else dp16[i % J] = Op<T>::mma(f, vf[(i - N) / J], dp16[i % J]);
                    });
                    constexpr int WN = J * RowsT::WSTEPS * RowsT::BLOCKS;
                    auto column = [&](const char *from, int i) { return RowsT::wread(from, tl, lane, (q2 + i / (RowsT::WSTEPS * RowsT::BLOCKS)) * 32, i % RowsT::BLOCKS, i / RowsT::BLOCKS % RowsT::WSTEPS); };
                    auto read_do = [&](int i) { return column(sDO, i); };
                    auto read_q = [&](int i) { return column(sQ, i); };
                    auto do_ahead = ahead<WN, kAheadCols, typename RowsT::WFrag>(read_do);
                    Weights<T> w[J];
#pragma unroll
                    for (int u = 0; u < J; u++) {
#pragma unroll
                        for (int e = 0; e < 16; e++) s[u][e] = fast_exp2(s[u][e] * a.scale_log2);
                        w[u] = Weights<T>(s[u]);
                    }
                    do_ahead.run([&](int i, typename RowsT::WFrag f) {
                        dv[i % RowsT::BLOCKS] = RowsT::wmma(f, w[i / (RowsT::WSTEPS * RowsT::BLOCKS)], i / RowsT::BLOCKS % RowsT::WSTEPS, dv[i % RowsT::BLOCKS]);
                    });
                    auto q_ahead = ahead<WN, kAheadCols, typename RowsT::WFrag>(read_q);
#pragma unroll
                    for (int u = 0; u < J; u++) {
#pragma unroll
                        for (int e = 0; e < 16; e++) s[u][e] *= dp16[u][e];
                        w[u] = Weights<T>(s[u]);
                    }
                    q_ahead.run([&](int i, typename RowsT::WFrag f) {
                        dk[i % RowsT::BLOCKS] = RowsT::wmma(f, w[i / (RowsT::WSTEPS * RowsT::BLOCKS)], i / RowsT::BLOCKS % RowsT::WSTEPS, dk[i % RowsT::BLOCKS]);
                    });
                }
            };
            walk<S::CONST>((tile1 - tile0 + KS - 1) / KS, tile);
        }
    }
    if (KS == 1) __syncthreads();  // (the ring is free)
    join_groups<NW, KS>(smem, dk, grp, wave, lane);
    if (!join_groups<NW, KS>(smem, dv, grp, wave, lane)) return;
    static_assert(kJoined<NW, KS, RowsT::BLOCKS> + NW * 32 * RowsT::ROWB <= KS * S::RING, "they fit the rings");
    const bool real = key < smp.length;
    char *const rows_lds = smem + kJoined<NW, KS, RowsT::BLOCKS> + wave * 32 * RowsT::ROWB;
    const int le = opaque(lane);
    store_rows<T, D>(rows_lds, le, dk, real, a.scale, (T *)a.dk + (size_t)b * a.sdk.batch + (size_t)kvh * a.sdk.head + (size_t)kw0 * a.sdk.row,
                     a.sdk.row, a.n_kv - kw0);
    store_rows<T, D>(rows_lds, le, dv, real, 1.f, (T *)a.dv + (size_t)b * a.sdv.batch + (size_t)kvh * a.sdv.head + (size_t)kw0 * a.sdv.row,
                     a.sdv.row, a.n_kv - kw0);
}

// Both roles in one launch, the longest tiles first: level l holds key tile l of every key head and query tile tiles_q - 1 - l of
// every head, which in the causal form have the same number of tiles to walk.
template <typename T, int D, int NW, int KS, bool CAUSAL>
__global__ __launch_bounds__(NW * KS * 64, sizeof(T) == 4 || D == 128 ? 1 : 2) void k_rel_bwd(RelBwdArgs a)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int nk = a.batch * a.kv_heads, nq = a.batch * a.heads, level = blockIdx.x / (nk + nq), x = blockIdx.x - level * (nk + nq);
    if (x < nk) {
        if (level < a.tiles_k) dkv_role<T, D, NW, KS, CAUSAL>(a, smem, x, level);
    } else if (level < a.tiles_q) {
        dq_role<T, D, NW, KS, CAUSAL>(a, smem, x - nk, a.tiles_q - 1 - level);
    }
}

// dbias of one head: the workgroups' sums by distance added up in their order, several runs of them side by side; then by bucket
__global__ __launch_bounds__(1024) void k_rel_dbias(RelBwdArgs a, int parts, bool causal)
{
    __shared__ f32x4 runs[1024];
    __shared__ int bucket[4096];
    const int tid = threadIdx.x, lane = tid & 63, h = blockIdx.x, nb = a.bias.n_buckets, M = a.bias.max_distance;
    const int len = table_length(M, causal), line = table_row(M, causal), cols = line / 4, n = min(1024 / cols, 16), run = tid / cols;
    for (int x = tid; x < len; x += 1024) {
        const int d = x - M - kPad;
        bucket[x] = causal && d > 0 ? -1 : bucket_of(a.bias, d);
    }
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (run < n) {
        const float *p = a.bins + (size_t)h * parts * line + 4 * (tid - run * cols);
#pragma unroll 4
        for (int i = run; i < parts; i += n) {
            const f32x4 y = *reinterpret_cast<const f32x4 *>(p + (size_t)i * line);
#pragma unroll
            for (int e = 0; e < 4; e++) sum[e] += y[e];
        }
    }
    runs[tid] = sum;
    __syncthreads();
    if (run == 0) {
        for (int i = 1; i < n; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) sum[e] += runs[i * cols + tid][e];
        runs[tid] = sum;
    }
    __syncthreads();
    const float *const by_distance = reinterpret_cast<const float *>(runs);
    for (int u = tid >> 6; u < nb; u += 16) {
        float s = 0.f;
        for (int x = lane; x < len; x += 64) s += bucket[x] == u ? by_distance[x] : 0.f;
        s = wave_sum(s);
        if (lane != 0) continue;
        if (a.bias.bf16)
            ((__bf16 *)a.d_bias)[(size_t)u * a.heads + h] = (__bf16)s;
        else
            ((float *)a.d_bias)[(size_t)u * a.heads + h] = s;
    }
}

template <typename T, int D, int NW, int KS>
hdt_status_t launch(const RelBwdArgs &a, bool causal, hipStream_t st)
{
    using S = BwdShape<T, D, NW, KS>;
    const int line = table_row(a.bias.max_distance, causal);
    const long long rows = (long long)a.batch * a.heads * a.n_pad;
    if (rows > 0) {
        HdtTimer t("hdt_rel_rows", st);
        constexpr int PER = kRowsU * 256 / (D * (int)sizeof(T) / 16);
        const unsigned groups = (unsigned)((rows + PER - 1) / PER);
        hipLaunchKernelGGL((k_rel_rows<T, D>), dim3(groups + (unsigned)a.heads), dim3(256), 0, st, a, rows, groups, causal);
        HDT_HIP_TRY(hipGetLastError());
    }
    const long long levels = std::max(a.heads ? a.tiles_q : 0, a.tiles_k), grid = levels * a.batch * (a.heads + a.kv_heads);
    if (grid > 0) {
        HdtTimer t("hdt_rel_bwd", st);
        const size_t lds_q = KS * S::RING + (size_t)line * (1 + 2 * NW * KS) * sizeof(float), lds_k = KS * (S::RING + S::SCALARS) + (size_t)line * sizeof(float);
        const size_t lds = lds_q > lds_k ? lds_q : lds_k;
        const void *f = causal ? (const void *)k_rel_bwd<T, D, NW, KS, true> : (const void *)k_rel_bwd<T, D, NW, KS, false>;
        if (lds > 65536) HDT_HIP_TRY(hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        if (causal)
            hipLaunchKernelGGL((k_rel_bwd<T, D, NW, KS, true>), dim3((unsigned)grid), dim3(S::THREADS), lds, st, a);
        else
            hipLaunchKernelGGL((k_rel_bwd<T, D, NW, KS, false>), dim3((unsigned)grid), dim3(S::THREADS), lds, st, a);
        HDT_HIP_TRY(hipGetLastError());
    }
    if (a.heads == 0) return HDT_OK;
    HdtTimer t("hdt_rel_dbias", st);
    static_assert(2 * kMostDistance + 2 * kPad <= 4096, "a head's distances fit k_rel_dbias");
    hipLaunchKernelGGL(k_rel_dbias, dim3((unsigned)a.heads), dim3(1024), 0, st, a, a.batch * a.tiles_q, causal);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

template <typename T, int D>
hdt_status_t launch_shape(const RelBwdArgs &a, int nw, bool causal, hipStream_t st)
{
    if (nw == 4) return launch<T, D, 4, 1>(a, causal, st);
    if (nw == 2) return launch<T, D, 2, 2>(a, causal, st);
    return launch<T, D, D == 64 ? 1 : 2, D == 64 ? 4 : 2>(a, causal, st);
}

}  // namespace

RelBwdPlan hdt_rel_bwd_plan(const hdt_rel_attn_t &d)
{
    RelBwdPlan p;
    auto tiles = [&](long long bm) { return d.batch * (d.heads * ((d.n_q + bm - 1) / bm) + d.kv_heads * ((d.n_kv + bm - 1) / bm)); };
    p.waves = hdt_rel_row_waves(tiles(64), tiles(32), d);
    // (a ring for each group, the table, and a row of sums by distance for each half-wave have to fit a compute unit's LDS)
    const size_t ring = (size_t)4 * (d.dtype == HDT_BF16 ? 64 * 2 : 32 * 4) * d.head_dim, line = table_row(d.max_distance, d.causal != 0) * sizeof(float);
    while (p.waves < 4 && 4 / p.waves * ring + 9 * line > 160 * 1024) p.waves *= 2;
    const int bm = 32 * p.waves;
    p.tiles_q = (d.n_q + bm - 1) / bm;
    p.tiles_k = (d.n_kv + bm - 1) / bm;
    p.n_pad = (d.n_q + 127) & ~127;
    const size_t rows = (size_t)d.batch * d.heads * p.n_pad;
    p.tables_at = (4 * rows * sizeof(float) + 255) & ~(size_t)255;
    p.bins_at = p.tables_at + (rows ? d.heads * line : 0);
    p.bytes = p.bins_at + (size_t)d.heads * d.batch * p.tiles_q * line;
    return p;
}

hdt_status_t hdt_launch_rel_bwd(const hdt_rel_attn_t &d, const RelBwdArgs &a, int waves, hipStream_t st)
{
    const bool causal = d.causal != 0;
    if (d.dtype == HDT_BF16) return d.head_dim == 64 ? launch_shape<__bf16, 64>(a, waves, causal, st) : launch_shape<__bf16, 128>(a, waves, causal, st);
    return d.head_dim == 64 ? launch_shape<float, 64>(a, waves, causal, st) : launch_shape<float, 128>(a, waves, causal, st);
}
