// Backward pass of self-attention with a relative position bias:
//     D_i = sum_c dO_ic O_ic,  P = exp(S - LSE),  dP = dO V^T,  dS = P o (dP - D),
//     dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO,  dbias[u][h] = sum of dS over the pairs of head h in bucket u.
// No atomics on memory: the results do not depend on the order in which workgroups run.
#include <algorithm>
#include <type_traits>

#include "hdt_rel.h"
#include "hdt_rel_args.h"

namespace {

using namespace hdt_rel;

// Four numbers of every row, four arrays of [batch][heads][n_pad]: n = -LSE log2(e), minus infinity for a row without keys (its pairs then
// weigh exp2(-inf) = 0); -D; and n with the bias of far keys behind and ahead, what the exponent of a far block starts from.  Every
// head's rows are filled up to whole tiles with rows without keys.
constexpr int kRowsU = 2;  // rows a thread has in flight
template <typename T, int D>
__global__ __launch_bounds__(256) void k_rel_rows(RelBwdArgs a, long long rows)
{
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
        const bool dead = ri[u] < smp.lo || ri[u] >= smp.hi || lse[u] == -INFINITY;
        const float n = dead ? -INFINITY : -lse[u] * LOG2E;
        a.row_scalars[r] = n;
        a.row_scalars[rows + r] = dead ? 0.f : -d;
        a.row_scalars[2 * rows + r] = n + bias_of(a.bias, -a.bias.max_distance, h) * a.scale_log2;
        a.row_scalars[3 * rows + r] = n + bias_of(a.bias, a.bias.max_distance, h) * a.scale_log2;
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

template <typename T, int D, int NW_>
struct BwdShape {
    static constexpr int NW = NW_, BM = 32 * NW, BN = sizeof(T) == 4 && D == 128 ? 32 : 64;
    static constexpr int RING = 2 * Pair<T, D, BN, NW>::STAGE, SCALARS = 2 * 4 * 256;  // two stages of four arrays of 64 floats
    static constexpr int KB = BN / 32, J = sizeof(T) == 2 && D == 64 ? KB : 1;          // blocks of a tile, and how many at a time
};

// dQ of a tile of query rows, and the sums of its dS by bucket
template <typename T, int D, int NW_, bool CAUSAL>
__device__ __forceinline__ void dq_role(const RelBwdArgs &a, char *smem, int bh, int I)
{
    using S = BwdShape<T, D, NW_>;
    using RowsT = Rows<T, D>;
    constexpr int BM = S::BM, BN = S::BN, NW = S::NW, KB = S::KB, J = S::J;
    const int M = a.bias.max_distance, len = table_length(M, CAUSAL);
    float *const tab = reinterpret_cast<float *>(smem + S::RING), *const bins = tab + len;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    const int b = bh / a.heads, h = bh - b * a.heads;
    const Sample smp = sample_of(a.lengths, a.starts, b, a.n_q, a.n_kv);
    const int r0 = I * BM, first = max(r0, smp.lo), last = min(r0 + BM, smp.hi) - 1;
    const int row = r0 + wave * 32 + (lane & 31);
    const bool own = row < a.n_q, real = row >= first && row <= last;
    const int seen = first <= last ? (CAUSAL ? smp.start + last + 1 : smp.length) : 0, tiles = (seen + BN - 1) / BN;

    f32x16 acc[RowsT::BLOCKS];
#pragma unroll
    for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[j][e] = 0.f;
    float behind = 0.f, ahead = 0.f;                       // this lane's sums of dS in the far tiles
    float *const my_bins = bins + (wave * 2 + hf) * len;   // one copy for each half-wave: no two lanes of an instruction meet
    for (int x = tid; x < len * NW * 2; x += NW * 64) bins[x] = 0.f;

    if (tiles > 0) {
        const int rc = min(max(row, first), last), pos = smp.start + rc;
        const int w0 = max(r0 + wave * 32, first), w1 = min(r0 + wave * 32 + 31, last), p0 = smp.start + w0, p1 = smp.start + w1;
        const size_t kvh = (size_t)(h / a.group);
        Pair<T, D, BN, NW> kv;
        kv.init((const T *)a.k + (size_t)b * a.sk.batch + kvh * a.sk.head, a.sk.row, (const T *)a.v + (size_t)b * a.sv.batch + kvh * a.sv.head,
                a.sv.row, smem, wave, lane);
        typename RowsT::Frag qf[RowsT::STEPS], dof[RowsT::STEPS];
        const char *qp = (const char *)((const T *)a.q + (size_t)b * a.sq.batch + (size_t)h * a.sq.head + (size_t)rc * a.sq.row);
        const char *dp = (const char *)((const T *)a.d_o + (size_t)b * a.sdo.batch + (size_t)h * a.sdo.head + (size_t)rc * a.sdo.row);
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) {
            qf[st] = *reinterpret_cast<const typename RowsT::Frag *>(qp + (2 * st + hf) * 16);
            dof[st] = *reinterpret_cast<const typename RowsT::Frag *>(dp + (2 * st + hf) * 16);
        }
        const size_t at_row = (size_t)bh * a.n_pad + rc, rows = (size_t)a.batch * a.heads * a.n_pad;
        const float nl = real ? a.row_scalars[at_row] : -INFINITY, nd = a.row_scalars[rows + at_row];
        fill_table<CAUSAL>(tab, a.bias, h, 1, tid, NW * 64);
        kv.request(0, 0, seen - 1, 0);
        const float *const my_tab = tab + 4 * hf - pos + M + kPad;
        float *const diagonal = my_bins + 4 * hf - (lane & 31) - (smp.start + r0 + wave * 32) + M + kPad;  // of key 0 and j = 0
        const RowLane rl = row_lane<RowsT::CPR>(lane);
        const TrLane tl = tr_lane<RowsT::CPR>(lane);
        __syncthreads();
        const float c_behind = tab[0] * a.scale_log2, c_ahead = tab[len - 1] * a.scale_log2;

        auto tile = [&](int t, auto stage) {
            constexpr int ST = decltype(stage)::value;
            wait_vmcnt<0>();
            wg_barrier();
            if (t + 1 < tiles) kv.request((t + 1) * BN, 0, seen - 1, 1 - ST);
            const char *sK = smem + ST * kv.STAGE, *sV = sK + kv.TILE;
            const Kind kind = kind_of<CAUSAL, BN>(t * BN, p0, p1, M, smp.length);
            if (kind == Kind::SKIP || w0 > w1) return;  // (nor has a wave without real rows anything to do)
            const float off = nl + (kind == Kind::FAR_BEHIND ? c_behind : kind == Kind::FAR_AHEAD ? c_ahead : 0.f);
#pragma unroll
            for (int k2 = 0; k2 < KB; k2 += J) {
                const int k0 = t * BN + 32 * k2;
                f32x16 s[J], dp16[J];
                if (kind == Kind::NEAR) {
#pragma unroll
                    for (int u = 0; u < J; u++) {
#pragma unroll
                        for (int e = 0; e < 16; e++) s[u][e] = my_tab[k0 + 32 * u + 8 * (e >> 2) + (e & 3)];
                        s[u] = Op<T>::mma(RowsT::read(sK, rl, (k2 + u) * 32, 0), qf[0], s[u]);
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < J; u++) {
#pragma unroll
                        for (int e = 0; e < 16; e++) s[u][e] = 0.f;
                        s[u] = Op<T>::mma(RowsT::read(sK, rl, (k2 + u) * 32, 0), qf[0], s[u]);
                    }
                }
#pragma unroll
                for (int u = 0; u < J; u++)
#pragma unroll
                    for (int e = 0; e < 16; e++) dp16[u][e] = nd;
#pragma unroll
                for (int st = 1; st < RowsT::STEPS; st++)
#pragma unroll
                    for (int u = 0; u < J; u++) s[u] = Op<T>::mma(RowsT::read(sK, rl, (k2 + u) * 32, st), qf[st], s[u]);
#pragma unroll
                for (int st = 0; st < RowsT::STEPS; st++)
#pragma unroll
                    for (int u = 0; u < J; u++) dp16[u] = Op<T>::mma(RowsT::read(sV, rl, (k2 + u) * 32, st), dof[st], dp16[u]);
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
                    else ahead += sum;
                }
#pragma unroll
                for (int u = 0; u < J; u++) {
                    const Weights<T> w(s[u]);
#pragma unroll
                    for (int j = 0; j < RowsT::BLOCKS; j++) acc[j] = RowsT::weigh(sK, tl, lane, (k2 + u) * 32, j, w, acc[j]);
                }
            }
        };
        int t = 0;
        for (; t + 1 < tiles; t += 2) {
            tile(t, std::integral_constant<int, 0>());
            tile(t + 1, std::integral_constant<int, 1>());
        }
        if (t < tiles) tile(t, std::integral_constant<int, 0>());
    }
    // the far tiles' sums join the bins at the two ends of the table
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        behind += __shfl_xor(behind, m);
        if (!CAUSAL) ahead += __shfl_xor(ahead, m);
    }
    __syncthreads();
    if (lane == 0) {
        bins[wave * 2 * len] += behind;
        if (!CAUSAL) bins[wave * 2 * len + len - 1] += ahead;
    }
    __syncthreads();
    // sums over the copies, by distance; their buckets beside them (the ring is free)
    int *const bucket = reinterpret_cast<int *>(smem);
    for (int x = tid; x < len; x += NW * 64) {
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < NW * 2; u++) sum += bins[u * len + x];
        const int d = x - M - kPad;
        bins[x] = sum;
        bucket[x] = CAUSAL && d > 0 ? -1 : bucket_of(a.bias, d);
    }
    __syncthreads();
    float *const out = a.bins + ((size_t)h * a.batch * a.tiles_q + (size_t)b * a.tiles_q + I) * a.bias.n_buckets;
    for (int u = wave; u < a.bias.n_buckets; u += NW) {
        float sum = 0.f;
        for (int x = lane; x < len; x += 64) sum += bucket[x] == u ? bins[x] : 0.f;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
        if (lane == 0) out[u] = sum;
    }
    if (!own) return;
    T *dq = (T *)a.dq + (size_t)b * a.sdq.batch + (size_t)h * a.sdq.head + (size_t)row * a.sdq.row;
    const float mult = real ? a.scale : 0.f;
#pragma unroll
    for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
        for (int q4 = 0; q4 < 4; q4++)
            store4(dq + 32 * j + 8 * q4 + 4 * hf, acc[j][q4 * 4] * mult, acc[j][q4 * 4 + 1] * mult, acc[j][q4 * 4 + 2] * mult, acc[j][q4 * 4 + 3] * mult);
}

// dK and dV of a tile of keys of one key head: over the query rows of every head that shares it
template <typename T, int D, int NW_, bool CAUSAL>
__device__ __forceinline__ void dkv_role(const RelBwdArgs &a, char *smem, int bk, int J0)
{
    using S = BwdShape<T, D, NW_>;
    using RowsT = Rows<T, D>;
    constexpr int BM = S::BM, BN = S::BN, NW = S::NW, KB = S::KB, J = S::J;
    constexpr bool LEAN = D == 128;  // what can be computed anew from the lane number is: registers are short
    const int M = a.bias.max_distance, len = table_length(M, CAUSAL);
    float *const scal = reinterpret_cast<float *>(smem + S::RING), *const tab = scal + S::SCALARS / 4;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
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
        const size_t rows = (size_t)a.batch * a.heads * a.n_pad;
        for (int h = kvh * a.group; h < (kvh + 1) * a.group; h++) {
            Pair<T, D, BN, NW> qd;
            qd.init((const T *)a.q + (size_t)b * a.sq.batch + (size_t)h * a.sq.head, a.sq.row,
                    (const T *)a.d_o + (size_t)b * a.sdo.batch + (size_t)h * a.sdo.head, a.sdo.row, smem, wave, lane);
            const float *rs = a.row_scalars + ((size_t)b * a.heads + h) * a.n_pad;
            auto request = [&](int t, int stage) {
                // (rows that are not real: copies, weighed zero)
                qd.request(t * BN, smp.lo, smp.hi - 1, stage);
                for (int w = wave; w < 4; w += NW)
                    dma4(rs + w * rows + t * BN, (uint32_t)(lane & (BN - 1)) * 4u, qd.lds + S::RING + (stage * 4 + w) * 256);
            };
            __syncthreads();  // the head before is done with the table and the ring
            fill_table<CAUSAL>(tab, a.bias, h, 1, tid, NW * 64);
            request(tile0, 0);
            __syncthreads();
            auto tile = [&](int t, auto stage) {
                constexpr int ST = decltype(stage)::value;
                wait_vmcnt<0>();
                wg_barrier();
                if (t + 1 < tile1) request(t + 1, 1 - ST);
                const char *sQ = smem + ST * qd.STAGE, *sDO = sQ + qd.TILE;
                const int q0 = smp.start + t * BN;  // position of the tile's first row
                // seen from the wave's 32 keys: the kinds of keys kw0 .. kw0 + 31 against positions q0 .. q0 + BN - 1
                const Kind kind = (CAUSAL && kw0 > q0 + BN - 1) || kw0 >= smp.length ? Kind::SKIP
                                  : kw0 + 31 - q0 <= -M                              ? Kind::FAR_BEHIND
                                  : !CAUSAL && kw0 - (q0 + BN - 1) >= M              ? Kind::FAR_AHEAD
                                                                                     : Kind::NEAR;
                if (kind == Kind::SKIP) return;
                const float *const st4 = scal + ST * 256, *const nd = st4 + 64;
                const float *const nl = kind == Kind::FAR_BEHIND ? st4 + 128 : kind == Kind::FAR_AHEAD ? st4 + 192 : st4;
                const int ol = LEAN ? opaque(lane) : lane;
                const RowLane rl = row_lane<RowsT::CPR>(ol);
                const TrLane tl = tr_lane<RowsT::CPR>(ol);
#pragma unroll
                for (int q2 = 0; q2 < KB; q2 += J) {
                    f32x16 s[J], dp16[J];
                    if (kind == Kind::NEAR) {
                        const float *my = tab + key - (q0 + 32 * q2) - 4 * hf + M + kPad;
#pragma unroll
                        for (int u = 0; u < J; u++) {
#pragma unroll
                            for (int e = 0; e < 16; e++) s[u][e] = my[-(32 * u + 8 * (e >> 2) + (e & 3))];
                            s[u] = Op<T>::mma(RowsT::read(sQ, rl, (q2 + u) * 32, 0), kf[0], s[u]);
                        }
                    } else {
#pragma unroll
                        for (int u = 0; u < J; u++) {
#pragma unroll
                            for (int e = 0; e < 16; e++) s[u][e] = 0.f;
                            s[u] = Op<T>::mma(RowsT::read(sQ, rl, (q2 + u) * 32, 0), kf[0], s[u]);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < J; u++)
#pragma unroll
                        for (int q4 = 0; q4 < 4; q4++) {
                            const f32x4 x = *reinterpret_cast<const f32x4 *>(nd + (q2 + u) * 32 + 4 * hf + 8 * q4);
#pragma unroll
                            for (int e = 0; e < 4; e++) dp16[u][4 * q4 + e] = x[e];
                        }
#pragma unroll
                    for (int st = 1; st < RowsT::STEPS; st++)
#pragma unroll
                        for (int u = 0; u < J; u++) s[u] = Op<T>::mma(RowsT::read(sQ, rl, (q2 + u) * 32, st), kf[st], s[u]);
#pragma unroll
                    for (int st = 0; st < RowsT::STEPS; st++)
#pragma unroll
                        for (int u = 0; u < J; u++) dp16[u] = Op<T>::mma(RowsT::read(sDO, rl, (q2 + u) * 32, st), vf[st], dp16[u]);
#pragma unroll
                    for (int u = 0; u < J; u++) {
#pragma unroll
                        for (int q4 = 0; q4 < 4; q4++) {
                            const f32x4 x = *reinterpret_cast<const f32x4 *>(nl + (q2 + u) * 32 + 4 * hf + 8 * q4);
#pragma unroll
                            for (int e = 0; e < 4; e++) s[u][4 * q4 + e] = fast_exp2(fmaf(s[u][4 * q4 + e], a.scale_log2, x[e]));
                        }
                        const Weights<T> w(s[u]);
#pragma unroll
                        for (int j = 0; j < RowsT::BLOCKS; j++) dv[j] = RowsT::weigh(sDO, tl, lane, (q2 + u) * 32, j, w, dv[j]);
                    }
#pragma unroll
                    for (int u = 0; u < J; u++) {
#pragma unroll
                        for (int e = 0; e < 16; e++) s[u][e] *= dp16[u][e];
                        const Weights<T> w(s[u]);
#pragma unroll
                        for (int j = 0; j < RowsT::BLOCKS; j++) dk[j] = RowsT::weigh(sQ, tl, lane, (q2 + u) * 32, j, w, dk[j]);
                    }
                }
            };
            int t = tile0;
            for (; t + 1 < tile1; t += 2) {
                tile(t, std::integral_constant<int, 0>());
                tile(t + 1, std::integral_constant<int, 1>());
            }
            if (t < tile1) tile(t, std::integral_constant<int, 0>());
        }
    }
    if (key >= a.n_kv) return;
    const bool real = key < smp.length;
    T *ok = (T *)a.dk + (size_t)b * a.sdk.batch + (size_t)kvh * a.sdk.head + (size_t)key * a.sdk.row;
    T *ov = (T *)a.dv + (size_t)b * a.sdv.batch + (size_t)kvh * a.sdv.head + (size_t)key * a.sdv.row;
    const float mk = real ? a.scale : 0.f, mv = real ? 1.f : 0.f;
#pragma unroll
    for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
        for (int q4 = 0; q4 < 4; q4++) {
            store4(ok + 32 * j + 8 * q4 + 4 * hf, dk[j][q4 * 4] * mk, dk[j][q4 * 4 + 1] * mk, dk[j][q4 * 4 + 2] * mk, dk[j][q4 * 4 + 3] * mk);
            store4(ov + 32 * j + 8 * q4 + 4 * hf, dv[j][q4 * 4] * mv, dv[j][q4 * 4 + 1] * mv, dv[j][q4 * 4 + 2] * mv, dv[j][q4 * 4 + 3] * mv);
        }
}

// Both roles in one launch, the longest tiles first: level l holds key tile l of every key head and query tile tiles_q - 1 - l of
// every head, which in the causal form have the same number of tiles to walk.
template <typename T, int D, int NW, bool CAUSAL>
__global__ __launch_bounds__(NW * 64, sizeof(T) == 4 ? 1 : 2) void k_rel_bwd(RelBwdArgs a)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int nk = a.batch * a.kv_heads, nq = a.batch * a.heads, level = blockIdx.x / (nk + nq), x = blockIdx.x - level * (nk + nq);
    if (x < nk) {
        if (level < a.tiles_k) dkv_role<T, D, NW, CAUSAL>(a, smem, x, level);
    } else if (level < a.tiles_q) {
        dq_role<T, D, NW, CAUSAL>(a, smem, x - nk, a.tiles_q - 1 - level);
    }
}

// dbias of one head: the workgroups' sums by bucket added up in their order, 16 runs of them
__global__ __launch_bounds__(1024) void k_rel_dbias(RelBwdArgs a, int parts)
{
    __shared__ float lds[16][64];
    const int lane = threadIdx.x & 63, run = threadIdx.x >> 6, u = blockIdx.y * 64 + lane, h = blockIdx.x, nb = a.bias.n_buckets;
    float sum = 0.f;
    if (u < nb) {
        const float *p = a.bins + (size_t)h * parts * nb + u;
        for (int i = run; i < parts; i += 16) sum += p[(size_t)i * nb];
    }
    lds[run][lane] = sum;
    __syncthreads();
    if (run != 0 || u >= nb) return;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i++) sum += lds[i][lane];
    if (a.bias.bf16)
        ((__bf16 *)a.d_bias)[(size_t)u * a.heads + h] = (__bf16)sum;
    else
        ((float *)a.d_bias)[(size_t)u * a.heads + h] = sum;
}

template <typename T, int D, int NW>
hdt_status_t launch(const RelBwdArgs &a, bool causal, hipStream_t st)
{
    using S = BwdShape<T, D, NW>;
    const int len = table_length(a.bias.max_distance, causal);
    const long long rows = (long long)a.batch * a.heads * a.n_pad;
    if (rows > 0) {
        HdtTimer t("hdt_rel_rows", st);
        constexpr int PER = kRowsU * 256 / (D * (int)sizeof(T) / 16);
        hipLaunchKernelGGL((k_rel_rows<T, D>), dim3((unsigned)((rows + PER - 1) / PER)), dim3(256), 0, st, a, rows);
        HDT_HIP_TRY(hipGetLastError());
    }
    const long long levels = std::max(a.heads ? a.tiles_q : 0, a.tiles_k), grid = levels * a.batch * (a.heads + a.kv_heads);
    if (grid > 0) {
        HdtTimer t("hdt_rel_bwd", st);
        const size_t lds_q = S::RING + (size_t)len * (1 + 2 * NW) * sizeof(float), lds_k = S::RING + S::SCALARS + (size_t)len * sizeof(float);
        const size_t lds = lds_q > lds_k ? lds_q : lds_k;
        const void *f = causal ? (const void *)k_rel_bwd<T, D, NW, true> : (const void *)k_rel_bwd<T, D, NW, false>;
        if (lds > 65536) HDT_HIP_TRY(hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        if (causal)
            hipLaunchKernelGGL((k_rel_bwd<T, D, NW, true>), dim3((unsigned)grid), dim3(NW * 64), lds, st, a);
        else
            hipLaunchKernelGGL((k_rel_bwd<T, D, NW, false>), dim3((unsigned)grid), dim3(NW * 64), lds, st, a);
        HDT_HIP_TRY(hipGetLastError());
    }
    if (a.heads == 0) return HDT_OK;
    HdtTimer t("hdt_rel_dbias", st);
    hipLaunchKernelGGL(k_rel_dbias, dim3((unsigned)a.heads, (unsigned)(a.bias.n_buckets + 63) / 64), dim3(1024), 0, st, a, a.batch * a.tiles_q);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

template <typename T, int D>
hdt_status_t launch_shape(const RelBwdArgs &a, int nw, bool causal, hipStream_t st)
{
    return nw == 4 ? launch<T, D, 4>(a, causal, st) : launch<T, D, 2>(a, causal, st);
}

}  // namespace

RelBwdPlan hdt_rel_bwd_plan(const hdt_rel_attn_t &d)
{
    RelBwdPlan p;
    // tiles of 64 rows where 128 would leave compute units without work
    const long long tiles = (long long)d.batch * d.heads * ((d.n_q + 127) / 128) + (long long)d.batch * d.kv_heads * ((d.n_kv + 127) / 128);
    p.waves = tiles < 768 ? 2 : 4;
    const int bm = 32 * p.waves;
    p.tiles_q = (d.n_q + bm - 1) / bm;
    p.tiles_k = (d.n_kv + bm - 1) / bm;
    p.n_pad = (d.n_q + 127) & ~127;
    const size_t rows = (size_t)d.batch * d.heads * p.n_pad;
    p.bins_at = (4 * rows * sizeof(float) + 255) & ~(size_t)255;
    p.bytes = p.bins_at + (size_t)d.heads * d.batch * p.tiles_q * d.n_buckets * sizeof(float);
    return p;
}

hdt_status_t hdt_launch_rel_bwd(const hdt_rel_attn_t &d, const RelBwdArgs &a, int waves, hipStream_t st)
{
    const bool causal = d.causal != 0;
    if (d.dtype == HDT_BF16) return d.head_dim == 64 ? launch_shape<__bf16, 64>(a, waves, causal, st) : launch_shape<__bf16, 128>(a, waves, causal, st);
    return d.head_dim == 64 ? launch_shape<float, 64>(a, waves, causal, st) : launch_shape<float, 128>(a, waves, causal, st);
}
