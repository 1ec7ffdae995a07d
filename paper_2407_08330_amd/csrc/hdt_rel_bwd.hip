// Backward pass of self-attention with a relative position bias:
//     D_i = sum_c dO_ic O_ic,  P = exp(S - LSE),  dP = dO V^T,  dS = P o (dP - D),
//     dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO,  dbias[u][h] = sum of dS over the pairs of head h in bucket u.
// No atomics on memory: the results do not depend on the order in which workgroups run.
#include "hdt_rel.h"
#include "hdt_rel_args.h"

namespace {

using namespace hdt_rel;

// Two numbers of every row: -LSE log2(e), minus infinity for a row without keys (its pairs then weigh exp2(-inf) = 0), and -D.  Every
// head's rows are filled up to whole tiles with rows without keys.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_rel_rows(RelBwdArgs a, long long rows)
{
    constexpr int LANES = D / 8, PER = 256 / LANES;
    const long long r = (long long)blockIdx.x * PER + threadIdx.x / LANES;
    const int c = threadIdx.x % LANES;
    float d = 0.f;
    const int bh = (int)(min(r, rows - 1) / a.n_pad), ri = (int)(min(r, rows - 1) - (long long)bh * a.n_pad), i = min(ri, a.n_q - 1);
    const int b = bh / a.heads, h = bh - b * a.heads;
    const T *o = (const T *)a.o + (size_t)b * a.so.batch + (size_t)h * a.so.head + (size_t)i * a.so.row + 8 * c;
    const T *g = (const T *)a.d_o + (size_t)b * a.sdo.batch + (size_t)h * a.sdo.head + (size_t)i * a.sdo.row + 8 * c;
#pragma unroll
    for (int e = 0; e < 8; e++) d = fmaf((float)o[e], (float)g[e], d);
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) d += __shfl_xor(d, m);
    const Sample smp = sample_of(a.lengths, a.starts, b, a.n_q, a.n_kv);
    const float lse = a.lse[(size_t)bh * a.n_q + i];
    const bool dead = ri < smp.lo || ri >= smp.hi || lse == -INFINITY;
    if (c == 0 && r < rows) {
        a.row_scalars[r] = dead ? -INFINITY : -lse * LOG2E;
        a.row_scalars[rows + r] = dead ? 0.f : -d;
    }
}

template <typename T, int D>
struct BwdShape {
    static constexpr int NW = 4, BM = 32 * NW, BN = sizeof(T) == 4 && D == 128 ? 32 : 64;
    static constexpr int TILE = BN * Rows<T, D>::ROWB, RING = 4 * TILE, SCALARS = 1024;  // two stages of two rows' worth of 64 floats
};

// dQ of a tile of query rows, and the sums of its dS by distance
template <typename T, int D, bool CAUSAL>
__global__ __launch_bounds__(256, 1) void k_rel_dq(RelBwdArgs a)
{
    using S = BwdShape<T, D>;
    using RowsT = Rows<T, D>;
    constexpr int BM = S::BM, BN = S::BN, NW = S::NW;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int M = a.bias.max_distance, len = table_length(M, CAUSAL);
    float *const tab = reinterpret_cast<float *>(smem + S::RING), *const bins = tab + len;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    const int I = blockIdx.x % a.tiles_q, bh = blockIdx.x / a.tiles_q, b = bh / a.heads, h = bh - b * a.heads;
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
    float behind = 0.f, ahead = 0.f;  // sums of dS in the far blocks
    float *const my_bins = bins + (wave * 2 + hf) * len;  // one copy for each half-wave: no two lanes of an instruction meet
    for (int x = tid; x < len * NW * 2; x += NW * 64) bins[x] = 0.f;

    if (tiles > 0) {
        const int rc = min(max(row, first), last), pos = smp.start + rc;
        const int p0 = smp.start + min(max(r0 + wave * 32, first), last), p1 = smp.start + min(max(r0 + wave * 32 + 31, first), last);
        const size_t kvh = (size_t)(h / a.group);
        const char *kb = (const char *)a.k + ((size_t)b * a.sk.batch + kvh * a.sk.head) * sizeof(T);
        const char *vb = (const char *)a.v + ((size_t)b * a.sv.batch + kvh * a.sv.head) * sizeof(T);
        const uint32_t krow = (uint32_t)a.sk.row * sizeof(T), vrow = (uint32_t)a.sv.row * sizeof(T);
        const uint32_t lds = lds_addr(smem);
        auto request = [&](int t) {
            const uint32_t at = lds + (uint32_t)(t & 1) * 2 * S::TILE;
            RowsT::template load<BN, NW>(kb + (size_t)t * BN * krow, krow, 0, seen - 1 - t * BN, at, wave, lane);
            RowsT::template load<BN, NW>(vb + (size_t)t * BN * vrow, vrow, 0, seen - 1 - t * BN, at + S::TILE, wave, lane);
        };
        typename RowsT::Frag qf[RowsT::STEPS], dof[RowsT::STEPS];
        const char *qp = (const char *)a.q + ((size_t)b * a.sq.batch + (size_t)h * a.sq.head + (size_t)rc * a.sq.row) * sizeof(T);
        const char *dp = (const char *)a.d_o + ((size_t)b * a.sdo.batch + (size_t)h * a.sdo.head + (size_t)rc * a.sdo.row) * sizeof(T);
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) {
            qf[st] = *reinterpret_cast<const typename RowsT::Frag *>(qp + (2 * st + hf) * 16);
            dof[st] = *reinterpret_cast<const typename RowsT::Frag *>(dp + (2 * st + hf) * 16);
        }
        const size_t at_row = (size_t)bh * a.n_pad + rc, rows = (size_t)a.batch * a.heads * a.n_pad;
        const float nl = real ? a.row_scalars[at_row] : -INFINITY, nd = a.row_scalars[rows + at_row];
        fill_table<CAUSAL>(tab, a.bias, h, 1, tid, NW * 64);
        request(0);
        const int to_bin = 4 * hf - pos + M + kPad;
        const RowLane rl = row_lane<RowsT::CPR>(lane);
        const TrLane tl = tr_lane<RowsT::CPR>(lane);
        __syncthreads();
        const float c_behind = tab[0] * a.scale_log2, c_ahead = tab[len - 1] * a.scale_log2;

        for (int t = 0; t < tiles; t++) {
            wait_vmcnt<0>();
            wg_barrier();
            if (t + 1 < tiles) request(t + 1);
            const char *sK = smem + (t & 1) * 2 * S::TILE, *sV = sK + S::TILE;
#pragma unroll
            for (int kb32 = 0; kb32 < BN / 32; kb32++) {
                const int k0 = t * BN + kb32 * 32;
                const Kind kind = kind_of<CAUSAL>(k0, p0, p1, M, smp.length);
                if (kind == Kind::SKIP) continue;
                f32x16 s, dp16;
#pragma unroll
                for (int e = 0; e < 16; e++) dp16[e] = nd;
                if (kind == Kind::NEAR) {
#pragma unroll
                    for (int e = 0; e < 16; e++) s[e] = tab[to_bin + k0 + 8 * (e >> 2) + (e & 3)];
                } else {
#pragma unroll
                    for (int e = 0; e < 16; e++) s[e] = 0.f;
                }
                const float off = nl + (kind == Kind::FAR_BEHIND ? c_behind : kind == Kind::FAR_AHEAD ? c_ahead : 0.f);
#pragma unroll
                for (int st = 0; st < RowsT::STEPS; st++) {
                    s = Op<T>::mma(RowsT::read(sK, rl, kb32 * 32, st), qf[st], s);
                    dp16 = Op<T>::mma(RowsT::read(sV, rl, kb32 * 32, st), dof[st], dp16);
                }
                if (!CAUSAL && k0 + 32 > smp.length) {
#pragma unroll
                    for (int e = 0; e < 16; e++) s[e] = k0 + 4 * hf + 8 * (e >> 2) + (e & 3) < smp.length ? s[e] : -INFINITY;
                }
#pragma unroll
                for (int e = 0; e < 16; e++) s[e] = fast_exp2(fmaf(s[e], a.scale_log2, off)) * dp16[e];  // dS^T
                if (kind == Kind::NEAR) {
#pragma unroll
                    for (int e = 0; e < 16; e++) __hip_atomic_fetch_add(my_bins + to_bin + k0 + 8 * (e >> 2) + (e & 3), s[e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                } else {
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 16; e++) sum += s[e];
                    if (kind == Kind::FAR_BEHIND) behind += sum;
                    else ahead += sum;
                }
                const Weights<T> w(s);
#pragma unroll
                for (int j = 0; j < RowsT::BLOCKS; j++) acc[j] = RowsT::weigh(sK, tl, lane, kb32 * 32, j, w, acc[j]);
            }
        }
    }
    // the far blocks' sums join the bins at the two ends of the table
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        behind += __shfl_xor(behind, m);
        ahead += __shfl_xor(ahead, m);
    }
    __syncthreads();
    if (lane == 0) {
        bins[wave * 2 * len] += behind;
        if (!CAUSAL) bins[wave * 2 * len + len - 1] += ahead;
    }
    __syncthreads();
    float *out = a.bins + ((size_t)h * a.batch * a.tiles_q + (size_t)b * a.tiles_q + I) * len;
    for (int x = tid; x < len; x += NW * 64) {
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < NW * 2; u++) sum += bins[u * len + x];
        out[x] = sum;
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
template <typename T, int D, bool CAUSAL>
__global__ __launch_bounds__(256, 1) void k_rel_dkv(RelBwdArgs a)
{
    using S = BwdShape<T, D>;
    using RowsT = Rows<T, D>;
    constexpr int BM = S::BM, BN = S::BN, NW = S::NW;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int M = a.bias.max_distance, len = table_length(M, CAUSAL);
    float *const scal = reinterpret_cast<float *>(smem + S::RING), *const tab = scal + S::SCALARS / 4;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    const int J = blockIdx.x % a.tiles_k, bk = blockIdx.x / a.tiles_k, b = bk / a.kv_heads, kvh = bk - b * a.kv_heads;
    const Sample smp = sample_of(a.lengths, a.starts, b, a.n_q, a.n_kv);
    const int key0 = J * BM, key = key0 + wave * 32 + (lane & 31), kc = min(key, smp.length - 1);
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
        const char *kp = (const char *)a.k + ((size_t)b * a.sk.batch + (size_t)kvh * a.sk.head + (size_t)kc * a.sk.row) * sizeof(T);
        const char *vp = (const char *)a.v + ((size_t)b * a.sv.batch + (size_t)kvh * a.sv.head + (size_t)kc * a.sv.row) * sizeof(T);
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) {
            kf[st] = *reinterpret_cast<const typename RowsT::Frag *>(kp + (2 * st + hf) * 16);
            vf[st] = *reinterpret_cast<const typename RowsT::Frag *>(vp + (2 * st + hf) * 16);
        }
        const uint32_t lds = lds_addr(smem);
        const uint32_t qrow = (uint32_t)a.sq.row * sizeof(T), drow = (uint32_t)a.sdo.row * sizeof(T);
        const size_t rows = (size_t)a.batch * a.heads * a.n_pad;
        const RowLane rl = row_lane<RowsT::CPR>(lane);
        const TrLane tl = tr_lane<RowsT::CPR>(lane);
        const int kw0 = key0 + wave * 32;
        for (int h = kvh * a.group; h < (kvh + 1) * a.group; h++) {
            const char *qb = (const char *)a.q + ((size_t)b * a.sq.batch + (size_t)h * a.sq.head) * sizeof(T);
            const char *db = (const char *)a.d_o + ((size_t)b * a.sdo.batch + (size_t)h * a.sdo.head) * sizeof(T);
            const float *rs = a.row_scalars + ((size_t)b * a.heads + h) * a.n_pad;
            auto request = [&](int t) {
                // rows that are not real are taken to be the nearest one that is: their weights are zero, what they hold may be anything
                const uint32_t at = lds + (uint32_t)(t & 1) * 2 * S::TILE;
                const int r0 = t * BN, low = max(smp.lo - r0, 0);
                RowsT::template load<BN, NW>(qb + (size_t)r0 * qrow, qrow, low, smp.hi - 1 - r0, at, wave, lane);
                RowsT::template load<BN, NW>(db + (size_t)r0 * drow, drow, low, smp.hi - 1 - r0, at + S::TILE, wave, lane);
                if (wave < 2) {  // wave 0: -LSE, wave 1: -D of the tile's rows
                    dma4(rs + wave * rows + r0, (uint32_t)(lane & (BN - 1)) * 4u, lds + S::RING + ((t & 1) * 2 + wave) * 256);
                }
            };
            __syncthreads();  // the head before is done with the table and the ring
            fill_table<CAUSAL>(tab, a.bias, h, 1, tid, NW * 64);
            request(tile0);
            __syncthreads();
            const float t_behind = tab[0], t_ahead = tab[len - 1];
            for (int t = tile0; t < tile1; t++) {
                wait_vmcnt<0>();
                wg_barrier();
                if (t + 1 < tile1) request(t + 1);
                const char *sQ = smem + (t & 1) * 2 * S::TILE, *sDO = sQ + S::TILE;
                const float *nl = scal + (t & 1) * 128, *nd = nl + 64;
#pragma unroll
                for (int qb32 = 0; qb32 < BN / 32; qb32++) {
                    const int q0 = smp.start + t * BN + qb32 * 32;  // positions of the block's rows
                    // the kinds as seen from the queries: keys kw0 .. kw0 + 31 against positions q0 .. q0 + 31
                    const Kind kind = kind_of<CAUSAL>(kw0, q0, q0 + 31, M, smp.length);
                    if (kind == Kind::SKIP) continue;
                    f32x16 s, dp16;
                    if (kind == Kind::NEAR) {
                        const float *my = tab + key - q0 - 4 * hf + M + kPad;
#pragma unroll
                        for (int e = 0; e < 16; e++) s[e] = my[-(8 * (e >> 2) + (e & 3))];
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; e++) s[e] = kind == Kind::FAR_BEHIND ? t_behind : t_ahead;
                    }
#pragma unroll
                    for (int q4 = 0; q4 < 4; q4++) {
                        const f32x4 x = *reinterpret_cast<const f32x4 *>(nd + qb32 * 32 + 4 * hf + 8 * q4);
#pragma unroll
                        for (int e = 0; e < 4; e++) dp16[4 * q4 + e] = x[e];
                    }
#pragma unroll
                    for (int st = 0; st < RowsT::STEPS; st++) {
                        s = Op<T>::mma(RowsT::read(sQ, rl, qb32 * 32, st), kf[st], s);
                        dp16 = Op<T>::mma(RowsT::read(sDO, rl, qb32 * 32, st), vf[st], dp16);
                    }
#pragma unroll
                    for (int q4 = 0; q4 < 4; q4++) {
                        const f32x4 x = *reinterpret_cast<const f32x4 *>(nl + qb32 * 32 + 4 * hf + 8 * q4);
#pragma unroll
                        for (int e = 0; e < 4; e++) s[4 * q4 + e] = fast_exp2(fmaf(s[4 * q4 + e], a.scale_log2, x[e]));
                    }
                    {
                        const Weights<T> w(s);
#pragma unroll
                        for (int j = 0; j < RowsT::BLOCKS; j++) dv[j] = RowsT::weigh(sDO, tl, lane, qb32 * 32, j, w, dv[j]);
                    }
#pragma unroll
                    for (int e = 0; e < 16; e++) s[e] *= dp16[e];
                    const Weights<T> w(s);
#pragma unroll
                    for (int j = 0; j < RowsT::BLOCKS; j++) dk[j] = RowsT::weigh(sQ, tl, lane, qb32 * 32, j, w, dk[j]);
                }
            }
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

// dbias of one head: the workgroups' sums by distance added up in their order, then the distances of a bucket
__global__ __launch_bounds__(1024) void k_rel_dbias(RelBwdArgs a, int parts, int len, int causal)
{
    extern __shared__ float dist[];  // [len]
    const int h = blockIdx.x, tid = threadIdx.x, M = a.bias.max_distance;
    for (int x = tid; x < len; x += 1024) {
        float sum = 0.f;
        const float *p = a.bins + (size_t)h * parts * len + x;
        for (int u = 0; u < parts; u++) sum += p[(size_t)u * len];
        dist[x] = sum;
    }
    __syncthreads();
    const int lane = tid & 63;
    for (int u = tid >> 6; u < a.bias.n_buckets; u += 16) {
        float sum = 0.f;
        for (int x = lane; x < len; x += 64) {
            const int d = x - M - kPad;
            if (causal && d > 0) continue;
            if (min(max(a.bias.table[min(max(d, -M), M) + M], 0), a.bias.n_buckets - 1) == u) sum += dist[x];
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
        if (lane == 0) {
            if (a.bias.bf16)
                ((__bf16 *)a.d_bias)[(size_t)u * a.heads + h] = (__bf16)sum;
            else
                ((float *)a.d_bias)[(size_t)u * a.heads + h] = sum;
        }
    }
}

template <typename T, int D>
hdt_status_t launch(const RelBwdArgs &a, bool causal, hipStream_t st)
{
    using S = BwdShape<T, D>;
    const int len = table_length(a.bias.max_distance, causal);
    const long long rows = (long long)a.batch * a.heads * a.n_pad;
    if (rows > 0) {
        HdtTimer t("hdt_rel_rows", st);
        constexpr int PER = 256 / (D / 8);
        hipLaunchKernelGGL((k_rel_rows<T, D>), dim3((unsigned)((rows + PER - 1) / PER)), dim3(256), 0, st, a, rows);
        HDT_HIP_TRY(hipGetLastError());
    }
    const size_t lds_q = S::RING + (size_t)len * (1 + 2 * S::NW) * sizeof(float), lds_k = S::RING + S::SCALARS + (size_t)len * sizeof(float);
    if (rows > 0) {
        HdtTimer t("hdt_rel_dq", st);
        const dim3 grid((unsigned)((long long)a.batch * a.heads * a.tiles_q));
        const void *f = causal ? (const void *)k_rel_dq<T, D, true> : (const void *)k_rel_dq<T, D, false>;
        if (lds_q > 65536) HDT_HIP_TRY(hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_q));
        if (causal)
            hipLaunchKernelGGL((k_rel_dq<T, D, true>), grid, dim3(S::NW * 64), lds_q, st, a);
        else
            hipLaunchKernelGGL((k_rel_dq<T, D, false>), grid, dim3(S::NW * 64), lds_q, st, a);
        HDT_HIP_TRY(hipGetLastError());
    }
    if (a.batch > 0 && a.tiles_k > 0) {
        HdtTimer t("hdt_rel_dkv", st);
        const dim3 grid((unsigned)((long long)a.batch * a.kv_heads * a.tiles_k));
        const void *f = causal ? (const void *)k_rel_dkv<T, D, true> : (const void *)k_rel_dkv<T, D, false>;
        if (lds_k > 65536) HDT_HIP_TRY(hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_k));
        if (causal)
            hipLaunchKernelGGL((k_rel_dkv<T, D, true>), grid, dim3(S::NW * 64), lds_k, st, a);
        else
            hipLaunchKernelGGL((k_rel_dkv<T, D, false>), grid, dim3(S::NW * 64), lds_k, st, a);
        HDT_HIP_TRY(hipGetLastError());
    }
    if (a.heads == 0) return HDT_OK;
    HdtTimer t("hdt_rel_dbias", st);
    hipLaunchKernelGGL(k_rel_dbias, dim3((unsigned)a.heads), dim3(1024), len * sizeof(float), st, a, a.batch * a.tiles_q, len, causal ? 1 : 0);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

}  // namespace

RelBwdPlan hdt_rel_bwd_plan(const hdt_rel_attn_t &d)
{
    RelBwdPlan p;
    p.tiles_q = (d.n_q + 127) / 128;
    p.tiles_k = (d.n_kv + 127) / 128;
    p.n_pad = (d.n_q + 127) & ~127;
    const size_t rows = (size_t)d.batch * d.heads * p.n_pad;
    p.bins_at = (2 * rows * sizeof(float) + 255) & ~(size_t)255;
    p.bytes = p.bins_at + (size_t)d.heads * d.batch * p.tiles_q * table_length(d.max_distance, d.causal != 0) * sizeof(float);
    return p;
}

hdt_status_t hdt_launch_rel_bwd(const hdt_rel_attn_t &d, const RelBwdArgs &a, hipStream_t st)
{
    const bool causal = d.causal != 0;
    if (d.dtype == HDT_BF16) return d.head_dim == 64 ? launch<__bf16, 64>(a, causal, st) : launch<__bf16, 128>(a, causal, st);
    return d.head_dim == 64 ? launch<float, 64>(a, causal, st) : launch<float, 128>(a, causal, st);
}
