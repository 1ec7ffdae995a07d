// Forward pass of self-attention with a relative position bias (hdt_rel.h has the mathematics and the block kinds).
//
// Work split: one workgroup per (sample, head block, tile of 128 rows, piece of the keys); wave w owns rows 32w .. 32w + 31 of the
// tile.  Rows are the queries of one head, or, where a head has fewer queries than a tile has rows, the queries of all heads that
// share a key head, so that the keys are read once for them (PACK: row r is query r / gp of head r % gp).  Key tiles of BN rows
// go through a ring of two stages in LDS.
#include <type_traits>

#include "hdt_rel.h"
#include "hdt_rel_args.h"

namespace {

using namespace hdt_rel;

template <typename T, int D>
struct FwdShape {
    static constexpr int NW = 4, BM = 32 * NW, BN = sizeof(T) == 4 && D == 128 ? 32 : 64;
    static constexpr int RING = 2 * Pair<T, D, BN, NW>::STAGE;
};

template <typename T, int D, bool CAUSAL>
__global__ __launch_bounds__(256, sizeof(T) == 4 && D == 128 ? 1 : 2) void k_rel_fwd(RelFwdArgs a)
{
    using S = FwdShape<T, D>;
    using RowsT = Rows<T, D>;
    constexpr int BM = S::BM, BN = S::BN, NW = S::NW, KB = BN / 32;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    float *const tab = reinterpret_cast<float *>(smem + S::RING);

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    // the longest tiles first; the head blocks side by side, so that with a multiple of 8 of them each stays on one XCD and in its L2
    const unsigned heads = (unsigned)(a.batch * a.head_blocks), tp = blockIdx.x / heads, piece = tp % a.pieces;
    const int bh = blockIdx.x - tp * heads, I = a.tiles - 1 - (int)(tp / a.pieces), b = bh / a.head_blocks, hb = bh - b * a.head_blocks;
    const int gp = a.gp, n_rows = a.n_q * gp, M = a.bias.max_distance;
    const Sample smp = sample_of(a.lengths, a.starts, b, a.n_q, a.n_kv);

    const int r0 = I * BM, first = max(r0, smp.lo * gp), last = min(r0 + BM, smp.hi * gp) - 1;
    const int row = r0 + wave * 32 + (lane & 31);
    const bool own = row < n_rows, real = row >= first && row <= last;
    int tile0 = 0, tile1 = 0, seen = 0;
    if (first <= last) {
        seen = CAUSAL ? smp.start + last / gp + 1 : smp.length;
        const int all = (seen + BN - 1) / BN, per = (all + (int)a.pieces - 1) / (int)a.pieces;
        tile0 = min((int)piece * per, all);
        tile1 = min(tile0 + per, all);
    }
    // rows that are not real take part as copies of one that is, and are not stored
    const int rc = min(max(row, first), max(first, last)), qi = rc / gp, g = rc - qi * gp, pos = smp.start + qi;
    const int w0 = max(r0 + wave * 32, first), w1 = min(r0 + wave * 32 + 31, last), p0 = smp.start + w0 / gp, p1 = smp.start + w1 / gp;

    f32x16 acc[RowsT::BLOCKS];
#pragma unroll
    for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[j][e] = 0.f;
    float m_ref = -INFINITY, l_part = 0.f;

    if (tile0 < tile1) {
        const size_t kvh = (size_t)(hb * gp / a.group);
        Pair<T, D, BN, NW> kv;
        kv.init((const T *)a.k + (size_t)b * a.sk.batch + kvh * a.sk.head, a.sk.row, (const T *)a.v + (size_t)b * a.sv.batch + kvh * a.sv.head,
                a.sv.row, smem, wave, lane);
        typename RowsT::Frag qf[RowsT::STEPS];
        const char *qp = (const char *)((const T *)a.q + (size_t)b * a.sq.batch + (size_t)(hb * gp + g) * a.sq.head + (size_t)qi * a.sq.row);
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) qf[st] = *reinterpret_cast<const typename RowsT::Frag *>(qp + (2 * st + hf) * 16);
        fill_table<CAUSAL>(tab, a.bias, hb * gp, gp, tid, NW * 64);
        kv.request(tile0 * BN, 0, seen - 1, 0);
        const int len = table_length(M, CAUSAL);
        const float *const my_tab = tab + g * len + 4 * hf - pos + M + kPad;
        const RowLane rl = row_lane<RowsT::CPR>(lane);
        const TrLane tl = tr_lane<RowsT::CPR>(lane);
        __syncthreads();
        const float c_behind = tab[g * len] * a.scale_log2, c_ahead = CAUSAL ? 0.f : tab[g * len + len - 1] * a.scale_log2;

        // one tile of keys, in stage ST of the ring (a constant: the LDS addresses of both stages are then offsets of the same registers)
        auto tile = [&](int t, auto stage) {
            constexpr int ST = decltype(stage)::value;
            wait_vmcnt<0>();
            wg_barrier();
            if (t + 1 < tile1) kv.request((t + 1) * BN, 0, seen - 1, 1 - ST);
            const char *sK = smem + ST * kv.STAGE, *sV = sK + kv.TILE;
            const int k0 = t * BN;
            const Kind kind = kind_of<CAUSAL, BN>(k0, p0, p1, M, smp.length);
            if (kind == Kind::SKIP || w0 > w1) return;  // (nor has a wave without real rows anything to do)
            f32x16 s[KB];
            float c = 0.f;
            if (kind == Kind::NEAR) {
#pragma unroll
                for (int kb = 0; kb < KB; kb++) {
#pragma unroll
                    for (int e = 0; e < 16; e++) s[kb][e] = my_tab[k0 + 32 * kb + 8 * (e >> 2) + (e & 3)];
                    s[kb] = Op<T>::mma(RowsT::read(sK, rl, kb * 32, 0), qf[0], s[kb]);
                }
            } else {
                c = kind == Kind::FAR_BEHIND ? c_behind : c_ahead;
#pragma unroll
                for (int kb = 0; kb < KB; kb++) {
#pragma unroll
                    for (int e = 0; e < 16; e++) s[kb][e] = 0.f;
                    s[kb] = Op<T>::mma(RowsT::read(sK, rl, kb * 32, 0), qf[0], s[kb]);
                }
            }
#pragma unroll
            for (int st = 1; st < RowsT::STEPS; st++)
#pragma unroll
                for (int kb = 0; kb < KB; kb++) s[kb] = Op<T>::mma(RowsT::read(sK, rl, kb * 32, st), qf[st], s[kb]);
            if (!CAUSAL && k0 + BN > smp.length) {
#pragma unroll
                for (int kb = 0; kb < KB; kb++)
#pragma unroll
                    for (int e = 0; e < 16; e++) s[kb][e] = k0 + 32 * kb + 4 * hf + 8 * (e >> 2) + (e & 3) < smp.length ? s[kb][e] : -INFINITY;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < KB; kb++)
#pragma unroll
                for (int e = 0; e < 16; e += 2) mx = fmaxf(mx, fmaxf(s[kb][e], s[kb][e + 1]));
            mx = fmaf(max_halves(mx), a.scale_log2, c);
            if (__any(mx > m_ref + 8.f)) {
                const float m_new = fmaxf(m_ref, mx), alpha = m_new == -INFINITY ? 1.f : fast_exp2(m_ref - m_new);
                m_ref = m_new;
                l_part *= alpha;
#pragma unroll
                for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
                    for (int e = 0; e < 16; e++) acc[j][e] *= alpha;
            }
            const float off = c - (m_ref == -INFINITY ? 0.f : m_ref);
#pragma unroll
            for (int kb = 0; kb < KB; kb++) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    s[kb][e] = fast_exp2(fmaf(s[kb][e], a.scale_log2, off));
                    sum += s[kb][e];
                }
                l_part += sum;
                const Weights<T> w(s[kb]);
#pragma unroll
                for (int j = 0; j < RowsT::BLOCKS; j++) acc[j] = RowsT::weigh(sV, tl, lane, kb * 32, j, w, acc[j]);
            }
        };
        int t = tile0;
        for (; t + 1 < tile1; t += 2) {
            tile(t, std::integral_constant<int, 0>());
            tile(t + 1, std::integral_constant<int, 1>());
        }
        if (t < tile1) tile(t, std::integral_constant<int, 0>());
    }

    const float l_tot = sum_halves(l_part);
    const float inv = real && l_tot > 0.f ? 1.f / l_tot : 0.f;
    const float lse = real && l_tot > 0.f ? (m_ref + __builtin_amdgcn_logf(l_tot)) * LN2 : -INFINITY;
    if (!own) return;
    const int oi = row / gp, og = row - oi * gp, head = hb * gp + og;
    if (a.pieces > 1) {
        const size_t at = ((size_t)bh * n_rows + row) * a.pieces + piece;
        float *o = a.part_o + at * D;
#pragma unroll
        for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
            for (int q4 = 0; q4 < 4; q4++) {
                f32x4 x;
#pragma unroll
                for (int e = 0; e < 4; e++) x[e] = acc[j][q4 * 4 + e] * inv;
                *reinterpret_cast<f32x4 *>(o + 32 * j + 8 * q4 + 4 * hf) = x;
            }
        if (hf == 0) a.part_lse[at] = lse;
        return;
    }
    T *o = (T *)a.o + (size_t)b * a.so.batch + (size_t)head * a.so.head + (size_t)oi * a.so.row;
#pragma unroll
    for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
        for (int q4 = 0; q4 < 4; q4++)
            store4(o + 32 * j + 8 * q4 + 4 * hf, acc[j][q4 * 4] * inv, acc[j][q4 * 4 + 1] * inv, acc[j][q4 * 4 + 2] * inv, acc[j][q4 * 4 + 3] * inv);
    if (hf == 0) a.lse[((size_t)b * a.heads + head) * a.n_q + oi] = lse;
}

// O = sum_p exp(LSE_p - LSE) O_p, LSE = log sum_p exp(LSE_p) over the pieces of a row's keys, in their order
template <typename T, int D>
__global__ __launch_bounds__(256) void k_rel_join(RelFwdArgs a, long long rows)
{
    constexpr int LANES = D / 4, PER = 256 / LANES;
    const long long r = (long long)blockIdx.x * PER + threadIdx.x / LANES;
    if (r >= rows) return;
    const int c = threadIdx.x % LANES, n_rows = a.n_q * a.gp;
    const float *pl = a.part_lse + r * a.pieces;
    float top = -INFINITY;
    for (unsigned p = 0; p < a.pieces; p++) top = fmaxf(top, pl[p]);
    float sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (unsigned p = 0; p < a.pieces; p++) {
        const float l = pl[p];
        if (l == -INFINITY) continue;
        const float w = fast_exp2((l - top) * LOG2E);
        const f32x4 x = *reinterpret_cast<const f32x4 *>(a.part_o + ((size_t)r * a.pieces + p) * D + 4 * c);
        sum += w;
#pragma unroll
        for (int e = 0; e < 4; e++) acc[e] = fmaf(w, x[e], acc[e]);
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const int bh = (int)(r / n_rows), row = (int)(r - (long long)bh * n_rows), b = bh / a.head_blocks, hb = bh - b * a.head_blocks;
    const int i = row / a.gp, head = hb * a.gp + row - i * a.gp;
    store4((T *)a.o + (size_t)b * a.so.batch + (size_t)head * a.so.head + (size_t)i * a.so.row + 4 * c, acc[0] * inv, acc[1] * inv,
           acc[2] * inv, acc[3] * inv);
    if (c == 0) a.lse[((size_t)b * a.heads + head) * a.n_q + i] = sum > 0.f ? top + __builtin_amdgcn_logf(sum) * LN2 : -INFINITY;
}

template <typename T, int D>
hdt_status_t launch(const RelFwdArgs &a, bool causal, hipStream_t st)
{
    using S = FwdShape<T, D>;
    const size_t lds = S::RING + (size_t)a.gp * table_length(a.bias.max_distance, causal) * sizeof(float);
    const long long bh = (long long)a.batch * a.head_blocks;
    const dim3 grid((unsigned)(bh * a.tiles * a.pieces)), block(S::NW * 64);
    {
        HdtTimer t("hdt_rel_fwd", st);
        const void *f = causal ? (const void *)k_rel_fwd<T, D, true> : (const void *)k_rel_fwd<T, D, false>;
        if (lds > 65536) HDT_HIP_TRY(hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        if (causal)
            hipLaunchKernelGGL((k_rel_fwd<T, D, true>), grid, block, lds, st, a);
        else
            hipLaunchKernelGGL((k_rel_fwd<T, D, false>), grid, block, lds, st, a);
        HDT_HIP_TRY(hipGetLastError());
    }
    if (a.pieces > 1) {
        HdtTimer t("hdt_rel_join", st);
        const long long rows = bh * a.n_q * a.gp;
        constexpr int PER = 256 / (D / 4);
        hipLaunchKernelGGL((k_rel_join<T, D>), dim3((unsigned)((rows + PER - 1) / PER)), dim3(256), 0, st, a, rows);
        HDT_HIP_TRY(hipGetLastError());
    }
    return HDT_OK;
}

}  // namespace

RelFwdPlan hdt_rel_fwd_plan(const hdt_rel_attn_t &d)
{
    RelFwdPlan p;
    constexpr int BM = 128, BN = 64;
    const int group = d.heads / d.kv_heads;
    // queries of the heads that share a key head together, where one head's do not fill a tile of rows (and the heads' tables fit)
    p.gp = d.n_q < BM && (size_t)group * table_length(d.max_distance, d.causal != 0) * sizeof(float) <= 32768 ? group : 1;
    p.head_blocks = d.heads / p.gp;
    p.tiles = (d.n_q * p.gp + BM - 1) / BM;
    const long long items = (long long)d.batch * p.head_blocks * p.tiles, key_tiles = (d.n_kv + BN - 1) / BN;
    long long pieces = items >= 512 ? 1 : (512 + items - 1) / items;
    if (pieces > (key_tiles + 1) / 2) pieces = (key_tiles + 1) / 2;
    p.pieces = pieces < 1 ? 1 : (unsigned)pieces;
    const size_t rows = (size_t)d.batch * d.heads * d.n_q;
    p.lse_at = rows * p.pieces * d.head_dim * sizeof(float);
    p.bytes = p.pieces > 1 ? p.lse_at + rows * p.pieces * sizeof(float) : 0;
    return p;
}

hdt_status_t hdt_launch_rel_fwd(const hdt_rel_attn_t &d, const RelFwdArgs &a, hipStream_t st)
{
    const bool causal = d.causal != 0;
    if (d.dtype == HDT_BF16) return d.head_dim == 64 ? launch<__bf16, 64>(a, causal, st) : launch<__bf16, 128>(a, causal, st);
    return d.head_dim == 64 ? launch<float, 64>(a, causal, st) : launch<float, 128>(a, causal, st);
}
