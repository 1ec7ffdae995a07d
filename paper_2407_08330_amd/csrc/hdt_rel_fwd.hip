// Forward pass of self-attention with a relative position bias (hdt_rel.h has the mathematics and the block kinds).
//
// Work split: one workgroup per (sample, head block, tile of rows, piece of the keys); a wave owns 32 rows, whose S, P and O stay in its
// registers: S^T = K Q^T leaves a row's pairs in one lane pair, so that the softmax needs one exchange a tile, and P^T is already the operand
// of O^T += V^T P^T.  A tile is 128 rows of 4 waves, or 64 or 32 rows whose workgroup has as many waves, which take every second or fourth
// key tile and join in LDS (hdt_rel_row_waves).  Rows are the queries of one head, or, where a head has fewer queries than a tile has rows,
// the queries of all heads that share a key head, so that the keys are read once for them (row r is query r / gp of head r % gp).  Key tiles
// of BN rows go through a ring of two stages in LDS, loaded directly.
//
// P is rounded to bf16 for its product with V (as the operand of the fast contraction has to be), after its sum is taken in fp32; the
// reference of the exponentials follows the maximum only from a factor 2^8 on, which saves rescaling and costs nothing in fp32 or bf16.
//
// What bounds it: vector instructions (an exponential, a fused multiply-add, a sum, half a maximum and half a conversion for each pair) next
// to the matrix ones.  24 heads x 8192 x 64, causal: 232-243 us, 0.85-0.89 PFLOP/s, vector pipe issuing 68 % and matrix pipe busy 41 % of all
// clocks.  32 heads x 4096 x 128: 150 us, 0.91.  (Tried on the first: no maximum unless a row's sum is large, with the contraction taken
// again then, 170 registers and a wave less a SIMD: 231 -> 243; sums by dot products of the rounded weights: 2 % quicker, but LSE then has
// bf16's errors; two blocks of rows a wave, which share the operands from LDS,
// at two waves a SIMD: 241 -> 257; more operands ahead, wave priorities around the contractions: within 1 %.)
#include <algorithm>
#include <type_traits>

#include "hdt_rel.h"
#include "hdt_rel_args.h"

namespace {

using namespace hdt_rel;

constexpr int kAheadK = 4, kAheadV = 4;  // operands on their way from LDS

// KS: groups of NW waves that take every KS-th key tile, each through a ring of its own, and join at the end.  Where there are few row
// tiles a wave's walk along the keys is what takes the time, and this shortens it.
template <typename T, int D, int NW_, int KS_>
struct FwdShape {
    static constexpr int NW = NW_, KS = KS_, THREADS = NW * KS * 64, BM = 32 * NW, BN = sizeof(T) == 4 ? 32 : 64;
    static constexpr int RING = 2 * Pair<T, D, BN, NW>::STAGE;
};

template <typename T, int D, int NW_, int KS_, bool CAUSAL>
__global__ __launch_bounds__(NW_ * KS_ * 64, sizeof(T) == 4 && D == 128 ? 1 : 2) void k_rel_fwd(RelFwdArgs a)
{
    using S = FwdShape<T, D, NW_, KS_>;
    using RowsT = Rows<T, D>;
    constexpr int BM = S::BM, BN = S::BN, NW = S::NW, KS = S::KS, KB = BN / 32;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    float *const tab = reinterpret_cast<float *>(smem + KS * S::RING);

    const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
    const int wave_all = __builtin_amdgcn_readfirstlane(tid >> 6), grp = KS > 1 ? wave_all / NW : 0, wave = wave_all - grp * NW;
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
                a.sv.row, smem + grp * S::RING, wave, lane);
        typename RowsT::Frag qf[RowsT::STEPS];
        const char *qp = (const char *)((const T *)a.q + (size_t)b * a.sq.batch + (size_t)(hb * gp + g) * a.sq.head + (size_t)qi * a.sq.row);
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) qf[st] = *reinterpret_cast<const typename RowsT::Frag *>(qp + (2 * st + hf) * 16);
        if (tile0 + grp < tile1) kv.request((tile0 + grp) * BN, 0, seen - 1, 0);
        fill_table(tab, a.bias, hb * gp, gp, CAUSAL, tid, S::THREADS);
        const int len = table_length(M, CAUSAL);
        const float *const my_tab = tab + g * len + 4 * hf - pos + M + kPad;
        const RowLane rl = row_lane<RowsT::CPR>(lane);
        const TrLane tl = tr_lane<RowsT::CPR>(lane);
        __syncthreads();
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) settle(qf[st]);
        const float c_behind = tab[g * len] * a.scale_log2, c_ahead = CAUSAL ? 0.f : tab[g * len + len - 1] * a.scale_log2;

        auto tile = [&](int round, auto stage) {  // one tile of keys
            const int ST = stage, t = tile0 + round * KS + grp;
            wait_vmcnt<0>();
            wg_barrier();
            if (t + KS < tile1) kv.request((t + KS) * BN, 0, seen - 1, 1 - ST);
            const char *sK = smem + grp * S::RING + ST * kv.STAGE, *sV = sK + kv.TILE;
            const int k0 = t * BN;
            const Kind kind = kind_of<CAUSAL, BN>(k0, p0, p1, M, smp.length);
            if (kind == Kind::SKIP || w0 > w1 || (KS > 1 && t >= tile1)) return;  // (nor has a wave without real rows anything to do)
            f32x16 s[KB];
            float c = 0.f;
            auto read_k = [&](int i) { return RowsT::read(sK, rl, i % KB * 32, i / KB); };
            auto k_ahead = ahead<KB * RowsT::STEPS, kAheadK, typename RowsT::Frag>(read_k);
            if (kind == Kind::NEAR) {
#pragma unroll
                for (int kb = 0; kb < KB; kb++)
#pragma unroll
                    for (int e = 0; e < 16; e++) s[kb][e] = my_tab[k0 + 32 * kb + 8 * (e >> 2) + (e & 3)];
                k_ahead.run([&](int i, typename RowsT::Frag f) { s[i % KB] = Op<T>::mma(f, qf[i / KB], s[i % KB]); });
            } else {
                c = kind == Kind::FAR_BEHIND ? c_behind : c_ahead;
                const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                k_ahead.run([&](int i, typename RowsT::Frag f) { s[i % KB] = Op<T>::mma(f, qf[i / KB], i < KB ? zero : s[i % KB]); });
            }
            auto read_v = [&](int i) { return RowsT::wread(sV, tl, lane, i / (RowsT::WSTEPS * RowsT::BLOCKS) * 32, i % RowsT::BLOCKS, i / RowsT::BLOCKS % RowsT::WSTEPS); };
            auto v_ahead = ahead<KB * RowsT::WSTEPS * RowsT::BLOCKS, kAheadV, typename RowsT::WFrag>(read_v);
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
            Weights<T> w[KB];
#pragma unroll
            for (int kb = 0; kb < KB; kb++) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    s[kb][e] = fast_exp2(fmaf(s[kb][e], a.scale_log2, off));
                    sum += s[kb][e];
                }
                l_part += sum;
                w[kb] = Weights<T>(s[kb]);
            }
            v_ahead.run([&](int i, typename RowsT::WFrag f) {
                acc[i % RowsT::BLOCKS] = RowsT::wmma(f, w[i / (RowsT::WSTEPS * RowsT::BLOCKS)], i / RowsT::BLOCKS % RowsT::WSTEPS, acc[i % RowsT::BLOCKS]);
            });
        };
        walk<true>((tile1 - tile0 + KS - 1) / KS, tile);  // (barriers are the whole workgroup's: every group takes the same number of rounds)
    }

    if constexpr (KS > 1) {  // the groups' results, in their order, a wave's beside those of the same rows
        constexpr int REGS = 16 * RowsT::BLOCKS + 2;
        static_assert((KS - 1) * NW * REGS * 256 <= KS * S::RING, "they fit the rings");
        float *const at = reinterpret_cast<float *>(smem) + lane;
        __syncthreads();
        if (grp > 0) {
            float *const to = at + ((grp - 1) * NW + wave) * REGS * 64;
            to[0] = m_ref, to[64] = l_part;
#pragma unroll
            for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
                for (int e = 0; e < 16; e++) to[(2 + 16 * j + e) * 64] = acc[j][e];
        }
        __syncthreads();
        if (grp > 0) return;
#pragma unroll
        for (int k = 1; k < KS; k++) {
            const float *const from = at + ((k - 1) * NW + wave) * REGS * 64;
            const float m = from[0], top = fmaxf(m, m_ref), w = m == -INFINITY ? 0.f : fast_exp2(m - top), own_w = m_ref == -INFINITY ? 0.f : fast_exp2(m_ref - top);
            m_ref = top;
            l_part = l_part * own_w + from[64] * w;
#pragma unroll
            for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
                for (int e = 0; e < 16; e++) acc[j][e] = acc[j][e] * own_w + from[(2 + 16 * j + e) * 64] * w;
        }
    }
    // rows on their way out: behind what the joining used
    char *const out_lds = smem + (KS - 1) * NW * (16 * RowsT::BLOCKS + 2) * 256 + wave * 32 * D * 4;
    static_assert((KS - 1) * NW * (16 * RowsT::BLOCKS + 2) * 256 + NW * 32 * D * 4 <= KS * S::RING, "they fit the rings");
    const float l_tot = sum_halves(l_part);
    const bool any = real && !no_weight(l_tot);  // (a NaN in the row or in a key it sees: O and LSE are NaN)
    const float inv = 1.f / l_tot, lse = any ? (m_ref + __builtin_amdgcn_logf(l_tot)) * LN2 : -INFINITY;
    const int oi = row / gp, og = row - oi * gp, head = hb * gp + og;
    if (a.pieces > 1) {
        if (KS == 1) __syncthreads();  // (the ring is free)
        const size_t at = (size_t)bh * n_rows + r0 + wave * 32;
        store_rows<float, D>(out_lds, lane, acc, any, inv, a.part_o + (at * a.pieces + piece) * D, (int64_t)a.pieces * D, n_rows - r0 - wave * 32);
        if (own && hf == 0) a.part_lse[(at + (lane & 31)) * a.pieces + piece] = lse;
        return;
    }
    if (own && hf == 0) a.lse[((size_t)b * a.heads + head) * a.n_q + oi] = lse;
    T *const o = (T *)a.o + (size_t)b * a.so.batch;
    if (gp == 1) {
        if (KS == 1) __syncthreads();
        store_rows<T, D>(out_lds, lane, acc, any, inv, o + (size_t)hb * a.so.head + (size_t)(r0 + wave * 32) * a.so.row, a.so.row, n_rows - r0 - wave * 32);
        return;
    }
    if (!own) return;
    T *const to = o + (size_t)head * a.so.head + (size_t)oi * a.so.row;  // (rows of several heads)
#pragma unroll
    for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
        for (int q4 = 0; q4 < 4; q4++)
            store4(to + 32 * j + 8 * q4 + 4 * hf, any ? acc[j][q4 * 4] * inv : 0.f, any ? acc[j][q4 * 4 + 1] * inv : 0.f,
                   any ? acc[j][q4 * 4 + 2] * inv : 0.f, any ? acc[j][q4 * 4 + 3] * inv : 0.f);
}

// Few rows (at most 32 in a head block: new tokens): the waves of a workgroup divide the keys instead of the rows.  Each walks blocks of
// 32 keys through a ring of its own (no barriers; 128 KB of blocks in flight a workgroup, which the stream from memory wants) and they join
// what they have in LDS.  8 waves with two blocks of 128-byte rows each, or one of 256: those take turns (us, rows of 256 bytes, 4 waves of
// two | 8 of one: 1000 keys of 1 head 14.2 | 12.3, 8192 keys of 256 186 | 186; rows of 128, 8 of two | 16 of one: 8.2 | 8.4, 92 | 95).
// Bound by reading K and V once: 32 x 4 key heads of 128, 8192 ragged keys (403 MB), 80 us and 4 for joining the pieces, 4.8 TB/s.  One
// token over 1000 keys of 12 heads of 64: 8 us: arguments and lengths 1.2, bias by distance and first keys 1.5, four blocks a wave 2.6,
// the join 1.9.
template <typename T, int D>
struct FewShape {
    static constexpr int ROWB = Rows<T, D>::ROWB, NI = 32 * ROWB / 1024, TILE = 32 * ROWB, STAGE = 2 * TILE;
    static constexpr int NW = ROWB <= 256 ? 8 : 4, STAGES = 128 * 1024 / (NW * STAGE), RING = STAGES * STAGE;
    static_assert(STAGES == 1 || STAGES == 2, "as the kernel's waits count");
    static_assert(NW * 32 * (D + 2) * 4 <= NW * RING + 8192, "the waves' references, sums and O fit");
    static constexpr int LDS = NW * RING + 8192;
};

template <typename T, int D, bool CAUSAL>
__global__ __launch_bounds__((FewShape<T, D>::NW * 64)) void k_rel_few(RelFwdArgs a)
{
    using S = FewShape<T, D>;
    using RowsT = Rows<T, D>;
    constexpr int NW = S::NW, NI = S::NI;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    float *const tab = reinterpret_cast<float *>(smem + S::LDS);

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5;
    const unsigned heads = (unsigned)(a.batch * a.head_blocks), piece = blockIdx.x / heads;
    const int bh = blockIdx.x - piece * heads, b = bh / a.head_blocks, hb = bh - b * a.head_blocks;
    const int gp = a.gp, n_rows = a.n_q * gp, M = a.bias.max_distance;
    const Sample smp = sample_of(a.lengths, a.starts, b, a.n_q, a.n_kv);
    const int first = smp.lo * gp, last = smp.hi * gp - 1;
    int block0 = 0, block1 = 0, seen = 0;  // this piece's blocks of 32 keys
    if (first <= last) {
        seen = CAUSAL ? smp.start + last / gp + 1 : smp.length;
        const int all = (seen + 31) / 32, per = (all + (int)a.pieces - 1) / (int)a.pieces;
        block0 = min((int)piece * per, all);
        block1 = min(block0 + per, all);
    }
    const int row = lane & 31, rc = min(max(row, first), max(first, last)), qi = rc / gp, g = rc - qi * gp, pos = smp.start + qi;
    const int p0 = smp.start + smp.lo, p1 = smp.start + smp.hi - 1;

    f32x16 acc[RowsT::BLOCKS];
#pragma unroll
    for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[j][e] = 0.f;
    float m_ref = -INFINITY, l_part = 0.f;

    if (block0 < block1) {
        const size_t kvh = (size_t)(hb * gp / a.group);
        const char *kb = (const char *)((const T *)a.k + (size_t)b * a.sk.batch + kvh * a.sk.head);
        const char *vb = (const char *)((const T *)a.v + (size_t)b * a.sv.batch + kvh * a.sv.head);
        const uint32_t krow = (uint32_t)a.sk.row * sizeof(T), vrow = (uint32_t)a.sv.row * sizeof(T);
        const char *const mine = smem + wave * S::RING;
        const uint32_t lds = lds_addr(mine);
        auto request = [&](int blk, int stage) {
            const uint32_t at = lds + (uint32_t)(stage * S::STAGE);
            const char *pk = kb + (size_t)blk * 32 * krow, *pv = vb + (size_t)blk * 32 * vrow;
            const int left = seen - 1 - blk * 32, c = lane % RowsT::CPR;
#pragma unroll
            for (int i = 0; i < NI; i++) {
                const int r = i * RowsT::RPI + lane / RowsT::CPR;
                const uint32_t from = (uint32_t)min(r, left), chunk = (uint32_t)((c ^ swz<RowsT::CPR>(r)) << 4);
                dma16(pk, from * krow + chunk, at + i * 1024);
                dma16(pv, from * vrow + chunk, at + S::TILE + i * 1024);
            }
        };
        if (block0 + wave < block1) request(block0 + wave, 0);
        typename RowsT::Frag qf[RowsT::STEPS];
        const char *qp = (const char *)((const T *)a.q + (size_t)b * a.sq.batch + (size_t)(hb * gp + g) * a.sq.head + (size_t)qi * a.sq.row);
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) qf[st] = *reinterpret_cast<const typename RowsT::Frag *>(qp + (2 * st + hf) * 16);
        fill_table(tab, a.bias, hb * gp, gp, CAUSAL, tid, NW * 64);
        const int len = table_length(M, CAUSAL);
        const float *const my_tab = tab + g * len + 4 * hf - pos + M + kPad;
        const RowLane rl = row_lane<RowsT::CPR>(lane);
        const TrLane tl = tr_lane<RowsT::CPR>(lane);
        __syncthreads();
#pragma unroll
        for (int st = 0; st < RowsT::STEPS; st++) settle(qf[st]);
        const float c_behind = tab[g * len] * a.scale_log2, c_ahead = CAUSAL ? 0.f : tab[g * len + len - 1] * a.scale_log2;

        int stage = 0;
        for (int blk = block0 + wave; blk < block1; blk += NW, stage ^= S::STAGES - 1) {
            if (S::STAGES == 2) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the block before last has been read)
                if (blk + NW < block1) {
                    request(blk + NW, stage ^ 1);
                    wait_vmcnt<2 * NI>();
                } else {
                    wait_vmcnt<0>();
                }
            } else {
                if (blk != block0 + wave) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the block before has been read)
                    request(blk, 0);
                }
                wait_vmcnt<0>();
            }
            const char *sK = mine + stage * S::STAGE, *sV = sK + S::TILE;
            const int k0 = blk * 32;
            const Kind kind = kind_of<CAUSAL, 32>(k0, p0, p1, M, smp.length);
            if (kind == Kind::SKIP) continue;
            f32x16 s;
            float c = 0.f;
            if (kind == Kind::NEAR) {
#pragma unroll
                for (int e = 0; e < 16; e++) s[e] = my_tab[k0 + 8 * (e >> 2) + (e & 3)];
            } else {
                c = kind == Kind::FAR_BEHIND ? c_behind : c_ahead;
#pragma unroll
                for (int e = 0; e < 16; e++) s[e] = 0.f;
            }
#pragma unroll
            for (int st = 0; st < RowsT::STEPS; st++) s = Op<T>::mma(RowsT::read(sK, rl, 0, st), qf[st], s);
            if (!CAUSAL && k0 + 32 > smp.length) {
#pragma unroll
                for (int e = 0; e < 16; e++) s[e] = k0 + 4 * hf + 8 * (e >> 2) + (e & 3) < smp.length ? s[e] : -INFINITY;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; e += 2) mx = fmaxf(mx, fmaxf(s[e], s[e + 1]));
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
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 16; e++) {
                s[e] = fast_exp2(fmaf(s[e], a.scale_log2, off));
                sum += s[e];
            }
            l_part += sum;
            const Weights<T> w(s);
#pragma unroll
            for (int x = 0; x < RowsT::WSTEPS; x++)
#pragma unroll
                for (int j = 0; j < RowsT::BLOCKS; j++) acc[j] = RowsT::wmma(RowsT::wread(sV, tl, lane, 0, j, x), w, x, acc[j]);
        }
    }

    // the waves' results: references and sums [wave][32], O [wave][row][D], chunk c of four at c ^ (row & 15); joined in their order
    float *const ms = reinterpret_cast<float *>(smem), *const ls = ms + NW * 32, *const os = ls + NW * 32;
    const float l_tot = sum_halves(l_part);
    __syncthreads();
    if (hf == 0) ms[wave * 32 + row] = m_ref, ls[wave * 32 + row] = l_tot;
    if (row < n_rows) {
        float *const o = os + (wave * 32 + row) * D;
#pragma unroll
        for (int j = 0; j < RowsT::BLOCKS; j++)
#pragma unroll
            for (int q4 = 0; q4 < 4; q4++)
                *reinterpret_cast<f32x4 *>(o + (((8 * j + 2 * q4 + hf) ^ (row & 15)) << 2)) = f32x4{acc[j][4 * q4], acc[j][4 * q4 + 1], acc[j][4 * q4 + 2], acc[j][4 * q4 + 3]};
    }
    __syncthreads();
    for (int x = tid; x < n_rows * (D / 4); x += NW * 64) {
        const int r = x / (D / 4), c = x - r * (D / 4);
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; w++) top = fmaxf(top, ms[w * 32 + r]);
        float sum = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; w++) {
            const float m = ms[w * 32 + r], weight = m == -INFINITY ? 0.f : fast_exp2(m - top);
            const f32x4 y = *reinterpret_cast<const f32x4 *>(os + (w * 32 + r) * D + ((c ^ (r & 15)) << 2));
            sum = fmaf(weight, ls[w * 32 + r], sum);
#pragma unroll
            for (int e = 0; e < 4; e++) o[e] = fmaf(weight, y[e], o[e]);
        }
        const bool any = r >= first && r <= last && !no_weight(sum);
        const float inv = 1.f / sum, lse = any ? (top + __builtin_amdgcn_logf(sum)) * LN2 : -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] = any ? o[e] * inv : 0.f;
        const int i = r / gp, head = hb * gp + r - i * gp;
        if (a.pieces > 1) {
            const size_t at = ((size_t)bh * n_rows + r) * a.pieces + piece;
            *reinterpret_cast<f32x4 *>(a.part_o + at * D + 4 * c) = o;
            if (c == 0) a.part_lse[at] = lse;
        } else {
            store4((T *)a.o + (size_t)b * a.so.batch + (size_t)head * a.so.head + (size_t)i * a.so.row + 4 * c, o[0], o[1], o[2], o[3]);
            if (c == 0) a.lse[((size_t)b * a.heads + head) * a.n_q + i] = lse;
        }
    }
}

// O = sum_p exp(LSE_p - LSE) O_p, LSE = log sum_p exp(LSE_p) over the pieces of a row's keys, in their order, eight pieces requested at
// a time
template <typename T, int D>
__global__ __launch_bounds__(256) void k_rel_join(RelFwdArgs a, long long rows)
{
    constexpr int LANES = D / 4, PER = 256 / LANES, U = 8;
    const long long r = (long long)blockIdx.x * PER + threadIdx.x / LANES;
    if (r >= rows) return;
    const int c = threadIdx.x % LANES, n_rows = a.n_q * a.gp, pieces = (int)a.pieces;
    const float *pl = a.part_lse + r * pieces;
    const f32x4 *po = reinterpret_cast<const f32x4 *>(a.part_o + (size_t)r * pieces * D) + c;
    float top = -INFINITY, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < pieces; p0 += U) {
        f32x4 x[U];
        float l[U], most = top;
        bool any = false;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int p = min(p0 + u, pieces - 1);
            x[u] = po[p * LANES];
            l[u] = pl[p];
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (p0 + u >= pieces) l[u] = -INFINITY;
            most = fmaxf(most, l[u]);  // (passes over a NaN; what is made of it below is one)
            any |= !minus_infinity(l[u]);
        }
        if (!any) continue;
        const float old = fast_exp2((top - most) * LOG2E);  // (nothing so far: 0)
        sum *= old;
#pragma unroll
        for (int e = 0; e < 4; e++) acc[e] *= old;
        top = most;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const float w = fast_exp2((l[u] - top) * LOG2E);  // (a piece without keys: 0, its O is 0)
            sum += w;
#pragma unroll
            for (int e = 0; e < 4; e++) acc[e] = fmaf(w, x[u][e], acc[e]);
        }
    }
    const bool any = !no_weight(sum);
    const float inv = 1.f / sum;
#pragma unroll
    for (int e = 0; e < 4; e++) acc[e] = any ? acc[e] * inv : 0.f;
    const int bh = (int)(r / n_rows), row = (int)(r - (long long)bh * n_rows), b = bh / a.head_blocks, hb = bh - b * a.head_blocks;
    const int i = row / a.gp, head = hb * a.gp + row - i * a.gp;
    store4((T *)a.o + (size_t)b * a.so.batch + (size_t)head * a.so.head + (size_t)i * a.so.row + 4 * c, acc[0], acc[1], acc[2], acc[3]);
    if (c == 0) a.lse[((size_t)b * a.heads + head) * a.n_q + i] = any ? top + __builtin_amdgcn_logf(sum) * LN2 : -INFINITY;
}

template <typename K>
hdt_status_t launch_kernel(K kernel, const char *name, dim3 grid, int threads, size_t lds, const RelFwdArgs &a, hipStream_t st)
{
    HdtTimer t(name, st);
    if (lds > 65536) HDT_HIP_TRY(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, st, a);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

template <typename T, int D, int NW, int KS>
hdt_status_t launch_rows(const RelFwdArgs &a, bool causal, dim3 grid, size_t table, hipStream_t st)
{
    using S = FwdShape<T, D, NW, KS>;
    return launch_kernel(causal ? k_rel_fwd<T, D, NW, KS, true> : k_rel_fwd<T, D, NW, KS, false>, "hdt_rel_fwd", grid, S::THREADS, KS * S::RING + table, a, st);
}

template <typename T, int D>
hdt_status_t launch(const RelFwdArgs &a, int waves, bool causal, hipStream_t st)
{
    const size_t table = (size_t)a.gp * table_length(a.bias.max_distance, causal) * sizeof(float);
    const long long bh = (long long)a.batch * a.head_blocks;
    const dim3 grid((unsigned)(bh * a.tiles * a.pieces));
    hdt_status_t r;
    if (waves == 0)
        r = launch_kernel(causal ? k_rel_few<T, D, true> : k_rel_few<T, D, false>, "hdt_rel_few", grid, FewShape<T, D>::NW * 64,
                          FewShape<T, D>::LDS + table, a, st);
    else if (waves == 4)
        r = launch_rows<T, D, 4, 1>(a, causal, grid, table, st);
    else if (waves == 2)
        r = launch_rows<T, D, 2, 2>(a, causal, grid, table, st);
    else
        r = launch_rows<T, D, D == 64 ? 1 : 2, D == 64 ? 4 : 2>(a, causal, grid, table, st);
    if (r != HDT_OK || a.pieces == 1) return r;
    HdtTimer t("hdt_rel_join", st);
    const long long rows = bh * a.n_q * a.gp;
    constexpr int PER = 256 / (D / 4);
    hipLaunchKernelGGL((k_rel_join<T, D>), dim3((unsigned)((rows + PER - 1) / PER)), dim3(256), 0, st, a, rows);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

}  // namespace

RelFwdPlan hdt_rel_fwd_plan(const hdt_rel_attn_t &d)
{
    RelFwdPlan p;
    const int group = d.heads / d.kv_heads;
    const size_t table = table_length(d.max_distance, d.causal != 0) * sizeof(float);
    // queries of the heads that share a key head together, where one head's do not fill a tile of rows (and the heads' tables fit)
    p.gp = d.n_q < 128 && group * table <= 24576 ? group : 1;
    p.head_blocks = d.heads / p.gp;
    const long long rows = (long long)d.n_q * p.gp, heads = (long long)d.batch * p.head_blocks;
    long long pieces;
    if (rows <= 32) {
        p.waves = 0, p.tiles = 1;
        // Pieces of the keys in workgroups of their own, one a compute unit (its rings fill the LDS), and a second kernel that joins them:
        // for keys whose walk takes longer than that.  (us, one piece | these.  Heads of 64 x keys: 8 x 1000 8.7 | 9.8, 8 x 2000 11.8 | 10.1,
        // 8 x 8192 30.2 | 10.9, 32 x 8192 30.8 | 17.7; of 128: 128 x 8192 86 | 66.  4 workgroups a unit instead of one: 256 x 8192 92 | 100.)
        // (A launch is made of whole rounds of one workgroup a unit, which shows where heads are just above a multiple of 256: heads of 64 x
        // 8192 keys, 192 72 us, 252 102, 264 131 (4.2 TB/s), 384 149 (5.4), 504 192, 516 217 (5.0).)
        pieces = (long long)d.n_kv * d.head_dim < 96 * 1024 ? 1 : std::min<long long>(256 / heads, (d.n_kv + 511) / 512);
    } else {
        // Keys many times the rows (a chunk behind a long cache): tiles of 128 rows and pieces; otherwise the tile that hdt_rel_row_waves()
        // gives, and pieces only where that leaves units without work.  (us, such tiles | 64 rows: 48 heads x 200 rows x 4096 keys of 64 25 | 34,
        // 96 x 200 x 4096 of 128 62 | 88, but 32 x 1000 x 2048 of 64 30 | 24; pieces from 512 | 1024 keys: 1 x 200 x 4096 12.8 | 14.4, of 128
        // 16.2 | 21.3; up to 256 | 1024 workgroups: 16 x 512 x 8192 43 | 63.)
        p.waves = hdt_rel_row_waves(heads * ((rows + 63) / 64), heads * ((rows + 31) / 32), d);
        const bool chunk = rows > 64 && d.n_kv >= 8 * rows;
        if (chunk && d.n_kv >= 2048) p.waves = 4;
        p.tiles = (int)((rows + 32 * p.waves - 1) / (32 * p.waves));
        pieces = d.n_kv < 2048 ? 1 : std::min<long long>((!chunk ? 256 : d.head_dim == 64 ? 768 : 512) / (heads * p.tiles), d.n_kv / 512);
    }
    p.pieces = pieces < 1 ? 1 : (unsigned)pieces;
    const size_t all = (size_t)d.batch * d.heads * d.n_q;
    p.lse_at = all * p.pieces * d.head_dim * sizeof(float);
    p.bytes = p.pieces > 1 ? p.lse_at + all * p.pieces * sizeof(float) : 0;
    return p;
}

hdt_status_t hdt_launch_rel_fwd(const hdt_rel_attn_t &d, const RelFwdArgs &a, int waves, hipStream_t st)
{
    const bool causal = d.causal != 0;
    if (d.dtype == HDT_BF16) return d.head_dim == 64 ? launch<__bf16, 64>(a, waves, causal, st) : launch<__bf16, 128>(a, waves, causal, st);
    return d.head_dim == 64 ? launch<float, 64>(a, waves, causal, st) : launch<float, 128>(a, waves, causal, st);
}
