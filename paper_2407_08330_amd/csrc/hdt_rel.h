// Pieces shared by the kernels of self-attention with a relative position bias (hdt_rel_fwd.hip, hdt_rel_bwd.hip).
//
//     A_ij = scale q_i . k_j + bias[bucket(j - p_i)][head],   P = softmax over the visible j,   O = P V
//
// p_i = start + i is the position query i stands at; it is real iff 0 <= p_i < length; key j is visible to it iff j < length and,
// in the causal form, j <= p_i.  The bias depends on the distance j - p_i alone and is constant from max_distance on, so of the
// 32 x 32 blocks of pairs that a wave works on
//   * most are "far": one constant for the whole block, which joins the exponent's own constant and costs nothing;
//   * the few within max_distance of the diagonal are "near": the accumulators of Q K^T start from the head's bias by distance
//     (bias / scale, in LDS) instead of zero, so that they cost LDS reads but no arithmetic.  The causal mask is part of that
//     table: minus infinity at positive distances.  Every block that the diagonal crosses is a near one.
// Accumulators hold pairs with one side along the lanes (column l % 32) and the other along the registers (rows of C, hdt_mfma.h).
//
// bf16 tensors go through v_mfma_f32_32x32x16_bf16, fp32 ones through v_mfma_f32_32x32x2_f32, whose C layout is the same; a lane's
// 16 bytes of a row are 8 contraction values of one instruction in bf16 and one value of each of four in fp32 (Op<T>).
#pragma once

#include <type_traits>

#include "hdt_internal.h"
#include "hdt_lanes.h"
#include "hdt_mfma.h"
#include "hdt_tile.h"

namespace hdt_rel {

using namespace hdt_tile;
using namespace hdt_lanes;

typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kPad = 128;             // distances the table goes on beyond the last one that matters: as far as 64 x 32 pairs reach, rows that are not real among them
constexpr int kMostDistance = 1024;   // max_distance at most
constexpr float kHidden = 1e6f;       // a bias from -1e6 down hides a bucket, one from 1e6 up counts as 1e6

// one row-side operand fragment (16 bytes of a row) and the contractions it takes part in
template <typename T>
struct Op;
template <>
struct Op<__bf16> {
    typedef bf16x8 Frag;
    static constexpr int PER_STEP = 16;  // values of the contraction a step covers
    static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) { return mfma_32x32x16(a, b, c); }
};
template <>
struct Op<float> {
    typedef f32x4 Frag;
    static constexpr int PER_STEP = 8;
    static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c)
    {
#pragma unroll
        for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// What a kernel does with blocks of 32 x 32 held in C fragments (P, dS) as the B operand of the next contraction
template <typename T>
struct Weights;
template <>
struct Weights<__bf16> {  // rounded to bf16: the operand type of the fast contraction; its sum is taken before
    bf16x8 lo, hi;
    __device__ __forceinline__ Weights() = default;
    __device__ __forceinline__ explicit Weights(const f32x16 &p) : lo(pack_bf16x8(p, 0)), hi(pack_bf16x8(p, 8)) {}
};
template <>
struct Weights<float> {
    f32x16 p;
    __device__ __forceinline__ Weights() = default;
    __device__ __forceinline__ explicit Weights(const f32x16 &x) : p(x) {}
};

// Rows of a [.][D] tensor in LDS: tiles of R rows, 16-byte chunks permuted within a row against bank conflicts (swz).
template <typename T, int D>
struct Rows {
    static constexpr int ROWB = D * (int)sizeof(T), CPR = ROWB / 16, RPI = 1024 / ROWB;  // rows per wave-level load
    static constexpr int STEPS = D / Op<T>::PER_STEP, BLOCKS = D / 32;
    typedef typename Op<T>::Frag Frag;

    // 16 bytes of row r0 + l % 32: step st
    static __device__ __forceinline__ Frag read(const char *tile, const RowLane &r, int r0, int st)
    {
        return *reinterpret_cast<const Frag *>(tile + (r0 + r.row) * ROWB + ((((st << 1) ^ r.x)) << 4));
    }
    // acc += (rows r0 .. r0 + 31 of the tile, columns 32 j ..)^T times the weights of those rows, in WSTEPS contractions: the operand of
    // step s, and the contraction
    static constexpr int WSTEPS = sizeof(T) == 2 ? 2 : 16;
    typedef typename std::conditional<sizeof(T) == 2, bf16x8, float>::type WFrag;
    static __device__ __forceinline__ WFrag wread(const char *tile, const TrLane &t, int lane, int r0, int j, int s)
    {
        if constexpr (sizeof(T) == 2) {
            return read_tr<ROWB>(tile, t, r0 + 16 * s, j);
        } else {
            const int c = 8 * j + ((lane & 31) >> 2), r = r0 + 8 * (s >> 2) + (s & 3) + 4 * (lane >> 5);
            return *reinterpret_cast<const float *>(tile + r * ROWB + ((c ^ swz<CPR>(r & 31)) << 4) + (lane & 3) * 4);
        }
    }
    static __device__ __forceinline__ f32x16 wmma(WFrag a, const Weights<T> &w, int s, f32x16 acc)
    {
        if constexpr (sizeof(T) == 2) {
            return mfma_32x32x16(a, s ? w.hi : w.lo, acc);
        } else {
            return __builtin_amdgcn_mfma_f32_32x32x2f32(a, w.p[s], acc, 0, 0, 0);
        }
    }
};

// Two tensors whose rows travel together (K and V; Q and dO): tiles of R rows of each into a stage of a ring in LDS (tile of the
// first, tile of the second), this wave's share of NW.
template <typename T, int D, int R, int NW>
struct Pair {
    typedef Rows<T, D> RowsT;
    static constexpr int TILE = R * RowsT::ROWB, STAGE = 2 * TILE, NI = R / RowsT::RPI / NW;
    static_assert(NI >= 1 && R % (RowsT::RPI * NW) == 0, "a wave loads whole instructions");
    const char *a, *b;               // row 0 of the two
    uint32_t stride_a, stride_b;     // bytes
    uint32_t off_a[NI], off_b[NI];  // this lane's bytes of the rows it loads, from the tile's first row on
    uint32_t lds;
    int wave, lane;

    __device__ __forceinline__ void init(const void *pa, int64_t row_a, const void *pb, int64_t row_b, const char *smem, int w, int l)
    {
        a = (const char *)pa, b = (const char *)pb, stride_a = (uint32_t)row_a * sizeof(T), stride_b = (uint32_t)row_b * sizeof(T);
        lds = lds_addr(smem), wave = w, lane = l;
        const int c = l % RowsT::CPR;
#pragma unroll
        for (int i = 0; i < NI; i++) {
            const int r = (w * NI + i) * RowsT::RPI + l / RowsT::CPR;
            off_a[i] = (uint32_t)r * stride_a + (uint32_t)((c ^ swz<RowsT::CPR>(r & 31)) << 4);
            off_b[i] = (uint32_t)r * stride_b + (uint32_t)((c ^ swz<RowsT::CPR>(r & 31)) << 4);
        }
    }
    // Starts loading rows r0 .. r0 + R - 1.  Rows in front of row `low` or behind row `last` are not read: copies of those two stand
    // in their place.
    __device__ __forceinline__ void request(int r0, int low, int last, int stage) const
    {
        const char *pa = a + (size_t)r0 * stride_a, *pb = b + (size_t)r0 * stride_b;
        const uint32_t at = lds + (uint32_t)(stage * STAGE + wave * NI * 1024);
        if (low <= r0 && last >= r0 + R - 1) {
#pragma unroll
            for (int i = 0; i < NI; i++) {
                dma16(pa, off_a[i], at + i * 1024);
                dma16(pb, off_b[i], at + TILE + i * 1024);
            }
        } else {
            const int c = lane % RowsT::CPR;
#pragma unroll
            for (int i = 0; i < NI; i++) {
                const int r = (wave * NI + i) * RowsT::RPI + lane / RowsT::CPR, from = min(max(r, low - r0), last - r0);
                const uint32_t chunk = (uint32_t)((c ^ swz<RowsT::CPR>(r & 31)) << 4);
                dma16(pa, (uint32_t)from * stride_a + chunk, at + i * 1024);
                dma16(pb, (uint32_t)from * stride_b + chunk, at + TILE + i * 1024);
            }
        }
    }
};

// Values the compiler loads itself are waited for here, in front of a loop whose own loads it does not count: where it first used them,
// inside the loop, its wait would be repeated in every round, and would wait for the next tile.
template <typename F>
__device__ __forceinline__ void settle(const F &f)
{
    asm volatile("" ::"v"(f));
}

// N contractions whose operands come from LDS, AHEAD of them requested before the first is waited for and one more behind each
// contraction.  Left to itself the compiler asks for an operand where it needs it and waits for it on the spot (to keep registers few),
// which leaves a wave waiting for most of its time.  What may move across the fixed order is arithmetic (mask 0x406: vector, scalar and
// transcendental instructions).
template <int N, int AHEAD, typename Frag, typename Read>
struct Ahead {
    Frag buf[AHEAD];
    const Read &read;
    __device__ __forceinline__ explicit Ahead(const Read &r) : read(r)
    {
#pragma unroll
        for (int i = 0; i < AHEAD && i < N; i++) buf[i] = read(i);
        __builtin_amdgcn_sched_barrier(0x406);
    }
    template <typename Mma>
    __device__ __forceinline__ void run(const Mma &mma)
    {
#pragma unroll
        for (int i = 0; i < N; i++) {
            mma(i, buf[i % AHEAD]);
            if (i + AHEAD < N) buf[i % AHEAD] = read(i + AHEAD);
            __builtin_amdgcn_sched_barrier(0x406);
        }
    }
};
template <int N, int AHEAD, typename Frag, typename Read>
__device__ __forceinline__ Ahead<N, AHEAD, Frag, Read> ahead(const Read &read)
{
    return Ahead<N, AHEAD, Frag, Read>(read);
}

// The rounds of a walk along tiles that go through a ring of two stages: `tile(round, stage)`.  CONST: the stage is a constant for the
// compiler, and the LDS addresses of both stages are then offsets of the same registers, for twice the code.
template <bool CONST, typename Tile>
__device__ __forceinline__ void walk(int rounds, const Tile &tile)
{
    int i = 0;
    if constexpr (CONST) {
        for (; i + 1 < rounds; i += 2) {
            tile(i, std::integral_constant<int, 0>());
            tile(i + 1, std::integral_constant<int, 1>());
        }
        if (i < rounds) tile(i, std::integral_constant<int, 0>());
    } else {
        for (; i < rounds; i++) tile(i, i & 1);
    }
}

// A wave's 32 x D accumulators, held transposed (lane (row l % 32, hf), columns 32 j + 8 q + 4 hf ..), times the lane's `mult`, or zeros where it is
// not `real`, to rows of a tensor: through 32 rows of LDS of the wave's own, so that whole rows leave, 16 bytes a lane.  (From the registers, 8 bytes to each of 32
// rows an instruction, the stores took 40 of the 660 us of a backward of 4096 x 32 heads of 128.)  Row r keeps chunk c at c ^ (r & 7).
template <typename T, int D>
__device__ __forceinline__ void store_rows(char *wave_lds, int lane, const f32x16 (&acc)[D / 32], bool real, float mult, T *dst, int64_t stride, int rows_valid)
{
    typedef Rows<T, D> R;
    const int r = lane & 31, hf = lane >> 5;
    const uint32_t at = lds_addr(wave_lds) + (uint32_t)(r * R::ROWB);
#pragma unroll
    for (int j = 0; j < D / 32; j++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const int c = sizeof(T) == 2 ? 4 * j + q : 8 * j + 2 * q + hf;
            typedef T V __attribute__((ext_vector_type(4)));
            V v;
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = (T)(real ? acc[j][4 * q + e] * mult : 0.f);
            *(HDT_LDS V *)(uintptr_t)(at + (uint32_t)((c ^ (r & 7)) << 4) + (sizeof(T) == 2 ? hf * 8 : 0)) = v;
        }
    const int lr = lane / R::CPR, c = lane % R::CPR;
#pragma unroll
    for (int i = 0; i < 32 / R::RPI; i++) {
        const int row = i * R::RPI + lr;
        const u32x4 v = *reinterpret_cast<const u32x4 *>(wave_lds + row * R::ROWB + ((c ^ (row & 7)) << 4));
        if (row < rows_valid) *reinterpret_cast<u32x4 *>((char *)(dst + (int64_t)row * stride) + c * 16) = v;
    }
}

// By their bits, which the compiler cannot see through: the sources are compiled on the assumption that no value is a NaN
// (-fno-honor-nans), and a real row of the caller's may make one.  Nothing but zero weights, so that a row has no key; a NaN sum is not that.
__device__ __forceinline__ bool no_weight(float sum) { return hidden(__builtin_bit_cast(unsigned, sum)) << 1 == 0; }
__device__ __forceinline__ bool minus_infinity(float x) { return hidden(__builtin_bit_cast(unsigned, x)) == 0xff800000u; }

// The rows of a sample that stand for positions, and its keys
struct Sample {
    int start, length;  // position of query 0; keys
    int lo, hi;         // queries [lo, hi) are real
};
__device__ __forceinline__ Sample sample_of(const int32_t *lengths, const int32_t *starts, int b, int n_q, int n_kv)
{
    Sample s;
    s.length = lengths ? min(max(as_const(lengths)[b], 0), n_kv) : n_kv;
    const int64_t start = starts ? as_const(starts)[b] : 0;
    s.lo = (int)min(max(-start, (int64_t)0), (int64_t)n_q);
    s.hi = (int)min(max((int64_t)s.length - start, (int64_t)s.lo), (int64_t)n_q);
    s.start = (int)start;
    return s;
}

// bias by distance of `heads` heads from h0 on, as bias / scale: entry d + max_distance + kPad, distances -max_distance - kPad up
// to kPad - 1 (causal: minus infinity from 1 on) or max_distance + kPad - 1
__host__ __device__ __forceinline__ int table_length(int max_distance, bool causal) { return (causal ? 1 : 2) * max_distance + 2 * kPad; }

struct BiasArgs {
    const void *bias;      // [n_buckets][heads]
    const int32_t *table;  // [2 max_distance + 1]
    int n_buckets, heads, max_distance, bf16;
    float inv_scale;
};
__device__ __forceinline__ int bucket_of(const BiasArgs &a, int distance)
{
    const int M = a.max_distance;
    return min(max(a.table[min(max(distance, -M), M) + M], 0), a.n_buckets - 1);
}
__device__ __forceinline__ float bias_at(const BiasArgs &a, int bucket, int head)
{
    const size_t at = (size_t)bucket * a.heads + head;
    const float x = a.bf16 ? (float)((const __bf16 *)a.bias)[at] : ((const float *)a.bias)[at];
    // Values that stand for a mask are one (kHidden): a row that saw nothing else would have an LSE next to them, in whose fp32 the
    // logarithm of its sum is lost, and with it the row's gradients.
    // (a NaN is kept, told by its bits: the smaller of it and kHidden would be kHidden)
    const unsigned bits = hidden(__builtin_bit_cast(unsigned, x));
    const float y = x <= -kHidden ? -INFINITY : fminf(x, kHidden) * a.inv_scale;
    return __builtin_bit_cast(float, bits << 1 > 0xff000000u ? bits : __builtin_bit_cast(unsigned, y));
}
__device__ __forceinline__ float bias_of(const BiasArgs &a, int distance, int head) { return bias_at(a, bucket_of(a, distance), head); }
__device__ __forceinline__ void fill_table(float *to, const BiasArgs &a, int h0, int heads, bool causal, int tid, int threads)
{
    constexpr int U = 4;  // entries a thread has in flight: two loads each, the second at the first's word
    const int len = table_length(a.max_distance, causal), M = a.max_distance, all = heads * len;
    for (int x0 = tid; x0 < all; x0 += U * threads) {
        int bucket[U];
        float bias[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int x = x0 + u * threads, d = x % len - M - kPad;
            bucket[u] = x < all && !(causal && d > 0) ? bucket_of(a, d) : -1;
        }
#pragma unroll
        for (int u = 0; u < U; u++) bias[u] = bucket[u] >= 0 ? bias_at(a, bucket[u], h0 + (x0 + u * threads) / len) : -INFINITY;
#pragma unroll
        for (int u = 0; u < U; u++)
            if (x0 + u * threads < all) to[x0 + u * threads] = bias[u];
    }
}

enum class Kind { SKIP, NEAR, FAR_BEHIND, FAR_AHEAD };
// of W keys from k0 on and positions [p0, p1] (p1 - p0 <= 31, W <= 64)
template <bool CAUSAL, int W>
__device__ __forceinline__ Kind kind_of(int k0, int p0, int p1, int M, int length)
{
    if ((CAUSAL && k0 > p1) || k0 >= length) return Kind::SKIP;
    if (k0 + W - 1 - p0 <= -M) return Kind::FAR_BEHIND;
    if (!CAUSAL && k0 - p1 >= M) return Kind::FAR_AHEAD;
    return Kind::NEAR;
}

}  // namespace hdt_rel
