// Token embeddings: rows of a table by ids, scaled, and the table's gradient.
//
//   hdt_embed_fwd  out[t] = scale table[id[t]];  0 for ids outside [0, vocab)
//   hdt_embed_bwd  grad[v] = scale sum of d_out[t] over the t with id[t] = v, in ascending order of blocks of them (see k_embed_sum);
//                  0 for rows without a token, or (accumulate) added to what stands there
//
// Both are bound by memory.  Forward, 32768 bf16 rows of 768 columns out of 32768: 19 us with nothing in the caches (67 MB, 3.5 TB/s), 11 with the table there;
// 16384 rows of an fp32 table to bf16: 9.2 us.  The backward has no atomics on values: k_embed_sort puts the tokens of each row side by side, in the
// order in which they came; k_embed_sum adds up a block of consecutive ones a wave, so that a word that is a tenth of a text keeps no
// workgroup longer than one that comes twice; k_embed_join adds up the rows that span several blocks.  Sums are in fp32 in a fixed order.
// Same sizes, words as frequent as 1 / rank: sort 19.8 us (a third of it the zeros of rows without a token, 30 MB; else every workgroup reading all ids
// from the L2 and placing its own), sum 15.9 (50 MB read), join 6.  The sort grows with the tokens, and with the vocabulary beyond 131072 rows, where there are more
// shares than compute units: all three, 131072 tokens of 32768 rows 103 us, 131072 of 262144 190; 2^20 tokens of 64 columns, of 32768 rows 470, of 2^20 1290.
#include <algorithm>

#include "hdt_internal.h"
#include "hdt_rows.h"

namespace {

using namespace hdt_rows;

// ------------------------------------------------------------------------------------------ forward
struct FwdArgs {
    const int32_t *ids;
    const void *table;
    void *out;
    int64_t tokens;
    int vocab, width, chunks, rows;  // rows: tokens of a workgroup
    float scale;
};

// a workgroup's tokens, chunk by chunk of eight columns
template <typename W, typename T, bool WHOLE>
__global__ __launch_bounds__(256) void k_embed_fwd(FwdArgs a)
{
    for (int64_t t0 = (int64_t)blockIdx.x * a.rows; t0 < a.tokens; t0 += (int64_t)gridDim.x * a.rows) {
        const unsigned all = (unsigned)min((int64_t)a.rows, a.tokens - t0) * (unsigned)a.chunks;
        for (unsigned i = threadIdx.x; i < all; i += 256) {
            const unsigned r = i / (unsigned)a.chunks, c = (i - r * a.chunks) * 8;
            const int64_t t = t0 + r;
            const int id = a.ids[t], left = a.width - (int)c;
            Eight v = {};
            if ((unsigned)id < (unsigned)a.vocab) {
                const auto w = load8<WHOLE>((const W *)a.table + (size_t)id * a.width + c, left);
#pragma unroll
                for (int e = 0; e < 8; e++) v.x[e] = a.scale * (float)w[e];
            }
            store8<WHOLE>((T *)a.out + (size_t)t * a.width + c, v, left);
        }
    }
}

// ------------------------------------------------------------------------------------------ backward: the order
struct Entry {
    int32_t id, token;
};
struct BwdArgs {
    const int32_t *ids;
    const void *d_out;
    void *grad;
    Entry *entries;   // [tokens], ordered by (id mod shares, id, token); the rest of them is not written
    int32_t *n_real;  // how many there are; NULL without tokens
    float *parts;     // [blocks][2][width]: of a block's first row where that began before it, of its last where that goes on behind it
    int tokens, vocab, width, shares_log2, rows, accumulate, block;  // rows: of a share; block: entries that a wave adds up
    float scale;
};

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kMostRows = 512, kAhead = 8;

// Share s of the rows are those whose number is s modulo the number of shares (frequent words, which stand side by side in a vocabulary
// made by frequency, go to different ones).  Its workgroup reads all ids, twice, from the caches: the first time it counts, its waves by
// themselves and row by row, so that each wave knows where its tokens of a row go, and the second time it puts them there.  Nothing is
// shared between workgroups.
// HELD: a wave's STEPS x 256 ids are all it has, and stay in registers in between.
template <typename W, int STEPS, bool HELD>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(BwdArgs a)
{
    extern __shared__ int count[];  // [waves][rows], [rows]
    __shared__ int wave_below[kSortWaves], wave_total[kSortWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int share = blockIdx.x, mask = (1 << a.shares_log2) - 1;
    for (int i = threadIdx.x; i < kSortWaves * a.rows; i += kSortThreads) count[i] = 0;
    __syncthreads();

    // a step is 256 tokens, four consecutive ones a lane (one a lane: 131072 tokens 64 us for 59, 30000 of 200 rows 18.3 for 16.3)
    const int steps = (a.tokens + 255) / 256, per = (steps + kSortWaves - 1) / kSortWaves;
    const int first = min(wave * per, steps), last = min(first + per, steps);
    int *const mine = count + wave * a.rows, *const totals = count + kSortWaves * a.rows;
    typedef int Four __attribute__((ext_vector_type(4)));
    typedef Four FourAnywhere __attribute__((aligned(4)));
    Four id[STEPS];
    auto take = [&](int s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < STEPS; u++) {
            const int t = (s + u) * 256 + lane * 4;
            id[u] = Four{-1, -1, -1, -1};
            if (s + u >= last) continue;
            if (t + 4 <= a.tokens)
                id[u] = *reinterpret_cast<const FourAnywhere *>(a.ids + t);
            else
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (t + e < a.tokens) id[u][e] = a.ids[t + e];
        }
    };
    int below = 0;
    auto count_them = [&](int s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < STEPS; u++) {
            if (s + u >= last) break;  // (code that is not run is not fetched)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int of = (unsigned)id[u][e] < (unsigned)a.vocab ? id[u][e] & mask : mask + 1;
                if (of < share) below++;
                if (of == share) atomicAdd(&mine[id[u][e] >> a.shares_log2], 1);
            }
        }
    };
    if (HELD) {
        take(first);
        count_them(first);
    } else {
        for (int s = first; s < last; s += STEPS) {
            take(s);
            count_them(s);
        }
    }
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) below += __shfl_xor(below, s);
    if (lane == 0) wave_below[wave] = below;
    __syncthreads();

    // thread r: row r of the share.  Its tokens begin behind those of the shares and rows before it.
    int total = 0;
    if ((int)threadIdx.x < a.rows) {
        for (int w = 0; w < kSortWaves; w++) total += count[w * a.rows + threadIdx.x];
        totals[threadIdx.x] = total;
    }
    int before = total;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int o = __shfl_up(before, s);
        if (lane >= s) before += o;
    }
    if (lane == 63) wave_total[wave] = before;
    __syncthreads();
    int base = 0, all = 0;
    for (int w = 0; w < kSortWaves; w++) {
        base += wave_below[w] + (w < wave ? wave_total[w] : 0);
        all += wave_below[w] + wave_total[w];
    }
    before += base - total;
    if (a.n_real && share == mask && threadIdx.x == 0) *a.n_real = all;
    if ((int)threadIdx.x < a.rows)
        for (int w = 0; w < kSortWaves; w++) {
            const int n = count[w * a.rows + threadIdx.x];
            count[w * a.rows + threadIdx.x] = before;
            before += n;
        }
    __syncthreads();

    if (!a.accumulate)
        for (int r = wave; r < a.rows; r += kSortWaves) {  // rows without a token
            const int64_t v = ((int64_t)r << a.shares_log2) + share;
            if (v >= a.vocab || totals[r] != 0) continue;
            const Eight zero = {};
            for (int c = lane * 8; c < a.width; c += 512) store8<false>((W *)a.grad + (size_t)v * a.width + c, zero, a.width - c);
        }
    for (int s = first; s < last; s += STEPS) {
        if (!HELD) take(s);
#pragma unroll
        for (int u = 0; u < STEPS; u++) {
            if (s + u >= last) break;
            const unsigned long long before_me = (1ull << lane) - 1;
            int row[4];
            unsigned long long open[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                row[e] = (unsigned)id[u][e] < (unsigned)a.vocab && (id[u][e] & mask) == share ? id[u][e] >> a.shares_log2 : -1;
                open[e] = __ballot(row[e] >= 0);
            }
            while (open[0] | open[1] | open[2] | open[3]) {  // the tokens that have the row of the first open one
                const int at_lane = __builtin_ctzll(open[0] | open[1] | open[2] | open[3]);
                int r = 0;
#pragma unroll
                for (int e = 3; e >= 0; e--)
                    if (open[e] >> at_lane & 1) r = __builtin_amdgcn_readlane(row[e], at_lane);
                unsigned long long same[4];
                const int at = mine[r];
                int place = at, all_same = 0;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    same[e] = __ballot(row[e] == r);
                    place += __popcll(same[e] & before_me);
                    all_same += __popcll(same[e]);
                    open[e] &= ~same[e];
                }
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (row[e] == r) a.entries[place++] = {id[u][e], (s + u) * 256 + lane * 4 + e};
                hdt_lanes::wave_lds_barrier();  // (all lanes have read the row's place; lane 0 moves it on for the next row and step)
                if (lane == 0) mine[r] = at + all_same;
                hdt_lanes::wave_lds_barrier();
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ backward: the sums
// A wave adds up the rows of a block of entries, 512 columns of them.
template <typename W, bool WHOLE>
__device__ __forceinline__ void put_row(const BwdArgs &a, int id, int c, Eight v)
{
    W *g = (W *)a.grad + (size_t)id * a.width + c;
    const int left = a.width - c;
#pragma unroll
    for (int e = 0; e < 8; e++) v.x[e] *= a.scale;
    if (a.accumulate) {
        const auto old = load8<WHOLE>(g, left);
#pragma unroll
        for (int e = 0; e < 8; e++) v.x[e] += (float)old[e];
    }
    store8<WHOLE>(g, v, left);
}

template <typename W, typename T, bool WHOLE>
__global__ __launch_bounds__(256) void k_embed_sum(BwdArgs a, int slabs)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = (int)(unit / slabs), c = ((int)(unit % slabs) * 64 + lane) * 8, left = a.width - c;
    const int64_t n = *a.n_real, i0 = (int64_t)block * a.block;
    if (i0 >= n) return;
    const int count = (int)min((int64_t)a.block, n - i0);
    // the entries and their neighbours: entry i0 + j in lane j + 1
    Entry mine = {-1, 0};
    if (lane < a.block + 2 && i0 - 1 + lane >= 0 && i0 - 1 + lane < n) mine = a.entries[i0 - 1 + lane];
    auto id_of = [&](int j) { return __builtin_amdgcn_readlane(mine.id, j + 1); };
    float *const part = a.parts + (size_t)block * 2 * a.width + c;
    bool begun_before = id_of(-1) == id_of(0);
    Eight sum = {};
    for (int j0 = 0; j0 < count; j0 += kAhead) {
        typename Vec<T>::V v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            v[u] = typename Vec<T>::V{};
            const int64_t t = __builtin_amdgcn_readlane(mine.token, min(j0 + u, count - 1) + 1);
            if (left > 0) v[u] = load8<WHOLE>((const T *)a.d_out + (size_t)t * a.width + c, left);
        }
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            const int j = j0 + u;
            if (j >= count) break;
#pragma unroll
            for (int e = 0; e < 8; e++) sum.x[e] += (float)v[u][e];
            const int id = id_of(j);
            const bool goes_on = id_of(j + 1) == id;
            if (goes_on && j + 1 < count) continue;
            if (left > 0) {
                if (begun_before)
                    store8<WHOLE>(part, sum, left);
                else if (goes_on)
                    store8<WHOLE>(part + a.width, sum, left);
                else
                    put_row<W, WHOLE>(a, id, c, sum);
            }
            begun_before = false;
            sum = Eight{};
        }
    }
}

// The rows that span blocks: the workgroup of the block in which one begins adds up its parts, its four waves a quarter each.
template <typename W, bool WHOLE>
__global__ __launch_bounds__(256) void k_embed_join(BwdArgs a, int slabs)
{
    __shared__ float lds[4][512];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t block = blockIdx.x / (unsigned)slabs, n = *a.n_real, i0 = block * a.block, i1 = i0 + a.block;
    if (i1 >= n) return;  // (no block behind it)
    const int id = a.entries[i1].id;
    if (a.entries[i1 - 1].id != id) return;
    if (a.entries[i0].id == id && i0 > 0 && a.entries[i0 - 1].id == id) return;  // begun before
    int64_t more = 1;  // blocks behind this one that have a part
    for (;;) {
        const int64_t at = i1 + (more + lane) * a.block;
        const unsigned long long ends = __ballot(!(at < n && a.entries[at].id == id));
        if (ends) {
            more += __builtin_ctzll(ends);
            break;
        }
        more += 64;
    }
    const int c = ((int)(blockIdx.x % (unsigned)slabs) * 64 + lane) * 8, left = a.width - c;
    const int64_t per = (more + 3) / 4, k0 = min(wave * per, more), k1 = min(k0 + per, more);
    Eight sum = {};
    if (left > 0) {
        const float *p = a.parts + ((size_t)(block + 1 + k0) * 2) * a.width + c;
        for (int64_t k = k0; k < k1; k += kAhead) {
            typename Vec<float>::V v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; u++)
                v[u] = k + u < k1 ? load8<WHOLE>(p + (size_t)(k - k0 + u) * 2 * a.width, left) : typename Vec<float>::V{};
#pragma unroll
            for (int u = 0; u < kAhead; u++)
#pragma unroll
                for (int e = 0; e < 8; e++) sum.x[e] += v[u][e];
        }
    }
    store8<true>(&lds[wave][lane * 8], sum, 8);
    __syncthreads();
    if (wave != 0 || left <= 0) return;
    const auto head = load8<WHOLE>(a.parts + ((size_t)block * 2 + 1) * a.width + c, left);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        sum.x[e] = head[e];
#pragma unroll
        for (int w = 0; w < 4; w++) sum.x[e] += lds[w][lane * 8 + e];
    }
    put_row<W, WHOLE>(a, id, c, sum);
}

// ------------------------------------------------------------------------------------------ host
constexpr int kMostWidth = 32768, kMostVocab = 1 << 24;
constexpr int64_t kMostElements = 1ll << 35, kMostTokens = 1ll << 28;  // (a launch has fewer than 2^32 threads)

bool misaligned(const void *p, unsigned by = 16) { return ((uintptr_t)p & (by - 1)) != 0; }

hdt_status_t check_sizes(const char *fn, int64_t tokens, int32_t vocab, int32_t width, float scale, hdt_dtype_t table_dt, hdt_dtype_t dt)
{
    if (tokens < 0 || vocab < 0 || width < 0) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: negative size", fn);
    if (!hdt_finite(scale)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: scale = %g", fn, (double)scale);
    if (dt != HDT_BF16 && dt != HDT_F32) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, (int)dt);
    if (table_dt != HDT_BF16 && table_dt != HDT_F32) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d of the table", fn, (int)table_dt);
    if (width < 1 || width > kMostWidth) return hdt_fail(HDT_ERR_SHAPE, "%s: width %d outside [1, %d]", fn, width, kMostWidth);
    if (vocab < 1 || vocab > kMostVocab) return hdt_fail(HDT_ERR_SHAPE, "%s: vocab %d outside [1, 2^24]", fn, vocab);
    if (tokens > kMostTokens || tokens * width > kMostElements) return hdt_fail(HDT_ERR_SHAPE, "%s: more than 2^28 tokens or 2^35 elements", fn);
    return HDT_OK;
}

// shares of the vocabulary: one a compute unit, or as many as keep a share's counts in LDS
int shares_log2(int vocab)
{
    int l = 8;
    while (((int64_t)kMostRows << l) < vocab) l++;
    return l;
}
// entries a block: few tokens are spread over more waves, many have fewer rows to join (us of sum and join, blocks of 8 | 16 | 32, 768 bf16 columns, with
// about 5 of each for the events around it: 4096 tokens 14.4 | 15.6 | 19.9, 8192 16.5 | 16.4 | 19.8, 16384 22.3 | 19.6 | 21.4, 32768 31.0 | 25.8 | 25.1)
int block_of(int64_t tokens) { return tokens <= 4096 ? 8 : tokens <= 16384 ? 16 : 32; }
int64_t blocks_of(int64_t tokens) { return (tokens + block_of(tokens) - 1) / block_of(tokens); }
size_t entries_bytes(int64_t tokens) { return ((size_t)tokens * sizeof(Entry) + 15) / 16 * 16; }

#define HDT_EXPORT extern "C" __attribute__((visibility("default")))

template <typename W, typename T>
void launch_fwd(const FwdArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)std::min<int64_t>((a.tokens + a.rows - 1) / a.rows, 1 << 20)), block(256);
    if (a.width % 8 == 0)
        hipLaunchKernelGGL((k_embed_fwd<W, T, true>), grid, block, 0, st, a);
    else
        hipLaunchKernelGGL((k_embed_fwd<W, T, false>), grid, block, 0, st, a);
}
template <typename W, typename T, bool WHOLE>
hdt_status_t launch_bwd(const BwdArgs &a, hipStream_t st)
{
    const int slabs = (a.width + 511) / 512;
    const int64_t blocks = blocks_of(a.tokens);
    {
        HdtTimer t("hdt_embed_sort", st);
        const size_t lds = (size_t)(kSortWaves + 1) * a.rows * sizeof(int);
        const dim3 grid(1u << a.shares_log2), threads(kSortThreads);
        if (a.tokens <= 4 * kSortThreads)
            hipLaunchKernelGGL((k_embed_sort<W, 1, true>), grid, threads, lds, st, a);
        else if (a.tokens <= 32 * kSortThreads)
            hipLaunchKernelGGL((k_embed_sort<W, 8, true>), grid, threads, lds, st, a);
        else
            hipLaunchKernelGGL((k_embed_sort<W, 4, false>), grid, threads, lds, st, a);
        HDT_HIP_TRY(hipGetLastError());
    }
    if (blocks == 0) return HDT_OK;
    {
        HdtTimer t("hdt_embed_sum", st);
        hipLaunchKernelGGL((k_embed_sum<W, T, WHOLE>), dim3((unsigned)((blocks * slabs + 3) / 4)), dim3(256), 0, st, a, slabs);
        HDT_HIP_TRY(hipGetLastError());
    }
    if (blocks == 1) return HDT_OK;
    HdtTimer t("hdt_embed_join", st);
    hipLaunchKernelGGL((k_embed_join<W, WHOLE>), dim3((unsigned)((blocks - 1) * slabs)), dim3(256), 0, st, a, slabs);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

}  // namespace

HDT_EXPORT hdt_status_t hdt_embed_fwd(const int32_t *d_ids, int64_t tokens, const void *table, int32_t vocab, int32_t width, float scale, void *out,
                                      hdt_dtype_t table_dt, hdt_dtype_t dt, void *stream)
{
    const char *fn = "hdt_embed_fwd";
    if (hdt_status_t st = check_sizes(fn, tokens, vocab, width, scale, table_dt, dt)) return st;
    if (tokens == 0) return HDT_OK;
    if (!d_ids || !table || !out) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (misaligned(d_ids, 4) || misaligned(table) || misaligned(out)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned, the ids 4", fn);
    if (out == table || out == (const void *)d_ids) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: output aliases an input", fn);
    const int chunks = (width + 7) / 8;
    const FwdArgs a = {d_ids, table, out, tokens, vocab, width, chunks, std::max(1, 1024 / chunks), scale};
    hipStream_t st = (hipStream_t)stream;
    HdtTimer t("hdt_embed_fwd", st);
    if (table_dt == HDT_BF16)
        dt == HDT_BF16 ? launch_fwd<__bf16, __bf16>(a, st) : launch_fwd<__bf16, float>(a, st);
    else
        dt == HDT_BF16 ? launch_fwd<float, __bf16>(a, st) : launch_fwd<float, float>(a, st);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

HDT_EXPORT size_t hdt_embed_bwd_workspace_bytes(int64_t tokens, int32_t width)
{
    if (tokens <= 0 || tokens > kMostTokens || width < 1 || width > kMostWidth || tokens * width > kMostElements) return 0;
    return 16 + entries_bytes(tokens) + (size_t)blocks_of(tokens) * 2 * width * sizeof(float);
}

HDT_EXPORT hdt_status_t hdt_embed_bwd(const void *d_out, const int32_t *d_ids, int64_t tokens, int32_t vocab, int32_t width, float scale,
                                      int32_t accumulate, void *grad, hdt_dtype_t table_dt, hdt_dtype_t dt, void *workspace, size_t workspace_bytes,
                                      void *stream)
{
    const char *fn = "hdt_embed_bwd";
    if (hdt_status_t st = check_sizes(fn, tokens, vocab, width, scale, table_dt, dt)) return st;
    if ((int64_t)vocab * width > kMostElements) return hdt_fail(HDT_ERR_SHAPE, "%s: a table of more than 2^35 elements", fn);
    if (!grad) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (misaligned(grad)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned, the ids 4", fn);
    if (tokens == 0 && accumulate) return HDT_OK;
    const size_t need = hdt_embed_bwd_workspace_bytes(tokens, width);
    if (tokens > 0) {
        if (!d_out || !d_ids) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
        if (misaligned(d_out) || misaligned(d_ids, 4)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned, the ids 4", fn);
        if (grad == d_out || grad == (const void *)d_ids) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: output aliases an input", fn);
        if (!workspace || workspace_bytes < need || misaligned(workspace))
            return hdt_fail(HDT_ERR_INVALID_ARG, "%s: a 16-byte aligned workspace of %zu bytes needed, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
    }
    BwdArgs a = {};
    a.d_out = d_out, a.ids = d_ids, a.grad = grad;
    if (tokens > 0) {  // (without tokens no workspace is needed: one that is given may be of no bytes)
        a.n_real = (int32_t *)workspace;
        a.entries = (Entry *)((char *)workspace + 16);
        a.parts = (float *)((char *)workspace + 16 + entries_bytes(tokens));
    }
    a.tokens = (int)tokens, a.vocab = vocab, a.width = width, a.accumulate = accumulate != 0, a.block = block_of(tokens), a.scale = scale;
    a.shares_log2 = shares_log2(vocab);
    a.rows = (int)(((int64_t)vocab + (1 << a.shares_log2) - 1) >> a.shares_log2);
    hipStream_t st = (hipStream_t)stream;
    const bool whole = width % 8 == 0;
#define HDT_EMBED_BWD(W, T) (whole ? launch_bwd<W, T, true>(a, st) : launch_bwd<W, T, false>(a, st))
    if (table_dt == HDT_BF16) return dt == HDT_BF16 ? HDT_EMBED_BWD(__bf16, __bf16) : HDT_EMBED_BWD(__bf16, float);
    return dt == HDT_BF16 ? HDT_EMBED_BWD(float, __bf16) : HDT_EMBED_BWD(float, float);
}
