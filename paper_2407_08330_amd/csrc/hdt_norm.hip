// What stands between the attention calls of a pre-norm block: dropout from a counter-based generator, the residual, layer norm.
//
//   hdt_dropout_add   out = x + y o m                       (x may be missing; the gradient of y is the same call on the gradient)
//   hdt_add_norm_fwd  h = x + y o m,  n = (h - mean) rstd w + b
//   hdt_add_norm_bwd  g = dn w,  dx = dh + rstd (g - mean(g) - xhat mean(g xhat)),  dy = dx o m,  dw = sum dn xhat,  db = sum dn
//
// The mask m is never stored: both passes compute it from (seed, step, site, element).  Eight elements share one block of
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC 2011), 16 bits each; an element is kept iff its 16 bits are at least
// t = round(65536 p), and what is kept is multiplied by 65536 / (65536 - t), the inverse of the probability that 16 bits really give.
//
// All of it is bound by memory: a row is read once, held in registers between its statistics and its result, and written once.  On 32768
// bf16 rows of 768 columns: dropout with residual 26 us (151 MB, 5.7 TB/s), norm forward and backward 92 us (453 MB, 4.9 TB/s); a copy
// of 200 MB reaches 5.4 TB/s, one of 2 GB 4.9.  Two things are slower.  Above 8192 columns the backward's row does not fit the registers of
// its 1024 threads (128 each): 264 to 603 values a thread lie in scratch memory, 1.0-1.9 TB/s.  Widths that are no multiple of eight have
// their accesses aligned to an element only and every chunk's random numbers from two blocks: bf16 2.2 TB/s, fp32 2.8-3.8.
// Sums and statistics are in fp32; h is rounded once, when it is written (the norm is taken of the unrounded sum).
#include <algorithm>

#include "hdt_internal.h"
#include "hdt_lanes.h"
#include "hdt_mfma.h"

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;

struct Drop {
    const long long *rng;  // device: seed, step
    uint32_t site, threshold;  // threshold 0: nothing is dropped
    float keep_scale;
};
struct Key {
    uint32_t seed_lo, seed_hi, step_lo, step_hi;
};
__device__ __forceinline__ Key key_of(const Drop &d)
{
    if (d.threshold == 0) return {};
    const unsigned long long seed = (unsigned long long)d.rng[0], step = (unsigned long long)d.rng[1];
    return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)step, (uint32_t)(step >> 32)};
}

struct Block {
    uint32_t w[4];
};
__device__ __forceinline__ Block philox(uint32_t block, uint32_t site, const Key &k)
{
    uint32_t c0 = block, c1 = site, c2 = k.step_lo, c3 = k.step_hi, k0 = k.seed_lo, k1 = k.seed_hi;
#pragma unroll
    for (int i = 0; i < 10; i++) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}
// the 16-bit numbers of elements at .. at + 7; WHOLE: of one block
template <bool WHOLE>
__device__ __forceinline__ Block numbers(unsigned long long at, const Drop &d, const Key &k)
{
    const uint32_t block = (uint32_t)(at >> 3), off = (uint32_t)at & 7u;
    Block a = philox(block, d.site, k);
    if (WHOLE || off == 0) return a;
    const Block b = philox(block + 1, d.site, k);
    uint32_t w[8] = {a.w[0], a.w[1], a.w[2], a.w[3], b.w[0], b.w[1], b.w[2], b.w[3]};
#pragma unroll
    for (int s = 4; s >= 1; s >>= 1) {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i + s < 8) w[i] = (off >> 1) & s ? w[i + s] : w[i];
    }
#pragma unroll
    for (int i = 0; i < 4; i++) a.w[i] = off & 1 ? (w[i] >> 16) | (w[i + 1] << 16) : w[i];
    return a;
}
// the factors of elements e of a block
__device__ __forceinline__ float factor(const Block &b, int e, const Drop &d)
{
    const uint32_t u = e & 1 ? b.w[e >> 1] >> 16 : b.w[e >> 1] & 0xffffu;
    return u >= d.threshold ? d.keep_scale : 0.f;
}

// 8 consecutive elements as they are in memory; `left` of them exist (WHOLE: all).  The address is aligned to an element only.
template <typename T>
struct Vec {
    typedef T V __attribute__((ext_vector_type(8)));
    typedef V Any __attribute__((aligned(sizeof(T))));
};
template <bool WHOLE, typename T>
__device__ __forceinline__ typename Vec<T>::V load8(const T *p, int left)
{
    if (WHOLE || left >= 8) return *reinterpret_cast<const typename Vec<T>::Any *>(p);
    typename Vec<T>::V r;
#pragma unroll
    for (int e = 0; e < 8; e++) r[e] = e < left ? p[e] : (T)0.f;
    return r;
}
struct Eight {
    float x[8];
};
template <bool WHOLE, typename T>
__device__ __forceinline__ void store8(T *p, const Eight &r, int left)
{
    if (WHOLE || left >= 8) {
        typename Vec<T>::V v;
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (T)r.x[e];
        *reinterpret_cast<typename Vec<T>::Any *>(p) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (e < left) p[e] = (T)r.x[e];
}
template <bool WHOLE>
__device__ __forceinline__ Eight load_weight(const void *p, int bf16, int at, int left)
{
    Eight r;
    if (bf16) {
        const auto v = load8<WHOLE>((const __bf16 *)p + at, left);
#pragma unroll
        for (int e = 0; e < 8; e++) r.x[e] = (float)v[e];
    } else {
        const auto v = load8<WHOLE>((const float *)p + at, left);
#pragma unroll
        for (int e = 0; e < 8; e++) r.x[e] = v[e];
    }
    return r;
}

// ------------------------------------------------------------------------------------------ dropout + residual
template <typename T>
__global__ __launch_bounds__(256) void k_dropout_add(const T *y, const T *x, T *out, unsigned long long n, Drop d)
{
    const Key k = key_of(d);
    for (unsigned long long at = ((unsigned long long)blockIdx.x * 256 + threadIdx.x) * 8; at < n; at += (unsigned long long)gridDim.x * 2048) {
        const int left = (int)min(n - at, 8ull);
        const typename Vec<T>::V yv = load8<false>(y + at, left);
        typename Vec<T>::V xv = {};
        if (x) xv = load8<false>(x + at, left);
        Block b = {};
        if (d.threshold) b = philox((uint32_t)(at >> 3), d.site, k);
        Eight v;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            v.x[e] = (float)yv[e];
            if (d.threshold) v.x[e] *= factor(b, e, d);
            if (x) v.x[e] += (float)xv[e];
        }
        store8<false>(out + at, v, left);
    }
}

// ------------------------------------------------------------------------------------------ sums over a row
// the sum over the threads of a row: a wave, or (TPR > 64) the whole workgroup
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float *lds)
{
    x = hdt_lanes::wave_sum(x);
    if (TPR > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int i = 0; i < TPR / 64; i++) x += lds[i];
    }
    return x;
}

struct NormArgs {
    const void *x, *y, *weight, *bias, *dn, *dh, *h;
    void *h_out, *n, *dx, *dy, *d_weight, *d_bias;
    float *mean, *rstd, *parts;
    int rows, width, weight_bf16;
    float eps, inv_width;
    Drop drop;
};

// A row's TPR threads hold its chunks of eight columns c = thread + TPR u, u < NCH.  WHOLE: the width is a multiple of eight, so that
// chunks are whole, and a chunk's random numbers those of one block.
template <int TPR, int NCH>
struct Shape {
    static constexpr int FWD = TPR < 256 ? 256 : TPR, BWD = TPR > 64 ? TPR : NCH < 4 ? 512 : 256;  // threads of a workgroup
};

template <typename T, int TPR, int NCH, bool WHOLE, bool DROP>
__global__ __launch_bounds__((Shape<TPR, NCH>::FWD)) void k_add_norm_fwd(NormArgs a)
{
    constexpr int PER = Shape<TPR, NCH>::FWD / TPR;
    typedef typename Vec<T>::V V;
    __shared__ float lds[16];
    const int sub = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const Key k = DROP ? key_of(a.drop) : Key{};
    for (int64_t row = (int64_t)blockIdx.x * PER + sub; row < a.rows; row += (int64_t)gridDim.x * PER) {  // (the same for whole waves, and for a workgroup that has one row)
        const size_t at = (size_t)row * a.width;
        V x[NCH], y[NCH];
#pragma unroll
        for (int u = 0; u < NCH; u++) {
            const int c = (t + TPR * u) * 8, left = a.width - c;
            x[u] = V{}, y[u] = V{};
            if (left > 0) {
                x[u] = load8<WHOLE>((const T *)a.x + at + c, left);
                if (a.y) y[u] = load8<WHOLE>((const T *)a.y + at + c, left);
            }
        }
        Eight h[NCH];
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < NCH; u++) {
            const int c = (t + TPR * u) * 8, left = a.width - c;
            Block b = {};
            if (DROP && left > 0) b = numbers<WHOLE>(at + c, a.drop, k);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                h[u].x[e] = (float)x[u][e] + (DROP ? (float)y[u][e] * factor(b, e, a.drop) : (float)y[u][e]);
                sum += h[u].x[e];
            }
            if (a.y && left > 0) store8<WHOLE>((T *)a.h_out + at + c, h[u], left);
        }
        const float mean = row_sum<TPR>(sum, lds) * a.inv_width;
        float sq = 0.f;
#pragma unroll
        for (int u = 0; u < NCH; u++) {
            const int left = a.width - (t + TPR * u) * 8;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                h[u].x[e] = (WHOLE ? 0 : e) < left ? h[u].x[e] - mean : 0.f;
                sq = fmaf(h[u].x[e], h[u].x[e], sq);
            }
        }
        const float rstd = 1.f / sqrtf(row_sum<TPR>(sq, lds) * a.inv_width + a.eps);
#pragma unroll
        for (int u = 0; u < NCH; u++) {
            const int c = (t + TPR * u) * 8, left = a.width - c;
            if (left <= 0) continue;
            const Eight w = load_weight<WHOLE>(a.weight, a.weight_bf16, c, left);
            Eight b = {};
            if (a.bias) b = load_weight<WHOLE>(a.bias, a.weight_bf16, c, left);
#pragma unroll
            for (int e = 0; e < 8; e++) h[u].x[e] = fmaf(h[u].x[e] * rstd, w.x[e], b.x[e]);
            store8<WHOLE>((T *)a.n + at + c, h[u], left);
        }
        if (t == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
    }
}

// Rows blockIdx, blockIdx + gridDim, ... of a workgroup's wave (or of the workgroup), the columns' sums of dn xhat and dn in
// registers throughout; at the end a row of the workgroup's sums: parts[workgroup][2][width]
template <typename T, int TPR, int NCH, bool WHOLE, bool DROP>
__global__ __launch_bounds__((Shape<TPR, NCH>::BWD)) void k_add_norm_bwd(NormArgs a)
{
    constexpr int PER = Shape<TPR, NCH>::BWD / TPR;
    typedef typename Vec<T>::V V;
    extern __shared__ __attribute__((aligned(16))) float lds[];  // 32, then (PER > 1) PER rows of `width` up to whole chunks
    const int sub = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const Key k = DROP ? key_of(a.drop) : Key{};
    Eight w[NCH], sw[NCH] = {}, sb[NCH] = {};
#pragma unroll
    for (int u = 0; u < NCH; u++) {
        const int c = (t + TPR * u) * 8;
        if (c < a.width) w[u] = load_weight<WHOLE>(a.weight, a.weight_bf16, c, a.width - c);
    }
    for (int64_t row = (int64_t)blockIdx.x * PER + sub; row < a.rows; row += (int64_t)gridDim.x * PER) {
        const size_t at = (size_t)row * a.width;
        const float mean = a.mean[row], rstd = a.rstd[row];
        V hv[NCH], gv[NCH], dv[NCH];
#pragma unroll
        for (int u = 0; u < NCH; u++) {
            const int c = (t + TPR * u) * 8, left = a.width - c;
            hv[u] = V{}, gv[u] = V{}, dv[u] = V{};
            if (left > 0) {
                hv[u] = load8<WHOLE>((const T *)a.h + at + c, left);
                gv[u] = load8<WHOLE>((const T *)a.dn + at + c, left);
                if (a.dh) dv[u] = load8<WHOLE>((const T *)a.dh + at + c, left);
            }
        }
        Eight hat[NCH], g[NCH];
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int u = 0; u < NCH; u++) {
            const int left = a.width - (t + TPR * u) * 8;
            if (left <= 0) continue;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float dn = (float)gv[u][e];
                hat[u].x[e] = WHOLE || e < left ? ((float)hv[u][e] - mean) * rstd : 0.f;
                sw[u].x[e] = fmaf(dn, hat[u].x[e], sw[u].x[e]);
                sb[u].x[e] += dn;
                g[u].x[e] = dn * w[u].x[e];
                s0 += g[u].x[e];
                s1 = fmaf(g[u].x[e], hat[u].x[e], s1);
            }
        }
        s0 = row_sum<TPR>(s0, lds) * a.inv_width;
        s1 = row_sum<TPR>(s1, lds + 16) * a.inv_width;
#pragma unroll
        for (int u = 0; u < NCH; u++) {
            const int c = (t + TPR * u) * 8, left = a.width - c;
            if (left <= 0) continue;
            Eight d;
#pragma unroll
            for (int e = 0; e < 8; e++) d.x[e] = fmaf(rstd, g[u].x[e] - s0 - hat[u].x[e] * s1, (float)dv[u][e]);
            store8<WHOLE>((T *)a.dx + at + c, d, left);
            if (DROP) {
                const Block b = numbers<WHOLE>(at + c, a.drop, k);
#pragma unroll
                for (int e = 0; e < 8; e++) d.x[e] *= factor(b, e, a.drop);
                store8<WHOLE>((T *)a.dy + at + c, d, left);
            }
        }
    }
    float *out = a.parts + (size_t)blockIdx.x * 2 * a.width;
    if (PER == 1) {
#pragma unroll
        for (int u = 0; u < NCH; u++) {
            const int c = (t + TPR * u) * 8;
            if (c >= a.width) continue;
            store8<WHOLE>(out + c, sw[u], a.width - c);
            store8<WHOLE>(out + a.width + c, sb[u], a.width - c);
        }
        return;
    }
    const int whole = (a.width + 7) & ~7;
#pragma unroll
    for (int which = 0; which < 2; which++) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < NCH; u++) {
            const int c = (t + TPR * u) * 8;
            if (c < a.width) store8<true>(lds + 32 + (size_t)sub * whole + c, which ? sb[u] : sw[u], 8);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.width; c += TPR * PER) {
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < PER; u++) sum += lds[32 + (size_t)u * whole + c];
            out[which * a.width + c] = sum;
        }
    }
}

// The workgroups' sums added up in a fixed order: 16 columns a workgroup, 64 runs of parts.  (64 columns and 16 runs left most of the
// chip idle: 1536 sums of 1024 parts 20.4 us.)
constexpr int kPartColumns = 16, kPartRuns = 64;
__global__ __launch_bounds__(kPartColumns * kPartRuns) void k_norm_parts(NormArgs a, int parts)
{
    __shared__ float lds[kPartRuns][kPartColumns];
    const int lane = threadIdx.x % kPartColumns, run = threadIdx.x / kPartColumns, x = blockIdx.x * kPartColumns + lane;
    float sum = 0.f;
    if (x < 2 * a.width) {
#pragma unroll 8
        for (int p = run; p < parts; p += kPartRuns) sum += a.parts[(size_t)p * 2 * a.width + x];
    }
    lds[run][lane] = sum;
    __syncthreads();
    if (run != 0 || x >= 2 * a.width) return;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPartRuns; i++) sum += lds[i][lane];
    void *out = x < a.width ? a.d_weight : a.d_bias;
    const int c = x < a.width ? x : x - a.width;
    if (!out) return;
    if (a.weight_bf16)
        ((__bf16 *)out)[c] = (__bf16)sum;
    else
        ((float *)out)[c] = sum;
}

constexpr int kMostWidth = 32768, kMostParts = 512;
constexpr long long kMostElements = 1ll << 35;  // 2^32 blocks of eight

// threads a row and chunks a thread: a wave up to 2048 columns, then a workgroup of 256 or 1024 (us at 32768 bf16 rows, wave | workgroup of
// 256: 768 columns 36 | 91 forward, 48 | 93 backward; 2048 columns 99 | 129, 137 | 135; 4096 rows of 2048 14.7 | 17.7, 26 | 25).  TB/s
// forward, backward, dropping: bf16 16384 x 4096 5.6, 5.0; 8192 x 8192 5.4, 4.6; 4096 x 12288 4.2, 1.7; 2048 x 32768 4.7, 1.3; 16384 x 2049
// 2.2, 2.2; 8192 x 8193 2.1, 1.2; fp32 16384 x 4096 5.8, 5.3; 8192 x 8192 5.5, 4.9; 4096 x 12288 4.5, 1.5; 2048 x 32768 4.9, 1.6
struct RowShape {
    int tpr, nch;
};
RowShape row_shape(int width)
{
    const int chunks = (width + 7) / 8;
    if (chunks <= 64) return {64, 1};
    if (chunks <= 128) return {64, 2};
    if (chunks <= 256) return {64, 4};
    return chunks <= 1024 ? RowShape{256, 4} : RowShape{1024, 4};
}
// workgroups of the backward: two per compute unit, and no more sums to add up behind it than that takes (us at 32768 bf16 rows, 256 | 512 |
// 1024 workgroups: 768 columns 46 | 48 | 54, 2048 columns 184 | 137 | 143)
int norm_parts(int rows, int width)
{
    const RowShape s = row_shape(width);
    const int per = s.tpr == 64 ? (s.nch < 4 ? Shape<64, 1>::BWD : Shape<64, 4>::BWD) / 64 : 1;
    return (int)std::min<int64_t>(((int64_t)rows + per - 1) / per, kMostParts);
}

template <typename T, int TPR, int NCH, bool WHOLE, bool DROP>
void launch_one(const NormArgs &a, bool bwd, hipStream_t st)
{
    using S = Shape<TPR, NCH>;
    if (!bwd) {
        const int64_t grid = std::min<int64_t>(((int64_t)a.rows + S::FWD / TPR - 1) / (S::FWD / TPR), 1 << 20);
        hipLaunchKernelGGL((k_add_norm_fwd<T, TPR, NCH, WHOLE, DROP>), dim3((unsigned)grid), dim3(S::FWD), 0, st, a);
    } else {
        constexpr int PER = S::BWD / TPR;
        const size_t lds = (32 + (PER > 1 ? (size_t)PER * ((a.width + 7) & ~7) : 0)) * sizeof(float);
        hipLaunchKernelGGL((k_add_norm_bwd<T, TPR, NCH, WHOLE, DROP>), dim3((unsigned)norm_parts(a.rows, a.width)), dim3(S::BWD), lds, st, a);
    }
}
template <typename T, int TPR, int NCH>
void launch_shape(const NormArgs &a, bool bwd, hipStream_t st)
{
    const bool whole = a.width % 8 == 0, drop = a.drop.threshold != 0;
    if (whole)
        drop ? launch_one<T, TPR, NCH, true, true>(a, bwd, st) : launch_one<T, TPR, NCH, true, false>(a, bwd, st);
    else
        drop ? launch_one<T, TPR, NCH, false, true>(a, bwd, st) : launch_one<T, TPR, NCH, false, false>(a, bwd, st);
}
template <typename T>
void launch(const NormArgs &a, bool bwd, hipStream_t st)
{
    const RowShape s = row_shape(a.width);
    if (s.tpr == 64 && s.nch == 1) return launch_shape<T, 64, 1>(a, bwd, st);
    if (s.tpr == 64 && s.nch == 2) return launch_shape<T, 64, 2>(a, bwd, st);
    if (s.tpr == 64) return launch_shape<T, 64, 4>(a, bwd, st);
    if (s.tpr == 256) return launch_shape<T, 256, 4>(a, bwd, st);
    launch_shape<T, 1024, 4>(a, bwd, st);
}

bool misaligned(const void *p) { return ((uintptr_t)p & 15u) != 0; }

// any: there is an element to drop
hdt_status_t drop_of(const char *fn, double p, bool any, const int64_t *rng, uint32_t site, Drop *d)
{
    if (!hdt_finite(p) || p < 0. || p >= 1.) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: p = %g outside [0, 1)", fn, p);
    const uint32_t t = (uint32_t)(p * 65536. + 0.5);
    if (t > 65535) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: p = %g rounds to 1 in steps of 1/65536", fn, p);
    if (t > 0 && any && !rng) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL generator state", fn);
    if ((uintptr_t)rng & 7u) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: the generator's state must be 8-byte aligned", fn);
    *d = {(const long long *)rng, site, t, (float)(65536. / (65536. - t))};
    return HDT_OK;
}
hdt_status_t check_norm(const char *fn, int64_t rows, int32_t width, hdt_dtype_t dt, hdt_dtype_t wdt)
{
    if (rows < 0 || width < 0) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: negative size", fn);
    if (dt != HDT_BF16 && dt != HDT_F32) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, (int)dt);
    if (wdt != HDT_BF16 && wdt != HDT_F32) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d of the weight", fn, (int)wdt);
    if (width < 1 || width > kMostWidth) return hdt_fail(HDT_ERR_SHAPE, "%s: width %d outside [1, %d]", fn, width, kMostWidth);
    if (rows > INT32_MAX || rows * width > kMostElements) return hdt_fail(HDT_ERR_SHAPE, "%s: more than 2^31 rows or 2^35 elements", fn);
    return HDT_OK;
}

#define HDT_EXPORT extern "C" __attribute__((visibility("default")))

}  // namespace

HDT_EXPORT hdt_status_t hdt_dropout_add(const void *y, const void *x, void *out, int64_t n, double p, const int64_t *d_rng, uint32_t site,
                                        hdt_dtype_t dt, void *stream)
{
    const char *fn = "hdt_dropout_add";
    if (n < 0) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: negative size", fn);
    if (n > kMostElements) return hdt_fail(HDT_ERR_SHAPE, "%s: more than 2^35 elements", fn);
    if (dt != HDT_BF16 && dt != HDT_F32) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, (int)dt);
    Drop d;
    const bool any = n > 0;
    if (hdt_status_t st = drop_of(fn, p, any, d_rng, site, &d)) return st;
    if (n == 0) return HDT_OK;
    if (!y || !out) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (misaligned(y) || misaligned(x) || misaligned(out)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    hipStream_t st = (hipStream_t)stream;
    HdtTimer t("hdt_dropout_add", st);
    const dim3 grid((unsigned)(n > (1ll << 31) ? 1 << 20 : (n + 2047) / 2048)), block(256);  // (a launch has fewer than 2^32 threads)
    if (dt == HDT_BF16)
        hipLaunchKernelGGL(k_dropout_add<__bf16>, grid, block, 0, st, (const __bf16 *)y, (const __bf16 *)x, (__bf16 *)out, (unsigned long long)n, d);
    else
        hipLaunchKernelGGL(k_dropout_add<float>, grid, block, 0, st, (const float *)y, (const float *)x, (float *)out, (unsigned long long)n, d);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

HDT_EXPORT hdt_status_t hdt_add_norm_fwd(const void *x, const void *y, const void *weight, const void *bias, int64_t rows, int32_t width,
                                         float eps, double p, const int64_t *d_rng, uint32_t site, void *h, void *n, float *mean, float *rstd,
                                         hdt_dtype_t dt, hdt_dtype_t weight_dt, void *stream)
{
    const char *fn = "hdt_add_norm_fwd";
    if (hdt_status_t st = check_norm(fn, rows, width, dt, weight_dt)) return st;
    if (!hdt_finite(eps) || eps < 0.f) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: eps = %g", fn, (double)eps);
    NormArgs a = {};
    const bool any = rows > 0;
    if (hdt_status_t st = drop_of(fn, p, any, d_rng, site, &a.drop)) return st;
    if (rows == 0) return HDT_OK;
    if (!x || !weight || !n || !mean || !rstd || (y && !h)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    for (const void *q : {x, y, weight, bias, (const void *)h, (const void *)n})
        if (misaligned(q)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    if (n == x || n == y || (y && (h == x || h == y || h == n))) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: output aliases an input or the other output", fn);
    if (!y) a.drop.threshold = 0;
    a.x = x, a.y = y, a.weight = weight, a.bias = bias, a.h_out = h, a.n = n, a.mean = mean, a.rstd = rstd;
    a.rows = (int)rows, a.width = width, a.weight_bf16 = weight_dt == HDT_BF16, a.eps = eps, a.inv_width = 1.f / (float)width;
    hipStream_t st = (hipStream_t)stream;
    HdtTimer t("hdt_add_norm_fwd", st);
    dt == HDT_BF16 ? launch<__bf16>(a, false, st) : launch<float>(a, false, st);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

HDT_EXPORT size_t hdt_add_norm_bwd_workspace_bytes(int64_t rows, int32_t width)
{
    if (rows <= 0 || rows > INT32_MAX || width < 1 || width > kMostWidth) return 0;
    return (size_t)norm_parts((int)rows, width) * 2 * width * sizeof(float);
}

HDT_EXPORT hdt_status_t hdt_add_norm_bwd(const void *dn, const void *dh, const void *h, const void *weight, const float *mean,
                                         const float *rstd, int64_t rows, int32_t width, double p, const int64_t *d_rng, uint32_t site,
                                         void *dx, void *dy, void *d_weight, void *d_bias, hdt_dtype_t dt, hdt_dtype_t weight_dt,
                                         void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "hdt_add_norm_bwd";
    if (hdt_status_t st = check_norm(fn, rows, width, dt, weight_dt)) return st;
    NormArgs a = {};
    const bool any = rows > 0;
    if (hdt_status_t st = drop_of(fn, p, any, d_rng, site, &a.drop)) return st;
    if (!d_weight) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (rows > 0) {
        if (!dn || !h || !weight || !mean || !rstd || !dx || (a.drop.threshold && !dy)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
        const void *in[] = {dn, dh, h, weight, mean, rstd}, *out[] = {dx, a.drop.threshold ? dy : nullptr};
        for (const void *q : {dn, dh, h, weight, (const void *)dx, (const void *)dy})
            if (misaligned(q)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
        for (const void *o : out)
            for (const void *q : in)
                if (o && o == q) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: output aliases an input", fn);
        if (out[0] == out[1]) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: outputs alias each other", fn);
        const size_t need = hdt_add_norm_bwd_workspace_bytes(rows, width);
        if (!workspace || workspace_bytes < need || misaligned(workspace))
            return hdt_fail(HDT_ERR_INVALID_ARG, "%s: a 16-byte aligned workspace of %zu bytes needed, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
    }
    a.dn = dn, a.dh = dh, a.h = h, a.weight = weight, a.mean = (float *)mean, a.rstd = (float *)rstd, a.dx = dx, a.dy = dy;
    a.d_weight = d_weight, a.d_bias = d_bias, a.parts = (float *)workspace;
    a.rows = (int)rows, a.width = width, a.weight_bf16 = weight_dt == HDT_BF16, a.inv_width = 1.f / (float)width;
    hipStream_t st = (hipStream_t)stream;
    if (rows > 0) {
        HdtTimer t("hdt_add_norm_bwd", st);
        dt == HDT_BF16 ? launch<__bf16>(a, true, st) : launch<float>(a, true, st);
        HDT_HIP_TRY(hipGetLastError());
    }
    HdtTimer t("hdt_norm_parts", st);
    hipLaunchKernelGGL(k_norm_parts, dim3((unsigned)((2 * width + kPartColumns - 1) / kPartColumns)), dim3(kPartColumns * kPartRuns), 0, st, a, rows > 0 ? norm_parts((int)rows, width) : 0);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}
