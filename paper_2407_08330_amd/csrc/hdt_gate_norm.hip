// The norms around a block, its gate and the residual in one:
//
//   hdt_gate_norm_fwd  c = (y - mean) rstd w_post + b_post,  h = s x + gate o c,  n = (h - mean') rstd' w + b
//   hdt_gate_norm_bwd  g = dn w,        dh' = dh + rstd' (g - mean(g) - hhat mean(g hhat)),    dx = s dh'
//                      g' = dh' gate w_post,  dy = rstd (g' - mean(g') - yhat mean(g' yhat))
//                      with A = sum dh' yhat, B = sum dh' over the rows:  dw_post = gate A, db_post = gate B, dgate = w_post A + b_post B;
//                      dw = sum dn hhat, db = sum dn
//
// Layer norms, or (rms) without means.  Bound by memory: a row's tensors are read once, held in registers between the statistics, and
// written once.  32768 bf16 rows of 768 columns: forward 49 us (201 MB, 4.1 TB/s), backward 78 (302 MB, 3.9 TB/s) and 7 for the sums over rows; a
// copy of 1 GiB reaches 5.1 TB/s.  The backward's four column sums beside a row's four tensors take 190-220 registers: two waves a SIMD, hence the next
// row's values requested before this one's are worked on (88 -> 78 us).  The same in the forward, which has five waves, cost more
// than it gave (55 -> 69; a row a wave, its vectors requested with its values: 50).  Above 8192 columns the backward's rows do not fit the
// registers of 1024 threads and lie in scratch memory.  Sums and statistics are in fp32; h is rounded once, when it is written (the second norm is taken of the unrounded sum, its
// backward of the rounded one).
#include <algorithm>

#include "hdt_internal.h"
#include "hdt_rows.h"

namespace {

using namespace hdt_rows;

struct GateArgs {
    const void *x, *y, *post_weight, *post_bias, *weight, *bias, *gate, *dn, *dh, *h;
    void *h_out, *n, *dx, *dy, *d_post_weight, *d_post_bias, *d_weight, *d_bias, *d_gate;
    float *stats, *parts;  // [4][rows]: mean and rstd of y, mean and rstd of h; [parts][4][width]
    int64_t rows;
    int width, weight_bf16, rms;
    float eps, inv_width, scale;
};

// a row's TPR threads hold its chunks of eight columns c = thread + TPR u, u < NCH; WHOLE: the width is a multiple of eight
template <int TPR, int NCH, bool WHOLE>
struct Chunks {
    template <typename F>
    static __device__ __forceinline__ void each(int t, int width, F f)
    {
#pragma unroll
        for (int u = 0; u < NCH; u++) {
            const int c = (t + TPR * u) * 8;
            if (c < width) f(u, c, width - c);
        }
    }
};

// v -> (v - mean) of the columns there are, and rstd; mean 0 with rms
template <int TPR, int NCH, bool WHOLE>
__device__ __forceinline__ void statistics(Eight (&v)[NCH], const GateArgs &a, int t, float *lds, float *mean, float *rstd)
{
    using C = Chunks<TPR, NCH, WHOLE>;
    float m = 0.f;
    if (!a.rms) {
        C::each(t, a.width, [&](int u, int, int) {
#pragma unroll
            for (int e = 0; e < 8; e++) m += v[u].x[e];
        });
        m = row_sum<TPR>(m, lds) * a.inv_width;
    }
    float sq = 0.f;
    C::each(t, a.width, [&](int u, int, int left) {
#pragma unroll
        for (int e = 0; e < 8; e++) {
            v[u].x[e] = WHOLE || e < left ? v[u].x[e] - m : 0.f;
            sq = fmaf(v[u].x[e], v[u].x[e], sq);
        }
    });
    *mean = m;
    *rstd = 1.f / sqrtf(row_sum<TPR>(sq, lds + 16) * a.inv_width + a.eps);
}

constexpr int fwd_threads(int tpr) { return tpr < 256 ? 256 : tpr; }
constexpr int bwd_threads(int tpr) { return tpr < 512 ? (tpr == 64 ? 512 : tpr) : tpr; }

// a thread's columns of the vectors, as they are in memory: requested with a row's values, which is what a wave waits for
template <typename W, int NCH>
struct Vectors {
    typename Vec<W>::V post_weight[NCH], post_bias[NCH], gate[NCH], weight[NCH], bias[NCH];
    template <bool WHOLE>
    __device__ __forceinline__ void load(const GateArgs &a, int u, int c, int left)
    {
        post_weight[u] = load8<WHOLE>((const W *)a.post_weight + c, left);
        weight[u] = load8<WHOLE>((const W *)a.weight + c, left);
        post_bias[u] = bias[u] = typename Vec<W>::V{};
        if (a.post_bias) post_bias[u] = load8<WHOLE>((const W *)a.post_bias + c, left);
        if (a.bias) bias[u] = load8<WHOLE>((const W *)a.bias + c, left);
#pragma unroll
        for (int e = 0; e < 8; e++) gate[u][e] = (W)1.f;
        if (a.gate) gate[u] = load8<WHOLE>((const W *)a.gate + c, left);
    }
};

// whether a row's registers leave room for the next row's values, which are then requested before this one's are worked on
template <typename T>
constexpr bool rows_ahead(int tpr, int nch)
{
    return tpr == 64 && nch <= 2 && sizeof(T) == 2;
}

template <typename T, typename W, int TPR, int NCH, bool WHOLE>
__global__ __launch_bounds__(fwd_threads(TPR)) void k_gate_norm_fwd(GateArgs a)
{
    constexpr int PER = fwd_threads(TPR) / TPR;
    using C = Chunks<TPR, NCH, WHOLE>;
    typedef typename Vec<T>::V V;
    __shared__ float lds[32];
    const int sub = threadIdx.x / TPR, t = threadIdx.x % TPR;
    for (int64_t row = (int64_t)blockIdx.x * PER + sub; row < a.rows; row += (int64_t)gridDim.x * PER) {
        const size_t at = (size_t)row * a.width;
        V xv[NCH];
        Eight h[NCH];
        Vectors<W, NCH> v;
        C::each(t, a.width, [&](int u, int c, int left) {
            xv[u] = load8<WHOLE>((const T *)a.x + at + c, left);
            const V yv = load8<WHOLE>((const T *)a.y + at + c, left);
#pragma unroll
            for (int e = 0; e < 8; e++) h[u].x[e] = (float)yv[e];
        });
        C::each(t, a.width, [&](int u, int c, int left) { v.template load<WHOLE>(a, u, c, left); });
        float m0, r0, m1, r1;
        statistics<TPR, NCH, WHOLE>(h, a, t, lds, &m0, &r0);
        C::each(t, a.width, [&](int u, int c, int left) {
#pragma unroll
            for (int e = 0; e < 8; e++)
                h[u].x[e] = fmaf((float)v.gate[u][e], fmaf(h[u].x[e] * r0, (float)v.post_weight[u][e], (float)v.post_bias[u][e]), a.scale * (float)xv[u][e]);
            store8<WHOLE>((T *)a.h_out + at + c, h[u], left);
        });
        statistics<TPR, NCH, WHOLE>(h, a, t, lds, &m1, &r1);
        C::each(t, a.width, [&](int u, int c, int left) {
#pragma unroll
            for (int e = 0; e < 8; e++) h[u].x[e] = fmaf(h[u].x[e] * r1, (float)v.weight[u][e], (float)v.bias[u][e]);
            store8<WHOLE>((T *)a.n + at + c, h[u], left);
        });
        if (t == 0) {
            a.stats[row] = m0;
            a.stats[a.rows + row] = r0;
            a.stats[2 * a.rows + row] = m1;
            a.stats[3 * a.rows + row] = r1;
        }
    }
}

// The columns' four sums stay in registers over a workgroup's rows; the weights, gate among them, are read again for every row (they
// stay in the L1), which leaves those registers to the sums.
template <typename T, int TPR, int NCH, bool WHOLE>
__global__ __launch_bounds__(bwd_threads(TPR)) void k_gate_norm_bwd(GateArgs a)
{
    constexpr int PER = bwd_threads(TPR) / TPR;
    using C = Chunks<TPR, NCH, WHOLE>;
    typedef typename Vec<T>::V V;
    extern __shared__ __attribute__((aligned(16))) float lds[];  // 64, then (PER > 1) PER rows of `width` up to whole chunks
    const int sub = threadIdx.x / TPR, t = threadIdx.x % TPR;
    Eight sums[4][NCH] = {};
    constexpr bool AHEAD = rows_ahead<T>(TPR, NCH);
    const int64_t step = (int64_t)gridDim.x * PER, first = (int64_t)blockIdx.x * PER + sub;
    struct Row {
        V h[NCH], y[NCH], g[NCH], d[NCH];
        float m0, r0, m1, r1;
    } next;
    auto load = [&](Row &to, int64_t row) __attribute__((always_inline)) {
        const size_t at = (size_t)row * a.width;
        to.m0 = a.stats[row], to.r0 = a.stats[a.rows + row], to.m1 = a.stats[2 * a.rows + row], to.r1 = a.stats[3 * a.rows + row];
        C::each(t, a.width, [&](int u, int c, int left) {
            to.h[u] = load8<WHOLE>((const T *)a.h + at + c, left);
            to.g[u] = load8<WHOLE>((const T *)a.dn + at + c, left);
            to.d[u] = V{};
            if (a.dh) to.d[u] = load8<WHOLE>((const T *)a.dh + at + c, left);
            to.y[u] = load8<WHOLE>((const T *)a.y + at + c, left);
        });
    };
    if (AHEAD && first < a.rows) load(next, first);
    for (int64_t row = first; row < a.rows; row += step) {
        const size_t at = (size_t)row * a.width;
        Row now;
        if (AHEAD) {
            now = next;
            if (row + step < a.rows) load(next, row + step);
        } else {
            load(now, row);
        }
        const float m0 = now.m0, r0 = now.r0, m1 = now.m1, r1 = now.r1;
        Eight hat[NCH], g[NCH];
        float s0 = 0.f, s1 = 0.f;
        C::each(t, a.width, [&](int u, int c, int left) {
            const Eight w = load_weight<WHOLE>(a.weight, a.weight_bf16, c, left);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float dn = (float)now.g[u][e];
                hat[u].x[e] = WHOLE || e < left ? ((float)now.h[u][e] - m1) * r1 : 0.f;
                sums[2][u].x[e] = fmaf(dn, hat[u].x[e], sums[2][u].x[e]);
                sums[3][u].x[e] += dn;
                g[u].x[e] = dn * w.x[e];
                s0 += g[u].x[e];
                s1 = fmaf(g[u].x[e], hat[u].x[e], s1);
            }
        });
        s0 = a.rms ? 0.f : row_sum<TPR>(s0, lds) * a.inv_width;
        s1 = row_sum<TPR>(s1, lds + 16) * a.inv_width;
        float t0 = 0.f, t1 = 0.f;
        C::each(t, a.width, [&](int u, int c, int left) {
            Eight d;
            const Eight wp = load_weight<WHOLE>(a.post_weight, a.weight_bf16, c, left);
#pragma unroll
            for (int e = 0; e < 8; e++) d.x[e] = 1.f;
            if (a.gate) d = load_weight<WHOLE>(a.gate, a.weight_bf16, c, left);
            Eight out;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float f = d.x[e] * wp.x[e], dh = fmaf(r1, g[u].x[e] - s0 - hat[u].x[e] * s1, (float)now.d[u][e]);
                out.x[e] = a.scale * dh;
                hat[u].x[e] = WHOLE || e < left ? ((float)now.y[u][e] - m0) * r0 : 0.f;
                sums[0][u].x[e] = fmaf(dh, hat[u].x[e], sums[0][u].x[e]);
                sums[1][u].x[e] += dh;
                g[u].x[e] = WHOLE || e < left ? dh * f : 0.f;
                t0 += g[u].x[e];
                t1 = fmaf(g[u].x[e], hat[u].x[e], t1);
            }
            store8<WHOLE>((T *)a.dx + at + c, out, left);
        });
        t0 = a.rms ? 0.f : row_sum<TPR>(t0, lds + 32) * a.inv_width;
        t1 = row_sum<TPR>(t1, lds + 48) * a.inv_width;
        C::each(t, a.width, [&](int u, int c, int left) {
#pragma unroll
            for (int e = 0; e < 8; e++) g[u].x[e] = r0 * (g[u].x[e] - t0 - hat[u].x[e] * t1);
            store8<WHOLE>((T *)a.dy + at + c, g[u], left);
        });
    }
    float *out = a.parts + (size_t)blockIdx.x * 4 * a.width;
    if (PER == 1) {
#pragma unroll
        for (int which = 0; which < 4; which++)
            C::each(t, a.width, [&](int u, int c, int left) { store8<WHOLE>(out + (size_t)which * a.width + c, sums[which][u], left); });
        return;
    }
    const int whole = (a.width + 7) & ~7;
#pragma unroll
    for (int which = 0; which < 4; which++) {
        __syncthreads();
        C::each(t, a.width, [&](int u, int c, int) { store8<true>(lds + 64 + (size_t)sub * whole + c, sums[which][u], 8); });
        __syncthreads();
        for (int c = threadIdx.x; c < a.width; c += TPR * PER) {
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < PER; u++) sum += lds[64 + (size_t)u * whole + c];
            out[which * a.width + c] = sum;
        }
    }
}

// the workgroups' sums added up in a fixed order, 16 columns a workgroup, 16 runs of parts; from them the gradients
constexpr int kPartColumns = 16, kPartRuns = 16;
__global__ __launch_bounds__(4 * kPartColumns * kPartRuns) void k_gate_norm_parts(GateArgs a, int parts)
{
    __shared__ float lds[kPartRuns][4][kPartColumns];
    const int lane = threadIdx.x % kPartColumns, which = threadIdx.x / kPartColumns % 4, run = threadIdx.x / (4 * kPartColumns);
    const int c = blockIdx.x * kPartColumns + lane;
    float sum = 0.f;
    if (c < a.width) {
#pragma unroll 8
        for (int p = run; p < parts; p += kPartRuns) sum += a.parts[((size_t)p * 4 + which) * a.width + c];
    }
    lds[run][which][lane] = sum;
    __syncthreads();
    if (threadIdx.x >= kPartColumns || c >= a.width) return;
    float s[4];
#pragma unroll
    for (int w = 0; w < 4; w++) {
        s[w] = 0.f;
#pragma unroll
        for (int i = 0; i < kPartRuns; i++) s[w] += lds[i][w][lane];
    }
    auto value = [&](const void *p) { return a.weight_bf16 ? (float)((const __bf16 *)p)[c] : ((const float *)p)[c]; };
    auto put = [&](void *p, float v) {
        if (!p) return;
        if (a.weight_bf16)
            ((__bf16 *)p)[c] = (__bf16)v;
        else
            ((float *)p)[c] = v;
    };
    const float g = a.gate ? value(a.gate) : 1.f;
    put(a.d_post_weight, g * s[0]);
    put(a.d_post_bias, g * s[1]);
    if (a.d_gate) put(a.d_gate, fmaf(value(a.post_weight), s[0], a.post_bias ? value(a.post_bias) * s[1] : 0.f));
    put(a.d_weight, s[2]);
    put(a.d_bias, s[3]);
}

constexpr int kMostWidth = 32768, kMostParts = 512;
constexpr int64_t kMostElements = 1ll << 35;

// (threads a row, chunks a thread): a wave while its registers hold the row, then workgroups (backward, us, a wave | a workgroup of 256: 8192 x 2048 121 | 47,
// 8192 x 1536 89 | 42; as many sums to add up as two workgroups a compute unit make, 512 | 1024: 32768 x 768 91 | 105, 8192 x 2048 57 | 58)
struct RowShape {
    int tpr, nch;
};
RowShape fwd_shape(int width)
{
    const int chunks = (width + 7) / 8;
    if (chunks <= 64) return {64, 1};
    if (chunks <= 128) return {64, 2};
    if (chunks <= 256) return {64, 4};
    return chunks <= 1024 ? RowShape{256, 4} : RowShape{1024, 4};
}
RowShape bwd_shape(int width)
{
    const int chunks = (width + 7) / 8;
    if (chunks <= 64) return {64, 1};
    if (chunks <= 128) return {64, 2};
    if (chunks <= 256) return {256, 1};
    if (chunks <= 512) return {256, 2};
    return chunks <= 1024 ? RowShape{256, 4} : RowShape{1024, 4};
}
int parts_of(int64_t rows, int width)
{
    const int tpr = bwd_shape(width).tpr, per = bwd_threads(tpr) / tpr;
    return (int)std::min<int64_t>((rows + per - 1) / per, kMostParts);
}

template <typename T, int TPR, int NCH, bool WHOLE>
void launch_fwd(const GateArgs &a, hipStream_t st)
{
    constexpr int PER = fwd_threads(TPR) / TPR;
    const dim3 grid((unsigned)std::min<int64_t>((a.rows + PER - 1) / PER, 1 << 20)), block(fwd_threads(TPR));
    if (a.weight_bf16)
        hipLaunchKernelGGL((k_gate_norm_fwd<T, __bf16, TPR, NCH, WHOLE>), grid, block, 0, st, a);
    else
        hipLaunchKernelGGL((k_gate_norm_fwd<T, float, TPR, NCH, WHOLE>), grid, block, 0, st, a);
}
template <typename T, int TPR, int NCH, bool WHOLE>
void launch_bwd(const GateArgs &a, hipStream_t st)
{
    constexpr int PER = bwd_threads(TPR) / TPR;
    const size_t lds = (64 + (PER > 1 ? (size_t)PER * ((a.width + 7) & ~7) : 0)) * sizeof(float);
    hipLaunchKernelGGL((k_gate_norm_bwd<T, TPR, NCH, WHOLE>), dim3((unsigned)parts_of(a.rows, a.width)), dim3(bwd_threads(TPR)), lds, st, a);
}
template <typename T, bool WHOLE>
void launch(const GateArgs &a, bool bwd, hipStream_t st)
{
    const RowShape s = bwd ? bwd_shape(a.width) : fwd_shape(a.width);
    if (!bwd) {
        if (s.tpr == 64 && s.nch == 1) return launch_fwd<T, 64, 1, WHOLE>(a, st);
        if (s.tpr == 64 && s.nch == 2) return launch_fwd<T, 64, 2, WHOLE>(a, st);
        if (s.tpr == 64) return launch_fwd<T, 64, 4, WHOLE>(a, st);
        if (s.tpr == 256) return launch_fwd<T, 256, 4, WHOLE>(a, st);
        return launch_fwd<T, 1024, 4, WHOLE>(a, st);
    }
    if (s.tpr == 64 && s.nch == 1) return launch_bwd<T, 64, 1, WHOLE>(a, st);
    if (s.tpr == 64) return launch_bwd<T, 64, 2, WHOLE>(a, st);
    if (s.tpr == 256 && s.nch == 1) return launch_bwd<T, 256, 1, WHOLE>(a, st);
    if (s.tpr == 256 && s.nch == 2) return launch_bwd<T, 256, 2, WHOLE>(a, st);
    if (s.tpr == 256) return launch_bwd<T, 256, 4, WHOLE>(a, st);
    launch_bwd<T, 1024, 4, WHOLE>(a, st);
}
void launch(const GateArgs &a, bool bwd, hdt_dtype_t dt, hipStream_t st)
{
    const bool whole = a.width % 8 == 0;
    if (dt == HDT_BF16)
        whole ? launch<__bf16, true>(a, bwd, st) : launch<__bf16, false>(a, bwd, st);
    else
        whole ? launch<float, true>(a, bwd, st) : launch<float, false>(a, bwd, st);
}

bool misaligned(const void *p, unsigned by = 16) { return ((uintptr_t)p & (by - 1)) != 0; }

hdt_status_t check_sizes(const char *fn, int64_t rows, int32_t width, float scale, hdt_dtype_t dt, hdt_dtype_t wdt)
{
    if (rows < 0 || width < 0) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: negative size", fn);
    if (!hdt_finite(scale)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: scale = %g", fn, (double)scale);
    if (dt != HDT_BF16 && dt != HDT_F32) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, (int)dt);
    if (wdt != HDT_BF16 && wdt != HDT_F32) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d of the weights", fn, (int)wdt);
    if (width < 1 || width > kMostWidth) return hdt_fail(HDT_ERR_SHAPE, "%s: width %d outside [1, %d]", fn, width, kMostWidth);
    if (rows > INT32_MAX || rows * width > kMostElements) return hdt_fail(HDT_ERR_SHAPE, "%s: more than 2^31 rows or 2^35 elements", fn);
    return HDT_OK;
}

#define HDT_EXPORT extern "C" __attribute__((visibility("default")))

}  // namespace

HDT_EXPORT hdt_status_t hdt_gate_norm_fwd(const void *x, const void *y, const void *post_weight, const void *post_bias, const void *gate,
                                          const void *weight, const void *bias, int64_t rows, int32_t width, float eps, float scale, int32_t rms,
                                          void *h, void *n, float *stats, hdt_dtype_t dt, hdt_dtype_t weight_dt, void *stream)
{
    const char *fn = "hdt_gate_norm_fwd";
    if (hdt_status_t st = check_sizes(fn, rows, width, scale, dt, weight_dt)) return st;
    if (!hdt_finite(eps) || eps < 0.f) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: eps = %g", fn, (double)eps);
    if (rows == 0) return HDT_OK;
    if (!x || !y || !post_weight || !weight || !h || !n || !stats) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    const void *in[] = {x, y, post_weight, post_bias, gate, weight, bias}, *out[] = {h, n, stats};
    for (const void *p : in)
        if (misaligned(p)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    if (misaligned(h) || misaligned(n) || misaligned(stats, 4)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    for (const void *o : out)
        for (const void *p : in)
            if (o == p) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: output aliases an input", fn);
    if (h == n || stats == h || stats == n) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: outputs alias each other", fn);
    GateArgs a = {};
    a.x = x, a.y = y, a.post_weight = post_weight, a.post_bias = post_bias, a.gate = gate, a.weight = weight, a.bias = bias, a.h_out = h, a.n = n, a.stats = stats;
    a.rows = rows, a.width = width, a.weight_bf16 = weight_dt == HDT_BF16, a.rms = rms != 0, a.eps = eps, a.inv_width = 1.f / (float)width, a.scale = scale;
    hipStream_t st = (hipStream_t)stream;
    HdtTimer t("hdt_gate_norm_fwd", st);
    launch(a, false, dt, st);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

HDT_EXPORT size_t hdt_gate_norm_bwd_workspace_bytes(int64_t rows, int32_t width)
{
    if (rows <= 0 || rows > INT32_MAX || width < 1 || width > kMostWidth) return 0;
    return (size_t)parts_of(rows, width) * 4 * width * sizeof(float);
}

HDT_EXPORT hdt_status_t hdt_gate_norm_bwd(const void *dn, const void *dh, const void *h, const void *y, const float *stats, const void *post_weight,
                                          const void *post_bias, const void *gate, const void *weight, int64_t rows, int32_t width, float scale, int32_t rms,
                                          void *dx, void *dy, void *d_post_weight, void *d_post_bias, void *d_gate, void *d_weight, void *d_bias,
                                          hdt_dtype_t dt, hdt_dtype_t weight_dt, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "hdt_gate_norm_bwd";
    if (hdt_status_t st = check_sizes(fn, rows, width, scale, dt, weight_dt)) return st;
    if (!post_weight || !weight || !d_post_weight || !d_weight) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (d_gate && !gate) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: a gradient of a gate that is not there", fn);
    const void *in[] = {dn, dh, h, y, stats, post_weight, post_bias, gate, weight};
    const void *out[] = {rows > 0 ? dx : nullptr, rows > 0 ? dy : nullptr, d_post_weight, d_post_bias, d_gate, d_weight, d_bias};
    if (rows > 0) {
        if (!dn || !h || !y || !stats || !dx || !dy) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
        for (const void *p : {dn, dh, h, y, (const void *)dx, (const void *)dy})
            if (misaligned(p)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
        if (misaligned(stats, 4)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: misaligned statistics", fn);
    }
    for (const void *p : {post_weight, post_bias, gate, weight})
        if (misaligned(p)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    for (const void *p : {(const void *)d_post_weight, (const void *)d_post_bias, (const void *)d_gate, (const void *)d_weight, (const void *)d_bias})
        if (misaligned(p, weight_dt == HDT_BF16 ? 2 : 4)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: misaligned gradient", fn);
    for (int i = 0; i < 7; i++) {
        if (!out[i]) continue;
        for (const void *p : in)
            if (out[i] == p) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: output aliases an input", fn);
        for (int j = 0; j < i; j++)
            if (out[i] == out[j]) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: outputs alias each other", fn);
    }
    const size_t need = hdt_gate_norm_bwd_workspace_bytes(rows, width);
    if (rows > 0 && (!workspace || workspace_bytes < need || misaligned(workspace)))
        return hdt_fail(HDT_ERR_INVALID_ARG, "%s: a 16-byte aligned workspace of %zu bytes needed, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
    GateArgs a = {};
    a.dn = dn, a.dh = dh, a.h = h, a.y = y, a.stats = (float *)stats, a.post_weight = post_weight, a.post_bias = post_bias, a.gate = gate, a.weight = weight;
    a.dx = dx, a.dy = dy, a.d_post_weight = d_post_weight, a.d_post_bias = d_post_bias, a.d_gate = d_gate, a.d_weight = d_weight, a.d_bias = d_bias;
    a.parts = (float *)workspace;
    a.rows = rows, a.width = width, a.weight_bf16 = weight_dt == HDT_BF16, a.rms = rms != 0, a.inv_width = 1.f / (float)width, a.scale = scale;
    hipStream_t st = (hipStream_t)stream;
    if (rows > 0) {
        HdtTimer t("hdt_gate_norm_bwd", st);
        launch(a, true, dt, st);
        HDT_HIP_TRY(hipGetLastError());
    }
    HdtTimer t("hdt_gate_norm_parts", st);
    hipLaunchKernelGGL(k_gate_norm_parts, dim3((unsigned)((width + kPartColumns - 1) / kPartColumns)), dim3(4 * kPartColumns * kPartRuns), 0, st, a,
                       rows > 0 ? parts_of(rows, width) : 0);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}
