// Gated feed-forward block: checks, what kernel takes which product, the calls.  hdt_ffn.h has the mathematics.
#include <algorithm>

#include "hdt_ffn.h"
#include "hdt_ffn_plain.h"

namespace {

using namespace hdt_ffn;

constexpr int kMostSize = 65536;
constexpr int64_t kMostElements = 1ll << 35;

bool misaligned(const void *p) { return ((uintptr_t)p & 15u) != 0; }
size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

hdt_status_t check_sizes(const char *fn, int64_t rows, int32_t width, int32_t inner, hdt_act_t act, hdt_dtype_t dt)
{
    if (rows < 0 || width < 0 || inner < 0) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: negative size", fn);
    if (dt != HDT_BF16 && dt != HDT_F32) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, (int)dt);
    if (act != HDT_SILU && act != HDT_GELU && act != HDT_GELU_TANH) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown activation %d", fn, (int)act);
    if (width < 1 || width > kMostSize || inner < 1 || inner > kMostSize)
        return hdt_fail(HDT_ERR_SHAPE, "%s: width %d or inner %d outside [1, %d]", fn, width, inner, kMostSize);
    if (rows > (1 << 28) || rows * std::max(width, inner) > kMostElements) return hdt_fail(HDT_ERR_SHAPE, "%s: more than 2^28 rows or 2^35 elements", fn);
    return HDT_OK;
}

struct Sizes {
    int64_t rows;
    int width, inner;
    hdt_dtype_t dt;
    size_t hidden_bytes() const { return padded((size_t)rows * inner * (dt == HDT_BF16 ? 2 : 4)); }
};

template <int KIND, bool A_SLOW, bool B_SLOW>
hdt_status_t product(const char *name, const Product &p, hdt_dtype_t dt, hipStream_t st)
{
    HdtTimer t(name, st);
    dt == HDT_BF16 ? launch_plain<__bf16, KIND, A_SLOW, B_SLOW>(p, st) : launch_plain<float, KIND, A_SLOW, B_SLOW>(p, st);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

#define HDT_EXPORT extern "C" __attribute__((visibility("default")))

}  // namespace

HDT_EXPORT size_t hdt_ffn_fwd_workspace_bytes(int64_t rows, int32_t width, int32_t inner, int32_t train, hdt_dtype_t dt)
{
    if (check_sizes("hdt_ffn_fwd_workspace_bytes", rows, width, inner, HDT_SILU, dt) != HDT_OK || rows == 0) return 0;
    const Sizes s = {rows, width, inner, dt};
    return train ? 0 : s.hidden_bytes();
}

HDT_EXPORT hdt_status_t hdt_ffn_fwd(const void *x, const void *w_gate, const void *w_up, const void *w_down, int64_t rows, int32_t width, int32_t inner,
                                    hdt_act_t act, void *y, void *by_gate, void *by_up, void *hidden, hdt_dtype_t dt, void *workspace, size_t workspace_bytes,
                                    void *stream)
{
    const char *fn = "hdt_ffn_fwd";
    if (hdt_status_t st = check_sizes(fn, rows, width, inner, act, dt)) return st;
    const bool train = hidden != nullptr;
    if (rows == 0) return HDT_OK;
    if (!x || !w_gate || !w_up || !w_down || !y) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if ((by_gate != nullptr) != train || (by_up != nullptr) != train) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: by_gate, by_up and hidden are given together or not at all", fn);
    const void *in[] = {x, w_gate, w_up, w_down}, *out[] = {y, by_gate, by_up, hidden};
    for (const void *p : in)
        if (misaligned(p)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    for (int i = 0; i < 4; i++) {
        if (!out[i]) continue;
        if (misaligned(out[i])) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
        for (const void *p : in)
            if (out[i] == p) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: output aliases an input", fn);
        for (int j = 0; j < i; j++)
            if (out[i] == out[j]) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: outputs alias each other", fn);
    }
    const size_t need = hdt_ffn_fwd_workspace_bytes(rows, width, inner, train, dt);
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace)))
        return hdt_fail(HDT_ERR_INVALID_ARG, "%s: a 16-byte aligned workspace of %zu bytes needed, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
    hipStream_t st = (hipStream_t)stream;
    void *h = train ? hidden : workspace;
    Product p = {};
    p.a[0] = x, p.b[0] = w_gate, p.b[1] = w_up, p.lda = width, p.ldb = width, p.m = (int)rows, p.n = inner, p.k = width, p.ranges = 1;
    p.out[0] = by_gate, p.out[1] = by_up, p.out[2] = h, p.ldo = inner, p.act = act;
    if (hdt_status_t s = product<GATE, false, false>("hdt_ffn_gate", p, dt, st)) return s;
    p = {};
    p.a[0] = h, p.b[0] = w_down, p.lda = inner, p.ldb = inner, p.m = (int)rows, p.n = width, p.k = inner, p.ranges = 1, p.out[0] = y, p.ldo = width;
    return product<STORE, false, false>("hdt_ffn_down", p, dt, st);
}

HDT_EXPORT size_t hdt_ffn_bwd_workspace_bytes(int64_t rows, int32_t width, int32_t inner, hdt_dtype_t dt)
{
    if (check_sizes("hdt_ffn_bwd_workspace_bytes", rows, width, inner, HDT_SILU, dt) != HDT_OK || rows == 0) return 0;
    const Sizes s = {rows, width, inner, dt};
    return 2 * s.hidden_bytes();
}

HDT_EXPORT hdt_status_t hdt_ffn_bwd(const void *dy, const void *x, const void *w_gate, const void *w_up, const void *w_down, const void *by_gate,
                                    const void *by_up, const void *hidden, int64_t rows, int32_t width, int32_t inner, void *dx,
                                    void *dw_gate, void *dw_up, void *dw_down, hdt_dtype_t dt, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "hdt_ffn_bwd";
    if (hdt_status_t st = check_sizes(fn, rows, width, inner, HDT_SILU, dt)) return st;
    if (!w_gate || !w_up || !w_down || !dw_gate || !dw_up || !dw_down) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (rows > 0 && (!dy || !x || !by_gate || !by_up || !hidden || !dx)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    const void *in[] = {dy, x, w_gate, w_up, w_down, by_gate, by_up, hidden}, *out[] = {dw_gate, dw_up, dw_down, rows > 0 ? dx : nullptr};
    for (const void *p : in)
        if (misaligned(p)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    for (int i = 0; i < 4; i++) {
        if (!out[i]) continue;
        if (misaligned(out[i])) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
        for (const void *p : in)
            if (out[i] == p) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: output aliases an input", fn);
        for (int j = 0; j < i; j++)
            if (out[i] == out[j]) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: outputs alias each other", fn);
    }
    const size_t need = hdt_ffn_bwd_workspace_bytes(rows, width, inner, dt);
    if (rows > 0 && (!workspace || workspace_bytes < need || misaligned(workspace)))
        return hdt_fail(HDT_ERR_INVALID_ARG, "%s: a 16-byte aligned workspace of %zu bytes needed, %zu given", fn, need, workspace ? workspace_bytes : (size_t)0);
    const Sizes s = {rows, width, inner, dt};
    hipStream_t st = (hipStream_t)stream;
    void *dg = workspace, *du = (char *)workspace + s.hidden_bytes();
    Product p = {};
    if (rows > 0) {
        p.a[0] = dy, p.b[0] = w_down, p.lda = width, p.ldb = inner, p.m = (int)rows, p.n = inner, p.k = width, p.ranges = 1;
        p.out[0] = dg, p.out[1] = du, p.by_gate = by_gate, p.by_up = by_up, p.ldo = inner;
        if (hdt_status_t r = product<DGATE, false, true>("hdt_ffn_dgate", p, dt, st)) return r;
        p = {};
        p.a[0] = dg, p.a[1] = du, p.b[0] = w_gate, p.b[1] = w_up, p.lda = inner, p.ldb = width, p.m = (int)rows, p.n = width, p.k = inner, p.ranges = 2;
        p.out[0] = dx, p.ldo = width;
        if (hdt_status_t r = product<STORE, false, true>("hdt_ffn_dx", p, dt, st)) return r;
    }
    // (no rows: gradients of zero)
    const struct {
        const void *a, *b;
        void *c;
        int m, n;
    } of[] = {{dg, x, dw_gate, inner, width}, {du, x, dw_up, inner, width}, {dy, hidden, dw_down, width, inner}};
    for (const auto &w : of) {
        p = {};
        p.a[0] = w.a, p.b[0] = w.b, p.lda = w.m, p.ldb = w.n, p.m = w.m, p.n = w.n, p.k = (int)rows, p.ranges = 1, p.out[0] = w.c, p.ldo = w.n;
        if (hdt_status_t r = product<WEIGHT, true, true>("hdt_ffn_dweight", p, dt, st)) return r;
    }
    return HDT_OK;
}
