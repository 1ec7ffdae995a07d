// Gated feed-forward block: checks, launches, the calls.  hdt_ffn.h has the mathematics, hdt_ffn_plan.h what kernel takes which product.
#include <algorithm>

#include "hdt_ffn.h"
#include "hdt_ffn_few.h"
#include "hdt_ffn_plain.h"
#include "hdt_ffn_plan.h"
#include "hdt_ffn_tile.h"

namespace {

using namespace hdt_ffn;

constexpr int kMostSize = 65536;
constexpr int64_t kMostElements = 1ll << 35;

bool misaligned(const void *p) { return ((uintptr_t)p & 15u) != 0; }

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

template <int KIND, typename S, bool A_SLOW, bool B_SLOW, bool EVEN>
hdt_status_t launch_tiles(const char *name, const Product *of, int products, const Plan &plan, void *parts, hipStream_t st)
{
    TileArgs a = {};
    a.products = products, a.k = of[0].k, a.ranges = of[0].ranges, a.parts = (float *)parts;
    const unsigned chunk = hdt_tile::xcd_chunk(plan.direct, 64, 1);
    a.chunk = hdt_tile::FastDiv(chunk);
    a.direct = plan.direct, a.spread = hdt_tile::padded_grid(plan.direct, chunk), a.tiles = plan.tiles;
    a.piece_items = plan.piece_items, a.sharers = plan.sharers, a.pieces = plan.pieces, a.per = plan.per, a.rest = plan.rest;
    a.act = of[0].act, a.group = 4;  // (2, 4 or 8: the same but for dG and dU, 200, 196 and 215-250 us)
    unsigned first = 0;
    for (int i = 0; i < products; i++) {
        const Product &p = of[i];
        const int tiles_m = ceil_div(p.m, S::BM), tiles_n = ceil_div(KIND == GATE ? 2 * (int64_t)p.n : p.n, S::BN);
        a.p[i] = {{(const __bf16 *)p.a[0], (const __bf16 *)p.a[1]}, {(const __bf16 *)p.b[0], (const __bf16 *)p.b[1]},
                  {(__bf16 *)p.out[0], (__bf16 *)p.out[1], (__bf16 *)p.out[2]}, (const __bf16 *)p.by_gate, (const __bf16 *)p.by_up,
                  p.lda, p.ldb, p.ldo, p.m, p.n, tiles_m, tiles_n, first};
        first += (unsigned)tiles_m * tiles_n;
    }
    const auto kernel = k_ffn_tile<KIND, S, A_SLOW, B_SLOW, EVEN>;
    if (S::LDS > 65536) HDT_HIP_TRY(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS));
    {
        HdtTimer t(name, st);
        hipLaunchKernelGGL(kernel, dim3(a.spread + plan.piece_items + plan.sharers), dim3(S::THREADS), S::LDS, st, a);
        HDT_HIP_TRY(hipGetLastError());
    }
    if (plan.direct == plan.tiles) return HDT_OK;
    HdtTimer t("hdt_ffn_join", st);
    hipLaunchKernelGGL((k_ffn_join<S, EVEN>), dim3((plan.tiles - plan.direct) * S::MB * S::NB), dim3(S::THREADS), 0, st, a);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

template <int KIND>
hdt_status_t make_few(const char *name, const Product &p, bool even, hipStream_t st)
{
    HdtTimer t(name, st);
    even ? launch_few<KIND, true>(p, st) : launch_few<KIND, false>(p, st);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

template <int KIND, bool A_SLOW, bool B_SLOW>
hdt_status_t make(const char *name, const Product *of, int products, const Sizes &s, Plan (Sizes::*plan_fn)() const, void *parts, hipStream_t st)
{
    if (!s.tiled()) {
        HdtTimer t(name, st);
        return launch_plain<KIND, A_SLOW, B_SLOW>(of, products, st);
    }
    const Plan plan = (s.*plan_fn)();
    if (s.even())
        return plan.shape == 0 ? launch_tiles<KIND, Large, A_SLOW, B_SLOW, true>(name, of, products, plan, parts, st)
                               : launch_tiles<KIND, Small, A_SLOW, B_SLOW, true>(name, of, products, plan, parts, st);
    return plan.shape == 0 ? launch_tiles<KIND, Large, A_SLOW, B_SLOW, false>(name, of, products, plan, parts, st)
                           : launch_tiles<KIND, Small, A_SLOW, B_SLOW, false>(name, of, products, plan, parts, st);
}

#define HDT_EXPORT extern "C" __attribute__((visibility("default")))

}  // namespace

HDT_EXPORT size_t hdt_ffn_fwd_workspace_bytes(int64_t rows, int32_t width, int32_t inner, int32_t train, hdt_dtype_t dt)
{
    if (check_sizes("hdt_ffn_fwd_workspace_bytes", rows, width, inner, HDT_SILU, dt) != HDT_OK || rows == 0) return 0;
    const Sizes s = {rows, width, inner, dt};
    return s.fwd_bytes(train != 0);
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
    const Sizes s = {rows, width, inner, dt};
    hipStream_t st = (hipStream_t)stream;
    void *h = train ? hidden : workspace, *parts = train ? workspace : (char *)workspace + s.hidden_bytes();
    Product p = {};
    p.a[0] = x, p.b[0] = w_gate, p.b[1] = w_up, p.lda = width, p.ldb = width, p.m = (int)rows, p.n = inner, p.k = width, p.ranges = 1;
    p.out[0] = by_gate, p.out[1] = by_up, p.out[2] = h, p.ldo = inner, p.act = act;
    if (hdt_status_t r = s.few() ? make_few<GATE>("hdt_ffn_gate", p, s.even(), st) : make<GATE, false, false>("hdt_ffn_gate", &p, 1, s, &Sizes::plan_gate, nullptr, st)) return r;
    p = {};
    p.a[0] = h, p.b[0] = w_down, p.lda = inner, p.ldb = inner, p.m = (int)rows, p.n = width, p.k = inner, p.ranges = 1, p.out[0] = y, p.ldo = width;
    return s.few() ? make_few<STORE>("hdt_ffn_down", p, s.even(), st) : make<STORE, false, false>("hdt_ffn_down", &p, 1, s, &Sizes::plan_down, parts, st);
}

HDT_EXPORT size_t hdt_ffn_bwd_workspace_bytes(int64_t rows, int32_t width, int32_t inner, hdt_dtype_t dt)
{
    if (check_sizes("hdt_ffn_bwd_workspace_bytes", rows, width, inner, HDT_SILU, dt) != HDT_OK || rows == 0) return 0;
    const Sizes s = {rows, width, inner, dt};
    return s.bwd_bytes();
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
    void *dg = workspace, *du = (char *)workspace + s.hidden_bytes(), *parts = (char *)workspace + 2 * s.hidden_bytes();
    Product p = {};
    if (rows > 0) {
        p.a[0] = dy, p.b[0] = w_down, p.lda = width, p.ldb = inner, p.m = (int)rows, p.n = inner, p.k = width, p.ranges = 1;
        p.out[0] = dg, p.out[1] = du, p.by_gate = by_gate, p.by_up = by_up, p.ldo = inner;
        if (hdt_status_t r = make<DGATE, false, true>("hdt_ffn_dgate", &p, 1, s, &Sizes::plan_dgate, nullptr, st)) return r;
        p = {};
        p.a[0] = dg, p.a[1] = du, p.b[0] = w_gate, p.b[1] = w_up, p.lda = inner, p.ldb = width, p.m = (int)rows, p.n = width, p.k = inner, p.ranges = 2;
        p.out[0] = dx, p.ldo = width;
        if (hdt_status_t r = make<STORE, false, true>("hdt_ffn_dx", &p, 1, s, &Sizes::plan_dx, parts, st)) return r;
    }
    // (no rows: gradients of zero)
    const struct {
        const void *a, *b;
        void *c;
        int m, n;
    } of[] = {{dg, x, dw_gate, inner, width}, {du, x, dw_up, inner, width}, {dy, hidden, dw_down, width, inner}};
    Product w[3] = {};
    for (int i = 0; i < 3; i++) {
        w[i].a[0] = of[i].a, w[i].b[0] = of[i].b, w[i].lda = of[i].m, w[i].ldb = of[i].n, w[i].m = of[i].m, w[i].n = of[i].n, w[i].k = (int)rows, w[i].ranges = 1;
        w[i].out[0] = of[i].c, w[i].ldo = of[i].n;
    }
    return make<STORE, true, true>("hdt_ffn_dweight", w, 3, s, &Sizes::plan_weights, parts, st);
}
