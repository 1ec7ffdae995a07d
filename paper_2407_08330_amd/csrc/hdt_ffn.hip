// Gated feed-forward block: checks, what kernel takes which product, the calls.  hdt_ffn.h has the mathematics.
#include <algorithm>

#include "hdt_ffn.h"
#include "hdt_ffn_plain.h"
#include "hdt_ffn_tile.h"

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

using Large = Shape<2, 4, 4, 2>;  // 256 x 256, a workgroup a compute unit
using Small = Shape<2, 2, 2, 2>;  // 128 x 128, two of them

// Products that one launch makes in tiles, and how: the shape, and the pieces of k that are joined afterwards.
struct Plan {
    bool large;
    int splits, per;   // tiles of k a piece
    unsigned tiles;    // of all products
    size_t parts_bytes;
};
struct Dims {
    int m, n;  // n: columns of the tile's operand (of both weights, for GATE)
};
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

template <typename S>
void consider(const Dims *of, int products, int k_tiles, bool divisible, bool large, Plan *best, double *best_cost)
{
    int64_t tiles = 0;
    for (int i = 0; i < products; i++) tiles += (int64_t)ceil_div(of[i].m, S::BM) * ceil_div(of[i].n, S::BN);
    // clocks of a tile of k with every unit full, and of what stands around a tile's walk
    const int slots = large ? 256 : 512;
    const double step = large ? 2600 : 1500, around = large ? 9000 : 6000;
    for (int splits = 1; splits <= (divisible ? 32 : 1); splits++) {
        const int per = ceil_div(k_tiles, splits);
        if (splits > 1 && (ceil_div(k_tiles, per) != splits || per < 4)) continue;
        const double rounds = (double)((tiles * splits + slots - 1) / slots);
        // pieces: their sums written and read at about 2000 bytes a clock, and a launch
        const double join = splits > 1 ? (double)tiles * splits * S::BM * S::BN * 8 / 2000 + 8000 : 0;
        const double cost = rounds * (per * step + around) + join;
        if (*best_cost >= 0 && cost >= *best_cost) continue;
        *best_cost = cost;
        *best = {large, splits, per, (unsigned)tiles, splits > 1 ? (size_t)tiles * splits * S::BM * S::BN * sizeof(float) : 0};
    }
}
Plan plan_of(const Dims *of, int products, int k, int ranges, bool divisible)
{
    Plan best = {};
    double cost = -1;
    const int k_tiles = ranges * ceil_div(k, BK);
    consider<Large>(of, products, k_tiles, divisible, true, &best, &cost);
    consider<Small>(of, products, k_tiles, divisible, false, &best, &cost);
    return best;
}

struct Sizes {
    int64_t rows;
    int width, inner;
    hdt_dtype_t dt;
    size_t hidden_bytes() const { return padded((size_t)rows * inner * (dt == HDT_BF16 ? 2 : 4)); }
    // whether rows begin at multiples of 16 bytes, as direct loads need it
    bool tiled() const { return dt == HDT_BF16 && width % 8 == 0 && inner % 8 == 0; }
    Plan plan_gate() const
    {
        const Dims d = {(int)rows, 2 * inner};
        return plan_of(&d, 1, width, 1, false);
    }
    Plan plan_down() const
    {
        const Dims d = {(int)rows, width};
        return plan_of(&d, 1, inner, 1, true);
    }
    Plan plan_dgate() const
    {
        const Dims d = {(int)rows, inner};
        return plan_of(&d, 1, width, 1, false);
    }
    Plan plan_dx() const
    {
        const Dims d = {(int)rows, width};
        return plan_of(&d, 1, inner, 2, true);
    }
    Plan plan_weights() const
    {
        const Dims d[] = {{inner, width}, {inner, width}, {width, inner}};
        return plan_of(d, 3, (int)rows, 1, true);
    }
    size_t fwd_bytes(bool train) const { return (train ? 0 : hidden_bytes()) + (tiled() ? plan_down().parts_bytes : 0); }
    size_t bwd_bytes() const { return 2 * hidden_bytes() + (tiled() ? std::max(plan_dx().parts_bytes, plan_weights().parts_bytes) : 0); }
};

template <int KIND, typename S, bool A_SLOW, bool B_SLOW>
hdt_status_t launch_tiles(const char *name, const Product *of, int products, const Plan &plan, void *parts, hipStream_t st)
{
    TileArgs a = {};
    a.products = products, a.k = of[0].k, a.ranges = of[0].ranges, a.splits = plan.splits, a.per = plan.per, a.tiles = plan.tiles, a.parts = (float *)parts;
    a.act = of[0].act, a.group = 8;
    unsigned first = 0;
    for (int i = 0; i < products; i++) {
        const Product &p = of[i];
        const int tiles_m = ceil_div(p.m, S::BM), tiles_n = ceil_div(KIND == GATE ? 2 * (int64_t)p.n : p.n, S::BN);
        a.p[i] = {{(const __bf16 *)p.a[0], (const __bf16 *)p.a[1]}, {(const __bf16 *)p.b[0], (const __bf16 *)p.b[1]},
                  {(__bf16 *)p.out[0], (__bf16 *)p.out[1], (__bf16 *)p.out[2]}, (const __bf16 *)p.by_gate, (const __bf16 *)p.by_up,
                  p.lda, p.ldb, p.ldo, p.m, p.n, tiles_m, tiles_n, first};
        first += (unsigned)tiles_m * tiles_n;
    }
    const unsigned items = plan.tiles * plan.splits, chunk = hdt_tile::xcd_chunk(items, 64, 1);
    a.chunk = hdt_tile::FastDiv(chunk);
    a.by_split = hdt_tile::FastDiv(plan.splits);
    const auto kernel = k_ffn_tile<KIND, S, A_SLOW, B_SLOW>;
    if (S::LDS > 65536) HDT_HIP_TRY(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS));
    {
        HdtTimer t(name, st);
        hipLaunchKernelGGL(kernel, dim3(hdt_tile::padded_grid(items, chunk)), dim3(S::THREADS), S::LDS, st, a);
        HDT_HIP_TRY(hipGetLastError());
    }
    if (plan.splits == 1) return HDT_OK;
    HdtTimer t("hdt_ffn_join", st);
    hipLaunchKernelGGL(k_ffn_join<S>, dim3(plan.tiles * S::MB), dim3(S::THREADS), 0, st, a);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

template <int KIND, bool A_SLOW, bool B_SLOW>
hdt_status_t make(const char *name, const Product *of, int products, const Sizes &s, Plan (Sizes::*plan_fn)() const, void *parts, hipStream_t st)
{
    if (s.tiled() && of[0].m > 0 && of[0].k > 0) {
        const Plan plan = (s.*plan_fn)();
        return plan.large ? launch_tiles<KIND, Large, A_SLOW, B_SLOW>(name, of, products, plan, parts, st)
                          : launch_tiles<KIND, Small, A_SLOW, B_SLOW>(name, of, products, plan, parts, st);
    }
    for (int i = 0; i < products; i++) {
        HdtTimer t(name, st);
        s.dt == HDT_BF16 ? launch_plain<__bf16, KIND, A_SLOW, B_SLOW>(of[i], st) : launch_plain<float, KIND, A_SLOW, B_SLOW>(of[i], st);
        HDT_HIP_TRY(hipGetLastError());
    }
    return HDT_OK;
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
    if (hdt_status_t r = make<GATE, false, false>("hdt_ffn_gate", &p, 1, s, &Sizes::plan_gate, nullptr, st)) return r;
    p = {};
    p.a[0] = h, p.b[0] = w_down, p.lda = inner, p.ldb = inner, p.m = (int)rows, p.n = width, p.k = inner, p.ranges = 1, p.out[0] = y, p.ldo = width;
    return make<STORE, false, false>("hdt_ffn_down", &p, 1, s, &Sizes::plan_down, parts, st);
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
