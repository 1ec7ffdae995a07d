// C-ABI entry points of self-attention with a relative position bias: argument checks, the buckets of the distances, dispatch.
#include "hdt_rel.h"
#include "hdt_rel_args.h"

namespace {

// T5's buckets (Raffel et al., JMLR 2020, Sec. 2.1: half of them for one distance each, the others for ranges that grow with the
// logarithm up to a largest distance, all beyond it in the last one); in double precision, because the borders of the ranges can be
// whole distances: within 1e-9 of one counts as having reached it.
__global__ void k_rel_table(int32_t *table, int n_buckets, int max_distance, int both)
{
    const int x = blockIdx.x * blockDim.x + threadIdx.x;
    if (x > 2 * max_distance) return;
    const int d = x - max_distance, half = both ? n_buckets / 2 : n_buckets, exact = half / 2;
    const int away = both ? abs(d) : max(-d, 0);
    int bucket = away;
    if (away >= exact) {
        const double steps = log((double)away / exact) / log((double)max_distance / exact) * (half - exact);
        bucket = min(exact + (int)floor(steps + 1e-9), half - 1);
    }
    table[x] = bucket + (both && d > 0 ? half : 0);
}

constexpr int kMostRows = 1 << 24, kMostBuckets = 4096;
constexpr int64_t kMostGrid = (1 << 20) - 1;  // tiles of 128 rows
constexpr int64_t kMostRowStride = 1 << 20;  // elements: a tile's rows stay within 32-bit byte offsets

struct View {
    const char *name;
    const hdt_strides_t *given;
    int32_t heads, rows;
    bool written;
};

// the strides of a tensor, the dense ones if none are given
hdt_status_t strides_of(const char *fn, const hdt_rel_attn_t &d, const View &v, hdt_strides_t *s)
{
    *s = *v.given;
    if (s->batch == 0 && s->head == 0 && s->row == 0) *s = {(int64_t)v.heads * v.rows * d.head_dim, (int64_t)v.rows * d.head_dim, d.head_dim};
    const int64_t unit = d.dtype == HDT_BF16 ? 8 : 4;
    if (s->batch < 0 || s->head < 0 || s->row < 0 || s->batch % unit || s->head % unit || s->row % unit)
        return hdt_fail(HDT_ERR_INVALID_ARG, "%s: the strides of %s must be non-negative multiples of 16 bytes", fn, v.name);
    if (v.rows > 1 && (s->row < d.head_dim || s->row > kMostRowStride))
        return hdt_fail(HDT_ERR_INVALID_ARG, "%s: the row stride of %s must be between head_dim and %lld elements", fn, v.name, (long long)kMostRowStride);
    if (!v.written || d.batch == 0 || v.heads == 0 || v.rows == 0) return HDT_OK;
    // an output's rows must not overlap: sizes and strides from the smallest stride on, each beyond what lies within it
    struct Dim {
        int64_t stride, size;
    } dims[3] = {{s->row, v.rows}, {s->head, v.heads}, {s->batch, d.batch}};
    for (int i = 0; i < 3; i++)
        for (int j = i + 1; j < 3; j++)
            if (dims[j].stride < dims[i].stride) {
                const Dim t = dims[i];
                dims[i] = dims[j];
                dims[j] = t;
            }
    int64_t extent = d.head_dim;
    for (const Dim &x : dims) {
        if (x.size <= 1) continue;
        if (x.stride < extent) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: the rows of the output %s overlap", fn, v.name);
        extent = x.stride * (x.size - 1) + extent;
    }
    return HDT_OK;
}

hdt_status_t check(const char *fn, const hdt_rel_attn_t *d)
{
    if (!d) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL description", fn);
    if (d->batch < 0 || d->heads < 0 || d->n_q < 0 || d->n_kv < 0) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: negative size", fn);
    if (d->kv_heads <= 0 || d->heads % d->kv_heads)
        return hdt_fail(HDT_ERR_SHAPE, "%s: %d heads on %d key heads (a divisor of the heads is needed)", fn, d->heads, d->kv_heads);
    if (d->dtype != HDT_BF16 && d->dtype != HDT_F32) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, (int)d->dtype);
    if (d->bias_dtype != HDT_BF16 && d->bias_dtype != HDT_F32)
        return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d of the bias", fn, (int)d->bias_dtype);
    if (d->head_dim != 64 && d->head_dim != 128) return hdt_fail(HDT_ERR_UNSUPPORTED, "%s: head_dim %d (supported: 64, 128)", fn, d->head_dim);
    if (!hdt_finite(d->softmax_scale) || d->softmax_scale <= 1e-20f || d->softmax_scale >= 1e20f)
        return hdt_fail(HDT_ERR_INVALID_ARG, "%s: softmax_scale must be between 1e-20 and 1e20", fn);
    if (d->n_q > kMostRows || d->n_kv > kMostRows) return hdt_fail(HDT_ERR_SHAPE, "%s: more than %d rows", fn, kMostRows);
    if (d->max_distance < 1 || d->max_distance > hdt_rel::kMostDistance)
        return hdt_fail(HDT_ERR_SHAPE, "%s: max_distance %d outside [1, %d]", fn, d->max_distance, hdt_rel::kMostDistance);
    if (d->n_buckets < 1 || d->n_buckets > kMostBuckets)
        return hdt_fail(HDT_ERR_SHAPE, "%s: n_buckets %d outside [1, %d]", fn, d->n_buckets, kMostBuckets);
    // a launch has fewer than 2^32 threads
    const int64_t tiles_q = ((int64_t)d->n_q + 127) / 128, tiles_k = ((int64_t)d->n_kv + 127) / 128, both = (int64_t)d->batch * ((int64_t)d->heads + d->kv_heads);
    if (both > kMostGrid || both * (tiles_q > tiles_k ? tiles_q : tiles_k) > kMostGrid)
        return hdt_fail(HDT_ERR_SHAPE, "%s: batch * heads * rows exceeds the grid limit", fn);
    return HDT_OK;
}

hdt_rel::BiasArgs bias_args(const hdt_rel_attn_t &d)
{
    return {d.d_bias, d.d_table, d.n_buckets, d.heads, d.max_distance, d.bias_dtype == HDT_BF16, 1.f / d.softmax_scale};
}

bool misaligned(const void *p) { return ((uintptr_t)p & 15u) != 0; }

#define HDT_EXPORT extern "C" __attribute__((visibility("default")))

}  // namespace

HDT_EXPORT hdt_status_t hdt_rel_table(int32_t n_buckets, int32_t max_distance, int32_t both_ways, int32_t *d_table, void *stream)
{
    const int half = both_ways ? n_buckets / 2 : n_buckets;
    if (n_buckets < 0 || max_distance < 0) return hdt_fail(HDT_ERR_INVALID_ARG, "hdt_rel_table: negative size");
    if (n_buckets > kMostBuckets || half < 2 || (both_ways && n_buckets % 2))
        return hdt_fail(HDT_ERR_SHAPE, "hdt_rel_table: %d buckets (2 to %d; both ways an even number from 4 on)", n_buckets, kMostBuckets);
    if (max_distance > hdt_rel::kMostDistance || max_distance <= half / 2)
        return hdt_fail(HDT_ERR_SHAPE, "hdt_rel_table: max_distance %d outside (%d, %d]", max_distance, half / 2, hdt_rel::kMostDistance);
    if (!d_table) return hdt_fail(HDT_ERR_INVALID_ARG, "hdt_rel_table: NULL pointer");
    hipStream_t st = (hipStream_t)stream;
    HdtTimer t("hdt_rel_table", st);
    hipLaunchKernelGGL(k_rel_table, dim3((2 * max_distance + 256) / 256), dim3(256), 0, st, d_table, n_buckets, max_distance, both_ways != 0);
    HDT_HIP_TRY(hipGetLastError());
    return HDT_OK;
}

HDT_EXPORT size_t hdt_rel_attn_fwd_workspace_bytes(const hdt_rel_attn_t *d)
{
    if (check("hdt_rel_attn_fwd_workspace_bytes", d) != HDT_OK || d->batch == 0 || d->heads == 0 || d->n_q == 0) return 0;
    return hdt_rel_fwd_plan(*d).bytes;
}

HDT_EXPORT hdt_status_t hdt_rel_attn_fwd(const hdt_rel_attn_t *d, const void *q, const void *k, const void *v, void *o, float *lse,
                                         void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "hdt_rel_attn_fwd";
    if (hdt_status_t st = check(fn, d)) return st;
    RelFwdArgs a = {};
    const View views[] = {{"q", &d->q, d->heads, d->n_q, false}, {"k", &d->k, d->kv_heads, d->n_kv, false},
                          {"v", &d->v, d->kv_heads, d->n_kv, false}, {"o", &d->o, d->heads, d->n_q, true}};
    hdt_strides_t *to[] = {&a.sq, &a.sk, &a.sv, &a.so};
    for (int i = 0; i < 4; i++)
        if (hdt_status_t st = strides_of(fn, *d, views[i], to[i])) return st;
    if (d->batch == 0 || d->heads == 0 || d->n_q == 0) return HDT_OK;
    if (!q || !o || !lse || !d->d_bias || !d->d_table || (d->n_kv > 0 && (!k || !v))) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    for (const void *p : {q, k, v, (const void *)o, (const void *)workspace})
        if (misaligned(p)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    if ((uintptr_t)lse & 3u) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: lse must be 4-byte aligned", fn);
    if (o == q || o == k || o == v) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: output aliases an input", fn);
    RelFwdPlan p = hdt_rel_fwd_plan(*d);
    if (p.bytes > 0 && (!workspace || workspace_bytes < p.bytes)) p.pieces = 1;
    a.q = q, a.k = k, a.v = v, a.o = o, a.lse = lse;
    a.part_o = (float *)workspace;
    a.part_lse = (float *)((char *)workspace + p.lse_at);
    a.lengths = d->d_lengths, a.starts = d->d_q_start;
    a.bias = bias_args(*d);
    a.batch = d->batch, a.heads = d->heads, a.group = d->heads / d->kv_heads, a.n_q = d->n_q, a.n_kv = d->n_kv;
    a.gp = p.gp, a.head_blocks = p.head_blocks, a.tiles = p.tiles, a.pieces = p.pieces;
    a.scale_log2 = d->softmax_scale * hdt_rel::LOG2E;
    return hdt_launch_rel_fwd(*d, a, p.waves, (hipStream_t)stream);
}

HDT_EXPORT size_t hdt_rel_attn_bwd_workspace_bytes(const hdt_rel_attn_t *d)
{
    if (check("hdt_rel_attn_bwd_workspace_bytes", d) != HDT_OK) return 0;
    return hdt_rel_bwd_plan(*d).bytes;
}

HDT_EXPORT hdt_status_t hdt_rel_attn_bwd(const hdt_rel_attn_t *d, const void *q, const void *k, const void *v, const void *o,
                                         const float *lse, const void *d_o, void *dq, void *dk, void *dv, void *d_bias_grad,
                                         void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "hdt_rel_attn_bwd";
    if (hdt_status_t st = check(fn, d)) return st;
    RelBwdArgs a = {};
    const View views[] = {{"q", &d->q, d->heads, d->n_q, false},      {"k", &d->k, d->kv_heads, d->n_kv, false},
                          {"v", &d->v, d->kv_heads, d->n_kv, false},  {"o", &d->o, d->heads, d->n_q, false},
                          {"d_o", &d->d_o, d->heads, d->n_q, false},  {"dq", &d->dq, d->heads, d->n_q, true},
                          {"dk", &d->dk, d->kv_heads, d->n_kv, true}, {"dv", &d->dv, d->kv_heads, d->n_kv, true}};
    hdt_strides_t *to[] = {&a.sq, &a.sk, &a.sv, &a.so, &a.sdo, &a.sdq, &a.sdk, &a.sdv};
    for (int i = 0; i < 8; i++)
        if (hdt_status_t st = strides_of(fn, *d, views[i], to[i])) return st;
    const bool rows = d->batch > 0 && d->heads > 0 && d->n_q > 0, keys = d->batch > 0 && d->n_kv > 0;
    if ((d->heads > 0 && (!d->d_bias || !d->d_table || !d_bias_grad)) || (rows && (!q || !o || !lse || !d_o || !dq)) || (keys && (!k || !v || !dk || !dv)))
        return hdt_fail(HDT_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    const void *in[] = {q, k, v, o, d_o}, *out[] = {dq, dk, dv};
    for (const void *p : in)
        if (misaligned(p)) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    if ((uintptr_t)lse & 3u) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: lse must be 4-byte aligned", fn);
    for (int i = 0; i < 3; i++) {
        if (misaligned(out[i])) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
        for (const void *p : in)
            if (out[i] && out[i] == p) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: output aliases an input", fn);
        for (int j = 0; j < i; j++)
            if (out[i] && out[i] == out[j]) return hdt_fail(HDT_ERR_INVALID_ARG, "%s: outputs alias each other", fn);
    }
    const RelBwdPlan p = hdt_rel_bwd_plan(*d);
    if (p.bytes > 0 && (!workspace || workspace_bytes < p.bytes || misaligned(workspace)))
        return hdt_fail(HDT_ERR_INVALID_ARG, "%s: a 16-byte aligned workspace of %zu bytes needed, %zu given", fn, p.bytes, workspace ? workspace_bytes : (size_t)0);
    a.q = q, a.k = k, a.v = v, a.o = o, a.d_o = d_o, a.lse = lse, a.dq = dq, a.dk = dk, a.dv = dv, a.d_bias = d_bias_grad;
    a.row_scalars = (float *)workspace;
    a.tables = (float *)((char *)workspace + p.tables_at);
    a.bins = (float *)((char *)workspace + p.bins_at);
    a.lengths = d->d_lengths, a.starts = d->d_q_start;
    a.bias = bias_args(*d);
    a.batch = d->batch, a.heads = d->heads, a.kv_heads = d->kv_heads, a.group = d->heads / d->kv_heads, a.n_q = d->n_q, a.n_kv = d->n_kv;
    a.tiles_q = p.tiles_q, a.tiles_k = p.tiles_k, a.n_pad = p.n_pad;
    a.scale = d->softmax_scale, a.scale_log2 = d->softmax_scale * hdt_rel::LOG2E;
    return hdt_launch_rel_bwd(*d, a, p.waves, (hipStream_t)stream);
}
