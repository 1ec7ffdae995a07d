// Arguments of the relative-bias attention's kernels, and what the host lays out for them.
#pragma once

#include "hdt_rel.h"

struct RelFwdArgs {
    const void *q, *k, *v;
    void *o;
    float *lse;                       // [batch][heads][n_q]
    float *part_o, *part_lse;         // [rows][pieces][head_dim], [rows][pieces]
    const int32_t *lengths, *starts;  // [batch] or NULL
    hdt_strides_t sq, sk, sv, so;
    hdt_rel::BiasArgs bias;
    int32_t batch, heads, group;      // group: heads per key head
    int32_t n_q, n_kv;
    int32_t gp, head_blocks, tiles;   // rows of a tile: queries of gp heads; head_blocks = heads / gp
    uint32_t pieces;                  // of every row tile's keys
    float scale_log2;
};

struct RelFwdPlan {
    int32_t gp, head_blocks, tiles;
    int32_t waves;         // of a workgroup, 32 rows each; 0: few rows, the waves divide the keys
    uint32_t pieces;
    size_t lse_at, bytes;  // of the workspace
};
RelFwdPlan hdt_rel_fwd_plan(const hdt_rel_attn_t &d);
hdt_status_t hdt_launch_rel_fwd(const hdt_rel_attn_t &d, const RelFwdArgs &a, int waves, hipStream_t st);

struct RelBwdArgs {
    const void *q, *k, *v, *o, *d_o;
    const float *lse;
    void *dq, *dk, *dv, *d_bias;
    float *row_scalars;               // four arrays of [batch][heads][n_pad], see k_rel_rows
    float *bins;                      // [heads][batch * tiles_q][n_buckets]: sums of dS
    const int32_t *lengths, *starts;
    hdt_strides_t sq, sk, sv, so, sdo, sdq, sdk, sdv;
    hdt_rel::BiasArgs bias;
    int32_t batch, heads, kv_heads, group, n_q, n_kv;
    int32_t tiles_q, tiles_k, n_pad;  // n_pad: n_q up to whole tiles
    float scale, scale_log2;
};

struct RelBwdPlan {
    int32_t tiles_q, tiles_k, n_pad, waves;  // waves of a workgroup, 32 rows each
    size_t bins_at, bytes;
};
RelBwdPlan hdt_rel_bwd_plan(const hdt_rel_attn_t &d);
hdt_status_t hdt_launch_rel_bwd(const hdt_rel_attn_t &d, const RelBwdArgs &a, int waves, hipStream_t st);

namespace hdt_rel {

__device__ __forceinline__ void store4(__bf16 *p, float x, float y, float z, float w)
{
    bf16x4 v = {(__bf16)x, (__bf16)y, (__bf16)z, (__bf16)w};
    *reinterpret_cast<bf16x4 *>(p) = v;
}
__device__ __forceinline__ void store4(float *p, float x, float y, float z, float w)
{
    f32x4 v = {x, y, z, w};
    *reinterpret_cast<f32x4 *>(p) = v;
}

}  // namespace hdt_rel
