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

// Waves of 32 rows a workgroup's tile has: 4, or 2 or 1 whose workgroups divide the walk along the other side among groups of waves, which
// is quicker for a tile, where all of them fit the card at once.  A compute unit holds two workgroups of 2 waves of 64 columns and one of
// the others; in fp32, whose walk is bound by the matrix instructions, a second round of small tiles still pays.
// (us, 4 | 2 | 1 waves.  Backward bf16, heads x rows of 64: 128 x 512 47.6 | 58.8 | 136, 64 x 512 35.8 | 36.1 | 71, 32 x 512 27.5 | 26.5 | 39.9,
// 16 x 512 27.1 | 22.2 | 25.9, 8 x 512 26.7 | 22.4 | 19.3; of 128: 32 x 512 36.0 | 41.9, 16 x 512 34.5 | 29.2.  fp32 of 64: 64 x 512
// 112 | 116 | 152, 32 x 512 88 | 64 | 82, 16 x 512 87 | 54 | 47.  Forward bf16 of 64: 128 x 512 13.8 | 18.1 | 51, 64 x 512 12.2 | 10.9 | 26,
// 16 x 512 11.6 | 9.6 | 8.8.  Calls of more rows take the rule as it is: its figures are of 512.)
inline int hdt_rel_row_waves(long long tiles64, long long tiles32, const hdt_rel_attn_t &d)
{
    if (d.head_dim == 64 && tiles32 <= (d.dtype == HDT_BF16 ? 256 : 512)) return 1;
    return tiles64 <= (d.head_dim == 64 ? 512 : 256) ? 2 : 4;
}

struct RelBwdArgs {
    const void *q, *k, *v, *o, *d_o;
    const float *lse;
    void *dq, *dk, *dv, *d_bias;
    float *row_scalars;               // four arrays of [batch][heads][n_pad], see k_rel_rows
    float *tables;                    // [heads][row]: bias by distance over the scale, row = table_row()
    float *bins;                      // [heads][batch * tiles_q][row]: sums of dS by distance
    const int32_t *lengths, *starts;
    hdt_strides_t sq, sk, sv, so, sdo, sdq, sdk, sdv;
    hdt_rel::BiasArgs bias;
    int32_t batch, heads, kv_heads, group, n_q, n_kv;
    int32_t tiles_q, tiles_k, n_pad;  // n_pad: n_q up to whole tiles
    float scale, scale_log2;
};

struct RelBwdPlan {
    int32_t tiles_q, tiles_k, n_pad, waves;  // waves of a workgroup, 32 rows each
    size_t tables_at, bins_at, bytes;
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
