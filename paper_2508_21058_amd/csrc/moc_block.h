// Arguments and launchers of the operators around the layer: head norms with rotation (moc_rope.hip) and cross attention
// (moc_cross_fwd.hip, moc_cross_bwd.hip, moc_cross_dkdv.hip).
#pragma once
#include "moc_internal.h"

namespace moc {

// ---- head norms with rotation -------------------------------------------------------------------
// One of q, k and v on its way through a pass. Strides count elements.
struct HeadPart {
    const void *x = nullptr;                   // the projection (backward: only where it is normalised)
    const void *g = nullptr;                   // backward: gradient of the output, contiguous [B, heads, N, d]
    void *out = nullptr;                       // forward: the output; backward: gradient of the projection
    long long x_b = 0, x_h = 0, x_n = 0;
    long long o_b = 0, o_h = 0, o_n = 0;
    const float *weight = nullptr;
    int heads = 0;                             // 0: the part is left out
};
struct RowArgs {
    HeadPart part[3];                          // q, k: normalised and turned, or turned only; v: copied
    const int32_t *positions;                  // nullptr: nothing is turned
    const double *freq;
    float *partial;                            // backward: [workgroups][2][d] sums for the weights' gradients
    int n_axes, axis_end[MOC_MAX_AXES];        // pairs [axis_end[a - 1], axis_end[a]) turn with axis a
    int N, n_tokens;                           // n_tokens = B * N
    int heads_total, heads_per_group, blocks;
    float eps, sign;                           // sign -1: the inverse rotation
};
// How a pass is cut: workgroups take `tokens` tokens of heads_per_group of all heads at a time.
struct RowGrid { int tokens, blocks, groups, per_group, grid_x; };
RowGrid row_grid(int B, int N, int heads_total, int d, bool bwd);
size_t rows_partial_bytes(int d);
hipError_t launch_rows(RowArgs a, int B, int d, int dtype, bool norm, bool halves, hipStream_t st);
hipError_t launch_rows_bwd(RowArgs a, int B, int d, int dtype, bool halves, float *dq_weight, float *dk_weight, hipStream_t st);

// ---- cross attention ----------------------------------------------------------------------------
struct CrossRange { int32_t first, end; };
// A tile of states of the wide key-stationary pass and the segments that attend all of it (none: its gradients are zero). The
// tiles of a sample cover its states once.
struct CrossKeys {
    int32_t start, len, pad[2];
    uint32_t segments[MOC_MAX_CROSS_SEGMENTS / 32];
};
struct CrossCount { int32_t live, idle; };             // of a sample: tiles of segments (the first ones) and without any
struct CrossArgs {
    const void *q, *k, *v, *o_in, *d_o;
    void *o, *dq, *dk, *dv;
    float *lse;                        // forward: out
    const float *lse_in;               // backward
    float *stats;                      // [B * H * N + 1] records (lse * log2 e, delta, query of the key head << 5, 0); last one (+inf, 0, 0, 0)
    float *part, *part_lse;            // split calls: [split][B * H * N][d], [split][B * H * N]
    float *kpart;                      // split dK / dV: [split][B * Hk * M][2][d]
    CrossKeys *items;                  // wide tiles: [B][max_items]
    CrossCount *item_counts;           // [B]
    int max_items;
    const CrossRange *ranges;          // [B][n_seg] or nullptr
    long long rows;                    // B * H * N
    int N, M, n_seg;                   // tokens of a query head (all heads of a group where copies is 1 and H > Hk), states
    int copies;                        // query heads of a key head that are walked one by one
    int Hk, BHk, tiles;                // tiles: query tiles of one copy
    int split;                         // parts of a range of states (forward, dQ) or of the queries (dK / dV)
    bool joined;                       // neighbouring segments with one range are one run of queries (a segment is short)
    bool dealt;                        // items are dealt to the XCDs one by one
    int cut_at;                        // dQ: workgroups from here on cut the states, a sample each
    float scale, scale_log2;
    int32_t q_off[MOC_MAX_CROSS_SEGMENTS + 1];
    int32_t tile_at[MOC_MAX_CROSS_SEGMENTS + 1];      // first query tile of a segment
};
void cross_tiles(CrossArgs &a);        // cuts the segments into query tiles
// Terms of a sum over states or queries that are added one after the other: 2^16 matrix additions of 16 products each in bf16, 2^14 of two in float.
// n additions in a row are off by at most n 2^-24 of the terms' magnitudes, and by a quarter of that where all terms are alike (2^-10, 2^-12).
constexpr int kChainTerms = 1 << 20, kChainTermsF32 = 1 << 15;
// Sizes of a call that follow from its arguments alone, and the places in its workspace (byte offsets).
struct CrossPlan {
    int split_q, split_kv;
    bool wide;                         // dK and dV in tiles of 256 states (moc_cross_dkdv.hip)
    int key_waves, max_items;          // else waves of 32 states of a workgroup
    bool fits;                         // no launch is larger than launches can be
    size_t stats, part, part_lse, kpart, items, item_counts, total;
};
CrossPlan cross_plan(int B, int H, int Hk, int N, int M, int d, int S, int dtype, bool with_bwd);
hipError_t launch_cross_fwd(CrossArgs a, int d, int dtype, hipStream_t st);
void launch_cross_dkdv_wide(const CrossArgs &a, hipStream_t st);
hipError_t launch_cross_bwd(CrossArgs a, const CrossPlan &p, int d, int dtype, hipStream_t st);

}  // namespace moc
