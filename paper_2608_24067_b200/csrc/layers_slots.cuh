// Launchers of layers_slots.cu.
#pragma once

#include "layers_internal.cuh"

namespace lay {

// xp[row] = x[token of row's slot]; unless dy is NULL the same of dy, and zeros in both up to whole steps of 64 rows
int launch_gather(som_layers* l, const SlotPlan& p, int64_t slots, int E, int k, int64_t D, const void* x, int64_t ldx, void* xp,
                  const void* dy, int64_t lddy, void* dyp, cudaStream_t st);
// Sums that end an operator.  Parts whose output is NULL are left out.
struct EndArgs {
    SlotPlan p;  // without p.seg: one group of `rows` rows
    int64_t T, rows;
    int k, D, E, bf16;
    // y[t] = residual[t] + the sum of part over token t's rows
    const float* part;
    const uint16_t* residual;
    uint16_t* y;
    int64_t ldr, ldy;
    // dweights[slot] = the sum of dot over the slot's row + <b2[expert], dy[t]>
    const float* dot;
    const int32_t* indices;
    const uint16_t *b2, *dy;
    void* dweights;
    int64_t lddy;
    int dots, weights_type;
    // v_sums[e][c] = sum of row weight * v[row][c] over the rows of expert e
    const uint16_t* v;
    uint16_t* v_sums;
    int64_t ldv;
    int v_cols;
    // the same from the products' sums over 32 rows
    const float* sums;
    uint16_t* sums_out;
    int sums_cols;
    int join_blocks, dweights_blocks, v_blocks, sums_blocks;  // set by launch_ends
};
int launch_ends(som_layers* l, EndArgs a, cudaStream_t st);

int launch_route(som_layers* l, int type, int score, int64_t T, int E, int k, const void* logits, int64_t ld, const float* bias,
                 int groups, int top_groups, int group_best, int renorm, float scale, float* weights, int32_t* indices,
                 int32_t* counts, cudaStream_t st);
int launch_route_backward(som_layers* l, int type, int score, int64_t T, int E, int k, const void* logits, int64_t ld,
                          const int32_t* indices, const float* dweights, int renorm, float scale, void* dlogits, cudaStream_t st);

}  // namespace lay
