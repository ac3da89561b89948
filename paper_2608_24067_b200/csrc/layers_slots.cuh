// Launchers of layers_slots.cu.
#pragma once

#include "layers_internal.cuh"

namespace lay {

// xp[row] = x[token of row's slot], the same of dy unless it is NULL; zeros up to whole steps of 64 rows
int launch_gather(som_layers* l, const SlotPlan& p, int k, int64_t D, const void* x, int64_t ldx, void* xp, const void* dy,
                  int64_t lddy, void* dyp, cudaStream_t st);
int launch_join(som_layers* l, const SlotPlan& p, int64_t T, int k, int64_t D, const float* part, const void* residual, int64_t ldr,
                void* y, int64_t ldy, int bf16, cudaStream_t st);
int launch_dweights(som_layers* l, const SlotPlan& p, const int32_t* indices, int64_t T, int k, int64_t D, const float* dot, int parts,
                    const void* b2, const void* dy, int64_t lddy, void* dweights, int weights_type, int bf16, cudaStream_t st);
// out[e][c] = sum of row weight * v[row][c] over the rows of expert e; without p.seg the sum over [0, rows)
int launch_column_sums(som_layers* l, const SlotPlan& p, int E, int64_t rows, const void* v, int64_t ld, int64_t cols, void* out,
                       int bf16, cudaStream_t st);
// the same from the products' sums over 32 rows
int launch_join_sums(som_layers* l, const SlotPlan& p, int E, int64_t rows, const float* part, int64_t cols, void* out, int bf16,
                     cudaStream_t st);

int launch_route(som_layers* l, int type, int score, int64_t T, int E, int k, const void* logits, int64_t ld, const float* bias,
                 int groups, int top_groups, int group_best, int renorm, float scale, float* weights, int32_t* indices,
                 int32_t* counts, cudaStream_t st);
int launch_route_backward(som_layers* l, int type, int score, int64_t T, int E, int k, const void* logits, int64_t ld,
                          const int32_t* indices, const float* dweights, int renorm, float scale, void* dlogits, cudaStream_t st);

}  // namespace lay
