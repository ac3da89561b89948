// Launchers of layers_few.cu: the linear unit and the experts' products for a handful of rows.
#pragma once

#include "layers_internal.cuh"

namespace lay {

constexpr int FEW_ROWS = 8;              // rows of x that share a read of the weights
constexpr int FEW_SMEM = 128 * 1024;     // most bytes of rows (or hidden values) in shared memory

struct FewArgs {
    const uint16_t* x;
    int64_t ldx;
    const uint16_t* w;     // [E][halves * F][D]
    const uint16_t* bias;  // [E][halves * F] or nullptr
    // som_linear: `rows` rows to y; som_experts: a slot a group, its hidden values times its weight to hidden[slot][F]
    const uint16_t* residual;
    int64_t ldr;
    uint16_t* y;
    int64_t ldy;
    float* hidden;
    const int32_t* indices;
    const void* weights;
    int weights_type, k, E;
    int rows, D, F, act, bf16, share;
    int* flags;
};

struct FewDownArgs {
    const float* hidden;  // [T * k][I]
    const int32_t* indices;
    const void* weights;
    const uint16_t *w2, *b2, *residual;
    uint16_t* y;
    int64_t ldr, ldy;
    int weights_type, k, E, D, I, bf16, share;
};

cudaError_t prepare_few();  // once per handle
int launch_few(som_layers* l, FewArgs a, int groups, bool gated, cudaStream_t st);
int launch_few_down(som_layers* l, FewDownArgs a, int64_t T, cudaStream_t st);

}  // namespace lay
