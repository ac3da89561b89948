// Internal declarations of the dense operators (som_linear, som_route, som_experts and their gradients).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "som_internal.cuh"

// bits of som_layers::flags
#define LAY_FLAG_BAD_EXPERT 1 /* an expert index outside [-1, E) was treated as -1 */
#define LAY_FLAG_GAVE_UP 2    /* a bounded wait inside a kernel ran out: the call's outputs are not valid */

struct som_layers {
    int device;
    int sm_count;
    int pairs;  // pairs of blocks that the products' kernels can have resident
    void* ws;  // grow-only device workspace of all calls on the handle
    size_t ws_bytes;
    int* flags;  // device, sticky LAY_FLAG_* bits
    int last_cuda_error;
    int64_t launches;
    void* encode;  // cuTensorMapEncodeTiled
};

namespace lay {

// Rows of the experts' work ("slots" = (token, place) pairs with an expert) in the experts' order, every expert's
// segment padded to whole row tiles.  All on the device, written by launch_plan.
struct SlotPlan {
    int* seg;          // [E + 1] first row of every expert's segment, multiples of the row tile
    int* count;        // [E] slots of every expert
    int* tiles;        // [1] row tiles in use
    int* tile_expert;  // [max tiles]
    int* pos;          // [T * k] row of a slot, -1 = none
    int* row_slot;     // [max rows] slot of a row in use
    float* row_weight; // [max rows] the slot's routing weight
    int* block_counts; // [plan_blocks][E] scratch of the plan
    int max_rows;      // upper bound that the host sizes buffers and grids by
    int tile;          // rows of a tile
};

cudaError_t prepare_product(som_layers* l);  // once per handle

cudaError_t prepare_plan();  // once per handle
int plan_blocks(int64_t slots);  // rows of SlotPlan::block_counts
int launch_plan(som_layers* l, const SlotPlan& p, const int32_t* indices, const void* weights, int weights_type, int64_t T,
                int k, int E, cudaStream_t st);

}  // namespace lay
