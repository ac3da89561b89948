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
    int64_t rounds[6][3];  // most tiles a block walked, by ProdMode and ProdShape; most rounds of som_route's two forms
    void* encode;  // cuTensorMapEncodeTiled
};

namespace lay {

// Every kernel of the dense operators is launched so that its blocks may come in while the kernel before it ends
// (programmatic stream serialization), and begins with enter(): nothing is read or written before all earlier work in the
// stream is complete, and the next kernel's launch is let through only after that.  What such a kernel reads may have been
// written while it was already resident, so none of them uses the read-only data path.
__device__ __forceinline__ void enter()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <class... P, class... A>
cudaError_t launch(som_layers* l, void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, const A&... args)
{
    cudaLaunchConfig_t c = {};
    c.gridDim = grid;
    c.blockDim = dim3((unsigned)threads);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    c.attrs = attr;
    c.numAttrs = cluster > 1 ? 2 : 1;
    ++l->launches;
    return cudaLaunchKernelEx(&c, kernel, P(args)...);
}

// a launch's outcome as a status, the error kept on the handle (and not left for the check of another call's launch)
inline int outcome(som_layers* l, cudaError_t e)
{
    if (e == cudaSuccess) return SOM_OK;
    l->last_cuda_error = (int)e;
    (void)cudaGetLastError();
    return SOM_ERR_CUDA;
}

// Rows of the experts' work ("slots" = (token, place) pairs with an expert) in the experts' order, every expert's
// segment padded to whole row tiles.  All on the device, written by launch_plan.
struct SlotPlan {
    int* seg;          // [E + 1] first row of every expert's segment, multiples of the row tile
    int* count;        // [E] slots of every expert
    int* tiles;        // [1] row tiles in use
    int* tile_expert;  // [max tiles]
    int* pos;          // [T * k] row of a slot, -1 = none
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
