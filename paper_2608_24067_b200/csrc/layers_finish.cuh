// Joining the parts of a product whose sum was split over blocks (ProdArgs::splits).
#pragma once

#include "layers_internal.cuh"

namespace lay {

enum FinishMode { FINISH_SUM = 0, FINISH_FWD = 1, FINISH_DZ = 2 };

struct FinishArgs {
    const float* part;  // [splits][rows][n]
    int64_t rows;
    int splits, n, cols;  // n: columns of the parts; cols: of the output (gated: n = 2 cols)
    const uint16_t* bias;
    const uint16_t* extra;  // FINISH_FWD: residual or nullptr; FINISH_DZ: dy
    int64_t ld_extra;
    uint16_t* out;  // [rows][ld]; FINISH_DZ: dz with n columns
    int64_t ld;
    int mode, act, gated, bf16;
};

int launch_finish(som_layers* l, const FinishArgs& a, cudaStream_t st);

}  // namespace lay
