// The matrix products of the dense operators on tcgen05: launch descriptions shared by the kernels and the C ABI.
#pragma once

#include "layers_internal.cuh"

namespace lay {

enum ProdMode {
    PROD_FWD = 0,     // out[row, n] = epilogue(sum_k A[row, k] B[n, k])
    PROD_DZ = 1,      // the same product, epilogue multiplies dy by the activation's derivative
    PROD_DZ_TWO = 2,  // two products over the same rows: z = x W1^T and g = dy W2; epilogue of the experts' gradient
    PROD_DX = 3,      // out[row, n] = sum_k A[row, k] B[k, n]
    PROD_DW = 4       // out[e][m, n] = sum_rows A[row, m] B[row, n] over the rows of expert e
};

// Output tiles: NARROW 128 x 128 and WIDE 128 x 256 by one block, PAIR 256 x 256 by two blocks of a cluster.
enum ProdShape { NARROW = 0, WIDE = 1, PAIR = 2 };
__host__ __device__ constexpr int shape_rows(int shape) { return shape == PAIR ? 256 : 128; }
__host__ __device__ constexpr int shape_cols(int shape) { return shape == NARROW ? 128 : 256; }

// Rows of a box of A where experts' rows are multiplied: boxes without rows in use are not fetched.  96 tokens x 6 of 64 experts of
// 2048 x 1024: 171 us, 177 with boxes of 128 rows, 173 with boxes of 32; 4096 tokens x 8: 589 us, 593 and 627 (more copies to issue).
constexpr int LEFT_BOX = 64;
constexpr int EPI_TURNS = 2;  // epilogue warps per 32 rows of a block's tile; they take its pieces of 32 columns in turn

// Rows of a box of a K-major B: what a block takes of consecutive rows, up to 128 (a copy more a step and the thread that issues
// them is what the products wait for)
__host__ __device__ constexpr int right_box(int mode, int shape, bool gated)
{
    const int share = shape_cols(shape) / (mode == PROD_DZ_TWO && !gated ? 2 : 1) / (shape == PAIR || gated ? 2 : 1);
    return share < 128 ? share : 128;
}

// partial sums of h * g that a tile of PROD_DZ_TWO (half as wide as others) leaves for a row
__host__ __device__ constexpr int tile_dots(int shape)
{
    return shape_cols(shape) / 2 / 32 < EPI_TURNS ? shape_cols(shape) / 2 / 32 : EPI_TURNS;
}

struct ProdArgs {
    CUtensorMap a, b;         // operands (of the first product)
    CUtensorMap a2, b2;       // second product of PROD_DZ_TWO, or a second one of PROD_DW over the same experts' rows
    CUtensorMap o;            // output of PROD_FWD, PROD_DX, PROD_DW
    CUtensorMap o2map;        // output of PROD_DW's second product, of rows2 x cols2
    int row_tiles2, col_tiles2, rows2, cols2;
    void* o0;                 // PROD_DZ, PROD_DZ_TWO: dz [rows][ld0], the gated half gate_rows columns on
    void* o2;                 // PROD_DZ_TWO: weighted hidden values [rows][ld2]
    int64_t ld0, ld2;
    const int* tiles;         // grouped rows: number of row tiles on the device; nullptr = row_tiles
    const int* tile_expert;   // grouped rows: expert of a row tile; nullptr = 0
    const int* seg;           // grouped rows: first row of every expert
    const int* count;         // and its rows in use; nullptr = one group of `rows` rows (PROD_DW: k1)
    const uint16_t* bias;     // [experts][bias_ld] or nullptr
    const uint16_t* extra;    // residual (PROD_FWD) or dy (PROD_DZ), [rows][ld_extra], or nullptr
    const float* row_weight;  // [rows] or nullptr
    float* dot;               // PROD_DZ_TWO: [rows][dots] partial sums of h * g, tile_dots a tile
    float* column_sums;       // PROD_DZ, PROD_DZ_TWO: [rows / 32][2 cols or cols] sums of dz over 32 rows, or nullptr
    int64_t ld_extra;
    int bias_ld, dots;
    int shape;
    int right_box;  // rows of a box of a K-major B: right_box()
    int row_tiles, col_tiles, experts;
    int splits;      // blocks that share a tile's sum (PROD_FWD, PROD_DX, PROD_DW; not grouped): part s goes to batch s of the output
    int rows, cols;  // extent of the outputs (PROD_DW: of one expert's)
    int gate_rows;   // gated: rows of B between a feature's gate row and its other row; 0 = not gated
    int k1, k2;      // length of the products' sums
    int act, bf16, out32;
    // B and the plan were complete before the kernel in front began its work (that kernel writes neither): the first stages' columns
    // are loaded while it still runs (96 tokens x 6 of 64 experts of 2048 x 1024: 169.1 us, 171.9 without)
    int columns_first;
    int weigh;  // row_weight multiplies: 1 the result, 2 the bias
    int* flags;
};

int launch_product(som_layers* l, ProdMode mode, const ProdArgs& args, cudaStream_t st);

// 3-d tensor map over [batch][rows][cols] of 16-bit (bytes = 2) or fp32 (4) elements in boxes of [1][box_rows] rows of 128 bytes
int make_map(som_layers* l, CUtensorMap* map, const void* base, int bytes, int64_t cols, int64_t rows, int64_t batch, int64_t ld,
             int64_t batch_stride, int box_rows);

}  // namespace lay
