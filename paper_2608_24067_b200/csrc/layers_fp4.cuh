// 4-bit matrices: layout of the scales, conversions, and the launches that the C entries share.
#pragma once

#include "layers_host.cuh"
#include "layers_math.cuh"

namespace lay {

constexpr int FP4_BLOCK = 32;       // values that share a power of two
constexpr int FP4_SCALE_TILE = 1024;  // bytes of the scales of 128 rows and 256 columns

// Byte of block j (columns 32 j to 32 j + 31) of a row; tiles = (D + 255) / 256
__host__ __device__ __forceinline__ int64_t fp4_scale_at(int64_t row, int64_t j, int64_t tiles)
{
    const int r = (int)(row & 127);
    return ((row >> 7) * tiles + (j >> 3)) * FP4_SCALE_TILE + ((j >> 2) & 1) * 512 + (r & 31) * 16 + (r >> 5) * 4 + (j & 3);
}

__host__ __device__ __forceinline__ int64_t fp4_tiles(int64_t D) { return (D + 255) / 256; }
inline int64_t fp4_scale_bytes(int64_t rows, int64_t D) { return (rows + 127) / 128 * fp4_tiles(D) * FP4_SCALE_TILE; }

// 2^(e - 127); 255 is NaN
__device__ __forceinline__ float fp4_power(uint32_t e) { return __uint_as_float(e == 255u ? 0x7fc00000u : e ? e << 23 : 0x00400000u); }

// the scale's byte of a block whose largest magnitude has these bits (infinity and NaN: 255)
__device__ __forceinline__ uint32_t fp4_scale_of(uint32_t most)
{
    if (most >= 0x7f800000u) return 255u;
    const int e = (int)((most + 0x200000u) >> 23) - 2;  // (a fraction of 0.75 and more carries into the exponent)
    return e < 0 ? 0u : e > 252 ? 252u : (uint32_t)e;  // (beyond 2^125 four of them would be infinite)
}

// what the values of such a block are multiplied by: 2^(127 - e), e <= 252
__device__ __forceinline__ float fp4_inverse(uint32_t e) { return __uint_as_float(e < 254u ? (254u - e) << 23 : 0u); }

// eight values, multiplied already, as eight codes: the first in the lowest four bits
__device__ __forceinline__ uint32_t fp4_codes(const float (&v)[8])
{
    uint32_t w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return w;
}

// The value of a code (its low four bits) over the block's power of two: the bits of its magnitude are the top of a number of the two
// smallest exponents, which 2^126 lifts to [0, 6].
__device__ __forceinline__ float fp4_value(uint32_t code) { return __uint_as_float(((code & 7u) << 22) | ((code & 8u) << 28)) * 0x1p126f; }

// The values of eight codes over their blocks' power of two, the first in the lowest four bits.  All of them have to be used: where the results of the two
// upper bytes are not, the optimising assembler (12.9) gives zeros for the lower two as well, however the codes were loaded (unoptimised, or with
// the upper two looked at, all 65536 codes of the lower two are right).
__device__ __forceinline__ void fp4_values(uint32_t w, float2 (&v)[4])
{
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
}

// A product of two matrices in 4 bits with som_linear's epilogue.
struct Fp4Product {
    const uint8_t *x_codes, *x_scales, *w_codes, *w_scales;
    const uint16_t *bias, *residual;
    uint16_t* y;
    int64_t T, D, F, ldr, ldy;
    int act, gated, bf16;
};

cudaError_t prepare_fp4_product(som_layers* l);  // once per handle
size_t fp4_product_bytes(const som_layers* l, const Fp4Product& p);  // workspace
int launch_fp4_product(som_layers* l, const Fp4Product& p, unsigned char* ws, cudaStream_t st);

constexpr int FP4_FEW = 4;  // the most rows of launch_fp4_few
cudaError_t prepare_fp4_few();            // once per handle
bool fp4_few_rows(const Fp4Product& p);   // whether launch_fp4_few takes them (it quantises x itself)
int launch_fp4_few(som_layers* l, const Fp4Product& p, const uint16_t* x, int64_t ldx, cudaStream_t st);

int launch_fp4_quantize(som_layers* l, int type, int64_t T, int64_t D, const void* x, int64_t ldx, uint8_t* codes, uint8_t* scales, cudaStream_t st);

}  // namespace lay
