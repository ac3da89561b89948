// Matrices in 4 bits: quantisation by blocks of 32 values with a power of two each, and back.
//
// Bound by HBM: 2.53 bytes a value from bf16 or to it.  A thread takes eight consecutive values (16 bytes of a 16-bit type), four threads
// share a block of 32; a warp takes 256 columns of a row, which are one row of a tile of the scales.
#include "layers_fp4.cuh"

namespace lay {
namespace {

struct QuantArgs {
    const void* x;
    int64_t ldx, T, D;
    uint8_t *codes, *scales;
    int bf16;
};

struct ValuesArgs {
    const uint8_t *codes, *scales;
    void* y;
    int64_t ldy, T, D;
    int bf16;
};

constexpr int Q_THREADS = 256;

template <bool WIDE>
__global__ void __launch_bounds__(Q_THREADS) k_fp4_quantize(const QuantArgs a)
{
    enter();
    const int lane = threadIdx.x & 31;
    const int64_t tiles = fp4_tiles(a.D), warps = a.T * tiles;
    for (int64_t i = ((int64_t)blockIdx.x * Q_THREADS + threadIdx.x) >> 5; i < warps; i += (int64_t)gridDim.x * (Q_THREADS / 32)) {
        const int64_t row = i / tiles, tile = i - row * tiles, col = tile * 256 + lane * 8;
        const bool in = col < a.D;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (in) {
            if (WIDE) {
                const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(a.x) + row * a.ldx + col);
                const float4 x0 = p[0], x1 = p[1];
                v[0] = x0.x, v[1] = x0.y, v[2] = x0.z, v[3] = x0.w, v[4] = x1.x, v[5] = x1.y, v[6] = x1.z, v[7] = x1.w;
            } else {
                load8(static_cast<const uint16_t*>(a.x) + row * a.ldx + col, v, a.bf16);
            }
        }
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(v[j]) & 0x7fffffffu);
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const uint32_t e = fp4_scale_of(most);
        const float by = fp4_inverse(e);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= by;
        if (in) *reinterpret_cast<uint32_t*>(a.codes + (row * a.D + col) / 2) = e == 255u ? 0u : fp4_codes(v);
        // four blocks' bytes lie next to each other
        uint32_t four = e << (8 * ((lane >> 2) & 3));
        four |= __shfl_xor_sync(0xffffffffu, four, 4);
        four |= __shfl_xor_sync(0xffffffffu, four, 8);
        if ((lane & 15) == 0) *reinterpret_cast<uint32_t*>(a.scales + fp4_scale_at(row, tile * 8 + lane / 4, tiles)) = four;
    }
}

template <bool WIDE>
__global__ void __launch_bounds__(Q_THREADS) k_fp4_values(const ValuesArgs a)
{
    enter();
    const int lane = threadIdx.x & 31;
    const int64_t tiles = fp4_tiles(a.D), warps = a.T * tiles;
    for (int64_t i = ((int64_t)blockIdx.x * Q_THREADS + threadIdx.x) >> 5; i < warps; i += (int64_t)gridDim.x * (Q_THREADS / 32)) {
        const int64_t row = i / tiles, tile = i - row * tiles, col = tile * 256 + lane * 8;
        if (col >= a.D) continue;
        const uint32_t w = *reinterpret_cast<const uint32_t*>(a.codes + (row * a.D + col) / 2);
        const float by = fp4_power(a.scales[fp4_scale_at(row, tile * 8 + lane / 4, tiles)]);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fp4_value(w >> (4 * j)) * by;
        if (WIDE) {
            float4* p = reinterpret_cast<float4*>(static_cast<float*>(a.y) + row * a.ldy + col);
            p[0] = make_float4(v[0], v[1], v[2], v[3]);
            p[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.y) + row * a.ldy + col) =
                make_uint4(pack2(v[0], v[1], a.bf16), pack2(v[2], v[3], a.bf16), pack2(v[4], v[5], a.bf16), pack2(v[6], v[7], a.bf16));
        }
    }
}

unsigned blocks_for(const som_layers* l, int64_t warps)
{
    const int64_t want = tiles_of(warps, Q_THREADS / 32), most = (int64_t)l->sm_count * 64;
    return (unsigned)(want < most ? want : most);
}

int check_fp4(const som_layers* l, int type, int64_t T, int64_t D)
{
    if (!l || T < 0 || D <= 0 || type < SOM_F32 || type > SOM_BF16) return SOM_ERR_INVALID_ARG;
    return T >= MOST_ROWS || D > MOST_COLS || D % FP4_BLOCK != 0 ? SOM_ERR_UNSUPPORTED : SOM_OK;
}

int check_rows_of(int type, const void* p, int64_t ld, int64_t D, int64_t T)
{
    if (T == 0) return SOM_OK;
    if (!p || ld < D) return SOM_ERR_INVALID_ARG;
    return !aligned16(p) || ld % (type == SOM_F32 ? 4 : 8) != 0 || ld >= (int64_t)1 << 32 ? SOM_ERR_UNSUPPORTED : SOM_OK;
}

int check_quantized(const void* codes, const void* scales, int64_t rows)
{
    if (rows == 0) return SOM_OK;
    if (!codes || !scales) return SOM_ERR_INVALID_ARG;
    return aligned16(codes) && (reinterpret_cast<uintptr_t>(scales) & 127u) == 0 ? SOM_OK : SOM_ERR_UNSUPPORTED;
}

}  // namespace

int launch_fp4_quantize(som_layers* l, int type, int64_t T, int64_t D, const void* x, int64_t ldx, uint8_t* codes, uint8_t* scales, cudaStream_t st)
{
    const QuantArgs a = {x, ldx, T, D, codes, scales, type == SOM_BF16};
    const dim3 grid(blocks_for(l, T * fp4_tiles(D)));
    return outcome(l, type == SOM_F32 ? launch(l, k_fp4_quantize<true>, grid, Q_THREADS, 0, st, 1, a) : launch(l, k_fp4_quantize<false>, grid, Q_THREADS, 0, st, 1, a));
}

}  // namespace lay

using namespace lay;

extern "C" {

int64_t som_fp4_scale_bytes(int64_t rows, int64_t D)
{
    return rows < 0 || D <= 0 || rows >= MOST_ROWS || D > MOST_COLS || D % FP4_BLOCK != 0 ? -1 : fp4_scale_bytes(rows, D);
}

int som_fp4_quantize(som_layers* l, int type, int64_t T, int64_t D, const void* x, int64_t ldx, void* codes, void* scales, void* stream)
{
    LAY_TRY(check_fp4(l, type, T, D));
    LAY_TRY(check_rows_of(type, x, ldx, D, T));
    LAY_TRY(check_quantized(codes, scales, T));
    if (T == 0) return SOM_OK;
    Guard g(l->device);
    return launch_fp4_quantize(l, type, T, D, x, ldx, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales), reinterpret_cast<cudaStream_t>(stream));
}

int som_fp4_values(som_layers* l, int type, int64_t T, int64_t D, const void* codes, const void* scales, void* y, int64_t ldy, void* stream)
{
    LAY_TRY(check_fp4(l, type, T, D));
    LAY_TRY(check_rows_of(type, y, ldy, D, T));
    LAY_TRY(check_quantized(codes, scales, T));
    if (T == 0) return SOM_OK;
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const ValuesArgs a = {static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), y, ldy, T, D, type == SOM_BF16};
    const dim3 grid(blocks_for(l, T * fp4_tiles(D)));
    return outcome(l, type == SOM_F32 ? launch(l, k_fp4_values<true>, grid, Q_THREADS, 0, st, 1, a) : launch(l, k_fp4_values<false>, grid, Q_THREADS, 0, st, 1, a));
}

int som_fp4_linear(som_layers* l, int type, int act, int gated, int64_t T, int64_t D, int64_t F, const void* x, int64_t ldx,
                   const void* w_codes, const void* w_scales, const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy,
                   void* stream)
{
    LAY_TRY(check_common(l, type, act, T));
    LAY_TRY(check_sizes(D, F));
    LAY_TRY(check_fp4(l, type, T, D));
    LAY_TRY(check_quantized(w_codes, w_scales, 1));
    LAY_TRY(check_rows(x, ldx, D, T));
    LAY_TRY(check_rows(y, ldy, F, T));
    if (residual) LAY_TRY(check_rows(residual, ldr, F, T));
    if (!aligned16(bias)) return SOM_ERR_UNSUPPORTED;
    if (T == 0) return SOM_OK;
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    Fp4Product p = {};
    p.w_codes = static_cast<const uint8_t*>(w_codes);
    p.w_scales = static_cast<const uint8_t*>(w_scales);
    p.bias = static_cast<const uint16_t*>(bias);
    p.residual = static_cast<const uint16_t*>(residual);
    p.y = static_cast<uint16_t*>(y);
    p.T = T, p.D = D, p.F = F, p.ldr = ldr, p.ldy = ldy;
    p.act = act, p.gated = gated != 0, p.bf16 = type == SOM_BF16;
    uint8_t *codes = nullptr, *scales = nullptr;
    unsigned char* parts = nullptr;
    auto carve = [&](Carver c) {
        codes = c.take<uint8_t>(T * D / 2);
        scales = c.take<uint8_t>(fp4_scale_bytes(T, D));
        parts = c.take<unsigned char>((int64_t)fp4_product_bytes(l, p));
        return c.used;
    };
    LAY_TRY(ensure(l, carve(Carver{nullptr, 0})));
    carve(Carver{static_cast<unsigned char*>(l->ws), 0});
    LAY_TRY(launch_fp4_quantize(l, type, T, D, x, ldx, codes, scales, st));
    p.x_codes = codes;
    p.x_scales = scales;
    return launch_fp4_product(l, p, parts, st);
}

}  // extern "C"
