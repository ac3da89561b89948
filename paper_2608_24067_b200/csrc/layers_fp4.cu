// Matrices in 4 bits: quantisation by blocks of 32 values with a power of two each, and back.
//
// Bound by HBM: 2.53 bytes a value from bf16 or to it.  A thread takes eight consecutive values (16 bytes of a 16-bit type) of four rows that are
// 32 apart, whose bytes of scales lie next to each other; four threads share a block of 32, a warp takes 256 columns of the rows, one row each
// of a tile of the scales.  All four rows are on their way before the first is worked on, as they came (in fp32 they took twice
// the registers, 55 us).  16384 x 4096: from bf16 32 us (5.4 TB/s), from fp32 44 (6.8); to bf16 28 (6.1), to fp32 49 (6.2).
#include "layers_fp4.cuh"

namespace lay {
namespace {

struct QuantArgs {
    const void* x;
    int64_t ldx, T, D;
    uint32_t tiles, units;
    uint8_t *codes, *scales;
};

struct ValuesArgs {
    const uint8_t *codes, *scales;
    void* y;
    int64_t ldy, T, D;
    uint32_t tiles, units;
};

constexpr int Q_THREADS = 256, Q_ROWS = 4;

// Unit u of the work: a tile of 256 columns of the rows row, row + 32, row + 64 and row + 96, whose bytes of scales lie next to each other.
struct Unit {
    int64_t row, tile;
    __device__ __forceinline__ Unit(uint32_t u, uint32_t tiles)
    {
        const uint32_t r = u / tiles;
        tile = u - r * tiles;
        row = (int64_t)(r >> 5) * 128 + (r & 31);
    }
};

// TYPE: SOM_F32, SOM_F16 or SOM_BF16
template <int TYPE>
__global__ void __launch_bounds__(Q_THREADS, TYPE == SOM_F32 ? 4 : 5) k_fp4_quantize(const QuantArgs a)
{
    constexpr bool WIDE = TYPE == SOM_F32;
    enter();
    const int lane = threadIdx.x & 31;
    for (uint32_t u = (blockIdx.x * Q_THREADS + threadIdx.x) >> 5; u < a.units; u += gridDim.x * (Q_THREADS / 32)) {
        const Unit at(u, a.tiles);
        const int64_t col = at.tile * 256 + lane * 8;
        const bool in = col < a.D;
        uint4 raw[Q_ROWS][WIDE ? 2 : 1];  // eight values of each row
#pragma unroll
        for (int i = 0; i < Q_ROWS; ++i) {
            const int64_t row = at.row + 32 * i;
#pragma unroll
            for (int h = 0; h < (WIDE ? 2 : 1); ++h)
                raw[i][h] = !in || row >= a.T ? make_uint4(0u, 0u, 0u, 0u)
                            : WIDE            ? *(reinterpret_cast<const uint4*>(static_cast<const float*>(a.x) + row * a.ldx + col) + h)
                                              : *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.x) + row * a.ldx + col);
        }
        uint32_t four[Q_ROWS];
#pragma unroll
        for (int i = 0; i < Q_ROWS; ++i) {
            float v[8];
            if (WIDE) {
                const uint4 x0 = raw[i][0], x1 = raw[i][WIDE ? 1 : 0];
                v[0] = __uint_as_float(x0.x), v[1] = __uint_as_float(x0.y), v[2] = __uint_as_float(x0.z), v[3] = __uint_as_float(x0.w);
                v[4] = __uint_as_float(x1.x), v[5] = __uint_as_float(x1.y), v[6] = __uint_as_float(x1.z), v[7] = __uint_as_float(x1.w);
            } else {
                widen8(raw[i][0], v, TYPE == SOM_BF16);
            }
            float top = largest(v[0], v[1], v[2]);
            top = largest(top, v[3], v[4]);
            top = largest(largest(top, v[5], v[6]), v[7], 0.f);
            uint32_t most = __float_as_uint(top);
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const uint32_t e = fp4_scale_of(most);
            const float by = fp4_inverse(e);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float2 s = __fmul2_rn(make_float2(v[j], v[j + 1]), make_float2(by, by));
                v[j] = s.x, v[j + 1] = s.y;
            }
            const int64_t row = at.row + 32 * i;
            if (in && row < a.T) *reinterpret_cast<uint32_t*>(a.codes + (row * a.D + col) / 2) = e == 255u ? 0u : fp4_codes(v);
            // four blocks' bytes lie next to each other
            four[i] = e << (8 * ((lane >> 2) & 3));
            four[i] |= __shfl_xor_sync(0xffffffffu, four[i], 4);
            four[i] |= __shfl_xor_sync(0xffffffffu, four[i], 8);
        }
        if ((lane & 15) == 0) {
            uint32_t* to = reinterpret_cast<uint32_t*>(a.scales + fp4_scale_at(at.row, at.tile * 8 + lane / 4, a.tiles));
            if (at.row + 96 < a.T) {
                *reinterpret_cast<uint4*>(to) = make_uint4(four[0], four[1], four[2], four[3]);
            } else {
#pragma unroll
                for (int i = 0; i < Q_ROWS; ++i)
                    if (at.row + 32 * i < a.T) to[i] = four[i];
            }
        }
    }
}

template <int TYPE>
__global__ void __launch_bounds__(Q_THREADS) k_fp4_values(const ValuesArgs a)
{
    constexpr bool WIDE = TYPE == SOM_F32;
    enter();
    const int lane = threadIdx.x & 31;
    for (uint32_t u = (blockIdx.x * Q_THREADS + threadIdx.x) >> 5; u < a.units; u += gridDim.x * (Q_THREADS / 32)) {
        const Unit at(u, a.tiles);
        // Eight columns a lane; fp32: four and, 128 further on, four, so that a store of the warp is 512 bytes in a row.
        constexpr int PARTS = WIDE ? 2 : 1, N = 8 / PARTS;
        uint32_t w[Q_ROWS][PARTS];
        uint4 e[PARTS];
#pragma unroll
        for (int h = 0; h < PARTS; ++h) {
            const int64_t col = at.tile * 256 + h * 128 + lane * N;
            const bool in = col < a.D;
#pragma unroll
            for (int i = 0; i < Q_ROWS; ++i) {
                w[i][h] = 0u;
                if (in && at.row + 32 * i < a.T) {
                    const uint8_t* p = a.codes + ((at.row + 32 * i) * a.D + col) / 2;
                    w[i][h] = WIDE ? *reinterpret_cast<const uint16_t*>(p) : *reinterpret_cast<const uint32_t*>(p);
                }
            }
            // (the bytes of rows beyond the last are there, and not used)
            if (in) e[h] = *reinterpret_cast<const uint4*>(a.scales + fp4_scale_at(at.row, at.tile * 8 + (WIDE ? 4 * h : lane / 16 * 4), a.tiles));
        }
#pragma unroll
        for (int h = 0; h < PARTS; ++h) {
            const int64_t col = at.tile * 256 + h * 128 + lane * N;
            if (col >= a.D) continue;
            const uint32_t es[Q_ROWS] = {e[h].x, e[h].y, e[h].z, e[h].w};
            const int shift = 8 * (WIDE ? lane >> 3 : (lane >> 2) & 3);
#pragma unroll
            for (int i = 0; i < Q_ROWS; ++i) {
                const int64_t row = at.row + 32 * i;
                if (row >= a.T) break;
                const float by = fp4_power((es[i] >> shift) & 255u);
                if constexpr (WIDE) {  // by bits (four codes: see fp4_values)
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = fp4_value(w[i][h] >> (4 * j)) * by;
                    *reinterpret_cast<float4*>(static_cast<float*>(a.y) + row * a.ldy + col) = make_float4(v[0], v[1], v[2], v[3]);
                } else {
                    float2 v[4];
                    fp4_values(w[i][h], v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = __fmul2_rn(v[j], make_float2(by, by));
                    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.y) + row * a.ldy + col) =
                        make_uint4(pack2(v[0].x, v[0].y, TYPE == SOM_BF16), pack2(v[1].x, v[1].y, TYPE == SOM_BF16), pack2(v[2].x, v[2].y, TYPE == SOM_BF16),
                                   pack2(v[3].x, v[3].y, TYPE == SOM_BF16));
                }
            }
        }
    }
}

// units of T rows: 32 of every 128 rows, or as many as there are
uint32_t units_of(int64_t T, int64_t D)
{
    const int64_t rest = T % 128;
    return (uint32_t)((T / 128 * 32 + (rest < 32 ? rest : 32)) * fp4_tiles(D));
}

unsigned blocks_for(const som_layers* l, uint32_t units)
{
    const int64_t want = tiles_of(units, Q_THREADS / 32), most = (int64_t)l->sm_count * 64;
    return (unsigned)(want < most ? want : most);
}

int check_fp4(const som_layers* l, int type, int64_t T, int64_t D)
{
    if (!l || T < 0 || D <= 0 || type < SOM_F32 || type > SOM_BF16) return SOM_ERR_INVALID_ARG;
    return T >= MOST_ROWS || D > MOST_COLS || D % FP4_BLOCK != 0 || T * fp4_tiles(D) >= (int64_t)1 << 33 ? SOM_ERR_UNSUPPORTED : SOM_OK;
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
    const QuantArgs a = {x, ldx, T, D, (uint32_t)fp4_tiles(D), units_of(T, D), codes, scales};
    const dim3 grid(blocks_for(l, a.units));
    return outcome(l, launch(l, type == SOM_F32 ? k_fp4_quantize<SOM_F32> : type == SOM_F16 ? k_fp4_quantize<SOM_F16> : k_fp4_quantize<SOM_BF16>, grid, Q_THREADS, 0, st, 1, a));
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
    const ValuesArgs a = {static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), y, ldy, T, D, (uint32_t)fp4_tiles(D), units_of(T, D)};
    const dim3 grid(blocks_for(l, a.units));
    return outcome(l, launch(l, type == SOM_F32 ? k_fp4_values<SOM_F32> : type == SOM_F16 ? k_fp4_values<SOM_F16> : k_fp4_values<SOM_BF16>, grid, Q_THREADS, 0, st, 1, a));
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
    if (fp4_few_rows(p)) return launch_fp4_few(l, p, static_cast<const uint16_t*>(x), ldx, st);
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
