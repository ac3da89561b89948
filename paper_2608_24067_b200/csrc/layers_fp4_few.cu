// The linear layer in 4 bits for one to a few rows, on the CUDA cores: single tokens while decoding.
//
// What counts is the weights' bytes and the launch.  A warp takes four rows of the weights that are 32 apart (their scales of four blocks
// are 16 bytes in a row), all loads of 4096 columns on their way at once, a lane one block of 32 values a row and step of 1024 columns.
// Products are whole numbers: twice a 4-bit value is one of 0, 1, 2, 3, 4, 6, 8, 12 and their negatives, which byte permutation looks up from a
// code (its sign bit selects 0, so that positive and negative values come in two words), and four products are added by one
// instruction; a block's sum is exact.  x is quantised by every block for itself, into shared memory, while the weights travel.
// Several warps share a row's columns where there are few rows, and a feature's gate and its other half where there is one.
//
// One row of 4096 against 4096 gated features: 8.2 us from a graph (17.8 MB; the bf16 weights' 67 MB take 13.5).  Of that the launch, x and the
// first loads' way are 4; two and more waves of blocks add their starts (4096 -> 16384 15 us).  Values by the conversion to fp16 and packed
// products instead: 7.7 us for one row, 17.0 instead of 15.7 for four; a place loaded again as soon as it is used, smaller steps
// with more blocks an SM: 8.5 to 10.5.
#include <type_traits>

#include "layers_fp4.cuh"

namespace lay {
namespace {

constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int STEPS = 4;  // of 1024 columns that a warp has on their way

struct FewFp4Args {
    const uint16_t* x;
    const uint8_t *w, *ws;
    const uint16_t *bias, *residual;
    uint16_t* y;
    int64_t ldx, ldr, ldy;
    int rows, D, F, share, act, bf16;
};

// The sums are held times this: a block's sum (4608 at most, of doubled values) times the weights' power of two alone is then finite, and only what
// the row's sum itself is may be infinite.  Sums below 2^-116 keep steps of 2^-139; half the smallest output is 2^-134 (bf16).
constexpr float DOWN = 0x1p-10f;

constexpr uint32_t LOW = 0x03020100u, HIGH = 0x0c080604u;  // twice the values of the codes 0 to 7

// twice the positive and the negative values of four codes (the lowest 16 bits), the others 0
__device__ __forceinline__ uint32_t doubled(uint32_t codes)
{
    uint32_t v;  // (a selector's highest bit takes the byte's sign alone: 0)
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(v) : "r"(LOW), "r"(HIGH), "r"(codes));
    return v;
}

template <int ROWS, int HALVES>
__global__ void __launch_bounds__(THREADS, 2) k_fp4_few(const FewFp4Args a)
{
    extern __shared__ __align__(16) unsigned char xs[];  // [ROWS][2][D / 32][16] doubled values (the halves of all blocks), then [ROWS][D / 32] powers of two
    __shared__ float part[WARPS][4 * ROWS];
    float* powers = reinterpret_cast<float*>(xs + ROWS * a.D);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, blocks = a.D / 32, tiles = (a.D + 255) / 256;
    const int each = HALVES * a.share, unit = warp / each, half = warp % HALVES, piece = warp % each / HALVES;  // units a block: WARPS / each
    // features f, f + 32, f + 64, f + 96
    const int q = blockIdx.x * (WARPS / each) + unit, f = q / 32 * 128 + q % 32, row0 = half * a.F + f;
    enter();
    uint4 w[STEPS][4], s[STEPS];
    auto fetch = [&](int j0) {
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int j = j0 + 32 * a.share * k;
            const bool in = j < blocks && f < a.F;
            s[k] = in ? *reinterpret_cast<const uint4*>(a.ws + fp4_scale_at(row0, j & ~3, tiles)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[k][i] = in && f + 32 * i < a.F ? __ldcs(reinterpret_cast<const uint4*>(a.w + ((int64_t)(row0 + 32 * i) * a.D + j * 32) / 2)) : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    int j0 = piece * 32 + lane;
    fetch(j0);
    for (int c = threadIdx.x; c < ROWS * (a.D / 8); c += THREADS) {  // (D / 8 is a multiple of four: a block of 32 is four lanes')
        const int r = ROWS == 1 ? 0 : c / (a.D / 8), col = (ROWS == 1 ? c : c - r * (a.D / 8)) * 8;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (r < a.rows) load8(a.x + r * a.ldx + col, v, a.bf16);
        float top = largest(v[0], v[1], v[2]);
        top = largest(top, v[3], v[4]);
        top = largest(largest(top, v[5], v[6]), v[7], 0.f);
        uint32_t most = __float_as_uint(top);
        const uint32_t four = 0xfu << (lane & ~3);
        most = max(most, __shfl_xor_sync(four, most, 1));
        most = max(most, __shfl_xor_sync(four, most, 2));
        const uint32_t e = fp4_scale_of(most);
        const float by = fp4_inverse(e);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= by;
        const uint32_t codes = e == 255u ? 0u : fp4_codes(v), other = codes ^ 0x88888888u;
        *reinterpret_cast<uint2*>(xs + r * a.D + (col & 16) * blocks + (col >> 5) * 16 + (col & 8)) =
            make_uint2(__vsub4(doubled(codes), doubled(other)), __vsub4(doubled(codes >> 16), doubled(other >> 16)));
        if ((lane & 3) == 0) powers[r * blocks + col / 32] = fp4_power(e);
    }
    __syncthreads();
    float acc[4][ROWS];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) acc[i][r] = 0.f;
    for (;;) {
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int j = j0 + 32 * a.share * k;
            if (j >= blocks) break;
            const uint32_t es[4] = {s[k].x, s[k].y, s[k].z, s[k].w};
            int sum[4][ROWS];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < ROWS; ++r) sum[i][r] = 0;
#pragma unroll
            for (int p = 0; p < 4; ++p) {  // eight columns
                uint2 xv[ROWS];  // (two loads become one of 16 bytes)
#pragma unroll
                for (int r = 0; r < ROWS; ++r) xv[r] = *(reinterpret_cast<const uint2*>(xs + r * a.D + (p >> 1) * (16 * blocks) + j * 16) + (p & 1));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t codes = p == 0 ? w[k][i].x : p == 1 ? w[k][i].y : p == 2 ? w[k][i].z : w[k][i].w, other = codes ^ 0x88888888u;
                    const uint32_t up0 = doubled(codes), up1 = doubled(codes >> 16), down0 = doubled(other), down1 = doubled(other >> 16);
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) {
                        sum[i][r] = __dp4a((int)up1, (int)xv[r].y, __dp4a((int)up0, (int)xv[r].x, sum[i][r]));
                        sum[i][r] -= __dp4a((int)down1, (int)xv[r].y, __dp4a((int)down0, (int)xv[r].x, 0));
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float by = fp4_power((es[i] >> (8 * (j & 3))) & 255u) * (0.25f * DOWN);  // (both were doubled)
#pragma unroll
                for (int r = 0; r < ROWS; ++r) acc[i][r] = fmaf((float)sum[i][r] * by, powers[r * blocks + j], acc[i][r]);
            }
        }
        j0 += 32 * a.share * STEPS;
        if (j0 - lane >= blocks) break;
        fetch(j0);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) acc[i][r] += __shfl_xor_sync(0xffffffffu, acc[i][r], d);
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) part[warp][i * ROWS + r] = acc[i][r];
    __syncthreads();
    // a thread an output of the block's units; the pieces in their order
    const int outs = WARPS / each * 4 * ROWS;
    if (threadIdx.x >= outs) return;
    const int u = threadIdx.x / (4 * ROWS), i = threadIdx.x % (4 * ROWS) / ROWS, r = threadIdx.x % ROWS;
    const int uq = blockIdx.x * (WARPS / each) + u, col = uq / 32 * 128 + uq % 32 + 32 * i;
    if (col >= a.F || r >= a.rows) return;
    float z = 0.f, g = 0.f;
    for (int k = 0; k < a.share; ++k) {
        z += part[u * each + k * HALVES][i * ROWS + r];
        if (HALVES == 2) g += part[u * each + k * HALVES + HALVES - 1][i * ROWS + r];
    }
    z *= 1.f / DOWN;
    g *= 1.f / DOWN;
    if (a.bias) {
        z += unpack1(a.bias[col], a.bf16);
        if (HALVES == 2) g += unpack1(a.bias[a.F + col], a.bf16);
    }
    float y = 0.f;
    with_act(a.act, [&](auto tag) { y = act_of<decltype(tag)::value>(z); });
    if (HALVES == 2) y *= g;
    if (a.residual) y += unpack1(a.residual[r * a.ldr + col], a.bf16);
    a.y[r * a.ldy + col] = (uint16_t)pack2(y, 0.f, a.bf16);
}

constexpr int MOST_SMEM = 96 << 10;

int few_bytes(int rows, int64_t D) { return (int)(rows * (D + D / 32 * 4)); }

template <int ROWS, int HALVES>
cudaError_t prepare_as()
{
    return cudaFuncSetAttribute(k_fp4_few<ROWS, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST_SMEM);
}

}  // namespace

cudaError_t prepare_fp4_few()
{
    cudaError_t e = prepare_as<1, 1>();
    if (e == cudaSuccess) e = prepare_as<2, 1>();
    if (e == cudaSuccess) e = prepare_as<4, 1>();
    if (e == cudaSuccess) e = prepare_as<1, 2>();
    if (e == cudaSuccess) e = prepare_as<2, 2>();
    return e == cudaSuccess ? prepare_as<4, 2>() : e;
}

// Rows so few that the CUDA cores take them, and not the tensor cores' tiles (x's quantisation, the product, often k_finish): a row costs
// them as many instructions as weights.  In us from a graph, this / tiles, bf16, `*` where tiles are taken:
//   D -> outputs            1 row          2 rows         3 or 4
//   4096 -> 8192 (gated)   8.2 / 12.4    10.5 / 12.4    15.7 / 12.4 *
//   4096 -> 4096           5.8 / 9.2      7.6 / 9.2     11.4 / 9.2 *
//   2048 -> 4096           3.8 / 7.7      4.7 / 7.7      6.9 / 7.7 *
//   4096 -> 16384         15.0 / 15.5    19.5 / 15.5 *  29.5 / 15.7 *
//   8192 -> 1024           5.1 / 9.7      7.7 / 9.7     13.2 / 9.7 *
//   1024 -> 1024           2.7 / 6.9      3.0 / 6.9      4.3 / 6.9
bool fp4_few_rows(const Fp4Product& p)
{
    if (p.T > FP4_FEW || (p.gated && p.F % 128 != 0)) return false;  // (a feature's gate and its other row lie alike in their 128 rows of scales)
    const int rows = p.T <= 2 ? (int)p.T : 4;
    return few_bytes(rows, p.D) <= MOST_SMEM && rows * p.D * (p.gated ? 2 * p.F : p.F) <= (rows <= 2 ? (int64_t)72 : (int64_t)20) << 20;
}

int launch_fp4_few(som_layers* l, const Fp4Product& p, const uint16_t* x, int64_t ldx, cudaStream_t st)
{
    const int halves = p.gated ? 2 : 1, rows = p.T <= 2 ? (int)p.T : 4, quads = (int)(tiles_of(p.F, 128) * 32);
    // warps that share a row's columns: where there are not eight warps an SM otherwise, and each keeps a step of 1024 columns
    int share = 1;
    while (share * 2 * halves <= WARPS && (int64_t)quads * halves * share * 2 <= (int64_t)8 * l->sm_count && share * 1024 < p.D) share *= 2;
    const FewFp4Args a = {x, p.w_codes, p.w_scales, p.bias, p.residual, p.y, ldx, p.ldr, p.ldy, (int)p.T, (int)p.D, (int)p.F, share, p.act, p.bf16};
    const dim3 grid((unsigned)tiles_of((int64_t)quads * halves * share, WARPS));
    const size_t smem = few_bytes(rows, p.D);
    auto run = [&](auto r, auto h) { return launch(l, k_fp4_few<decltype(r)::value, decltype(h)::value>, grid, THREADS, smem, st, 1, a); };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    if (halves == 1) return outcome(l, rows == 1 ? run(One(), One()) : rows == 2 ? run(Two(), One()) : run(Four(), One()));
    return outcome(l, rows == 1 ? run(One(), Two()) : rows == 2 ? run(Two(), Two()) : run(Four(), Two()));
}

}  // namespace lay
