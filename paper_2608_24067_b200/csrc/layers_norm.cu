// Layer norm over the rows of a matrix, and its gradient.
//
//   h = x + residual, rounded to the matrix's type (it is an output, and the gradient starts from it); over a row of D values
//   mean = sum h / D, variance = sum (h - mean)^2 / D, n = (h - mean) r with r = 1 / sqrt(variance + eps), y = n weight + bias.
//   Gradient, with d = dy weight: dx = r (d - sum d / D - n sum (d n) / D) + dsum, dweight = sum over rows of dy n, dbias of dy.
//
// Bound by HBM: a few operations a value.  Everything between input and output is fp32; the variance is summed from the differences
// to the mean, not from squares, so that a row far from zero keeps its digits.
#include "layers_host.cuh"

namespace lay {
namespace {

struct NormArgs {
    const void *x, *residual, *weight, *bias;
    void *sum, *y;
    int64_t ldx, ldr, lds, ldy;
    int D;
    float eps;
};

struct NormBackArgs {
    const void *x, *weight, *dy, *dsum;
    void* dx;
    float* stats;  // [T][2] mean and r of every row, or nullptr
    int64_t ldx, lddy, ldds;
    int64_t T;
    int D;
    float eps;
};

struct ColumnArgs {
    const void *x, *dy;
    const float* stats;
    float* part;  // [parts][2][D]
    int64_t ldx, lddy, T;
    int D, parts;
};

struct ColumnJoinArgs {
    const float* part;
    void *dweight, *dbias;
    int D, parts;
};

__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ float wide(__half v) { return __half2float(v); }
__device__ __forceinline__ float wide(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class E>
__device__ __forceinline__ E narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

constexpr int ROW_THREADS = 256;

// the sums of N values over the block, to every thread, in a fixed order
template <int N, int THREADS>
__device__ __forceinline__ void block_sums(float (&v)[N])
{
    __shared__ float part[THREADS / 32][N];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
    __syncthreads();  // the last call's parts have been read
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) part[threadIdx.x >> 5][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.f;
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) v[i] += part[w][i];
    }
}

// Any row length and alignment: a block a row, which it walks three times (from L1 or L2 after the first).
template <class E, class W>
__global__ void __launch_bounds__(ROW_THREADS) k_norm_any(const NormArgs a)
{
    enter();
    const int64_t row = blockIdx.x;
    const E* x = static_cast<const E*>(a.x) + row * a.ldx;
    const E* res = a.residual ? static_cast<const E*>(a.residual) + row * a.ldr : nullptr;
    E* sum = a.sum ? static_cast<E*>(a.sum) + row * a.lds : nullptr;
    E* y = static_cast<E*>(a.y) + row * a.ldy;
    auto value = [&](int i) { return res ? wide(narrow<E>(wide(x[i]) + wide(res[i]))) : wide(x[i]); };
    float s[1] = {0.f};
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) s[0] += value(i);
    block_sums<1, ROW_THREADS>(s);
    const float mean = s[0] / (float)a.D;
    s[0] = 0.f;
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) {
        const float c = value(i) - mean;
        s[0] = fmaf(c, c, s[0]);
    }
    block_sums<1, ROW_THREADS>(s);
    const float r = 1.f / sqrtf(s[0] / (float)a.D + a.eps);
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) {
        const float h = value(i);
        float n = (h - mean) * r;
        if (a.weight) n *= wide(static_cast<const W*>(a.weight)[i]);
        if (a.bias) n += wide(static_cast<const W*>(a.bias)[i]);
        y[i] = narrow<E>(n);
        if (sum) sum[i] = narrow<E>(h);
    }
}

template <class E, class W>
__global__ void __launch_bounds__(ROW_THREADS) k_norm_back_any(const NormBackArgs a)
{
    enter();
    const int64_t row = blockIdx.x;
    const E* x = static_cast<const E*>(a.x) + row * a.ldx;
    const E* dy = static_cast<const E*>(a.dy) + row * a.lddy;
    const E* dsum = a.dsum ? static_cast<const E*>(a.dsum) + row * a.ldds : nullptr;
    const W* w = static_cast<const W*>(a.weight);
    const float n = (float)a.D;  // (divided by, not multiplied by its inverse: the mean of equal values is that value)
    float s[2] = {0.f, 0.f};
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) {
        s[0] += wide(x[i]);
        s[1] += w ? wide(dy[i]) * wide(w[i]) : wide(dy[i]);
    }
    block_sums<2, ROW_THREADS>(s);
    const float mean = s[0] / n, d_mean = s[1] / n;
    s[0] = s[1] = 0.f;
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) {
        const float c = wide(x[i]) - mean, d = w ? wide(dy[i]) * wide(w[i]) : wide(dy[i]);
        s[0] = fmaf(c, c, s[0]);
        s[1] = fmaf(c, d, s[1]);
    }
    block_sums<2, ROW_THREADS>(s);
    const float r = 1.f / sqrtf(s[0] / n + a.eps), along = s[1] / n * r * r;  // n sum (d n) / D = (h - mean) r^2 sum (d (h - mean)) / D
    if (a.stats && threadIdx.x == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, r);
    if (!a.dx) return;
    E* dx = static_cast<E*>(a.dx) + row * a.D;
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) {
        const float c = wide(x[i]) - mean, d = w ? wide(dy[i]) * wide(w[i]) : wide(dy[i]);
        float g = r * (d - d_mean - c * along);
        if (dsum) g += wide(dsum[i]);
        dx[i] = narrow<E>(g);
    }
}

// The columns' sums from the rows' statistics: 32 columns a block, eight rows at a time of one of `parts` stretches of the rows.
template <class E>
__global__ void __launch_bounds__(256) k_norm_columns(const ColumnArgs a)
{
    __shared__ float part[8][2][32];
    enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    const int64_t from = a.T * blockIdx.y / a.parts, to = a.T * (blockIdx.y + 1) / a.parts;
    float dw = 0.f, db = 0.f;
    if (col < a.D)
        for (int64_t row = from + warp; row < to; row += 8) {
            const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * row);
            const float d = wide(static_cast<const E*>(a.dy)[row * a.lddy + col]);
            dw = fmaf(d, (wide(static_cast<const E*>(a.x)[row * a.ldx + col]) - st.x) * st.y, dw);
            db += d;
        }
    part[warp][0][lane] = dw;
    part[warp][1][lane] = db;
    __syncthreads();
    if (warp < 2 && col < a.D) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += part[i][warp][lane];
        a.part[((int64_t)blockIdx.y * 2 + warp) * a.D + col] = s;
    }
}

// the parts' sum, in their order
template <class W>
__global__ void __launch_bounds__(256) k_norm_join(const ColumnJoinArgs a)
{
    __shared__ float part[8][32];
    enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t i = (int64_t)blockIdx.x * 32 + lane;  // of 2 D sums
    float s = 0.f;
    if (i < 2 * (int64_t)a.D)
        for (int p = warp; p < a.parts; p += 8) s += a.part[(int64_t)p * 2 * a.D + i];
    part[warp][lane] = s;
    __syncthreads();
    if (warp > 0 || i >= 2 * (int64_t)a.D) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += part[w][lane];
    W* to = static_cast<W*>(i < a.D ? a.dweight : a.dbias);
    if (to) to[i < a.D ? i : i - a.D] = narrow<W>(s);
}

// f(E(), W()) of the matrix's and the weights' types
template <class F>
cudaError_t by_types(int type, int weights_type, F&& f)
{
    if (type == SOM_F32) return f(float(), float());
    if (type == SOM_F16) return weights_type == SOM_F32 ? f(__half(), float()) : f(__half(), __half());
    return weights_type == SOM_F32 ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
}

int check_norm(const som_layers* l, int type, int weights_type, int64_t T, int64_t D, float eps)
{
    if (!l || T < 0 || D <= 0 || type < SOM_F32 || type > SOM_BF16 || (weights_type != SOM_F32 && weights_type != type) || !(eps >= 0.f))
        return SOM_ERR_INVALID_ARG;
    return T >= MOST_ROWS || D > MOST_COLS ? SOM_ERR_UNSUPPORTED : SOM_OK;
}

// rows of a norm's matrix: present, and long enough
int check_row(const void* p, int64_t ld, int64_t D, int64_t T)
{
    if (T == 0) return SOM_OK;
    if (!p || ld < D) return SOM_ERR_INVALID_ARG;
    return ld >= (int64_t)1 << 32 ? SOM_ERR_UNSUPPORTED : SOM_OK;
}

}  // namespace
}  // namespace lay

using namespace lay;

extern "C" {

int som_norm(som_layers* l, int type, int64_t T, int64_t D, const void* x, int64_t ldx, const void* weight, const void* bias,
             int weights_type, const void* residual, int64_t ldr, float eps, void* sum, int64_t lds, void* y, int64_t ldy, void* stream)
{
    LAY_TRY(check_norm(l, type, weights_type, T, D, eps));
    LAY_TRY(check_row(x, ldx, D, T));
    LAY_TRY(check_row(y, ldy, D, T));
    if (residual) LAY_TRY(check_row(residual, ldr, D, T));
    if (sum) LAY_TRY(check_row(sum, lds, D, T));
    if (T == 0) return SOM_OK;
    Guard g(l->device);
    const NormArgs a = {x, residual, weight, bias, sum, y, ldx, ldr, lds, ldy, (int)D, eps};
    return outcome(l, by_types(type, weights_type, [&](auto e, auto w) {
                       return launch(l, k_norm_any<decltype(e), decltype(w)>, dim3((unsigned)T), ROW_THREADS, 0, reinterpret_cast<cudaStream_t>(stream), 1, a);
                   }));
}

int som_norm_backward(som_layers* l, int type, int64_t T, int64_t D, const void* x, int64_t ldx, const void* weight, int weights_type,
                      const void* dy, int64_t lddy, const void* dsum, int64_t ldds, float eps, void* dx, void* dweight, void* dbias,
                      void* stream)
{
    LAY_TRY(check_norm(l, type, weights_type, T, D, eps));
    LAY_TRY(check_row(x, ldx, D, T));
    LAY_TRY(check_row(dy, lddy, D, T));
    if (dsum) LAY_TRY(check_row(dsum, ldds, D, T));
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const size_t wide_bytes = weights_type == SOM_F32 ? 4 : 2;
    if (T == 0) {
        if (dweight) SOM_CK(l, cudaMemsetAsync(dweight, 0, D * wide_bytes, st));
        if (dbias) SOM_CK(l, cudaMemsetAsync(dbias, 0, D * wide_bytes, st));
        return SOM_OK;
    }
    const bool columns = dweight || dbias;
    int64_t parts = 4 * (int64_t)l->sm_count / tiles_of(D, 32);
    if (parts > T / 64) parts = T / 64;
    if (parts < 1) parts = 1;
    Carver c{nullptr, 0};
    c.take<float>(2 * T);
    c.take<float>(parts * 2 * D);
    if (columns) LAY_TRY(ensure(l, c.used));
    c = Carver{static_cast<unsigned char*>(l->ws), 0};
    float* stats = columns ? c.take<float>(2 * T) : nullptr;
    float* part = columns ? c.take<float>(parts * 2 * D) : nullptr;
    const NormBackArgs a = {x, weight, dy, dsum, dx, stats, ldx, lddy, ldds, T, (int)D, eps};
    const ColumnArgs b = {x, dy, stats, part, ldx, lddy, T, (int)D, (int)parts};
    const ColumnJoinArgs j = {part, dweight, dbias, (int)D, (int)parts};
    return outcome(l, by_types(type, weights_type, [&](auto e, auto w) {
                       using E = decltype(e);
                       using W = decltype(w);
                       cudaError_t r = launch(l, k_norm_back_any<E, W>, dim3((unsigned)T), ROW_THREADS, 0, st, 1, a);
                       if (r != cudaSuccess || !columns) return r;
                       r = launch(l, k_norm_columns<E>, dim3((unsigned)tiles_of(D, 32), (unsigned)parts), 256, 0, st, 1, b);
                       if (r != cudaSuccess) return r;
                       return launch(l, k_norm_join<W>, dim3((unsigned)tiles_of(2 * D, 32)), 256, 0, st, 1, j);
                   }));
}

}  // extern "C"
