// Products with few output tiles and a long sum (a few dozen tokens, a narrow output) keep most SMs idle while the others walk
// the sum; so the sum is split over blocks, which leave fp32 parts, and this kernel adds the parts in their order and applies
// what the product's epilogue would have.  A thread takes eight columns of a row.  Bound by its launch (about 3 us).
#include "layers_finish.cuh"
#include "layers_math.cuh"

namespace lay {
namespace {

__device__ __forceinline__ void add_parts(const float* p, int64_t stride, int splits, float (&v)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float4 a = *reinterpret_cast<const float4*>(p + s * stride), b = *reinterpret_cast<const float4*>(p + s * stride + 4);
        v[0] += a.x, v[1] += a.y, v[2] += a.z, v[3] += a.w;
        v[4] += b.x, v[5] += b.y, v[6] += b.z, v[7] += b.w;
    }
}

__device__ __forceinline__ void store8(uint16_t* to, const float (&v)[8], int bf16)
{
    *reinterpret_cast<uint4*>(to) = make_uint4(pack2(v[0], v[1], bf16), pack2(v[2], v[3], bf16), pack2(v[4], v[5], bf16), pack2(v[6], v[7], bf16));
}

__global__ void __launch_bounds__(256) k_finish(const FinishArgs a)
{
    enter();
    const int chunks = a.cols / 8;
    const int64_t stride = a.rows * a.n;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < a.rows * chunks; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t row = i / chunks;
        const int col = (int)(i - row * chunks) * 8;
        float v[8], u[8];
        add_parts(a.part + row * a.n + col, stride, a.splits, v);
        if (a.gated) add_parts(a.part + row * a.n + a.cols + col, stride, a.splits, u);
        if (a.bias) {
            float b[8];
            load8(a.bias + col, b, a.bf16);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += b[j];
            if (a.gated) {
                load8(a.bias + a.cols + col, b, a.bf16);
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] += b[j];
            }
        }
        if (a.mode == FINISH_FWD) {
            with_act(a.act, [&](auto tag) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = act_of<decltype(tag)::value>(v[j]);
            });
            if (a.gated) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= u[j];
            }
            if (a.extra) {
                float r[8];
                load8(a.extra + row * a.ld_extra + col, r, a.bf16);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += r[j];
            }
        } else if (a.mode == FINISH_DZ) {
            float g[8];
            load8(a.extra + row * a.ld_extra + col, g, a.bf16);
            with_act(a.act, [&](auto tag) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float h, dh;
                    act_both<decltype(tag)::value>(v[j], h, dh);
                    v[j] = a.gated ? g[j] * (dh * u[j]) : g[j] * dh;
                    if (a.gated) u[j] = g[j] * h;
                }
            });
            if (a.gated) store8(a.out + row * a.ld + a.cols + col, u, a.bf16);
        }
        // (FINISH_DZ: dz in 16 bits, as the next products' operand; see the products' own epilogue)
        store8(a.out + row * a.ld + col, v, a.bf16);
    }
}

}  // namespace

int launch_finish(som_layers* l, const FinishArgs& a, cudaStream_t st)
{
    const int64_t want = (a.rows * (a.cols / 8) + 255) / 256, most = (int64_t)l->sm_count * 8;
    return outcome(l, launch(l, k_finish, dim3((unsigned)(want < most ? want : most)), 256, 0, st, 1, a));
}

}  // namespace lay
