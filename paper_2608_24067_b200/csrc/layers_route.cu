// som_route and som_route_backward: one warp a token, the row's logits in registers (lane l holds experts l, l + 32, ...).
//
// The choice is k rounds of a warp-wide maximum of (key, lowest index): the keys as order-preserving 32-bit integers, so
// that a round is two integer warp reductions.  Scores that the choice goes by are computed in fp64 and rounded to fp32
// (an expert's rank then does not depend on the last bits of one exponential); where the logits order the experts
// themselves only the chosen experts' scores are computed, in fp32.
#include "layers_math.cuh"
#include "layers_slots.cuh"

namespace lay {
namespace {

constexpr unsigned ALL = 0xffffffffu;
constexpr int ROUTE_WARPS = 8;

template <int TYPE>
__device__ __forceinline__ float logit_at(const void* p, int64_t i)
{
    if (TYPE == SOM_F32) return __ldg(static_cast<const float*>(p) + i);
    return unpack1(__ldg(static_cast<const uint16_t*>(p) + i), TYPE == SOM_BF16);
}

__device__ __forceinline__ float from_ordered(uint32_t u)
{
    return __uint_as_float((u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(ALL, v, d);
    return v;
}

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(ALL, v, d);
    return v;
}

// exp(x - top), with the limit 1 where both are infinite
__device__ __forceinline__ float exp_from(float x, float top) { return x == top ? 1.f : expf(x - top); }

struct RouteArgs {
    const void* logits;
    int64_t ld, T;
    const float* bias;
    float* weights;
    int32_t* indices;
    int32_t* counts;
    int E, k, score, groups, top_groups, group_best, renorm;
    float scale;
};

template <int TYPE, int V>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) k_route(const RouteArgs a)
{
    extern __shared__ int hist[];  // [E] when counts are wanted
    const int lane = threadIdx.x & 31;
    if (a.counts) {
        for (int i = threadIdx.x; i < a.E; i += 32 * ROUTE_WARPS) hist[i] = 0;
        __syncthreads();
    }
    const bool by_score = a.bias || (a.groups > 1 && a.group_best == 2);
    for (int64_t t = (int64_t)blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5); t < a.T; t += (int64_t)gridDim.x * ROUTE_WARPS) {
        const int64_t row = t * a.ld;
        float x[V];
        uint32_t key[V];  // 0 = masked out or taken
        uint32_t top_u = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = v * 32 + lane;
            x[v] = i < a.E ? logit_at<TYPE>(a.logits, row + i) : -INFINITY;
            const bool live = x[v] > -INFINITY;  // (false for NaN)
            key[v] = live ? som_ordered_bits(x[v] + 0.f) : 0u;  // + 0: the two zeros tie
            top_u = max(top_u, key[v]);
        }
        top_u = __reduce_max_sync(ALL, top_u);
        const float top = top_u ? from_ordered(top_u) : 0.f;
        float total = 1.f;  // softmax: sum of exp(x - top)
        if (by_score) {
            double e[V], sum = 0.0;
            if (a.score == SOM_SCORE_SOFTMAX) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    e[v] = key[v] ? (x[v] == top ? 1.0 : exp((double)x[v] - (double)top)) : 0.0;
                    sum += e[v];
                }
                sum = warp_sum(sum);
                total = (float)sum;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!key[v]) continue;
                float s = a.score == SOM_SCORE_SOFTMAX ? (float)(e[v] / sum) : (float)(1.0 / (1.0 + exp(-(double)x[v])));
                if (a.bias) s += __ldg(a.bias + v * 32 + lane);
                key[v] = s == s ? som_ordered_bits(s + 0.f) : 0u;
            }
        } else if (a.score == SOM_SCORE_SOFTMAX && !a.renorm) {
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) sum += key[v] ? exp_from(x[v], top) : 0.f;
            total = warp_sum(sum);
        }
        if (a.groups > 1 && a.top_groups < a.groups) {
            const int size = a.E / a.groups;
            uint32_t mine = 0;  // lane g: key of group g
            for (int g = 0; g < a.groups; ++g) {
                uint32_t m1 = 0, m2 = 0;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int i = v * 32 + lane - g * size;
                    if (i >= 0 && i < size) {
                        m2 = max(m2, min(m1, key[v]));
                        m1 = max(m1, key[v]);
                    }
                }
                const uint32_t b1 = __reduce_max_sync(ALL, m1);
                uint32_t gk = b1;
                if (a.group_best == 2 && b1) {
                    const int owner = __ffs(__ballot_sync(ALL, m1 == b1)) - 1;
                    const uint32_t b2 = __reduce_max_sync(ALL, lane == owner ? m2 : m1);
                    if (b2) {
                        const float s = from_ordered(b1) + from_ordered(b2);
                        gk = s == s ? som_ordered_bits(s + 0.f) : 0u;
                    }
                }
                if (lane == g) mine = gk;
            }
            int rank = 0;
            for (int g = 0; g < a.groups; ++g) {
                const uint32_t other = __shfl_sync(ALL, mine, g);
                rank += other > mine || (other == mine && g < lane);
            }
            const unsigned kept = __ballot_sync(ALL, lane < a.groups && rank < a.top_groups);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int i = v * 32 + lane;
                if (i < a.E && !((kept >> (i / size)) & 1u)) key[v] = 0u;
            }
        }
        int at = -1;  // lane j: the j-th choice
        for (int j = 0; j < a.k; ++j) {
            uint32_t best = 0;
            int bi = 0x7fffffff;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (key[v] > best) {
                    best = key[v];
                    bi = v * 32 + lane;
                }
            const uint32_t m = __reduce_max_sync(ALL, best);
            if (m == 0) break;
            const int i = (int)__reduce_min_sync(ALL, (unsigned)(best == m ? bi : 0x7fffffff));
            if (lane == j) at = i;
            if ((i & 31) == lane) {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (v == (i >> 5)) key[v] = 0u;
            }
        }
        float s = 0.f;
        const float xj = at >= 0 ? logit_at<TYPE>(a.logits, row + at) : -INFINITY;
        if (a.score == SOM_SCORE_SIGMOID) {
            if (at >= 0) s = 1.f / (1.f + expf(-xj));
        } else if (a.renorm) {
            // only ratios of the chosen experts' scores count: taken from the largest of them
            float m = xj;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(ALL, m, d));
            if (at >= 0 && (m == top || top < INFINITY)) s = exp_from(xj, m);  // (beside an infinite logit all others score 0)
        } else if (at >= 0) {
            s = exp_from(xj, top) / total;
        }
        if (a.renorm) {
            const float sum = warp_sum(s);
            s = sum > 0.f ? s / sum : 0.f;
        }
        if (lane < a.k) {
            a.weights[t * a.k + lane] = s * a.scale;
            a.indices[t * a.k + lane] = at;
            if (a.counts && at >= 0) atomicAdd(&hist[at], 1);
        }
    }
    if (a.counts) {
        __syncthreads();
        for (int i = threadIdx.x; i < a.E; i += 32 * ROUTE_WARPS) {
            if (gridDim.x == 1) a.counts[i] = hist[i];
            else if (hist[i]) atomicAdd(&a.counts[i], hist[i]);
        }
    }
}

struct RouteGradArgs {
    const void* logits;
    int64_t ld, T;
    const int32_t* indices;
    const float* dweights;
    void* dlogits;
    int E, k, score, renorm;
    float scale;
    int* flags;
};

template <int TYPE>
__device__ __forceinline__ void put_logit(void* p, int64_t i, float v)
{
    if (TYPE == SOM_F32) static_cast<float*>(p)[i] = v;
    else static_cast<uint16_t*>(p)[i] = (uint16_t)pack2(v, 0.f, TYPE == SOM_BF16);
}

// Lane j holds choice j.  The row is written as if nothing had been chosen, then the chosen elements are written over it.
template <int TYPE, int V>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) k_route_backward(const RouteGradArgs a)
{
    const int lane = threadIdx.x & 31;
    for (int64_t t = (int64_t)blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5); t < a.T; t += (int64_t)gridDim.x * ROUTE_WARPS) {
        const int64_t row = t * a.ld, out = t * a.E;
        int at = lane < a.k ? a.indices[t * a.k + lane] : -1;
        const bool bad = at < -1 || at >= a.E;
        som_raise(a.flags, bad, LAY_FLAG_BAD_EXPERT);
        if (bad) at = -1;
        const float d = at >= 0 ? a.dweights[t * a.k + lane] * a.scale : 0.f;
        const float xj = at >= 0 ? logit_at<TYPE>(a.logits, row + at) : -INFINITY;
        const bool live = xj > -INFINITY;
        float g;  // the chosen element's gradient
        if (a.score == SOM_SCORE_SOFTMAX && !a.renorm) {
            float x[V], top = -INFINITY;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int i = v * 32 + lane;
                x[v] = i < a.E ? logit_at<TYPE>(a.logits, row + i) : -INFINITY;
                top = fmaxf(top, x[v]);  // (a NaN is left out)
            }
#pragma unroll
            for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(ALL, top, m));
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                x[v] = x[v] > -INFINITY ? exp_from(x[v], top) : 0.f;
                sum += x[v];
            }
            sum = warp_sum(sum);
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
            const float p = live ? exp_from(xj, top) * inv : 0.f;
            const float dot = warp_sum(live ? p * d : 0.f);
            g = 0.f;
            for (int j = 0; j < a.k; ++j) {  // an expert named twice gets both
                const int o = __shfl_sync(ALL, at, j);
                const float od = __shfl_sync(ALL, d, j);
                if (o == at) g += od;
            }
            g = p * (g - dot);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int i = v * 32 + lane;
                if (i < a.E) put_logit<TYPE>(a.dlogits, out + i, x[v] > 0.f ? -(x[v] * inv) * dot : 0.f);
            }
        } else {
            float q = 0.f, top = 0.f;
            if (a.score == SOM_SCORE_SOFTMAX) {
                top = xj;
#pragma unroll
                for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(ALL, top, m));
                if (live) q = exp_from(xj, top);
            } else if (live) {
                q = 1.f / (1.f + expf(-xj));
            }
            float e = d;
            if (a.renorm) {
                const float sum = warp_sum(q), inv = sum > 0.f ? 1.f / sum : 0.f;
                const float mean = warp_sum(live ? d * q : 0.f) * inv;
                e = (d - mean) * inv;
            }
            // softmax with renormalisation: the mean over all experts of the scores' gradient is zero
            e = live ? (a.score == SOM_SCORE_SOFTMAX ? q * e : q * (1.f / (1.f + expf(xj))) * e) : 0.f;
            g = 0.f;
            for (int j = 0; j < a.k; ++j) {
                const int o = __shfl_sync(ALL, at, j);
                const float oe = __shfl_sync(ALL, e, j);
                if (o == at) g += oe;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int i = v * 32 + lane;
                if (i < a.E) put_logit<TYPE>(a.dlogits, out + i, 0.f);
            }
        }
        __syncwarp();
        if (at >= 0) put_logit<TYPE>(a.dlogits, out + at, live ? g : 0.f);
    }
}

int done(som_layers* l, cudaError_t e)
{
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess) return SOM_OK;
    l->last_cuda_error = (int)e;
    return SOM_ERR_CUDA;
}

// the warp's registers for a row: the smallest power of two of 32 experts that holds it
template <template <int, int> class K, int TYPE, class A>
cudaError_t by_size(int E, const A& a, int grid, size_t smem, cudaStream_t st)
{
    if (E <= 32) return K<TYPE, 1>::go(a, grid, smem, st);
    if (E <= 64) return K<TYPE, 2>::go(a, grid, smem, st);
    if (E <= 128) return K<TYPE, 4>::go(a, grid, smem, st);
    if (E <= 256) return K<TYPE, 8>::go(a, grid, smem, st);
    if (E <= 512) return K<TYPE, 16>::go(a, grid, smem, st);
    return K<TYPE, 32>::go(a, grid, smem, st);
}

template <template <int, int> class K, class A>
cudaError_t by_type(int type, int E, const A& a, int grid, size_t smem, cudaStream_t st)
{
    if (type == SOM_F32) return by_size<K, SOM_F32>(E, a, grid, smem, st);
    if (type == SOM_F16) return by_size<K, SOM_F16>(E, a, grid, smem, st);
    return by_size<K, SOM_BF16>(E, a, grid, smem, st);
}

template <int TYPE, int V>
struct Route {
    static cudaError_t go(const RouteArgs& a, int grid, size_t smem, cudaStream_t st)
    {
        k_route<TYPE, V><<<grid, 32 * ROUTE_WARPS, smem, st>>>(a);
        return cudaGetLastError();
    }
};

template <int TYPE, int V>
struct RouteGrad {
    static cudaError_t go(const RouteGradArgs& a, int grid, size_t smem, cudaStream_t st)
    {
        k_route_backward<TYPE, V><<<grid, 32 * ROUTE_WARPS, smem, st>>>(a);
        return cudaGetLastError();
    }
};

int route_grid(const som_layers* l, int64_t T)
{
    const int64_t want = (T + ROUTE_WARPS - 1) / ROUTE_WARPS, most = (int64_t)l->sm_count * 8;
    return (int)(want < most ? want : most);
}

}  // namespace

int launch_route(som_layers* l, int type, int score, int64_t T, int E, int k, const void* logits, int64_t ld, const float* bias,
                 int groups, int top_groups, int group_best, int renorm, float scale, float* weights, int32_t* indices,
                 int32_t* counts, cudaStream_t st)
{
    const int grid = T > 0 ? route_grid(l, T) : 0;
    cudaError_t e = cudaSuccess;
    if (counts && grid != 1) e = cudaMemsetAsync(counts, 0, (size_t)E * sizeof(int32_t), st);  // one block writes its counts itself
    if (e == cudaSuccess && grid) {
        const RouteArgs a{logits, ld, T, bias, weights, indices, counts, E, k, score, groups, top_groups, group_best, renorm, scale};
        e = by_type<Route>(type, E, a, grid, counts ? (size_t)E * sizeof(int) : 0, st);
        ++l->launches;
    }
    return done(l, e);
}

int launch_route_backward(som_layers* l, int type, int score, int64_t T, int E, int k, const void* logits, int64_t ld,
                          const int32_t* indices, const float* dweights, int renorm, float scale, void* dlogits, cudaStream_t st)
{
    if (T == 0) return SOM_OK;
    const RouteGradArgs a{logits, ld, T, indices, dweights, dlogits, E, k, score, renorm, scale, l->flags};
    const cudaError_t e = by_type<RouteGrad>(type, E, a, route_grid(l, T), 0, st);
    ++l->launches;
    return done(l, e);
}

}  // namespace lay
