// som_route and som_route_backward: one warp a token, the row's logits in registers.  Lane l holds the V experts from l * V,
// so that a lane's order and the lanes' order are the experts' order and a tie goes to the lowest lane.
//
// The choice is k rounds of a warp-wide maximum over the keys as order-preserving 32-bit integers: one integer warp
// reduction, one ballot, one shuffle a round; the lane that gave the maximum looks for its next one.
//
// Where the choice goes by scores (not by the logits themselves), it is that of the scores rounded from 64 bits, so that it
// does not hang on the last bits of one exponential.  Computing every score in fp64 took 61 us for 16384 tokens of 256
// experts, four fifths of it fp64 arithmetic.  So the scores are first computed in fp32, off by less than 2^-19, and the
// rounds also look at the gaps between consecutive choices (the first one not taken among them) and between the last group
// kept and the first one dropped: a gap beyond twice the errors cannot change sign.  Only a token with a smaller gap, about
// one in a hundred, goes through the fp64 scores.
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

// the rare path's arithmetic, out of line: unrolled into the kernel it would take the registers of the common path
__device__ __noinline__ double exp64(float x, float top) { return x == top ? 1.0 : exp((double)x - (double)top); }
__device__ __noinline__ float sigmoid64(float x) { return (float)(1.0 / (1.0 + exp(-(double)x))); }

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

// The V logits from `at` on (-inf beyond the row's end); `whole`: rows and their pieces lie on the vector loads' grid.
template <int TYPE, int V>
__device__ __forceinline__ void load_row(const void* p, int64_t row, int at, int E, bool whole, float (&x)[V])
{
    constexpr int SIZE = TYPE == SOM_F32 ? 4 : 2, WORDS = V * SIZE / 4;
    if (WORDS >= 1 && whole && at + V <= E) {
        uint32_t w[WORDS ? WORDS : 1];
        const char* q = static_cast<const char*>(p) + (row + at) * SIZE;
        if (WORDS >= 4) {
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) {
                const uint4 u = __ldg(reinterpret_cast<const uint4*>(q) + i);
                w[4 * i] = u.x, w[4 * i + 1] = u.y, w[4 * i + 2] = u.z, w[4 * i + 3] = u.w;
            }
        } else if (WORDS == 2) {
            const uint2 u = __ldg(reinterpret_cast<const uint2*>(q));
            w[0] = u.x, w[WORDS > 1 ? 1 : 0] = u.y;
        } else {
            w[0] = __ldg(reinterpret_cast<const uint32_t*>(q));
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (SIZE == 4) {
                x[v] = __uint_as_float(w[v]);
            } else {
                const float2 f = unpack2(w[v / 2], TYPE == SOM_BF16);
                x[v] = v & 1 ? f.y : f.x;
            }
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = at + v < E ? logit_at<TYPE>(p, row + at + v) : -INFINITY;
    }
}

// whether load_row may use vector loads on this matrix
template <int TYPE, int V>
__device__ __forceinline__ bool whole_rows(const void* p, int64_t ld)
{
    constexpr int SIZE = TYPE == SOM_F32 ? 4 : 2, BYTES = V * SIZE < 16 ? V * SIZE : 16;
    return (reinterpret_cast<uintptr_t>(p) % BYTES) == 0 && (ld * SIZE) % BYTES == 0;
}

// the two largest keys of (m1 >= m2) and (o1 >= o2)
__device__ __forceinline__ void merge2(uint32_t& m1, uint32_t& m2, uint32_t o1, uint32_t o2)
{
    m2 = max(min(m1, o1), max(m2, o2));
    m1 = max(m1, o1);
}

__device__ __forceinline__ uint32_t group_key(uint32_t b1, uint32_t b2, int best)
{
    if (best == 1 || b2 == 0) return b1;
    const float s = from_ordered(b1) + from_ordered(b2);
    return s == s ? som_ordered_bits(s + 0.f) : 0u;
}

// Whether two keys from fp32 scores may be ordered otherwise by the exact ones; `errors`: scores in each of them.
__device__ __forceinline__ bool too_near(uint32_t above, uint32_t below, int errors)
{
    if (above == 0 || below == 0) return false;  // nothing left below: no order to mistake
    const float f = from_ordered(above), g = from_ordered(below);
    return !(f - g > errors * 0x1p-18f * (1.f + fabsf(f)));
}

template <int TYPE, int V>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) k_route(const RouteArgs a)
{
    extern __shared__ int hist[];  // [E] when counts are wanted
    const int lane = threadIdx.x & 31, first = lane * V;
    if (a.counts) {
        for (int i = threadIdx.x; i < a.E; i += 32 * ROUTE_WARPS) hist[i] = 0;
        __syncthreads();
    }
    const bool whole = whole_rows<TYPE, V>(a.logits, a.ld);
    const bool by_groups = a.groups > 1 && a.top_groups < a.groups;
    const bool by_score = a.bias || (a.groups > 1 && a.group_best == 2);
    const int size = a.E / a.groups;
    const int lanes = size % V == 0 ? size / V : 0;  // lanes of a group, where no lane spans two
    const int my_group = lanes ? lane / lanes : 0, my_place = lanes ? lane - my_group * lanes : 0;
    float bias[V];
#pragma unroll
    for (int v = 0; v < V; ++v) bias[v] = a.bias && first + v < a.E ? __ldg(a.bias + first + v) : 0.f;

    for (int64_t t = (int64_t)blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5); t < a.T; t += (int64_t)gridDim.x * ROUTE_WARPS) {
        const int64_t row = t * a.ld;
        float x[V];
        load_row<TYPE, V>(a.logits, row, first, a.E, whole, x);
        uint32_t top_u = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) top_u = max(top_u, x[v] > -INFINITY ? som_ordered_bits(x[v]) : 0u);  // (a NaN is not)
        top_u = __reduce_max_sync(ALL, top_u);
        const float top = top_u ? from_ordered(top_u) : 0.f;
        float total = 1.f;  // softmax: sum of exp(x - top)
        if (a.score == SOM_SCORE_SOFTMAX && (by_score || !a.renorm)) {
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) sum += x[v] > -INFINITY ? exp_from(x[v], top) : 0.f;
            total = warp_sum(sum);
        }
        int at;  // lane j: the j-th choice
#pragma unroll 1
        for (int exact = 0;; exact = 1) {
            uint32_t key[V];  // 0 = masked out or taken
            if (!by_score) {
#pragma unroll
                for (int v = 0; v < V; ++v) key[v] = x[v] > -INFINITY ? som_ordered_bits(x[v] + 0.f) : 0u;  // + 0: the two zeros tie
            } else {
                double sum = 1.0;
                if (exact && a.score == SOM_SCORE_SOFTMAX) {
                    sum = 0.0;
#pragma unroll
                    for (int v = 0; v < V; ++v) sum += x[v] > -INFINITY ? exp64(x[v], top) : 0.0;
                    sum = warp_sum(sum);
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float s;
                    if (a.score == SOM_SCORE_SOFTMAX) s = exact ? (float)(exp64(x[v], top) / sum) : __fdividef(exp_from(x[v], top), total);
                    else s = exact ? sigmoid64(x[v]) : __fdividef(1.f, 1.f + __expf(-x[v]));
                    s += bias[v];
                    key[v] = x[v] > -INFINITY && s == s ? som_ordered_bits(s + 0.f) : 0u;
                }
            }
            bool unsure = false;
            if (by_groups) {
                uint32_t mine = 0;  // lane g: key of group g
                if (lanes) {
                    uint32_t m1 = 0, m2 = 0;
#pragma unroll
                    for (int v = 0; v < V; ++v) merge2(m1, m2, key[v], 0u);
                    for (int d = 1; d < lanes; d <<= 1) {
                        const uint32_t o1 = __shfl_down_sync(ALL, m1, d), o2 = __shfl_down_sync(ALL, m2, d);
                        if (my_place + d < lanes) merge2(m1, m2, o1, o2);
                    }
                    m1 = group_key(m1, m2, a.group_best);
                    mine = __shfl_sync(ALL, m1, lane * lanes & 31);
                    if (lane >= a.groups) mine = 0;
                } else {
                    for (int g = 0; g < a.groups; ++g) {
                        uint32_t m1 = 0, m2 = 0;
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            const int i = first + v - g * size;
                            if (i >= 0 && i < size) merge2(m1, m2, key[v], 0u);
                        }
                        const uint32_t b1 = __reduce_max_sync(ALL, m1);
                        const int owner = __ffs(__ballot_sync(ALL, m1 == b1)) - 1;
                        const uint32_t b2 = __reduce_max_sync(ALL, lane == owner ? m2 : m1);
                        if (lane == g) mine = group_key(b1, b2, a.group_best);
                    }
                }
                int rank = 0;
                for (int g = 0; g < a.groups; ++g) {
                    const uint32_t other = __shfl_sync(ALL, mine, g);
                    rank += other > mine || (other == mine && g < lane);
                }
                const bool keep = lane < a.groups && rank < a.top_groups;
                const unsigned kept = __ballot_sync(ALL, keep);
                if (by_score && !exact) {
                    const uint32_t low = __reduce_min_sync(ALL, keep ? mine : 0xffffffffu);
                    const uint32_t next = __reduce_max_sync(ALL, !keep && lane < a.groups ? mine : 0u);
                    unsure = too_near(low, next, 2);
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int g = lanes ? my_group : min((first + v) / size, 31);
                    if (!((kept >> g) & 1u)) key[v] = 0u;
                }
            }
            at = -1;
            uint32_t best = 0, last = 0;
            int bv = 0;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (key[v] > best) best = key[v], bv = v;
            const int rounds = by_score && !exact && a.k < a.E ? a.k + 1 : a.k;  // (the first one not taken is looked at)
            for (int j = 0; j < rounds && !unsure; ++j) {
                const uint32_t m = __reduce_max_sync(ALL, best);
                if (m == 0) break;
                if (by_score && !exact && j > 0 && too_near(last, m, 1)) unsure = true;
                last = m;
                const int owner = __ffs(__ballot_sync(ALL, best == m)) - 1;
                const int i = owner * V + __shfl_sync(ALL, bv, owner);
                if (lane == j && j < a.k) at = i;
                if (lane == owner) {
                    const int gone = bv;
                    best = 0;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (v == gone) key[v] = 0u;
                        if (key[v] > best) best = key[v], bv = v;
                    }
                }
            }
            if (!unsure) break;
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
