// som_route and som_route_backward: one warp a token, the row's logits in registers.  Lane l holds the V experts from l * V,
// so that a lane's order and the lanes' order are the experts' order.
//
// The choice takes k rounds of a warp-wide maximum.  What bounds it is instructions, not bytes (16384 tokens x 256 experts
// are 17 MB, 2.6 us), so a round has to be short.  A key and its expert are packed into 32 bits, 22 of key and 10 of index,
// so that one integer reduction finds the winner with ties to the lowest index; each lane's keys are sorted beforehand
// (minima and maxima only), so that the winner's lane just moves up its list.  16-bit logits fit such a key exactly.  Others
// become fixed-point distances from an upper bound, and scores come from fast fp32 exponentials; so the gaps between
// consecutive choices (the first one not taken among them) and between the last group kept and the first dropped are
// compared with the errors of both keys.  Where a gap is smaller, the contested groups or places are settled from the exact keys
// of those that contest them (of all experts where that is not enough): logits as order-preserving integers, scores in fp64
// rounded to fp32, so that the choice does not hang on the last bits of one exponential.  2048 tokens x 256 experts with bias
// and groups: 12.3 us; 20.5 us where a small gap sends the whole token to the exact keys; 16384 tokens: 61 us with every score
// in fp64.
#include "layers_math.cuh"
#include "layers_slots.cuh"

namespace lay {
namespace {

constexpr unsigned ALL = 0xffffffffu;
constexpr int ROUTE_WARPS = 8;

template <int TYPE>
__device__ __forceinline__ float logit_at(const void* p, int64_t i)
{
    if (TYPE == SOM_F32) return static_cast<const float*>(p)[i];
    return unpack1(static_cast<const uint16_t*>(p)[i], TYPE == SOM_BF16);
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


// Where scores are renormalised only the chosen ones' ratios count, also where the scores themselves are below fp32's range; but
// scores that are 0 in 64 bits as well (a logit of the type's lowest value as a mask, chosen for its bias) weigh 0: those below
// exp(NO_SCORE), against the row's largest logit for the softmax.
constexpr float NO_SCORE = -700.f;
__device__ __forceinline__ bool scores_at(float most, float top) { return most == top || most > top + NO_SCORE; }

// sigmoid(x) as a multiple of exp(most), most <= 0 the largest chosen logit or 0; needed from LOW_LOGIT down
constexpr float LOW_LOGIT = -80.f;
__device__ __forceinline__ float sigmoid_from(float x, float most)
{
    return most < NO_SCORE ? 0.f : expf(fminf(x, 0.f) - most) / (1.f + expf(-fabsf(x)));
}

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(ALL, v, d));
    return v;
}

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
                const uint4 u = *(reinterpret_cast<const uint4*>(q) + i);
                w[4 * i] = u.x, w[4 * i + 1] = u.y, w[4 * i + 2] = u.z, w[4 * i + 3] = u.w;
            }
        } else if (WORDS == 2) {
            const uint2 u = *(reinterpret_cast<const uint2*>(q));
            w[0] = u.x, w[WORDS > 1 ? 1 : 0] = u.y;
        } else {
            w[0] = *(reinterpret_cast<const uint32_t*>(q));
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

// The choice from exact keys: lane j returns the j-th.  Rare, so what it costs is fetching its code: loops, nothing unrolled,
// the keys in local memory.  (Unrolled, it added 17 us to 20 us for 16384 tokens of which one in a hundred came here.)
template <int TYPE>
__device__ __noinline__ int choose_exact(const RouteArgs& a, int64_t row, float top, bool by_score, bool by_groups, int lane)
{
    const int n = (a.E + 31) / 32, first = lane * n;
    uint32_t key[32];  // 0 = masked out or taken
    double sum = 1.0;
#pragma unroll 1
    for (int pass = by_score && a.score == SOM_SCORE_SOFTMAX ? 0 : 1; pass < 2; ++pass) {  // the scores' sum, the keys
        if (pass == 0) sum = 0.0;
#pragma unroll 1
        for (int v = 0; v < n; ++v) {
            const float x = first + v < a.E ? logit_at<TYPE>(a.logits, row + first + v) : -INFINITY;
            const bool live = x > -INFINITY;
            float s = x;
            if (by_score) {
                const bool soft = a.score == SOM_SCORE_SOFTMAX;
                const double e = soft && x == top ? 1.0 : exp(soft ? (double)x - (double)top : -(double)x);
                if (pass == 0) {
                    if (live) sum += e;
                    continue;
                }
                s = (float)((soft ? e : 1.0) / (soft ? sum : 1.0 + e));
                if (a.bias && first + v < a.E) s += *(a.bias + first + v);
            }
            key[v] = live && s > -INFINITY ? som_ordered_bits(s + 0.f) : 0u;  // + 0: the two zeros tie
        }
        if (pass == 0) sum = warp_sum(sum);
    }
    if (by_groups) {
        const int size = a.E / a.groups;
        uint32_t mine = 0;  // lane g: key of group g
#pragma unroll 1
        for (int g = 0; g < a.groups; ++g) {
            uint32_t m1 = 0, m2 = 0;
#pragma unroll 1
            for (int v = max(0, g * size - first); v < min(n, (g + 1) * size - first); ++v) merge2(m1, m2, key[v], 0u);
            const uint32_t b1 = __reduce_max_sync(ALL, m1);
            const int owner = __ffs(__ballot_sync(ALL, m1 == b1)) - 1;
            const uint32_t b2 = __reduce_max_sync(ALL, lane == owner ? m2 : m1);
            if (lane == g) mine = group_key(b1, b2, a.group_best);
        }
        int rank = 0;
#pragma unroll 1
        for (int g = 0; g < a.groups; ++g) {
            const uint32_t other = __shfl_sync(ALL, mine, g);
            rank += other > mine || (other == mine && g < lane);
        }
        const unsigned kept = __ballot_sync(ALL, lane < a.groups && rank < a.top_groups);
#pragma unroll 1
        for (int v = 0; v < n; ++v)
            if (!((kept >> min((first + v) / size, 31)) & 1u)) key[v] = 0u;
    }
    int at = -1;
#pragma unroll 1
    for (int j = 0; j < a.k; ++j) {
        uint32_t best = 0;
        int bv = 0;
#pragma unroll 1
        for (int v = 0; v < n; ++v)
            if (key[v] > best) best = key[v], bv = v;
        const uint32_t m = __reduce_max_sync(ALL, best);
        if (m == 0) break;
        const int owner = __ffs(__ballot_sync(ALL, best == m)) - 1;  // the lowest lane holds the lowest index
        const int i = owner * n + __shfl_sync(ALL, bv, owner);
        if (lane == j) at = i;
        if (lane == owner) key[bv] = 0u;
    }
    return at;
}

// Errors of two fp32 keys together, per unit of 1 + |bias|.  Sigmoid: 2^-22 of the exponential times s (1 - s), 2^-22.5 of the
// division, 2^-24 each for the bias and for the exact key's own two roundings: below 2^-21 a key.  Softmax: the sum of up
// to 1024 exponentials (37 additions in a row at most) and the exponential are off by 2^-18.5 of a score, and the scores of two
// experts are at most 1 together.
__device__ __forceinline__ float key_errors(int score) { return score == SOM_SCORE_SOFTMAX ? 0x1p-18f : 0x1p-20f; }

constexpr int KEY_BITS = 22, INDEX_BITS = 10;
constexpr uint32_t KEY_MOST = (1u << KEY_BITS) - 1u, INDEX_MASK = (1u << INDEX_BITS) - 1u;

// How scores and biases are packed.  Keys lie between the lowest bias and 1 + the highest, with 0 among them.  Biases below FAR_BIAS
// (-1e9 switches an expert off) do not count for that range: such an expert's key is the lowest, 1, which no key within the range
// gets, and where the choice, or a kept group's key, would hang on it, exact keys are taken.  (16384 tokens x 256 experts with groups,
// one bias of -1e9: 27 us; 121 where it counts for the range, and so every token takes the exact keys.)
struct Packing {
    float ceiling, scale;
    uint32_t margin;  // key units: rounding of the distances and the scores' errors
    bool fits;        // (not with biases of 2.6e5 and more)
};
constexpr float FAR_BIAS = -64.f;

// from a lane's lowest bias that counts and its highest
__device__ __forceinline__ Packing packing_of(float low, float high, int score)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        high = fmaxf(high, __shfl_xor_sync(ALL, high, d));
        low = fminf(low, __shfl_xor_sync(ALL, low, d));
    }
    Packing p;
    p.ceiling = 1.f + high;
    p.scale = (float)(KEY_MOST - 8u) / (p.ceiling - low);
    p.margin = 3 + (uint32_t)(p.scale * key_errors(score) * fmaxf(p.ceiling, 1.f - low));
    p.fits = p.scale > 16.f;
    return p;
}

// beyond the keys' range
__device__ __forceinline__ bool far_key(uint32_t packed) { return (packed >> INDEX_BITS) <= 1u; }

__device__ __forceinline__ void order2(uint32_t& a, uint32_t& b)
{
    const uint32_t hi = max(a, b), lo = min(a, b);
    a = hi;
    b = lo;
}

// descending: Batcher's odd-even merge sort, unrolled
template <int V>
__device__ __forceinline__ void sort_down(uint32_t (&k)[V])
{
#pragma unroll
    for (int p = 1; p < V; p <<= 1)
#pragma unroll
        for (int q = p; q >= 1; q >>= 1)
#pragma unroll
            for (int j = q % p; j + q < V; j += 2 * q)
#pragma unroll
                for (int i = 0; i < q; ++i)
                    if (i + j + q < V && (i + j) / (2 * p) == (i + j + q) / (2 * p)) order2(k[i + j], k[i + j + q]);
}

// 16-bit logits (exact as floats) as order-preserving 16-bit integers
template <int TYPE>
__device__ __forceinline__ uint32_t ordered16(float x)
{
    uint32_t u;
    if (TYPE == SOM_BF16) {
        u = __float_as_uint(x) >> 16;
    } else {
        const __half h = __float2half_rn(x);
        u = *reinterpret_cast<const uint16_t*>(&h);
    }
    return u & 0x8000u ? ~u & 0xffffu : u | 0x8000u;
}

// The exact key of one expert as an order-preserving integer, where it needs no other expert: a logit, or sigmoid + bias.
template <int TYPE>
__device__ __noinline__ uint32_t exact_key(const RouteArgs& a, int64_t row, int i, bool by_score)
{
    const float x = logit_at<TYPE>(a.logits, row + i);
    float s = x;
    if (by_score) {
        s = (float)(1.0 / (1.0 + exp(-(double)x)));
        if (a.bias) s += a.bias[i];
    }
    return x > -INFINITY && s > -INFINITY ? som_ordered_bits(s + 0.f) : 0u;  // (a bias of -inf or NaN: never chosen)
}

// Which groups are kept, by one warp for one token: lane g holds the key of group g; `low` and `next` are the smallest key
// kept and the largest one dropped, nearer than `margin`.  Groups beyond the margin on either side stay where they are.
template <int TYPE>
__device__ __noinline__ unsigned settle_groups(const RouteArgs& a, int64_t row, uint32_t key, uint32_t low, uint32_t next, uint32_t margin, int lane)
{
    const bool there = lane < a.groups && key;
    const bool above = there && key >= next + margin, open = there && !above && key + margin > low;
    unsigned kept = __ballot_sync(ALL, above), todo = __ballot_sync(ALL, open);
    const int size = a.E / a.groups;
    uint32_t mine = 0;
    for (unsigned left = todo; left; left &= left - 1) {
        const int g = __ffs(left) - 1;
        uint32_t m1 = 0, m2 = 0;
#pragma unroll 1
        for (int i = lane; i < size; i += 32) merge2(m1, m2, exact_key<TYPE>(a, row, g * size + i, true), 0u);
        const uint32_t b1 = __reduce_max_sync(ALL, m1);
        const int owner = __ffs(__ballot_sync(ALL, m1 == b1)) - 1;
        const uint32_t b2 = __reduce_max_sync(ALL, lane == owner ? m2 : m1);
        if (lane == g) mine = group_key(b1, b2, a.group_best);
    }
    for (int n = a.top_groups - __popc(kept); n > 0; --n) {
        const uint32_t m = __reduce_max_sync(ALL, open ? mine : 0u);
        if (m == 0) break;
        const int g = __ffs(__ballot_sync(ALL, open && mine == m)) - 1;
        kept |= 1u << g;
        if (lane == g) mine = 0;
    }
    return kept;
}

// Puts candidates (lanes 0 to n - 1: expert `index`) into the order of their exact keys; returns to lane j the j-th of k, or -1.
template <int TYPE>
__device__ __noinline__ int settle_places(const RouteArgs& a, int64_t row, int index, int n, bool by_score, int lane)
{
    uint32_t key = 0;
    if (lane < n) key = exact_key<TYPE>(a, row, index, by_score);
    __syncwarp();
    int rank = 0;
    for (int i = 0; i < n; ++i) {
        const uint32_t k = __shfl_sync(ALL, key, i);
        const int o = __shfl_sync(ALL, index, i);
        rank += k > key || (k == key && k && o < index);
    }
    int at = -1;
    for (int i = 0; i < a.k && i < n; ++i) {
        const unsigned is = __ballot_sync(ALL, key && rank == i);
        const int v = __shfl_sync(ALL, index, is ? __ffs(is) - 1 : 0);
        if (lane == i && is) at = v;
    }
    return at;
}

template <int TYPE, int V>
__global__ void __launch_bounds__(32 * ROUTE_WARPS, V <= 8 ? 4 : 2) k_route(const RouteArgs a)
{
    enter();
    extern __shared__ int hist[];  // [E] when counts are wanted
    const int lane = threadIdx.x & 31, first = lane * V;
    if (a.counts) {
        for (int i = threadIdx.x; i < a.E; i += 32 * ROUTE_WARPS) hist[i] = 0;
        __syncthreads();
    }
    const bool whole = whole_rows<TYPE, V>(a.logits, a.ld);
    const bool by_groups = a.groups > 1 && a.top_groups < a.groups;
    const bool by_score = a.bias || (a.groups > 1 && a.group_best == 2);
    const bool exact16 = TYPE != SOM_F32 && !by_score;
    int lanes = 0, my_group = 0, my_place = 0;  // lanes of a group, where no lane spans two
    if (by_groups) {
        const int size = a.E / a.groups;
        lanes = size % V == 0 ? size / V : 0;
        my_group = lanes ? lane / lanes : 0;
        my_place = lane - my_group * lanes;
    }
    float bias[V];
    float high = 0.f, low = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        bias[v] = a.bias && first + v < a.E ? *(a.bias + first + v) : 0.f;
        high = fmaxf(high, bias[v]);
        if (bias[v] >= FAR_BIAS) low = fminf(low, bias[v]);
    }
    // packed keys: scores and biases; or logits, of which those up to 64 below the row's largest are told apart
    Packing pack{0.f, (float)KEY_MOST / 64.f, 3, true};
    if (by_score) pack = packing_of(low, high, a.score);
    const float ceiling = pack.ceiling, scale = pack.scale;
    const uint32_t margin = pack.margin;
    const bool packs = (!by_groups || lanes) && a.k < 32 && pack.fits;

    for (int64_t t = (int64_t)blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5); t < a.T; t += (int64_t)gridDim.x * ROUTE_WARPS) {
        const int64_t row = t * a.ld;
        float x[V];
        load_row<TYPE, V>(a.logits, row, first, a.E, whole, x);
        float top = -INFINITY;
#pragma unroll
        for (int v = 0; v < V; ++v) top = fmaxf(top, x[v]);  // (a NaN is left out)
        const uint32_t top_u = __reduce_max_sync(ALL, top > -INFINITY ? som_ordered_bits(top) : 0u);
        top = top_u ? from_ordered(top_u) : 0.f;
        float total = 1.f;  // softmax: sum of exp(x - top)
        if (a.score == SOM_SCORE_SOFTMAX && (by_score || !a.renorm)) {
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) sum += x[v] > -INFINITY ? exp_from(x[v], top) : 0.f;
            total = warp_sum(sum);
        }
        int at = -1;  // lane j: the j-th choice
        bool sure = packs && top < INFINITY;
        if (sure) {
            uint32_t key[V];  // 0 = masked out or taken
            if (exact16) {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    key[v] = x[v] > -INFINITY ? ordered16<TYPE>(x[v] + 0.f) << 16 | (INDEX_MASK - first - v) : 0u;  // + 0: the two zeros tie
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float d;  // distance from the upper bound
                    if (!by_score) d = top - x[v];
                    else if (a.score == SOM_SCORE_SOFTMAX) d = ceiling - (__fdividef(exp_from(x[v], top), total) + bias[v]);
                    else d = ceiling - (__fdividef(1.f, 1.f + __expf(-x[v])) + bias[v]);
                    const uint32_t u = KEY_MOST - min((uint32_t)(d * scale), KEY_MOST - 1u);
                    key[v] = x[v] > -INFINITY && d < INFINITY ? u << INDEX_BITS | (INDEX_MASK - first - v) : 0u;
                }
            }
            if (by_groups) {
                uint32_t m1 = 0, m2 = 0;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    m2 = max(m2, min(m1, key[v]));
                    m1 = max(m1, key[v]);
                }
                for (int d = 1; d < lanes; d <<= 1) {
                    const uint32_t o1 = __shfl_down_sync(ALL, m1, d), o2 = __shfl_down_sync(ALL, m2, d);
                    if (my_place + d < lanes) merge2(m1, m2, o1, o2);
                }
                // a lone expert's distance is not comparable with the sum of two
                if (a.group_best == 2 && __any_sync(ALL, my_place == 0 && m1 && !m2)) sure = false;
                const uint32_t gk = a.group_best == 2 ? (m1 >> INDEX_BITS) + (m2 >> INDEX_BITS) : m1;
                uint32_t mine = __shfl_sync(ALL, gk, lane * lanes & 31);  // lane g: group g
                if (lane >= a.groups) mine = 0;
                const uint32_t all = mine;
                unsigned kept = 0;
                uint32_t last = 0;
                for (int r = 0; r < a.top_groups; ++r) {
                    last = __reduce_max_sync(ALL, mine);
                    if (last == 0) break;
                    const int g = __ffs(__ballot_sync(ALL, mine == last)) - 1;
                    kept |= 1u << g;
                    if (lane == g) mine = 0;
                }
                // (with the lowest key in it, a sum is an upper bound of the group's key: enough for a group that is not kept)
                if (a.group_best == 2 && __any_sync(ALL, my_place == 0 && ((kept >> my_group) & 1u) && far_key(m2))) sure = false;
                const uint32_t next = last ? __reduce_max_sync(ALL, mine) : 0u;
                if (!exact16 && next && sure) {
                    const int shift = a.group_best == 2 ? 0 : INDEX_BITS;
                    const uint32_t apart = a.group_best == 2 ? 2 * margin : margin;
                    if ((last >> shift) - (next >> shift) < apart) {
                        if (by_score && a.score == SOM_SCORE_SIGMOID) kept = settle_groups<TYPE>(a, row, all >> shift, last >> shift, next >> shift, apart, lane);
                        else sure = false;
                    }
                }
                if (!((kept >> my_group) & 1u)) {
#pragma unroll
                    for (int v = 0; v < V; ++v) key[v] = 0u;
                }
            }
            if (sure) {
                sort_down<V>(key);
                uint32_t won = 0;
                const int rounds = exact16 ? a.k : a.k + 1;  // (the first one not taken is looked at)
                for (int j = 0; j < rounds; ++j) {
                    const uint32_t m = __reduce_max_sync(ALL, key[0]);
                    if (m == 0) break;
                    if (lane == j) won = m;
                    if (key[0] == m) {
#pragma unroll
                        for (int v = 0; v + 1 < V; ++v) key[v] = key[v + 1];
                        key[V - 1] = 0u;
                    }
                }
                at = won ? (int)(INDEX_MASK - (won & INDEX_MASK)) : -1;
                if (!exact16) {
                    if (__any_sync(ALL, won && lane < a.k && far_key(won))) sure = false;
                    uint32_t above = __shfl_up_sync(ALL, won, 1);
                    // contested places: lane j's winner and the one above it
                    unsigned near = __ballot_sync(ALL, won && lane > 0 && (above >> INDEX_BITS) - (won >> INDEX_BITS) < margin);
                    if (near && sure) {
                        if (by_score && a.score == SOM_SCORE_SOFTMAX) {
                            sure = false;
                        } else {
                            // the contest for the last place: more winners, until one stands apart or none is left
                            int n = __popc(__ballot_sync(ALL, won != 0));
                            bool open = n > a.k && (near >> a.k & 1u);
                            while (open && n < 32) {
                                const uint32_t m = __reduce_max_sync(ALL, key[0]);
                                if (m == 0) break;
                                const uint32_t before = __shfl_sync(ALL, won, n - 1);
                                open = (before >> INDEX_BITS) - (m >> INDEX_BITS) < margin;
                                if (!open) break;
                                if (lane == n) won = m;
                                ++n;
                                if (key[0] == m) {
#pragma unroll
                                    for (int v = 0; v + 1 < V; ++v) key[v] = key[v + 1];
                                    key[V - 1] = 0u;
                                }
                            }
                            if (n == 32) sure = false;
                            else at = settle_places<TYPE>(a, row, (int)(INDEX_MASK - (won & INDEX_MASK)), n, by_score, lane);
                        }
                    }
                }
                if (lane >= a.k) at = -1;
            }
        }
        if (!sure) at = choose_exact<TYPE>(a, row, top, by_score, by_groups, lane);
        float s = 0.f;
        const float xj = at >= 0 ? logit_at<TYPE>(a.logits, row + at) : -INFINITY;
        if (a.score == SOM_SCORE_SIGMOID) {
            if (at >= 0) s = 1.f / (1.f + expf(-xj));
            if (a.renorm && __any_sync(ALL, at >= 0 && xj < LOW_LOGIT)) {
                const float m = fminf(warp_max(xj), 0.f);
                if (at >= 0) s = sigmoid_from(xj, m);
            }
        } else if (a.renorm) {
            // only ratios of the chosen experts' scores count: taken from the largest of them
            const float m = warp_max(xj);
            if (at >= 0 && scores_at(m, top)) s = exp_from(xj, m);  // (beside an infinite logit all others score 0)
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

// ---- many tokens ----------------------------------------------------------------------------------------------
//
// Four lanes a token, eight tokens a warp: the rounds of the warp-wide choice cost the same instructions for one token as
// this form spends on eight.  A lane takes the row's experts in pieces of eight (its eight of every 32), sorts a piece and
// merges it into its list of the L largest keys; two exchanges make the four lanes' lists one.  The two largest keys that fell
// out are kept for the certificate.  With groups the first walk finds the groups' keys and the second one walks only the chosen
// groups.  What the certificate leaves open, the whole warp settles for one token at a time: contested groups by their exact
// keys, and contested places by the exact keys of the list, one candidate a lane.  Only where the contest reaches beyond the
// list, or scores need a sum over all experts, are all keys of the token computed exactly.
//
// 16384 tokens x 256 experts, 8 of 4 of 8 groups, bias: 27 us (0.7 TB/s).  Latency of the sorting networks, the grid leaving too few
// warps to cover it: 2048 warps are 256 blocks on 148 SMs, one on some and two on the others (two are resident by their registers),
// which issue in 20 and 39 % of the cycles; and with groups a row is walked, and the kept experts' scores are computed, twice.

// a (descending) becomes the L largest of a and b (descending), descending; rest >= rest2: the largest of those left out
template <int L>
__device__ __forceinline__ void merge_down(uint32_t (&a)[L], const uint32_t (&b)[L], uint32_t& rest, uint32_t& rest2)
{
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const uint32_t out = min(a[i], b[L - 1 - i]);
        rest2 = max(rest2, min(rest, out));
        rest = max(rest, out);
        a[i] = max(a[i], b[L - 1 - i]);
    }
#pragma unroll
    for (int h = L / 2; h >= 1; h >>= 1)
#pragma unroll
        for (int i = 0; i < L; ++i)
            if (!(i & h)) order2(a[i], a[i + h]);
}

constexpr int QUAD_WARPS = 8, QUAD_ROWS = 8 * QUAD_WARPS;

template <int TYPE, int L>
__global__ void __launch_bounds__(32 * QUAD_WARPS) k_route_many(const RouteArgs a)
{
    enter();
    extern __shared__ int hist[];  // [E] when counts are wanted
    __shared__ uint32_t group_keys[QUAD_ROWS][33];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane >> 2, part = lane & 3;
    if (a.counts) {
        for (int i = threadIdx.x; i < a.E; i += 32 * QUAD_WARPS) hist[i] = 0;
        __syncthreads();
    }
    const bool whole = whole_rows<TYPE, 8>(a.logits, a.ld) && (reinterpret_cast<uintptr_t>(a.bias) & 15u) == 0;
    const bool by_groups = a.groups > 1 && a.top_groups < a.groups;
    const bool by_score = a.bias || (a.groups > 1 && a.group_best == 2);
    const bool exact16 = TYPE != SOM_F32 && !by_score;
    const int pieces = (a.E + 31) / 32, size = a.E / a.groups, per_group = size / 32;
    Packing pack{0.f, (float)KEY_MOST / 64.f, 3, true};
    if (by_score) {
        float high = 0.f, low = 0.f;
        if (a.bias)
            for (int i = lane; i < a.E; i += 32) {
                const float b = *(a.bias + i);
                high = fmaxf(high, b);
                if (b >= FAR_BIAS) low = fminf(low, b);
            }
        pack = packing_of(low, high, a.score);
    }
    const float ceiling = pack.ceiling, scale = pack.scale;
    const uint32_t margin = pack.margin;
    // whether the row's largest logit has to be found first (where not, the largest chosen one is that)
    const bool has_top = a.score == SOM_SCORE_SOFTMAX ? by_score || !a.renorm || !exact16 || by_groups : !by_score && !exact16;

    for (int64_t t0 = ((int64_t)blockIdx.x * QUAD_WARPS + warp) * 8; t0 < a.T; t0 += (int64_t)gridDim.x * QUAD_ROWS) {
        const int64_t t = t0 + quad < a.T ? t0 + quad : a.T - 1, row = t * a.ld;  // (past the end: the last row again, not written)
        float top = 0.f, total = 1.f;
        if (has_top) {
            top = -INFINITY;
            for (int b = 0; b < pieces; ++b) {
                float x[8];
                load_row<TYPE, 8>(a.logits, row, b * 32 + part * 8, a.E, whole, x);
#pragma unroll
                for (int v = 0; v < 8; ++v) top = fmaxf(top, x[v]);
            }
            top = fmaxf(top, __shfl_xor_sync(ALL, top, 1));
            top = fmaxf(top, __shfl_xor_sync(ALL, top, 2));
            if (!(top > -INFINITY)) top = 0.f;
        }
        if (a.score == SOM_SCORE_SOFTMAX && (by_score || !a.renorm)) {
            total = 0.f;
            for (int b = 0; b < pieces; ++b) {
                float x[8];
                load_row<TYPE, 8>(a.logits, row, b * 32 + part * 8, a.E, whole, x);
#pragma unroll
                for (int v = 0; v < 8; ++v) x[v] = x[v] > -INFINITY ? exp_from(x[v], top) : 0.f;
                total += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
            }
            total += __shfl_xor_sync(ALL, total, 1);
            total += __shfl_xor_sync(ALL, total, 2);
        }
        bool full = !(pack.fits && top < INFINITY);  // all keys have to be computed exactly
        auto keys_of = [&](int piece, uint32_t (&key)[8]) {
            const int at = piece * 32 + part * 8;
            float x[8];
            load_row<TYPE, 8>(a.logits, row, at, a.E, whole, x);
            if (exact16) {
#pragma unroll
                for (int v = 0; v < 8; ++v) key[v] = x[v] > -INFINITY ? ordered16<TYPE>(x[v] + 0.f) << 16 | (INDEX_MASK - at - v) : 0u;
                return;
            }
            float bias[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) bias[v] = 0.f;
            if (a.bias) load_row<SOM_F32, 8>(a.bias, 0, at, a.E, whole, bias);
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                float d;
                if (!by_score) d = top - x[v];
                else if (a.score == SOM_SCORE_SOFTMAX) d = ceiling - (__fdividef(exp_from(x[v], top), total) + bias[v]);
                else d = ceiling - (__fdividef(1.f, 1.f + __expf(-x[v])) + bias[v]);
                const uint32_t u = KEY_MOST - min((uint32_t)(d * scale), KEY_MOST - 1u);
                key[v] = x[v] > -INFINITY && d < INFINITY ? u << INDEX_BITS | (INDEX_MASK - at - v) : 0u;
            }
        };
        unsigned kept = 0;
        if (by_groups) {
            uint32_t* mine = group_keys[warp * 8 + quad];
            bool lone = false;
            unsigned bounds = 0;  // groups whose sum has the lowest key in it: an upper bound of the group's key
            for (int g = 0; g < a.groups; ++g) {
                uint32_t m1 = 0, m2 = 0;
                for (int b = 0; b < per_group; ++b) {
                    uint32_t key[8];
                    keys_of(g * per_group + b, key);
#pragma unroll
                    for (int v = 0; v < 8; ++v) {
                        m2 = max(m2, min(m1, key[v]));
                        m1 = max(m1, key[v]);
                    }
                }
#pragma unroll
                for (int d = 1; d <= 2; d <<= 1) {
                    const uint32_t o1 = __shfl_xor_sync(ALL, m1, d), o2 = __shfl_xor_sync(ALL, m2, d);
                    merge2(m1, m2, o1, o2);
                }
                bounds |= (unsigned)(m1 && far_key(m2)) << g;
                lone |= m1 && !m2;  // a lone expert's distance is not comparable with the sum of two
                if (part == 0) mine[g] = a.group_best == 2 ? (m1 >> INDEX_BITS) + (m2 >> INDEX_BITS) : m1;
            }
            if (a.group_best == 2 && lone) full = true;
            __syncwarp();
            uint32_t low = 0xffffffffu, next = 0u;  // of the groups kept and of the others, this lane's quarter
            for (int g = part; g < a.groups; g += 4) {
                const uint32_t k = mine[g];
                int rank = 0;
                for (int o = 0; o < a.groups; ++o) rank += mine[o] > k || (mine[o] == k && o < g);
                if (rank < a.top_groups) {
                    kept |= 1u << g;
                    low = min(low, k);
                } else {
                    next = max(next, k);
                }
            }
#pragma unroll
            for (int d = 1; d <= 2; d <<= 1) {
                kept |= __shfl_xor_sync(ALL, kept, d);
                low = min(low, __shfl_xor_sync(ALL, low, d));
                next = max(next, __shfl_xor_sync(ALL, next, d));
            }
            if (a.group_best == 2 && (kept & bounds)) full = true;
            if (!exact16) {
                const uint32_t apart = a.group_best == 2 ? 2 * margin : margin;
                const int shift = a.group_best == 2 ? 0 : INDEX_BITS;
                const bool open = !full && low != 0xffffffffu && low && next && (low >> shift) - (next >> shift) < apart;
                if (a.score == SOM_SCORE_SOFTMAX || !by_score) {
                    full |= open;
                } else {
                    for (unsigned todo = __ballot_sync(ALL, open && part == 0); todo; todo &= todo - 1) {
                        const int who = __ffs(todo) - 1;
                        const int64_t its_row = __shfl_sync(ALL, row, who);
                        const uint32_t its_low = __shfl_sync(ALL, low, who) >> shift, its_next = __shfl_sync(ALL, next, who) >> shift;
                        const unsigned got = settle_groups<TYPE>(a, its_row, lane < a.groups ? group_keys[warp * 8 + (who >> 2)][lane] >> shift : 0u,
                                                                 its_low, its_next, apart, lane);
                        if (quad == who >> 2) kept = got;
                    }
                }
            }
            __syncwarp();  // the keys have been read: the next token may write its own
        }
        uint32_t list[L], rest = 0, rest2 = 0;
#pragma unroll
        for (int i = 0; i < L; ++i) list[i] = 0u;
        const int walk = by_groups ? a.top_groups * per_group : pieces;
        unsigned left = kept;
        int within = 0;
        for (int b = 0; b < walk; ++b) {
            int piece = b;
            if (by_groups) {  // (each token walks its own groups)
                piece = left ? (__ffs(left) - 1) * per_group + within : pieces;  // (beyond the row: no experts)
                if (++within == per_group) within = 0, left &= left - 1;
            }
            uint32_t key[8], more[L];
            keys_of(piece, key);
            sort_down<8>(key);
#pragma unroll
            for (int i = 0; i < L; ++i) more[i] = i < 8 ? key[i] : 0u;
            merge_down<L>(list, more, rest, rest2);
        }
#pragma unroll
        for (int d = 1; d <= 2; d <<= 1) {
            uint32_t more[L];
#pragma unroll
            for (int i = 0; i < L; ++i) more[i] = __shfl_xor_sync(ALL, list[i], d);
            const uint32_t r1 = __shfl_xor_sync(ALL, rest, d), r2 = __shfl_xor_sync(ALL, rest2, d);
            merge2(rest, rest2, r1, r2);
            merge_down<L>(list, more, rest, rest2);
        }
        int at[L];
#pragma unroll
        for (int i = 0; i < L; ++i) at[i] = i < a.k && list[i] ? (int)(INDEX_MASK - (list[i] & INDEX_MASK)) : -1;
        const bool there = t0 + quad < a.T;
        if (!exact16) {
            bool near = false;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const uint32_t next = i + 1 < L ? list[i + 1 < L ? i + 1 : i] : rest;
                if (i < a.k && list[i]) {
                    near |= next && (list[i] >> INDEX_BITS) - (next >> INDEX_BITS) < margin;
                    full |= far_key(list[i]);
                }
            }
            if (by_score && a.score == SOM_SCORE_SOFTMAX) full |= near;
            for (unsigned todo = __ballot_sync(ALL, near && !full && there && part == 0); todo; todo &= todo - 1) {
                const int who = __ffs(todo) - 1;
                uint32_t mine = __shfl_sync(ALL, rest, who), next = __shfl_sync(ALL, rest2, who);  // lanes 0 to L: the candidates
#pragma unroll
                for (int i = 0; i < L; ++i) {
                    const uint32_t v = __shfl_sync(ALL, list[i], who);
                    if (lane == i) mine = v;
                }
                const uint32_t below = __shfl_down_sync(ALL, mine, 1);
                if (lane < L) next = below;
                // the contest for the last place has to end within the list
                const unsigned clear = __ballot_sync(ALL, lane <= L && (!next || (mine >> INDEX_BITS) - (next >> INDEX_BITS) >= margin));
                if (!(clear >> (a.k - 1))) {
                    if (quad == who >> 2) full = true;
                    continue;
                }
                const int index = (int)(INDEX_MASK - (mine & INDEX_MASK));
                const int n = __popc(__ballot_sync(ALL, lane <= L && mine));
                const int got = settle_places<TYPE>(a, __shfl_sync(ALL, row, who), index, n, by_score, lane);
#pragma unroll
                for (int i = 0; i < L; ++i) {
                    const int v = __shfl_sync(ALL, got, i);
                    if (quad == who >> 2) at[i] = i < a.k ? v : -1;
                }
            }
        }
        for (unsigned todo = __ballot_sync(ALL, full && part == 0 && there); todo; todo &= todo - 1) {
            const int who = __ffs(todo) - 1;
            const int got = choose_exact<TYPE>(a, __shfl_sync(ALL, row, who), __shfl_sync(ALL, top, who), by_score, by_groups, lane);
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int v = __shfl_sync(ALL, got, i);
                if (quad == who >> 2) at[i] = i < a.k ? v : -1;
            }
        }
        // lane `part` writes choices part, part + 4, ...
        float s[L / 4], x[L / 4], most = -INFINITY, least = INFINITY;
        int mine[L / 4];
#pragma unroll
        for (int i = 0; i < L; ++i)
            if ((i & 3) == part) mine[i >> 2] = at[i];
#pragma unroll
        for (int i = 0; i < L / 4; ++i) {
            x[i] = mine[i] >= 0 ? logit_at<TYPE>(a.logits, row + mine[i]) : -INFINITY;
            most = fmaxf(most, x[i]);
            if (mine[i] >= 0) least = fminf(least, x[i]);
        }
#pragma unroll
        for (int d = 1; d <= 2; d <<= 1) {
            most = fmaxf(most, __shfl_xor_sync(ALL, most, d));
            least = fminf(least, __shfl_xor_sync(ALL, least, d));
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < L / 4; ++i) {
            s[i] = 0.f;
            if (mine[i] >= 0) {
                if (a.score == SOM_SCORE_SIGMOID) s[i] = a.renorm && least < LOW_LOGIT ? sigmoid_from(x[i], fminf(most, 0.f)) : 1.f / (1.f + expf(-x[i]));
                else if (!a.renorm) s[i] = exp_from(x[i], top) / total;
                else if (!has_top || scores_at(most, top)) s[i] = exp_from(x[i], most);  // only ratios count
            }
            sum += s[i];
        }
        sum += __shfl_xor_sync(ALL, sum, 1);
        sum += __shfl_xor_sync(ALL, sum, 2);
        if (t0 + quad < a.T) {
#pragma unroll
            for (int i = 0; i < L / 4; ++i) {
                const int j = 4 * i + part;
                if (j < a.k) {
                    const float v = a.renorm ? (sum > 0.f ? s[i] / sum : 0.f) : s[i];
                    a.weights[t * a.k + j] = v * a.scale;
                    a.indices[t * a.k + j] = mine[i];
                    if (a.counts && mine[i] >= 0) atomicAdd(&hist[mine[i]], 1);
                }
            }
        }
    }
    if (a.counts) {
        __syncthreads();
        for (int i = threadIdx.x; i < a.E; i += 32 * QUAD_WARPS)
            if (hist[i]) atomicAdd(&a.counts[i], hist[i]);
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

// ds = scale dw for the chosen, 0 for others; renormalised: scale (dw - sum of w dw) / (sum of the chosen s).  dlogit = s (1 - s) ds for
// the sigmoid, s (ds - sum of s ds) for the softmax.  Lane j holds choice j.  The row is written as if nothing had been chosen, then
// the chosen elements are written over it.  16381 tokens x 100 bf16 logits: 7.3 MB, 9.0 us a call on the device (calls one after
// the other in a graph; the host's call takes about as long).  Bound by instructions: issued in 75 % of the cycles that an SM is busy.
template <int TYPE, int V>
__global__ void __launch_bounds__(32 * ROUTE_WARPS) k_route_backward(const RouteGradArgs a)
{
    enter();
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
            float q = 0.f;  // (renormalised: any multiple of the scores will do)
            if (a.score == SOM_SCORE_SOFTMAX) {
                const float most = warp_max(xj);
                bool scores = true;
                if (most < NO_SCORE + 100.f) {  // (above that only a row's largest logit beyond 100 could leave no score)
                    float top = most;
                    for (int i = lane; i < a.E; i += 32) top = fmaxf(top, logit_at<TYPE>(a.logits, row + i));
                    scores = scores_at(most, warp_max(top));
                }
                if (live && scores) q = exp_from(xj, most);
            } else {
                if (live) q = 1.f / (1.f + expf(-xj));
                if (a.renorm && __any_sync(ALL, live && xj < LOW_LOGIT)) {
                    const float m = fminf(warp_max(xj), 0.f);
                    if (live) q = sigmoid_from(xj, m);
                }
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

// the warp's registers for a row: the smallest power of two of 32 experts that holds it
template <template <int, int> class K, int TYPE, class A>
cudaError_t by_size(som_layers* l, int E, const A& a, int grid, size_t smem, cudaStream_t st)
{
    if (E <= 32) return K<TYPE, 1>::go(l, a, grid, smem, st);
    if (E <= 64) return K<TYPE, 2>::go(l, a, grid, smem, st);
    if (E <= 128) return K<TYPE, 4>::go(l, a, grid, smem, st);
    if (E <= 256) return K<TYPE, 8>::go(l, a, grid, smem, st);
    if (E <= 512) return K<TYPE, 16>::go(l, a, grid, smem, st);
    return K<TYPE, 32>::go(l, a, grid, smem, st);
}

template <template <int, int> class K, class A>
cudaError_t by_type(som_layers* l, int type, int E, const A& a, int grid, size_t smem, cudaStream_t st)
{
    if (type == SOM_F32) return by_size<K, SOM_F32>(l, E, a, grid, smem, st);
    if (type == SOM_F16) return by_size<K, SOM_F16>(l, E, a, grid, smem, st);
    return by_size<K, SOM_BF16>(l, E, a, grid, smem, st);
}

template <int TYPE, int V>
struct Route {
    static cudaError_t go(som_layers* l, const RouteArgs& a, int grid, size_t smem, cudaStream_t st)
    {
        return launch(l, k_route<TYPE, V>, dim3(grid), 32 * ROUTE_WARPS, smem, st, 1, a);
    }
};

template <int TYPE, int V>
struct RouteGrad {
    static cudaError_t go(som_layers* l, const RouteGradArgs& a, int grid, size_t smem, cudaStream_t st)
    {
        return launch(l, k_route_backward<TYPE, V>, dim3(grid), 32 * ROUTE_WARPS, smem, st, 1, a);
    }
};

// Tokens from which on four lanes a token (k_route_many) are faster than a warp a token (k_route).  k_route_many takes one pass of
// long latency, the longer the more it walks a row (groups: twice), k_route time by tokens x experts.  8 chosen, fp32, k_route_many
// / k_route in us (`*` where k_route_many is taken; calls of up to about 15 us are the host's):
//   experts, keys            6000 tokens      8192            12288           16384           32768
//   64, logits               15 / 15          15 / 15 *       15 / 15 *       15 / 17 *       19 / 25 *
//   128, sigmoid             16 / 16          16 / 16 *       16 / 17 *       17 / 19 *       26 / 29 *
//   128, sigmoid, groups     17 / 16          17 / 16         19 / 19         19 / 22 *       31 / 36 *
//   256, logits              17 / 15          17 / 17 *       19 / 21 *       20 / 23 *       32 / 34 *
//   256, sigmoid             19 / 17          19 / 20 *       22 / 23 *       23 / 25 *       37 / 40 *
//   256, sigmoid, groups     23 / 19          23 / 22         27 / 25         27 / 29 *       46 / 48 *
//   384, sigmoid             24 / 27          24 / 34 *       29 / 42 *       29 / 51 *       50 / 89 *
//   512, sigmoid, groups     35 / 31          35 / 37 *       41 / 48 *       41 / 58 *       78 / 103 *
//   1024, sigmoid            48 / 65          48 / 80 *       57 / 108 *      58 / 139 *      123 / 260 *
//   1024, sigmoid, groups    62 / 70          62 / 85 *       72 / 115 *      71 / 150 *      155 / 281 *
// Softmax scores with a bias or groups by two walk a row up to four times, and near ties of them take all exact keys of a token,
// which is the whole warp's work in either form:
//   64                       16 / 16          16 / 16         18 / 19         17 / 21 *       27 / 33 *
//   256                      40 / 25          40 / 27         44 / 32         44 / 41         67 / 65
//   256, groups              41 / 29          54 / 33         57 / 39         58 / 54         81 / 70
//   512                      54 / 61          69 / 66         66 / 77         82 / 88 *       126 / 148 *
//   512, groups              90 / 57          91 / 81         91 / 91         104 / 108 *     158 / 163 *
//   1024, groups             138 / 123        180 / 179       192 / 222       193 / 245 *     355 / 435 *
// (256 experts, 65536 tokens: 111 / 104, with groups 141 / 125.)
bool takes_many(int64_t T, int E, bool by_groups, bool softmax_keys)
{
    if (softmax_keys) return T >= 16384 && (E <= 128 || E >= 512);
    return T >= (by_groups && E <= 256 ? 16384 : 8192);
}

void note_rounds(som_layers* l, int form, int64_t rounds)
{
    if (rounds > l->rounds[5][form]) l->rounds[5][form] = rounds;
}

// What a warp sets up (biases, groups, the block's counts) is shared by its tokens: no more blocks than are resident.
int route_grid(const som_layers* l, int64_t T, int per_sm)
{
    const int64_t want = (T + ROUTE_WARPS - 1) / ROUTE_WARPS, most = (int64_t)l->sm_count * per_sm;
    return (int)(want < most ? want : most);
}

}  // namespace

template <int TYPE, int L>
cudaError_t go_many(som_layers* l, const RouteArgs& a, int grid, size_t smem, cudaStream_t st)
{
    return launch(l, k_route_many<TYPE, L>, dim3(grid), 32 * QUAD_WARPS, smem, st, 1, a);
}

template <int TYPE>
cudaError_t route_many(som_layers* l, const RouteArgs& a, int grid, size_t smem, cudaStream_t st)
{
    return a.k <= 8 ? go_many<TYPE, 8>(l, a, grid, smem, st) : go_many<TYPE, 16>(l, a, grid, smem, st);
}

int launch_route(som_layers* l, int type, int score, int64_t T, int E, int k, const void* logits, int64_t ld, const float* bias,
                 int groups, int top_groups, int group_best, int renorm, float scale, float* weights, int32_t* indices,
                 int32_t* counts, cudaStream_t st)
{
    const int grid = T > 0 ? route_grid(l, T, E <= 256 ? 4 : 2) : 0;
    cudaError_t e = cudaSuccess;
    if (counts && grid != 1) e = cudaMemsetAsync(counts, 0, (size_t)E * sizeof(int32_t), st);  // one block writes its counts itself
    if (e == cudaSuccess && grid) {
        const RouteArgs a{logits, ld, T, bias, weights, indices, counts, E, k, score, groups, top_groups, group_best, renorm, scale};
        const size_t smem = counts ? (size_t)E * sizeof(int) : 0;
        const bool by_groups = groups > 1 && top_groups < groups;
        const bool by_score = bias || (groups > 1 && group_best == 2);
        // Not four lanes a token where pieces of 32 experts span groups, and not where scores of 16-bit logits without a bias decide: equal
        // logits are common there, and only the other form settles them without exact keys.
        if (takes_many(T, E, by_groups, by_score && score == SOM_SCORE_SOFTMAX) && k <= 16 && (!by_groups || E / groups % 32 == 0) &&
            (type == SOM_F32 || bias || !by_score)) {
            // (two blocks an SM are resident; with four an SM the last ones even out: 65536 tokens x 256 experts 60 us, 63 with two)
            const int64_t want = (T + QUAD_ROWS - 1) / QUAD_ROWS, most = (int64_t)l->sm_count * 4;
            const int blocks = (int)(want < most ? want : most);
            note_rounds(l, 1, (want + blocks - 1) / blocks);
            e = type == SOM_F32 ? route_many<SOM_F32>(l, a, blocks, smem, st) : type == SOM_F16 ? route_many<SOM_F16>(l, a, blocks, smem, st) : route_many<SOM_BF16>(l, a, blocks, smem, st);
        } else {
            note_rounds(l, 0, ((T + ROUTE_WARPS - 1) / ROUTE_WARPS + grid - 1) / grid);
            e = by_type<Route>(l, type, E, a, grid, smem, st);
        }
    }
    return outcome(l, e);
}

int launch_route_backward(som_layers* l, int type, int score, int64_t T, int E, int k, const void* logits, int64_t ld,
                          const int32_t* indices, const float* dweights, int renorm, float scale, void* dlogits, cudaStream_t st)
{
    if (T == 0) return SOM_OK;
    const RouteGradArgs a{logits, ld, T, indices, dweights, dlogits, E, k, score, renorm, scale, l->flags};
    const cudaError_t e = by_type<RouteGrad>(l, type, E, a, route_grid(l, T, 8), 0, st);
    return outcome(l, e);
}

}  // namespace lay
