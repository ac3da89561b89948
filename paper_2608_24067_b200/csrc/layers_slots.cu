// What surrounds the experts' products: the plan that orders the tokens' slots by expert, the gather into that order, the
// join of a token's results and the small gradients.
#include "layers_math.cuh"
#include "layers_slots.cuh"

namespace lay {
namespace {

constexpr int PLAN_THREADS = 1024, PLAN_WARPS = PLAN_THREADS / 32;

__device__ __forceinline__ float load_weight(const void* w, int type, int64_t i)
{
    if (type == SOM_F32) return static_cast<const float*>(w)[i];
    return unpack1(static_cast<const uint16_t*>(w)[i], type == SOM_BF16);
}

// A stable counting sort of the slots by expert in one block: every warp owns a contiguous run of slots, counts it into a
// row of its own in shared memory, the rows are turned into starting places, and the warp walks its run again.
// Stable, so that the rows of an expert (and the sums over them) have one order.  Latency: 6 us for 576 slots of 64 experts.
__global__ void __launch_bounds__(PLAN_THREADS) k_slot_plan(SlotPlan p, const int32_t* indices, const void* weights,
                                                           int weights_type, int64_t slots, int E, int* flags)
{
    enter();
    extern __shared__ int hist[];  // [PLAN_WARPS][E], then [E] segment starts
    __shared__ int warp_sum[PLAN_WARPS];
    int* start = hist + PLAN_WARPS * E;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < PLAN_WARPS * E; i += PLAN_THREADS) hist[i] = 0;
    __syncthreads();
    const int64_t run = (slots + PLAN_THREADS - 1) / PLAN_THREADS * 32;
    const int64_t lo = warp * run, hi = lo + run < slots ? lo + run : slots;
    int* mine = hist + warp * E;
    bool bad = false;
    for (int64_t s = lo + lane; s < hi; s += 32) {
        const int e = indices[s];
        if (e >= 0 && e < E) atomicAdd(&mine[e], 1);
        bad |= e < -1 || e >= E;
    }
    som_raise(flags, bad, LAY_FLAG_BAD_EXPERT);
    __syncthreads();
    // thread e: starting places of expert e's slots by warp; segments padded to whole tiles
    int count = 0;
    const int e = threadIdx.x;
    if (e < E)
        for (int w = 0; w < PLAN_WARPS; ++w) {
            const int c = hist[w * E + e];
            hist[w * E + e] = count;
            count += c;
        }
    const int tiles = (count + p.tile - 1) / p.tile;
    int sum = tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += v;
    }
    if (lane == 31) warp_sum[warp] = sum;
    __syncthreads();
    int before = sum - tiles;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    if (e < E) {
        start[e] = before * p.tile;
        p.seg[e] = before * p.tile;
        p.count[e] = count;
        for (int i = 0; i < tiles; ++i) p.tile_expert[before + i] = e;
        if (e == E - 1) {
            p.seg[E] = (before + tiles) * p.tile;
            *p.tiles = before + tiles;
        }
    }
    __syncthreads();
    for (int64_t s0 = lo; s0 < hi; s0 += 32) {
        const int64_t s = s0 + lane;
        int x = s < hi ? indices[s] : -1;
        if (x < 0 || x >= E) x = -1;
        const unsigned same = __match_any_sync(0xffffffffu, x);
        const int rank = __popc(same & ((1u << lane) - 1u));
        int at = 0;
        if (x >= 0) at = mine[x];
        __syncwarp();
        if (x >= 0 && rank == 0) mine[x] = at + __popc(same);
        __syncwarp();
        if (s < hi) {
            const int row = x >= 0 ? start[x] + at + rank : -1;
            p.pos[s] = row;
            if (row >= 0) p.row_weight[row] = load_weight(weights, weights_type, s);
        }
    }
}

// The same for many slots, in three launches over blocks of PLACE_SLOTS consecutive slots: every block counts its slots by
// expert, one block turns the counts into segments and the blocks' starting places, every block places its slots.  (One
// block alone took 60 us for 32768 slots; these take 3 + 5 + 9.)
constexpr int PLACE_SLOTS = 1024, PLACE_WARPS = 8;

__global__ void __launch_bounds__(32 * PLACE_WARPS) k_slot_count(const int32_t* indices, int64_t slots, int E, int* counts, int* flags)
{
    enter();
    extern __shared__ int hist[];  // [E]
    for (int i = threadIdx.x; i < E; i += 32 * PLACE_WARPS) hist[i] = 0;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * PLACE_SLOTS, hi = lo + PLACE_SLOTS < slots ? lo + PLACE_SLOTS : slots;
    bool bad = false;
    for (int64_t s = lo + threadIdx.x; s < hi; s += 32 * PLACE_WARPS) {
        const int e = indices[s];
        if (e >= 0 && e < E) atomicAdd(&hist[e], 1);
        bad |= e < -1 || e >= E;
    }
    som_raise(flags, bad, LAY_FLAG_BAD_EXPERT);
    __syncthreads();
    for (int i = threadIdx.x; i < E; i += 32 * PLACE_WARPS) counts[(size_t)blockIdx.x * E + i] = hist[i];
}

// counts[block][e] -> first place of the block's slots within expert e; the segments
__global__ void __launch_bounds__(PLAN_THREADS) k_slot_segments(SlotPlan p, int E, int blocks, int* counts)
{
    enter();
    __shared__ int warp_sum[PLAN_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, e = threadIdx.x;
    int count = 0;
    if (e < E)
        for (int b0 = 0; b0 < blocks; b0 += 8) {
            int c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = b0 + i < blocks ? counts[(size_t)(b0 + i) * E + e] : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (b0 + i < blocks) {
                    counts[(size_t)(b0 + i) * E + e] = count;
                    count += c[i];
                }
        }
    const int tiles = (count + p.tile - 1) / p.tile;
    int sum = tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += v;
    }
    if (lane == 31) warp_sum[warp] = sum;
    __syncthreads();
    int before = sum - tiles;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    if (e < E) {
        p.seg[e] = before * p.tile;
        p.count[e] = count;
        for (int i = 0; i < tiles; ++i) p.tile_expert[before + i] = e;
        if (e == E - 1) {
            p.seg[E] = (before + tiles) * p.tile;
            *p.tiles = before + tiles;
        }
    }
}

__global__ void __launch_bounds__(32 * PLACE_WARPS) k_slot_place(SlotPlan p, const int32_t* indices, const void* weights, int weights_type,
                                                                int64_t slots, int E, const int* places)
{
    enter();
    extern __shared__ int hist[];  // [PLACE_WARPS][E]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < PLACE_WARPS * E; i += 32 * PLACE_WARPS) hist[i] = 0;
    __syncthreads();
    constexpr int RUN = PLACE_SLOTS / PLACE_WARPS;
    const int64_t lo = (int64_t)blockIdx.x * PLACE_SLOTS + warp * RUN;
    int* mine = hist + warp * E;
    int x[RUN / 32], same[RUN / 32];
#pragma unroll
    for (int i = 0; i < RUN / 32; ++i) {
        const int64_t s = lo + i * 32 + lane;
        x[i] = s < slots ? indices[s] : -1;
        if (x[i] < 0 || x[i] >= E) x[i] = -1;
        same[i] = (int)__match_any_sync(0xffffffffu, x[i]);
        if (x[i] >= 0 && (same[i] & ((1 << lane) - 1)) == 0) mine[x[i]] += __popc(same[i]);
        __syncwarp();
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += 32 * PLACE_WARPS) {
        int at = p.seg[e] + places[(size_t)blockIdx.x * E + e];
        for (int w = 0; w < PLACE_WARPS; ++w) {
            const int c = hist[w * E + e];
            hist[w * E + e] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RUN / 32; ++i) {
        const int64_t s = lo + i * 32 + lane;
        const int rank = __popc(same[i] & ((1 << lane) - 1));
        int row = -1;
        if (x[i] >= 0) row = mine[x[i]] + rank;
        __syncwarp();
        if (x[i] >= 0 && rank == 0) mine[x[i]] += __popc(same[i]);
        __syncwarp();
        if (s < slots) {
            p.pos[s] = row;
            if (row >= 0) p.row_weight[row] = load_weight(weights, weights_type, s);
        }
    }
}

// Rows of x (blockIdx.z == 0) and of dy (1) in the slots' order, a warp a slot: what it reads does not wait for where it goes.  With
// `zeros` up to whole steps of 64 rows of an expert are zeros (the sums over an expert's rows run in such steps; rows of products
// do not mix).  Bound by the writes: 32768 rows of 2048 in 28 us, 134 MB
// written and 17 read (5.4 TB/s); by rows, each asking for its slot, 31.  (Rows fetched one by one by the products' copies instead took
// longer than both.)
__global__ void __launch_bounds__(256) k_gather(SlotPlan p, int64_t slots, int E, int k, int D, const uint16_t* x, int64_t ldx, uint16_t* xp,
                                                const uint16_t* dy, int64_t lddy, uint16_t* dyp, int zeros)
{
    enter();
    const int lane = threadIdx.x & 31, chunks = D / 8;
    const uint16_t* from = blockIdx.z ? dy : x;
    const int64_t ld = blockIdx.z ? lddy : ldx, all = slots + (zeros ? (int64_t)E * 64 : 0);
    uint16_t* to = blockIdx.z ? dyp : xp;
    for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < all; i += (int64_t)gridDim.x * 8) {
        if (i < slots) {
            const uint4* in = reinterpret_cast<const uint4*>(from + (size_t)(i / k) * ld);
            const int row = p.pos[i];
            for (int c = lane; c < chunks; c += 128) {
                uint4 u[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + 32 * j < chunks) u[j] = *(in + c + 32 * j);
                if (row < 0) break;
                uint4* out = reinterpret_cast<uint4*>(to + (size_t)row * D);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + 32 * j < chunks) out[c + 32 * j] = u[j];
            }
        } else {
            const int e = (int)((i - slots) >> 6), n = p.count[e], r = n + (int)((i - slots) & 63);
            if (r >= ((n + 63) & ~63)) continue;
            uint4* out = reinterpret_cast<uint4*>(to + (size_t)(p.seg[e] + r) * D);
            for (int c = lane; c < chunks; c += 32) out[c] = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

// y[t] = residual[t] + sum over j of part[pos[t][j]], in the order of j.  The parts are fp32 so that a token's result is rounded
// once.  Bound by HBM: 4096 tokens x 8 x 2048 in 48 us, 285 MB (5.9 TB/s).
__device__ __forceinline__ void join_rows(const EndArgs& a, int block)
{
    const int chunks = a.D / 8;
    for (int64_t i = (int64_t)block * blockDim.x + threadIdx.x; i < a.T * chunks; i += (int64_t)a.join_blocks * blockDim.x) {
        const int64_t t = i / chunks;
        const int c = (int)(i % chunks);
        float v[8];
        if (a.residual) {
            load8(a.residual + (size_t)t * a.ldr + 8 * c, v, a.bf16);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.f;
        }
        for (int j = 0; j < a.k; ++j) {
            const int row = a.p.pos[t * a.k + j];
            if (row < 0) continue;
            const float4* q = reinterpret_cast<const float4*>(a.part + (size_t)row * a.D + 8 * c);
            const float4 x = q[0], y = q[1];
            v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
            v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
        }
        uint4 u;
        u.x = pack2(v[0], v[1], a.bf16);
        u.y = pack2(v[2], v[3], a.bf16);
        u.z = pack2(v[4], v[5], a.bf16);
        u.w = pack2(v[6], v[7], a.bf16);
        *reinterpret_cast<uint4*>(a.y + (size_t)t * a.ldy + 8 * c) = u;
    }
}

// dweights[slot] = sum of the slot's partial <h, W2^T dy> + <b2, dy>; one warp a slot
__device__ __forceinline__ void slot_dweights(const EndArgs& a, int block)
{
    const int lane = threadIdx.x & 31;
    for (int64_t s = ((int64_t)block * blockDim.x + threadIdx.x) >> 5; s < a.T * a.k; s += ((int64_t)a.dweights_blocks * blockDim.x) >> 5) {
        const int row = a.p.pos[s];
        float v = 0.f;
        if (row >= 0) {
            for (int i = lane; i < a.dots; i += 32) v += a.dot[(size_t)row * a.dots + i];
            if (a.b2) {
                const uint16_t* b = a.b2 + (size_t)a.indices[s] * a.D;
                const uint16_t* g = a.dy + (size_t)(s / a.k) * a.lddy;
                for (int i = lane * 8; i < a.D; i += 256) {
                    float u[8], w[8];
                    load8(b + i, u, a.bf16);
                    load8(g + i, w, a.bf16);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v = fmaf(u[j], w[j], v);
                }
            }
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        if (lane == 0) {
            if (a.weights_type == SOM_F32) static_cast<float*>(a.dweights)[s] = v;
            else static_cast<uint16_t*>(a.dweights)[s] = (uint16_t)pack2(v, 0.f, a.bf16);
        }
    }
}

// out[e][c] = sum over the rows of expert e of weight[row] * v[row][c]; a block sums 64 columns of one expert, 32 rows at
// a time, in a fixed order
__device__ __forceinline__ void column_sums(const EndArgs& a, int block, float* part)
{
    const int across = (a.v_cols + 63) / 64, e = block / across, c0 = (block - e * across) * 64;
    const int c = c0 + (threadIdx.x & 7) * 8, r = threadIdx.x >> 3;
    const int64_t lo = a.p.seg ? a.p.seg[e] : 0, hi = a.p.seg ? lo + a.p.count[e] : a.rows;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < a.v_cols)
#pragma unroll 4
        for (int64_t i = lo + r; i < hi; i += 32) {
            float u[8];
            load8(a.v + (size_t)i * a.ldv + c, u, a.bf16);
            const float w = a.p.seg ? a.p.row_weight[i] : 1.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = fmaf(w, u[j], s[j]);
        }
#pragma unroll
    for (int j = 0; j < 8; ++j) part[r * 65 + (threadIdx.x & 7) * 8 + j] = s[j];
    __syncthreads();
    if (threadIdx.x < 64 && c0 + threadIdx.x < a.v_cols) {
        float sum = 0.f;
        for (int i = 0; i < 32; ++i) sum += part[i * 65 + threadIdx.x];
        a.v_sums[(size_t)e * a.v_cols + c0 + threadIdx.x] = (uint16_t)pack2(sum, 0.f, a.bf16);
    }
}

// out[e][c] = sum of part[g][c] over the expert's groups of 32 rows (of 32-row sums); 32 columns a block, 8 groups at a time
__device__ __forceinline__ void join_sums(const EndArgs& a, int block, float* sums)
{
    const int across = (a.sums_cols + 31) / 32, e = block / across;
    const int c = (block - e * across) * 32 + (threadIdx.x & 31), r = threadIdx.x >> 5;
    const int64_t lo = a.p.seg ? a.p.seg[e] / 32 : 0, hi = a.p.seg ? lo + (a.p.count[e] + 31) / 32 : (a.rows + 31) / 32;
    float s = 0.f;
    if (c < a.sums_cols)
        for (int64_t i = lo + r; i < hi; i += 8) s += a.sums[(size_t)i * a.sums_cols + c];
    sums[r * 33 + (threadIdx.x & 31)] = s;
    __syncthreads();
    if (r == 0 && c < a.sums_cols) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += sums[i * 33 + threadIdx.x];
        a.sums_out[(size_t)e * a.sums_cols + c] = (uint16_t)pack2(s, 0.f, a.bf16);
    }
}

// What nothing follows, in one launch, each part by blocks of its own: the parts that take longest a block come first.
__global__ void __launch_bounds__(256) k_ends(const __grid_constant__ EndArgs a)
{
    enter();
    extern __shared__ float shared[];
    int block = blockIdx.x;
    if (block < a.v_blocks) return column_sums(a, block, shared);
    block -= a.v_blocks;
    if (block < a.sums_blocks) return join_sums(a, block, shared);
    block -= a.sums_blocks;
    if (block < a.dweights_blocks) return slot_dweights(a, block);
    join_rows(a, block - a.dweights_blocks);
}

// blocks of `per` items each, at most eight per SM: the kernels walk the rest
int grid_for(const som_layers* l, int64_t items, int per)
{
    const int64_t want = (items + per - 1) / per, most = (int64_t)l->sm_count * 8;
    return (int)(want < 1 ? 1 : want < most ? want : most);
}

}  // namespace

cudaError_t prepare_plan()
{
    return cudaFuncSetAttribute(k_slot_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, (PLAN_WARPS + 1) * 1024 * (int)sizeof(int));
}

// One block for up to 4096 slots (5 to 12 us; three launches take about 14), blocks of PLACE_SLOTS beyond.
int plan_blocks(int64_t slots) { return slots <= 4096 ? 0 : (int)((slots + PLACE_SLOTS - 1) / PLACE_SLOTS); }

int launch_plan(som_layers* l, const SlotPlan& p, const int32_t* indices, const void* weights, int weights_type, int64_t T,
                int k, int E, cudaStream_t st)
{
    const int blocks = plan_blocks(T * k);
    if (blocks == 0) {
        const size_t smem = (size_t)(PLAN_WARPS + 1) * E * sizeof(int);
        return outcome(l, launch(l, k_slot_plan, dim3(1), PLAN_THREADS, smem, st, 1, p, indices, weights, weights_type, T * k, E, l->flags));
    }
    cudaError_t e = launch(l, k_slot_count, dim3(blocks), 32 * PLACE_WARPS, (size_t)E * sizeof(int), st, 1, indices, T * k, E, p.block_counts, l->flags);
    if (e == cudaSuccess) e = launch(l, k_slot_segments, dim3(1), PLAN_THREADS, 0, st, 1, p, E, blocks, p.block_counts);
    if (e == cudaSuccess)
        e = launch(l, k_slot_place, dim3(blocks), 32 * PLACE_WARPS, (size_t)PLACE_WARPS * E * sizeof(int), st, 1, p, indices, weights, weights_type,
                   T * k, E, p.block_counts);
    return outcome(l, e);
}

int launch_gather(som_layers* l, const SlotPlan& p, int64_t slots, int E, int k, int64_t D, const void* x, int64_t ldx, void* xp,
                  const void* dy, int64_t lddy, void* dyp, cudaStream_t st)
{
    const int zeros = dy != nullptr;
    const dim3 grid(grid_for(l, slots + (zeros ? (int64_t)E * 64 : 0), 8), 1, dy ? 2 : 1);
    return outcome(l, launch(l, k_gather, grid, 256, 0, st, 1, p, slots, E, k, (int)D, static_cast<const uint16_t*>(x), ldx,
                             static_cast<uint16_t*>(xp), static_cast<const uint16_t*>(dy), lddy, static_cast<uint16_t*>(dyp), zeros));
}

int launch_ends(som_layers* l, EndArgs a, cudaStream_t st)
{
    a.join_blocks = a.y ? grid_for(l, a.T * (a.D / 8), 256) : 0;
    a.dweights_blocks = a.dweights ? grid_for(l, a.T * a.k, 8) : 0;
    a.sums_blocks = a.sums_out ? a.E * ((a.sums_cols + 31) / 32) : 0;
    a.v_blocks = a.v_sums ? a.E * ((a.v_cols + 63) / 64) : 0;
    const int64_t blocks = (int64_t)a.join_blocks + a.dweights_blocks + a.sums_blocks + a.v_blocks;
    // (blocks without shared memory are brought in while the products still have theirs: 3 us of a join after products)
    const size_t smem = a.v_blocks ? 32 * 65 * sizeof(float) : a.sums_blocks ? 8 * 33 * sizeof(float) : 0;
    return outcome(l, launch(l, k_ends, dim3((unsigned)blocks), 256, smem, st, 1, a));
}

}  // namespace lay
