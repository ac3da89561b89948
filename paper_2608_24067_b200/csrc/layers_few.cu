// The linear unit for a handful of rows, on the CUDA cores: single tokens while decoding.
//
// With so few rows a weight is used once or a few times, so the weights' bytes are all that counts and the tensor cores'
// tiles would be almost empty.  A warp owns one output feature (its gate row and its other row together) and reads those
// weight rows once, 16 bytes a lane and several loads in flight, against the tokens' rows in shared memory; a few warps
// share a feature where there are too few features to keep the memory busy.  k_few computes act(x W^T + b) (+ residual),
// for one group of rows (som_linear) or for every slot with its expert's weights (som_experts, first product); k_few_down
// the experts' second product, one warp an output of one token over all of the token's experts, so that neither a join nor a
// second pass over y follows.  The experts' hidden values stay in fp32 between the two.
//
// Bound by HBM and the launch: one row against 4096 gated features of 4096 takes 13.5 us a call (67 MB, 5.0 TB/s with the launch; 17 us
// alone under a profiler); one token's 8 of 64 experts of 2048 x 1024, both kernels, 25.4 us (101 MB, 4.0 TB/s).
#include "layers_few.cuh"
#include "layers_math.cuh"

namespace lay {
namespace {

constexpr int FEW_WARPS = 8, FEW_THREADS = 32 * FEW_WARPS;
__host__ __device__ constexpr int few_resident(int rows) { return rows <= 2 ? 3 : 2; }  // by its registers
constexpr int DOWN_WARPS = 24, DOWN_THREADS = 32 * DOWN_WARPS;  // k_few_down: one block an SM shares the token's hidden values

// weights are read once: past L1
__device__ __forceinline__ uint4 stream16(const uint16_t* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

__device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// ROWS rows of x against one feature a warp; HALVES = 2 when gated.  `share` warps of the block split the sum over D.
// Blocks stay and walk the features, and a weight's place in the registers is loaded again as soon as it has been used, with
// the next feature's weights at the end of a row: the loads never drain.
template <int ROWS, int HALVES>
__global__ void __launch_bounds__(FEW_THREADS, few_resident(ROWS)) k_few(const FewArgs a)
{
    extern __shared__ __align__(16) uint16_t xs[];  // [ROWS][D]
    __shared__ float part[FEW_WARPS][ROWS * HALVES];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    enter();
    int64_t first = 0;  // first row of x and of the output
    const uint16_t *w = a.w, *bias = a.bias;
    float weight = 1.f;
    if (a.indices) {  // one slot a block column
        const int e = a.indices[blockIdx.y];
        if (e < 0 || e >= a.E) {
            if ((e < -1 || e >= a.E) && threadIdx.x == 0 && blockIdx.x == 0) atomicOr(a.flags, LAY_FLAG_BAD_EXPERT);
            return;
        }
        first = blockIdx.y / a.k;
        w += (size_t)e * (HALVES * a.F) * a.D;
        if (bias) bias += (size_t)e * HALVES * a.F;
        weight = a.weights_type == SOM_F32 ? static_cast<const float*>(a.weights)[blockIdx.y]
                                           : unpack1(static_cast<const uint16_t*>(a.weights)[blockIdx.y], a.weights_type == SOM_BF16);
    }
    constexpr int DEEP = 8 / HALVES;  // eight 16-byte loads in flight
    const int share = a.share, features = FEW_WARPS / share, part_of = warp % share;
    const int step = 256 * share, rounds = (a.D + DEEP * step - 1) / (DEEP * step);
    const int c0 = part_of * 256 + lane * 8, stride = gridDim.x * features;
    uint4 buf[DEEP][HALVES];
    auto fetch = [&](int f, int round, int i) {
        const int c = c0 + (round * DEEP + i) * step;
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
            buf[i][h] = f < a.F && c < a.D ? stream16(w + (size_t)(f + h * a.F) * a.D + c) : make_uint4(0u, 0u, 0u, 0u);
    };
    int f = blockIdx.x * features + warp / share;
#pragma unroll
    for (int i = 0; i < DEEP; ++i) fetch(f, 0, i);  // the first weights travel while the rows of x are brought in
    for (int i = threadIdx.x; i < ROWS * (a.D / 8); i += FEW_THREADS) {
        const int r = ROWS == 1 ? 0 : i / (a.D / 8), q = ROWS == 1 ? i : i % (a.D / 8);
        *reinterpret_cast<uint4*>(xs + (size_t)i * 8) =
            r < a.rows ? *(reinterpret_cast<const uint4*>(a.x + (size_t)(first + r) * a.ldx) + q) : make_uint4(0u, 0u, 0u, 0u);
    }
    __syncthreads();
    for (int f_block = blockIdx.x * features; f_block < a.F; f_block += stride, f += stride) {
        float acc[ROWS][HALVES];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int h = 0; h < HALVES; ++h) acc[r][h] = 0.f;
        for (int round = 0; round < rounds; ++round) {
            const bool last = round + 1 == rounds;
            const int next_f = last ? f + stride : f, next_round = last ? 0 : round + 1;
#pragma unroll
            for (int i = 0; i < DEEP; ++i) {
                const int c = c0 + (round * DEEP + i) * step;
                float wv[HALVES][8];
#pragma unroll
                for (int h = 0; h < HALVES; ++h) widen8(buf[i][h], wv[h], a.bf16);
                fetch(next_f, next_round, i);
                if (c < a.D) {
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) {
                        float xv[8];
                        load8(xs + (size_t)r * a.D + c, xv, a.bf16);
#pragma unroll
                        for (int h = 0; h < HALVES; ++h)
#pragma unroll
                            for (int j = 0; j < 8; ++j) acc[r][h] = fmaf(wv[h][j], xv[j], acc[r][h]);
                    }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int h = 0; h < HALVES; ++h) acc[r][h] = lanes_sum(acc[r][h]);
        if (share > 1) {  // the warps' parts, added in their order
            __syncthreads();  // the last feature's parts have been read
            if (lane == 0) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) part[warp][r * HALVES + h] = acc[r][h];
            }
            __syncthreads();
            if (part_of) continue;
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int h = 0; h < HALVES; ++h) {
                    float s = part[warp][r * HALVES + h];
                    for (int i = 1; i < share; ++i) s += part[warp + i][r * HALVES + h];
                    acc[r][h] = s;
                }
        }
        if (f >= a.F || lane >= a.rows) continue;
        float z = acc[0][0], u = HALVES == 2 ? acc[0][HALVES - 1] : 1.f;  // lane r: row r
#pragma unroll
        for (int r = 1; r < ROWS; ++r)
            if (lane == r) {
                z = acc[r][0];
                if (HALVES == 2) u = acc[r][HALVES - 1];
            }
        if (bias) {
            z += unpack1(*(bias + f), a.bf16);
            if (HALVES == 2) u += unpack1(*(bias + a.F + f), a.bf16);
        }
        float y = 0.f;
        with_act(a.act, [&](auto tag) { y = act_of<decltype(tag)::value>(z); });
        if (HALVES == 2) y *= u;
        if (a.hidden) {
            a.hidden[(size_t)blockIdx.y * a.F + f] = y * weight;
        } else {
            if (a.residual) y += unpack1(*(a.residual + (size_t)lane * a.ldr + f), a.bf16);
            a.y[(size_t)lane * a.ldy + f] = (uint16_t)pack2(y, 0.f, a.bf16);
        }
    }
}

// y[t][d] = residual + sum_j (<w2[e_j][d], hidden[t, j]> + weight_j b2[e_j][d]); `share` warps of the block share an output,
// each a part of the k * I products.  Blocks stay, as above: the token's hidden values are brought in once a block.  The
// first weights are read before the kernel in front, which writes the hidden values, is waited for.  (What that overlaps is its end: a
// block here takes 768 x 72 registers, and comes in on an SM when k_few's blocks there, 61440 registers together, have left.)
__global__ void __launch_bounds__(DOWN_THREADS, 1) k_few_down(const FewDownArgs a)
{
    extern __shared__ __align__(16) float hs[];  // [k][2][I / 2]: of every eight values the first four, then the other four
    __shared__ float part[DOWN_WARPS];
    __shared__ int64_t base[32];  // the experts' weights, -1 = none
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t t = blockIdx.y;
    // (The kernel before, k_few, was let in only after all earlier work: indices and weights are there.  It does not write them.)
    if (threadIdx.x < a.k) {
        const int e = a.indices[t * a.k + threadIdx.x];
        base[threadIdx.x] = e >= 0 && e < a.E ? (int64_t)e * a.D * a.I : -1;
    }
    __syncthreads();
    constexpr int DEEP = 8;
    const int share = a.share, outputs = DOWN_WARPS / share, part_of = warp % share;
    const int span = (a.I + 255) / 256 * 256, all = a.k * (span / 256);  // pieces of 256 products, a piece within one expert
    const int rounds = (all + DEEP * share - 1) / (DEEP * share), stride = gridDim.x * outputs;
    // a warp's pieces are part_of, part_of + share, ...: place (j, c) of the next one to read and of the next one to use
    struct Place {
        int j, c;
        __device__ __forceinline__ void settle(int span)
        {
            while (c >= span) c -= span, ++j;
        }
    };
    Place from{0, part_of * 256};
    from.settle(span);
    const Place start = from;
    uint4 buf[DEEP];
    auto fetch = [&](int d, uint4& to) {
        const int c = from.c + lane * 8;
        to = make_uint4(0u, 0u, 0u, 0u);
        if (d < a.D && from.j < a.k && c < a.I) {
            const int64_t b = base[from.j];
            if (b >= 0) to = stream16(a.w2 + b + (int64_t)d * a.I + c);
        }
        from.c += 256 * share;
        from.settle(span);
    };
    int d = blockIdx.x * outputs + warp / share;
#pragma unroll
    for (int i = 0; i < DEEP; ++i) fetch(d, buf[i]);
    enter();
    for (int i = threadIdx.x; i < a.k * (a.I / 4); i += DOWN_THREADS) {
        const int j = i / (a.I / 4), q = i - j * (a.I / 4);
        reinterpret_cast<float4*>(hs)[j * (a.I / 4) + (q & 1) * (a.I / 8) + (q >> 1)] =
            base[j] >= 0 ? __ldcg(reinterpret_cast<const float4*>(a.hidden + t * a.k * a.I) + i) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncthreads();
    for (int d_block = blockIdx.x * outputs; d_block < a.D; d_block += stride, d += stride) {
        float acc = 0.f;
        Place use = start;
        for (int round = 0; round < rounds; ++round) {
            const bool last = round + 1 == rounds;
            if (last) from = start;
            const int next_d = last ? d + stride : d;
#pragma unroll
            for (int i = 0; i < DEEP; ++i) {
                float wv[8];
                widen8(buf[i], wv, a.bf16);
                fetch(next_d, buf[i]);
                const int c = use.c + lane * 8;
                if (use.j < a.k && c < a.I) {
                    const float* h = hs + (size_t)use.j * a.I + c / 2;
                    const float4 h0 = *reinterpret_cast<const float4*>(h), h1 = *reinterpret_cast<const float4*>(h + a.I / 2);
                    acc = fmaf(wv[0], h0.x, acc), acc = fmaf(wv[1], h0.y, acc), acc = fmaf(wv[2], h0.z, acc), acc = fmaf(wv[3], h0.w, acc);
                    acc = fmaf(wv[4], h1.x, acc), acc = fmaf(wv[5], h1.y, acc), acc = fmaf(wv[6], h1.z, acc), acc = fmaf(wv[7], h1.w, acc);
                }
                use.c += 256 * share;
                use.settle(span);
            }
        }
        acc = lanes_sum(acc);
        if (share > 1) {
            __syncthreads();
            if (lane == 0) part[warp] = acc;
            __syncthreads();
            if (part_of) continue;
            acc = part[warp];
            for (int i = 1; i < share; ++i) acc += part[warp + i];
        }
        if (d >= a.D || lane) continue;
        if (a.b2)
            for (int j = 0; j < a.k; ++j) {
                if (base[j] < 0) continue;
                const float wt = a.weights_type == SOM_F32 ? static_cast<const float*>(a.weights)[t * a.k + j]
                                                           : unpack1(static_cast<const uint16_t*>(a.weights)[t * a.k + j], a.weights_type == SOM_BF16);
                acc = fmaf(wt, unpack1(*(a.b2 + (size_t)a.indices[t * a.k + j] * a.D + d), a.bf16), acc);
            }
        if (a.residual) acc += unpack1(*(a.residual + (size_t)t * a.ldr + d), a.bf16);
        a.y[(size_t)t * a.ldy + d] = (uint16_t)pack2(acc, 0.f, a.bf16);
    }
}

// rows of the instance that takes `rows` rows
int rows_taken(int rows) { return rows <= 2 ? rows : rows <= 4 ? 4 : FEW_ROWS; }

template <int HALVES>
cudaError_t go(som_layers* l, const FewArgs& a, dim3 grid, size_t smem, cudaStream_t st)
{
    switch (rows_taken(a.rows)) {
        case 1: return launch(l, k_few<1, HALVES>, grid, FEW_THREADS, smem, st, 1, a);
        case 2: return launch(l, k_few<2, HALVES>, grid, FEW_THREADS, smem, st, 1, a);
        case 4: return launch(l, k_few<4, HALVES>, grid, FEW_THREADS, smem, st, 1, a);
        default: return launch(l, k_few<FEW_ROWS, HALVES>, grid, FEW_THREADS, smem, st, 1, a);
    }
}

template <int HALVES>
cudaError_t allow()
{
    cudaError_t e = cudaFuncSetAttribute(k_few<1, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_few<2, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_few<4, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_few<8, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM);
    return e;
}

// Warps that share an output: as many as it takes for three outputs' parts to every resident warp (24 on an SM), so that
// the last ones do not leave the others idle for long, each part no shorter than the loads that a warp has in flight.
int share_of(const som_layers* l, int64_t outputs, int64_t length, int in_flight)
{
    int s = 1;
    while (s < FEW_WARPS && outputs * s < (int64_t)l->sm_count * 24 * 3 && length / (2 * s) >= in_flight) s *= 2;
    return s;
}

constexpr size_t SM_SMEM = 228 * 1024, FEW_STATIC = 2048;  // shared memory of an SM; more than k_few's own and what a block reserves

// Blocks for `outputs` of them, `each` a block at a time, in `groups` columns: no more than are resident.
dim3 few_grid(const som_layers* l, int64_t outputs, int each, int64_t groups, int per_sm)
{
    const int64_t want = (outputs + each - 1) / each, most = (int64_t)l->sm_count * per_sm / groups;
    return dim3((unsigned)(want < most ? want : most > 0 ? most : 1), (unsigned)groups);
}

}  // namespace

cudaError_t prepare_few()
{
    cudaError_t e = allow<1>();
    if (e == cudaSuccess) e = allow<2>();
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_few_down, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM);
    return e;
}

int launch_few(som_layers* l, FewArgs a, int groups, bool gated, cudaStream_t st)
{
    a.share = share_of(l, (int64_t)a.F * groups, (int64_t)a.D, gated ? 1024 : 2048);
    const size_t smem = (size_t)rows_taken(a.rows) * a.D * 2;
    // With a third block an SM for more than two rows, where two are resident, the last third of the blocks brought the rows in once
    // more and ran by itself: 4 rows, 4096 -> 4096, 20 us instead of 17, gated 34 instead of 26; 8 rows gated 62 instead of 47.
    const int by_smem = (int)(SM_SMEM / (smem + FEW_STATIC)), by_registers = few_resident(rows_taken(a.rows));
    const dim3 grid = few_grid(l, a.F, FEW_WARPS / a.share, groups, by_smem < by_registers ? by_smem : by_registers);
    return outcome(l, gated ? go<2>(l, a, grid, smem, st) : go<1>(l, a, grid, smem, st));
}

int launch_few_down(som_layers* l, FewDownArgs a, int64_t T, cudaStream_t st)
{
    a.share = share_of(l, a.D * T, (int64_t)a.k * a.I, 2048);
    return outcome(l, launch(l, k_few_down, few_grid(l, a.D, DOWN_WARPS / a.share, T, 1), DOWN_THREADS, (size_t)a.k * a.I * sizeof(float), st, 1, a));
}

}  // namespace lay
