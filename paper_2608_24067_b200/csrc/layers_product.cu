// Matrix products of the dense operators on the 5th-generation tensor cores.
//
// One persistent block per SM walks the output tiles (128 rows x 256 columns of accumulator).  Warp 0 issues the TMA
// copies of a four-stage ring (64 k of both operands a stage, 48 KB, 128-byte swizzle), warp 1 issues the matrix
// instructions (tcgen05.mma, 128 x 256 x 16, fp32 accumulators in tensor memory), eight warps run the epilogue.  The
// accumulator is double-buffered (2 x 256 of the 512 columns of tensor memory), so that the epilogue of a tile runs
// under the products of the next; PROD_DZ_PAIR keeps two products of a tile side by side and has one buffer.  Operands
// enter K-major (a row holds consecutive k) or M/N-major (a row holds consecutive rows of the product), as they lie in
// memory: no operand is transposed beforehand.  Every wait is bounded.
#include "layers_math.cuh"
#include "layers_product.cuh"
#include "layers_ptx.cuh"

namespace lay {
namespace {

constexpr int BM = 128, BN = 256, BK = 64, STAGES = 4;
constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int BOX = 64 * 128;  // bytes of a box of 64 rows
constexpr int EPI_WARPS = 8, THREADS = 32 * (2 + EPI_WARPS);
constexpr int OUT_BYTES = 32 * 128;  // an epilogue warp's staged output: 32 rows of 128 bytes
constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + EPI_WARPS * OUT_BYTES;

struct Tile {
    int row, col, expert;  // first row and column of the output, expert
    int k0, k;             // PROD_DW: first row of the sum and its length
};

template <int MODE>
__device__ __forceinline__ int tile_count(const ProdArgs& p)
{
    if (MODE == PROD_DW) return p.experts * p.row_tiles * p.col_tiles;
    return (p.tiles ? *p.tiles : p.row_tiles) * p.col_tiles;
}

template <int MODE>
__device__ __forceinline__ Tile tile_at(const ProdArgs& p, int idx, int width)
{
    Tile t;
    if (MODE == PROD_DW) {
        const int per = p.row_tiles * p.col_tiles;
        t.expert = idx / per;
        const int rest = idx - t.expert * per;
        t.row = (rest / p.col_tiles) * BM;
        t.col = (rest % p.col_tiles) * width;
        t.k0 = p.seg ? p.seg[t.expert] : 0;
        t.k = p.seg ? p.seg[t.expert + 1] - t.k0 : p.k1;
    } else {
        const int rt = idx / p.col_tiles;
        t.row = rt * BM;
        t.col = (idx - rt * p.col_tiles) * width;
        t.expert = p.tile_expert ? p.tile_expert[rt] : 0;
        t.k0 = 0;
        t.k = p.k1;
    }
    return t;
}

// An epilogue warp's way out: 32 rows (lane l holds row l) of 32 columns are staged in shared memory and stored by TMA,
// which leaves out what lies outside the tensor.  16-bit pieces (64-byte rows, 64-byte swizzle) alternate between the
// two halves of the buffer, so that a piece is staged while the one before is read; fp32 pieces (128-byte rows) fill it.
struct Stager {
    unsigned char* buf;
    int lane, turn;
    __device__ __forceinline__ void put16(const CUtensorMap* map, const float (&v)[32], int col, int row, int batch, const ProdArgs& p)
    {
        unsigned char* to = buf + turn * (OUT_BYTES / 2);
        turn ^= 1;
        if (lane == 0) store_wait_read<1>();
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint4 u;
            u.x = pack2(v[8 * j], v[8 * j + 1], p.bf16);
            u.y = pack2(v[8 * j + 2], v[8 * j + 3], p.bf16);
            u.z = pack2(v[8 * j + 4], v[8 * j + 5], p.bf16);
            u.w = pack2(v[8 * j + 6], v[8 * j + 7], p.bf16);
            *reinterpret_cast<uint4*>(to + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = u;
        }
        send(map, to, col, row, batch, p);
    }
    __device__ __forceinline__ void put32(const CUtensorMap* map, const float (&v)[32], int col, int row, int batch, const ProdArgs& p)
    {
        if (lane == 0) store_wait_read<0>();
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j)
            *reinterpret_cast<float4*>(buf + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        send(map, buf, col, row, batch, p);
    }
    __device__ __forceinline__ void send(const CUtensorMap* map, const unsigned char* from, int col, int row, int batch, const ProdArgs& p)
    {
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
            if (col < p.cols && row < p.rows) tma_store(map, from, col, row, batch);
            store_commit();
        }
    }
};

// v[j] += bias[col + j] * s for the columns below `cols` (a multiple of 8)
__device__ __forceinline__ void add_row(float (&v)[32], const uint16_t* bias, int col, int cols, float s, int bf16)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (col + 8 * j < cols) {
            float b[8];
            load8(bias + col + 8 * j, b, bf16);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[8 * j + i] = fmaf(b[i], s, v[8 * j + i]);
        }
}

template <int MODE>
__global__ void __launch_bounds__(THREADS, 1) k_product(const __grid_constant__ ProdArgs p)
{
    constexpr bool A_MN = MODE == PROD_DW, B_MN = MODE == PROD_DX || MODE == PROD_DW;
    constexpr int BUFFERS = MODE == PROD_DZ_PAIR ? 1 : 2;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty[2], drained;
    __shared__ uint32_t tmem_sh;
    __shared__ int gave_up_sh;
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    unsigned char* staged = ring + STAGES * STAGE_BYTES;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            bar_init(&full[i], 1);
            bar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(&acc_full[i], 1);
            bar_init(&acc_empty[i], EPI_WARPS);
        }
        bar_init(&drained, 1);
        gave_up_sh = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(&tmem_sh, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_sh;
    volatile int* gave_up = &gave_up_sh;

    const bool gated = p.gate_rows != 0;
    // output columns of a tile: a gated product spends half of the accumulator's columns on the other half of its rows
    const int width = gated && (MODE == PROD_FWD || MODE == PROD_DZ || MODE == PROD_DZ_PAIR) ? BN / 2 : BN;
    const int total = tile_count<MODE>(p);
    const int n2 = width;  // columns of the second product of PROD_DZ_PAIR

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            int64_t issued = 0;
            bool ok = true;
            for (int idx = blockIdx.x; ok && idx < total; idx += gridDim.x) {
                const Tile t = tile_at<MODE>(p, idx, width);
                const int it1 = (t.k + BK - 1) / BK, it2 = MODE == PROD_DZ_PAIR ? (p.k2 + BK - 1) / BK : 0;
                for (int it = 0; it < it1 + it2; ++it) {
                    if (!bar_wait(&empty[stage], phase ^ 1u, gave_up)) {
                        ok = false;
                        break;
                    }
                    unsigned char* sa = ring + stage * STAGE_BYTES;
                    unsigned char* sb = sa + A_BYTES;
                    uint64_t* bar = &full[stage];
                    if (MODE == PROD_DZ_PAIR && it >= it1) {
                        const int k = (it - it1) * BK;
                        bar_expect(bar, A_BYTES + n2 * BK * 2);
                        tma_load(sa, &p.a2, bar, k, t.row, 0);
                        for (int j = 0; j < n2 / 64; ++j) tma_load(sb + j * BOX, &p.b2, bar, t.col + 64 * j, k, t.expert);
                    } else {
                        const int k = t.k0 + it * BK;
                        bar_expect(bar, STAGE_BYTES);
                        if (A_MN) {
                            tma_load(sa, &p.a, bar, t.row, k, 0);
                            tma_load(sa + BOX, &p.a, bar, t.row + 64, k, 0);
                        } else {
                            tma_load(sa, &p.a, bar, k, t.row, 0);
                        }
                        if (B_MN) {
                            for (int j = 0; j < 4; ++j)
                                tma_load(sb + j * BOX, &p.b, bar, t.col + 64 * j, k, MODE == PROD_DW ? 0 : t.expert);
                        } else {
                            tma_load(sb, &p.b, bar, k, t.col, t.expert);
                            tma_load(sb + 2 * BOX, &p.b, bar, k, gated ? t.col + p.gate_rows : t.col + 128, t.expert);
                        }
                    }
                    ++issued;
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
            if (!ok) {  // copies still in flight write this block's shared memory: let them land before it leaves
                const long long t0 = clock64();
                for (int s = 0; s < STAGES; ++s) {
                    const int64_t uses = issued / STAGES + (s < (int)(issued % STAGES) ? 1 : 0);
                    while (uses > 0 && !bar_try(&full[s], (uint32_t)(uses - 1) & 1u) && clock64() - t0 < WAIT_CYCLES) {}
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            int stage = 0, n_acc = 0;
            uint32_t phase = 0;
            bool ok = true;
            const uint32_t idesc1 = mma_desc(p.bf16, A_MN, B_MN, BM, BN);
            const uint32_t idesc2 = mma_desc(p.bf16, 0, 1, BM, n2);
            for (int idx = blockIdx.x; ok && idx < total; idx += gridDim.x, ++n_acc) {
                const Tile t = tile_at<MODE>(p, idx, width);
                const int buf = BUFFERS == 2 ? n_acc & 1 : 0;
                const uint32_t use = (uint32_t)(n_acc / BUFFERS) & 1u;
                if (!bar_wait(&acc_empty[buf], use ^ 1u, gave_up)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const int it1 = (t.k + BK - 1) / BK, it2 = MODE == PROD_DZ_PAIR ? (p.k2 + BK - 1) / BK : 0;
                for (int it = 0; it < it1 + it2; ++it) {
                    if (!bar_wait(&full[stage], phase, gave_up)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t sa = smem_addr(ring + stage * STAGE_BYTES), sb = sa + A_BYTES;
                    const bool second = MODE == PROD_DZ_PAIR && it >= it1;
                    const uint32_t d = tmem + (uint32_t)(buf * BN) + (second ? (uint32_t)BN : 0u);
                    const bool first = it == 0 || (MODE == PROD_DZ_PAIR && it == it1);
#pragma unroll
                    for (int kk = 0; kk < BK / 16; ++kk) {
                        const uint64_t da = A_MN ? mat_desc(sa + kk * 2048, BOX, 1024) : mat_desc(sa + kk * 32, 16, 1024);
                        const uint64_t db =
                            B_MN || second ? mat_desc(sb + kk * 2048, BOX, 1024) : mat_desc(sb + kk * 32, 16, 1024);
                        mma(d, da, db, second ? idesc2 : idesc1, !(first && kk == 0));
                    }
                    mma_commit(&empty[stage]);
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                mma_commit(&acc_full[buf]);
            }
            if (!ok) {  // instructions in flight read shared memory and write tensor memory
                mma_commit(&drained);
                const long long t0 = clock64();
                while (!bar_try(&drained, 0) && clock64() - t0 < WAIT_CYCLES) {}
            }
        }
    } else {
        const int w = warp - 2, q = warp & 3, half = w >> 2;  // a warp may read the 32 lanes of its quarter only
        Stager s{staged + w * OUT_BYTES, lane, 0};
        int n_acc = 0;
        for (int idx = blockIdx.x; idx < total; idx += gridDim.x, ++n_acc) {
            const Tile t = tile_at<MODE>(p, idx, width);
            const int buf = BUFFERS == 2 ? n_acc & 1 : 0;
            if (!bar_wait(&acc_full[buf], (uint32_t)(n_acc / BUFFERS) & 1u, gave_up)) break;
            __syncwarp();
            tc_fence_after();
            const uint32_t acc = tmem + (uint32_t)(buf * BN) + ((uint32_t)(32 * q) << 16);
            const int row0 = t.row + 32 * q, row = row0 + lane;
            const bool inside = row < p.rows;
            const bool counts = inside && (!p.row_slot || p.row_slot[row] >= 0);
            const float rw = p.row_weight && inside ? p.row_weight[row] : 1.f;
            const uint16_t* bias = p.bias ? p.bias + (size_t)t.expert * p.bias_ld : nullptr;

            if (MODE == PROD_FWD || MODE == PROD_DX || MODE == PROD_DW) {
                const int each = width / 2;  // columns of this warp
#pragma unroll 1
                for (int c = 0; c < each; c += 32) {
                    const int at = half * each + c, col = t.col + at;
                    float v[32];
                    tmem_ld32(acc + at, v);
                    if (MODE == PROD_FWD && gated) {
                        float u[32];
                        tmem_ld32(acc + BN / 2 + at, u);
                        tmem_wait_ld();
                        if (bias) {
                            add_row(v, bias, col, p.cols, 1.f, p.bf16);
                            add_row(u, bias + p.gate_rows, col, p.cols, 1.f, p.bf16);
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = act_of(v[j], p.act) * u[j];
                    } else {
                        tmem_wait_ld();
                        if (MODE == PROD_DW && t.k == 0) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = 0.f;  // an expert without a token: nothing was summed
                        }
                        if (MODE == PROD_FWD) {
                            if (bias) add_row(v, bias, col, p.cols, p.weigh == 2 ? rw : 1.f, p.bf16);
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = act_of(v[j], p.act);
                        }
                    }
                    if (MODE == PROD_FWD) {
                        if (p.extra && inside) add_row(v, p.extra + (size_t)row * p.ld_extra, col, p.cols, 1.f, p.bf16);
                        if (p.weigh == 1) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = counts ? v[j] * rw : 0.f;
                        }
                    }
                    if (p.out32) s.put32(&p.o0, v, col, row0, MODE == PROD_DW ? t.expert : 0, p);
                    else s.put16(&p.o0, v, col, row0, MODE == PROD_DW ? t.expert : 0, p);
                }
            } else {
                // PROD_DZ, PROD_DZ_PAIR.  dh = the gradient that reaches the activation's output.
                const int each = width / 2;
                float dot = 0.f;
#pragma unroll 1
                for (int c = 0; c < each; c += 32) {
                    const int at = half * each + c, col = t.col + at;
                    float v[32], u[32], g[32];
                    tmem_ld32(acc + at, v);
                    if (gated) tmem_ld32(acc + BN / 2 + at, u);
                    if (MODE == PROD_DZ_PAIR) tmem_ld32(acc + BN + at, g);
                    tmem_wait_ld();
                    if (bias) {
                        add_row(v, bias, col, p.cols, 1.f, p.bf16);
                        if (gated) add_row(u, bias + p.gate_rows, col, p.cols, 1.f, p.bf16);
                    }
                    if (MODE == PROD_DZ) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) g[j] = 0.f;
                        if (inside) add_row(g, p.extra + (size_t)row * p.ld_extra, col, p.cols, 1.f, p.bf16);
                    }
                    // v: z (or the gate) -> dz of it; u: the gated half -> dz of it; hidden values on the way
                    float hid[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        float a, da;
                        act_both(v[j], p.act, a, da);
                        const float other = gated ? u[j] : 1.f;
                        const float hj = a * other;
                        if (MODE == PROD_DZ_PAIR) {
                            if (col + j < p.cols) dot = fmaf(hj, g[j], dot);
                            hid[j] = counts ? hj * rw : 0.f;
                            g[j] = counts ? g[j] * rw : 0.f;
                        }
                        v[j] = counts ? g[j] * other * da : 0.f;
                        if (gated) u[j] = counts ? g[j] * a : 0.f;
                    }
                    s.put16(&p.o0, v, col, row0, 0, p);
                    if (gated) s.put16(&p.o1, u, col, row0, 0, p);
                    if (MODE == PROD_DZ_PAIR) s.put16(&p.o2, hid, col, row0, 0, p);
                }
                if (MODE == PROD_DZ_PAIR && inside)
                    p.dot[(size_t)row * (2 * p.col_tiles) + 2 * (t.col / width) + half] = dot;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(&acc_empty[buf]);
        }
        if (lane == 0) store_wait_all();
    }
    __syncthreads();
    if (threadIdx.x == 0 && gave_up_sh) atomicOr(p.flags, LAY_FLAG_GAVE_UP);
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_free(tmem, 512);
    }
}

template <int MODE>
int launch_mode(som_layers* l, const ProdArgs& args, cudaStream_t st)
{
    cudaError_t e = cudaFuncSetAttribute(k_product<MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e == cudaSuccess) {
        int64_t most = (int64_t)args.row_tiles * args.col_tiles * (MODE == PROD_DW ? args.experts : 1);
        const int grid = (int)(most < l->sm_count ? most : l->sm_count);
        k_product<MODE><<<grid, THREADS, SMEM, st>>>(args);
        ++l->launches;
        e = cudaGetLastError();
    }
    if (e != cudaSuccess) {
        l->last_cuda_error = (int)e;
        return SOM_ERR_CUDA;
    }
    return SOM_OK;
}

}  // namespace

int launch_product(som_layers* l, ProdMode mode, const ProdArgs& args, cudaStream_t st)
{
    switch (mode) {
        case PROD_FWD: return launch_mode<PROD_FWD>(l, args, st);
        case PROD_DZ: return launch_mode<PROD_DZ>(l, args, st);
        case PROD_DZ_PAIR: return launch_mode<PROD_DZ_PAIR>(l, args, st);
        case PROD_DX: return launch_mode<PROD_DX>(l, args, st);
        default: return launch_mode<PROD_DW>(l, args, st);
    }
}

}  // namespace lay
