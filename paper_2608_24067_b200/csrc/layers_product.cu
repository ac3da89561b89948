// Matrix products of the dense operators on the 5th-generation tensor cores.
//
// Persistent blocks, one per SM, walk the output tiles.  Warp 0 issues the TMA copies of a six-stage ring (64 k of both
// operands a stage, 32 KB, 128-byte swizzle), warp 1 issues the matrix instructions (tcgen05.mma, fp32 accumulators in
// tensor memory), eight warps run the epilogue.  The accumulator is double-buffered, so that the epilogue of a tile runs
// under the products of the next; PROD_DZ_TWO keeps two products of a tile side by side and has one buffer.  Operands enter
// K-major (a row holds consecutive k) or M/N-major (a row holds consecutive rows of the product), as they lie in memory: no
// operand is transposed beforehand.  Every wait is bounded.
//
// Two tile shapes.  PAIR: two blocks of a cluster share a tile of 256 x 256; each loads its own 128 rows of A and one half of
// B, and the matrix instruction reads both halves (cta_group::2).  A single block on 128 x 256 moves 48 KB into and 48 KB out
// of its shared memory for 512 clocks of matrix work, 192 bytes a clock where shared memory gives 128: 4096 x 4096 x 4096
// took 134 us so.  With the pair it is 32 KB each way, 128 bytes a clock.  SINGLE: 128 x 128 by one block, for products
// that have too few tiles to fill the SMs with pairs or too few rows per expert.
#include "layers_math.cuh"
#include "layers_product.cuh"
#include "layers_ptx.cuh"

namespace lay {
namespace {

constexpr int BM = 128, BK = 64, STAGES = 6;
constexpr int HALF = 128 * BK * 2;  // bytes of a block's share of an operand in a stage
constexpr int STAGE_BYTES = 2 * HALF;
constexpr int BOX = 64 * 128;  // bytes of a box of 64 rows
constexpr int EPI_WARPS = 8, THREADS = 32 * (2 + EPI_WARPS);
constexpr int OUT_BYTES = 32 * 128;  // an epilogue warp's staged output: 32 rows of 128 bytes
constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + EPI_WARPS * OUT_BYTES;

struct Tile {
    int row, col, expert;  // this block's first row and the tile's first column of the output, expert
    int k0, k;             // PROD_DW: first row of the sum; length of the first product's sum
    int live, store;       // rows below `live` are in use, rows below `store` are written (zeros from `live` on)
};

__device__ __forceinline__ int round64(int n) { return (n + 63) & ~63; }

template <int MODE>
__device__ __forceinline__ int tile_count(const ProdArgs& p)
{
    if (MODE == PROD_DW) return p.experts * p.row_tiles * p.col_tiles;
    return (p.tiles ? *p.tiles : p.row_tiles) * p.col_tiles;
}

template <int MODE, bool PAIR>
__device__ __forceinline__ Tile tile_at(const ProdArgs& p, int idx, int width, int rank)
{
    constexpr int ROWS = PAIR ? PAIR_ROWS : SINGLE_ROWS;
    Tile t;
    if (MODE == PROD_DW) {
        const int per = p.row_tiles * p.col_tiles;
        t.expert = idx / per;
        const int rest = idx - t.expert * per, rt = rest / p.col_tiles;
        t.row = rt * ROWS + rank * BM;
        t.col = (rest - rt * p.col_tiles) * width;
        t.k0 = p.seg ? p.seg[t.expert] : 0;
        t.k = p.seg ? round64(p.count[t.expert]) : p.k1;
        t.live = t.store = p.rows;
    } else {
        const int rt = idx / p.col_tiles;
        t.row = rt * ROWS + rank * BM;
        t.col = (idx - rt * p.col_tiles) * width;
        t.expert = p.tile_expert ? p.tile_expert[rt] : 0;
        t.k0 = 0;
        t.k = p.k1;
        t.live = t.store = p.rows;
        if (p.seg) {
            const int s = p.seg[t.expert], n = p.count[t.expert];
            t.live = s + n;
            // the sums over an expert's rows (PROD_DW) run over whole steps of 64 rows
            t.store = MODE == PROD_DZ_TWO ? s + round64(n) : t.live;
        }
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

// 32 values of a row of a 16-bit matrix, fetched before they are needed; zeros beyond `cols` (a multiple of 8)
struct Row32 {
    uint4 w[4];
    __device__ __forceinline__ void fetch(const uint16_t* row, int col, int cols, bool want)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = want && col + 8 * j < cols ? __ldg(reinterpret_cast<const uint4*>(row + col) + j) : make_uint4(0u, 0u, 0u, 0u);
    }
    // v += s * values
    __device__ __forceinline__ void add(float (&v)[32], float s, int bf16) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t u[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = unpack2(u[i], bf16);
                v[8 * j + 2 * i] = fmaf(f.x, s, v[8 * j + 2 * i]);
                v[8 * j + 2 * i + 1] = fmaf(f.y, s, v[8 * j + 2 * i + 1]);
            }
        }
    }
};

// Lane l holds v[0..31] of row l; returns to lane l the sum of column l over the 32 rows (31 exchanges, fixed order).
__device__ __forceinline__ float column_sum(float (&v)[32], int lane)
{
#pragma unroll
    for (int h = 16; h >= 1; h >>= 1) {
        const bool up = lane & h;
#pragma unroll
        for (int j = 0; j < h; ++j) {
            const float give = up ? v[j] : v[j + h], keep = up ? v[j + h] : v[j];
            v[j] = keep + __shfl_xor_sync(0xffffffffu, give, h);
        }
    }
    return v[0];
}

template <int MODE, bool PAIR>
__global__ void __launch_bounds__(THREADS, 1) k_product(const __grid_constant__ ProdArgs p)
{
    constexpr bool A_MN = MODE == PROD_DW, B_MN = MODE == PROD_DX || MODE == PROD_DW;
    constexpr int BUFFERS = MODE == PROD_DZ_TWO ? 1 : 2;
    constexpr int BN = PAIR ? PAIR_COLS : SINGLE_COLS;
    constexpr uint32_t TMEM_COLUMNS = 2 * BN;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty[2], drained;
    __shared__ uint32_t tmem_sh;
    __shared__ int gave_up_sh;
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    unsigned char* staged = ring + STAGES * STAGE_BYTES;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)cluster_rank() : 0;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            bar_init(&full[i], 1);
            bar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(&acc_full[i], 1);
            bar_init(&acc_empty[i], EPI_WARPS * (PAIR ? 2 : 1));
        }
        bar_init(&drained, 1);
        gave_up_sh = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<PAIR>(&tmem_sh, TMEM_COLUMNS);
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();  // the other block's barriers are ready
    tc_fence_after();
    const uint32_t tmem = tmem_sh;
    volatile int* gave_up = &gave_up_sh;

    const bool gated = p.gate_rows != 0;
    // output columns of a tile: a gated product spends half of the accumulator's columns on the other half of its rows
    const int width = gated && (MODE == PROD_FWD || MODE == PROD_DZ || MODE == PROD_DZ_TWO) ? BN / 2 : BN;
    const int total = tile_count<MODE>(p);
    const int n2 = width;  // columns of the second product of PROD_DZ_TWO
    const int step = PAIR ? gridDim.x >> 1 : gridDim.x, first_tile = PAIR ? blockIdx.x >> 1 : blockIdx.x;
    const int share2 = PAIR ? n2 / 2 : n2;  // columns of the second product's B in this block

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            int64_t issued = 0;
            bool ok = true;
            for (int idx = first_tile; ok && idx < total; idx += step) {
                const Tile t = tile_at<MODE, PAIR>(p, idx, width, rank);
                // first row (K-major) or column of this block's 128 columns of B
                const int b0 = !PAIR ? t.col : gated && !B_MN ? t.col + rank * p.gate_rows : t.col + rank * 128;
                const int b1 = !PAIR && gated && !B_MN ? t.col + p.gate_rows : b0 + 64;
                const int it1 = (t.k + BK - 1) / BK, it2 = MODE == PROD_DZ_TWO ? (p.k2 + BK - 1) / BK : 0;
                for (int it = 0; it < it1 + it2; ++it) {
                    if (!bar_wait(&empty[stage], phase ^ 1u, gave_up)) {
                        ok = false;
                        break;
                    }
                    unsigned char* sa = ring + stage * STAGE_BYTES;
                    unsigned char* sb = sa + HALF;
                    // the leader's barrier counts both blocks' bytes
                    const uint32_t bar = PAIR ? cluster_addr(smem_addr(&full[stage]), 0) : smem_addr(&full[stage]);
                    if (MODE == PROD_DZ_TWO && it >= it1) {
                        const int k = (it - it1) * BK;
                        if (rank == 0) bar_expect(&full[stage], (PAIR ? 2 : 1) * (HALF + share2 * BK * 2));
                        tma_load<PAIR>(sa, &p.a2, bar, k, t.row, 0);
                        for (int j = 0; j < share2; j += 64) tma_load<PAIR>(sb + j * 128, &p.b2, bar, t.col + rank * share2 + j, k, t.expert);
                    } else {
                        const int k = t.k0 + it * BK;
                        if (rank == 0) bar_expect(&full[stage], (PAIR ? 2 : 1) * STAGE_BYTES);
                        if (A_MN) {
                            tma_load<PAIR>(sa, &p.a, bar, t.row, k, 0);
                            tma_load<PAIR>(sa + BOX, &p.a, bar, t.row + 64, k, 0);
                        } else {
                            tma_load<PAIR>(sa, &p.a, bar, k, t.row, 0);
                        }
                        if (B_MN) {
                            tma_load<PAIR>(sb, &p.b, bar, b0, k, MODE == PROD_DW ? 0 : t.expert);
                            tma_load<PAIR>(sb + BOX, &p.b, bar, b1, k, MODE == PROD_DW ? 0 : t.expert);
                        } else {
                            tma_load<PAIR>(sb, &p.b, bar, k, b0, t.expert);
                            tma_load<PAIR>(sb + BOX, &p.b, bar, k, b1, t.expert);
                        }
                    }
                    ++issued;
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
            if (!ok && rank == 0) {  // copies still in flight write shared memory: let them land before the block leaves
                const long long t0 = clock64();
                for (int s = 0; s < STAGES; ++s) {
                    const int64_t uses = issued / STAGES + (s < (int)(issued % STAGES) ? 1 : 0);
                    while (uses > 0 && !bar_try(&full[s], (uint32_t)(uses - 1) & 1u) && clock64() - t0 < WAIT_CYCLES) {}
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            int stage = 0, n_acc = 0;
            uint32_t phase = 0;
            bool ok = true;
            const uint32_t idesc1 = mma_desc(p.bf16, A_MN, B_MN, PAIR ? 256 : 128, BN);
            const uint32_t idesc2 = mma_desc(p.bf16, 0, 1, PAIR ? 256 : 128, n2);
            for (int idx = first_tile; ok && idx < total; idx += step, ++n_acc) {
                const Tile t = tile_at<MODE, PAIR>(p, idx, width, rank);
                const int buf = BUFFERS == 2 ? n_acc & 1 : 0;
                const uint32_t use = (uint32_t)(n_acc / BUFFERS) & 1u;
                if (!bar_wait(&acc_empty[buf], use ^ 1u, gave_up)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const int it1 = (t.k + BK - 1) / BK, it2 = MODE == PROD_DZ_TWO ? (p.k2 + BK - 1) / BK : 0;
                for (int it = 0; it < it1 + it2; ++it) {
                    if (!bar_wait(&full[stage], phase, gave_up)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t sa = smem_addr(ring + stage * STAGE_BYTES), sb = sa + HALF;
                    const bool second = MODE == PROD_DZ_TWO && it >= it1;
                    const uint32_t d = tmem + (uint32_t)(buf * BN) + (second ? (uint32_t)BN : 0u);
                    const bool first = it == 0 || (MODE == PROD_DZ_TWO && it == it1);
#pragma unroll
                    for (int kk = 0; kk < BK / 16; ++kk) {
                        const uint64_t da = A_MN ? mat_desc(sa + kk * 2048, BOX, 1024) : mat_desc(sa + kk * 32, 16, 1024);
                        const uint64_t db =
                            B_MN || second ? mat_desc(sb + kk * 2048, BOX, 1024) : mat_desc(sb + kk * 32, 16, 1024);
                        mma<PAIR>(d, da, db, second ? idesc2 : idesc1, !(first && kk == 0));
                    }
                    mma_commit<PAIR>(&empty[stage]);
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                mma_commit<PAIR>(&acc_full[buf]);
            }
            if (!ok) {  // instructions in flight read shared memory and write tensor memory
                mma_commit<PAIR>(&drained);
                const long long t0 = clock64();
                while (!bar_try(&drained, 0) && clock64() - t0 < WAIT_CYCLES) {}
            }
        }
    } else {
        const int w = warp - 2, q = warp & 3, half = w >> 2;  // a warp may read the 32 lanes of its quarter only
        Stager s{staged + w * OUT_BYTES, lane, 0};
        int n_acc = 0;
        for (int idx = first_tile; idx < total; idx += step, ++n_acc) {
            const Tile t = tile_at<MODE, PAIR>(p, idx, width, rank);
            const int buf = BUFFERS == 2 ? n_acc & 1 : 0;
            const uint32_t acc = tmem + (uint32_t)(buf * BN) + ((uint32_t)(32 * q) << 16);
            const int row0 = t.row + 32 * q, row = row0 + lane;
            const bool counts = row < t.live;
            const float rw = p.row_weight && counts ? p.row_weight[row] : 1.f;
            const uint16_t* bias = p.bias ? p.bias + (size_t)t.expert * p.bias_ld : nullptr;
            const uint16_t* extra = p.extra ? p.extra + (size_t)row * p.ld_extra : nullptr;
            const int each = width / 2;  // columns of this warp
            const int batch = MODE == PROD_DW ? t.expert : 0;
            if (!bar_wait(&acc_full[buf], (uint32_t)(n_acc / BUFFERS) & 1u, gave_up)) break;
            __syncwarp();
            tc_fence_after();
            if (row0 < t.store) {
                float dot = 0.f;
#pragma unroll 1
                for (int c = 0; c < each; c += 32) {
                    const int at = half * each + c, col = t.col + at;
                    Row32 add, b0, b1;
                    if (MODE == PROD_FWD || MODE == PROD_DZ) add.fetch(extra, col, p.cols, extra && counts);
                    if (MODE != PROD_DX && MODE != PROD_DW) {
                        b0.fetch(bias, col, p.cols, bias != nullptr);
                        b1.fetch(bias ? bias + p.gate_rows : bias, col, p.cols, bias && gated);
                    }
                    float v[32], u[32];
                    tmem_ld32(acc + at, v);
                    if (MODE == PROD_DX || MODE == PROD_DW) {
                        tmem_wait_ld();
                        if (MODE == PROD_DW && t.k == 0) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = 0.f;  // an expert without a token: nothing was summed
                        }
                    } else if (MODE == PROD_FWD) {
                        if (gated) {
                            tmem_ld32(acc + BN / 2 + at, u);
                            tmem_wait_ld();
                            if (bias) {
                                b0.add(v, 1.f, p.bf16);
                                b1.add(u, 1.f, p.bf16);
                            }
                            with_act(p.act, [&](auto tag) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) v[j] = act_of<decltype(tag)::value>(v[j]) * u[j];
                            });
                        } else {
                            tmem_wait_ld();
                            if (bias) b0.add(v, p.weigh == 2 ? rw : 1.f, p.bf16);
                            if (p.act != SOM_ACT_NONE)
                                with_act(p.act, [&](auto tag) {
#pragma unroll
                                    for (int j = 0; j < 32; ++j) v[j] = act_of<decltype(tag)::value>(v[j]);
                                });
                        }
                        if (extra) add.add(v, 1.f, p.bf16);
                        if (p.weigh == 1) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] *= rw;
                        }
                    } else {
                        // PROD_DZ, PROD_DZ_TWO: v = z (or the gate's z) becomes dz, u = the gated half's
                        float g[32];
                        if (gated) tmem_ld32(acc + BN / 2 + at, u);
                        if (MODE == PROD_DZ_TWO) tmem_ld32(acc + BN + at, g);
                        tmem_wait_ld();
                        if (bias) {
                            b0.add(v, 1.f, p.bf16);
                            if (gated) b1.add(u, 1.f, p.bf16);
                        }
                        if (MODE == PROD_DZ) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) g[j] = 0.f;
                            add.add(g, 1.f, p.bf16);
                        }
                        float hid[32];
                        with_act(p.act, [&](auto tag) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                float a, da;
                                act_both<decltype(tag)::value>(v[j], a, da);
                                if (gated) {
                                    hid[j] = a * u[j];
                                    v[j] = u[j] * da;
                                    u[j] = a;
                                } else {
                                    hid[j] = a;
                                    v[j] = da;
                                }
                            }
                        });
                        if (MODE == PROD_DZ_TWO) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                if (col + j < p.cols) dot = fmaf(hid[j], g[j], dot);
                                hid[j] = counts ? hid[j] * rw : 0.f;
                                g[j] *= rw;
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            v[j] = counts ? v[j] * g[j] : 0.f;
                            if (gated) u[j] = counts ? u[j] * g[j] : 0.f;
                        }
                        if (MODE == PROD_DZ_TWO) s.put16(&p.o2, hid, col, row0, 0, p);
                        if (gated) s.put16(&p.o1, u, col, row0, 0, p);
                    }
                    if (p.out32) s.put32(&p.o0, v, col, row0, batch, p);
                    else s.put16(&p.o0, v, col, row0, batch, p);
                    if ((MODE == PROD_DZ || MODE == PROD_DZ_TWO) && p.column_sums) {
                        // (outputs were rounded; the sums are over the unrounded values)
                        float* to = p.column_sums + (size_t)(row0 / 32) * (p.cols + p.gate_rows);
                        const float sv = column_sum(v, lane);
                        if (col + lane < p.cols) to[col + lane] = sv;
                        if (gated) {
                            const float su = column_sum(u, lane);
                            if (col + lane < p.cols) to[p.gate_rows + col + lane] = su;
                        }
                    }
                }
                if (MODE == PROD_DZ_TWO && counts) p.dot[(size_t)row * (2 * p.col_tiles) + 2 * (t.col / width) + half] = dot;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIR) bar_arrive_remote(cluster_addr(smem_addr(&acc_empty[buf]), 0));
                else bar_arrive(&acc_empty[buf]);
            }
        }
        if (lane == 0) store_wait_all();
    }
    __syncthreads();
    if (threadIdx.x == 0 && gave_up_sh) atomicOr(p.flags, LAY_FLAG_GAVE_UP);
    __syncwarp();
    if (PAIR) cluster_sync();  // no block leaves while the other may still reach its memory
    if (warp == 1) {
        tc_fence_after();
        tmem_free<PAIR>(tmem, TMEM_COLUMNS);
    }
}

template <int MODE, bool PAIR>
cudaError_t launch_mode(som_layers* l, const ProdArgs& args, cudaStream_t st)
{
    const int64_t tiles = (int64_t)args.row_tiles * args.col_tiles * (MODE == PROD_DW ? args.experts : 1);
    const int most = PAIR ? l->pairs : l->sm_count;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)(tiles < most ? tiles : most) * (PAIR ? 2 : 1));
    c.blockDim = dim3(THREADS);
    c.dynamicSmemBytes = SMEM;
    c.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    c.attrs = attr;
    c.numAttrs = PAIR ? 1 : 0;
    return cudaLaunchKernelEx(&c, k_product<MODE, PAIR>, args);
}

template <int MODE>
cudaError_t prepare_mode(int* pairs)
{
    cudaError_t e = cudaFuncSetAttribute(k_product<MODE, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_product<MODE, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(2);
    c.blockDim = dim3(THREADS);
    c.dynamicSmemBytes = SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    c.attrs = attr;
    c.numAttrs = 1;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, k_product<MODE, true>, &c);
    if (n < *pairs) *pairs = n;
    return e;
}

}  // namespace

cudaError_t prepare_product(som_layers* l)
{
    l->pairs = l->sm_count / 2;
    cudaError_t e = prepare_mode<PROD_FWD>(&l->pairs);
    if (e == cudaSuccess) e = prepare_mode<PROD_DZ>(&l->pairs);
    if (e == cudaSuccess) e = prepare_mode<PROD_DZ_TWO>(&l->pairs);
    if (e == cudaSuccess) e = prepare_mode<PROD_DX>(&l->pairs);
    if (e == cudaSuccess) e = prepare_mode<PROD_DW>(&l->pairs);
    return l->pairs > 0 ? e : cudaErrorNotSupported;
}

int launch_product(som_layers* l, ProdMode mode, const ProdArgs& a, cudaStream_t st)
{
    cudaError_t e;
    switch (mode) {
        case PROD_FWD: e = a.pair ? launch_mode<PROD_FWD, true>(l, a, st) : launch_mode<PROD_FWD, false>(l, a, st); break;
        case PROD_DZ: e = a.pair ? launch_mode<PROD_DZ, true>(l, a, st) : launch_mode<PROD_DZ, false>(l, a, st); break;
        case PROD_DZ_TWO: e = a.pair ? launch_mode<PROD_DZ_TWO, true>(l, a, st) : launch_mode<PROD_DZ_TWO, false>(l, a, st); break;
        case PROD_DX: e = a.pair ? launch_mode<PROD_DX, true>(l, a, st) : launch_mode<PROD_DX, false>(l, a, st); break;
        default: e = a.pair ? launch_mode<PROD_DW, true>(l, a, st) : launch_mode<PROD_DW, false>(l, a, st); break;
    }
    ++l->launches;
    if (e == cudaSuccess) return SOM_OK;
    l->last_cuda_error = (int)e;
    return SOM_ERR_CUDA;
}

}  // namespace lay
