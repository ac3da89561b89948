// The product of two matrices in 4 bits on the 5th-generation tensor cores (tcgen05.mma kind::mxf4, fp32 accumulators).
//
// Persistent blocks walk the output tiles as the 16-bit products do (layers_product.cu): warp 0 issues the TMA copies of a ring, warp 1 the
// matrix instructions, sixteen warps run the epilogue; every wait is bounded.  A stage holds 256 k of both operands (rows of 128 bytes) and their
// scales, 1 KB for 128 rows as they lie in memory; copies from shared to tensor memory (tcgen05.cp) bring the scales in front of the
// instructions that use them, a set of columns for each place of the ring.
//
// PAIR: 256 x 256 tiles by two blocks of a cluster (cta_group::2); each loads its own 128 rows of A, one half of B, and the scales of its rows of
// A and of all of B.  NARROW: 128 x 128 by one block, for products with few tiles; where SMs still idle the sum is
// split over blocks, which leave fp32 parts for k_finish.
#include "layers_epilogue.cuh"
#include "layers_finish.cuh"
#include "layers_fp4.cuh"
#include "layers_product.cuh"

namespace lay {
namespace {

constexpr int BM = 128, BK = 256, STEPS = BK / 64;
constexpr int PART_BYTES = BM * BK / 2;  // 128 rows of a stage
constexpr int STAGES = 5, STAGE_BYTES = 2 * PART_BYTES, SCALE_BYTES = 3 * FP4_SCALE_TILE;
constexpr int TURNS = 4, EPI_WARPS = 4 * TURNS, THREADS = 32 * (2 + EPI_WARPS);
constexpr int ROW_BYTES = 64, OUT_BYTES = 32 * ROW_BYTES;  // an epilogue warp's staged output: 32 rows of 32 columns (fp32: 16)
constexpr int SMEM = 1024 + STAGES * (STAGE_BYTES + SCALE_BYTES) + EPI_WARPS * OUT_BYTES;

struct Fp4Args {
    CUtensorMap a, b, sa, sb, o;
    const uint16_t *bias, *residual;
    int64_t ldr;
    int row_tiles, col_tiles, splits;
    int rows, cols;   // of the output
    int gate_rows;    // gated: rows of B between a feature's gate row and its other row; 0 = not gated
    int steps;        // stages of the whole sum
    int act;
    int* flags;
};

struct Tile {
    int row, col, split, from, n;
};

template <bool PAIRED>
__device__ __forceinline__ Tile tile_at(const Fp4Args& p, int idx, int width, int rank)
{
    Tile t;
    t.split = 0;
    if (p.splits > 1) {
        t.split = idx % p.splits;
        idx /= p.splits;
    }
    const int rt = idx / p.col_tiles;
    t.row = rt * (PAIRED ? 2 * BM : BM) + rank * BM;
    t.col = (idx - rt * p.col_tiles) * width;
    t.from = p.steps * t.split / p.splits;
    t.n = p.steps * (t.split + 1) / p.splits - t.from;
    return t;
}

// What a kernel makes of the sums: outputs, outputs of features with a gate (pairs), fp32 parts without an epilogue (single blocks).
enum Ends { PLAIN = 0, GATED = 1, PARTS = 2 };

template <bool PAIRED, int ENDS, bool BF16>
__global__ void __launch_bounds__(THREADS, 1) k_fp4_product(const __grid_constant__ Fp4Args p)
{
    constexpr int BN = PAIRED ? 256 : 128;
    constexpr int BUFFERS = PAIRED ? 1 : 2;  // accumulators
    constexpr uint32_t SCALES = BUFFERS * BN, SCALES_A = 8, SCALES_SET = SCALES_A + BN / 16;  // first column of the stages' scales
    static_assert(SCALES + STAGES * SCALES_SET <= 512, "tensor memory");
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_free[2], drained;
    __shared__ uint32_t tmem_sh;
    __shared__ int gave_up_sh, summed[2];
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    unsigned char* scales = ring + STAGES * STAGE_BYTES;
    unsigned char* staged = scales + STAGES * SCALE_BYTES;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = PAIRED ? (int)cluster_rank() : 0;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            bar_init(&full[i], 1);
            bar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(&acc_full[i], 1);
            bar_init(&acc_free[i], EPI_WARPS * (PAIRED ? 2 : 1));
        }
        bar_init(&drained, 1);
        gave_up_sh = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&p.a);
        prefetch_map(&p.b);
        prefetch_map(&p.sa);
        prefetch_map(&p.sb);
    }
    if (warp == 1) tmem_alloc<PAIRED>(&tmem_sh, 512);
    tc_fence_before();
    __syncthreads();
    if (PAIRED) cluster_sync();  // the other block's barriers are ready
    tc_fence_after();
    if (warp > 0) enter();
    const uint32_t tmem = tmem_sh;
    volatile int* gave_up = &gave_up_sh;

    constexpr int WIDTH = ENDS == GATED ? BN / 2 : BN;  // output columns of a tile
    const int step = PAIRED ? gridDim.x >> 1 : gridDim.x, first_tile = PAIRED ? blockIdx.x >> 1 : blockIdx.x;
    const int total = p.row_tiles * p.col_tiles * p.splits;

    if (warp == 0) {
        if (lane == 0) {
            // The leader's barrier counts both blocks' bytes.  Rows of scales come in ones or twos of 128 (beyond the last: zeros).
            constexpr int SHARE = PAIRED ? BN / 2 : BN;  // columns of B in this block
            constexpr int BYTES = (PAIRED ? 2 : 1) * (PART_BYTES + SHARE * BK / 2 + FP4_SCALE_TILE * (1 + BN / 128));
            const uint32_t full0 = PAIRED ? cluster_addr(smem_addr(&full[0]), 0) : smem_addr(&full[0]);
            auto load_columns = [&](const Tile& t, int it, int s) {
                unsigned char *sb = ring + s * STAGE_BYTES + PART_BYTES, *ss = scales + s * SCALE_BYTES + FP4_SCALE_TILE;
                const uint32_t bar = full0 + 8 * s;
                const int k = (t.from + it) * (BK / 4);
                if (rank == 0) bar_expect(&full[s], BYTES);
                if (ENDS != GATED) {
                    tma_load<PAIRED>(sb, &p.b, bar, k, t.col + rank * SHARE, 0);
                    tma_load<PAIRED>(ss, &p.sb, bar, 0, t.from + it, t.col / 128);
                } else {  // the first block has the gate's rows, the second the others
                    tma_load<PAIRED>(sb, &p.b, bar, k, t.col + rank * p.gate_rows, 0);
                    tma_load<PAIRED>(ss, &p.sb, bar, 0, t.from + it, t.col / 128);
                    tma_load<PAIRED>(ss + FP4_SCALE_TILE, &p.sb, bar, 0, t.from + it, (t.col + p.gate_rows) / 128);
                }
            };
            auto load_rows = [&](const Tile& t, int it, int s) {
                const uint32_t bar = full0 + 8 * s;
                tma_load<PAIRED>(ring + s * STAGE_BYTES, &p.a, bar, (t.from + it) * (BK / 4), t.row, 0);
                tma_load<PAIRED>(scales + s * SCALE_BYTES, &p.sa, bar, 0, t.from + it, t.row / 128);
            };
            int stage = 0, ahead = 0;
            uint32_t phase = 0;
            int64_t issued = 0;
            bool ok = true;
            // The weights were complete before the kernel in front (x's quantisation, which the same call launched) began its work.
            if (first_tile < total) {
                const Tile t = tile_at<PAIRED>(p, first_tile, WIDTH, rank);
                for (; ahead < STAGES && ahead < t.n; ++ahead) load_columns(t, ahead, ahead);
            }
            enter();
            for (int idx = first_tile; ok && idx < total; idx += step) {
                const Tile t = tile_at<PAIRED>(p, idx, WIDTH, rank);
                for (int it = 0; it < t.n; ++it) {
                    if (!bar_wait(&empty[stage], phase ^ 1u, gave_up)) {
                        ok = false;
                        break;
                    }
                    load_rows(t, it, stage);
                    if (issued >= ahead) load_columns(t, it, stage);
                    ++issued;
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
            if (issued < ahead) issued = ahead;
            if (!ok && rank == 0) {  // copies still in flight write shared memory: let them land before the block leaves
                const long long t0 = clock64();
                for (int s = 0; s < STAGES; ++s) {
                    const int64_t uses = issued / STAGES + (s < (int)(issued % STAGES) ? 1 : 0);
                    while (uses > 0 && !bar_try(&full[s], (uint32_t)(uses - 1) & 1u) && clock64() - t0 < WAIT_CYCLES) {}
                }
            }
        }
    } else if (warp == 1) {
        // The whole warp walks the stages and one lane issues: addresses and descriptors then stay in the warp's own registers.  With one
        // lane alone in the loop an instruction took 60 to 70 clocks to issue, 940 a stage: 8192 x 16384 x 4096 took 239 us.
        if (rank == 0) {
            int stage = 0, n_acc = 0;
            uint32_t phase = 0;
            bool ok = true;
            const bool lead = elect_lane();
            constexpr uint32_t idesc[2] = {mma_fp4_desc(PAIRED ? 256 : 128, BN, 0), mma_fp4_desc(PAIRED ? 256 : 128, BN, 1)};
            for (int idx = first_tile; ok && idx < total; idx += step, ++n_acc) {
                const Tile t = tile_at<PAIRED>(p, idx, WIDTH, rank);
                const int buf = n_acc % BUFFERS;
                const uint32_t d = tmem + buf * BN;
                ok = __all_sync(0xffffffffu, bar_wait<PAIRED>(&acc_free[buf], (uint32_t)(n_acc / BUFFERS) & 1u ^ 1u, gave_up));  // all go on or all leave
                tc_fence_after();
                for (int it = 0; ok && it < t.n; ++it) {
                    ok = __all_sync(0xffffffffu, bar_wait(&full[stage], phase, gave_up));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sa = smem_addr(ring) + stage * STAGE_BYTES, sb = sa + PART_BYTES, ss = smem_addr(scales) + stage * SCALE_BYTES;
                    // A stage's scales have a set of columns for each place of the ring: what used it is done when the place is loaded again.
                    // (The next stage's in front of this stage's instructions, where it is here, was slower.)
                    const uint32_t ta = tmem + SCALES + stage * SCALES_SET, tb = ta + SCALES_A;
                    if (lead) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            tmem_put_scales<PAIRED>(ta + 4 * h, ss + 512 * h);
#pragma unroll
                            for (int c = 0; c < BN / 128; ++c) tmem_put_scales<PAIRED>(tb + h * (BN / 32) + 4 * c, ss + FP4_SCALE_TILE * (1 + c) + 512 * h);
                        }
#pragma unroll
                        for (int kk = 0; kk < STEPS; ++kk)
                            mma_fp4<PAIRED>(d, mat_desc(sa + kk * 32, 16, 1024), mat_desc(sb + kk * 32, 16, 1024), idesc[kk & 1], ta + 4 * (kk >> 1), tb + (kk >> 1) * (BN / 32),
                                            !(it == 0 && kk == 0));
                        mma_commit<PAIRED>(&empty[stage]);
                    }
                    __syncwarp();
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                if (!ok) break;
                if (lead) mma_commit<PAIRED>(&acc_full[buf]);
                __syncwarp();
            }
            if (!ok && lead) {  // instructions in flight read shared memory and write tensor memory
                mma_commit<PAIRED>(&drained);
                const long long t0 = clock64();
                while (!bar_try(&drained, 0) && clock64() - t0 < WAIT_CYCLES) {}
            }
            __syncwarp();
        }
    } else {
        // A warp may read the 32 lanes of its quarter only; the four warps of a quarter take a fourth of the tile's columns each, into
        // registers at once, so that the accumulator is free again before any of the epilogue's work.
        constexpr int PIECE = WIDTH / TURNS, SENT = ENDS == PARTS ? 16 : 32;  // columns of a warp, and of what it stages at once
        const int q = warp & 3, turn = (warp - 2) >> 2;
        Stager<1, ROW_BYTES> s{staged + (warp - 2) * OUT_BYTES, lane, 0};
        int n_acc = 0;
        for (int idx = first_tile; idx < total; idx += step, ++n_acc) {
            const Tile t = tile_at<PAIRED>(p, idx, WIDTH, rank);
            const int buf = n_acc % BUFFERS, at = turn * PIECE, col = t.col + at;
            const uint32_t acc = tmem + buf * BN + ((uint32_t)(32 * q) << 16);
            const int row0 = t.row + 32 * q, row = row0 + lane;
            const bool counts = row < p.rows;
            const uint16_t* extra = ENDS != PARTS && p.residual ? p.residual + (size_t)row * p.ldr : nullptr;
            RowPart<16> add, b0, b1;
            auto fetch = [&](int col) {
                add.fetch(extra, col, p.cols, extra && counts);
                b0.fetch(p.bias, col, p.cols, p.bias);
                if (ENDS == GATED) b1.fetch(p.bias + p.gate_rows, col, p.cols, p.bias);
            };
            if (ENDS != PARTS) {  // the first columns' while the products still run, the others on the way to L2
                fetch(col);
                if (extra && counts && col < p.cols) prefetch_l2(extra + col);
            }
            // One lane waits, the others for it at a hardware barrier; all go on or all leave by the word that it writes (two words in turn).
            if (warp == 2 && lane == 0) summed[n_acc & 1] = bar_wait(&acc_full[buf], (uint32_t)(n_acc / BUFFERS) & 1u, gave_up);
            asm volatile("bar.sync 1, %0;" ::"n"(32 * EPI_WARPS) : "memory");
            if (!summed[n_acc & 1]) break;
            tc_fence_after();
            float v[PIECE], u[ENDS == GATED ? PIECE : 16];
#pragma unroll
            for (int h = 0; h < PIECE; h += 32) {
                tmem_ld(acc + at + h, reinterpret_cast<float(&)[32]>(v[h]));
                if constexpr (ENDS == GATED) tmem_ld(acc + BN / 2 + at + h, reinterpret_cast<float(&)[32]>(u[h]));
            }
            tmem_wait_ld();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIRED) bar_arrive_remote(cluster_addr(smem_addr(&acc_free[buf]), 0));
                else bar_arrive(&acc_free[buf]);
            }
#pragma unroll
            for (int c = 0; c < PIECE / 16; ++c) {
                float(&z)[16] = reinterpret_cast<float(&)[16]>(v[16 * c]);
                const bool first = c * 16 % SENT == 0, last = (c + 1) * 16 % SENT == 0;
                if (first && (ENDS == PARTS || c == 0)) s.begin();
                if constexpr (ENDS == PARTS) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) s.put(k, z + 4 * k);
                } else {
                    if (p.bias) b0.template add<BF16>(z);
                    if (p.act != SOM_ACT_NONE)
                        with_act(p.act, [&](auto tag) {
#pragma unroll
                            for (int k = 0; k < 16; ++k) z[k] = act_of<decltype(tag)::value>(z[k]);
                        });
                    if constexpr (ENDS == GATED) {
                        float(&w)[16] = reinterpret_cast<float(&)[16]>(u[16 * c]);
                        if (p.bias) b1.template add<BF16>(w);
#pragma unroll
                        for (int k = 0; k < 16; ++k) z[k] *= w[k];
                    }
                    if (extra) add.template add<BF16>(z);
                    if (c + 1 < PIECE / 16) fetch(col + 16 * (c + 1));
                    if (first && c > 0) s.begin();
                    s.put(2 * (c & 1), pack8<BF16>(z));
                    s.put(2 * (c & 1) + 1, pack8<BF16>(z + 8));
                }
                if (last) s.send(&p.o, col + 16 * (c + 1) - SENT, row0, t.split, p.rows, p.cols);
            }
        }
    }
    if (warp >= 2 && lane == 0) store_wait_all();
    __syncthreads();
    if (threadIdx.x == 0 && gave_up_sh) atomicOr(p.flags, LAY_FLAG_GAVE_UP);
    __syncwarp();
    if (PAIRED) cluster_sync();  // no block leaves while the other may still reach its memory
    if (warp == 1) {
        tc_fence_after();
        tmem_free<PAIRED>(tmem, 512);
    }
}

// [rows of 128][steps of 256 columns][256 words] scales, `blocks` rows of 128 a box
int map_scales(som_layers* l, CUtensorMap* map, const void* base, int64_t rows, int64_t D, int blocks)
{
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    const cuuint64_t dims[3] = {FP4_SCALE_TILE / 4, (cuuint64_t)fp4_tiles(D), (cuuint64_t)tiles_of(rows, 128)};
    const cuuint64_t strides[2] = {FP4_SCALE_TILE, (cuuint64_t)(fp4_tiles(D) * FP4_SCALE_TILE)};
    const cuuint32_t box[3] = {FP4_SCALE_TILE / 4, 1u, (cuuint32_t)blocks}, step[3] = {1u, 1u, 1u};
    const CUresult r = reinterpret_cast<Encode>(l->encode)(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<void*>(base), dims, strides, box, step,
                                                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                                                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r == CUDA_SUCCESS) return SOM_OK;
    l->last_cuda_error = (int)cudaErrorInvalidValue;
    return SOM_ERR_CUDA;
}

// How a product is cut: pairs once narrow tiles pass the SMs (as the 16-bit products); blocks that share a sum where tiles leave SMs idle, four
// steps of 256 k each at the least.  `joined`: fp32 parts and k_finish, for split sums and for gated products that are not made by pairs
// (a single block's tile holds no two halves; of pairs each half has to begin on 128 rows of scales).
// Parts of at least 2 / 4 / 8 steps / none, in us from a graph with x's quantisation: 8 rows, 8192 -> 1024 10.1 / 8.7 / 9.3 / 11.4; 64 rows, 2048 -> 4096
// 8.6 / 8.3 / 8.4 / 8.4; 200 rows, 1024 -> 1024 8.2 / 7.2 / 7.2 / 7.2; 64 rows, 4096 -> 2 x 1000 10.6 / 8.9 / 10.3 / 11.6.
struct Cut {
    bool paired, joined;
    int row_tiles, col_tiles, splits;
};

Cut cut_of(const som_layers* l, const Fp4Product& p)
{
    const int64_t outputs = p.gated ? 2 * p.F : p.F, steps = tiles_of(p.D, BK);
    Cut c = {};
    const int64_t narrow = tiles_of(p.T, 128) * tiles_of(outputs, 128);
    c.paired = narrow > l->sm_count && !(p.gated && p.F % 128 != 0);
    c.splits = 1;
    if (!c.paired) {
        int64_t s = l->sm_count / narrow;
        if (s > steps / 4) s = steps / 4;
        if (s > 16) s = 16;
        if (s > 1) c.splits = (int)s;
        c.joined = c.splits > 1 || p.gated;
    }
    c.row_tiles = (int)tiles_of(p.T, c.paired ? 256 : 128);
    c.col_tiles = (int)(c.paired ? tiles_of(p.F, p.gated ? 128 : 256) : tiles_of(outputs, 128));
    return c;
}

dim3 grid_of(const som_layers* l, const Fp4Args& a, bool paired)
{
    const int64_t tiles = (int64_t)a.row_tiles * a.col_tiles * a.splits, most = paired ? l->fp4_pairs : l->sm_count;
    return dim3((unsigned)((tiles < most ? tiles : most) * (paired ? 2 : 1)));
}

template <bool PAIRED, int ENDS>
cudaError_t launch_as(som_layers* l, const Fp4Args& a, bool bf16, cudaStream_t st)
{
    const dim3 grid = grid_of(l, a, PAIRED);
    return bf16 ? launch(l, k_fp4_product<PAIRED, ENDS, true>, grid, THREADS, SMEM, st, PAIRED ? 2 : 1, a)
                : launch(l, k_fp4_product<PAIRED, ENDS, false>, grid, THREADS, SMEM, st, PAIRED ? 2 : 1, a);
}

// (and, of pairs, how many can be resident)
template <bool PAIRED, int ENDS, bool BF16>
cudaError_t prepare_as(int* pairs)
{
    const cudaError_t e = cudaFuncSetAttribute(k_fp4_product<PAIRED, ENDS, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e != cudaSuccess || !PAIRED) return e;
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
    const cudaError_t f = cudaOccupancyMaxActiveClusters(&n, k_fp4_product<PAIRED, ENDS, BF16>, &c);
    if (n < *pairs) *pairs = n;
    return f;
}

}  // namespace

cudaError_t prepare_fp4_product(som_layers* l)
{
    int n = l->sm_count / 2;
    cudaError_t e = prepare_as<false, PLAIN, true>(&n);
    if (e == cudaSuccess) e = prepare_as<false, PLAIN, false>(&n);
    if (e == cudaSuccess) e = prepare_as<false, PARTS, true>(&n);
    if (e == cudaSuccess) e = prepare_as<true, PLAIN, true>(&n);
    if (e == cudaSuccess) e = prepare_as<true, PLAIN, false>(&n);
    if (e == cudaSuccess) e = prepare_as<true, GATED, true>(&n);
    if (e == cudaSuccess) e = prepare_as<true, GATED, false>(&n);
    l->fp4_pairs = n;
    return e == cudaSuccess && n < 1 ? cudaErrorNotSupported : e;
}

size_t fp4_product_bytes(const som_layers* l, const Fp4Product& p)
{
    const Cut c = cut_of(l, p);
    return c.joined ? (size_t)c.splits * p.T * (p.gated ? 2 * p.F : p.F) * sizeof(float) : 0;
}

int launch_fp4_product(som_layers* l, const Fp4Product& p, unsigned char* ws, cudaStream_t st)
{
    const Cut c = cut_of(l, p);
    const int64_t outputs = p.gated ? 2 * p.F : p.F;
    Fp4Args a = {};
    LAY_TRY(make_map(l, &a.a, p.x_codes, 2, p.D / 4, p.T, 1, p.D / 4, p.T * p.D / 4, 128));
    LAY_TRY(make_map(l, &a.b, p.w_codes, 2, p.D / 4, outputs, 1, p.D / 4, outputs * p.D / 4, 128));
    LAY_TRY(map_scales(l, &a.sa, p.x_scales, p.T, p.D, 1));
    LAY_TRY(map_scales(l, &a.sb, p.w_scales, outputs, p.D, c.paired && !p.gated ? 2 : 1));
    a.row_tiles = c.row_tiles;
    a.col_tiles = c.col_tiles;
    a.splits = c.splits;
    a.rows = (int)p.T;
    a.steps = (int)tiles_of(p.D, BK);
    a.flags = l->flags;
    if (c.joined) {
        a.cols = (int)outputs;
        LAY_TRY(make_map(l, &a.o, ws, 4, outputs, p.T, c.splits, outputs, p.T * outputs, 32, ROW_BYTES));
        LAY_TRY(outcome(l, launch(l, k_fp4_product<false, PARTS, true>, grid_of(l, a, false), THREADS, SMEM, st, 1, a)));
        FinishArgs f = {};
        f.part = reinterpret_cast<const float*>(ws);
        f.rows = p.T;
        f.splits = c.splits;
        f.n = (int)outputs;
        f.cols = (int)p.F;
        f.bias = p.bias;
        f.extra = p.residual;
        f.ld_extra = p.ldr;
        f.out = p.y;
        f.ld = p.ldy;
        f.mode = FINISH_FWD;
        f.act = p.act;
        f.gated = p.gated;
        f.bf16 = p.bf16;
        return launch_finish(l, f, st);
    }
    a.cols = (int)p.F;
    a.gate_rows = p.gated ? (int)p.F : 0;
    a.act = p.act;
    a.bias = p.bias;
    a.residual = p.residual;
    a.ldr = p.ldr;
    LAY_TRY(make_map(l, &a.o, p.y, 2, p.F, p.T, 1, p.ldy, p.T * p.ldy, 32, ROW_BYTES));
    return outcome(l, !c.paired ? launch_as<false, PLAIN>(l, a, p.bf16, st) : p.gated ? launch_as<true, GATED>(l, a, p.bf16, st) : launch_as<true, PLAIN>(l, a, p.bf16, st));
}

}  // namespace lay
