// Matrix products of the dense operators on the 5th-generation tensor cores.
//
// Persistent blocks, one per SM, walk the output tiles.  Warp 0 issues the TMA copies of a ring (64 k of both operands a stage,
// 128-byte swizzle: 32 KB, or 48 for wide tiles), warp 1 issues the matrix instructions (tcgen05.mma, fp32 accumulators in
// tensor memory), eight warps run the epilogue (sixteen were no faster where the epilogue counts, and slower elsewhere).  The
// accumulator is double-buffered, so that the epilogue of a tile runs under the products of the next.  PROD_DZ_TWO keeps two
// products of a tile side by side, z with one buffer and g with two: the next tile's g is multiplied while the epilogue reads
// this tile's z and g (16384 rows of 32 experts of 2048 x 1024: 250 us, with one buffer for both 301).  Operands enter K-major
// (a row holds consecutive k) or M/N-major (a row holds consecutive rows of the product), as they lie in memory: no operand is
// transposed beforehand.  Every wait is bounded.
//
// Three tile shapes.  PAIR: two blocks of a cluster share a tile of 256 x 256; each loads its own 128 rows of A and one half of
// B, and the matrix instruction reads both halves (cta_group::2).  A single block on 128 x 256 moves 48 KB into and 48 KB out
// of its shared memory for 512 clocks of matrix work, 192 bytes a clock where shared memory gives 128: 4096 x 4096 x 4096
// took 134 us so, 103 in pairs (no epilogue).  With the pair it is 32 KB each way, 128 bytes a clock.  WIDE: that single block,
// for experts with fewer rows than a pair's tile, where the weights' bytes count.  NARROW: 128 x 128 by one block, for products
// with few tiles.
//
// What bounds them.  Pairs: the matrix pipe and the card's power.  4096 x 4096 x 4096 bf16 with bias, gelu and residual takes 123 us
// at 1.61 GHz (1.11 PFLOP/s, pipe busy for 57 % of the time, of the 86 % that 256 tiles leave to 74 pairs), 131 us call after call,
// where the clock falls further.  The experts' products of 4096 tokens x 8 of 64: 253 + 146 us, 1.03 PFLOP/s of use and 1.31 with
// the padding of each expert to 256 rows.  Wide, 9 rows an expert: the weights, 520 MB in 92 us (5.6 TB/s) and 260 in 54 (4.8).
#include "layers_math.cuh"
#include "layers_product.cuh"
#include "layers_ptx.cuh"

namespace lay {
namespace {

constexpr int BM = 128, BK = 64;
constexpr int BOX = 64 * 128;      // bytes of a box of 64 rows
constexpr int A_BYTES = 2 * BOX;   // a block's rows of A in a stage
// Bytes of the ring and buffers of an epilogue warp.  PROD_DW, whose sums may be short (an expert's rows), gives a stage of its
// ring for a second buffer, so that a piece is staged while the one before is read.
__host__ __device__ constexpr int ring_bytes(int mode) { return (mode == PROD_DW ? 5 : 6) * 2 * A_BYTES; }
__host__ __device__ constexpr int out_buffers(int mode) { return mode == PROD_DW ? 2 : 1; }
constexpr int EPI_WARPS = 4 * EPI_TURNS, THREADS = 32 * (2 + EPI_WARPS);
constexpr int OUT_BYTES = 32 * 128;  // an epilogue warp's staged output: 32 rows of 128 bytes
constexpr int SMEM = 1024 + ring_bytes(PROD_FWD) + EPI_WARPS * OUT_BYTES;
static_assert(SMEM == 1024 + ring_bytes(PROD_DW) + EPI_WARPS * 2 * OUT_BYTES, "one size for all modes");

struct Tile {
    int row, col, expert;  // this block's first row and the tile's first column of the output, expert
    int k0, k;             // PROD_DW: first row of the sum; length of the first product's sum
    int split;             // part of the sum
    bool second;           // PROD_DW: a tile of the second product
    int live, store;       // rows below `live` are in use, rows below `store` are written (zeros from `live` on)
};

__device__ __forceinline__ int round64(int n) { return (n + 63) & ~63; }

// EARLY: the plan is read before the kernel in front is over, past what this SM's L1 holds
template <bool EARLY>
__device__ __forceinline__ int plan_at(const int* p)
{
    return EARLY ? __ldcg(p) : *p;
}

template <int MODE, bool EARLY = false>
__device__ __forceinline__ int tile_count(const ProdArgs& p)
{
    if (MODE == PROD_DW) return p.experts * (p.row_tiles * p.col_tiles + p.row_tiles2 * p.col_tiles2) * p.splits;
    return (p.tiles ? plan_at<EARLY>(p.tiles) : p.row_tiles) * p.col_tiles * p.splits;
}

template <int MODE, int SHAPE, bool EARLY = false>
__device__ __forceinline__ Tile tile_at(const ProdArgs& p, int idx, int width, int rank)
{
    constexpr int ROWS = shape_rows(SHAPE);
    Tile t;
    t.split = 0;
    t.second = false;
    if (p.splits > 1) {
        t.split = idx % p.splits;
        idx /= p.splits;
    }
    if (MODE == PROD_DW) {
        const int all = p.experts * p.row_tiles * p.col_tiles;
        t.second = idx >= all;
        if (t.second) idx -= all;
        const int col_tiles = t.second ? p.col_tiles2 : p.col_tiles, per = (t.second ? p.row_tiles2 : p.row_tiles) * col_tiles;
        t.expert = idx / per;
        const int rest = idx - t.expert * per, rt = rest / col_tiles;
        t.row = rt * ROWS + rank * BM;
        t.col = (rest - rt * col_tiles) * width;
        t.k0 = p.seg ? plan_at<EARLY>(p.seg + t.expert) : 0;
        t.k = p.seg ? round64(plan_at<EARLY>(p.count + t.expert)) : p.k1;
        t.live = t.store = t.second ? p.rows2 : p.rows;
    } else {
        const int rt = idx / p.col_tiles;
        t.row = rt * ROWS + rank * BM;
        t.col = (idx - rt * p.col_tiles) * width;
        t.expert = p.tile_expert ? plan_at<EARLY>(p.tile_expert + rt) : 0;
        t.k0 = 0;
        t.k = p.k1;
        t.live = t.store = p.rows;
        if (p.seg) {
            const int s = plan_at<EARLY>(p.seg + t.expert), n = plan_at<EARLY>(p.count + t.expert);
            t.live = s + n;
            // the sums over an expert's rows (PROD_DW) run over whole steps of 64 rows
            t.store = MODE == PROD_DZ_TWO ? s + round64(n) : t.live;
        }
    }
    if (p.splits > 1) {
        const int steps = (p.k1 + BK - 1) / BK, from = steps * t.split / p.splits, to = steps * (t.split + 1) / p.splits;
        t.k0 = from * BK;
        t.k = (to - from) * BK;
    }
    return t;
}

// Ways out of the epilogue.  Staged: 32 rows (lane l holds row l) of 64 16-bit or 32 fp32 columns go through shared memory
// (128-byte rows, 128-byte swizzle) to a TMA store, which leaves out what lies outside the tensor.  Direct: a lane writes 8
// columns at a time.  Direct stores take the load/store pipe 32 cycles an instruction: too much where a tile's products are short
// (PROD_DW at 512 rows an expert: 134 us staged, 178 us direct), but no waits, and no shared memory for up to three outputs
// at once (PROD_DZ, PROD_DZ_TWO).
template <int BUFFERS>
struct Stager {
    unsigned char* buf;
    int lane, other;  // other: distance to the other buffer
    // the last store from this buffer has read it
    __device__ __forceinline__ void begin()
    {
        if (BUFFERS == 2) {
            buf += other;
            other = -other;
        }
        if (lane == 0) store_wait_read<BUFFERS - 1>();
        __syncwarp();
    }
    // 16 bytes of this lane's row
    __device__ __forceinline__ void put(int chunk, uint4 v) { *reinterpret_cast<uint4*>(buf + lane * 128 + ((chunk ^ (lane & 7)) << 4)) = v; }
    __device__ __forceinline__ void put(int chunk, const float* v)
    {
        put(chunk, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
    }
    __device__ __forceinline__ void send(const CUtensorMap* map, int col, int row, int batch, int rows, int cols)
    {
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
            if (col < cols && row < rows) tma_store(map, buf, col, row, batch);
            store_commit();
        }
    }
};

template <bool BF16>
__device__ __forceinline__ uint4 pack8(const float* v)
{
    return make_uint4(pack2(v[0], v[1], BF16), pack2(v[2], v[3], BF16), pack2(v[4], v[5], BF16), pack2(v[6], v[7], BF16));
}

// 8 consecutive values of a lane's row -> global memory
template <bool BF16>
__device__ __forceinline__ void store8(uint16_t* to, const float (&v)[8])
{
    *reinterpret_cast<uint4*>(to) = pack8<BF16>(v);
}

// N values of a row of a 16-bit matrix, fetched before they are needed; zeros beyond `cols` (a multiple of 8)
template <int N>
struct RowPart {
    uint4 w[N / 8];
    __device__ __forceinline__ void fetch(const uint16_t* row, int col, int cols, bool want)
    {
#pragma unroll
        for (int j = 0; j < N / 8; ++j)
            w[j] = want && col + 8 * j < cols ? *(reinterpret_cast<const uint4*>(row + col) + j) : make_uint4(0u, 0u, 0u, 0u);
    }
    template <bool BF16>
    __device__ __forceinline__ void get(float (&v)[N]) const
    {
#pragma unroll
        for (int j = 0; j < N / 8; ++j) widen8(w[j], reinterpret_cast<float(&)[8]>(v[8 * j]), BF16);
    }
    template <bool BF16>
    __device__ __forceinline__ void add(float (&v)[N]) const
    {
        float f[N];
        get<BF16>(f);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] += f[j];
    }
};

// Lane l holds v[0..7] of row l; returns to the lanes with l % 8 = c the sum of column c over the 32 rows (fixed order).
__device__ __forceinline__ float column_sum(float (&v)[8], int lane)
{
#pragma unroll
    for (int h = 4; h >= 1; h >>= 1) {
        const bool up = lane & h;
#pragma unroll
        for (int j = 0; j < h; ++j) {
            const float give = up ? v[j] : v[j + h], keep = up ? v[j + h] : v[j];
            v[j] = keep + __shfl_xor_sync(0xffffffffu, give, h);
        }
    }
    v[0] += __shfl_xor_sync(0xffffffffu, v[0], 8);
    return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 16);
}

template <int MODE, int SHAPE, bool BF16>
__global__ void __launch_bounds__(THREADS, 1) k_product(const __grid_constant__ ProdArgs p)
{
    constexpr bool A_MN = MODE == PROD_DW, B_MN = MODE == PROD_DX || MODE == PROD_DW;
    constexpr int BUFFERS = MODE == PROD_DZ_TWO ? 1 : 2;  // of the first product
    constexpr bool PAIRED = SHAPE == PAIR;
    constexpr int BN = shape_cols(SHAPE);
    constexpr int SHARE = PAIRED ? BN / 2 : BN;  // columns of B in this block
    constexpr int STAGE_BYTES = A_BYTES + SHARE * 128, STAGES = ring_bytes(MODE) / STAGE_BYTES;
    constexpr uint32_t TMEM_COLUMNS = 2 * BN;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty[2], drained;
    __shared__ uint32_t tmem_sh;
    __shared__ int gave_up_sh, summed[2];  // summed: whether a tile's products came, for the epilogue
    unsigned char* ring = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);

    unsigned char* staged = ring + ring_bytes(MODE);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = PAIRED ? (int)cluster_rank() : 0;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            bar_init(&full[i], 1);
            bar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(&acc_full[i], 1);
            bar_init(&acc_empty[i], EPI_WARPS * (PAIRED ? 2 : 1));
        }
        bar_init(&drained, 1);
        gave_up_sh = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<PAIRED>(&tmem_sh, TMEM_COLUMNS);
    if (threadIdx.x == 0) {
        prefetch_map(&p.a);
        prefetch_map(&p.b);
    }
    tc_fence_before();
    __syncthreads();
    if (PAIRED) cluster_sync();  // the other block's barriers are ready
    tc_fence_after();
    if (warp > 0) enter();
    const uint32_t tmem = tmem_sh;
    volatile int* gave_up = &gave_up_sh;

    const bool gated = p.gate_rows != 0;
    // Output columns of a tile: a gated product spends half of the accumulator's columns on the other half of its rows.
    // PROD_DZ_TWO: half in any case; the second product takes the other BN columns of tensor memory in turns of BN / 2.
    const int width = MODE == PROD_DZ_TWO || (gated && (MODE == PROD_FWD || MODE == PROD_DZ)) ? BN / 2 : BN;
    const int n1 = MODE == PROD_DZ_TWO && !gated ? BN / 2 : BN;  // accumulator columns of the first product
    constexpr int N2 = BN / 2, SHARE2 = PAIRED ? N2 / 2 : N2;  // columns of the second product, and of its B in this block
    const int step = PAIRED ? gridDim.x >> 1 : gridDim.x, first_tile = PAIRED ? blockIdx.x >> 1 : blockIdx.x;

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            int64_t issued = 0;
            bool ok = true;
            constexpr int A_ALL = A_BYTES * (PAIRED ? 2 : 1);
            // the same for all tiles: steps of the second product (which comes first); columns of the first product's B in this block,
            // and how many of them are the gate's (gated: a pair's second block has the other half, in a single block they follow)
            const int it2 = MODE == PROD_DZ_TWO ? (p.k2 + BK - 1) / BK : 0;
            const int share = PAIRED ? n1 / 2 : n1, gates = !PAIRED && gated && !B_MN ? share / 2 : share;
            const int from = !PAIRED ? 0 : gated && !B_MN ? p.gate_rows : share;
            const int box = B_MN ? 64 : p.right_box, all1 = A_ALL + (PAIRED ? 2 : 1) * share * 128, all2 = A_ALL + N2 * 128;
            // the leader's barrier counts both blocks' bytes
            const uint32_t full0 = PAIRED ? cluster_addr(smem_addr(&full[0]), 0) : smem_addr(&full[0]);
            auto load_columns = [&](const Tile& t, int it, int s) {
                unsigned char* sb = ring + s * STAGE_BYTES + A_BYTES;
                const uint32_t bar = full0 + 8 * s;
                if (MODE == PROD_DZ_TWO && it < it2) {
                    if (rank == 0) bar_expect(&full[s], all2);
                    for (int j = 0; j < SHARE2; j += 64) tma_load<PAIRED>(sb + j * 128, &p.b2, bar, t.col + rank * SHARE2 + j, it * BK, t.expert);
                    return;
                }
                const int b0 = t.col + rank * from, k = t.k0 + (it - it2) * BK;
                if (rank == 0) bar_expect(&full[s], all1);
                for (int j = 0; j < share; j += box) {
                    if (B_MN) tma_load<PAIRED>(sb + j * 128, t.second ? &p.b2 : &p.b, bar, b0 + j, k, MODE == PROD_DW ? 0 : t.expert);
                    else tma_load<PAIRED>(sb + j * 128, &p.b, bar, k, j < gates ? b0 + j : b0 + j - gates + p.gate_rows, t.expert);
                }
            };
            auto load_rows = [&](const Tile& t, int it, int s) {
                unsigned char* sa = ring + s * STAGE_BYTES;
                const uint32_t bar = full0 + 8 * s;
                const bool second = MODE == PROD_DZ_TWO && it < it2;
                const CUtensorMap* map = second || t.second ? &p.a2 : &p.a;
                const int k = second ? it * BK : t.k0 + (it - it2) * BK;
                if (A_MN) {
                    tma_load<PAIRED>(sa, map, bar, t.row, k, 0);
                    tma_load<PAIRED>(sa + BOX, map, bar, t.row + 64, k, 0);
                } else if (p.seg) {
                    // Experts' rows come in boxes of LEFT_BOX; where none of a box is in use it is read from beyond the matrix, which
                    // gives zeros without traffic (and multiplying zeros takes less power).
#pragma unroll
                    for (int r = 0; r < BM; r += LEFT_BOX) tma_load<PAIRED>(sa + r * 128, map, bar, k, t.row + r < t.live ? t.row + r : p.rows, 0);
                } else {
                    tma_load<PAIRED>(sa, map, bar, k, t.row, 0);
                }
            };
            int ahead = 0;  // stages of the first tile whose columns are on their way
            if (p.columns_first && first_tile < tile_count<MODE, true>(p)) {
                const Tile t = tile_at<MODE, SHAPE, true>(p, first_tile, width, rank);
                const int n = (t.k + BK - 1) / BK + it2;
                for (; ahead < STAGES && ahead < n; ++ahead) load_columns(t, ahead, ahead);
            }
            enter();
            const int total = tile_count<MODE>(p);
            for (int idx = first_tile; ok && idx < total; idx += step) {
                const Tile t = tile_at<MODE, SHAPE>(p, idx, width, rank);
                const int n = (t.k + BK - 1) / BK + it2;
                for (int it = 0; it < n; ++it) {
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
        if (lane == 0 && rank == 0) {
            int stage = 0, n_acc = 0;
            uint32_t phase = 0;
            bool ok = true;
            const int total = tile_count<MODE>(p);
            const uint32_t idesc1 = mma_desc(BF16, A_MN, B_MN, PAIRED ? 256 : 128, n1);
            const uint32_t idesc2 = mma_desc(BF16, 0, 1, PAIRED ? 256 : 128, N2);
            for (int idx = first_tile; ok && idx < total; idx += step, ++n_acc) {
                const Tile t = tile_at<MODE, SHAPE>(p, idx, width, rank);
                const int buf = BUFFERS == 2 ? n_acc & 1 : 0;
                const uint32_t use = (uint32_t)(n_acc / BUFFERS) & 1u;
                const int it1 = (t.k + BK - 1) / BK, it2 = MODE == PROD_DZ_TWO ? (p.k2 + BK - 1) / BK : 0;
                // (the second product's turn was read by the epilogue of the tile before the last, which is over)
                for (int it = 0; it < it1 + it2; ++it) {
                    if (it == it2) {  // the first product's columns have been read
                        ok = bar_wait<PAIRED>(&acc_empty[buf], use ^ 1u, gave_up);
                        tc_fence_after();
                    }
                    if (!ok || !bar_wait(&full[stage], phase, gave_up)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t sa = smem_addr(ring + stage * STAGE_BYTES), sb = sa + A_BYTES;
                    const bool second = MODE == PROD_DZ_TWO && it < it2;
                    const uint32_t d = second ? tmem + (uint32_t)(BN + (n_acc & 1) * N2) : tmem + (uint32_t)(buf * BN);
                    const bool first = it == 0 || it == it2;
#pragma unroll
                    for (int kk = 0; kk < BK / 16; ++kk) {
                        const uint64_t da = A_MN ? mat_desc(sa + kk * 2048, BOX, 1024) : mat_desc(sa + kk * 32, 16, 1024);
                        const uint64_t db =
                            B_MN || second ? mat_desc(sb + kk * 2048, BOX, 1024) : mat_desc(sb + kk * 32, 16, 1024);
                        mma<PAIRED>(d, da, db, second ? idesc2 : idesc1, !(first && kk == 0));
                    }
                    mma_commit<PAIRED>(&empty[stage]);
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                if (!ok) break;
                if (it1 + it2 == 0 && !bar_wait<PAIRED>(&acc_empty[buf], use ^ 1u, gave_up)) {  // nothing to sum
                    ok = false;
                    break;
                }
                mma_commit<PAIRED>(&acc_full[buf]);
            }
            if (!ok) {  // instructions in flight read shared memory and write tensor memory
                mma_commit<PAIRED>(&drained);
                const long long t0 = clock64();
                while (!bar_try(&drained, 0) && clock64() - t0 < WAIT_CYCLES) {}
            }
        }
    } else {
        // A warp may read the 32 lanes of its quarter only; the warps of a quarter take the tile's pieces in turn: 128 bytes
        // of staged outputs, or 32 columns of direct ones, in steps of as many columns as the registers hold.
        constexpr int STEP = MODE == PROD_FWD ? 16 : 8;
        const int piece = MODE == PROD_DZ || MODE == PROD_DZ_TWO || p.out32 ? 32 : 64, round = EPI_TURNS * piece;
        const int q = warp & 3, turn = (warp - 2) >> 2, total = tile_count<MODE>(p);
        Stager<out_buffers(MODE)> s{staged + (warp - 2) * out_buffers(MODE) * OUT_BYTES, lane, OUT_BYTES};
        int n_acc = 0;
        for (int idx = first_tile; idx < total; idx += step, ++n_acc) {
            const Tile t = tile_at<MODE, SHAPE>(p, idx, width, rank);
            const int buf = BUFFERS == 2 ? n_acc & 1 : 0;
            const uint32_t acc = tmem + (uint32_t)(buf * BN) + ((uint32_t)(32 * q) << 16);
            const uint32_t acc2 = tmem + (uint32_t)(BN + (n_acc & 1) * N2) + ((uint32_t)(32 * q) << 16);
            const int row0 = t.row + 32 * q, row = row0 + lane;
            const bool counts = row < t.live;
            // padding rows weigh nothing (what they hold is zeros, or the bias's image of them)
            const float rw = !p.row_weight ? 1.f : counts ? p.row_weight[row] : 0.f;
            const uint16_t* bias = p.bias ? p.bias + (size_t)t.expert * p.bias_ld : nullptr;
            const uint16_t* extra = p.extra ? p.extra + (size_t)row * p.ld_extra : nullptr;
            const bool any = row0 < t.store && turn * piece < width;
            // what the epilogue reads from memory is fetched ahead: the first step's before the products are done
            RowPart<STEP> add, b0, b1;
            auto fetch = [&](int at) {
                const int col = t.col + at;
                if (MODE == PROD_FWD || MODE == PROD_DZ) add.fetch(extra, col, p.cols, extra && counts && at < width);
                if (MODE != PROD_DX && MODE != PROD_DW) {
                    b0.fetch(bias, col, p.cols, bias && at < width);
                    b1.fetch(bias ? bias + p.gate_rows : bias, col, p.cols, bias && gated && at < width);
                }
            };
            if (any) {
                fetch(turn * piece);
                if ((MODE == PROD_FWD || MODE == PROD_DZ) && extra && counts)  // the rest on its way to L2
                    for (int at = turn * piece + round; at < width && t.col + at < p.cols; at += round) prefetch_l2(extra + t.col + at);
            }
            // One lane waits for the products, the other warps for that lane at a hardware barrier: trying the mbarrier
            // takes shared-memory cycles (sixteen warps that did slowed the products by 5 %).  All go on or all leave, by that lane's
            // word: *gave_up may be raised between two warps' looks at it, and one that had left would be missing at the next barrier.
            // (Two words in turn: a word is written again only after every warp has passed the other tile's barrier.)
            if (warp == 2 && lane == 0) summed[n_acc & 1] = bar_wait(&acc_full[buf], (uint32_t)(n_acc / BUFFERS) & 1u, gave_up);
            asm volatile("bar.sync 1, %0;" ::"n"(32 * EPI_WARPS) : "memory");
            if (!summed[n_acc & 1]) break;
            tc_fence_after();
            if (!any) {
                // none of this warp's rows or columns
            } else if constexpr (MODE == PROD_DX || MODE == PROD_DW) {
                const int batch = MODE == PROD_DW ? t.expert + t.split : t.split, cols = t.second ? p.cols2 : p.cols;
                const CUtensorMap* map = t.second ? &p.o2map : &p.o;
                float next[32];
                tmem_ld(acc + turn * piece, next);
                for (int at = turn * piece; at < width;) {
                    float v[32];
                    const int half = p.out32 ? 0 : (at >> 5) & 1, step_on = !p.out32 && half == 0 ? 32 : round - 32 * half;
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = MODE == PROD_DW && t.k == 0 ? 0.f : next[j];  // (no token: nothing was summed)
                    if (at + step_on < width) tmem_ld(acc + at + step_on, next);
                    if (half == 0) s.begin();
                    if (p.out32) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) s.put(j, v + 4 * j);
                        s.send(map, t.col + at, row0, batch, t.second ? p.rows2 : p.rows, cols);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) s.put(4 * half + j, pack8<BF16>(v + 8 * j));
                        if (half == 1) s.send(map, t.col + at - 32, row0, batch, t.second ? p.rows2 : p.rows, cols);
                    }
                    at += step_on;
                }
            } else if constexpr (MODE == PROD_FWD) {
#pragma unroll 1
                for (int at = turn * piece; at < width;) {
                    const int col = t.col + at, done = (at & (piece - 1)) + 16;  // columns of the piece after this step
                    const int step_on = done == piece ? round - piece + 16 : 16;
                    float v[STEP], u[STEP];
                    tmem_ld(acc + at, v);
                    if (gated) tmem_ld(acc + BN / 2 + at, u);
                    tmem_wait_ld();
                    if (bias) {
                        float f[STEP];
                        b0.template get<BF16>(f);
                        const float by = p.weigh == 2 ? rw : 1.f;
#pragma unroll
                        for (int j = 0; j < STEP; ++j) v[j] = fmaf(f[j], by, v[j]);
                        if (gated) b1.template add<BF16>(u);
                    }
                    if (p.act != SOM_ACT_NONE)
                        with_act(p.act, [&](auto tag) {
#pragma unroll
                            for (int j = 0; j < STEP; ++j) v[j] = act_of<decltype(tag)::value>(v[j]);
                        });
                    if (gated) {
#pragma unroll
                        for (int j = 0; j < STEP; ++j) v[j] *= u[j];
                    }
                    if (extra) add.template add<BF16>(v);
                    fetch(at + step_on);
                    // The experts' hidden values are rounded to 16 bits below: the next product's instructions take no wider operands (two
                    // 16-bit terms a value would double its work).  Weighted before: a weight of at most 1 keeps large values in fp16's
                    // range, and what a small one loses below that range, 2^-25, is what y's own rounding loses there.
                    if (p.weigh == 1) {
#pragma unroll
                        for (int j = 0; j < STEP; ++j) v[j] *= rw;
                    }
                    if (done == 16) s.begin();
                    if (p.out32) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) s.put((done - 16) / 4 + j, v + 4 * j);
                    } else {
                        s.put((done - 16) / 8, pack8<BF16>(v));
                        s.put((done - 16) / 8 + 1, pack8<BF16>(v + 8));
                    }
                    if (done == piece) s.send(&p.o, col + 16 - piece, row0, t.split, p.rows, p.cols);
                    at += step_on;
                }
            } else {
                // PROD_DZ, PROD_DZ_TWO: v = z (or the gate's z) becomes dz, u = the gated half's
                const bool writes = row < t.store;
                uint16_t* out = static_cast<uint16_t*>(p.o0) + (size_t)row * p.ld0;
                uint16_t* out2 = static_cast<uint16_t*>(p.o2) + (size_t)row * p.ld2;
                float dot = 0.f;
#pragma unroll 1
                for (int at = turn * 32; at < width; at += (at & 24) == 24 ? round - 24 : 8) {
                    const int col = t.col + at;
                    float v[8], u[8], g[8], hid[8];
                    tmem_ld(acc + at, v);
                    if (gated) tmem_ld(acc + BN / 2 + at, u);
                    if (MODE == PROD_DZ_TWO) tmem_ld(acc2 + at, g);
                    tmem_wait_ld();
                    if (bias) {
                        b0.template add<BF16>(v);
                        if (gated) b1.template add<BF16>(u);
                    }
                    if (MODE == PROD_DZ) add.template get<BF16>(g);
                    fetch(at + ((at & 24) == 24 ? round - 24 : 8));
                    with_act(p.act, [&](auto tag) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            float a, da;
                            act_both<decltype(tag)::value>(v[j], a, da);
                            hid[j] = a;
                            v[j] = da;
                        }
                    });
                    if (gated) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float a = hid[j];
                            hid[j] = a * u[j];
                            v[j] *= u[j];
                            u[j] = a;
                        }
                    }
                    if (MODE == PROD_DZ_TWO) {
                        // (columns beyond the last have g = 0: W2 is filled with zeros there)
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            dot = fmaf(hid[j], g[j], dot);
                            g[j] *= rw;
                            hid[j] *= rw;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        v[j] *= g[j];
                        if (gated) u[j] *= g[j];
                    }
                    // dz and the weighted h are rounded to 16 bits here, as operands of the products that follow (those would take twice the
                    // instructions for two terms a value): dx and dw are off by 2.3e-3 (bf16) and 2.9e-4 (fp16) against 64 bits in the
                    // relative norm, where one rounding of exact results is off by 1.7e-3 and 2.1e-4.
                    if (writes && col < p.cols) {
                        store8<BF16>(out + col, v);
                        if (gated) store8<BF16>(out + p.gate_rows + col, u);
                        if (MODE == PROD_DZ_TWO) store8<BF16>(out2 + col, hid);
                    }
                    if (p.column_sums) {
                        // (outputs were rounded; the sums are over the unrounded values; rows that do not count hold zeros)
                        float* to = p.column_sums + (size_t)(row0 / 32) * (p.cols + p.gate_rows) + col;
                        const float sv = column_sum(v, lane);
                        if (lane < 8 && col < p.cols) to[lane] = sv;
                        if (gated) {
                            const float su = column_sum(u, lane);
                            if (lane < 8 && col < p.cols) to[p.gate_rows + lane] = su;
                        }
                    }
                }
                if (MODE == PROD_DZ_TWO && counts) p.dot[(size_t)row * p.dots + (t.col / width) * tile_dots(SHAPE) + turn] = dot;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIRED) bar_arrive_remote(cluster_addr(smem_addr(&acc_empty[buf]), 0));
                else bar_arrive(&acc_empty[buf]);
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
        tmem_free<PAIRED>(tmem, TMEM_COLUMNS);
    }
}

template <int MODE, int SHAPE, bool BF16>
cudaError_t launch_as(som_layers* l, const ProdArgs& args, cudaStream_t st)
{
    const int64_t tiles = ((int64_t)args.row_tiles * args.col_tiles + (int64_t)args.row_tiles2 * args.col_tiles2) * (MODE == PROD_DW ? args.experts : 1) * args.splits;
    const int most = SHAPE == PAIR ? l->pairs : l->sm_count, blocks = SHAPE == PAIR ? 2 : 1;
    const int64_t at_once = tiles < most ? tiles : most, rounds = (tiles + at_once - 1) / at_once;
    if (rounds > l->rounds[MODE][SHAPE]) l->rounds[MODE][SHAPE] = rounds;
    return launch(l, k_product<MODE, SHAPE, BF16>, dim3((unsigned)at_once * blocks), THREADS, SMEM, st, blocks, args);
}

// wide tiles are for grouped rows
template <int MODE>
constexpr bool HAS_WIDE = MODE == PROD_FWD || MODE == PROD_DZ_TWO || MODE == PROD_DX;

template <int MODE>
cudaError_t launch_mode(som_layers* l, const ProdArgs& a, cudaStream_t st)
{
    if constexpr (HAS_WIDE<MODE>)
        if (a.shape == WIDE) return a.bf16 ? launch_as<MODE, WIDE, true>(l, a, st) : launch_as<MODE, WIDE, false>(l, a, st);
    if (a.shape == PAIR) return a.bf16 ? launch_as<MODE, PAIR, true>(l, a, st) : launch_as<MODE, PAIR, false>(l, a, st);
    return a.bf16 ? launch_as<MODE, NARROW, true>(l, a, st) : launch_as<MODE, NARROW, false>(l, a, st);
}

template <int MODE, bool BF16>
cudaError_t prepare_as(int* pairs)
{
    cudaError_t e = cudaFuncSetAttribute(k_product<MODE, NARROW, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if constexpr (HAS_WIDE<MODE>)
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_product<MODE, WIDE, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_product<MODE, PAIR, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
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
    e = cudaOccupancyMaxActiveClusters(&n, k_product<MODE, PAIR, BF16>, &c);
    if (n < *pairs) *pairs = n;
    return e;
}

template <int MODE>
cudaError_t prepare_mode(int* pairs)
{
    const cudaError_t e = prepare_as<MODE, true>(pairs);
    return e == cudaSuccess ? prepare_as<MODE, false>(pairs) : e;
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
        case PROD_FWD: e = launch_mode<PROD_FWD>(l, a, st); break;
        case PROD_DZ: e = launch_mode<PROD_DZ>(l, a, st); break;
        case PROD_DZ_TWO: e = launch_mode<PROD_DZ_TWO>(l, a, st); break;
        case PROD_DX: e = launch_mode<PROD_DX>(l, a, st); break;
        default: e = launch_mode<PROD_DW>(l, a, st); break;
    }
    return outcome(l, e);
}

}  // namespace lay
