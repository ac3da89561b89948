// Layer norm over the rows of a matrix, and its gradient.
//
//   h = x + residual, rounded to the matrix's type (it is an output, and the gradient starts from it); over a row of D values
//   mean = sum h / D, variance = sum (h - mean)^2 / D, n = (h - mean) r with r = 1 / sqrt(variance + eps), y = n weight + bias.
//   Gradient, with d = dy weight: dx = r (d - sum d / D - n sum (d n) / D) + dsum, dweight = sum over rows of dy n, dbias of dy.
//
// Bound by HBM: a few operations a value.  Everything between input and output is fp32; the variance is summed from the differences
// to the mean, not from squares, so that a row far from zero keeps its digits.
//
// A row is held in registers by a group of threads, 16 values each, loaded in 16 bytes where rows lie on them and value by value else; longer
// rows are walked.  8192 x 4096 bf16 with a residual 49 us (5.5 TB/s), its gradient 59 to 61 (4.5); rows of 4095 86 and 167.  The gradient is bound by
// its chain of sums, with four rows an SM at a time (one of 8192 columns): 31 instructions a value, half of the issue slots.  In fp32 and off 16 bytes it
// spills 44 to 152 bytes: 8192 x 4096 fp32 104 us (5.2 TB/s), 4096 x 8001 173.  Rows beyond the registers: 2000 x 65536 bf16 346 us and 882, 1.5 and
// 0.9 TB/s.
#include <initializer_list>
#include <type_traits>

#include "layers_host.cuh"
#include "layers_math.cuh"

namespace lay {
namespace {

struct NormArgs {
    const void *x, *residual, *weight, *bias;
    void *sum, *y;
    int64_t ldx, ldr, lds, ldy, T;
    int D, log;  // log: of the threads of a row (k_norm)
    float inv, eps;  // inv = 1 / D
};

struct NormBackArgs {
    const void *x, *weight, *dy, *dsum;
    void* dx;
    float* stats;  // [T][2] mean and r of every row, or nullptr (k_norm_back_any)
    float* part;   // [blocks][2][D] sums of the block's rows, or nullptr (k_norm_back)
    int64_t ldx, lddy, ldds;
    int64_t T;
    int D, log;
    float inv, eps;
};

struct ColumnArgs {
    const void *x, *dy;
    const float* stats;
    float* part;  // [parts][2][D]
    int64_t ldx, lddy, T;
    int D, parts;
};

struct ColumnJoinArgs {
    const float* part;
    void *dweight, *dbias;
    int D, parts;
};

__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ float wide(__half v) { return __half2float(v); }
__device__ __forceinline__ float wide(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class E>
__device__ __forceinline__ E narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

constexpr int ROW_THREADS = 256;

// the sums of N values over the block, to every thread, in a fixed order
template <int N, int THREADS>
__device__ __forceinline__ void block_sums(float (&v)[N])
{
    __shared__ float part[THREADS / 32][N];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
    __syncthreads();  // the last call's parts have been read
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) part[threadIdx.x >> 5][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.f;
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) v[i] += part[w][i];
    }
}

// ---- rows held in registers ------------------------------------------------------------------------------------------

constexpr int HELD = 16;  // values that a thread holds of a row: HELD * sizeof(E) / 16 pieces of 16 bytes, a group's threads apart

template <class E>
struct Piece {
    static constexpr int N = 16 / (int)sizeof(E), PAIRS = N / 2, COUNT = HELD / N;
    uint4 w;
    __device__ __forceinline__ void load(const E* p) { w = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(E* p) const { *reinterpret_cast<uint4*>(p) = w; }
    __device__ __forceinline__ void get(float2* v) const
    {
        if constexpr (sizeof(E) == 4) {
            v[0] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y)), v[1] = make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
        } else {
            v[0] = unpack2(w.x, BF16), v[1] = unpack2(w.y, BF16), v[2] = unpack2(w.z, BF16), v[3] = unpack2(w.w, BF16);
        }
    }
    __device__ __forceinline__ void put(const float2* v)
    {
        if constexpr (sizeof(E) == 4) w = make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
        else w = make_uint4(pack2(v[0].x, v[0].y, BF16), pack2(v[1].x, v[1].y, BF16), pack2(v[2].x, v[2].y, BF16), pack2(v[3].x, v[3].y, BF16));
    }
    static constexpr int BF16 [[maybe_unused]] = std::is_same<E, __nv_bfloat16>::value;
};

// Which columns of a row a thread holds.  LINED: rows on 16 bytes, of whole pieces; pieces lie a group's threads apart.  Else any row: single values
// that are a group's threads apart, each load and store of a warp 32 values in a row.
template <class E, bool LINED>
struct Held {
    using P = Piece<E>;
    int t, threads, D;
    __device__ __forceinline__ int column(int c, int j) const { return LINED ? (c * threads + t) * P::N + j : (c * P::N + j) * threads + t; }
    __device__ __forceinline__ bool has(int c) const { return column(c, 0) < D; }  // any of piece c
    // all of it: asked once a piece in fp32 (gradient of 16384 x 333 47.5 -> 38.7 us); 16-bit pieces are twice as long, and it cost registers (87 -> 98)
    __device__ __forceinline__ bool full(int c) const { return sizeof(E) == 4 && column(c, P::N - 1) < D; }
    // a value of piece c that is not in the row counts as 0
    __device__ __forceinline__ float2 only(int c, int pair, float2 v) const
    {
        return LINED || full(c) ? v : make_float2(column(c, 2 * pair) < D ? v.x : 0.f, column(c, 2 * pair + 1) < D ? v.y : 0.f);
    }
    __device__ __forceinline__ void load(const E* row, int c, P& q) const
    {
        if constexpr (LINED) {
            if (has(c)) q.load(row + column(c, 0));
        } else {
            uint32_t w[P::N];
            if (full(c)) {
                const uint32_t* from = reinterpret_cast<const uint32_t*>(row) + column(c, 0);
#pragma unroll
                for (int j = 0; j < P::N; ++j) w[j] = from[j * threads];
            } else {
#pragma unroll
                for (int j = 0; j < P::N; ++j) {
                    const int i = column(c, j);
                    if constexpr (sizeof(E) == 4) w[j] = i < D ? *(reinterpret_cast<const uint32_t*>(row) + i) : 0u;
                    else w[j] = i < D ? *(reinterpret_cast<const uint16_t*>(row) + i) : 0u;
                }
            }
            if constexpr (sizeof(E) == 4) q.w = make_uint4(w[0], w[1], w[2], w[3]);
            else q.w = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4 % P::N] | w[5 % P::N] << 16, w[6 % P::N] | w[7 % P::N] << 16);
        }
    }
    __device__ __forceinline__ void store(E* row, int c, const P& q) const
    {
        if constexpr (LINED) {
            if (has(c)) q.store(row + column(c, 0));
        } else {
            const uint32_t w[4] = {q.w.x, q.w.y, q.w.z, q.w.w};
            if (full(c)) {
                uint32_t* to = reinterpret_cast<uint32_t*>(row) + column(c, 0);
#pragma unroll
                for (int j = 0; j < P::N; ++j) to[j * threads] = w[j % 4];
            } else {
#pragma unroll
                for (int j = 0; j < P::N; ++j) {
                    const int i = column(c, j);
                    if constexpr (sizeof(E) == 4) {
                        if (i < D) *(reinterpret_cast<uint32_t*>(row) + i) = w[j % 4];
                    } else {
                        if (i < D) *(reinterpret_cast<uint16_t*>(row) + i) = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
                    }
                }
            }
        }
    }
    // weights of piece c (of a piece that is in the row)
    template <class W>
    __device__ __forceinline__ void weights(const void* base, int c, float2 (&v)[P::PAIRS]) const
    {
        const W* p = static_cast<const W*>(base);
        if constexpr (LINED) {
#pragma unroll
            for (int j = 0; j < P::PAIRS; j += Piece<W>::PAIRS) {
                Piece<W> q;
                q.load(p + column(c, 2 * j));
                q.get(v + j);
            }
        } else {
#pragma unroll
            for (int j = 0; j < P::PAIRS; ++j) {
                const int i = column(c, 2 * j), k = column(c, 2 * j + 1);
                v[j] = make_float2(i < D ? wide(p[i]) : 0.f, k < D ? wide(p[k]) : 0.f);
            }
        }
    }
};

// The arithmetic goes in pairs (one instruction for two values): what bounds these kernels next to HBM is the issue of instructions.
__device__ __forceinline__ float2 twice(float v) { return make_float2(v, v); }

// The sums of N = 1 or 2 values over the `warps` warps of a row's group, to every thread of it; `part` is this group's own, and another one
// than that of the sums before and after (which is what lets one barrier do).  Two values: after the first exchange the lower lanes sum the one
// and the upper lanes the other.
template <int N>
__device__ __forceinline__ void group_sums(float (&v)[N], float (*part)[N], int warps, int warp, int barrier)
{
    const int lane = threadIdx.x & 31;
    float s = v[0];
    if (N == 2) {
        const float give = lane < 16 ? v[N - 1] : v[0];
        s = (lane < 16 ? v[0] : v[N - 1]) + __shfl_xor_sync(0xffffffffu, give, 16);
    } else {
        s += __shfl_xor_sync(0xffffffffu, s, 16);
    }
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if (warps == 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = N == 1 ? s : __shfl_sync(0xffffffffu, s, 16 * i);
        return;
    }
    if (N == 1 ? lane == 0 : (lane & 15) == 0) part[warp][lane / 16 % N] = s;
    asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(32 * warps) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
    for (int w = 0; w < warps; ++w) {
        if constexpr (N == 2) {
            const float2 q = *reinterpret_cast<const float2*>(part[w]);
            v[0] += q.x;
            v[1] += q.y;
        } else {
            v[0] += part[w][0];
        }
    }
}

// s / n by n's inverse and one step of correction: the mean of equal values is that value
__device__ __forceinline__ float over(float s, float n, float inv)
{
    const float q = s * inv;
    return fmaf(fmaf(-q, n, s), inv, q);
}

constexpr int FRONT_THREADS = 256, FRONT_MOST = 1024;  // a block holds as many rows as groups fit into 256 threads, or one

template <class E, class W, bool LINED>
__global__ void __launch_bounds__(FRONT_MOST) k_norm(const NormArgs a)
{
    __shared__ float part0[FRONT_MOST / 32][1], part1[FRONT_MOST / 32][1];
    using P = Piece<E>;
    const int group = threadIdx.x >> a.log, threads = 1 << a.log, t = threadIdx.x & (threads - 1), warps = threads / 32, first = group * warps;
    const Held<E, LINED> held = {t, threads, a.D};
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x >> a.log) + group;
    enter();
    if (row >= a.T) return;  // (a whole group)
    const E* x = static_cast<const E*>(a.x) + row * a.ldx;
    const E* res = a.residual ? static_cast<const E*>(a.residual) + row * a.ldr : nullptr;
    P px[P::COUNT], pr[P::COUNT];
#pragma unroll
    for (int c = 0; c < P::COUNT; ++c) {
        held.load(x, c, px[c]);
        if (res) held.load(res, c, pr[c]);
    }
    float2 v[P::COUNT][P::PAIRS], s2 = twice(0.f);
#pragma unroll
    for (int c = 0; c < P::COUNT; ++c)
        if (held.has(c)) {
            px[c].get(v[c]);
            if (res) {
                float2 r[P::PAIRS];
                pr[c].get(r);
#pragma unroll
                for (int j = 0; j < P::PAIRS; ++j) v[c][j] = __fadd2_rn(v[c][j], r[j]);
                px[c].put(v[c]);
                px[c].get(v[c]);
            }
            if (a.sum) held.store(static_cast<E*>(a.sum) + row * a.lds, c, px[c]);
#pragma unroll
            for (int j = 0; j < P::PAIRS; ++j) s2 = __fadd2_rn(s2, v[c][j]);
        }
    float s[1] = {s2.x + s2.y};
    group_sums(s, part0 + first, warps, threadIdx.x / 32 - first, 1 + group);
    const float mean = over(s[0], (float)a.D, a.inv);
    s2 = twice(0.f);
#pragma unroll
    for (int c = 0; c < P::COUNT; ++c)
        if (held.has(c))
#pragma unroll
            for (int j = 0; j < P::PAIRS; ++j) {
                v[c][j] = held.only(c, j, __fadd2_rn(v[c][j], twice(-mean)));
                s2 = __ffma2_rn(v[c][j], v[c][j], s2);
            }
    s[0] = s2.x + s2.y;
    group_sums(s, part1 + first, warps, threadIdx.x / 32 - first, 1 + group);
    const float r = rsqrtf(s[0] * a.inv + a.eps);
#pragma unroll
    for (int c = 0; c < P::COUNT; ++c) {
        if (!held.has(c)) continue;
        float2 w[P::PAIRS];
#pragma unroll
        for (int j = 0; j < P::PAIRS; ++j) v[c][j] = __fmul2_rn(v[c][j], twice(r));
        if (a.weight) {
            held.template weights<W>(a.weight, c, w);
#pragma unroll
            for (int j = 0; j < P::PAIRS; ++j) v[c][j] = __fmul2_rn(v[c][j], w[j]);
        }
        if (a.bias) {
            held.template weights<W>(a.bias, c, w);
#pragma unroll
            for (int j = 0; j < P::PAIRS; ++j) v[c][j] = __fadd2_rn(v[c][j], w[j]);
        }
        px[c].put(v[c]);
        held.store(static_cast<E*>(a.y) + row * a.ldy, c, px[c]);
    }
}

// The gradient in one pass: blocks stay, and so do a thread's columns, so that dweight and dbias are summed in registers.  A thread brings its
// own pieces of the next rows into shared memory (cp.async), three rows ahead (fp32: one), and reads them there itself: no barrier, no registers for
// what is on its way.  A block's groups add up through shared memory and leave one part a block.
constexpr int BACK_THREADS = 512;
template <class E>
constexpr int back_smem()
{
    return 8 / (int)sizeof(E) * 3 * Piece<E>::COUNT * BACK_THREADS * 16;
}

template <int OFFSET>
__device__ __forceinline__ void copy16(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0 + %2], [%1], 16;" ::"r"(to), "l"(from), "n"(OFFSET) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Rows that are not LINED are loaded when their turn comes.
template <class E, class W, bool LINED>
__global__ void __launch_bounds__(BACK_THREADS, 1) k_norm_back(const NormBackArgs a)
{
    __shared__ __align__(8) float part0[BACK_THREADS / 32][2], part1[BACK_THREADS / 32][2];
    extern __shared__ __align__(16) uint4 ring[];  // [DEPTH][x, dy, dsum][COUNT][BACK_THREADS]; at the end the columns' sums, [2][D]
    using P = Piece<E>;
    constexpr int DEPTH = 8 / (int)sizeof(E);
    const int group = threadIdx.x >> a.log, threads = 1 << a.log, t = threadIdx.x & (threads - 1), warps = threads / 32, first = group * warps, groups = BACK_THREADS >> a.log;
    const int warp = threadIdx.x / 32 - first;
    const Held<E, LINED> held = {t, threads, a.D};
    enter();
    float2 w[P::COUNT][P::PAIRS], dw[P::COUNT][P::PAIRS], db[P::COUNT][P::PAIRS];
    const float n = (float)a.D, inv = a.inv;
    constexpr int WHAT = P::COUNT * BACK_THREADS * 16, STAGE = 3 * WHAT, RING = DEPTH * STAGE;  // bytes of one of x, dy and dsum, of a row's place, of all
    unsigned char* mine = reinterpret_cast<unsigned char*>(ring) + threadIdx.x * 16;
    const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
    auto piece = [&](int stage, int what, int c) { return reinterpret_cast<uint4*>(mine + stage + what * WHAT + c * (BACK_THREADS * 16)); };
    const int i0 = t * P::N, far = threads * P::N;  // this thread's first column, and from one of its pieces to the next
#pragma unroll
    for (int c = 0; c < P::COUNT; ++c) {
#pragma unroll
        for (int j = 0; j < P::PAIRS; ++j) w[c][j] = twice(1.f), dw[c][j] = db[c][j] = twice(0.f);
        if (a.weight && held.has(c)) held.template weights<W>(a.weight, c, w[c]);
    }
    if constexpr (LINED) {  // what is not copied stays zero: columns beyond the row's end, and dsum where there is none
#pragma unroll
        for (int stage = 0; stage < RING; stage += STAGE)
#pragma unroll
            for (int what = 0; what < 3; ++what)
#pragma unroll
                for (int c = 0; c < P::COUNT; ++c)
                    if (!held.has(c) || (what == 2 && !a.dsum)) *piece(stage, what, c) = make_uint4(0u, 0u, 0u, 0u);
    }
    int64_t row = (int64_t)blockIdx.x * groups + group;
    const int64_t step = (int64_t)gridDim.x * groups;
    // the next row to fetch, and where it lies
    int64_t ahead = row;
    const E *fx = static_cast<const E*>(a.x) + row * a.ldx + i0, *fg = static_cast<const E*>(a.dy) + row * a.lddy + i0;
    const E* fs = a.dsum ? static_cast<const E*>(a.dsum) + row * a.ldds + i0 : nullptr;
    E* to = a.dx ? static_cast<E*>(a.dx) + row * a.D : nullptr;
    auto fetch = [&](int stage) {
        if (ahead < a.T) {
            auto copy = [&](auto c) {
                constexpr int C = decltype(c)::value, AT = C * (BACK_THREADS * 16);
                if (i0 + C * far < a.D) {
                    copy16<AT>(mine_at + stage, fx + C * far);
                    copy16<AT + WHAT>(mine_at + stage, fg + C * far);
                    if (fs) copy16<AT + 2 * WHAT>(mine_at + stage, fs + C * far);
                }
            };
            copy(std::integral_constant<int, 0>());
            copy(std::integral_constant<int, 1>());
            if constexpr (P::COUNT == 4) {
                copy(std::integral_constant<int, 2>());
                copy(std::integral_constant<int, 3>());
            }
            ahead += step;
            fx += step * a.ldx;
            fg += step * a.lddy;
            if (fs) fs += step * a.ldds;
        }
        copies_end();
    };
    static_assert(P::COUNT == 2 || P::COUNT == 4, "pieces of a thread");
    if constexpr (LINED)
#pragma unroll
        for (int k = 0; k < DEPTH - 1; ++k) fetch(k * STAGE);
    int stage = 0;
    for (; row < a.T; row += step) {
        P qx[P::COUNT], qg[P::COUNT], qs[P::COUNT];
        if constexpr (LINED) {
            fetch(stage == 0 ? RING - STAGE : stage - STAGE);  // (the place of the row before)
            copies_wait<DEPTH - 1>();
        } else {
#pragma unroll
            for (int c = 0; c < P::COUNT; ++c) {
                held.load(static_cast<const E*>(a.x) + row * a.ldx, c, qx[c]);
                held.load(static_cast<const E*>(a.dy) + row * a.lddy, c, qg[c]);
                qs[c].w = make_uint4(0u, 0u, 0u, 0u);
                if (a.dsum) held.load(static_cast<const E*>(a.dsum) + row * a.ldds, c, qs[c]);
            }
        }
        float2 v[P::COUNT][P::PAIRS], g[P::COUNT][P::PAIRS], s0 = twice(0.f), s1 = twice(0.f);
#pragma unroll
        for (int c = 0; c < P::COUNT; ++c) {
            if constexpr (LINED) {
                qx[c].w = *piece(stage, 0, c);
                qg[c].w = *piece(stage, 1, c);
            }
            qx[c].get(v[c]);
            qg[c].get(g[c]);
#pragma unroll
            for (int j = 0; j < P::PAIRS; ++j) {
                s0 = __fadd2_rn(s0, v[c][j]);
                s1 = __ffma2_rn(g[c][j], w[c][j], s1);
            }
        }
        float s[2] = {s0.x + s0.y, s1.x + s1.y};
        group_sums(s, part0 + first, warps, warp, 1 + group);
        const float mean = over(s[0], n, inv), d_mean = over(s[1], n, inv);
        s0 = s1 = twice(0.f);
#pragma unroll
        for (int c = 0; c < P::COUNT; ++c)
            if (held.has(c))
#pragma unroll
                for (int j = 0; j < P::PAIRS; ++j) {
                    v[c][j] = held.only(c, j, __fadd2_rn(v[c][j], twice(-mean)));
                    s0 = __ffma2_rn(v[c][j], v[c][j], s0);
                    s1 = __ffma2_rn(v[c][j], __fmul2_rn(g[c][j], w[c][j]), s1);
                }
        s[0] = s0.x + s0.y, s[1] = s1.x + s1.y;
        group_sums(s, part1 + first, warps, warp, 1 + group);
        // n sum (d n) / D = (h - mean) r^2 sum (d (h - mean)) / D
        const float r = rsqrtf(s[0] * inv + a.eps), along = -(s[1] * inv) * r * r;
#pragma unroll
        for (int c = 0; c < P::COUNT; ++c) {
            float2 out[P::PAIRS];
            P q;
            q.w = LINED ? *piece(stage, 2, c) : qs[c].w;
            q.get(out);
#pragma unroll
            for (int j = 0; j < P::PAIRS; ++j) {
                const float2 d = __ffma2_rn(g[c][j], w[c][j], twice(-d_mean));
                dw[c][j] = __ffma2_rn(g[c][j], __fmul2_rn(v[c][j], twice(r)), dw[c][j]);
                db[c][j] = __fadd2_rn(db[c][j], g[c][j]);
                out[j] = __ffma2_rn(twice(r), __ffma2_rn(v[c][j], twice(along), d), out[j]);
            }
            if (to) {
                q.put(out);
                held.store(to, c, q);
            }
        }
        if (to) to += step * a.D;
        stage = stage + STAGE == RING ? 0 : stage + STAGE;
    }
    copies_wait<0>();
    float* columns = reinterpret_cast<float*>(ring);
    __syncthreads();  // every thread is done with its places of the ring
    if (!a.part) return;
    for (int k = 0; k < groups; ++k) {  // one group after the other, in their order
        if (group == k)
#pragma unroll
            for (int c = 0; c < P::COUNT; ++c)
#pragma unroll
                for (int j = 0; j < P::N; ++j) {
                    const int i = held.column(c, j);
                    const float dwi = j & 1 ? dw[c][j / 2].y : dw[c][j / 2].x, dbi = j & 1 ? db[c][j / 2].y : db[c][j / 2].x;
                    if (i < a.D) {
                        columns[i] = k ? columns[i] + dwi : dwi;
                        columns[a.D + i] = k ? columns[a.D + i] + dbi : dbi;
                    }
                }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < 2 * a.D; i += BACK_THREADS) a.part[(int64_t)blockIdx.x * 2 * a.D + i] = columns[i];
}

// ---- rows too long for the registers ---------------------------------------------------------------------------------

// A block a row, which it walks three times (from L1 or L2 after the first).
template <class E, class W>
__global__ void __launch_bounds__(ROW_THREADS) k_norm_any(const NormArgs a)
{
    enter();
    const int64_t row = blockIdx.x;
    const E* x = static_cast<const E*>(a.x) + row * a.ldx;
    const E* res = a.residual ? static_cast<const E*>(a.residual) + row * a.ldr : nullptr;
    E* sum = a.sum ? static_cast<E*>(a.sum) + row * a.lds : nullptr;
    E* y = static_cast<E*>(a.y) + row * a.ldy;
    auto value = [&](int i) { return res ? wide(narrow<E>(wide(x[i]) + wide(res[i]))) : wide(x[i]); };
    float s[1] = {0.f};
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) s[0] += value(i);
    block_sums<1, ROW_THREADS>(s);
    const float mean = s[0] / (float)a.D;
    s[0] = 0.f;
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) {
        const float c = value(i) - mean;
        s[0] = fmaf(c, c, s[0]);
    }
    block_sums<1, ROW_THREADS>(s);
    const float r = 1.f / sqrtf(s[0] / (float)a.D + a.eps);
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) {
        const float h = value(i);
        float n = (h - mean) * r;
        if (a.weight) n *= wide(static_cast<const W*>(a.weight)[i]);
        if (a.bias) n += wide(static_cast<const W*>(a.bias)[i]);
        y[i] = narrow<E>(n);
        if (sum) sum[i] = narrow<E>(h);
    }
}

template <class E, class W>
__global__ void __launch_bounds__(ROW_THREADS) k_norm_back_any(const NormBackArgs a)
{
    enter();
    const int64_t row = blockIdx.x;
    const E* x = static_cast<const E*>(a.x) + row * a.ldx;
    const E* dy = static_cast<const E*>(a.dy) + row * a.lddy;
    const E* dsum = a.dsum ? static_cast<const E*>(a.dsum) + row * a.ldds : nullptr;
    const W* w = static_cast<const W*>(a.weight);
    const float n = (float)a.D;  // (divided by, not multiplied by its inverse: the mean of equal values is that value)
    float s[2] = {0.f, 0.f};
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) {
        s[0] += wide(x[i]);
        s[1] += w ? wide(dy[i]) * wide(w[i]) : wide(dy[i]);
    }
    block_sums<2, ROW_THREADS>(s);
    const float mean = s[0] / n, d_mean = s[1] / n;
    s[0] = s[1] = 0.f;
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) {
        const float c = wide(x[i]) - mean, d = w ? wide(dy[i]) * wide(w[i]) : wide(dy[i]);
        s[0] = fmaf(c, c, s[0]);
        s[1] = fmaf(c, d, s[1]);
    }
    block_sums<2, ROW_THREADS>(s);
    const float r = 1.f / sqrtf(s[0] / n + a.eps), along = s[1] / n * r * r;  // n sum (d n) / D = (h - mean) r^2 sum (d (h - mean)) / D
    if (a.stats && threadIdx.x == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, r);
    if (!a.dx) return;
    E* dx = static_cast<E*>(a.dx) + row * a.D;
    for (int i = threadIdx.x; i < a.D; i += ROW_THREADS) {
        const float c = wide(x[i]) - mean, d = w ? wide(dy[i]) * wide(w[i]) : wide(dy[i]);
        float g = r * (d - d_mean - c * along);
        if (dsum) g += wide(dsum[i]);
        dx[i] = narrow<E>(g);
    }
}

// The columns' sums from the rows' statistics: 32 columns a block, eight rows at a time of one of `parts` stretches of the rows.
template <class E>
__global__ void __launch_bounds__(256) k_norm_columns(const ColumnArgs a)
{
    __shared__ float part[8][2][32];
    enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    const int64_t from = a.T * blockIdx.y / a.parts, to = a.T * (blockIdx.y + 1) / a.parts;
    float dw = 0.f, db = 0.f;
    if (col < a.D)
        for (int64_t row = from + warp; row < to; row += 8) {
            const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * row);
            const float d = wide(static_cast<const E*>(a.dy)[row * a.lddy + col]);
            dw = fmaf(d, (wide(static_cast<const E*>(a.x)[row * a.ldx + col]) - st.x) * st.y, dw);
            db += d;
        }
    part[warp][0][lane] = dw;
    part[warp][1][lane] = db;
    __syncthreads();
    if (warp < 2 && col < a.D) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += part[i][warp][lane];
        a.part[((int64_t)blockIdx.y * 2 + warp) * a.D + col] = s;
    }
}

constexpr int JOIN_AHEAD = 20;  // parts of a warp: all of 148 at once

// the parts' sum, in a fixed order
template <class W>
__global__ void __launch_bounds__(256) k_norm_join(const ColumnJoinArgs a)
{
    __shared__ float part[8][32];
    enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t i = (int64_t)blockIdx.x * 32 + lane;  // of 2 D sums
    float s = 0.f;
    if (i < 2 * (int64_t)a.D)
        for (int p = warp; p < a.parts; p += 8 * JOIN_AHEAD) {
            float v[JOIN_AHEAD];  // on their way at once (beyond the last part its values again, without a branch)
#pragma unroll
            for (int k = 0; k < JOIN_AHEAD; ++k) v[k] = a.part[(int64_t)min(p + 8 * k, a.parts - 1) * 2 * a.D + i];
#pragma unroll
            for (int k = 0; k < JOIN_AHEAD; ++k) s += p + 8 * k < a.parts ? v[k] : 0.f;
        }
    part[warp][lane] = s;
    __syncthreads();
    if (warp > 0 || i >= 2 * (int64_t)a.D) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += part[w][lane];
    W* to = static_cast<W*>(i < a.D ? a.dweight : a.dbias);
    if (to) to[i < a.D ? i : i - a.D] = narrow<W>(s);
}

// f(E(), W()) of the matrix's and the weights' types
template <class F>
cudaError_t by_types(int type, int weights_type, F&& f)
{
    if (type == SOM_F32) return f(float(), float());
    if (type == SOM_F16) return weights_type == SOM_F32 ? f(__half(), float()) : f(__half(), __half());
    return weights_type == SOM_F32 ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
}

int check_norm(const som_layers* l, int type, int weights_type, int64_t T, int64_t D, float eps)
{
    if (!l || T < 0 || D <= 0 || type < SOM_F32 || type > SOM_BF16 || (weights_type != SOM_F32 && weights_type != type) || !(eps >= 0.f))
        return SOM_ERR_INVALID_ARG;
    return T >= MOST_ROWS || D > MOST_COLS ? SOM_ERR_UNSUPPORTED : SOM_OK;
}

// Logarithm of the threads of a row that is held in registers: as many warps, a power of two, as hold it.  0: too long
int group_of(int64_t D, int most)
{
    if (D > (int64_t)most * HELD) return 0;
    int log = 5;
    while (((int64_t)HELD << log) < D) ++log;
    return log;
}

// whether rows lie on 16 bytes and are whole pieces of them
bool lined(int64_t D, int bytes, std::initializer_list<const void*> rows, std::initializer_list<int64_t> lds)
{
    bool on = D * bytes % 16 == 0;
    for (const void* p : rows) on = on && aligned16(p);
    for (int64_t ld : lds) on = on && ld * bytes % 16 == 0;
    return on;
}

// rows of a norm's matrix: present, and long enough
int check_row(const void* p, int64_t ld, int64_t D, int64_t T)
{
    if (T == 0) return SOM_OK;
    if (!p || ld < D) return SOM_ERR_INVALID_ARG;
    return ld >= (int64_t)1 << 32 ? SOM_ERR_UNSUPPORTED : SOM_OK;
}

template <class E, class W>
cudaError_t prepare_as()
{
    static_assert(back_smem<E>() >= 2 * BACK_THREADS * HELD * (int)sizeof(float), "the columns' sums take the ring's place");
    const cudaError_t e = cudaFuncSetAttribute(k_norm_back<E, W, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, back_smem<E>());
    return e == cudaSuccess ? cudaFuncSetAttribute(k_norm_back<E, W, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, back_smem<E>()) : e;
}

}  // namespace

cudaError_t prepare_norm()
{
    cudaError_t e = prepare_as<float, float>();
    if (e == cudaSuccess) e = prepare_as<__half, __half>();
    if (e == cudaSuccess) e = prepare_as<__half, float>();
    if (e == cudaSuccess) e = prepare_as<__nv_bfloat16, __nv_bfloat16>();
    return e == cudaSuccess ? prepare_as<__nv_bfloat16, float>() : e;
}

}  // namespace lay

using namespace lay;

extern "C" {

int som_norm(som_layers* l, int type, int64_t T, int64_t D, const void* x, int64_t ldx, const void* weight, const void* bias,
             int weights_type, const void* residual, int64_t ldr, float eps, void* sum, int64_t lds, void* y, int64_t ldy, void* stream)
{
    LAY_TRY(check_norm(l, type, weights_type, T, D, eps));
    LAY_TRY(check_row(x, ldx, D, T));
    LAY_TRY(check_row(y, ldy, D, T));
    if (residual) LAY_TRY(check_row(residual, ldr, D, T));
    if (sum) LAY_TRY(check_row(sum, lds, D, T));
    if (T == 0) return SOM_OK;
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    int log = group_of(D, FRONT_MOST);
    const bool on16 = lined(D, type == SOM_F32 ? 4 : 2, {x, residual, weight, bias, sum, y}, {ldx, residual ? ldr : 0, sum ? lds : 0, ldy});
    // Rows of 16-bit values that are not on 16 bytes: loads of two bytes are what costs, and beyond this length three walks with more threads are as
    // fast.  Held / walked, with a residual: 16384 x 1001 47 / 66 us, 16384 x 2001 91 / 94, 8192 x 4095 90 / 86, 2000 x 12001 113 / 78; fp32 4096 x 8001 104 / 146.
    if (!on16 && type != SOM_F32 && D > 2048) log = 0;
    const NormArgs a = {x, residual, weight, bias, sum, y, ldx, ldr, lds, ldy, T, (int)D, log, 1.f / (float)D, eps};
    return outcome(l, by_types(type, weights_type, [&](auto e, auto w) {
                       using E = decltype(e);
                       using W = decltype(w);
                       if (!log) return launch(l, k_norm_any<E, W>, dim3((unsigned)T), ROW_THREADS, 0, st, 1, a);
                       const int threads = (1 << log) < FRONT_THREADS ? FRONT_THREADS : 1 << log;
                       return launch(l, on16 ? k_norm<E, W, true> : k_norm<E, W, false>, dim3((unsigned)tiles_of(T, threads >> log)), threads, 0, st, 1, a);
                   }));
}

int som_norm_backward(som_layers* l, int type, int64_t T, int64_t D, const void* x, int64_t ldx, const void* weight, int weights_type,
                      const void* dy, int64_t lddy, const void* dsum, int64_t ldds, float eps, void* dx, void* dweight, void* dbias,
                      void* stream)
{
    LAY_TRY(check_norm(l, type, weights_type, T, D, eps));
    LAY_TRY(check_row(x, ldx, D, T));
    LAY_TRY(check_row(dy, lddy, D, T));
    if (dsum) LAY_TRY(check_row(dsum, ldds, D, T));
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const size_t wide_bytes = weights_type == SOM_F32 ? 4 : 2;
    if (T == 0) {
        if (dweight) SOM_CK(l, cudaMemsetAsync(dweight, 0, D * wide_bytes, st));
        if (dbias) SOM_CK(l, cudaMemsetAsync(dbias, 0, D * wide_bytes, st));
        return SOM_OK;
    }
    const bool columns = dweight || dbias;
    // Held whatever the alignment.  Rows off 16 bytes with dsum, held / walked, in us: bf16 16384 x 101 30 / 46, 16384 x 1001 87 / 123, 8192 x 4095 166 / 207,
    // 4096 x 8001 176 / 197; fp32 16384 x 1001 84 / 132, 4096 x 8001 173 / 235.
    const int log = group_of(D, BACK_THREADS);
    const bool on16 = lined(D, type == SOM_F32 ? 4 : 2, {x, dy, dsum, dx, weight}, {ldx, lddy, dsum ? ldds : 0});
    int64_t parts;
    if (log) {
        parts = tiles_of(T, BACK_THREADS >> log);
        if (parts > l->sm_count) parts = l->sm_count;
    } else {
        parts = 4 * (int64_t)l->sm_count / tiles_of(D, 32);
        // A thread adds at most a 64th of the rows one after the other (or eight), which is what bounds the sums' error.  As many as fill the SMs / this, in us:
        // 2000 x 12000 bf16 170 / 125, 8192 x 8200 355 / 309, 2000 x 65536 915 / 882.
        if (parts < 8) parts = 8;
        if (parts > T / 64) parts = T / 64;
        if (parts < 1) parts = 1;
    }
    float *stats = nullptr, *part = nullptr;
    auto carve = [&](Carver c) {
        if (!log) stats = c.take<float>(2 * T);
        part = c.take<float>(parts * 2 * D);
        return c.used;
    };
    if (columns) {
        LAY_TRY(ensure(l, carve(Carver{nullptr, 0})));
        carve(Carver{static_cast<unsigned char*>(l->ws), 0});
    }
    const NormBackArgs a = {x, weight, dy, dsum, dx, stats, part, ldx, lddy, ldds, T, (int)D, log, 1.f / (float)D, eps};
    const ColumnArgs b = {x, dy, stats, part, ldx, lddy, T, (int)D, (int)parts};
    const ColumnJoinArgs j = {part, dweight, dbias, (int)D, (int)parts};
    return outcome(l, by_types(type, weights_type, [&](auto e, auto w) {
                       using E = decltype(e);
                       using W = decltype(w);
                       cudaError_t r;
                       if (log) {
                           r = launch(l, on16 ? k_norm_back<E, W, true> : k_norm_back<E, W, false>, dim3((unsigned)parts), BACK_THREADS, back_smem<E>(), st, 1, a);
                       } else {
                           r = launch(l, k_norm_back_any<E, W>, dim3((unsigned)T), ROW_THREADS, 0, st, 1, a);
                           if (r == cudaSuccess && columns) r = launch(l, k_norm_columns<E>, dim3((unsigned)tiles_of(D, 32), (unsigned)parts), 256, 0, st, 1, b);
                       }
                       if (r != cudaSuccess || !columns) return r;
                       return launch(l, k_norm_join<W>, dim3((unsigned)tiles_of(2 * D, 32)), 256, 0, st, 1, j);
                   }));
}

}  // extern "C"
