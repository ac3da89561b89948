// A step of AdamW over many tensors in one launch, with its moments in 32 bits or in 8.
//
//   g = scale grad, m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2,
//   p = p (1 - rate decay) - rate (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps); a 16-bit copy of p where one is wanted.
//
// Moments in 8 bits: 256 consecutive elements share a power of two, that of their largest magnitude (the next where it is above the
// largest code, which could not be rounded up, and a growing moment would stay at it); an element's code is a
// small floating-point number below it: m a sign, 4 bits of exponent and 3 of fraction, v 5 and 3 (it spans twice m's powers), both
// with gradual underflow, 2^-17 and 2^-33 of the block's power at the least.  Rounding to the nearest would hold v still for ever: a
// step moves it by a thousandth, a code is a sixteenth apart.  So a value is rounded up with the probability that makes the code
// right in the mean, by 16 random bits that are a function of (seed, tensor, element): the same call gives the same codes.  A
// positive v never becomes 0 (the quotient would lose its measure).  The fp32 value that a code is made from is the one that the step used.
//
// Products and sums that the codes come from are rounded one by one (no fused multiply-add): which code is taken is then a matter of
// the definition, not of the compiler.  With moments in 32 bits all operations are, the parameter's too: a 16-bit copy that a fused last product
// moves to its other neighbour now and then (5 of a million) is not the one of the formula in fp32.
//
// Bound by HBM: 28 bytes an element with fp32 parameters, a bf16 copy and bf16 gradients, 10 with 8-bit moments and bf16
// parameters.  A block takes 2048 elements of one tensor, a thread eight in a row, a warp the 256 that share a power; the tensors'
// addresses are the kernel's own parameters (no table to copy, and a captured graph keeps them).
#include "layers_host.cuh"
#include "layers_math.cuh"

namespace lay {
namespace {

constexpr int ADAM_THREADS = 256, ADAM_BLOCK = 256, ADAM_CHUNK = 8 * ADAM_THREADS;

struct Hyper {
    float keep, rate, b1, c1, b2, c2, k1, k2, eps;  // keep = 1 - rate decay; c = 1 - b; k = 1 / (1 - b^t)
    uint32_t seed;
};

struct HyperPairs {
    float2 keep, minus_rate, b1, c1, b2, c2, k1, k2, eps;
};

template <int CAP>
struct AdamTable {
    som_adamw_tensor item[CAP];  // first_chunk: the launch's chunks before the tensor
    int count;
    int param_bf16, grad_bf16, copy_bf16;
    Hyper h;
    HyperPairs pairs;  // the same
    const Hyper* h_at;  // in its place where the host does not know it
    const float* scale;
};

template <int CAP>
struct MomentTable {
    som_adamw_tensor item[CAP];  // param, copy: where m and v go
    int count;
};

struct HyperArgs {
    Hyper* to;
    double rate, b1, b2, eps, decay;
    int64_t step;
    const float* rate_at;
    const int64_t* step_at;
    uint32_t seed;
};

__host__ __device__ inline Hyper hyper_of(double rate, double b1, double b2, double eps, double decay, int64_t step, uint32_t seed)
{
    return {(float)(1.0 - rate * decay), (float)rate, (float)b1, (float)(1.0 - b1), (float)b2, (float)(1.0 - b2),
            (float)(1.0 / (1.0 - pow(b1, (double)step))), (float)(1.0 / (1.0 - pow(b2, (double)step))), (float)eps, seed};
}

__host__ __device__ inline HyperPairs pairs_of(const Hyper& h)
{
    auto two = [](float v) { return make_float2(v, v); };
    return {two(h.keep), two(-h.rate), two(h.b1), two(h.c1), two(h.b2), two(h.c2), two(h.k1), two(h.k2), two(h.eps)};
}

__global__ void k_adamw_hyper(const HyperArgs a)
{
    enter();
    const int64_t step = a.step_at ? max(*a.step_at, (int64_t)1) : a.step;
    *a.to = hyper_of(a.rate_at ? (double)*a.rate_at : a.rate, a.b1, a.b2, a.eps, a.decay, step, a.step_at ? a.seed + (uint32_t)step : a.seed);
}

// mix(x) = y ^ (y >> 16) with y = mix_half(x)
__device__ __forceinline__ uint32_t mix_half(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x9E3779B9u;
    x ^= x >> 15;
    return x * 0xBB67AE85u;
}
__device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x = mix_half(x);
    return x ^ (x >> 16);
}

// eight consecutive values as fp32; `left` of them exist (vector loads only where all do)
__device__ __forceinline__ void read8(const float* p, float (&v)[8], bool whole, int left)
{
    if (whole) {
        const float4 a = *reinterpret_cast<const float4*>(p), b = *(reinterpret_cast<const float4*>(p) + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
    }
}
__device__ __forceinline__ void read8(const uint16_t* p, float (&v)[8], bool whole, int left, int bf16)
{
    if (whole) {
        load8(p, v, bf16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? unpack1(p[i], bf16) : 0.f;
    }
}
__device__ __forceinline__ void write8(float* p, const float (&v)[8], bool whole, int left)
{
    if (whole) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *(reinterpret_cast<float4*>(p) + 1) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = v[i];
    }
}
__device__ __forceinline__ void write8(uint16_t* p, const float (&v)[8], bool whole, int left, int bf16)
{
    const uint4 w = make_uint4(pack2(v[0], v[1], bf16), pack2(v[2], v[3], bf16), pack2(v[4], v[5], bf16), pack2(v[6], v[7], bf16));
    if (whole) {
        *reinterpret_cast<uint4*>(p) = w;
    } else {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (uint16_t)(u[i / 2] >> (16 * (i & 1)));
    }
}
__device__ __forceinline__ uint2 read_codes(const uint8_t* p, bool whole, int left)
{
    if (whole) return *reinterpret_cast<const uint2*>(p);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) w[i / 4] |= (uint32_t)p[i] << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void write_codes(uint8_t* p, uint2 c, bool whole, int left)
{
    if (whole) {
        *reinterpret_cast<uint2*>(p) = c;
    } else {
        const uint32_t w[2] = {c.x, c.y};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (uint8_t)(w[i / 4] >> (8 * (i & 3)));
    }
}

__device__ __forceinline__ float fast_rsqrt(float x)
{
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// off by 2^-22, also where x is subnormal
__device__ __forceinline__ float near_sqrt(float x)
{
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 2^(e - 127) of an exponent byte; 255 (a block that holds an infinity or NaN) gives infinity, and 0 times it NaN
__device__ __forceinline__ float power_of(uint32_t e) { return __uint_as_float(max(e << 23, 0x00400000u)); }
// 2^(127 - e), e <= 254
__device__ __forceinline__ float power_below(uint32_t e) { return __int_as_float(max((254 - (int)e) * (1 << 23), 0x00400000)); }

__device__ __forceinline__ float2 twice(float v) { return make_float2(v, v); }

// The sum of two products that are rounded by themselves.  (Of a packed product and a packed sum the compiler makes one rounding, whatever they say.)
__device__ __forceinline__ float2 sum2(float2 a, float2 b) { return make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)); }

// the values of eight codes: a code's bits are the top of a number of the smallest exponents, which 2^112 (or 2^96) lifts to [0, 2)
template <bool SIGNED>
__device__ __forceinline__ void decode8(uint2 c, uint32_t e, float2 (&v)[4])
{
    const float2 by = twice(power_of(e)), top = twice(SIGNED ? 0x1p112f : 0x1p96f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? c.x : c.y;
        const int at = 16 * (i & 1);  // of the lower byte
        uint32_t lo, hi;
        if (SIGNED) {  // the sign to the top, the other seven bits to 20..26
            lo = (uint32_t)((int32_t)(w * (1u << (24 - at))) >> 4) & 0x87f00000u;
            hi = (uint32_t)((int32_t)(w * (1u << (16 - at))) >> 4) & 0x87f00000u;
        } else {  // (products: shifts have a pipe of half the width)
            lo = (w & (0xffu << at)) * (1u << (20 - at));
            hi = at ? (w >> 4) & 0x0ff00000u : (w & 0xff00u) * (1u << 12);
        }
        v[i] = __fmul2_rn(__fmul2_rn(make_float2(__uint_as_float(lo), __uint_as_float(hi)), top), by);
    }
}

// 16 x; a product, since shifts have a pipe of half the width, and an instruction of its own, since the compiler (12.9) took the top bytes of x
// itself for those of 16 x where x was negative, in an expression that took the sign from x in the same step.  (In this one the plain product gives the
// right codes too; the tests compare every bit.)
__device__ __forceinline__ uint32_t times16(uint32_t x)
{
    uint32_t r;
    asm("mul.lo.u32 %0, %1, 16;" : "=r"(r) : "r"(x));
    return r;
}

__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// codes of eight values of a block of a warp's 256, and the block's exponent; h: 16 random bits for each.
// (A code above the largest is met only where the exponent is 255.)
template <bool SIGNED>
__device__ __forceinline__ uint32_t encode8(const float2 (&v)[4], const uint32_t (&h)[8], uint2& codes)
{
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = largest(most, v[i].x, v[i].y);
    // a fraction of 7 / 8 and more carries into the exponent
    const uint32_t e = (min(__reduce_max_sync(0xffffffffu, __float_as_uint(most)), 0x7f800000u) + 0x100000u) >> 23;
    const float2 up = twice(power_below(e)), top = twice(SIGNED ? 0x1p-112f : 0x1p-96f);
    uint32_t u[8], bits[8];  // u: the code in the top byte, but for the sign
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = __fmul2_rn(__ffma2_rn(v[i], up, twice(0.f)), top);  // (-0 becomes 0)
        bits[2 * i] = __float_as_uint(a.x), bits[2 * i + 1] = __float_as_uint(a.y);
#pragma unroll
        for (int k = 2 * i; k < 2 * i + 2; ++k) u[k] = times16(bits[k]) + h[k] * 256u;
    }
    codes = make_uint2(top_bytes(u[0], u[1], u[2], u[3]), top_bytes(u[4], u[5], u[6], u[7]));
    if (SIGNED) {  // (the signs of four at a time)
        codes.x |= top_bytes(bits[0], bits[1], bits[2], bits[3]) & 0x80808080u;
        codes.y |= top_bytes(bits[4], bits[5], bits[6], bits[7]) & 0x80808080u;
    }
    if (!SIGNED) {  // a code of 0 becomes 1 where the value is not 0
        if ((((codes.x - 0x01010101u) & ~codes.x) | ((codes.y - 0x01010101u) & ~codes.y)) & 0x80808080u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t& w = i < 2 ? codes.x : codes.y;
                const int at = 16 * (i & 1);
                if (v[i].x > 0.f && !(w & (0xffu << at))) w |= 1u << at;
                if (v[i].y > 0.f && !(w & (0xff00u << at))) w |= 0x100u << at;
            }
        }
    }
    return e;
}

// the tensor that a chunk of the launch belongs to
template <class TABLE>
__device__ __forceinline__ int tensor_of(const TABLE& t, uint32_t chunk)
{
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.item[mid].first_chunk <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Where a thread's eight elements lie, and how many of them there are.
struct Place {
    int64_t at;
    int left;
    bool whole;  // all eight, in vectors
};
__device__ __forceinline__ bool on16(const som_adamw_tensor& it)
{
    return ((reinterpret_cast<uintptr_t>(it.param) | reinterpret_cast<uintptr_t>(it.grad) | reinterpret_cast<uintptr_t>(it.copy) |
             reinterpret_cast<uintptr_t>(it.m) | reinterpret_cast<uintptr_t>(it.v)) & 15u) == 0;
}
__device__ __forceinline__ Place place_of(const som_adamw_tensor& it, int64_t at)
{
    const int left = it.n - at >= 8 ? 8 : it.n > at ? (int)(it.n - at) : 0;
    return {at, left, left == 8 && on16(it)};
}

// (BF16: the 16-bit tensors are bf16; else the table says what each is)
template <bool P16, bool G16, bool BF16, class TABLE>
__device__ __forceinline__ void read_params(const TABLE& t, const som_adamw_tensor& it, const Place& q, float (&p)[8], float (&g)[8])
{
    if (P16) read8(static_cast<const uint16_t*>(it.param) + q.at, p, q.whole, q.left, BF16 || t.param_bf16);
    else read8(static_cast<const float*>(it.param) + q.at, p, q.whole, q.left);
    if (G16) read8(static_cast<const uint16_t*>(it.grad) + q.at, g, q.whole, q.left, BF16 || t.grad_bf16);
    else read8(static_cast<const float*>(it.grad) + q.at, g, q.whole, q.left);
}

template <bool P16, bool COPY, bool BF16, class TABLE>
__device__ __forceinline__ void write_params(const TABLE& t, const som_adamw_tensor& it, const Place& q, const float (&p)[8])
{
    if (P16) write8(static_cast<uint16_t*>(it.param) + q.at, p, q.whole, q.left, BF16 || t.param_bf16);
    else write8(static_cast<float*>(it.param) + q.at, p, q.whole, q.left);
    if (COPY) write8(static_cast<uint16_t*>(it.copy) + q.at, p, q.whole, q.left, BF16 || t.copy_bf16);
}

// P16, G16: 16-bit parameters, gradients; COPY: a 16-bit copy of fp32 parameters
template <bool P16, bool G16, bool COPY, int CAP>
__global__ void __launch_bounds__(ADAM_THREADS) k_adamw(const __grid_constant__ AdamTable<CAP> t)
{
    enter();
    const som_adamw_tensor& it = t.item[tensor_of(t, blockIdx.x)];
    const Place q = place_of(it, (int64_t)(blockIdx.x - it.first_chunk) * ADAM_CHUNK + threadIdx.x * 8);
    const float scale = t.scale ? *t.scale : 1.f;
    if (!(fabsf(scale) <= 3.4028235e38f) || q.left == 0) return;  // (an infinity or NaN: the step is left out)
    const Hyper h = t.h_at ? *t.h_at : t.h;
    float p[8], g[8], m[8], v[8];
    read_params<P16, G16, false>(t, it, q, p, g);
    read8(static_cast<const float*>(it.m) + q.at, m, q.whole, q.left);
    read8(static_cast<const float*>(it.v) + q.at, v, q.whole, q.left);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (t.scale) g[i] = __fmul_rn(g[i], scale);
        m[i] = __fadd_rn(__fmul_rn(m[i], h.b1), __fmul_rn(g[i], h.c1));
        v[i] = __fadd_rn(__fmul_rn(v[i], h.b2), __fmul_rn(__fmul_rn(g[i], g[i]), h.c2));
        const float change = __fmul_rn(m[i], h.k1) / __fadd_rn(sqrtf(__fmul_rn(v[i], h.k2)), h.eps);
        p[i] = __fsub_rn(__fmul_rn(p[i], h.keep), __fmul_rn(change, h.rate));
    }
    write_params<P16, COPY, false>(t, it, q, p);
    write8(static_cast<float*>(it.m) + q.at, m, q.whole, q.left);
    write8(static_cast<float*>(it.v) + q.at, v, q.whole, q.left);
}

// The same with moments in 8 bits.  Bound by the issue of instructions (67 an element, slots 76 % busy) as much as by HBM: arithmetic goes in
// pairs, square root and quotient are the approximations (2^-22 of the change).  AT: the step's numbers come from memory; else they are
// the kernel's parameters, in pairs.  BF16: 16-bit parameters and gradients are bf16 (with fp32 parameters the choice at run time was
// faster: 546 us, 643 with registers spilled).  Forms with fp16 parameters, with 16-bit gradients beside fp32 parameters or with the step's numbers in
// memory spill 4 to 16 bytes.  210 million elements: bf16 parameters 496 us (4.2 TB/s), fp32 with a bf16 copy 546 (6.1 TB/s).
// Slower: the arithmetic in scalars (560 and 644), two and four times eight elements a thread (506 to 570 and 610 to 870), 5, 7 or 8 blocks an SM.
template <bool P16, bool G16, bool COPY, bool BF16, int CAP, bool AT>
__global__ void __launch_bounds__(ADAM_THREADS, 6) k_adamw8(const __grid_constant__ AdamTable<CAP> t)
{
    enter();
    const som_adamw_tensor& it = t.item[tensor_of(t, blockIdx.x)];
    const float scale = t.scale ? *t.scale : 1.f;
    if (!(fabsf(scale) <= 3.4028235e38f)) return;
    HyperPairs at_h;
    if (AT) at_h = pairs_of(*t.h_at);
    const HyperPairs& h = AT ? at_h : t.pairs;
    const uint32_t seed = AT ? t.h_at->seed : t.h.seed;
    // (the warp's number by a shuffle: what hangs on it alone is then computed once a warp)
    const int lane = threadIdx.x & 31, off = threadIdx.x * 8, warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0);
    const int64_t base = (int64_t)(blockIdx.x - it.first_chunk) * ADAM_CHUNK, blocks = (it.n + ADAM_BLOCK - 1) / ADAM_BLOCK;
    const int here = (int)(it.n - base < ADAM_CHUNK ? it.n - base : ADAM_CHUNK) - off;  // elements of the tensor from this thread's first on
    if (here + lane * 8 <= 0) return;  // none of the warp's
    const Place q = {base + off, here < 8 ? (here > 0 ? here : 0) : 8, here >= 8 && on16(it)};
    uint8_t* em = it.exponents + base / ADAM_BLOCK + warp;
    uint8_t* ev = em + blocks;
    float p[8], g[8];
    read_params<P16, G16, BF16>(t, it, q, p, g);
    const float top = largest(largest(largest(g[0], g[1], g[2]), g[3], g[4]), largest(g[5], g[6], g[7]), 0.f);
    const uint32_t e_v = *ev;
    // (otherwise v k2 is below 2 power k2 + 1e36, and so finite; a NaN among the gradients counts as a large one)
    const bool by_root = h.eps.x < 0.999e-8f || !(top * fabsf(scale) < 1e18f) || !(power_of(e_v) * h.k2.x < 1e38f);
    float2 m[4], v[4];
    {
        const uint2 mc = read_codes(static_cast<const uint8_t*>(it.m) + q.at, q.whole, q.left), vc = read_codes(static_cast<const uint8_t*>(it.v) + q.at, q.whole, q.left);
        decode8<true>(mc, *em, m);
        decode8<false>(vc, e_v, v);
    }
    auto moves = [&](auto root_of) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 gi = __fmul2_rn(make_float2(g[2 * i], g[2 * i + 1]), twice(scale));  // (by 1 where there is none)
            m[i] = sum2(__fmul2_rn(m[i], h.b1), __fmul2_rn(gi, h.c1));
            v[i] = sum2(__fmul2_rn(v[i], h.b2), __fmul2_rn(__fmul2_rn(gi, gi), h.c2));
            const float2 up = __fmul2_rn(m[i], h.k1), root = __fadd2_rn(root_of(__fmul2_rn(v[i], h.k2)), h.eps);
            const float2 change = __fmul2_rn(up, make_float2(fast_rcp(root.x), fast_rcp(root.y)));
            const float2 now = __ffma2_rn(change, h.minus_rate, __fmul2_rn(make_float2(p[2 * i], p[2 * i + 1]), h.keep));
            p[2 * i] = now.x, p[2 * i + 1] = now.y;
        }
    };
    if (by_root) {
        moves([](float2 x) { return make_float2(near_sqrt(x.x), near_sqrt(x.y)); });
    } else {  // as x / sqrt(x + 1e-37): roots below 1e-15 are not right, and nothing next to eps; an infinite x would give NaN
        moves([](float2 x) {
            const float2 more = __fadd2_rn(x, twice(1e-37f));
            return __fmul2_rn(x, make_float2(fast_rsqrt(more.x), fast_rsqrt(more.y)));
        });
    }
    write_params<P16, COPY, BF16>(t, it, q, p);
    const uint32_t key = mix(mix((uint32_t)(base / ADAM_BLOCK) + warp) ^ (seed + it.number * 0x9E3779B9u)) + lane * (8u * 0x6A09E667u);
    uint32_t rm[8], rv[8];  // the lower and the upper half of mix()
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t y = mix_half(key + i * 0x6A09E667u);
        rv[i] = y >> 16;
        rm[i] = (y ^ rv[i]) & 0xffffu;
    }
    if (q.left < 8) {  // (beyond the tensor's end)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (2 * i >= q.left) m[i].x = v[i].x = 0.f;
            if (2 * i + 1 >= q.left) m[i].y = v[i].y = 0.f;
        }
    }
    uint2 codes;
    const uint32_t e1 = encode8<true>(m, rm, codes);
    write_codes(static_cast<uint8_t*>(it.m) + q.at, codes, q.whole, q.left);
    const uint32_t e2 = encode8<false>(v, rv, codes);
    write_codes(static_cast<uint8_t*>(it.v) + q.at, codes, q.whole, q.left);
    if (lane == 0) {
        *em = (uint8_t)e1;
        *ev = (uint8_t)e2;
    }
}

// What the 8-bit moments stand for, as bf16 values, which hold them exactly.
template <int CAP>
__global__ void __launch_bounds__(ADAM_THREADS) k_adamw_moments(const __grid_constant__ MomentTable<CAP> t)
{
    enter();
    const som_adamw_tensor& it = t.item[tensor_of(t, blockIdx.x)];
    const int64_t at = (int64_t)(blockIdx.x - it.first_chunk) * ADAM_CHUNK + threadIdx.x * 8;
    if (at >= it.n) return;
    const int left = it.n - at >= 8 ? 8 : (int)(it.n - at);
    const uintptr_t all = reinterpret_cast<uintptr_t>(it.param) | reinterpret_cast<uintptr_t>(it.copy) | reinterpret_cast<uintptr_t>(it.m) | reinterpret_cast<uintptr_t>(it.v);
    const bool whole = left == 8 && (all & 15u) == 0;
    const int64_t blocks = (it.n + ADAM_BLOCK - 1) / ADAM_BLOCK, block = at / ADAM_BLOCK;
    const uint2 mc = read_codes(static_cast<const uint8_t*>(it.m) + at, whole, left), vc = read_codes(static_cast<const uint8_t*>(it.v) + at, whole, left);
    const uint32_t em = it.exponents[block], ev = it.exponents[blocks + block];
    float2 m[4], v[4];
    decode8<true>(mc, em, m);
    decode8<false>(vc, ev, v);
    write8(static_cast<uint16_t*>(it.param) + at, reinterpret_cast<const float(&)[8]>(m), whole, left, 1);
    write8(static_cast<uint16_t*>(it.copy) + at, reinterpret_cast<const float(&)[8]>(v), whole, left, 1);
}

// Tensors a launch: what a kernel's parameters hold (32764 bytes), and fewer where there are few, since a launch copies them.  In us a call, small / large
// table: 5 tensors 10.8 / 14.7, 15 tensors 16.0 / 20.0, 24 tensors 20.9 / 24.6; on the device they are alike.  300 tensors of 100000 elements, bf16
// gradients, on the device: 119 us, with 8-bit moments 91 (floors 119 and 64); the call takes 165.
constexpr int FEW_TENSORS = 24, MOST_TENSORS = 500;
static_assert(sizeof(AdamTable<MOST_TENSORS>) <= 32764, "kernel parameters");

template <bool P16, bool G16, bool COPY, bool BF16, bool AT, int CAP>
cudaError_t launch_8(som_layers* l, const AdamTable<CAP>& t, unsigned chunks, cudaStream_t st)
{
    return launch(l, k_adamw8<P16, G16, COPY, BF16, CAP, AT>, dim3(chunks), ADAM_THREADS, 0, st, 1, t);
}

template <bool P16, bool G16, bool COPY, int BITS, int CAP>
cudaError_t launch_table(som_layers* l, const AdamTable<CAP>& t, unsigned chunks, cudaStream_t st)
{
    if (BITS == 32) return launch(l, k_adamw<P16, G16, COPY, CAP>, dim3(chunks), ADAM_THREADS, 0, st, 1, t);
    if (P16 && t.param_bf16) return t.h_at ? launch_8<P16, G16, COPY, P16, true>(l, t, chunks, st) : launch_8<P16, G16, COPY, P16, false>(l, t, chunks, st);
    return t.h_at ? launch_8<P16, G16, COPY, false, true>(l, t, chunks, st) : launch_8<P16, G16, COPY, false, false>(l, t, chunks, st);
}

template <bool P16, bool G16, bool COPY, int BITS>
cudaError_t launch_adamw(som_layers* l, const AdamTable<MOST_TENSORS>& t, unsigned chunks, cudaStream_t st)
{
    if (t.count > FEW_TENSORS) return launch_table<P16, G16, COPY, BITS>(l, t, chunks, st);
    AdamTable<FEW_TENSORS> s;
    for (int i = 0; i < t.count; ++i) s.item[i] = t.item[i];
    s.count = t.count;
    s.param_bf16 = t.param_bf16, s.grad_bf16 = t.grad_bf16, s.copy_bf16 = t.copy_bf16;
    s.h = t.h;
    s.pairs = t.pairs;
    s.h_at = t.h_at;
    s.scale = t.scale;
    return launch_table<P16, G16, COPY, BITS>(l, s, chunks, st);
}

template <int BITS>
cudaError_t launch_types(som_layers* l, const AdamTable<MOST_TENSORS>& t, bool p16, bool g16, bool copy, unsigned chunks, cudaStream_t st)
{
    if (p16) return g16 ? launch_adamw<true, true, false, BITS>(l, t, chunks, st) : launch_adamw<true, false, false, BITS>(l, t, chunks, st);
    if (copy) return g16 ? launch_adamw<false, true, true, BITS>(l, t, chunks, st) : launch_adamw<false, false, true, BITS>(l, t, chunks, st);
    return g16 ? launch_adamw<false, true, false, BITS>(l, t, chunks, st) : launch_adamw<false, false, false, BITS>(l, t, chunks, st);
}

constexpr int64_t MOST_CHUNKS = ((int64_t)1 << 31) - 1;

bool off_by(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// Hands the tensors out to launches: run(first, count, chunks) with their first_chunk written to `to`
template <class TABLE, class RUN>
int in_launches(const som_adamw_tensor* tensors, int32_t count, TABLE& t, RUN&& run)
{
    int32_t i = 0;
    while (i < count) {
        int64_t chunks = 0;
        t.count = 0;
        for (; i < count && t.count < MOST_TENSORS; ++i) {
            if (tensors[i].n == 0) continue;
            const int64_t more = (tensors[i].n + ADAM_CHUNK - 1) / ADAM_CHUNK;
            if (chunks + more > MOST_CHUNKS) break;
            som_adamw_tensor& to = t.item[t.count++];
            to = tensors[i];
            to.first_chunk = (uint32_t)chunks;
            chunks += more;
        }
        if (t.count) LAY_TRY(run((unsigned)chunks));
    }
    return SOM_OK;
}

int check_tensors(const som_adamw_tensor* t, int32_t count)
{
    if (count < 0 || (count > 0 && !t)) return SOM_ERR_INVALID_ARG;
    for (int32_t i = 0; i < count; ++i) {
        if (t[i].n < 0) return SOM_ERR_INVALID_ARG;
        if (t[i].n > (int64_t)1 << 40) return SOM_ERR_UNSUPPORTED;
    }
    return SOM_OK;
}

}  // namespace
}  // namespace lay

using namespace lay;

extern "C" {

int som_adamw(som_layers* l, int param_type, int grad_type, int copy_type, int bits, int32_t count, const som_adamw_tensor* tensors,
              const som_adamw_step* step, void* stream)
{
    if (!l || !step || param_type < SOM_F32 || param_type > SOM_BF16 || grad_type < SOM_F32 || grad_type > SOM_BF16 || copy_type > SOM_BF16)
        return SOM_ERR_INVALID_ARG;
    const bool copy = copy_type >= 0;
    if ((bits != 8 && bits != 32) || copy_type == SOM_F32 || (copy && param_type != SOM_F32)) return SOM_ERR_INVALID_ARG;
    if (half_type(param_type) && half_type(grad_type) && grad_type != param_type) return SOM_ERR_INVALID_ARG;
    const double b1 = step->beta1, b2 = step->beta2;
    if (!(b1 >= 0.0 && b1 < 1.0) || !(b2 >= 0.0 && b2 < 1.0) || !(step->eps >= 0.0) || !(step->decay >= 0.0) || (!step->step_at && step->step < 1))
        return SOM_ERR_INVALID_ARG;
    LAY_TRY(check_tensors(tensors, count));
    const int param_bytes = param_type == SOM_F32 ? 4 : 2, grad_bytes = grad_type == SOM_F32 ? 4 : 2;
    for (int32_t i = 0; i < count; ++i) {
        const som_adamw_tensor& t = tensors[i];
        if (t.n == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v || (copy && !t.copy) || (bits == 8 && !t.exponents)) return SOM_ERR_INVALID_ARG;
        if (off_by(t.param, param_bytes) || off_by(t.grad, grad_bytes) || off_by(copy ? t.copy : nullptr, 2) || off_by(t.m, bits / 8) || off_by(t.v, bits / 8))
            return SOM_ERR_UNSUPPORTED;
    }
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    AdamTable<MOST_TENSORS> t;
    t.param_bf16 = param_type == SOM_BF16, t.grad_bf16 = grad_type == SOM_BF16, t.copy_bf16 = copy_type == SOM_BF16;
    t.scale = step->scale;
    t.h_at = nullptr;
    if (step->rate_at || step->step_at) {
        LAY_TRY(ensure(l, sizeof(Hyper)));
        const HyperArgs a = {static_cast<Hyper*>(l->ws), step->rate, b1, b2, step->eps, step->decay, step->step, step->rate_at, step->step_at, step->seed};
        LAY_TRY(outcome(l, launch(l, k_adamw_hyper, dim3(1), 1, 0, st, 1, a)));
        t.h_at = a.to;
    }
    t.h = hyper_of(step->rate, b1, b2, step->eps, step->decay, step->step_at ? 1 : step->step, step->seed);
    t.pairs = pairs_of(t.h);
    return in_launches(tensors, count, t, [&](unsigned chunks) {
        for (int i = 0; i < t.count; ++i)
            if (!copy) t.item[i].copy = nullptr;
        return outcome(l, bits == 8 ? launch_types<8>(l, t, param_type != SOM_F32, grad_type != SOM_F32, copy, chunks, st)
                                    : launch_types<32>(l, t, param_type != SOM_F32, grad_type != SOM_F32, copy, chunks, st));
    });
}

int som_adamw_moments(som_layers* l, int32_t count, const som_adamw_tensor* tensors, void* const* m, void* const* v, void* stream)
{
    if (!l || (count > 0 && (!m || !v))) return SOM_ERR_INVALID_ARG;
    LAY_TRY(check_tensors(tensors, count));
    for (int32_t i = 0; i < count; ++i) {
        if (tensors[i].n == 0) continue;
        if (!tensors[i].m || !tensors[i].v || !tensors[i].exponents || !m[i] || !v[i]) return SOM_ERR_INVALID_ARG;
        if (off_by(m[i], 2) || off_by(v[i], 2)) return SOM_ERR_UNSUPPORTED;
    }
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    int32_t from = 0;
    // The small table alone (the outputs' addresses take the places of param and copy): 5 tensors 20.1 us a call, with the large one 24.0; 500 tensors of
    // 100000 elements take 88 us on the device, 54 in one launch, of a call of 1060.
    while (from < count) {
        som_adamw_tensor some[FEW_TENSORS];
        const int32_t n = count - from < FEW_TENSORS ? count - from : FEW_TENSORS;
        for (int32_t i = 0; i < n; ++i) {
            some[i] = tensors[from + i];
            some[i].param = m[from + i];
            some[i].copy = v[from + i];
        }
        MomentTable<MOST_TENSORS> t;
        LAY_TRY(in_launches(some, n, t, [&](unsigned chunks) {
            MomentTable<FEW_TENSORS> s;
            for (int i = 0; i < t.count; ++i) s.item[i] = t.item[i];
            s.count = t.count;
            return outcome(l, launch(l, k_adamw_moments<FEW_TENSORS>, dim3(chunks), ADAM_THREADS, 0, st, 1, s));
        }));
        from += n;
    }
    return SOM_OK;
}

}  // extern "C"
