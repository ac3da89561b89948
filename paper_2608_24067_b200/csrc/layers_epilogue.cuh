// What the products' epilogues share: ways out to memory, and rows fetched ahead.
#pragma once

#include "layers_math.cuh"
#include "layers_ptx.cuh"

namespace lay {

// Ways out of the epilogue.  Staged: 32 rows (lane l holds row l) of 64 16-bit or 32 fp32 columns go through shared memory
// (128-byte rows, 128-byte swizzle) to a TMA store, which leaves out what lies outside the tensor.  Direct: a lane writes 8
// columns at a time.  Direct stores take the load/store pipe 32 cycles an instruction: too much where a tile's products are short
// (PROD_DW at 512 rows an expert: 134 us staged, 178 us direct), but no waits, and no shared memory for up to three outputs
// at once (PROD_DZ, PROD_DZ_TWO).
// ROW_BYTES 64: half as many columns, 64-byte rows under the 64-byte swizzle.
template <int BUFFERS, int ROW_BYTES = 128>
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
    __device__ __forceinline__ void put(int chunk, uint4 v)
    {
        *reinterpret_cast<uint4*>(buf + lane * ROW_BYTES + ((chunk ^ (ROW_BYTES == 128 ? lane & 7 : (lane >> 1) & 3)) << 4)) = v;
    }
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

}  // namespace lay
