// Host-side pieces that the C entries of the dense operators share: device guard, workspace, checks of arguments.
#pragma once

#include "layers_internal.cuh"

namespace lay {

struct Guard {  // the handle's device for the length of a call
    int prev;
    bool switched;
    explicit Guard(int dev) : prev(-1), switched(false)
    {
        if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) switched = cudaSetDevice(dev) == cudaSuccess;
    }
    ~Guard()
    {
        if (switched) cudaSetDevice(prev);
    }
};

// Hands out pieces of the workspace; run once without a base to learn the size.
struct Carver {
    unsigned char* base;
    size_t used;
    template <class T>
    T* take(int64_t n)
    {
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += som_align_up((size_t)n * sizeof(T), 1024);
        return p;
    }
};

inline int ensure(som_layers* l, size_t need)
{
    if (need <= l->ws_bytes) return SOM_OK;
    if (l->ws) {
        SOM_CK(l, cudaFree(l->ws));  // synchronises: earlier work in it is done
        l->ws = nullptr;
        l->ws_bytes = 0;
    }
    need = som_align_up(need + need / 8, 1 << 20);
    SOM_CK(l, cudaMalloc(&l->ws, need));
    l->ws_bytes = need;
    return SOM_OK;
}

#define LAY_TRY(call)                   \
    do {                                \
        const int rc__ = (call);        \
        if (rc__ != SOM_OK) return rc__; \
    } while (0)

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool half_type(int type) { return type == SOM_F16 || type == SOM_BF16; }
constexpr int64_t MOST_ROWS = (int64_t)1 << 30, MOST_COLS = (int64_t)1 << 24;

inline int check_common(const som_layers* l, int type, int act, int64_t T)
{
    if (!l || T < 0 || act < SOM_ACT_NONE || act > SOM_ACT_SILU || !half_type(type)) return SOM_ERR_INVALID_ARG;
    return SOM_OK;
}

// a [T][cols] 16-bit operand of a product: present, long enough rows, and laid out as the copies need it
inline int check_rows(const void* p, int64_t ld, int64_t cols, int64_t T)
{
    if (T == 0) return SOM_OK;
    if (!p || ld < cols) return SOM_ERR_INVALID_ARG;
    if (!aligned16(p) || ld % 8 != 0 || ld >= (int64_t)1 << 32) return SOM_ERR_UNSUPPORTED;
    return SOM_OK;
}

inline int check_weight(const void* p)
{
    if (!p) return SOM_ERR_INVALID_ARG;
    return aligned16(p) ? SOM_OK : SOM_ERR_UNSUPPORTED;
}

inline int check_sizes(int64_t a, int64_t b)
{
    if (a <= 0 || b <= 0) return SOM_ERR_INVALID_ARG;
    if (a % 8 != 0 || b % 8 != 0 || a > MOST_COLS || b > MOST_COLS) return SOM_ERR_UNSUPPORTED;
    return SOM_OK;
}

inline int64_t tiles_of(int64_t n, int64_t width) { return (n + width - 1) / width; }

}  // namespace lay
