// Host side of the dense operators declared in include/som.h: handle, argument checks, workspace, tensor maps, launches.
#include <new>

#include "layers_few.cuh"
#include "layers_finish.cuh"
#include "layers_fp4.cuh"
#include "layers_host.cuh"
#include "layers_product.cuh"
#include "layers_slots.cuh"

namespace lay {

int make_map(som_layers* l, CUtensorMap* map, const void* base, int bytes, int64_t cols, int64_t rows, int64_t batch, int64_t ld,
             int64_t batch_stride, int box_rows, int row_bytes)
{
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)batch};
    const cuuint64_t strides[2] = {(cuuint64_t)(ld * bytes), (cuuint64_t)(batch_stride * bytes)};
    const cuuint32_t box[3] = {(cuuint32_t)(row_bytes / bytes), (cuuint32_t)box_rows, 1u};
    const cuuint32_t step[3] = {1u, 1u, 1u};
    const CUresult r = reinterpret_cast<Encode>(l->encode)(
        map, bytes == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims,
        strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, row_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r == CUDA_SUCCESS) return SOM_OK;
    l->last_cuda_error = (int)cudaErrorInvalidValue;
    return SOM_ERR_CUDA;
}

namespace {

// 16-bit operands of the products: the left one K-major in boxes of 128 rows (LEFT_BOX where they are the experts'); the right
// one, and M/N-major ones, of 64
int map_left(som_layers* l, CUtensorMap* m, const void* p, int64_t cols, int64_t rows, int64_t ld, int box = 128)
{
    return make_map(l, m, p, 2, cols, rows, 1, ld, rows * ld, box);
}
int map_right(som_layers* l, ProdArgs* a, ProdMode mode, bool gated, const void* p, int64_t cols, int64_t rows, int64_t batch = 1)
{
    a->right_box = right_box(mode, a->shape, gated);
    return make_map(l, &a->b, p, 2, cols, rows, batch, cols, rows * cols, a->right_box);
}
int map_64(som_layers* l, CUtensorMap* m, const void* p, int64_t cols, int64_t rows, int64_t ld, int64_t batch = 1)
{
    return make_map(l, m, p, 2, cols, rows, batch, ld, rows * ld, 64);
}
int map_out(som_layers* l, CUtensorMap* m, void* p, int bytes, int64_t cols, int64_t rows, int64_t ld, int64_t batch = 1)
{
    return make_map(l, m, p, bytes, cols, rows, batch, ld, rows * ld, 32);
}

// The tiles of a product of `rows` x `cols` outputs (`batch` of them).  Pairs of blocks do twice a single block's work per
// byte that they load, but need tiles enough for every SM: narrow single tiles where every SM has one at most.  1024 rows, sums of
// 2048, narrow tiles / pairs: 1024 columns 13.6 / 16.2 us, 2048 (128 narrow tiles) 15.2 / 16.4, 2560 (160) 25.3 / 17.7.
void set_tiles(const som_layers* l, ProdArgs* a, int64_t rows, int64_t cols, bool gated, int64_t batch = 1)
{
    const int halves = gated ? 2 : 1;
    a->shape = tiles_of(rows, 128) * tiles_of(cols, 128 / halves) * batch > l->sm_count ? PAIR : NARROW;
    a->row_tiles = tiles_of(rows, shape_rows(a->shape));
    a->col_tiles = tiles_of(cols, shape_cols(a->shape) / halves);
    a->rows = (int)rows;
    a->cols = (int)cols;
    a->splits = 1;
}

// Blocks that share each tile's sum, for products whose tiles leave SMs idle: worth its second launch (about 3 us, with a
// step of 64 k at about 0.3 us) where it takes at least 14 steps off the longest sum.  In parts / in one: 32 x 4096 outputs, sums of
// 4096, 13.5 / 24.1 us; 64 x 8192, 4096, 19.3 / 24.9; 256 x 1024, 2048, 11.6 / 14.2; 128 x 1024, 1024 (not split) 11.8 / 9.3.
int splits_of(const som_layers* l, const ProdArgs& a, int64_t k)
{
    if (a.shape != NARROW) return 1;
    const int64_t tiles = (int64_t)a.row_tiles * a.col_tiles, steps = tiles_of(k, 64);
    int64_t s = l->sm_count / tiles;
    if (s > steps / 4) s = steps / 4;
    if (s > 16) s = 16;
    return s > 1 && steps - steps / s >= 14 ? (int)s : 1;
}

// Runs a product in a.splits parts of [rows][n] fp32 at `parts` and joins them by `f`.
int run_split(som_layers* l, ProdMode mode, ProdArgs a, FinishArgs f, unsigned char* parts, cudaStream_t st)
{
    const int rc = make_map(l, &a.o, parts, 4, f.n, f.rows, a.splits, f.n, f.rows * f.n, 32);
    if (rc != SOM_OK) return rc;
    a.out32 = 1;
    f.part = reinterpret_cast<const float*>(parts);
    f.splits = a.splits;
    f.bf16 = a.bf16;
    const int done = launch_product(l, mode, a, st);
    return done != SOM_OK ? done : launch_finish(l, f, st);
}

// Rows so few that the CUDA cores take them, a warp an output, and not the tensor cores' tiles.  One and two rows are bound by the
// weights' bytes, unless the rows are short and the outputs many; with more a warp's instructions count, a reduction over its
// lanes for each row and output among them, about as much as 1024 products.  In us, k_few / tiles, bf16, `*` where tiles are taken:
//   D -> outputs            1 row         2 rows        3 or 4          5 to 8
//   4096 -> 4096           9.8 / 14.5   11.6 / 14.4   17.1 / 14.6 *   30.2 / 14.6 *
//   4096 -> 8192 (gated)  14.1 / 22.5   18.0 / 22.6   25.6 / 22.7 *   47.2 / 22.2 *
//   4096 -> 32768         45.2 / 82.5   53.1 / 70.9   79.0 / 76.5 *    152 / 68.9 *
//   4096 -> 2048           9.5 / 14.0    9.5 / 14.2   11.0 / 14.2     18.4 / 12.7 *
//   2048 -> 4096           9.6 / 12.0    9.7 / 12.1    9.8 / 11.9     15.1 / 11.9 *
//   2048 -> 2048          12.2 / 18.4   11.0 / 11.9    9.6 / 11.9      9.9 / 12.0
//   4096 -> 1024           9.6 / 12.3    9.9 / 12.1    9.7 / 12.1     11.8 / 12.1
//   8192 -> 1024           9.6 / 12.8    9.6 / 12.9   12.8 / 12.9     36.7 / 12.8 *
//   1392 -> 3728 (gated)   9.9 / 12.5    9.7 / 12.3    9.9 / 12.3      9.9 / 12.3 *
//   1024 -> 16384         11.2 / 13.7   13.1 / 13.7   17.1 / 13.7 *   26.4 / 13.4 *
//   512 -> 16384           9.7 / 9.8    11.2 / 10.0   13.8 / 10.0 *   19.1 / 9.9 *
//   256 -> 32768          15.0 / 12.3   17.2 / 12.1 * 21.6 / 12.3 *   28.0 / 11.7 *
//   2048 -> 256, 512 -> 512: launches alone, 9.7 / 10 to 12 at 1 to 8 rows
bool few_rows(int64_t T, int64_t D, int64_t outputs)
{
    if (T > FEW_ROWS || T * D * 2 > FEW_SMEM / 2) return false;  // (the rows lie in shared memory)
    const int64_t rows = T <= 2 ? T : T <= 4 ? 4 : FEW_ROWS;
    return (T <= 2 && D >= 1024) || rows * outputs * (D + 1024) <= (int64_t)48 << 20;
}

}  // namespace
}  // namespace lay

using namespace lay;

extern "C" {

int som_layers_create(som_layers** out)
{
    if (!out) return SOM_ERR_INVALID_ARG;
    *out = nullptr;
    int dev = 0, major = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || major != 10)
        return SOM_ERR_NO_DEVICE;
    som_layers* l = new (std::nothrow) som_layers();
    if (!l) return SOM_ERR_INVALID_ARG;
    l->device = dev;
    l->sm_count = sms;
    cudaDriverEntryPointQueryResult found;
    cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &l->encode, cudaEnableDefault, &found);
    if (e == cudaSuccess && (found != cudaDriverEntryPointSuccess || !l->encode)) e = cudaErrorNotSupported;
    if (e == cudaSuccess) e = prepare_product(l);
    if (e == cudaSuccess) e = prepare_fp4_product(l);
    if (e == cudaSuccess) e = prepare_norm();
    if (e == cudaSuccess) e = prepare_fp4_few();
    if (e == cudaSuccess) e = prepare_few();
    if (e == cudaSuccess) e = prepare_plan();
    if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void**>(&l->flags), 256);
    if (e == cudaSuccess) e = cudaMemset(l->flags, 0, 256);
    if (e != cudaSuccess) {
        som_layers_destroy(l);
        (void)cudaGetLastError();
        return SOM_ERR_CUDA;
    }
    *out = l;
    return SOM_OK;
}

int som_layers_destroy(som_layers* l)
{
    if (!l) return SOM_OK;
    Guard g(l->device);
    cudaFree(l->flags);
    cudaFree(l->ws);
    delete l;
    return SOM_OK;
}

int som_layers_last_cuda_error(const som_layers* l) { return l ? l->last_cuda_error : 0; }
int64_t som_layers_launch_count(const som_layers* l) { return l ? l->launches : 0; }
int64_t som_layers_rounds(const som_layers* l, int product, int tiles)
{
    return l && product >= 0 && product < 6 && tiles >= 0 && tiles < 3 ? l->rounds[product][tiles] : -1;
}

int som_layers_device_flags(som_layers* l, void* stream)
{
    if (!l) return SOM_ERR_INVALID_ARG;
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    int flags = 0;
    SOM_CK(l, cudaMemcpyAsync(&flags, l->flags, sizeof(int), cudaMemcpyDeviceToHost, st));
    SOM_CK(l, cudaMemsetAsync(l->flags, 0, sizeof(int), st));
    SOM_CK(l, cudaStreamSynchronize(st));
    if (flags & LAY_FLAG_GAVE_UP) return SOM_ERR_CUDA;
    return flags & LAY_FLAG_BAD_EXPERT ? SOM_ERR_INVALID_ARG : SOM_OK;
}

int som_linear(som_layers* l, int type, int act, int gated, int64_t T, int64_t D, int64_t F, const void* x, int64_t ldx,
               const void* w, const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy, void* stream)
{
    LAY_TRY(check_common(l, type, act, T));
    LAY_TRY(check_sizes(D, F));
    LAY_TRY(check_weight(w));
    LAY_TRY(check_rows(x, ldx, D, T));
    LAY_TRY(check_rows(y, ldy, F, T));
    if (residual) LAY_TRY(check_rows(residual, ldr, F, T));
    if (!aligned16(bias) || T >= MOST_ROWS) return SOM_ERR_UNSUPPORTED;
    if (T == 0) return SOM_OK;
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int64_t rows = gated ? 2 * F : F;
    if (few_rows(T, D, rows)) {
        FewArgs f = {};
        f.x = static_cast<const uint16_t*>(x);
        f.ldx = ldx;
        f.w = static_cast<const uint16_t*>(w);
        f.bias = static_cast<const uint16_t*>(bias);
        f.residual = static_cast<const uint16_t*>(residual);
        f.ldr = ldr;
        f.y = static_cast<uint16_t*>(y);
        f.ldy = ldy;
        f.rows = (int)T;
        f.D = (int)D;
        f.F = (int)F;
        f.act = act;
        f.bf16 = type == SOM_BF16;
        f.flags = l->flags;
        return launch_few(l, f, 1, gated, st);
    }
    ProdArgs a = {};
    LAY_TRY(map_left(l, &a.a, x, D, T, ldx));
    a.bf16 = type == SOM_BF16;
    a.flags = l->flags;
    a.experts = 1;
    a.k1 = (int)D;
    set_tiles(l, &a, T, rows, false);
    a.splits = splits_of(l, a, D);
    if (a.splits > 1) {
        LAY_TRY(ensure(l, (size_t)a.splits * T * rows * sizeof(float)));
        LAY_TRY(map_right(l, &a, PROD_FWD, false, w, D, rows));
        FinishArgs f = {};
        f.rows = T;
        f.n = (int)rows;
        f.cols = (int)F;
        f.bias = static_cast<const uint16_t*>(bias);
        f.extra = static_cast<const uint16_t*>(residual);
        f.ld_extra = ldr;
        f.out = static_cast<uint16_t*>(y);
        f.ld = ldy;
        f.mode = FINISH_FWD;
        f.act = act;
        f.gated = gated;
        return run_split(l, PROD_FWD, a, f, static_cast<unsigned char*>(l->ws), st);
    }
    LAY_TRY(map_out(l, &a.o, y, 2, F, T, ldy));
    a.bias = static_cast<const uint16_t*>(bias);
    a.extra = static_cast<const uint16_t*>(residual);
    a.ld_extra = ldr;
    set_tiles(l, &a, T, F, gated);
    LAY_TRY(map_right(l, &a, PROD_FWD, gated, w, D, rows));
    a.gate_rows = gated ? (int)F : 0;
    a.act = act;
    return launch_product(l, PROD_FWD, a, st);
}

int som_linear_backward(som_layers* l, int type, int act, int gated, int64_t T, int64_t D, int64_t F, const void* x,
                        int64_t ldx, const void* w, const void* bias, const void* dy, int64_t lddy, void* dx, void* dw,
                        void* dbias, void* stream)
{
    LAY_TRY(check_common(l, type, act, T));
    LAY_TRY(check_sizes(D, F));
    LAY_TRY(check_weight(w));
    LAY_TRY(check_rows(x, ldx, D, T));
    LAY_TRY(check_rows(dy, lddy, F, T));
    if (!aligned16(bias) || !aligned16(dx) || !aligned16(dw) || T >= MOST_ROWS) return SOM_ERR_UNSUPPORTED;
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int64_t rows = gated ? 2 * F : F;
    if (T == 0) {
        if (dw) SOM_CK(l, cudaMemsetAsync(dw, 0, (size_t)rows * D * 2, st));
        if (dbias) SOM_CK(l, cudaMemsetAsync(dbias, 0, (size_t)rows * 2, st));
        return SOM_OK;
    }
    const bool again = act != SOM_ACT_NONE || gated;  // dz is not dy itself
    const void* dz = dy;
    int64_t lddz = lddy;
    ProdArgs a = {};
    a.experts = 1;
    a.act = act;
    a.bf16 = type == SOM_BF16;
    a.flags = l->flags;
    // the three products and the blocks that share their tiles' sums
    ProdArgs z = a, px = a, pw = a;
    z.k1 = (int)D;
    set_tiles(l, &z, T, rows, false);
    z.splits = splits_of(l, z, D);
    px.k1 = (int)rows;
    set_tiles(l, &px, T, D, false);
    px.splits = splits_of(l, px, rows);
    pw.k1 = (int)T;
    set_tiles(l, &pw, rows, D, false);
    pw.splits = splits_of(l, pw, T);
    uint16_t* z_grad;
    float* sums;
    unsigned char* parts;
    Carver c{nullptr, 0};
    for (int pass = 0; pass < 2; ++pass) {
        c.used = 0;
        z_grad = c.take<uint16_t>(again ? T * rows : 0);
        sums = c.take<float>(again && dbias && z.splits == 1 ? tiles_of(T, 32) * rows : 0);
        int64_t most = again && z.splits > 1 ? (int64_t)z.splits * T * rows : 0;
        if (dx && px.splits > 1 && (int64_t)px.splits * T * D > most) most = (int64_t)px.splits * T * D;
        if (dw && pw.splits > 1 && (int64_t)pw.splits * rows * D > most) most = (int64_t)pw.splits * rows * D;
        parts = reinterpret_cast<unsigned char*>(c.take<float>(most));
        if (pass == 0) {
            LAY_TRY(ensure(l, c.used));
            c.base = static_cast<unsigned char*>(l->ws);
        }
    }
    FinishArgs f = {};
    if (again) {
        dz = z_grad;
        lddz = rows;
        LAY_TRY(map_left(l, &z.a, x, D, T, ldx));
        if (z.splits > 1) {
            LAY_TRY(map_right(l, &z, PROD_FWD, false, w, D, rows));
            f.rows = T;
            f.n = (int)rows;
            f.cols = (int)F;
            f.bias = static_cast<const uint16_t*>(bias);
            f.extra = static_cast<const uint16_t*>(dy);
            f.ld_extra = lddy;
            f.out = z_grad;
            f.ld = rows;
            f.mode = FINISH_DZ;
            f.act = act;
            f.gated = gated;
            z.act = SOM_ACT_NONE;
            LAY_TRY(run_split(l, PROD_FWD, z, f, parts, st));
        } else {
            z.o0 = z_grad;
            z.ld0 = rows;
            z.bias = static_cast<const uint16_t*>(bias);
            z.extra = static_cast<const uint16_t*>(dy);
            z.ld_extra = lddy;
            z.column_sums = dbias ? sums : nullptr;
            set_tiles(l, &z, T, F, gated);
            LAY_TRY(map_right(l, &z, PROD_DZ, gated, w, D, rows));
            z.gate_rows = gated ? (int)F : 0;
            LAY_TRY(launch_product(l, PROD_DZ, z, st));
        }
    }
    if (dbias) {
        EndArgs s = {};
        s.rows = T;
        s.E = 1;
        s.bf16 = a.bf16;
        if (again && z.splits == 1) {
            s.sums = sums;
            s.sums_cols = (int)rows;
            s.sums_out = static_cast<uint16_t*>(dbias);
        } else {
            s.v = static_cast<const uint16_t*>(dz);
            s.ldv = lddz;
            s.v_cols = (int)rows;
            s.v_sums = static_cast<uint16_t*>(dbias);
        }
        LAY_TRY(launch_ends(l, s, st));
    }
    f = FinishArgs();
    f.mode = FINISH_SUM;
    px.act = pw.act = SOM_ACT_NONE;
    if (dx) {
        LAY_TRY(map_left(l, &px.a, dz, rows, T, lddz));
        LAY_TRY(map_64(l, &px.b, w, D, rows, D));
        if (px.splits > 1) {
            f.rows = T;
            f.n = f.cols = (int)D;
            f.out = static_cast<uint16_t*>(dx);
            f.ld = D;
            LAY_TRY(run_split(l, PROD_DX, px, f, parts, st));
        } else {
            LAY_TRY(map_out(l, &px.o, dx, 2, D, T, D));
            LAY_TRY(launch_product(l, PROD_DX, px, st));
        }
    }
    if (dw) {
        LAY_TRY(map_64(l, &pw.a, dz, rows, T, lddz));
        LAY_TRY(map_64(l, &pw.b, x, D, T, ldx));
        if (pw.splits > 1) {
            f.rows = rows;
            f.n = f.cols = (int)D;
            f.out = static_cast<uint16_t*>(dw);
            f.ld = D;
            LAY_TRY(run_split(l, PROD_DW, pw, f, parts, st));
        } else {
            LAY_TRY(map_out(l, &pw.o, dw, 2, D, rows, D));
            LAY_TRY(launch_product(l, PROD_DW, pw, st));
        }
    }
    return SOM_OK;
}

static int check_route(const som_layers* l, int type, int score, int64_t T, int32_t E, int32_t k, const void* logits, int64_t ld)
{
    if (!l || type < SOM_F32 || type > SOM_BF16 || (score != SOM_SCORE_SOFTMAX && score != SOM_SCORE_SIGMOID) || T < 0 || E < 1 ||
        k < 1 || k > E || (T > 0 && (!logits || ld < E)))
        return SOM_ERR_INVALID_ARG;
    return E > 1024 || k > 32 || T >= MOST_ROWS ? SOM_ERR_UNSUPPORTED : SOM_OK;
}

int som_route(som_layers* l, int type, int score, int64_t T, int32_t E, int32_t k, const void* logits, int64_t ld,
              const float* bias, int32_t groups, int32_t top_groups, int32_t group_best, int renorm, float scale,
              float* weights, int32_t* indices, int32_t* counts, void* stream)
{
    LAY_TRY(check_route(l, type, score, T, E, k, logits, ld));
    if (groups < 1 || E % groups != 0 || top_groups < 1 || top_groups > groups || (group_best != 1 && group_best != 2) ||
        (T > 0 && (!weights || !indices)))
        return SOM_ERR_INVALID_ARG;
    if (groups > 32) return SOM_ERR_UNSUPPORTED;
    Guard g(l->device);
    return launch_route(l, type, score, T, E, k, logits, ld, bias, groups, top_groups, group_best, renorm, scale, weights, indices,
                        counts, reinterpret_cast<cudaStream_t>(stream));
}

int som_route_backward(som_layers* l, int type, int score, int64_t T, int32_t E, int32_t k, const void* logits, int64_t ld,
                       const int32_t* indices, const float* dweights, int renorm, float scale, void* dlogits, void* stream)
{
    LAY_TRY(check_route(l, type, score, T, E, k, logits, ld));
    if (T > 0 && (!indices || !dweights || !dlogits)) return SOM_ERR_INVALID_ARG;
    Guard g(l->device);
    return launch_route_backward(l, type, score, T, E, k, logits, ld, indices, dweights, renorm, scale, dlogits,
                                 reinterpret_cast<cudaStream_t>(stream));
}

static int check_experts(const som_layers* l, int type, int act, int64_t T, int32_t E, int32_t k, int64_t D, int64_t I,
                         const void* x, int64_t ldx, const int32_t* indices, const void* weights, int weights_type,
                         const void* w1, const void* b1, const void* w2, const void* b2)
{
    LAY_TRY(check_common(l, type, act, T));
    if (E < 1 || k < 1 || (weights_type != SOM_F32 && weights_type != type) || (T > 0 && (!indices || !weights)))
        return SOM_ERR_INVALID_ARG;
    LAY_TRY(check_sizes(D, I));
    LAY_TRY(check_weight(w1));
    LAY_TRY(check_weight(w2));
    LAY_TRY(check_rows(x, ldx, D, T));
    if (!aligned16(b1) || !aligned16(b2) || E > 1024 || k > 32 || T * k >= MOST_ROWS - (int64_t)E * 128) return SOM_ERR_UNSUPPORTED;
    return SOM_OK;
}

// the plan's arrays for row tiles of `tile` rows
static SlotPlan carve_plan(Carver& c, int64_t T, int E, int k, int tile)
{
    SlotPlan p = {};
    const int64_t slots = T * k, used = slots < E ? slots : E;  // experts that can have a slot
    p.tile = tile;
    p.max_rows = (int)((slots + used * (tile - 1)) / tile * tile);
    p.seg = c.take<int>(E + 1);
    p.count = c.take<int>(E);
    p.tiles = c.take<int>(1);
    p.tile_expert = c.take<int>(p.max_rows / tile);
    p.pos = c.take<int>(slots);
    p.row_weight = c.take<float>(p.max_rows);
    p.block_counts = c.take<int>((int64_t)plan_blocks(slots) * E);
    return p;
}

// So few slots that most experts in use have one: each slot reads its expert's weights by itself (a weight that two slots
// read comes from L2 the second time).  In us, each slot by itself / slots ordered by expert, at D 2048, I 1024 unless said:
// 32 slots of 128 experts (1024, 512) 25 / 40; 64 slots of 64 experts 128 / 124; 96 of 64 189 / 138; 16 slots of 8 experts 35 / 39;
// 32 of 8 61 / 40; 16 of 8 (1024, 512) 19 / 27; 48 of 8 28 / 28.
static bool few_slots(int64_t T, int E, int k) { return T * k <= 16 || (T * k <= 64 && T * k <= E); }

// Rows of an expert's tiles: a pair's once the experts have rows enough; with fewer, a pair would mostly multiply padding, and
// the weights' bytes bound the product, not the tensor cores.  Where the two meet depends on how the experts' rows fall into tiles, so
// no one number is right everywhere: 256 is within 15 % of the better shape in all of these.  In us, single blocks / pairs, D 2048
// and I 1024, gated, unless said:
//   rows an expert                  64           128          192          256          384          512
//   64 experts                   181 / 202    219 / 219    268 / 278    315 / 337    438 / 448    552 / 540
//   16 experts                    68 / 80      90 / 84      94 / 105    113 / 102    139 / 127    143 / 146
//   8 experts (1024, 2048)        49 / 55      58 / 58      60 / 66      78 / 68      83 / 71      86 / 89
//   12 experts (1000, 712)        44 / 43      48 / 55      66 / 58      70 / 67      84 / 74      91 / 75
//   64 experts, gradient         496 / 557    602 / 641    737 / 792    869 / 911   1079 / 1068  1432 / 1362
//   32 experts (1024, 512), grad. 90 / 103    116 / 111    128 / 141    158 / 151    178 / 186    228 / 242
//   16 experts, gradient         138 / 155    175 / 162    189 / 214    243 / 225    273 / 313    355 / 386
//   12 experts (1000, 712), grad. 73 / 68      84 / 86      90 / 94     113 / 99     130 / 131    163 / 145
static int tile_rows(int64_t T, int E, int k) { return T * k >= (int64_t)256 * E ? shape_rows(PAIR) : shape_rows(WIDE); }

// A product over the slots' rows.  Single blocks are wide where that leaves a tile for every SM, by the tiles to expect.
static ProdArgs grouped(const som_layers* l, const SlotPlan& p, int64_t slots, int E, int type, int64_t cols, bool gated)
{
    ProdArgs a = {};
    a.tiles = p.tiles;
    a.tile_expert = p.tile_expert;
    a.seg = p.seg;
    a.count = p.count;
    a.row_weight = p.row_weight;
    const int64_t expected = (slots < E ? slots : E) + slots / 256;
    const int halves = gated ? 2 : 1;
    // Wide tiles once they are two thirds of the SMs.  Gated, D 2048 and I 1024 unless said, wide / narrow: 8 experts with 8 or 16 rows
    // (64 wide tiles) 45 / 39 us, 12 with 33 (1000, 712; 78) 38 / 33, 16 with 8 (128) 54.8 / 57.8, 32 with 4 (256) 82.4 / 83.6, 64 with 9
    // (512) 159.4 / 164
    a.shape = p.tile == shape_rows(PAIR) ? PAIR : 3 * expected * tiles_of(cols, shape_cols(WIDE) / halves) >= 2 * l->sm_count ? WIDE : NARROW;
    a.row_tiles = p.max_rows / p.tile;
    a.col_tiles = tiles_of(cols, shape_cols(a.shape) / halves);
    a.rows = p.max_rows;
    a.cols = (int)cols;
    a.splits = 1;
    a.columns_first = 1;  // (all its products follow the gather or a later kernel)
    a.bf16 = type == SOM_BF16;
    a.flags = l->flags;
    return a;
}

int som_experts(som_layers* l, int type, int act, int gated, int64_t T, int32_t E, int32_t k, int64_t D, int64_t I,
                const void* x, int64_t ldx, const int32_t* indices, const void* weights, int weights_type, const void* w1,
                const void* b1, const void* w2, const void* b2, const void* residual, int64_t ldr, void* y, int64_t ldy,
                void* stream)
{
    LAY_TRY(check_experts(l, type, act, T, E, k, D, I, x, ldx, indices, weights, weights_type, w1, b1, w2, b2));
    LAY_TRY(check_rows(y, ldy, D, T));
    if (residual) LAY_TRY(check_rows(residual, ldr, D, T));
    if (T == 0) return SOM_OK;
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int64_t rows1 = gated ? 2 * I : I;
    if (few_slots(T, E, k) && D * 2 <= FEW_SMEM && k * I * 4 <= FEW_SMEM) {
        LAY_TRY(ensure(l, (size_t)(T * k * I) * sizeof(float)));
        FewArgs f = {};
        f.x = static_cast<const uint16_t*>(x);
        f.ldx = ldx;
        f.w = static_cast<const uint16_t*>(w1);
        f.bias = static_cast<const uint16_t*>(b1);
        f.hidden = static_cast<float*>(l->ws);
        f.indices = indices;
        f.weights = weights;
        f.weights_type = weights_type;
        f.k = k;
        f.E = E;
        f.rows = 1;
        f.D = (int)D;
        f.F = (int)I;
        f.act = act;
        f.bf16 = type == SOM_BF16;
        f.flags = l->flags;
        LAY_TRY(launch_few(l, f, (int)(T * k), gated, st));
        FewDownArgs d = {};
        d.hidden = f.hidden;
        d.indices = indices;
        d.weights = weights;
        d.w2 = static_cast<const uint16_t*>(w2);
        d.b2 = static_cast<const uint16_t*>(b2);
        d.residual = static_cast<const uint16_t*>(residual);
        d.y = static_cast<uint16_t*>(y);
        d.ldr = ldr;
        d.ldy = ldy;
        d.weights_type = weights_type;
        d.k = k;
        d.E = E;
        d.D = (int)D;
        d.I = (int)I;
        d.bf16 = f.bf16;
        return launch_few_down(l, d, T, st);
    }
    SlotPlan p;
    uint16_t *xp, *h;
    float* part;
    Carver c{nullptr, 0};
    for (int pass = 0; pass < 2; ++pass) {
        c.used = 0;
        p = carve_plan(c, T, E, k, tile_rows(T, E, k));
        xp = c.take<uint16_t>((int64_t)p.max_rows * D);
        h = c.take<uint16_t>((int64_t)p.max_rows * I);
        part = c.take<float>((int64_t)p.max_rows * D);
        if (pass == 0) {
            LAY_TRY(ensure(l, c.used));
            c.base = static_cast<unsigned char*>(l->ws);
        }
    }
    LAY_TRY(launch_plan(l, p, indices, weights, weights_type, T, k, E, st));
    LAY_TRY(launch_gather(l, p, T * k, E, k, D, x, ldx, xp, nullptr, 0, nullptr, st));
    ProdArgs a = grouped(l, p, T * k, E, type, I, gated);
    LAY_TRY(map_left(l, &a.a, xp, D, p.max_rows, D, LEFT_BOX));
    LAY_TRY(map_right(l, &a, PROD_FWD, gated, w1, D, rows1, E));
    LAY_TRY(map_out(l, &a.o, h, 2, I, p.max_rows, I));
    a.bias = static_cast<const uint16_t*>(b1);
    a.bias_ld = (int)rows1;
    a.gate_rows = gated ? (int)I : 0;
    a.k1 = (int)D;
    a.act = act;
    a.weigh = 1;
    LAY_TRY(launch_product(l, PROD_FWD, a, st));
    a = grouped(l, p, T * k, E, type, D, false);
    LAY_TRY(map_left(l, &a.a, h, I, p.max_rows, I, LEFT_BOX));
    LAY_TRY(map_right(l, &a, PROD_FWD, false, w2, I, D, E));
    LAY_TRY(map_out(l, &a.o, part, 4, D, p.max_rows, D));
    a.bias = static_cast<const uint16_t*>(b2);
    a.bias_ld = (int)D;
    a.k1 = (int)I;
    a.weigh = 2;
    a.out32 = 1;
    LAY_TRY(launch_product(l, PROD_FWD, a, st));
    EndArgs s = {};
    s.p = p;
    s.T = T;
    s.k = k;
    s.D = (int)D;
    s.bf16 = a.bf16;
    s.part = part;
    s.residual = static_cast<const uint16_t*>(residual);
    s.ldr = ldr;
    s.y = static_cast<uint16_t*>(y);
    s.ldy = ldy;
    return launch_ends(l, s, st);
}

int som_experts_backward(som_layers* l, int type, int act, int gated, int64_t T, int32_t E, int32_t k, int64_t D, int64_t I,
                         const void* x, int64_t ldx, const int32_t* indices, const void* weights, int weights_type,
                         const void* w1, const void* b1, const void* w2, const void* b2, const void* dy, int64_t lddy,
                         void* dx, void* dweights, void* dw1, void* db1, void* dw2, void* db2, void* stream)
{
    LAY_TRY(check_experts(l, type, act, T, E, k, D, I, x, ldx, indices, weights, weights_type, w1, b1, w2, b2));
    LAY_TRY(check_rows(dy, lddy, D, T));
    if (!dw1 || !dw2 || (T > 0 && (!dx || !dweights))) return SOM_ERR_INVALID_ARG;
    if (!aligned16(dx) || !aligned16(dw1) || !aligned16(dw2)) return SOM_ERR_UNSUPPORTED;
    Guard g(l->device);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int64_t rows1 = gated ? 2 * I : I;
    if (T == 0) {
        SOM_CK(l, cudaMemsetAsync(dw1, 0, (size_t)E * rows1 * D * 2, st));
        SOM_CK(l, cudaMemsetAsync(dw2, 0, (size_t)E * D * I * 2, st));
        if (db1) SOM_CK(l, cudaMemsetAsync(db1, 0, (size_t)E * rows1 * 2, st));
        if (db2) SOM_CK(l, cudaMemsetAsync(db2, 0, (size_t)E * D * 2, st));
        return SOM_OK;
    }
    SlotPlan p;
    uint16_t *xp, *dyp, *h, *dz;
    float *part, *dot, *sums;
    ProdArgs z;  // z and g = W2^T dy side by side, in tiles of half the width
    Carver c{nullptr, 0};
    for (int pass = 0; pass < 2; ++pass) {
        c.used = 0;
        p = carve_plan(c, T, E, k, tile_rows(T, E, k));
        z = grouped(l, p, T * k, E, type, I, true);
        z.dots = z.col_tiles * tile_dots(z.shape);
        xp = c.take<uint16_t>((int64_t)p.max_rows * D);
        dyp = c.take<uint16_t>((int64_t)p.max_rows * D);
        h = c.take<uint16_t>((int64_t)p.max_rows * I);
        dz = c.take<uint16_t>((int64_t)p.max_rows * rows1);
        part = c.take<float>((int64_t)p.max_rows * D);
        dot = c.take<float>((int64_t)p.max_rows * z.dots);
        sums = c.take<float>(db1 ? p.max_rows / 32 * rows1 : 0);
        if (pass == 0) {
            LAY_TRY(ensure(l, c.used));
            c.base = static_cast<unsigned char*>(l->ws);
        }
    }
    LAY_TRY(launch_plan(l, p, indices, weights, weights_type, T, k, E, st));
    LAY_TRY(launch_gather(l, p, T * k, E, k, D, x, ldx, xp, dy, lddy, dyp, st));
    // -> dz, the weighted h, partial sums of <h, g>
    ProdArgs a = z;
    LAY_TRY(map_left(l, &a.a, xp, D, p.max_rows, D, LEFT_BOX));
    LAY_TRY(map_right(l, &a, PROD_DZ_TWO, gated, w1, D, rows1, E));
    LAY_TRY(map_left(l, &a.a2, dyp, D, p.max_rows, D, LEFT_BOX));
    LAY_TRY(map_64(l, &a.b2, w2, I, D, I, E));
    a.o0 = dz;
    a.ld0 = rows1;
    a.o2 = h;
    a.ld2 = I;
    a.bias = static_cast<const uint16_t*>(b1);
    a.bias_ld = (int)rows1;
    a.dot = dot;
    a.column_sums = db1 ? sums : nullptr;
    a.gate_rows = gated ? (int)I : 0;
    a.k1 = a.k2 = (int)D;
    a.act = act;
    LAY_TRY(launch_product(l, PROD_DZ_TWO, a, st));
    // dx; with its join all other sums
    a = grouped(l, p, T * k, E, type, D, false);
    LAY_TRY(map_left(l, &a.a, dz, rows1, p.max_rows, rows1, LEFT_BOX));
    LAY_TRY(map_64(l, &a.b, w1, D, rows1, D, E));
    LAY_TRY(map_out(l, &a.o, part, 4, D, p.max_rows, D));
    a.k1 = (int)rows1;
    a.out32 = 1;
    LAY_TRY(launch_product(l, PROD_DX, a, st));
    EndArgs s = {};
    s.p = p;
    s.T = T;
    s.k = k;
    s.D = (int)D;
    s.E = E;
    s.bf16 = a.bf16;
    s.part = part;
    s.y = static_cast<uint16_t*>(dx);
    s.ldy = D;
    s.dot = dot;
    s.dots = z.dots;
    s.indices = indices;
    s.b2 = static_cast<const uint16_t*>(b2);
    s.dy = static_cast<const uint16_t*>(dy);
    s.lddy = lddy;
    s.dweights = dweights;
    s.weights_type = weights_type;
    s.sums = sums;
    s.sums_cols = (int)rows1;
    s.sums_out = static_cast<uint16_t*>(db1);
    s.v = dyp;
    s.ldv = D;
    s.v_cols = (int)D;
    s.v_sums = static_cast<uint16_t*>(db2);
    LAY_TRY(launch_ends(l, s, st));
    // dw1 = dz^T x and dw2 = dy^T (weighted h), in one launch
    a = ProdArgs();
    a.seg = p.seg;
    a.count = p.count;
    a.experts = E;
    a.columns_first = 1;
    a.bf16 = type == SOM_BF16;
    a.flags = l->flags;
    LAY_TRY(map_64(l, &a.a, dz, rows1, p.max_rows, rows1));
    LAY_TRY(map_64(l, &a.b, xp, D, p.max_rows, D));
    LAY_TRY(map_out(l, &a.o, dw1, 2, D, rows1, D, E));
    set_tiles(l, &a, rows1, D, false, E);
    LAY_TRY(map_64(l, &a.a2, dyp, D, p.max_rows, D));
    LAY_TRY(map_64(l, &a.b2, h, I, p.max_rows, I));
    LAY_TRY(map_out(l, &a.o2map, dw2, 2, I, D, I, E));
    a.rows2 = (int)D;
    a.cols2 = (int)I;
    a.row_tiles2 = tiles_of(D, shape_rows(a.shape));
    a.col_tiles2 = tiles_of(I, shape_cols(a.shape));
    return launch_product(l, PROD_DW, a, st);
}

}  // extern "C"
