// Microscaled formats: a matrix to codes and scales, and back.  A block of 32 values shares the power of two
// 2^E with E = floor(log2(max |x|)) - emax; a code is x * 2^-E rounded to the format.  Both directions are
// streams bound by HBM: four neighbouring lanes hold a block, eight values each, so that a lane's load is 16 or 32
// bytes, its codes are one store of 4 or 8, and the block's maximum takes two exchanges inside a quad.
#include "pv_ops.h"

namespace {

constexpr int kBlock = 256;

// One wave per stretch of 64 * 8 values of a row: the row and the stretch come from scalar arithmetic, and a lane
// only has to look whether its eight values lie inside the row.  Lanes behind the row's last block do nothing; those
// inside it and behind `cols` write zero codes.
struct span {
    int64_t row;
    int unit;        // of eight values, in the row
    int valid;       // values of them inside the row; may be below 0
    bool live;       // the unit belongs to one of the row's blocks
};

__device__ __forceinline__ span wave_span(int64_t rows, int cols, int nblk, int waves_a_row)
{
    const int64_t w = (int64_t)blockIdx.x * (kBlock / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    span s;
    s.row = w / waves_a_row;
    s.unit = (int)(w - s.row * waves_a_row) * 64 + (threadIdx.x & 63);
    s.valid = cols - s.unit * 8;
    s.live = s.row < rows && s.unit < nblk * 4;
    return s;
}

template <int FMT, class T>
__global__ __launch_bounds__(kBlock) void k_quantize_mx(const T *__restrict__ X, uint8_t *__restrict__ codes,
                                                        uint8_t *__restrict__ scales, int64_t rows, int64_t cols,
                                                        int nblk, int waves_a_row)
{
    const span s = wave_span(rows, (int)cols, nblk, waves_a_row);
    if (!s.live) return;
    float v[8];
    pv_load8(X + s.row * cols + (int64_t)s.unit * 8, s.valid, v);
    const unsigned scale = pv_mx_scale<FMT>(pv_mx_largest(v));
    const pv_u2 c = pv_mx_encode<FMT>(v, scale);
    const int64_t u = s.row * nblk * 4 + s.unit;
    if constexpr (FMT == PV_MX_E2M1) reinterpret_cast<unsigned *>(codes)[u] = c.x;
    else reinterpret_cast<pv_u2 *>(codes)[u] = c;
    if ((s.unit & 3) == 0) scales[u >> 2] = (uint8_t)scale;
}

template <int FMT, class T>
__global__ __launch_bounds__(kBlock) void k_dequantize_mx(const uint8_t *__restrict__ codes,
                                                          const uint8_t *__restrict__ scales, T *__restrict__ out,
                                                          int64_t rows, int64_t cols, int nblk, int waves_a_row)
{
    const span s = wave_span(rows, (int)cols, nblk, waves_a_row);
    if (!s.live) return;
    const int64_t u = s.row * nblk * 4 + s.unit;
    pv_u2 c = {0u, 0u};
    if constexpr (FMT == PV_MX_E2M1) c.x = reinterpret_cast<const unsigned *>(codes)[u];
    else c = reinterpret_cast<const pv_u2 *>(codes)[u];
    float v[8];
    pv_mx_decode<FMT>(c, pv_mx_power(scales[u >> 2]), v);
    pv_store8<true>(out + s.row * cols + (int64_t)s.unit * 8, s.valid, v);
}

__global__ __launch_bounds__(kBlock) void k_zero(uint16_t *p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlock) p[i] = 0;
}

struct plan {
    int nblk, waves_a_row;
    unsigned blocks;
};

pv_status make_plan(pv_ctx *ctx, int64_t rows, int64_t cols, plan *p)
{
    p->nblk = (int)pv_mx_blocks(cols);
    p->waves_a_row = (p->nblk * 4 + 63) / 64;
    const int64_t blocks = (rows * p->waves_a_row + kBlock / 64 - 1) / (kBlock / 64);
    if (blocks >= (int64_t)1 << 31) return pv_fail(ctx, PV_ERR_UNSUPPORTED, "%lld rows are too many", (long long)rows);
    p->blocks = (unsigned)blocks;
    return PV_OK;
}

}  // namespace

pv_status pv_launch_quantize_mx(pv_ctx *ctx, int64_t rows, int64_t cols, int format, int x_type, const void *X,
                                uint8_t *codes, uint8_t *scales)
{
    plan p;
    const pv_status st = make_plan(ctx, rows, cols, &p);
    if (st != PV_OK) return st;
    pv_timed t(ctx, PV_K_MX_CONVERT);
    return pv_for_dtype(x_type, [&](auto v) {
        using T = decltype(v);
        const auto k = format == PV_MX_E2M1 ? k_quantize_mx<PV_MX_E2M1, T> : k_quantize_mx<PV_MX_E4M3, T>;
        hipLaunchKernelGGL(k, dim3(p.blocks), dim3(kBlock), 0, ctx->stream, static_cast<const T *>(X), codes, scales,
                           rows, cols, p.nblk, p.waves_a_row);
        PV_HIP(ctx, hipGetLastError());
        return PV_OK;
    });
}

pv_status pv_launch_dequantize_mx(pv_ctx *ctx, int64_t rows, int64_t cols, int format, const uint8_t *codes,
                                  const uint8_t *scales, int out_type, void *out)
{
    plan p;
    const pv_status st = make_plan(ctx, rows, cols, &p);
    if (st != PV_OK) return st;
    pv_timed t(ctx, PV_K_MX_CONVERT);
    return pv_for_dtype(out_type, [&](auto v) {
        using T = decltype(v);
        const auto k = format == PV_MX_E2M1 ? k_dequantize_mx<PV_MX_E2M1, T> : k_dequantize_mx<PV_MX_E4M3, T>;
        hipLaunchKernelGGL(k, dim3(p.blocks), dim3(kBlock), 0, ctx->stream, codes, scales, static_cast<T *>(out), rows,
                           cols, p.nblk, p.waves_a_row);
        PV_HIP(ctx, hipGetLastError());
        return PV_OK;
    });
}

pv_status pv_launch_zero(pv_ctx *ctx, void *p, int64_t bytes)
{
    const int64_t n = bytes / 2, blocks = (n + kBlock - 1) / kBlock;
    hipLaunchKernelGGL(k_zero, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(kBlock), 0, ctx->stream,
                       static_cast<uint16_t *>(p), n);
    PV_HIP(ctx, hipGetLastError());
    return PV_OK;
}
