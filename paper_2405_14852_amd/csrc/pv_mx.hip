// Microscaled formats: a matrix to codes and scales, and back.  A block of 32 values shares the power of two
// 2^E with E = floor(log2(max |x|)) - emax; a code is x * 2^-E rounded to the format.  Both directions are
// streams bound by HBM: four neighbouring lanes hold a block, eight values each, so that a lane's load is 16 or 32
// bytes, its codes are one store of 4 or 8, and the block's maximum takes two exchanges inside a quad.
#include "pv_ops.h"

namespace {

constexpr int kBlock = 256;

// One wave per stretch of 64 * 8 values of a row: the row and the stretch come from scalar arithmetic, and a lane
// only has to look whether its eight values lie inside the row.  Lanes behind the row's last block do nothing; those
// inside it and behind `cols` write zero codes.  A matrix whose rows end with a block is one stretch after another, whatever
// its rows: it is taken as rows of 512, the last of them cut by `units` (2^20 rows of 64, bf16 to e4m3: 161 -> 32.4 us, back
// 118 -> 30.4).
struct span {
    int64_t row;
    int unit;        // of eight values, in the row
    int valid;       // values of them inside the row; may be below 0
    int64_t at;      // the unit among all of the matrix's
    bool live;       // it belongs to one of the row's blocks
};

struct plan {
    int64_t rows, units;
    int cols, nblk, waves_a_row;
};

__device__ __forceinline__ span wave_span(const plan &p)
{
    const int64_t w = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kBlock / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    span s;
    s.row = p.waves_a_row == 1 ? w : w / p.waves_a_row;
    s.unit = (int)(w - s.row * p.waves_a_row) * 64 + (threadIdx.x & 63);
    s.valid = p.cols - s.unit * 8;
    s.at = s.row * p.nblk * 4 + s.unit;
    s.live = s.row < p.rows && s.unit < p.nblk * 4 && s.at < p.units;
    return s;
}

template <int FMT, class T>
__global__ __launch_bounds__(kBlock) void k_quantize_mx(const T *__restrict__ X, uint8_t *__restrict__ codes,
                                                        uint8_t *__restrict__ scales, plan p)
{
    const span s = wave_span(p);
    if (!s.live) return;
    float v[8];
    pv_load8(X + s.row * p.cols + (int64_t)s.unit * 8, s.valid, v);
    const unsigned scale = pv_mx_scale<FMT>(pv_mx_largest(v));
    const pv_u2 c = pv_mx_encode<FMT>(v, scale);
    if constexpr (FMT == PV_MX_E2M1) reinterpret_cast<unsigned *>(codes)[s.at] = c.x;
    else reinterpret_cast<pv_u2 *>(codes)[s.at] = c;
    if ((s.unit & 3) == 0) scales[s.at >> 2] = (uint8_t)scale;
}

template <int FMT, class T>
__global__ __launch_bounds__(kBlock) void k_dequantize_mx(const uint8_t *__restrict__ codes,
                                                          const uint8_t *__restrict__ scales, T *__restrict__ out,
                                                          plan p)
{
    const span s = wave_span(p);
    if (!s.live) return;
    pv_u2 c = {0u, 0u};
    if constexpr (FMT == PV_MX_E2M1) c.x = reinterpret_cast<const unsigned *>(codes)[s.at];
    else c = reinterpret_cast<const pv_u2 *>(codes)[s.at];
    float v[8];
    pv_mx_decode<FMT>(c, pv_mx_power(scales[s.at >> 2]), v);
    pv_store8<true>(out + s.row * p.cols + (int64_t)s.unit * 8, s.valid, v);
}

__global__ __launch_bounds__(kBlock) void k_zero(uint16_t *p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlock) p[i] = 0;
}

// The grid has a second direction where the first, whose threads are counted in 32 bits, would not do
pv_status make_plan(pv_ctx *ctx, int64_t rows, int64_t cols, plan *p, dim3 *grid)
{
    constexpr int64_t kWide = 1 << 22;
    p->units = rows * pv_mx_blocks(cols) * 4;
    if (cols % kMxBlock == 0) {
        cols = 512;
        rows = (p->units + 63) / 64;
    }
    p->rows = rows;
    p->cols = (int)cols;
    p->nblk = (int)pv_mx_blocks(cols);
    p->waves_a_row = (p->nblk * 4 + 63) / 64;
    const int64_t blocks = (rows * p->waves_a_row + kBlock / 64 - 1) / (kBlock / 64);
    if (blocks >= (int64_t)1 << 31) return pv_fail(ctx, PV_ERR_UNSUPPORTED, "%lld rows are too many", (long long)rows);
    *grid = blocks <= kWide ? dim3((unsigned)blocks) : dim3((unsigned)kWide, (unsigned)((blocks + kWide - 1) / kWide));
    return PV_OK;
}

}  // namespace

pv_status pv_launch_quantize_mx(pv_ctx *ctx, int64_t rows, int64_t cols, int format, int x_type, const void *X,
                                uint8_t *codes, uint8_t *scales)
{
    plan p;
    dim3 grid;
    const pv_status st = make_plan(ctx, rows, cols, &p, &grid);
    if (st != PV_OK) return st;
    pv_timed t(ctx, PV_K_MX_CONVERT);
    return pv_for_dtype(x_type, [&](auto v) {
        using T = decltype(v);
        const auto k = format == PV_MX_E2M1 ? k_quantize_mx<PV_MX_E2M1, T> : k_quantize_mx<PV_MX_E4M3, T>;
        hipLaunchKernelGGL(k, grid, dim3(kBlock), 0, ctx->stream, static_cast<const T *>(X), codes, scales,
                           p);
        PV_HIP(ctx, hipGetLastError());
        return PV_OK;
    });
}

pv_status pv_launch_dequantize_mx(pv_ctx *ctx, int64_t rows, int64_t cols, int format, const uint8_t *codes,
                                  const uint8_t *scales, int out_type, void *out)
{
    plan p;
    dim3 grid;
    const pv_status st = make_plan(ctx, rows, cols, &p, &grid);
    if (st != PV_OK) return st;
    pv_timed t(ctx, PV_K_MX_CONVERT);
    return pv_for_dtype(out_type, [&](auto v) {
        using T = decltype(v);
        const auto k = format == PV_MX_E2M1 ? k_dequantize_mx<PV_MX_E2M1, T> : k_dequantize_mx<PV_MX_E4M3, T>;
        hipLaunchKernelGGL(k, grid, dim3(kBlock), 0, ctx->stream, codes, scales, static_cast<T *>(out), p);
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
