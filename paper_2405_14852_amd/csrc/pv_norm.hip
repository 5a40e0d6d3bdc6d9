// Root-mean-square norm with the residual's addition and an output in 8 or 4 bits, and its gradients.
//   h = x + r,  rstd = (mean h^2 + eps)^(-1/2),  y = h rstd w
//   dx = dh + rstd (dy w - n mean(dy w n)),  dw = sum over rows of dy n,  n = h rstd
// Streams bound by HBM: a row is read once and stays in the registers of the lanes that share it, eight
// consecutive values a lane, so a block of 32 values lies in four neighbouring lanes as pv_quantize_mx wants it.
#include "pv_ops.h"

namespace {

constexpr int kBlock = 256;

// TPR threads share a row (64: four rows a block, no barrier; kBlock: one row a block), each with NV times eight values.
template <class T, int TPR, int NV, int FMT>
__global__ __launch_bounds__(kBlock) void k_rms_norm(const T *x, const T *residual, const float *__restrict__ weight,
                                                     float eps, T *h, T *y, uint8_t *__restrict__ codes,
                                                     uint8_t *__restrict__ scales, float *__restrict__ rstd_out,
                                                     int64_t rows, int64_t cols, int nblk)
{
    __shared__ float part[kBlock / 64];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (kBlock / TPR) + threadIdx.x / TPR;
    if (row >= rows) return;             // a whole wave, and a whole block where they meet in barriers
    const int64_t base = row * cols;
    const int units = nblk * 4;
    // every load before the first store: the outputs may lie on the inputs, so the compiler keeps their order
    float v[NV][8], r[NV][8];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int unit = u * TPR + t, valid = (int)cols - unit * 8;
        pv_load8(x + base + (int64_t)unit * 8, valid, v[u]);
        if (residual) pv_load8(residual + base + (int64_t)unit * 8, valid, r[u]);
    }
    float sum = 0.0f;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int unit = u * TPR + t, valid = (int)cols - unit * 8;
        if (residual) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = (float)(T)(v[u][i] + r[u][i]);
        }
        if (h) pv_store8(h + base + (int64_t)unit * 8, valid, v[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(v[u][i], v[u][i], sum);
    }
    sum = pv_block_reduce<TPR>(sum, part, pv_add{});
    const float rstd = 1.0f / sqrtf(sum / (float)cols + eps);
    if (rstd_out && t == 0) rstd_out[row] = rstd;
    if (!y && !codes) return;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int unit = u * TPR + t, valid = (int)cols - unit * 8;
        float w[8];
        pv_load8(weight + (int64_t)unit * 8, valid, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] = (v[u][i] * rstd) * w[i];
        if (y) pv_store8(y + base + (int64_t)unit * 8, valid, v[u]);
        if (codes && unit < units) {
            const unsigned scale = pv_mx_scale<FMT>(pv_mx_largest(v[u]));
            const pv_u2 c = pv_mx_encode<FMT>(v[u], scale);
            const int64_t at = row * units + unit;
            if constexpr (FMT == PV_MX_E2M1) reinterpret_cast<unsigned *>(codes)[at] = c.x;
            else reinterpret_cast<pv_u2 *>(codes)[at] = c;
            if ((unit & 3) == 0) scales[at >> 2] = (uint8_t)scale;
        }
    }
}

// Rows that no block's registers hold: the sum first, then the row once more.  A lane that writes has read the
// same elements itself (x and residual again, before h or y over them), so the outputs may lie on the inputs.
template <class T, int FMT>
__global__ __launch_bounds__(1024) void k_rms_norm_long(const T *x, const T *residual,
                                                        const float *__restrict__ weight, float eps, T *h, T *y,
                                                        uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                        float *__restrict__ rstd_out, int64_t rows, int64_t cols,
                                                        int nblk)
{
    __shared__ float part[16];
    const int64_t row = blockIdx.x, base = row * cols;
    const int units = nblk * 4;
    auto load = [&](int unit, int valid, float (&v)[8]) {
        pv_load8(x + base + (int64_t)unit * 8, valid, v);
        if (!residual) return;
        float r[8];
        pv_load8(residual + base + (int64_t)unit * 8, valid, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)(T)(v[i] + r[i]);
    };
    float sum = 0.0f;
    for (int unit = threadIdx.x; unit < units; unit += 1024) {
        float v[8];
        load(unit, (int)cols - unit * 8, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(v[i], v[i], sum);
    }
    sum = pv_block_reduce<1024>(sum, part, pv_add{});
    const float rstd = 1.0f / sqrtf(sum / (float)cols + eps);
    if (rstd_out && threadIdx.x == 0) rstd_out[row] = rstd;
    for (int unit = threadIdx.x; unit < units; unit += 1024) {
        const int valid = (int)cols - unit * 8;
        float v[8], w[8];
        load(unit, valid, v);
        if (h) pv_store8(h + base + (int64_t)unit * 8, valid, v);
        pv_load8(weight + (int64_t)unit * 8, valid, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (v[i] * rstd) * w[i];
        if (y) pv_store8(y + base + (int64_t)unit * 8, valid, v);
        if (codes) {
            const unsigned scale = pv_mx_scale<FMT>(pv_mx_largest(v));
            const pv_u2 c = pv_mx_encode<FMT>(v, scale);
            const int64_t at = row * units + unit;
            if constexpr (FMT == PV_MX_E2M1) reinterpret_cast<unsigned *>(codes)[at] = c.x;
            else reinterpret_cast<pv_u2 *>(codes)[at] = c;
            if ((unit & 3) == 0) scales[at >> 2] = (uint8_t)scale;
        }
    }
}

// Backward: block b takes the rows b, b + gridDim.x, ... and keeps its sums for dweight in registers from row to row;
// they leave once, as one row of `partial`.
template <class T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void k_rms_norm_backward(const T *dy, const T *dh, const T *h,
                                                               const float *__restrict__ weight,
                                                               const float *__restrict__ rstd_in, T *dx,
                                                               float *__restrict__ partial, int64_t rows, int64_t cols)
{
    __shared__ float part[2][THREADS / 64];
    const int t = threadIdx.x;
    float acc[NV][8];
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[u][i] = 0.0f;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
        const int64_t base = row * cols;
        const float rstd = rstd_in[row];
        float g[NV][8], n[NV][8];
        float dot = 0.0f;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int64_t at = (int64_t)(u * THREADS + t) * 8;
            const int valid = (int)cols - (u * THREADS + t) * 8;
            pv_load8(dy + base + at, valid, g[u]);
            pv_load8(h + base + at, valid, n[u]);
        }
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int64_t at = (int64_t)(u * THREADS + t) * 8;
            const int valid = (int)cols - (u * THREADS + t) * 8;
            float w[8];
            pv_load8(weight + at, valid, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[u][i] *= rstd;
                acc[u][i] = fmaf(g[u][i], n[u][i], acc[u][i]);
                g[u][i] *= w[i];
                dot = fmaf(g[u][i], n[u][i], dot);
            }
        }
        if (!dx) continue;
        const float mean = pv_block_reduce<THREADS>(dot, part[turn], pv_add{}) / (float)cols;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int64_t at = (int64_t)(u * THREADS + t) * 8;
            const int valid = (int)cols - (u * THREADS + t) * 8;
            float d[8];
            if (dh) pv_load8(dh + base + at, valid, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e = rstd * fmaf(-n[u][i], mean, g[u][i]);
                d[i] = dh ? d[i] + e : e;
            }
            pv_store8(dx + base + at, valid, d);
        }
    }
    if (!partial) return;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int64_t at = (int64_t)(u * THREADS + t) * 8;
        pv_store8(partial + (int64_t)blockIdx.x * cols + at, (int)cols - (int)at, acc[u]);
    }
}

// Rows that no block's registers hold: the row's dot product, and then the row once more.  A block's sums for
// dweight are read and written in its row of `partial`, which it alone touches, each entry by one thread.
template <class T>
__global__ __launch_bounds__(1024) void k_rms_norm_backward_long(const T *dy, const T *dh, const T *h,
                                                                 const float *__restrict__ weight,
                                                                 const float *__restrict__ rstd_in, T *dx,
                                                                 float *__restrict__ partial, int64_t rows,
                                                                 int64_t cols)
{
    __shared__ float part[2][16];
    float *mine = partial ? partial + (int64_t)blockIdx.x * cols : nullptr;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
        const int64_t base = row * cols;
        const float rstd = rstd_in[row];
        const bool first = row == blockIdx.x;
        float dot = 0.0f;
        for (int64_t at = (int64_t)threadIdx.x * 8; at < cols; at += 8192) {
            const int valid = (int)(cols - at);
            float g[8], n[8], w[8], a[8];
            pv_load8(dy + base + at, valid, g);
            pv_load8(h + base + at, valid, n);
            pv_load8(weight + at, valid, w);
            if (mine && !first) pv_load8(mine + at, valid, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] *= rstd;
                a[i] = fmaf(g[i], n[i], mine && !first ? a[i] : 0.0f);
                dot = fmaf(g[i] * w[i], n[i], dot);
            }
            if (mine) pv_store8(mine + at, valid, a);
        }
        if (!dx) continue;
        const float mean = pv_block_reduce<1024>(dot, part[turn], pv_add{}) / (float)cols;
        for (int64_t at = (int64_t)threadIdx.x * 8; at < cols; at += 8192) {
            const int valid = (int)(cols - at);
            float g[8], n[8], w[8], d[8];
            pv_load8(dy + base + at, valid, g);
            pv_load8(h + base + at, valid, n);
            pv_load8(weight + at, valid, w);
            if (dh) pv_load8(dh + base + at, valid, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e = rstd * fmaf(-(n[i] * rstd), mean, g[i] * w[i]);
                d[i] = dh ? d[i] + e : e;
            }
            pv_store8(dx + base + at, valid, d);
        }
    }
}

// dweight: the blocks' sums added in the order of the blocks, 8 threads a column for an eighth of them each
__global__ __launch_bounds__(kBlock) void k_sum_partials(const float *__restrict__ partial, int parts, int64_t cols,
                                                         float *__restrict__ out)
{
    __shared__ float s[8][32];
    const int c = threadIdx.x & 31, e = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + c;
    float sum = 0.0f;
    if (col < cols)
#pragma unroll 8
        for (int p = e * parts / 8; p < (e + 1) * parts / 8; ++p) sum += partial[(int64_t)p * cols + col];
    s[e][c] = sum;
    __syncthreads();
    if (e == 0 && col < cols) {
#pragma unroll
        for (int i = 1; i < 8; ++i) sum += s[i][c];
        out[col] = sum;
    }
}

// f(integral_constant<int, NV>) for the smallest of 1, 2, 4, 8 that covers `units` with `threads`
template <class F>
pv_status for_nv(int units, int threads, F f)
{
    const int nv = (units + threads - 1) / threads;
    if (nv <= 1) return f(std::integral_constant<int, 1>{});
    if (nv <= 2) return f(std::integral_constant<int, 2>{});
    if (nv <= 4) return f(std::integral_constant<int, 4>{});
    return f(std::integral_constant<int, 8>{});
}

}  // namespace

pv_status pv_launch_rms_norm(pv_ctx *ctx, int64_t rows, int64_t cols, int type, const void *x, const void *residual,
                             const float *weight, float eps, void *h, void *y, int format, uint8_t *codes,
                             uint8_t *scales, float *rstd)
{
    const int nblk = (int)pv_mx_blocks(cols), units = nblk * 4;
    pv_timed t(ctx, PV_K_RMS_NORM);
    return pv_for_dtype(type, [&](auto v) {
        using T = decltype(v);
        auto launch = [&](auto k, unsigned blocks, int threads) {
            hipLaunchKernelGGL(k, dim3(blocks), dim3(threads), 0, ctx->stream, static_cast<const T *>(x),
                               static_cast<const T *>(residual), weight, eps, static_cast<T *>(h),
                               static_cast<T *>(y), codes, scales, rstd, rows, cols, nblk);
            PV_HIP(ctx, hipGetLastError());
            return PV_OK;
        };
        if (units > kBlock * 8) {
            const auto k = format == PV_MX_E2M1 ? k_rms_norm_long<T, PV_MX_E2M1> : k_rms_norm_long<T, PV_MX_E4M3>;
            return launch(k, (unsigned)rows, 1024);
        }
        // a wave a row where that fills the chip and its registers hold it
        if (units <= 64 * 8 && rows >= 1024)
            return for_nv(units, 64, [&](auto nv) {
                constexpr int NV = decltype(nv)::value;
                const auto k = format == PV_MX_E2M1 ? k_rms_norm<T, 64, NV, PV_MX_E2M1> : k_rms_norm<T, 64, NV, PV_MX_E4M3>;
                return launch(k, (unsigned)((rows + 3) / 4), kBlock);
            });
        return for_nv(units, kBlock, [&](auto nv) {
            constexpr int NV = decltype(nv)::value;
            const auto k = format == PV_MX_E2M1 ? k_rms_norm<T, kBlock, NV, PV_MX_E2M1> : k_rms_norm<T, kBlock, NV, PV_MX_E4M3>;
            return launch(k, (unsigned)rows, kBlock);
        });
    });
}

pv_status pv_launch_rms_norm_backward(pv_ctx *ctx, int64_t rows, int64_t cols, int type, const void *dy,
                                      const void *dh, const void *h, const float *weight, const float *rstd,
                                      void *dx, float *dweight)
{
    constexpr int kThreads = 512;
    constexpr int64_t kMaxBlocks = 512;      // two a compute unit
    const int64_t blocks = rows < kMaxBlocks ? rows : kMaxBlocks;
    float *partial = nullptr;
    if (dweight && blocks > 1) {
        void *p;
        const pv_status st = pv_ops_scratch(ctx, (size_t)(blocks * cols) * sizeof(float), &p);
        if (st != PV_OK) return st;
        partial = static_cast<float *>(p);
    } else {
        partial = dweight;
    }
    pv_timed t(ctx, PV_K_RMS_NORM);
    const int units = (int)((cols + 7) / 8);
    pv_status st = pv_for_dtype(type, [&](auto v) {
        using T = decltype(v);
        auto launch = [&](auto k, int threads) {
            hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(threads), 0, ctx->stream, static_cast<const T *>(dy),
                               static_cast<const T *>(dh), static_cast<const T *>(h), weight, rstd,
                               static_cast<T *>(dx), partial, rows, cols);
            PV_HIP(ctx, hipGetLastError());
            return PV_OK;
        };
        if (units > kThreads * 4) return launch(k_rms_norm_backward_long<T>, 1024);
        return for_nv(units, kThreads, [&](auto nv) {
            constexpr int NV = decltype(nv)::value < 4 ? decltype(nv)::value : 4;
            return launch(k_rms_norm_backward<T, kThreads, NV>, kThreads);
        });
    });
    if (st != PV_OK || partial == dweight) return st;
    hipLaunchKernelGGL(k_sum_partials, dim3((unsigned)((cols + 31) / 32)), dim3(kBlock), 0, ctx->stream, partial,
                       (int)blocks, cols, dweight);
    PV_HIP(ctx, hipGetLastError());
    return PV_OK;
}
