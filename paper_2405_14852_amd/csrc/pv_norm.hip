// Root-mean-square norm with the residual's addition and an output in 8 or 4 bits, and its gradients.
//   h = x + r,  rstd = (mean h^2 + eps)^(-1/2),  y = h rstd w
//   dx = dh + rstd (dy w - n mean(dy w n)),  dw = sum over rows of dy n,  n = h rstd
// Streams bound by HBM: a row is read once and stays in the registers of the lanes that share it, eight
// consecutive values a lane, so a block of 32 values lies in four neighbouring lanes as pv_quantize_mx wants it.
#include "pv_ops.h"

namespace {

constexpr int kBlock = 256;

// A row's rstd in two parts, the second what the first is rounded by: r (1 - r^2 m) / 2 with the roundings of r^2 and m kept.
// The squares of eight values are added in float32 and those sums in double, so that the mean is known beyond float32.
struct root {
    float hi, lo;
};

__device__ __forceinline__ root inverse_root(double mean)
{
    const float m = (float)mean, r = 1.0f / sqrtf(m), q = r * r;
    const float d = fmaf(-q, m, 1.0f) - fmaf(fmaf(r, r, -q), m, q * (float)(mean - m));
    return {r, fabsf(d) < 1.0f ? 0.5f * r * d : 0.0f};      // (of no number, an infinity, 0: none)
}

// h rstd w, rounded once; rest: what the rounding left
__device__ __forceinline__ float normed(float v, root rstd, float w, float &rest)
{
    const float n = v * rstd.hi, dn = fmaf(v, rstd.lo, fmaf(v, rstd.hi, -n));
    const float p = n * w, dp = fmaf(dn, w, fmaf(n, w, -p)), s = p + dp;
    rest = dp - (s - p);
    return fabsf(dp) < __builtin_inff() ? s : p;            // (p infinite: dp is so against it, or no number)
}

// One row's outputs from its stored sum v (a thread's eight values of it).  A code is that of the formula, not of a float32 that it
// rounds to: a value that float32 puts on a tie of the format is moved towards where it lies.  (8192 x 4096, e4m3: the roundings of
// float32 alone put 15 to 27 codes of the 33 million on the other side of a tie, each off by up to an eighth of its value; so 0 to 2, and
// 62.3 us instead of 60.2.)
template <class T, int FMT>
__device__ __forceinline__ void norm_out(const float (&v)[8], root rstd, const float (&w)[8], int valid, int unit, int units,
                                         int64_t row, int64_t cols, T *y, uint8_t *codes, uint8_t *scales)
{
    float o[8], rest;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = normed(v[i], rstd, w[i], rest);
    if (y) pv_store8<true>(y + row * cols + (int64_t)unit * 8, valid, o);
    if (codes && unit < units) {
        unsigned low = ~0u;                                 // a tie has 19 zero bits at its end in either format
#pragma unroll
        for (int i = 0; i < 8; ++i) low = min(low, __float_as_uint(o[i]) << 13);
        if (low == 0)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                normed(v[i], rstd, w[i], rest);
                const unsigned b = __float_as_uint(o[i]);
                if (b << 13 == 0 && fabsf(rest) > 0.0f && fabsf(o[i]) < __builtin_inff()) o[i] = __uint_as_float((rest < 0.0f) == (o[i] < 0.0f) ? b + 1 : b - 1);
            }
        const unsigned scale = pv_mx_scale<FMT>(pv_mx_largest(o));
        const pv_u2 c = pv_mx_encode<FMT>(o, scale);
        const int64_t at = row * units + unit;
        if constexpr (FMT == PV_MX_E2M1) reinterpret_cast<unsigned *>(codes)[at] = c.x;
        else reinterpret_cast<pv_u2 *>(codes)[at] = c;
        if ((unit & 3) == 0) scales[at >> 2] = (uint8_t)scale;
    }
}

// TPR threads share a row (up to 64: kBlock / TPR rows a block, no barrier; else the block's), each with NV times eight values.  A block
// goes from row to row, in steps of the grid, with its weights in registers and the next row already on its way while this
// one is summed (8192 x 4096, bf16 to e4m3: 63.8 us with a wave a row and the weights read for each).
template <class T, int TPR, int NV, int FMT>
__global__ __launch_bounds__(TPR <= 64 ? kBlock : TPR) void k_rms_norm(const T *x, const T *residual,
                                                                       const float *__restrict__ weight, float eps, T *h,
                                                                       T *y, uint8_t *__restrict__ codes,
                                                                       uint8_t *__restrict__ scales,
                                                                       float *__restrict__ rstd_out, int64_t rows,
                                                                       int64_t cols, int nblk)
{
    constexpr int kThreads = TPR <= 64 ? kBlock : TPR, kRows = kThreads / TPR;
    __shared__ double part[2][kThreads / 64];
    const double per = 1.0 / (double)cols;
    typedef typename pv_vec8<T>::raw raw;
    const int t = threadIdx.x % TPR, units = nblk * 4;
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    const int64_t stride = (int64_t)gridDim.x * kRows;
    raw a[NV], b[NV];
    auto load = [&](int64_t at) {
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int unit = u * TPR + t, valid = (int)cols - unit * 8;
            a[u] = pv_load8_raw(x + at * cols + (int64_t)unit * 8, valid);
            if (residual) b[u] = pv_load8_raw(residual + at * cols + (int64_t)unit * 8, valid);
        }
    };
    if (row < rows) load(row);
    float w[NV][8];
#pragma unroll
    for (int u = 0; u < NV; ++u) pv_load8(weight + (u * TPR + t) * 8, (int)cols - (u * TPR + t) * 8, w[u]);
    for (int turn = 0; row < rows; row += stride, turn ^= 1) {      // alike in all that share a row, and a whole block's where it meets in barriers
        float v[NV][8];
        double sum = 0.0;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            float eight = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[u][i] = (float)a[u][i];
                if (residual) v[u][i] = (float)(T)(v[u][i] + (float)b[u][i]);
                eight = fmaf(v[u][i], v[u][i], eight);
            }
            sum += eight;
        }
        if (row + stride < rows) load(row + stride);                // (another row: the outputs may lie on the inputs)
#pragma unroll
        for (int u = 0; u < NV; ++u)
            if (h) pv_store8<true>(h + row * cols + (u * TPR + t) * 8, (int)cols - (u * TPR + t) * 8, v[u]);
        sum = pv_block_reduce<TPR>(sum, part[turn], pv_add{});
        const root rstd = inverse_root(sum * per + eps);
        if (rstd_out && t == 0) rstd_out[row] = rstd.hi + rstd.lo;
#pragma unroll
        for (int u = 0; u < NV; ++u)
            norm_out<T, FMT>(v[u], rstd, w[u], (int)cols - (u * TPR + t) * 8, u * TPR + t, units, row, cols, y, codes, scales);
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
    __shared__ double part[2][16];
    const double per = 1.0 / (double)cols;
    const int units = nblk * 4;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
        const int64_t base = row * cols;
        auto load = [&](int unit, int valid, float (&v)[8]) {
            pv_load8(x + base + (int64_t)unit * 8, valid, v);
            if (!residual) return;
            float r[8];
            pv_load8(residual + base + (int64_t)unit * 8, valid, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)(T)(v[i] + r[i]);
        };
        double sum = 0.0;
        for (int unit = threadIdx.x; unit < units; unit += 1024) {
            float v[8], eight = 0.0f;
            load(unit, (int)cols - unit * 8, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) eight = fmaf(v[i], v[i], eight);
            sum += eight;
        }
        sum = pv_block_reduce<1024>(sum, part[turn], pv_add{});
        const root rstd = inverse_root(sum * per + eps);
        if (rstd_out && threadIdx.x == 0) rstd_out[row] = rstd.hi + rstd.lo;
        for (int unit = threadIdx.x; unit < units; unit += 1024) {
            const int valid = (int)cols - unit * 8;
            float v[8], w[8];
            load(unit, valid, v);
            if (h) pv_store8(h + base + (int64_t)unit * 8, valid, v);
            pv_load8(weight + (int64_t)unit * 8, valid, w);
            norm_out<T, FMT>(v, rstd, w, valid, unit, units, row, cols, y, codes, scales);
        }
    }
}

// Backward: block b takes the rows b, b + gridDim.x, ... (short rows, of TPR threads: kRows of them at a time) with the weights and
// its sums for dweight in registers from row to row; the sums leave once, as one row of `partial`.  A row stays as it was read, and the factors are formed twice, which takes
// half the registers.  Where they leave room for one block a compute unit only and for another row (kAhead), that row is on its
// way while this one is reduced.
template <class T, int THREADS, int NV, int TPR = THREADS>
__global__ __launch_bounds__(THREADS) void k_rms_norm_backward(const T *dy, const T *dh, const T *h,
                                                               const float *__restrict__ weight,
                                                               const float *__restrict__ rstd_in, T *dx,
                                                               float *__restrict__ partial, int64_t rows, int64_t cols)
{
    constexpr int kRows = THREADS / TPR;
    static_assert(kRows == 1 || (NV == 1 && TPR <= 64), "");
    __shared__ float part[2][THREADS / 64];
    typedef typename pv_vec8<T>::raw raw;
    const int t = threadIdx.x % TPR;
    const int64_t row0 = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR, stride = (int64_t)gridDim.x * kRows;
    float acc[NV][8], w[NV][8];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        pv_load8(weight + (u * TPR + t) * 8, (int)cols - (u * TPR + t) * 8, w[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[u][i] = 0.0f;
    }
    constexpr bool kAhead = NV == 3 && sizeof(T) == 2;
    raw next[kAhead ? 3 * NV : 1];
    auto load = [&](int64_t row, raw *a, raw *b, raw *c) {
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int first = (u * TPR + t) * 8, valid = (int)cols - first;
            a[u] = pv_load8_raw(dy + row * cols + first, valid);
            b[u] = pv_load8_raw(h + row * cols + first, valid);
            if (dh && dx) c[u] = pv_load8_raw(dh + row * cols + first, valid);
        }
    };
    if constexpr (kAhead) load(row0, next, next + NV, next + 2 * NV);
    int turn = 0;
    for (int64_t row = row0; row < rows; row += stride, turn ^= 1) {
        const float rstd = rstd_in[row];
        raw a[NV], b[NV], c[NV];
        if constexpr (kAhead) {
#pragma unroll
            for (int u = 0; u < NV; ++u) a[u] = next[u], b[u] = next[NV + u], c[u] = next[2 * NV + u];
            if (row + stride < rows) load(row + stride, next, next + NV, next + 2 * NV);      // (another row: dx may lie on an input)
        } else {
            load(row, a, b, c);
        }
        float dot = 0.0f;
#pragma unroll
        for (int u = 0; u < NV; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float n = (float)b[u][i] * rstd;
                acc[u][i] = fmaf((float)a[u][i], n, acc[u][i]);
                dot = fmaf((float)a[u][i] * w[u][i], n, dot);
            }
        if (!dx) continue;
        const float mean = pv_block_reduce<TPR>(dot, part[turn], pv_add{}) / (float)cols;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int first = (u * TPR + t) * 8;
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e = rstd * fmaf(-((float)b[u][i] * rstd), mean, (float)a[u][i] * w[u][i]);
                d[i] = dh ? (float)c[u][i] + e : e;
            }
            pv_store8<true>(dx + row * cols + first, (int)cols - first, d);
        }
    }
    if (!partial) return;
    if constexpr (kRows > 1) {                         // the block's rows together, in their order
        __shared__ float s[kRows][TPR * 8 + 4];        // (16 bytes behind a row: its first bank is another's)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[threadIdx.x / TPR][t * 8 + i] = acc[0][i];
        __syncthreads();
        for (int col = threadIdx.x; col < TPR * 8 && col < cols; col += THREADS) {
            float sum = s[0][col];
#pragma unroll
            for (int r = 1; r < kRows; ++r) sum += s[r][col];
            partial[(int64_t)blockIdx.x * cols + col] = sum;
        }
        return;
    }
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int first = (u * TPR + t) * 8;
        pv_store8(partial + (int64_t)blockIdx.x * cols + first, (int)cols - first, acc[u]);
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

// dweight: the blocks' sums added in the order of the blocks, 32 threads a column for a part of them each, and 32 columns at a time
__global__ __launch_bounds__(1024) void k_sum_partials(const float *__restrict__ partial, int parts, int64_t cols,
                                                         float *__restrict__ out)
{
    __shared__ float s[32][33];
    const int c = threadIdx.x & 31, e = threadIdx.x >> 5;
    for (int64_t first = (int64_t)blockIdx.x * 32; first < cols; first += (int64_t)gridDim.x * 32) {
        const int64_t col = first + c;
        float sum = 0.0f;
        if (col < cols)
#pragma unroll 8
            for (int p = e * parts / 32; p < (e + 1) * parts / 32; ++p) sum += partial[(int64_t)p * cols + col];
        s[e][c] = sum;
        __syncthreads();
        if (e == 0 && col < cols) {
#pragma unroll
            for (int i = 1; i < 32; ++i) sum += s[i][c];
            out[col] = sum;
        }
        __syncthreads();
    }
}

constexpr int kMostUnits = 2048;      // of eight values, of a row in registers

// f(integral_constant<int, NV>), NV = ceil(units / threads) <= MAX_NV
template <int MAX_NV, class F>
pv_status for_nv(int units, int threads, F f)
{
    if (units <= threads) return f(std::integral_constant<int, 1>{});
    if constexpr (MAX_NV > 2) {
        if (units > 2 * threads) {
            if constexpr (MAX_NV > 3) {
                if (units > 3 * threads) return f(std::integral_constant<int, 4>{});
            }
            return f(std::integral_constant<int, 3>{});
        }
    }
    return f(std::integral_constant<int, 2>{});
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
        if (units > kMostUnits) {
            const auto k = format == PV_MX_E2M1 ? k_rms_norm_long<T, PV_MX_E2M1> : k_rms_norm_long<T, PV_MX_E4M3>;
            return launch(k, (unsigned)(rows < 4096 ? rows : 4096), 1024);
        }
        // short rows, enough of them to fill the chip: a wave a row, or an eighth or a quarter of one (bf16, h and y: 2^20 rows of 64
        // 314 us with a wave, 109 with a quarter, 83 with an eighth; 2^19 of 128 170 with a wave, 83 with a quarter)
        if (units <= 128 && rows >= 1024) {
            auto wave = [&](auto lanes, auto nv) {
                constexpr int NV = decltype(nv)::value, TPR = decltype(lanes)::value, kRows = kBlock / TPR;
                const int64_t blocks = (rows + kRows - 1) / kRows;
                return launch(format == PV_MX_E2M1 ? k_rms_norm<T, TPR, NV, PV_MX_E2M1> : k_rms_norm<T, TPR, NV, PV_MX_E4M3>,
                              (unsigned)(blocks < 4096 ? blocks : 4096), kBlock);
            };
            constexpr std::integral_constant<int, 1> one{};
            constexpr std::integral_constant<int, 2> two{};
            constexpr std::integral_constant<int, 8> eighth{};
            constexpr std::integral_constant<int, 16> quarter{};
            constexpr std::integral_constant<int, 64> whole{};
            return units <= 8 ? wave(eighth, one) : units <= 16 ? wave(quarter, one) : units <= 32 ? wave(quarter, two) : units <= 64 ? wave(whole, one) : wave(whole, two);
        }
        auto block = [&](auto threads, auto nv) {
            constexpr int THREADS = decltype(threads)::value, NV = decltype(nv)::value;
            const int64_t most = 256 * (2048 / THREADS);      // as many threads as the chip holds
            return launch(format == PV_MX_E2M1 ? k_rms_norm<T, THREADS, NV, PV_MX_E2M1> : k_rms_norm<T, THREADS, NV, PV_MX_E4M3>,
                          (unsigned)(rows < most ? rows : most), THREADS);
        };
        if (units <= 1024) return for_nv<4>(units, 256, [&](auto nv) { return block(std::integral_constant<int, 256>{}, nv); });
        return for_nv<4>(units, 512, [&](auto nv) { return block(std::integral_constant<int, 512>{}, nv); });
    });
}

pv_status pv_launch_rms_norm_backward(pv_ctx *ctx, int64_t rows, int64_t cols, int type, const void *dy,
                                      const void *dh, const void *h, const float *weight, const float *rstd,
                                      void *dx, float *dweight)
{
    const int units = (int)((cols + 7) / 8);
    // each block leaves a row of sums that is written and read: no more of them than an eighth of the rows is worth
    const int64_t most = units > 1024 ? 256 : rows >= 4096 ? 1024 : 512;
    // threads a row of a block of 256: as many of 8, 16, 32, 64 as hold a short row, if there are enough of them to fill the chip
    // (bf16, 2^19 rows of 128 with the block a row 1096 us, with 16 threads 99)
    const int tpr = rows < 4096 || units > 64 ? 256 : units <= 8 ? 8 : units <= 16 ? 16 : units <= 32 ? 32 : 64;
    const int64_t groups = (rows + 256 / tpr - 1) / (256 / tpr), blocks = groups < most ? groups : most;
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
    pv_status st = pv_for_dtype(type, [&](auto v) {
        using T = decltype(v);
        auto launch = [&](auto k, int threads) {
            hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(threads), 0, ctx->stream, static_cast<const T *>(dy),
                               static_cast<const T *>(dh), static_cast<const T *>(h), weight, rstd,
                               static_cast<T *>(dx), partial, rows, cols);
            PV_HIP(ctx, hipGetLastError());
            return PV_OK;
        };
        if (units > kMostUnits) return launch(k_rms_norm_backward_long<T>, 1024);
        if (tpr == 8) return launch(k_rms_norm_backward<T, 256, 1, 8>, 256);
        if (tpr == 16) return launch(k_rms_norm_backward<T, 256, 1, 16>, 256);
        if (tpr == 32) return launch(k_rms_norm_backward<T, 256, 1, 32>, 256);
        if (tpr == 64) return launch(k_rms_norm_backward<T, 256, 1, 64>, 256);
        if (units <= 256) return launch(k_rms_norm_backward<T, 256, 1>, 256);
        return for_nv<4>(units, 512, [&](auto nv) { return launch(k_rms_norm_backward<T, 512, decltype(nv)::value>, 512); });
    });
    if (st != PV_OK || partial == dweight) return st;
    // (a launch's threads are counted in 32 bits: 2^21 blocks are half of that)
    const int64_t sums = (cols + 31) / 32;
    hipLaunchKernelGGL(k_sum_partials, dim3((unsigned)(sums < 1 << 21 ? sums : 1 << 21)), dim3(1024), 0, ctx->stream, partial,
                       (int)blocks, cols, dweight);
    PV_HIP(ctx, hipGetLastError());
    return PV_OK;
}
