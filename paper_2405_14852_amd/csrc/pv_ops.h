// Shared by the operators around the V step (microscaled formats, product, norm, distillation):
// typed loads and stores of eight consecutive elements, the rounding of a block of 32 values to codes,
// reductions over a wave and a block, and the launchers' declarations.
#pragma once

#include "pv_dpp.h"
#include "pv_internal.h"

// mx block length, in values
constexpr int kMxBlock = 32;

static inline int64_t pv_mx_blocks(int64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }

// whether a launch can be made: its threads are counted in 32 bits
static inline bool pv_grid_fits(int64_t blocks, int threads) { return blocks < ((int64_t)1 << 32) / threads; }

static inline int pv_dtype_size(int t) { return t == PV_F32 ? 4 : 2; }

// Scratch of these operators.  A block that a captured call has used stays until the context goes:
// a later, larger call must not free memory that a graph still writes.
pv_status pv_ops_scratch(pv_ctx *ctx, size_t bytes, void **ptr);

// ---------------------------------------------------------------- launchers
pv_status pv_launch_quantize_mx(pv_ctx *ctx, int64_t rows, int64_t cols, int format, int x_type, const void *X,
                                uint8_t *codes, uint8_t *scales);
pv_status pv_launch_dequantize_mx(pv_ctx *ctx, int64_t rows, int64_t cols, int format, const uint8_t *codes,
                                  const uint8_t *scales, int out_type, void *out);
pv_status pv_launch_mx_product(pv_ctx *ctx, int64_t tokens, int64_t out, int64_t in, int x_format,
                               const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *w_codes,
                               const uint8_t *w_scales, int y_type, void *Y);
pv_status pv_launch_mx_product_grads(pv_ctx *ctx, int64_t tokens, int64_t out, int64_t in, int x_format,
                                     const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *w_codes,
                                     const uint8_t *w_scales, const void *dY, int dx_type, void *dX, float *dW);
pv_status pv_launch_rms_norm(pv_ctx *ctx, int64_t rows, int64_t cols, int type, const void *x, const void *residual,
                             const float *weight, float eps, void *h, void *y, int format, uint8_t *codes,
                             uint8_t *scales, float *rstd);
pv_status pv_launch_rms_norm_backward(pv_ctx *ctx, int64_t rows, int64_t cols, int type, const void *dy,
                                      const void *dh, const void *h, const float *weight, const float *rstd,
                                      void *dx, float *dweight);
// row_weight: c_r of the call (loss, gradient), or grad_loss of the backward call, where loss is NULL
pv_status pv_launch_distill(pv_ctx *ctx, int64_t rows, int64_t vocab, int k, int type, const void *logits, int64_t ld,
                            const int32_t *ids, const float *top, float temperature, const float *row_weight,
                            float *loss, float *lse, const float *lse_in, void *grad, int64_t grad_ld);
// zeros by a kernel: a memset node in a captured graph is not used here
pv_status pv_launch_zero(pv_ctx *ctx, void *p, int64_t bytes);

#ifdef __HIPCC__
typedef __bf16 pv_bf16;
typedef _Float16 pv_f16;
typedef float pv_f2 __attribute__((ext_vector_type(2)));
typedef unsigned pv_u2 __attribute__((ext_vector_type(2)));
typedef unsigned pv_u4 __attribute__((ext_vector_type(4)));

// eight elements as one value that needs no more alignment than an element does: gfx950 loads and
// stores 16 bytes at any address, so rows of odd lengths take the same path as aligned ones
template <class T>
struct pv_vec8 {
    typedef T raw __attribute__((ext_vector_type(8)));
    typedef raw type __attribute__((aligned(sizeof(T))));
};

template <class T>
__device__ __forceinline__ void pv_load8(const T *p, int valid, float (&v)[8])
{
    if (valid >= 8) {
        const typename pv_vec8<T>::raw r = *reinterpret_cast<const typename pv_vec8<T>::type *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)r[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < valid ? (float)p[i] : 0.0f;
    }
}

// the same, not yet converted
template <class T>
__device__ __forceinline__ typename pv_vec8<T>::raw pv_load8_raw(const T *p, int valid)
{
    if (valid >= 8) return *reinterpret_cast<const typename pv_vec8<T>::type *>(p);
    typename pv_vec8<T>::raw r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = i < valid ? p[i] : (T)0.0f;
    return r;
}

// STREAM: past the caches, for what a kernel writes in whole lines and nobody reads soon: the inputs stay (dequantisation of
// 14336 x 4096 in a quantising pass 78.5 -> 68.3 us; outputs in parts of lines lose by it, a product's 180 -> 245)
template <bool STREAM = false, class T>
__device__ __forceinline__ void pv_store8(T *p, int valid, const float (&v)[8])
{
    if (valid >= 8) {
        typename pv_vec8<T>::raw r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = (T)v[i];
        if constexpr (STREAM) __builtin_nontemporal_store(r, reinterpret_cast<typename pv_vec8<T>::type *>(p));
        else *reinterpret_cast<typename pv_vec8<T>::type *>(p) = r;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = (T)v[i];
    }
}

// Bits of the largest magnitude of a block of 32 values that four neighbouring lanes (a quad) hold, eight
// each.  Magnitudes compare like their bits, and a NaN's are above all others: it is not lost.
__device__ __forceinline__ unsigned pv_mx_largest(const float (&v)[8])
{
    unsigned a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(v[i]) & 0x7fffffffu);
    a = max(a, (unsigned)pv_dpp<kDppXor1>((int)a));
    return max(a, (unsigned)pv_dpp<kDppXor2>((int)a));
}

// Scale byte of a block from those bits: floor(log2) is the exponent field, a subnormal's counts as 0 and
// is clamped like it; not finite: 255.
template <int FMT>
__device__ __forceinline__ unsigned pv_mx_scale(unsigned largest)
{
    constexpr int kEmax = FMT == PV_MX_E2M1 ? 2 : 8;
    const int e = (int)(largest >> 23);
    return e == 255 ? 255u : (unsigned)max(e - kEmax, 0);
}

// Codes of eight values under the scale byte `s`.  The multiplication by 2^(127 - s) is exact as long as the result is
// a normal number, and where it is not the code is 0; the conversions round to the nearest, ties to even.
template <int FMT>
__device__ __forceinline__ pv_u2 pv_mx_encode(const float (&v)[8], unsigned s)
{
    constexpr float kTop = FMT == PV_MX_E2M1 ? 6.0f : 448.0f;
    const float inv = __uint_as_float(s == 255u ? 0u : (254u - s) << 23);
    float c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = s == 255u ? 0.0f : fminf(fmaxf(v[i] * inv, -kTop), kTop);
    pv_u2 r = {0u, 0u};
    if constexpr (FMT == PV_MX_E2M1) {
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.x, c[0], c[1], 1.0f, 0);
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.x, c[2], c[3], 1.0f, 1);
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.x, c[4], c[5], 1.0f, 2);
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.x, c[6], c[7], 1.0f, 3);
    } else {
        r.x = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], (int)r.x, false);
        r.x = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], (int)r.x, true);
        r.y = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c[4], c[5], (int)r.y, false);
        r.y = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c[6], c[7], (int)r.y, true);
    }
    return r;
}

// 2^(s - 127); 255: NaN
__device__ __forceinline__ float pv_mx_power(unsigned s)
{
    return __uint_as_float(s == 255u ? 0x7fc00000u : s == 0u ? 0x00400000u : s << 23);
}

// values of eight codes (E2M1: r.x alone)
template <int FMT>
__device__ __forceinline__ void pv_mx_decode(pv_u2 r, float power, float (&v)[8])
{
    pv_f2 d[4];
    if constexpr (FMT == PV_MX_E2M1) {
        d[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x, 1.0f, 0);
        d[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x, 1.0f, 1);
        d[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x, 1.0f, 2);
        d[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x, 1.0f, 3);
    } else {
        d[0] = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.x, false);
        d[1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.x, true);
        d[2] = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.y, false);
        d[3] = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.y, true);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = d[i].x * power;
        v[2 * i + 1] = d[i].y * power;
    }
}

// over LANES neighbouring lanes
template <int LANES = 64, class V, class F>
__device__ __forceinline__ V pv_wave_reduce(V v, F f)
{
#pragma unroll
    for (int m = LANES / 2; m; m >>= 1) v = f(v, __shfl_xor(v, m));
    return v;
}

// over THREADS / 64 waves, or a part of a wave; `part` has one entry a wave and may be used again after another barrier
template <int THREADS, class V, class F>
__device__ __forceinline__ V pv_block_reduce(V v, V *part, F f)
{
    constexpr int kWaves = THREADS / 64;
    v = pv_wave_reduce<(THREADS < 64 ? THREADS : 64)>(v, f);
    if constexpr (kWaves <= 1) return v;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = f(v, part[w]);
    return v;
}

struct pv_add {
    template <class V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};
struct pv_max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// calls f(T{}) with the element type of `t`
template <class F>
static inline pv_status pv_for_dtype(int t, F f)
{
    return t == PV_F32 ? f(float{}) : t == PV_BF16 ? f(pv_bf16{}) : f(pv_f16{});
}
#endif
