// Distillation from a teacher's k largest logits: loss, and the gradient of the student's logits.
//   p = softmax_j(u_j / t) over the teacher's entries, q = softmax_v(z_v / t) over the vocabulary
//   loss = c t^2 sum_j p_j (ln p_j - ln q[id_j]),   grad_v = c t (q_v - sum_{j: id_j = v} p_j)
// Bound by HBM: the logits in, the gradient out, 2 or 4 bytes an entry each.  A block takes a row, and the
// row stays in its registers between the sum and the gradient where they hold it; the exponentials are formed twice
// instead of being kept, at 16 a clock and compute unit they cost a fraction of the bytes.
// The teacher's entries are k places of the row.  The sweep writes all of the row as if there were none; once its stores are
// done the first entry of each id writes its place again, less the sum of the entries with that id in the order of the
// list: one writer a place, no atomics on sums, the same bits every time.  (A sweep that leaves the places out
// splits a store of 16 bytes into single elements wherever one lies: 2048 x 32000 with 256 entries 76 us.)  A bit per place in
// LDS tells whether any place has two entries; only then are the lists compared.
#include "pv_ops.h"

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

template <class T>
struct unit_of {                                  // 16 bytes of a row, at any element's address
    static constexpr int n = 16 / sizeof(T);
    typedef T raw __attribute__((ext_vector_type(n)));
    typedef raw type __attribute__((aligned(sizeof(T))));
};

// past the caches (2048 x 32000: 61.5 -> 56.2 us)
template <class T>
__device__ __forceinline__ void store_unit(T *g, int unit, int vocab, const typename unit_of<T>::raw &r)
{
    constexpr int U = unit_of<T>::n;
    if ((unit + 1) * U <= vocab) {
        __builtin_nontemporal_store(r, reinterpret_cast<typename unit_of<T>::type *>(g + unit * U));
        return;
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
        if (unit * U + i < vocab) g[unit * U + i] = r[i];
}

// two values over a block, with one barrier
template <int WAVES, class F>
__device__ __forceinline__ void reduce_two(float &a, float &b, float *part, F f)
{
    a = pv_wave_reduce(a, f);
    b = pv_wave_reduce(b, f);
    if ((threadIdx.x & 63) == 0) {
        part[threadIdx.x >> 6] = a;
        part[WAVES + (threadIdx.x >> 6)] = b;
    }
    __syncthreads();
    a = part[0];
    b = part[WAVES];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
        a = f(a, part[w]);
        b = f(b, part[WAVES + w]);
    }
}

struct args {
    const int32_t *ids;
    const float *top, *row_weight, *lse_in;
    float *loss, *lse;
    int64_t ld, grad_ld;
    int vocab, k;
    float t;
    unsigned pieces;         // blocks a row (backward)
};

// NV > 0: the row lies in NV units a thread.  NV == 0: it passes by, with a running largest value and sum in each thread, and
// is read again for the gradient if there is one.
// LSE: the sum is given (the backward call), only the gradient is formed, by a block for every NV units a thread of a row.
// row, z, g: the block's row; c: its weight; first: the unit that the block begins with.
template <class T, int THREADS, int NV, bool LSE>
__device__ __forceinline__ void distill_row(const args &a, int64_t row, const T *z, T *g, float c, int first)
{
    constexpr int U = unit_of<T>::n, kWaves = THREADS / 64;
    constexpr float kNone = -__builtin_inff();
    typedef typename unit_of<T>::raw raw;
    typedef typename unit_of<T>::type loose;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    float *p = reinterpret_cast<float *>(lds);                        // [k] the teacher's logits
    float *zt = p + a.k;                                              // [k] the logits in their places
    int *id = reinterpret_cast<int *>(zt + a.k);                      // [k] their places, -1: none
    unsigned *mark = reinterpret_cast<unsigned *>(id + a.k);          // [ceil(vocab / 32)] places of the row
    __shared__ float part[3][2 * kWaves];
    __shared__ int s_twice;                                           // some place has two entries

    const int tid = threadIdx.x, V = a.vocab, k = a.k;
    const int units = LSE ? min((V + U - 1) / U, first + NV * THREADS) : (V + U - 1) / U;

    auto load = [&](int unit) {
        raw r;
        if ((unit + 1) * U <= V) return (raw)*reinterpret_cast<const loose *>(z + unit * U);
#pragma unroll
        for (int i = 0; i < U; ++i) r[i] = unit * U + i < V ? z[unit * U + i] : (T)kNone;
        return r;
    };
    auto store = [&](int unit, const raw &r) { store_unit(g, unit, V, r); };

    raw v[NV ? NV : 1];
    if constexpr (NV > 0) {
#pragma unroll
        for (int u = 0; u < NV; ++u)
            if (first + u * THREADS + tid < units) v[u] = load(first + u * THREADS + tid);
    }
    // the teacher's entries, while the row is on its way: a thread each, or more
    const float inv_t = 1.0f / a.t, scale = kLog2e * inv_t;
    float top = kNone, total = 0.0f, max_u = kNone, sum_u = 0.0f;
    for (int j = tid; j < k; j += THREADS) {
        const int i = a.ids[row * k + j];
        const bool in = i >= 0 && i < V;
        const float u = in ? a.top[row * k + j] : kNone;
        id[j] = in ? i : -1;
        p[j] = u;
        zt[j] = in ? (float)z[i] : 0.0f;
        max_u = fmaxf(max_u, u);
    }
    if (g)
        for (int w = tid; w < (V + 31) / 32; w += THREADS) mark[w] = 0;
    if (tid == 0) s_twice = 0;
    if constexpr (!LSE && NV > 0) {
#pragma unroll
        for (int u = 0; u < NV; ++u)
            if (u * THREADS + tid < units) {
#pragma unroll
                for (int i = 0; i < U; ++i) top = fmaxf(top, (float)v[u][i]);
            }
    } else if constexpr (!LSE) {
#pragma unroll 2
        for (int unit = tid; unit < units; unit += THREADS) {
            const raw r = load(unit);
            float m = top;
#pragma unroll
            for (int i = 0; i < U; ++i) m = fmaxf(m, (float)r[i]);
            total *= top == m ? 1.0f : __builtin_amdgcn_exp2f((top - m) * scale);
            top = m;
            // (as long as nothing but -infinity has passed, m is no number to subtract)
#pragma unroll
            for (int i = 0; i < U; ++i) total += (float)r[i] == kNone ? 0.0f : __builtin_amdgcn_exp2f(((float)r[i] - m) * scale);
        }
    }
    const float own_top = top;
    reduce_two<kWaves>(top, max_u, part[0], pv_max{});
    // the marks are clear, and the largest of either are known
    for (int j = tid; j < k; j += THREADS) {
        if (id[j] < 0) continue;
        const float u = p[j];
        sum_u += max_u > kNone || u != u ? expf((u - max_u) * inv_t) : 0.0f;
        if (g) {
            const unsigned bit = 1u << (id[j] & 31);
            if (atomicOr(&mark[id[j] >> 5], bit) & bit) s_twice = 1;
        }
    }
    // q_v = exp2(z_v * scale - shift) / total, one operation an exponent; a rounded shift is the same in q and in the total.  What it
    // is rounded by is a power of two in both: with a shift of 4096 or more (or one that is not finite) the largest logit is
    // subtracted first.  So it is in rows that pass by: their total was, and has nothing of a rounded shift.
    const float shift = top * scale;
    const bool far = (NV == 0 && !LSE) || !(fabsf(shift) < 4096.0f);
    auto weight = [&](float x, auto is_far) {
        return __builtin_amdgcn_exp2f(decltype(is_far)::value ? (x - top) * scale : fmaf(x, scale, -shift));
    };
    if constexpr (!LSE && NV > 0) {
        auto sum = [&](auto is_far) {
#pragma unroll
            for (int u = 0; u < NV; ++u)
                if (u * THREADS + tid < units) {
#pragma unroll
                    for (int i = 0; i < U; ++i) total += weight((float)v[u][i], is_far);
                }
        };
        if (far) sum(std::true_type{});
        else sum(std::false_type{});
    } else if constexpr (!LSE) {
        total *= __builtin_amdgcn_exp2f((own_top - top) * scale);
    }
    reduce_two<kWaves>(total, sum_u, part[1], pv_add{});
    // p_j = exp((u_j - max_u) / t - log_sum_u); q_v as above, or exp(z_v / t - lse) with the sum given
    const bool any = sum_u != 0.0f;               // (of the largest entry's 1, unless there is none)
    const float log_sum_u = logf(sum_u), inv_total = 1.0f / total, lse = LSE ? a.lse_in[row] : 0.0f;
    const float factor = any ? c * a.t : 0.0f;
    auto p_of = [&](int j) { return any && id[j] >= 0 ? expf((p[j] - max_u) * inv_t - log_sum_u) : 0.0f; };
    const float factor_q = LSE ? factor : factor * inv_total;
    auto grad_q = [&](float x, auto is_far) {
        if constexpr (LSE) return factor_q * __builtin_amdgcn_exp2f(fmaf(x, inv_t, -lse) * kLog2e);
        return factor_q * weight(x, is_far);
    };
    if (g) {
        auto sweep = [&](auto is_far) {
            auto emit = [&](int unit, const raw &r) {
                raw o;
#pragma unroll
                for (int i = 0; i < U; ++i) o[i] = (T)grad_q((float)r[i], is_far);
                store(unit, o);
            };
            if constexpr (NV > 0) {
#pragma unroll
                for (int u = 0; u < NV; ++u)
                    if (first + u * THREADS + tid < units) emit(first + u * THREADS + tid, v[u]);
            } else {
                for (int unit = tid; unit < units; unit += THREADS) emit(unit, load(unit));
            }
        };
        if (factor == 0.0f) {
            const raw zero = {};
            for (int unit = first + tid; unit < units; unit += THREADS) store(unit, zero);
        } else if (!LSE && far) {
            sweep(std::true_type{});
        } else {
            sweep(std::false_type{});
        }
    }
    if constexpr (!LSE) {
        // where the rounded shift was subtracted, the total is off by what it was rounded by (6e-8 of the largest logit)
        const float log_total = logf(total) - (far ? 0.0f : fmaf(top, scale, -shift) * 0.69314718055994530942f);
        // t (ln p - ln q), whose differences of logits need no division: nothing leaves float32 at a small t, and t^2 is not formed
        float loss = 0.0f;
        for (int j = tid; j < k; j += THREADS) {
            const float pj = p_of(j);
            if (pj != 0.0f) loss = fmaf(pj, fmaf(a.t, log_total - log_sum_u, (p[j] - max_u) - (zt[j] - top)), loss);
        }
        loss = pv_block_reduce<THREADS>(loss, part[2], pv_add{});
        if (tid == 0 && a.loss) {
            a.loss[row] = any ? c * a.t * loss : 0.0f;
            if (a.lse) a.lse[row] = top * inv_t + log_total;
        }
    }
    if (!g || factor == 0.0f) return;
    // The entries' own places, once each, by the first entry of a place, over what the sweep left there: its stores are done when the
    // waves meet.
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    for (int e = tid; e < k; e += THREADS) {
        int place = id[e];
        if (place < 0) continue;
        float sum = 0.0f;
        if (s_twice) {
            for (int j = 0; j < k; ++j)
                if (id[j] == place) {
                    if (j < e) {
                        place = -1;
                        break;
                    }
                    sum += p_of(j);
                }
        } else {
            sum = p_of(e);
        }
        if (place >= first * U && place < units * U) g[place] = (T)((far ? grad_q(zt[e], std::true_type{}) : grad_q(zt[e], std::false_type{})) - factor * sum);
    }
}

// A saved sum of this size or more is off by 2^-16 and more of what it should be in q, as a float32 logarithm has no more digits, and
// of a row of one far value it has none of the vocabulary's logarithm.
constexpr float kFarSum = 256.0f;

template <class T, int THREADS, int NV, bool LSE>
__global__ __launch_bounds__(THREADS) void k_distill(const T *logits, T *grad, args a)
{
    constexpr int U = unit_of<T>::n;
    const int64_t row = LSE ? blockIdx.x / a.pieces : blockIdx.x;
    const int first = LSE ? (int)(blockIdx.x % a.pieces) * (NV * THREADS) : 0;      // unit of this block
    const T *z = logits + row * a.ld;
    T *g = grad ? grad + row * a.grad_ld : nullptr;
    const float c = a.row_weight ? a.row_weight[row] : 1.0f;
    if (c == 0.0f) {
        const int all = (a.vocab + U - 1) / U, units = LSE ? min(all, first + NV * THREADS) : all;
        const typename unit_of<T>::raw zero = {};
        if (g)
            for (int unit = first + threadIdx.x; unit < units; unit += THREADS) store_unit(g, unit, a.vocab, zero);
        if (threadIdx.x == 0 && !LSE) {
            a.loss[row] = 0.0f;
            if (a.lse) a.lse[row] = 0.0f;
        }
        return;
    }
    if constexpr (LSE) {
        if (!(fabsf(a.lse_in[row]) < kFarSum)) {
            // the row's first block forms the sum again and the gradient of all of it; no other touches the row
            if (first == 0) distill_row<T, THREADS, 0, false>(a, row, z, g, c, 0);
            return;
        }
    }
    distill_row<T, THREADS, NV, LSE>(a, row, z, g, c, first);
}

}  // namespace

pv_status pv_launch_distill(pv_ctx *ctx, int64_t rows, int64_t vocab, int k, int type, const void *logits, int64_t ld,
                            const int32_t *ids, const float *top, float temperature, const float *row_weight,
                            float *loss, float *lse, const float *lse_in, void *grad, int64_t grad_ld)
{
    args a = {ids, top, row_weight, lse_in, loss, lse, ld, grad_ld, (int)vocab, k, temperature, 1};
    const size_t lds = 3 * (size_t)k * 4 + (grad ? (size_t)((vocab + 31) / 32) * 4 : 0);
    pv_timed t(ctx, PV_K_DISTILL);
    return pv_for_dtype(type, [&](auto v) {
        using T = decltype(v);
        const int units = (int)((vocab + unit_of<T>::n - 1) / unit_of<T>::n);
        auto launch = [&](auto kernel, int threads) {
            if (lds > 65536 - 1024)
                PV_HIP(ctx, hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                                hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
            // as many rows as a launch's threads, which are counted in 32 bits, allow
            const int64_t most = ((int64_t)1 << 31) / threads / a.pieces;
            for (int64_t row = 0; row < rows; row += most) {
                args b = a;
                b.ids += row * k;
                b.top += row * k;
                for (const float **q : {&b.row_weight, &b.lse_in})
                    if (*q) *q += row;
                for (float **q : {&b.loss, &b.lse})
                    if (*q) *q += row;
                hipLaunchKernelGGL(kernel, dim3((unsigned)((rows - row < most ? rows - row : most) * a.pieces)), dim3(threads), lds, ctx->stream,
                                   static_cast<const T *>(logits) + row * ld, grad ? static_cast<T *>(grad) + row * grad_ld : nullptr, b);
                PV_HIP(ctx, hipGetLastError());
            }
            return PV_OK;
        };
        if (lse_in) {
            const int threads = units <= 256 * 4 ? 256 : 512;
            a.pieces = (unsigned)((units + threads * 4 - 1) / (threads * 4));
            return threads == 256 ? launch(k_distill<T, 256, 4, true>, 256) : launch(k_distill<T, 512, 4, true>, 512);
        }
        // few threads a row, and many rows on a compute unit, as long as they hold theirs; the loss alone holds nothing
        if (units <= 256) return launch(k_distill<T, 256, 1, false>, 256);
        if (units <= 256 * 4) return launch(k_distill<T, 256, 4, false>, 256);
        if (units <= 512 * 4) return launch(k_distill<T, 512, 4, false>, 512);
        if (units <= 512 * 8) return launch(k_distill<T, 512, 8, false>, 512);
        if (!grad) return launch(k_distill<T, 512, 0, false>, 512);
        if (units <= 1024 * 8) return launch(k_distill<T, 1024, 8, false>, 1024);
        if (units <= 1024 * 16) return launch(k_distill<T, 1024, 16, false>, 1024);
        return launch(k_distill<T, 512, 0, false>, 512);
    });
}
