// Distillation from a teacher's k largest logits: loss, and the gradient of the student's logits.
//   p = softmax_j(u_j / t) over the teacher's entries, q = softmax_v(z_v / t) over the vocabulary
//   loss = c t^2 sum_j p_j (ln p_j - ln q[id_j]),   grad_v = c t (q_v - sum_{j: id_j = v} p_j)
// Bound by HBM: the logits in, the gradient out, 2 or 4 bytes an entry each.  A block takes a row, and the
// row stays in its registers between the sum and the gradient where they hold it; the exponentials are formed twice
// instead of being kept, at 16 a clock and compute unit they cost a fraction of the bytes.
// The teacher's entries are k places of the row: a bit per place marks them in LDS, the sweep that writes the gradient
// leaves marked places out, and the first entry of each id writes its place, less the sum of the entries with that id
// in the order of the list - one writer a place, no atomics on sums, and the same bits every time.
#include "pv_ops.h"

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2e = 1.44269504088896340736f;

template <class T>
struct unit_of {                                  // 16 bytes of a row, at any element's address
    static constexpr int n = 16 / sizeof(T);
    typedef T raw __attribute__((ext_vector_type(n)));
    typedef raw type __attribute__((aligned(sizeof(T))));
};

struct args {
    const int32_t *ids;
    const float *top, *row_weight, *lse_in;
    float *loss, *lse;
    int64_t ld, grad_ld;
    int vocab, k;
    float t;
};

// NV > 0: the row lies in NV units a thread.  NV == 0: the row is read again for the gradient.
// LSE: the sum is given (the backward call), only the gradient is formed.
template <class T, int NV, bool LSE>
__global__ __launch_bounds__(kThreads) void k_distill(const T *logits, T *grad, args a)
{
    constexpr int U = unit_of<T>::n;
    typedef typename unit_of<T>::raw raw;
    typedef typename unit_of<T>::type loose;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    float *part = reinterpret_cast<float *>(lds);                     // [2][kWaves]
    float *p = part + 2 * kWaves;                                     // [k] the teacher's probabilities
    float *zt = p + a.k;                                              // [k] the logits in their places
    int *id = reinterpret_cast<int *>(zt + a.k);                      // [k] their places, -1: none
    unsigned *mark = reinterpret_cast<unsigned *>(id + a.k);          // [ceil(vocab / 32)] places of the row

    __shared__ int twice;                                             // some place has two entries
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, V = a.vocab, k = a.k;
    const T *z = logits + row * a.ld;
    T *g = grad ? grad + row * a.grad_ld : nullptr;
    const float c = a.row_weight ? a.row_weight[row] : 1.0f;
    const int units = (V + U - 1) / U;

    auto load = [&](int unit) {
        raw r;
        if ((unit + 1) * U <= V) return (raw)*reinterpret_cast<const loose *>(z + unit * U);
#pragma unroll
        for (int i = 0; i < U; ++i) r[i] = unit * U + i < V ? z[unit * U + i] : (T)(-__builtin_inff());
        return r;
    };
    auto store = [&](int unit, const raw &r, unsigned skip) {
        if (skip == 0 && (unit + 1) * U <= V) {
            *reinterpret_cast<loose *>(g + unit * U) = r;
            return;
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (unit * U + i < V && !(skip >> i & 1)) g[unit * U + i] = r[i];
    };

    if (c == 0.0f) {
        const raw zero = {};
        if (g)
            for (int unit = tid; unit < units; unit += kThreads) store(unit, zero, 0);
        if (tid == 0 && !LSE) {
            a.loss[row] = 0.0f;
            if (a.lse) a.lse[row] = 0.0f;
        }
        return;
    }

    raw v[NV ? NV : 1];
    if constexpr (NV > 0) {
#pragma unroll
        for (int u = 0; u < NV; ++u)
            if (u * kThreads + tid < units) v[u] = load(u * kThreads + tid);
    }
    // the teacher's entries, while the row is on its way: the first wave forms their softmax
    const float inv_t = 1.0f / a.t;
    float log_sum_u = 0.0f, max_u = -__builtin_inff();
    if (g)
        for (int w = tid; w < (V + 31) / 32; w += kThreads) mark[w] = 0;
    if (tid == 0) twice = 0;
    if (tid < 64) {
        for (int j = tid; j < k; j += 64) {
            const int i = a.ids[row * k + j];
            const bool in = i >= 0 && i < V;
            const float u = in ? a.top[row * k + j] * inv_t : -__builtin_inff();
            id[j] = in ? i : -1;
            p[j] = u;
            zt[j] = in ? (float)z[i] : 0.0f;
            max_u = fmaxf(max_u, u);
        }
        max_u = pv_wave_reduce(max_u, pv_max{});
        float sum = 0.0f;
        for (int j = tid; j < k; j += 64) sum += id[j] >= 0 && max_u > -__builtin_inff() ? expf(p[j] - max_u) : 0.0f;
        sum = pv_wave_reduce(sum, pv_add{});
        log_sum_u = logf(sum);                    // -inf: no entry
    }

    // q_v = exp2(z_v * scale - shift)
    const float scale = kLog2e * inv_t;
    float top = -__builtin_inff(), lse, total = 0.0f;
    if constexpr (LSE) {
        lse = a.lse_in[row];
        __syncthreads();          // the marks are clear
    } else {
        auto largest = [&](const raw &r) {
#pragma unroll
            for (int i = 0; i < U; ++i) top = fmaxf(top, (float)r[i]);
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int u = 0; u < NV; ++u)
                if (u * kThreads + tid < units) largest(v[u]);
        } else {
            for (int unit = tid; unit < units; unit += kThreads) largest(load(unit));
        }
        top = pv_block_reduce<kThreads>(top, part, pv_max{});
        auto add = [&](const raw &r, int unit) {
#pragma unroll
            for (int i = 0; i < U; ++i) total += __builtin_amdgcn_exp2f(((float)r[i] - top) * scale);
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int u = 0; u < NV; ++u)
                if (u * kThreads + tid < units) add(v[u], u * kThreads + tid);
        } else {
            for (int unit = tid; unit < units; unit += kThreads) add(load(unit), unit);
        }
        total = pv_block_reduce<kThreads>(total, part + kWaves, pv_add{});
        lse = top * inv_t + logf(total);
    }

    // the loss, and the entries' probabilities in place of their logits
    if (tid < 64) {
        const bool any = log_sum_u != -__builtin_inff();
        float loss = 0.0f;
        for (int j = tid; j < k; j += 64) {
            const float log_p = p[j] - max_u - log_sum_u;
            const float pj = any && id[j] >= 0 ? expf(log_p) : 0.0f;
            if (!LSE && pj != 0.0f) {
                const float log_q = (zt[j] - top) * inv_t - logf(total);
                loss = fmaf(pj, log_p - log_q, loss);
            }
            p[j] = pj;
            if (g && pj != 0.0f) {
                const unsigned bit = 1u << (id[j] & 31);
                if (atomicOr(&mark[id[j] >> 5], bit) & bit) twice = 1;
            }
        }
        if constexpr (!LSE) {
            loss = pv_wave_reduce(loss, pv_add{});
            if (tid == 0) {
                a.loss[row] = any ? c * a.t * a.t * loss : 0.0f;
                if (a.lse) a.lse[row] = lse;
            }
        }
        if (tid == 0) part[0] = any ? c * a.t : 0.0f;
    }
    if (!g) return;
    __syncthreads();
    const float factor = part[0], inv_total = 1.0f / total;

    auto q_of = [&](float x) {
        // forward: relative to the largest, as the sum was taken; backward: from the log of the sum
        if constexpr (LSE) return __builtin_amdgcn_exp2f(fmaf(x, inv_t, -lse) * kLog2e);
        return __builtin_amdgcn_exp2f((x - top) * scale) * inv_total;
    };
    // the entries' own places, once each
    if (tid < k && p[tid] != 0.0f) {
        int place = id[tid];
        float sum = p[tid];
        if (twice) {
            sum = 0.0f;
            for (int j = 0; j < k; ++j)
                if (id[j] == place && p[j] != 0.0f) {
                    if (j < tid) {
                        place = -1;
                        break;
                    }
                    sum += p[j];
                }
        }
        if (place >= 0) g[place] = (T)(factor * (q_of(zt[tid]) - sum));
    }
    auto emit = [&](int unit, raw r) {
        const unsigned word = mark[unit * U >> 5] >> (unit * U & 31) & ((1u << U) - 1);
#pragma unroll
        for (int i = 0; i < U; ++i) r[i] = factor != 0.0f ? (T)(factor * q_of((float)r[i])) : (T)0.0f;
        store(unit, r, word);
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int u = 0; u < NV; ++u)
            if (u * kThreads + tid < units) emit(u * kThreads + tid, v[u]);
    } else {
        // a place that an entry has written already (grad may be logits) is read and left out
        for (int unit = tid; unit < units; unit += kThreads) emit(unit, load(unit));
    }
}

}  // namespace

pv_status pv_launch_distill(pv_ctx *ctx, int64_t rows, int64_t vocab, int k, int type, const void *logits, int64_t ld,
                            const int32_t *ids, const float *top, float temperature, const float *row_weight,
                            float *loss, float *lse, const float *lse_in, void *grad, int64_t grad_ld)
{
    const args a = {ids, top, row_weight, lse_in, loss, lse, ld, grad_ld, (int)vocab, k, temperature};
    const size_t lds = (2 * kWaves + 3 * (size_t)k) * 4 + (grad ? (size_t)((vocab + 31) / 32) * 4 : 0);
    pv_timed t(ctx, PV_K_DISTILL);
    return pv_for_dtype(type, [&](auto v) {
        using T = decltype(v);
        const int units = (int)((vocab + unit_of<T>::n - 1) / unit_of<T>::n), nv = (units + kThreads - 1) / kThreads;
        auto launch = [&](auto kernel) {
            if (lds > 65536)
                PV_HIP(ctx, hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                                hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
            hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(kThreads), lds, ctx->stream,
                               static_cast<const T *>(logits), static_cast<T *>(grad), a);
            PV_HIP(ctx, hipGetLastError());
            return PV_OK;
        };
        auto pick = [&](auto given) {
            constexpr bool LSE = decltype(given)::value;
            if (nv <= 1) return launch(k_distill<T, 1, LSE>);
            if (nv <= 2) return launch(k_distill<T, 2, LSE>);
            if (nv <= 4) return launch(k_distill<T, 4, LSE>);
            if (nv <= 8) return launch(k_distill<T, 8, LSE>);
            if (nv <= 16) return launch(k_distill<T, 16, LSE>);
            return launch(k_distill<T, 0, LSE>);
        };
        return lse_in ? pick(std::true_type{}) : pick(std::false_type{});
    });
}
