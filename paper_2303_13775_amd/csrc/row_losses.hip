// Losses over rows of logits with their gradients: clipped policy loss with a KL term, preference loss of paired log ratios.
// One row: m = max z, s = sum exp(z - m), log p = (z_a - m) - log s; the gradient is slope * (1[c = a] - exp(z_c - m) / s),
// where the slope d loss / d log p is one number a row (a pair).
#include <algorithm>

#include "op_checks.h"
#include "gsplit_internal.h"

namespace {

typedef __bf16 bf16;

struct Rows {
    const void *logits; int64_t ld;
    void *grad; int64_t gld;
    const int64_t *actions;
    int64_t n; int C;
};

struct Policy {
    const float *old_logp, *ref_logp, *advantage, *weight;
    float *loss, *logp, *kl;
    float lo, hi, kl_coef, even_weight;
};

constexpr int RT = 256;

// maximum and sum over a workgroup of RT threads
__device__ __forceinline__ float wg_max(float x, float *lds) {
    for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
    for (int w = 1; w < RT / 64; ++w) x = fmaxf(x, lds[w]);
    __syncthreads();
    return x;
}
template <class T>
__device__ __forceinline__ T wg_sum(T x, T *lds) {
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
    for (int w = 1; w < RT / 64; ++w) x += lds[w];
    __syncthreads();
    return x;
}

// (base, sum of exp(z - base)) of a row: base is its maximum, 0 for a row of -inf alone, whose sum is then 0: a row that has no
// distribution.  fmaxf drops a NaN, the sum shows it.
template <class T>
__device__ __forceinline__ float2 row_stats(const T *z, int C, float *lds) {
    float m = -INFINITY;
    for (int c = threadIdx.x; c < C; c += RT) m = fmaxf(m, (float)z[c]);
    m = wg_max(m, lds);
    if (m == -INFINITY) m = 0.f;
    float s = 0.f;
    for (int c = threadIdx.x; c < C; c += RT) s += __expf((float)z[c] - m);
    return {m, wg_sum(s, lds)};
}
// log p of a row from its statistics and its action's logit, in double: a KL term is a difference of nearly equal numbers
__device__ __forceinline__ double row_logp(float2 st, float za) { return ((double)za - (double)st.x) - log((double)st.y); }

// (slope 0 where a row takes no part, or its loss does not move: no class moves it either)
template <class T>
__device__ __forceinline__ void row_gradient(const T *z, T *g, int C, float2 st, float slope, int64_t a) {
    if (slope == 0.f) {
        for (int c = threadIdx.x; c < C; c += RT) g[c] = (T)0.f;
        return;
    }
    const float scale = slope / st.y;
    for (int c = threadIdx.x; c < C; c += RT) {
        const float p = __expf((float)z[c] - st.x) * scale;
        g[c] = (T)((c == a ? slope : 0.f) - p);
    }
}

// writes loss, log p and KL term of a row, returns its slope
__device__ __forceinline__ float policy_row(const Policy &P, int64_t r, double logp, float w) {
    const double adv = P.advantage[r], ratio = exp(logp - (double)P.old_logp[r]);
    const double free_ = -adv * ratio;
    const double held = -adv * fmin(fmax(ratio, 1.0 - (double)P.lo), 1.0 + (double)P.hi);
    double loss = held, slope = 0.0, kl = 0.0;
    if (!(free_ < held)) loss = slope = free_;      // (a NaN too)
    if (P.ref_logp) {
        const double d = (double)P.ref_logp[r] - logp, e = expm1(d);
        kl = e - d;
        if (P.kl_coef > 0.f) { loss += (double)P.kl_coef * kl; slope -= (double)P.kl_coef * e; }
    }
    if (P.loss) P.loss[r] = (float)((double)w * loss);
    if (P.logp) P.logp[r] = (float)logp;
    if (P.kl) P.kl[r] = (float)kl;
    return (float)((double)w * slope);
}
__device__ __forceinline__ void policy_left_out(const Policy &P, int64_t r) {
    if (P.loss) P.loss[r] = 0.f;
    if (P.logp) P.logp[r] = 0.f;
    if (P.kl) P.kl[r] = 0.f;
}

template <class T>
__global__ __launch_bounds__(RT) void k_policy_rows(Rows R, Policy P) {
    __shared__ float lds[RT / 64];
    __shared__ float lds_slope;
    for (int64_t r = blockIdx.x; r < R.n; r += gridDim.x) {
        const T *z = (const T *)R.logits + r * R.ld;
        const float w = P.weight ? P.weight[r] : P.even_weight;
        const int64_t a = R.actions[r];
        bool used = w != 0.f && a >= 0 && a < R.C;
        float2 st{0.f, 0.f};
        float za = 0.f;
        if (used) {
            za = (float)z[a];
            st = row_stats(z, R.C, lds);
            used = st.y != 0.f;
        }
        if (threadIdx.x == 0) {
            lds_slope = 0.f;
            if (used) lds_slope = policy_row(P, r, row_logp(st, za), w);
            else policy_left_out(P, r);
        }
        __syncthreads();
        if (R.grad) row_gradient(z, (T *)R.grad + r * R.gld, R.C, st, lds_slope, a);
        __syncthreads();
    }
}

struct Pairs {
    const int64_t *seq_ptr; int64_t n;
    const float *ref_logp, *weight;
    float *row_logp, *loss, *margin;
    float4 *work;               // a row: base, sum, log p (double); the pairs put the row's slope in its place
    float beta, smoothing, even_weight;
};

// offsets kept inside the buffers, whatever they hold
__device__ __forceinline__ int64_t seq_at(const Pairs &Q, int64_t q, int64_t n_rows) {
    return min(max(Q.seq_ptr[q], (int64_t)0), n_rows);
}

template <class T>
__global__ __launch_bounds__(RT) void k_preference_rows(Rows R, Pairs Q) {
    __shared__ float lds[RT / 64];
    const int64_t first = seq_at(Q, 0, R.n), last = seq_at(Q, 2 * Q.n, R.n);
    for (int64_t r = first + blockIdx.x; r < last; r += gridDim.x) {
        const T *z = (const T *)R.logits + r * R.ld;
        const int64_t a = R.actions[r];
        float2 st{0.f, 0.f};
        double logp = 0.0;
        if (a >= 0 && a < R.C) {
            const float za = (float)z[a];
            st = row_stats(z, R.C, lds);
            if (st.y != 0.f) logp = row_logp(st, za);
        }
        if (threadIdx.x == 0) {
            const float2 bits = __builtin_bit_cast(float2, logp);
            Q.work[r] = {st.x, st.y, bits.x, bits.y};
            if (Q.row_logp) Q.row_logp[r] = (float)logp;
        }
    }
}

__global__ __launch_bounds__(RT) void k_preference_pairs(Rows R, Pairs Q) {
    __shared__ double lds[RT / 64];
    for (int64_t p = blockIdx.x; p < Q.n; p += gridDim.x) {
        double sum[2];
        for (int k = 0; k < 2; ++k) {
            double x = 0.0;
            const int64_t end = seq_at(Q, 2 * p + k + 1, R.n);
            for (int64_t r = seq_at(Q, 2 * p + k, R.n) + threadIdx.x; r < end; r += RT)
                x += __builtin_bit_cast(double, make_float2(Q.work[r].z, Q.work[r].w));
            sum[k] = wg_sum(x, lds) - (Q.ref_logp ? (double)Q.ref_logp[2 * p + k] : 0.0);
        }
        const double h = (double)Q.beta * (sum[0] - sum[1]), e = Q.smoothing;
        const double w = Q.weight ? Q.weight[p] : Q.even_weight;
        const double soft = log1p(exp(-fabs(h)));
        if (threadIdx.x == 0) {
            if (Q.margin) Q.margin[p] = (float)h;
            if (Q.loss) Q.loss[p] = w == 0.0 ? 0.f : (float)(w * ((1.0 - e) * (soft + fmax(-h, 0.0)) + e * (soft + fmax(h, 0.0))));
        }
        // d loss / d margin = w (e - sigmoid(-margin))
        const float slope = w == 0.0 ? 0.f : (float)((double)Q.beta * w * (e - 1.0 / (1.0 + exp(h))));
        if (R.grad)
            for (int k = 0; k < 2; ++k) {
                const int64_t end = seq_at(Q, 2 * p + k + 1, R.n);
                for (int64_t r = seq_at(Q, 2 * p + k, R.n) + threadIdx.x; r < end; r += RT)
                    Q.work[r].z = Q.work[r].y == 0.f ? 0.f : k ? -slope : slope;
            }
    }
}

template <class T>
__global__ __launch_bounds__(RT) void k_preference_grad(Rows R, Pairs Q) {
    const int64_t first = seq_at(Q, 0, R.n), last = seq_at(Q, 2 * Q.n, R.n);
    for (int64_t r = first + blockIdx.x; r < last; r += gridDim.x) {
        const float4 k = Q.work[r];
        row_gradient((const T *)R.logits + r * R.ld, (T *)R.grad + r * R.gld, R.C, {k.x, k.y}, k.z, R.actions[r]);
    }
}

unsigned row_grid(const gsplit_ctx *ctx, int64_t n) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((int64_t)ctx->n_cu * 8, n)); }

}  // namespace

extern "C" int gsplit_policy_loss(gsplit_ctx *ctx, const gsplit_policy_config *c, const void *d_logits, int64_t n_rows,
                                  int32_t n_classes, int64_t logits_stride, const int64_t *d_actions, const float *d_old_logp,
                                  const float *d_ref_logp, const float *d_advantages, const float *d_row_weight,
                                  void *d_grad_logits, int64_t grad_stride, float *d_row_loss, float *d_row_logp,
                                  float *d_row_kl, void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        if (const char *e = op_check_policy(c, d_logits, n_rows, n_classes, logits_stride, d_actions, d_old_logp, d_ref_logp,
                                            d_advantages, d_row_weight, d_grad_logits, grad_stride, d_row_loss, d_row_logp, d_row_kl))
            return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_policy_loss: ") + e);
        if (n_rows == 0) return GSPLIT_OK;
        const Rows R{d_logits, logits_stride, d_grad_logits, grad_stride, d_actions, n_rows, n_classes};
        const Policy P{d_old_logp, d_ref_logp, d_advantages, d_row_weight, d_row_loss, d_row_logp, d_row_kl,
                       c->clip_low, c->clip_high, c->kl_coef, (float)(1.0 / (double)n_rows)};
        GsTimeScope ts(ctx, "policy_loss", -1, st);
        if (c->dtype == GSPLIT_F32) hipLaunchKernelGGL(k_policy_rows<float>, dim3(row_grid(ctx, n_rows)), dim3(RT), 0, st, R, P);
        else hipLaunchKernelGGL(k_policy_rows<bf16>, dim3(row_grid(ctx, n_rows)), dim3(RT), 0, st, R, P);
        return GSPLIT_OK;
    });
}

extern "C" int gsplit_preference_loss(gsplit_ctx *ctx, const gsplit_preference_config *c, const void *d_logits, int64_t n_rows,
                                      int32_t n_classes, int64_t logits_stride, const int64_t *d_actions,
                                      const int64_t *d_seq_ptr, int64_t n_pairs, const float *d_ref_logp,
                                      const float *d_pair_weight, void *d_grad_logits, int64_t grad_stride, float *d_row_logp,
                                      float *d_pair_loss, float *d_pair_margin, float *d_row_work, void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        if (const char *e = op_check_preference(c, d_logits, n_rows, n_classes, logits_stride, d_actions, d_seq_ptr, n_pairs,
                                                d_ref_logp, d_pair_weight, d_grad_logits, grad_stride, d_row_logp, d_pair_loss,
                                                d_pair_margin, d_row_work))
            return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_preference_loss: ") + e);
        if (n_pairs == 0) return GSPLIT_OK;
        const Rows R{d_logits, logits_stride, d_grad_logits, grad_stride, d_actions, n_rows, n_classes};
        const Pairs Q{d_seq_ptr, n_pairs, d_ref_logp, d_pair_weight, d_row_logp, d_pair_loss, d_pair_margin,
                      (float4 *)d_row_work, c->beta, c->label_smoothing, (float)(1.0 / (double)n_pairs)};
        const dim3 rows(row_grid(ctx, n_rows)), block(RT);
        const bool f32 = c->dtype == GSPLIT_F32;
        if (n_rows > 0) {
            GsTimeScope ts(ctx, "preference_rows", -1, st);
            if (f32) hipLaunchKernelGGL(k_preference_rows<float>, rows, block, 0, st, R, Q);
            else hipLaunchKernelGGL(k_preference_rows<bf16>, rows, block, 0, st, R, Q);
        }
        {
            GsTimeScope ts(ctx, "preference_pairs", -1, st);
            hipLaunchKernelGGL(k_preference_pairs, dim3(row_grid(ctx, n_pairs)), block, 0, st, R, Q);
        }
        if (n_rows > 0 && d_grad_logits) {
            GsTimeScope ts(ctx, "preference_grad", -1, st);
            if (f32) hipLaunchKernelGGL(k_preference_grad<float>, rows, block, 0, st, R, Q);
            else hipLaunchKernelGGL(k_preference_grad<bf16>, rows, block, 0, st, R, Q);
        }
        return GSPLIT_OK;
    });
}
