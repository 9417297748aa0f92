// Losses over rows of logits with their gradients: clipped policy loss with a KL term, preference loss of paired log ratios.
// One row: m = max z, s = sum exp(z - m), log p = (z_a - m) - log s; the gradient is slope * (1[c = a] - exp(z_c - m) / s),
// where the slope d loss / d log p is one number a row (a pair).
#include <algorithm>
#include <cmath>

#include "op_checks.h"
#include "gsplit_internal.h"
#include "row_pieces.h"
#include "row_rules.h"

namespace {

struct Rows {
    const void *logits; int64_t ld;
    void *grad; int64_t gld;
    const int64_t *actions;
    int64_t n; int C;
    int64_t first = 0;          // row of the launch's first team
};

struct Policy {
    const float *old_logp, *ref_logp, *advantage, *weight;
    float *loss, *logp, *kl;
    double log_lo, log_hi;      // logarithms of the clip's borders: a ratio's side is decided in double
    float lo, hi, kl_coef, even_weight;
};

// log p of a row from its statistics and its action's logit, in double: a KL term is a difference of nearly equal numbers
__device__ __forceinline__ double row_logp(RowStats st, float za) { return ((double)za - (double)base_of(st.m)) - log((double)st.s); }

// e^x - 1 - x without the cancellation near 0: its series up to |x| = 1 (the first term left out is 4e-9 of the value)
__device__ __forceinline__ float exp_above_tangent(float x) {
    if (fabsf(x) > 1.f) return (expf(x) - 1.f) - x;
    float y = 1.f / 39916800.f;
    const float c[] = {1.f / 3628800.f, 1.f / 362880.f, 1.f / 40320.f, 1.f / 5040.f, 1.f / 720.f, 1.f / 120.f, 1.f / 24.f, 1.f / 6.f, 0.5f};
    for (float k : c) y = fmaf(y, x, k);
    return x * x * y;
}

// Slope, and through *loss and *kl the loss and the KL term, of one row.  Differences of log-probabilities are formed in double and
// rounded once; what follows from them is float.
__device__ __forceinline__ float policy_row(const Policy &P, double logp, float old_logp, float ref_logp, float adv, float w, float *loss, float *kl) {
    const double d = logp - (double)old_logp;
    // an advantage above 0 gains nothing from a ratio over the upper border, one below 0 nothing from one under the lower
    const bool held = adv >= 0.f ? d > P.log_hi : d < P.log_lo;
    const float ratio = adv == 0.f ? (float)d : expf((float)d);     // (no advantage: 0 times any ratio, NaN stays)
    float l = -adv * (held ? (adv >= 0.f ? P.hi : P.lo) : ratio), slope = held ? 0.f : l;
    *kl = 0.f;
    if (P.ref_logp) {
        const float x = (float)((double)ref_logp - logp);
        *kl = exp_above_tangent(x);
        if (P.kl_coef > 0.f) { l += P.kl_coef * *kl; slope -= P.kl_coef * (*kl + x); }
    }
    *loss = w * l;
    return w * slope;
}

// Lanes LANES of a team take a row each time.  LANES <= 64: several teams a wave, all lanes form the row's numbers alike; else the
// team is the workgroup, and its first wave does.
template <class T, int THREADS, int LANES, int E>
__global__ __launch_bounds__(THREADS) void k_policy_rows(Rows R, Policy P) {
    constexpr bool WG = LANES > 64;
    constexpr bool HELD = E > 0;
    __shared__ RowStats lds[WG ? THREADS / 64 : 1];
    __shared__ float lds_slope;
    const int lane = WG ? threadIdx.x : threadIdx.x % LANES;
    constexpr int TEAMS = THREADS / LANES;
    // (no loop over rows: the compiler keeps what a loop needs in registers that the row is to have)
    const int64_t r = R.first + (int64_t)blockIdx.x * TEAMS + (WG ? 0 : threadIdx.x / LANES);
    if (r < R.n) {
        const T *z = (const T *)R.logits + r * R.ld;
        T *g = R.grad ? (T *)R.grad + r * R.gld : nullptr;
        const float w = P.weight ? P.weight[r] : P.even_weight;
        const int64_t a = R.actions[r];
        RowStats st{-INFINITY, 0.f};
        float za = 0.f, slope = 0.f;
        HeldRow<T, LANES, HELD ? E : PIECE<T>> row;
        if (w != 0.f && a >= 0 && a < R.C) {
            za = (float)z[a];
            if constexpr (HELD) { row.load(z, R.C, lane); st = row.stats(); }
            else st = StreamedRow<T, LANES, -E>::stats(z, R.C, lane);
            if constexpr (WG) st = join_waves<LANES>(st, lds);
            else st = join_lanes<LANES>(st);
        }
        if (!WG || threadIdx.x < 64) {
            float loss = 0.f, kl = 0.f, logp = 0.f;
            if (st.s != 0.f) {      // 0: the row is left out
                const double lp = row_logp(st, za);
                logp = (float)lp;
                slope = policy_row(P, lp, P.old_logp[r], P.ref_logp ? P.ref_logp[r] : 0.f, P.advantage[r], w, &loss, &kl);
            }
            if (lane == 0) {
                if (P.loss) P.loss[r] = loss;
                if (P.logp) P.logp[r] = logp;
                if (P.kl) P.kl[r] = kl;
            }
        }
        if constexpr (WG) {
            if (threadIdx.x == 0) lds_slope = slope;
            __syncthreads();
            slope = lds_slope;
        }
        if (g) {
            if (slope == 0.f) store_zeros<T, LANES>(g, R.C, lane);      // nothing moves it
            else if constexpr (HELD) row.store(g, R.C, lane, st, slope, (int)a, za);
            else StreamedRow<T, LANES, -E>::store(z, g, R.C, lane, st, slope, (int)a, za);
        }
    }
}

struct Pairs {
    const int64_t *seq_ptr; int64_t n;
    const float *ref_logp, *weight;
    float *row_logp, *loss, *margin;
    float4 *work;               // a row: maximum, sum, log p (double); the pairs put the row's slope in its place
    float beta, smoothing, even_weight;
};

// offsets kept inside the buffers, whatever they hold
__device__ __forceinline__ int64_t seq_at(const Pairs &Q, int64_t q, int64_t n_rows) {
    return min(max(Q.seq_ptr[q], (int64_t)0), n_rows);
}

// Statistics and log p of row r into its place in the working memory, by a team of LANES lanes; returns log p (0: left out)
template <class T, int LANES, int E>
__device__ __forceinline__ double preference_row(const Rows &R, const Pairs &Q, int64_t r, int lane, RowStats *lds) {
    const T *z = (const T *)R.logits + r * R.ld;
    const int64_t a = R.actions[r];
    RowStats st{-INFINITY, 0.f};
    float za = 0.f;
    if (a >= 0 && a < R.C) {
        za = (float)z[a];
        st = StreamedRow<T, LANES, E>::stats(z, R.C, lane);
        if constexpr (LANES > 64) { st = join_waves<LANES>(st, lds); __syncthreads(); }
        else st = join_lanes<LANES>(st);
    }
    const double logp = st.s != 0.f ? row_logp(st, za) : 0.0;
    if (lane == 0) {
        const float2 bits = __builtin_bit_cast(float2, logp);
        Q.work[r] = {st.m, st.s, bits.x, bits.y};
        if (Q.row_logp) Q.row_logp[r] = (float)logp;
    }
    return logp;
}
template <class T, int LANES, int E>
__device__ __forceinline__ void preference_row_grad(const Rows &R, int64_t r, int lane, RowStats st, float slope) {
    const T *z = (const T *)R.logits + r * R.ld;
    T *g = (T *)R.grad + r * R.gld;
    if (slope == 0.f) store_zeros<T, LANES>(g, R.C, lane);
    else {
        const int64_t a = R.actions[r];
        StreamedRow<T, LANES, E>::store(z, g, R.C, lane, st, slope, (int)a, (float)z[a]);
    }
}

// Writes loss and margin of a pair from the difference of its log ratios (first thread), returns d loss / d log p of its chosen rows
__device__ __forceinline__ float pair_row(const Pairs &Q, int64_t p, double ratio_gap) {
    const double h = (double)Q.beta * ratio_gap, e = Q.smoothing;
    const double w = Q.weight ? Q.weight[p] : Q.even_weight;
    if (threadIdx.x == 0) {
        const double soft = log1p(exp(-fabs(h)));
        if (Q.margin) Q.margin[p] = (float)h;
        if (Q.loss) Q.loss[p] = w == 0.0 ? 0.f : (float)(w * ((1.0 - e) * (soft + fmax(-h, 0.0)) + e * (soft + fmax(h, 0.0))));
    }
    // d loss / d margin = w (e - sigmoid(-margin))
    return w == 0.0 ? 0.f : (float)((double)Q.beta * w * (e - 1.0 / (1.0 + exp(h))));
}
__device__ __forceinline__ double reference_gap(const Pairs &Q, int64_t p) {
    return Q.ref_logp ? (double)Q.ref_logp[2 * p] - (double)Q.ref_logp[2 * p + 1] : 0.0;
}

// the rows of a pair, the chosen sequence's and then the rejected one's
struct PairRows {
    int64_t b0, n0, b1, n;
    __device__ __forceinline__ PairRows(const Pairs &Q, int64_t p, int64_t n_rows) {
        b0 = seq_at(Q, 2 * p, n_rows);
        b1 = seq_at(Q, 2 * p + 1, n_rows);
        n0 = max(b1 - b0, (int64_t)0);
        n = n0 + max(seq_at(Q, 2 * p + 2, n_rows) - b1, (int64_t)0);
    }
    __device__ __forceinline__ int64_t row(int64_t i) const { return i < n0 ? b0 + i : b1 + (i - n0); }
};

template <int THREADS>
__device__ __forceinline__ double wg_sum(double x, double *lds) {
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = lds[0];
        for (int w = 1; w < THREADS / 64; ++w) x += lds[w];
        __syncthreads();
    }
    return x;
}

// A pair from its rows' statistics to their gradient by one workgroup, THREADS / LANES rows at a time; the second reading of the
// rows comes from the caches.
template <class T, int THREADS, int LANES, int E>
__global__ __launch_bounds__(THREADS) void k_preference_whole(Rows R, Pairs Q) {
    __shared__ RowStats lds[LANES > 64 ? THREADS / 64 : 1];
    __shared__ double lds_sum[THREADS / 64];
    constexpr int TEAMS = THREADS / LANES;
    const int lane = LANES > 64 ? threadIdx.x : threadIdx.x % LANES, team = LANES > 64 ? 0 : threadIdx.x / LANES;
    const PairRows P(Q, blockIdx.x, R.n);
    double gap = 0.0;
    for (int64_t i = team; i < P.n; i += TEAMS) {
        const double logp = preference_row<T, LANES, E>(R, Q, P.row(i), lane, lds);
        if (lane == 0) gap += i < P.n0 ? logp : -logp;
    }
    gap = wg_sum<THREADS>(gap, lds_sum) - reference_gap(Q, blockIdx.x);
    const float slope = pair_row(Q, blockIdx.x, gap);
    if (!R.grad) return;
    __syncthreads();        // (the working memory of a row is written by its team's first lane)
    for (int64_t i = team; i < P.n; i += TEAMS) {
        const int64_t r = P.row(i);
        const float4 k = Q.work[r];
        preference_row_grad<T, LANES, E>(R, r, lane, {k.x, k.y}, k.y == 0.f ? 0.f : i < P.n0 ? slope : -slope);
    }
}

// The same as three launches, for pairs too few or too long for a workgroup each: all rows, all pairs, all rows again
template <class T, int THREADS, int LANES, int E>
__global__ __launch_bounds__(THREADS) void k_preference_rows(Rows R, Pairs Q) {
    __shared__ RowStats lds[LANES > 64 ? THREADS / 64 : 1];
    constexpr int TEAMS = THREADS / LANES;
    const int64_t first = seq_at(Q, 0, R.n), last = seq_at(Q, 2 * Q.n, R.n);
    for (int64_t r = first + (int64_t)blockIdx.x * TEAMS + (LANES > 64 ? 0 : threadIdx.x / LANES); r < last; r += (int64_t)gridDim.x * TEAMS)
        preference_row<T, LANES, E>(R, Q, r, threadIdx.x % LANES, lds);
}

constexpr int PT = 256;
__global__ __launch_bounds__(PT) void k_preference_pairs(Rows R, Pairs Q) {
    __shared__ double lds[PT / 64];
    for (int64_t p = blockIdx.x; p < Q.n; p += gridDim.x) {
        const PairRows P(Q, p, R.n);
        double gap = 0.0;
        for (int64_t i = threadIdx.x; i < P.n; i += PT) {
            const float4 k = Q.work[P.row(i)];
            const double logp = __builtin_bit_cast(double, make_float2(k.z, k.w));
            gap += i < P.n0 ? logp : -logp;
        }
        gap = wg_sum<PT>(gap, lds) - reference_gap(Q, p);
        const float slope = pair_row(Q, p, gap);
        if (!R.grad) continue;
        for (int64_t i = threadIdx.x; i < P.n; i += PT) {
            float4 &k = Q.work[P.row(i)];
            k.z = k.y == 0.f ? 0.f : i < P.n0 ? slope : -slope;
        }
    }
}

template <class T, int THREADS, int LANES, int E>
__global__ __launch_bounds__(THREADS) void k_preference_grad(Rows R, Pairs Q) {
    constexpr int TEAMS = THREADS / LANES;
    const int lane = LANES > 64 ? threadIdx.x : threadIdx.x % LANES;
    const int64_t first = seq_at(Q, 0, R.n), last = seq_at(Q, 2 * Q.n, R.n);
    // the last rows first: they are the ones that the pass before has left in the caches
    for (int64_t r = last - 1 - (int64_t)blockIdx.x * TEAMS - (LANES > 64 ? 0 : threadIdx.x / LANES); r >= first; r -= (int64_t)gridDim.x * TEAMS) {
        const float4 k = Q.work[r];
        preference_row_grad<T, LANES, E>(R, r, lane, {k.x, k.y}, k.z);
    }
}

unsigned row_grid(int64_t n, int teams, int64_t most) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(most, gs_ceil_div(n, teams))); }

template <int N> struct Int { static constexpr int value = N; };

// calls f(threads, lanes, elements a lane) with the constants of the form; -elements: streamed
template <class F>
void with_form(int form, F f) {
    switch (form) {
        case ROW_16x8: f(Int<256>{}, Int<16>{}, Int<8>{}); break;
        case ROW_16x16: f(Int<256>{}, Int<16>{}, Int<16>{}); break;
        case ROW_64x8: f(Int<256>{}, Int<64>{}, Int<8>{}); break;
        case ROW_64x16: f(Int<256>{}, Int<64>{}, Int<16>{}); break;
        case ROW_256x8: f(Int<256>{}, Int<256>{}, Int<8>{}); break;
        case ROW_256x16: f(Int<256>{}, Int<256>{}, Int<16>{}); break;
        case ROW_256x32: f(Int<256>{}, Int<256>{}, Int<32>{}); break;
        case ROW_512x32: f(Int<512>{}, Int<512>{}, Int<32>{}); break;
        case ROW_512x64: f(Int<512>{}, Int<512>{}, Int<64>{}); break;
        case ROW_1024x64: f(Int<1024>{}, Int<1024>{}, Int<64>{}); break;
        default: f(Int<1024>{}, Int<1024>{}, Int<-32>{}); break;
    }
}

// the same for kernels that stream rows: 16, 64 or 256 lanes a row, in workgroups of 64 or 256 threads
template <class F>
void with_part(int dtype, int lanes, int threads, F f) {
    const auto typed = [&](auto type) {
        if (lanes == 16 && threads == 64) f(type, Int<64>{}, Int<16>{}, Int<16>{});
        else if (lanes == 16) f(type, Int<256>{}, Int<16>{}, Int<16>{});
        else if (lanes == 64 && threads == 64) f(type, Int<64>{}, Int<64>{}, Int<16>{});
        else if (lanes == 64) f(type, Int<256>{}, Int<64>{}, Int<16>{});
        else f(type, Int<256>{}, Int<256>{}, Int<32>{});
    };
    if (dtype == GSPLIT_F32) typed(float{});
    else typed(bf16{});
}

template <class T>
void launch_policy(Rows R, const Policy &P, hipStream_t st) {
    with_form(row_form(R.C, PIECE<T>), [&](auto threads, auto lanes, auto e) {
        constexpr int TH = decltype(threads)::value, LA = decltype(lanes)::value, E = decltype(e)::value;
        constexpr int64_t MOST = 1 << 21;       // workgroups of a launch: it has less than 2^32 threads
        for (; R.first < R.n; R.first += MOST * (TH / LA))
            hipLaunchKernelGGL((k_policy_rows<T, TH, LA, E>), dim3(row_grid(R.n - R.first, TH / LA, MOST)), dim3(TH), 0, st, R, P);
    });
}

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
                       std::log(1.0 - (double)c->clip_low), std::log1p((double)c->clip_high), (float)(1.0 - (double)c->clip_low),
                       (float)(1.0 + (double)c->clip_high), c->kl_coef, (float)(1.0 / (double)n_rows)};
        GsTimeScope ts(ctx, "policy_loss", -1, st);
        if (c->dtype == GSPLIT_F32) launch_policy<float>(R, P, st);
        else launch_policy<bf16>(R, P, st);
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
        const int64_t most = (int64_t)ctx->n_cu * 32;
        const int whole = n_rows > 0 ? preference_whole(n_rows, n_pairs, (int64_t)n_classes * op_elem_size(c->dtype), ctx->n_cu) : 0;
        if (whole) {
            GsTimeScope ts(ctx, "preference_loss", -1, st);
            with_part(c->dtype, row_part(n_classes), whole, [&](auto type, auto threads, auto lanes, auto e) {
                using T = decltype(type);
                constexpr int TH = decltype(threads)::value, LA = decltype(lanes)::value, E = decltype(e)::value;
                hipLaunchKernelGGL((k_preference_whole<T, TH, LA, E>), dim3((unsigned)n_pairs), dim3(TH), 0, st, R, Q);
            });
            return GSPLIT_OK;
        }
        if (n_rows > 0) {
            GsTimeScope ts(ctx, "preference_rows", -1, st);
            with_part(c->dtype, row_part(n_classes), 256, [&](auto type, auto threads, auto lanes, auto e) {
                using T = decltype(type);
                constexpr int TH = decltype(threads)::value, LA = decltype(lanes)::value, E = decltype(e)::value;
                hipLaunchKernelGGL((k_preference_rows<T, TH, LA, E>), dim3(row_grid(n_rows, TH / LA, most)), dim3(TH), 0, st, R, Q);
            });
        }
        {
            GsTimeScope ts(ctx, "preference_pairs", -1, st);
            hipLaunchKernelGGL(k_preference_pairs, dim3(row_grid(n_pairs, 1, most)), dim3(PT), 0, st, R, Q);
        }
        if (n_rows > 0 && d_grad_logits) {
            GsTimeScope ts(ctx, "preference_grad", -1, st);
            with_part(c->dtype, row_part(n_classes), 256, [&](auto type, auto threads, auto lanes, auto e) {
                using T = decltype(type);
                constexpr int TH = decltype(threads)::value, LA = decltype(lanes)::value, E = decltype(e)::value;
                hipLaunchKernelGGL((k_preference_grad<T, TH, LA, E>), dim3(row_grid(n_rows, TH / LA, most)), dim3(TH), 0, st, R, Q);
            });
        }
        return GSPLIT_OK;
    });
}
