// Behind the backward pass: the global gradient norm over many tensors, clipping by it, and the AdamW update.
#include <algorithm>

#include "op_checks.h"
#include "gsplit_internal.h"

namespace {

typedef __bf16 bf16;

constexpr int UT = 256;
// The tensors of a launch travel in its arguments (up to 4 KB), so a captured call needs no table in device memory; more of them
// take more launches.
constexpr int NORM_TENSORS = 128;
constexpr int ADAMW_TENSORS = 56;

// How a launch's elements are dealt to workgroups: every tensor in chunks of `chunk` elements, numbered through
template <int N>
struct Chunks {
    int32_t first[N + 1];       // first chunk of a tensor
    int32_t n;
    int64_t chunk;
    int64_t len[N];
    __device__ __forceinline__ int tensor_of(int c) const {     // the last tensor with first <= c: tensors may be empty
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first[mid] <= c) lo = mid; else hi = mid;
        }
        return lo;
    }
};
struct Grads {
    Chunks<NORM_TENSORS> at;
    const void *g[NORM_TENSORS];
    void *out[NORM_TENSORS];
    uint32_t half[NORM_TENSORS / 32];
};
struct Adamw {
    Chunks<ADAMW_TENSORS> at;
    void *p[ADAMW_TENSORS];
    float *master[ADAMW_TENSORS];
    const void *g[ADAMW_TENSORS];
    float *m[ADAMW_TENSORS], *v[ADAMW_TENSORS];
    uint32_t half_p[2], half_g[2];
};
static_assert(sizeof(Grads) <= 4096 - 256 && sizeof(Adamw) <= 4096 - 256, "kernel arguments");

struct Hyper {
    double lr, beta1, beta2, weight_decay;
    float eps, max_norm;
    int64_t step;
    const int64_t *d_step;
    const float *d_lr;
};

template <class T>
__device__ __forceinline__ double sum_of_squares(const T *g, int64_t n) {
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += UT) { const double x = (float)g[i]; s += x * x; }
    return s;
}

__device__ __forceinline__ double wg_sum(double x, double *lds) {
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
    for (int w = 1; w < UT / 64; ++w) x += lds[w];
    __syncthreads();
    return x;
}

__device__ __forceinline__ bool bit_of(const uint32_t *w, int i) { return w[i >> 5] >> (i & 31) & 1; }

// slot b = workgroup b's sum; the launches of one call (`add` in all but the first) have the same grid
__global__ __launch_bounds__(UT) void k_grad_norm(Grads G, double *__restrict__ slots, bool add) {
    __shared__ double lds[UT / 64];
    double s = 0.0;
    for (int c = blockIdx.x; c < G.at.first[G.at.n]; c += gridDim.x) {
        const int t = G.at.tensor_of(c);
        const int64_t at = (int64_t)(c - G.at.first[t]) * G.at.chunk, n = min(G.at.chunk, G.at.len[t] - at);
        s += bit_of(G.half, t) ? sum_of_squares((const bf16 *)G.g[t] + at, n) : sum_of_squares((const float *)G.g[t] + at, n);
    }
    s = wg_sum(s, lds);
    if (threadIdx.x == 0) slots[blockIdx.x] = add ? slots[blockIdx.x] + s : s;
}

// the norm, from the slots of the kernel above
__device__ __forceinline__ float norm_of(const double *__restrict__ slots, int n_slots, double *lds) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n_slots; i += UT) s += slots[i];
    return (float)sqrt(wg_sum(s, lds));
}
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }
__device__ __forceinline__ float factor_of(float norm, float max_norm) {
    return is_finite(norm) && norm > max_norm ? max_norm / norm : 1.f;
}

__global__ __launch_bounds__(UT) void k_norm_of(const double *__restrict__ slots, int n_slots, float *__restrict__ norm) {
    __shared__ double lds[UT / 64];
    const float x = norm_of(slots, n_slots, lds);
    if (threadIdx.x == 0) *norm = x;
}

template <class T>
__device__ __forceinline__ void scale_run(const T *g, T *out, int64_t n, float f) {
    for (int64_t i = threadIdx.x; i < n; i += UT) out[i] = (T)((float)g[i] * f);
}

__global__ __launch_bounds__(UT) void k_clip(Grads G, const double *__restrict__ slots, int n_slots, float max_norm,
                                             float *__restrict__ norm_out) {
    __shared__ double lds[UT / 64];
    const float norm = norm_of(slots, n_slots, lds), f = factor_of(norm, max_norm);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    for (int c = blockIdx.x; c < G.at.first[G.at.n]; c += gridDim.x) {
        const int t = G.at.tensor_of(c);
        if (f == 1.f && G.out[t] == G.g[t]) continue;
        const int64_t at = (int64_t)(c - G.at.first[t]) * G.at.chunk, n = min(G.at.chunk, G.at.len[t] - at);
        if (bit_of(G.half, t)) scale_run((const bf16 *)G.g[t] + at, (bf16 *)G.out[t] + at, n, f);
        else scale_run((const float *)G.g[t] + at, (float *)G.out[t] + at, n, f);
    }
}

struct Steps { float f, keep, rate, b1, a1, b2, a2, root, eps; };      // of one launch's update

template <class T>
__device__ __forceinline__ void update_run(float *p, bf16 *half, const T *g, float *m, float *v, int64_t n, const Steps &S) {
    for (int64_t i = threadIdx.x; i < n; i += UT) {
        const float x = (float)g[i] * S.f;
        const float mi = S.b1 * m[i] + S.a1 * x, vi = S.b2 * v[i] + S.a2 * (x * x);
        const float pi = S.keep * p[i] - S.rate * mi / (sqrtf(vi * S.root) + S.eps);
        m[i] = mi; v[i] = vi; p[i] = pi;
        if (half) half[i] = (bf16)pi;
    }
}

__global__ __launch_bounds__(UT) void k_adamw(Adamw A, Hyper H, const double *__restrict__ slots, int n_slots,
                                              float *__restrict__ norm_out) {
    __shared__ double lds[UT / 64];
    Steps S;
    S.f = 1.f;
    if (n_slots) {
        const float norm = norm_of(slots, n_slots, lds);
        if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
        if (!is_finite(norm)) return;
        S.f = factor_of(norm, H.max_norm);
    }
    const double lr = H.d_lr ? (double)*H.d_lr : H.lr;
    const double t = (double)(H.d_step ? max(*H.d_step, (int64_t)1) : H.step);
    S.keep = (float)(1.0 - lr * H.weight_decay);
    S.rate = (float)(lr / (1.0 - pow(H.beta1, t)));
    S.root = (float)(1.0 / (1.0 - pow(H.beta2, t)));
    S.b1 = (float)H.beta1; S.a1 = (float)(1.0 - H.beta1);
    S.b2 = (float)H.beta2; S.a2 = (float)(1.0 - H.beta2);
    S.eps = H.eps;
    for (int c = blockIdx.x; c < A.at.first[A.at.n]; c += gridDim.x) {
        const int k = A.at.tensor_of(c);
        const int64_t at = (int64_t)(c - A.at.first[k]) * A.at.chunk, n = min(A.at.chunk, A.at.len[k] - at);
        float *p = bit_of(A.half_p, k) ? A.master[k] + at : (float *)A.p[k] + at;
        bf16 *half = bit_of(A.half_p, k) ? (bf16 *)A.p[k] + at : nullptr;
        if (bit_of(A.half_g, k)) update_run(p, half, (const bf16 *)A.g[k] + at, A.m[k] + at, A.v[k] + at, n, S);
        else update_run(p, half, (const float *)A.g[k] + at, A.m[k] + at, A.v[k] + at, n, S);
    }
}

int64_t chunk_of(int64_t total) {
    int64_t chunk = 4096;
    while (chunk < total / (4 * GS_NORM_SLOTS)) chunk *= 2;
    return chunk;
}

// Calls launch(group) for the tensors in groups of N, chunks laid out; fill(group, k, i): tensor i is the group's k-th
template <int N, class Group, class Len, class Fill, class Launch>
void in_groups(int64_t n_tensors, int64_t chunk, Len len, Fill fill, Launch launch) {
    for (int64_t from = 0; from < n_tensors || from == 0; from += N) {
        Group G{};
        G.at.chunk = chunk;
        int64_t chunks = 0;
        for (int64_t i = from; i < std::min<int64_t>(n_tensors, from + N); ++i) {
            const int k = G.at.n++;
            G.at.first[k] = (int32_t)chunks;
            G.at.len[k] = len(i);
            chunks += gs_ceil_div(len(i), chunk);
            fill(G, k, i);
        }
        G.at.first[G.at.n] = (int32_t)chunks;
        launch(G, from == 0);
    }
}

struct NormPlan { int64_t chunk; int slots; };

template <class Len>
NormPlan plan(int64_t n_tensors, Len len, int per_group) {
    int64_t total = 0, most = 0;
    for (int64_t i = 0; i < n_tensors; ++i) total += len(i);
    NormPlan p{chunk_of(total), 1};
    int64_t group = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        if (i % per_group == 0) group = 0;
        group += gs_ceil_div(len(i), p.chunk);
        most = std::max(most, group);
    }
    p.slots = (int)std::max<int64_t>(1, std::min<int64_t>(GS_NORM_SLOTS, most));
    return p;
}

template <class GradOf>
void launch_norm(gsplit_ctx *ctx, int64_t n_tensors, const NormPlan &p, GradOf grad, hipStream_t st) {
    in_groups<NORM_TENSORS, Grads>(
        n_tensors, p.chunk, [&](int64_t i) { return grad(i).n; },
        [&](Grads &G, int k, int64_t i) {
            const gsplit_grad_tensor t = grad(i);
            G.g[k] = t.d_grad;
            G.out[k] = t.d_out ? t.d_out : (void *)t.d_grad;
            if (t.dtype == GSPLIT_BF16) G.half[k >> 5] |= 1u << (k & 31);
        },
        [&](const Grads &G, bool first) {
            GsTimeScope ts(ctx, "grad_norm", -1, st);
            hipLaunchKernelGGL(k_grad_norm, dim3(p.slots), dim3(UT), 0, st, G, ctx->norm_part, !first);
        });
}

}  // namespace

extern "C" int gsplit_grad_norm(gsplit_ctx *ctx, const gsplit_grad_tensor *t, int64_t n_tensors, float *d_norm, void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        const char *e = op_check_grads(t, n_tensors, 0.0, false);
        if (!e && (!d_norm || op_misaligned(d_norm, 4))) e = "bad d_norm";
        if (e) return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_grad_norm: ") + e);
        const NormPlan p = plan(n_tensors, [&](int64_t i) { return t[i].n; }, NORM_TENSORS);
        launch_norm(ctx, n_tensors, p, [&](int64_t i) { return t[i]; }, st);
        GsTimeScope ts(ctx, "norm_of", -1, st);
        hipLaunchKernelGGL(k_norm_of, dim3(1), dim3(UT), 0, st, ctx->norm_part, p.slots, d_norm);
        return GSPLIT_OK;
    });
}

extern "C" int gsplit_clip_grads(gsplit_ctx *ctx, const gsplit_grad_tensor *t, int64_t n_tensors, double max_norm, float *d_norm,
                                 void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        const char *e = op_check_grads(t, n_tensors, max_norm, true);
        if (!e && op_misaligned(d_norm, 4)) e = "misaligned buffer";
        if (e) return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_clip_grads: ") + e);
        const NormPlan p = plan(n_tensors, [&](int64_t i) { return t[i].n; }, NORM_TENSORS);
        launch_norm(ctx, n_tensors, p, [&](int64_t i) { return t[i]; }, st);
        in_groups<NORM_TENSORS, Grads>(
            n_tensors, p.chunk, [&](int64_t i) { return t[i].n; },
            [&](Grads &G, int k, int64_t i) {
                G.g[k] = t[i].d_grad;
                G.out[k] = t[i].d_out ? t[i].d_out : (void *)t[i].d_grad;
                if (t[i].dtype == GSPLIT_BF16) G.half[k >> 5] |= 1u << (k & 31);
            },
            [&](const Grads &G, bool first) {
                GsTimeScope ts(ctx, "clip_grads", -1, st);
                hipLaunchKernelGGL(k_clip, dim3(p.slots), dim3(UT), 0, st, G, ctx->norm_part, p.slots, (float)max_norm,
                                   first ? d_norm : nullptr);
            });
        return GSPLIT_OK;
    });
}

extern "C" int gsplit_adamw_step(gsplit_ctx *ctx, const gsplit_adamw_config *c, const gsplit_adamw_tensor *t, int64_t n_tensors,
                                 float *d_norm, void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        const char *e = op_check_adamw(c, t, n_tensors);
        if (!e && op_misaligned(d_norm, 4)) e = "misaligned buffer";
        if (e) return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_adamw_step: ") + e);
        const auto len = [&](int64_t i) { return t[i].n; };
        int slots = 0;
        if (c->max_norm > 0.0) {
            const NormPlan p = plan(n_tensors, len, NORM_TENSORS);
            launch_norm(ctx, n_tensors, p, [&](int64_t i) {
                return gsplit_grad_tensor{t[i].d_grad, nullptr, t[i].n, t[i].grad_dtype};
            }, st);
            slots = p.slots;
        }
        const NormPlan p = plan(n_tensors, len, ADAMW_TENSORS);
        const Hyper H{c->lr, c->beta1, c->beta2, c->weight_decay, (float)c->eps, (float)c->max_norm, c->step, c->d_step, c->d_lr};
        in_groups<ADAMW_TENSORS, Adamw>(
            n_tensors, p.chunk, len,
            [&](Adamw &A, int k, int64_t i) {
                A.p[k] = t[i].d_param; A.master[k] = t[i].d_master; A.g[k] = t[i].d_grad; A.m[k] = t[i].d_m; A.v[k] = t[i].d_v;
                if (t[i].param_dtype == GSPLIT_BF16) A.half_p[k >> 5] |= 1u << (k & 31);
                if (t[i].grad_dtype == GSPLIT_BF16) A.half_g[k >> 5] |= 1u << (k & 31);
            },
            [&](const Adamw &A, bool first) {
                GsTimeScope ts(ctx, "adamw", -1, st);
                hipLaunchKernelGGL(k_adamw, dim3(p.slots), dim3(UT), 0, st, A, H, ctx->norm_part, slots, first ? d_norm : nullptr);
            });
        return GSPLIT_OK;
    });
}
