// Behind the backward pass: the global gradient norm over many tensors, clipping by it, and the AdamW update.
//
// Memory bounds all of it.  The factor needs every gradient before the first can be scaled, so gradients are read twice; the second
// pass begins with the chunks that the first has left in the 256 MB cache.  400 M gradients of two types in 387 tensors 606 us, 3.6 GB
// at 5.9 TB/s (a plain copy of that size 4.8); the update of 250 M 1355 us, 7.8 GB at 5.7 TB/s: eight streams of it, four read and
// four written.  Of small calls the launches are all: 10 k gradients clipped 4.2 us on the device, the update of 206 k 3.4 + 5.3.
#include <algorithm>
#include <cmath>
#include <limits>

#include "op_checks.h"
#include "gsplit_internal.h"
#include "row_pieces.h"
#include "update_rules.h"

namespace {

// The tensors of a launch travel in its arguments (up to 4 KB), so a captured call needs no table in device memory; more tensors
// take more launches.
constexpr int NORM_TENSORS = 224, CLIP_TENSORS = 144, ADAMW_TENSORS = 72;

// How the elements of a launch's tensors (none of them empty) are dealt: in chunks of `chunk` elements, numbered through
template <int N>
struct Chunks {
    int32_t first[N + 1];       // first chunk of a tensor
    int32_t tail[N];            // elements of its last chunk
    int32_t n, chunk;
    __host__ __device__ __forceinline__ int count() const { return first[n]; }
    __device__ __forceinline__ int tensor_of(int c) const {
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first[mid] <= c) lo = mid; else hi = mid;
        }
        return lo;
    }
    __device__ __forceinline__ int64_t start(int c, int t) const { return (int64_t)(c - first[t]) * chunk; }
    __device__ __forceinline__ int len(int c, int t) const { return c + 1 == first[t + 1] ? tail[t] : chunk; }
};
template <int N> struct Bits {
    uint32_t w[(N + 31) / 32];
    __device__ __forceinline__ bool operator[](int i) const { return w[i >> 5] >> (i & 31) & 1; }
    void set(int i) { w[i >> 5] |= 1u << (i & 31); }
};
struct Norm {
    const void *g[NORM_TENSORS];
    Chunks<NORM_TENSORS> at;
    Bits<NORM_TENSORS> half;
};
struct Clip {
    const void *g[CLIP_TENSORS];
    void *out[CLIP_TENSORS];
    Chunks<CLIP_TENSORS> at;
    Bits<CLIP_TENSORS> half;
};
struct Adamw {
    void *p[ADAMW_TENSORS];
    float *master[ADAMW_TENSORS];
    const void *g[ADAMW_TENSORS];
    float *m[ADAMW_TENSORS], *v[ADAMW_TENSORS];
    Chunks<ADAMW_TENSORS> at;
    Bits<ADAMW_TENSORS> half_p, half_g;
};
static_assert(sizeof(Norm) <= 4096 - 128 && sizeof(Clip) <= 4096 - 128 && sizeof(Adamw) <= 4096 - 256, "kernel arguments");

// -- the norm ---------------------------------------------------------------------------------

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

// Squares are formed and summed in double, which holds those of every float: neither 1e30 nor 1e-30 leaves its range, and the norm
// is the float next to the exact one.  (A conversion and a double multiply-add an element do not show: 400 M elements at 6 TB/s.)
template <class T>
__device__ __forceinline__ double squares(u32x4 q, double s) {
    float x[PIECE<T>];
    unpack<T>(q, x);
#pragma unroll
    for (int k = 0; k < PIECE<T>; ++k) s = fma((double)x[k], (double)x[k], s);
    return s;
}
// (a team of LANES lanes: a wave or the workgroup)
template <class T, int LANES>
__device__ __forceinline__ double sum_of_squares(const T *g, int n, int lane) {
    constexpr int V = PIECE<T>, DEEP = 4;       // pieces a thread has in flight
    const int nv = n / V;
    double s = 0.0;
    int j = lane;
    for (; j + (DEEP - 1) * LANES < nv; j += DEEP * LANES) {
        u32x4 q[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) q[i] = load_kept(g + (j + i * LANES) * V);
#pragma unroll
        for (int i = 0; i < DEEP; ++i) s = squares<T>(q[i], s);
    }
    for (; j < nv; j += LANES) s = squares<T>(load_kept(g + j * V), s);
    if (lane < n - nv * V) { const double x = (float)g[nv * V + lane]; s = fma(x, x, s); }
    return s;
}

template <int THREADS>
__device__ __forceinline__ double wg_sum(double x, double *lds) {
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
    for (int w = 1; w < THREADS / 64; ++w) x += lds[w];
    return x;
}

// a team's share of all squares, as one of `of` teams
template <int LANES, class Table, class Half>
__device__ __forceinline__ double share_of_squares(const Table &G, const Half &half, int which, int of) {
    const int lane = (int)threadIdx.x % LANES;
    double s = 0.0;
    for (int c = which; c < G.at.count(); c += of) {
        const int t = G.at.tensor_of(c);
        const int64_t at = G.at.start(c, t);
        s += half[t] ? sum_of_squares<bf16, LANES>((const bf16 *)G.g[t] + at, G.at.len(c, t), lane)
                     : sum_of_squares<float, LANES>((const float *)G.g[t] + at, G.at.len(c, t), lane);
    }
    return s;
}
// the wave's number, the same in all its lanes as far as the compiler can see
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

constexpr int UT = 256;

// slot b = workgroup b's sum; the launches of one call (`add` in all but the first) have the same grid
__global__ __launch_bounds__(UT) void k_grad_norm(Norm G, double *__restrict__ slots, bool add) {
    __shared__ double lds[UT / 64];
    const double s = wg_sum<UT>(share_of_squares<UT>(G, G.half, blockIdx.x, gridDim.x), lds);
    if (threadIdx.x == 0) slots[blockIdx.x] = add ? slots[blockIdx.x] + s : s;
}

// the norm, from the slots of the kernel above
template <int THREADS>
__device__ __forceinline__ float norm_of(const double *__restrict__ slots, int n_slots, double *lds) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n_slots; i += THREADS) s += slots[i];
    return (float)sqrt(wg_sum<THREADS>(s, lds));
}
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }
__device__ __forceinline__ float factor_of(float norm, float max_norm) {
    return is_finite(norm) && norm > max_norm ? max_norm / norm : 1.f;
}

// their sum, in the slot behind them: for passes of many workgroups, which would each add up a thousand slots
__global__ __launch_bounds__(UT) void k_sum_slots(double *__restrict__ slots, int n_slots) {
    __shared__ double lds[UT / 64];
    double s = 0.0;
    for (int i = threadIdx.x; i < n_slots; i += UT) s += slots[i];
    s = wg_sum<UT>(s, lds);
    if (threadIdx.x == 0) slots[GS_NORM_SLOTS] = s;
}

__global__ __launch_bounds__(UT) void k_norm_of(const double *__restrict__ slots, int n_slots, float *__restrict__ norm) {
    __shared__ double lds[UT / 64];
    const float x = norm_of<UT>(slots, n_slots, lds);
    if (threadIdx.x == 0) *norm = x;
}

// -- clipping ---------------------------------------------------------------------------------

template <class T>
__device__ __forceinline__ u32x4 scaled(u32x4 q, float f) {
    float x[PIECE<T>];
    unpack<T>(q, x);
#pragma unroll
    for (int k = 0; k < PIECE<T>; ++k) x[k] *= f;
    return pack<T>(x);
}
template <class T, int LANES>
__device__ __forceinline__ void scale_run(const T *g, T *out, int n, float f, int lane) {
    constexpr int V = PIECE<T>, DEEP = 4;
    const int nv = n / V;
    int j = lane;
    for (; j + (DEEP - 1) * LANES < nv; j += DEEP * LANES) {
        u32x4 q[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) q[i] = load_piece(g + (j + i * LANES) * V);
#pragma unroll
        for (int i = 0; i < DEEP; ++i) store_piece(out + (j + i * LANES) * V, scaled<T>(q[i], f));
    }
    for (; j < nv; j += LANES) store_piece(out + j * V, scaled<T>(load_piece(g + j * V), f));
    if (lane < n - nv * V) out[nv * V + lane] = (T)((float)g[nv * V + lane] * f);
}

template <int LANES>
__device__ __forceinline__ void scale_chunks(const Clip &G, float f, int which, int of) {
    const int lane = (int)threadIdx.x % LANES;
    // the last chunks first: the norm's pass has left them in the caches
    for (int c = G.at.count() - 1 - which; c >= 0; c -= of) {
        const int t = G.at.tensor_of(c);
        if (f == 1.f && G.out[t] == G.g[t]) continue;
        const int64_t at = G.at.start(c, t);
        if (G.half[t]) scale_run<bf16, LANES>((const bf16 *)G.g[t] + at, (bf16 *)G.out[t] + at, G.at.len(c, t), f, lane);
        else scale_run<float, LANES>((const float *)G.g[t] + at, (float *)G.out[t] + at, G.at.len(c, t), f, lane);
    }
}

__global__ __launch_bounds__(UT) void k_clip(Clip G, const double *__restrict__ slots, int n_slots, float max_norm,
                                             float *__restrict__ norm_out) {
    __shared__ double lds[UT / 64];
    const float norm = norm_of<UT>(slots, n_slots, lds);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    scale_chunks<UT>(G, factor_of(norm, max_norm), blockIdx.x, gridDim.x);
}

// Norm and clipping of few elements by one workgroup (several could not clip in place: one would scale what another still adds up),
// a chunk a wave: taken by the whole workgroup one after the other, the six tensors of 64-64-16 were twelve trips to memory in a
// row, 10.9 us.
constexpr int ST = 1024;
static_assert(UPDATE_CLIP_SMALL_CHUNKS <= CLIP_TENSORS, "one launch holds them");
__global__ __launch_bounds__(ST) void k_clip_small(Clip G, float max_norm, float *__restrict__ norm_out) {
    __shared__ double lds[ST / 64];
    const float norm = (float)sqrt(wg_sum<ST>(share_of_squares<64>(G, G.half, wave_id(), ST / 64), lds));
    if (norm_out && threadIdx.x == 0) *norm_out = norm;
    scale_chunks<64>(G, factor_of(norm, max_norm), wave_id(), ST / 64);
}

// -- the update -------------------------------------------------------------------------------

struct Hyper {
    double lr, beta1, beta2, weight_decay;
    int64_t step;
    const int64_t *d_step;
    const float *d_lr;
    float eps, max_norm;
};
struct Steps { float f, keep, rate, b1, a1, b2, a2, root, eps; };      // the numbers of a launch's update

__host__ __device__ inline Steps steps_of(const Hyper &H, double lr, double t) {
    return {1.f, (float)(1.0 - lr * H.weight_decay), (float)(lr / (1.0 - pow(H.beta1, t))), (float)H.beta1, (float)(1.0 - H.beta1),
            (float)H.beta2, (float)(1.0 - H.beta2), (float)(1.0 / (1.0 - pow(H.beta2, t))), H.eps};
}

// four elements of the gradient of either type
template <class T>
__device__ __forceinline__ void load4(const T *g, float *x) {
    if constexpr (sizeof(T) == 4) {
        unpack<float>(load_piece(g), x);
    } else {
        const u32x2 q = __builtin_nontemporal_load((const u32x2_any *)g);
        for (int k = 0; k < 2; ++k) { x[2 * k] = __uint_as_float(q[k] << 16); x[2 * k + 1] = __uint_as_float(q[k] & 0xffff0000u); }
    }
}
__device__ __forceinline__ void update1(float &p, float &m, float &v, float g, const Steps &S) {
    g *= S.f;
    m = S.b1 * m + S.a1 * g;
    v = S.b2 * v + S.a2 * (g * g);
    p = S.keep * p - S.rate * m / (sqrtf(v * S.root) + S.eps);
}
// LARGE: what is read and written will not be found in the caches by the next step, and is said not to be read again.
template <class T, bool HALF, int THREADS, bool LARGE>
__device__ __forceinline__ void update_run(float *p, bf16 *half, const T *g, float *m, float *v, int n, const Steps &S) {
    constexpr int DEEP = 2;
    const int nv = n / 4;
    const auto load = [](const float *from, float *x) { unpack<float>(LARGE ? load_piece(from) : load_kept(from), x); };
    const auto store = [](float *to, const float *x) { LARGE ? store_piece(to, pack<float>(x)) : store_kept(to, pack<float>(x)); };
    const auto step = [&](int j, auto deep) {
        constexpr int D = decltype(deep)::value;
        float pp[D][4], mm[D][4], vv[D][4], gg[D][4];
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const int e = (j + i * THREADS) * 4;
            load(p + e, pp[i]); load(m + e, mm[i]); load(v + e, vv[i]); load4(g + e, gg[i]);
        }
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const int e = (j + i * THREADS) * 4;
#pragma unroll
            for (int k = 0; k < 4; ++k) update1(pp[i][k], mm[i][k], vv[i][k], gg[i][k], S);
            store(p + e, pp[i]); store(m + e, mm[i]); store(v + e, vv[i]);
            if constexpr (HALF)
                __builtin_nontemporal_store((u32x2{bf16_pair(pp[i][0], pp[i][1]), bf16_pair(pp[i][2], pp[i][3])}), (u32x2_any *)(half + e));
        }
    };
    int j = threadIdx.x;
    for (; j + (DEEP - 1) * THREADS < nv; j += DEEP * THREADS) step(j, std::integral_constant<int, DEEP>{});
    for (; j < nv; j += THREADS) step(j, std::integral_constant<int, 1>{});
    if ((int)threadIdx.x < n - nv * 4) {
        const int e = nv * 4 + threadIdx.x;
        float pi = p[e], mi = m[e], vi = v[e];
        update1(pi, mi, vi, (float)g[e], S);
        p[e] = pi; m[e] = mi; v[e] = vi;
        if constexpr (HALF) half[e] = (bf16)pi;
    }
}

// How the norm reaches the update: not at all, from the slots, or formed by every workgroup anew (few elements)
enum : int { NORM_NONE, NORM_SLOTS, NORM_HERE };

template <int WHENCE, int THREADS, bool LARGE>
__global__ __launch_bounds__(THREADS) void k_adamw(Adamw A, Hyper H, Steps S, const double *__restrict__ slots, int n_slots,
                                              float *__restrict__ norm_out) {
    __shared__ double lds[THREADS / 64];
    if (H.d_step || H.d_lr) {
        __shared__ Steps shared;
        if (threadIdx.x == 0)
            shared = steps_of(H, H.d_lr ? (double)*H.d_lr : H.lr, (double)(H.d_step ? max(*H.d_step, (int64_t)1) : H.step));
        __syncthreads();
        S = shared;
    }
    if constexpr (WHENCE != NORM_NONE) {
        float norm;
        if constexpr (WHENCE == NORM_SLOTS) norm = norm_of<THREADS>(slots, n_slots, lds);
        else norm = (float)sqrt(wg_sum<THREADS>(share_of_squares<64>(A, A.half_g, wave_id(), THREADS / 64), lds));
        if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
        if (!is_finite(norm)) return;
        S.f = factor_of(norm, H.max_norm);
    }
    for (int c = A.at.count() - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
        const int t = A.at.tensor_of(c), n = A.at.len(c, t);
        const int64_t at = A.at.start(c, t);
        float *m = A.m[t] + at, *v = A.v[t] + at;
        const float *g = (const float *)A.g[t] + at;
        const bf16 *gh = (const bf16 *)A.g[t] + at;
        if (A.half_p[t]) {
            float *p = A.master[t] + at;
            bf16 *half = (bf16 *)A.p[t] + at;
            if (A.half_g[t]) update_run<bf16, true, THREADS, LARGE>(p, half, gh, m, v, n, S);
            else update_run<float, true, THREADS, LARGE>(p, half, g, m, v, n, S);
        } else {
            float *p = (float *)A.p[t] + at;
            if (A.half_g[t]) update_run<bf16, false, THREADS, LARGE>(p, nullptr, gh, m, v, n, S);
            else update_run<float, false, THREADS, LARGE>(p, nullptr, g, m, v, n, S);
        }
    }
}

// -- launches ---------------------------------------------------------------------------------

// Calls launch(group, first) for the tensors that are not empty, in groups of N (one empty group if there are none), the last
// ones first if `back`; fill(group, k, i): tensor i is the group's k-th.
template <int N, class Group, class Len, class Fill, class Launch>
void in_groups(int64_t n_tensors, int chunk, bool back, Len len, Fill fill, Launch launch) {
    bool first = true;
    int64_t i = back ? n_tensors - 1 : 0;
    const int64_t by = back ? -1 : 1;
    do {
        int64_t from = i, to = i;           // a group's tensors: their own order in either direction
        int found = 0;
        for (; to >= 0 && to < n_tensors && found < N; to += by) found += len(to) > 0;
        if (back) { const int64_t t = from; from = to + 1; to = t + 1; i = from - 1; }
        else i = to;
        Group G{};
        G.at.chunk = chunk;
        int64_t chunks = 0;
        for (int64_t x = from; x < to; ++x) {
            const int64_t n = len(x);
            if (n == 0) continue;
            const int k = G.at.n++;
            G.at.first[k] = (int32_t)chunks;
            chunks += gs_ceil_div(n, chunk);
            G.at.tail[k] = (int32_t)(n - (gs_ceil_div(n, chunk) - 1) * chunk);
            fill(G, k, x);
        }
        G.at.first[G.at.n] = (int32_t)chunks;
        launch(G, first);
        first = false;
    } while (i >= 0 && i < n_tensors);
}

struct Totals { int64_t elements = 0, tensors = 0; };       // tensors: those that are not empty
template <class Len>
Totals totals_of(int64_t n_tensors, Len len) {
    Totals t;
    for (int64_t i = 0; i < n_tensors; ++i) { t.elements += len(i); t.tensors += len(i) > 0; }
    return t;
}

// Where a pass finds the sum of all squares: at[0 .. n - 1]
struct Slots { const double *at; int n; };

// forms it; passes of `workgroups` workgroups will read it
template <class GradOf>
Slots launch_norm(gsplit_ctx *ctx, int64_t n_tensors, const Totals &total, int64_t workgroups, GradOf grad, hipStream_t st) {
    const auto len = [&](int64_t i) { return grad(i).n; };
    const int chunk = norm_chunk(total.elements, ctx->n_cu);
    // the grid of all launches: what the first one's chunks fill (a slot that a launch has nothing for keeps its sum)
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(GS_NORM_SLOTS, (int64_t)ctx->n_cu * 4),
                                                                 total.elements / chunk + total.tensors));
    in_groups<NORM_TENSORS, Norm>(
        n_tensors, chunk, false, len,
        [&](Norm &G, int k, int64_t i) {
            G.g[k] = grad(i).d_grad;
            if (grad(i).dtype == GSPLIT_BF16) G.half.set(k);
        },
        [&](const Norm &G, bool first) {
            GsTimeScope ts(ctx, "grad_norm", -1, st);
            hipLaunchKernelGGL(k_grad_norm, dim3(grid), dim3(UT), 0, st, G, ctx->norm_part, !first);
        });
    if (!norm_in_one_slot(workgroups, ctx->n_cu)) return {ctx->norm_part, grid};
    GsTimeScope ts(ctx, "sum_slots", -1, st);
    hipLaunchKernelGGL(k_sum_slots, dim3(1), dim3(UT), 0, st, ctx->norm_part, grid);
    return {ctx->norm_part + GS_NORM_SLOTS, 1};
}

}  // namespace

extern "C" int gsplit_grad_norm(gsplit_ctx *ctx, const gsplit_grad_tensor *t, int64_t n_tensors, float *d_norm, void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        const char *e = op_check_grads(t, n_tensors, 0.0, false);
        if (!e && (!d_norm || op_misaligned(d_norm, 4))) e = "bad d_norm";
        if (e) return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_grad_norm: ") + e);
        const Totals total = totals_of(n_tensors, [&](int64_t i) { return t[i].n; });
        const Slots slots = launch_norm(ctx, n_tensors, total, 1, [&](int64_t i) { return t[i]; }, st);
        GsTimeScope ts(ctx, "norm_of", -1, st);
        hipLaunchKernelGGL(k_norm_of, dim3(1), dim3(UT), 0, st, slots.at, slots.n, d_norm);
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
        const auto len = [&](int64_t i) { return t[i].n; };
        const Totals total = totals_of(n_tensors, len);
        const bool small = update_clip_small(total.elements, total.tensors);
        const int chunk = update_chunk(total.elements, 4096, ctx->n_cu);
        const Slots slots = small ? Slots{nullptr, 0} : launch_norm(ctx, n_tensors, total, total.elements / chunk, [&](int64_t i) { return t[i]; }, st);
        in_groups<CLIP_TENSORS, Clip>(
            n_tensors, chunk, true, len,
            [&](Clip &G, int k, int64_t i) {
                G.g[k] = t[i].d_grad;
                G.out[k] = t[i].d_out ? t[i].d_out : (void *)t[i].d_grad;
                if (t[i].dtype == GSPLIT_BF16) G.half.set(k);
            },
            [&](const Clip &G, bool first) {
                GsTimeScope ts(ctx, "clip_grads", -1, st);
                float *norm = first ? d_norm : nullptr;
                if (small) hipLaunchKernelGGL(k_clip_small, dim3(1), dim3(ST), 0, st, G, (float)max_norm, norm);
                else hipLaunchKernelGGL(k_clip, dim3(std::max(1, G.at.count())), dim3(UT), 0, st, G, slots.at, slots.n, (float)max_norm, norm);
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
        const Totals total = totals_of(n_tensors, len);
        const bool clip = c->max_norm > 0.0, here = clip && total.tensors <= ADAMW_TENSORS && update_norm_here(total.elements);
        const bool large = update_large(total.elements);
        const int chunk = update_chunk(total.elements, 2048, ctx->n_cu);
        Slots slots{nullptr, 0};
        if (clip && !here)
            slots = launch_norm(ctx, n_tensors, total, total.elements / chunk, [&](int64_t i) {
                return gsplit_grad_tensor{t[i].d_grad, nullptr, t[i].n, t[i].grad_dtype};
            }, st);
        // (an eps below the floats stays above 0: an element without gradient and moments is 0 / (0 + eps), which is no number for 0)
        const float eps = c->eps > 0.0 ? std::max((float)c->eps, std::numeric_limits<float>::denorm_min()) : 0.f;
        const Hyper H{c->lr, c->beta1, c->beta2, c->weight_decay, c->step, c->d_step, c->d_lr, eps, (float)c->max_norm};
        const Steps S = c->d_step || c->d_lr ? Steps{} : steps_of(H, H.lr, (double)H.step);
        in_groups<ADAMW_TENSORS, Adamw>(
            n_tensors, chunk, true, len,
            [&](Adamw &A, int k, int64_t i) {
                A.p[k] = t[i].d_param; A.master[k] = t[i].d_master; A.g[k] = t[i].d_grad; A.m[k] = t[i].d_m; A.v[k] = t[i].d_v;
                if (t[i].param_dtype == GSPLIT_BF16) A.half_p.set(k);
                if (t[i].grad_dtype == GSPLIT_BF16) A.half_g.set(k);
            },
            [&](const Adamw &A, bool first) {
                GsTimeScope ts(ctx, "adamw", -1, st);
                const auto kernel = here ? k_adamw<NORM_HERE, ST, false>
                                    : large ? clip ? k_adamw<NORM_SLOTS, UT, true> : k_adamw<NORM_NONE, UT, true>
                                            : clip ? k_adamw<NORM_SLOTS, UT, false> : k_adamw<NORM_NONE, UT, false>;
                hipLaunchKernelGGL(kernel, dim3(std::max(1, A.at.count())), dim3(here ? ST : UT), large ? UPDATE_LARGE_LDS : 0, st, A, H, S, slots.at, slots.n,
                                   first ? d_norm : nullptr);
            });
        return GSPLIT_OK;
    });
}
