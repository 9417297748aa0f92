// Losses over rows of logits with their gradients: clipped policy loss with a KL term, preference loss of paired log ratios.
// One row: m = max z, s = sum exp(z - m), log p = (z_a - m) - log s; the gradient is slope * (1[c = a] - exp(z_c - m) / s),
// where the slope d loss / d log p is one number a row (a pair).
//
// Memory bounds all of it: a row has to be read and its gradient written, some fifteen vector instructions an element go beside
// that.  So the policy loss reads a row once: its team of lanes holds it in registers while maximum, sum and slope are formed (16
// lanes for up to 512 classes, several rows a wave; a wave; a workgroup of up to 1024 threads, which is all registers of a compute
// unit, for 98304 floats).  8192 x 65536 float 700 us, 5.8 TB/s of reading and writing; 16384 x 8192 176 us, 6.1 TB/s; 4095 x 50001
// bfloat16 147 us, 5.3 TB/s.  Read twice, the second time from the caches, 16384 x 8192 takes 252.
// The preference loss knows no row's slope before all rows of its pair are read, so it reads rows twice: 16 pairs of up to 512 rows
// of 32768 bfloat16 classes 215 us, 1.29 GB moved at 6.0 TB/s.  (Its launches cut into groups of pairs that fit the 256 MB cache
// came out slower, 225 us in groups of 180 MB, 258 of 128.)
// Of small calls the launches are all: 1024 x 47 4.3 us on the device, 7.1 to 8.2 with the host.
#include <algorithm>
#include <cmath>

#include "op_checks.h"
#include "gsplit_internal.h"
#include "row_pieces.h"
#include "row_rules.h"

namespace {

enum : int { HELD, RAW, STREAMED };

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
__device__ __forceinline__ double row_logp(RowStats st, float za) { return ((double)za - (double)base_of(st.m)) - log(st.s); }

// e^x - 1 - x without the cancellation near 0: its series up to |x| = 1 (the first term left out is 4e-9 of the value)
__device__ __forceinline__ float exp_above_tangent(float x) {
    if (x > 80.f) return expf(x);       // (what is missing is nothing beside it, and inf - inf is no number)
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
    // (no number is on neither side: it shows in the gradient as in the loss)
    const bool held = adv >= 0.f ? d > P.log_hi : adv < 0.f && d < P.log_lo;
    const float ratio = adv == 0.f && d > 80.0 ? 1.f : expf((float)d);      // (no advantage: 0 times a ratio that leaves the floats)
    float l = -adv * (held ? (adv >= 0.f ? P.hi : P.lo) : ratio), slope = held ? 0.f : l;
    *kl = 0.f;
    if (P.ref_logp) {
        const float x = (float)((double)ref_logp - logp);
        *kl = exp_above_tangent(x);
        if (P.kl_coef > 0.f) { l += P.kl_coef * *kl; slope -= P.kl_coef * expm1f(x); }      // (kl + x, without their difference)
    }
    *loss = w * l;
    return w * slope;
}

// A team of LANES lanes takes a row.  LANES <= 64: one or more teams a wave, all lanes form the row's numbers alike; else the team is
// the workgroup, and its first wave does.
template <class T, int THREADS, int LANES, int E, int WAYS>
__global__ __launch_bounds__(THREADS) void k_policy_rows(Rows R, Policy P) {
    constexpr bool WG = LANES > 64;
    constexpr bool IN_REGS = WAYS != STREAMED;
    using Row = std::conditional_t<WAYS == RAW, RawRow<T, LANES, E>, HeldRow<T, LANES, E>>;
    __shared__ RowStats lds[WG ? THREADS / 64 : 1];
    __shared__ float lds_row[3];        // a workgroup's row: maximum, sum, slope
    const int lane = WG ? threadIdx.x : threadIdx.x % LANES;
    constexpr int TEAMS = THREADS / LANES;
    // (no loop over rows: the compiler keeps what a loop needs in registers that the row is to have)
    const int64_t r = R.first + (int64_t)blockIdx.x * TEAMS + (WG ? 0 : threadIdx.x / LANES);
    if (r < R.n) {
        const T *z = (const T *)R.logits + r * R.ld;
        T *g = R.grad ? (T *)R.grad + r * R.gld : nullptr;
        const float w = P.weight ? P.weight[r] : P.even_weight;
        const int64_t a = R.actions[r];
        RowStats st{-INFINITY, 0.0};
        float za = 0.f, slope = 0.f;
        Row row;
        if (w != 0.f && a >= 0 && a < R.C) {
            za = (float)z[a];
            if constexpr (IN_REGS) { row.load(z, R.C, lane); st = row.stats(); }
            else st = StreamedRow<T, LANES, E>::stats(z, R.C, lane);
            if constexpr (WG) st = join_waves<LANES>(st, lds);
            else st = join_lanes<LANES>(st);
        }
        if (!WG || threadIdx.x < 64) {
            float loss = 0.f, kl = 0.f, logp = 0.f;
            if (st.s != 0.0) {      // 0: the row is left out
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
            if (threadIdx.x == 0) { lds_row[0] = st.m; lds_row[1] = (float)st.s; lds_row[2] = slope; }
            __syncthreads();
            st = {lds_row[0], lds_row[1]};
            slope = lds_row[2];
        }
        if (g) {
            if (slope == 0.f) store_zeros<T, LANES>(g, R.C, lane);      // nothing moves it
            else if constexpr (IN_REGS) row.store(g, R.C, lane, st, slope, (int)a, za);
            else StreamedRow<T, LANES, E>::store(z, g, R.C, lane, st, slope, (int)a, za);
        }
    }
}

// Few rows of many classes: every row in `chunks` parts (at most 64) of `len` elements, a workgroup each.  One launch leaves the parts'
// statistics and the action's logit, which the next one might otherwise have overwritten when it reads it; the next joins them.
struct Parts {
    RowStats *st;       // [rows x chunks]
    float *za;          // [rows]
    int chunks, len;
    __device__ __forceinline__ int from() const { return (int)blockIdx.x * len; }
    __device__ __forceinline__ int size(int C) const { return min(len, C - from()); }
    // the statistics of row y of the launch: in all lanes of a wave, or by one thread
    __device__ __forceinline__ RowStats joined(int64_t y) const {
        const int lane = threadIdx.x & 63;
        return join_lanes<64>(lane < chunks ? st[y * chunks + lane] : RowStats{-INFINITY, 0.0});
    }
    __device__ __forceinline__ RowStats joined_alone(int64_t y) const {
        const RowStats *p = st + y * chunks;
        float m = -INFINITY;
        double s = 0.0;
        for (int k = 0; k < chunks; ++k) m = fmaxf(m, p[k].m);
        for (int k = 0; k < chunks; ++k) s += p[k].s * (double)share(p[k].m, base_of(m));
        return {m, s};
    }
};
constexpr int CT = 256, CE = 32;

template <class T>
__device__ __forceinline__ void part_stats(const Rows &R, const Parts &S, int64_t r, RowStats *lds) {
    const int64_t a = R.actions[r];
    if (a < 0 || a >= R.C) return;
    const T *z = (const T *)R.logits + r * R.ld;
    const RowStats st = join_waves<CT>(StreamedRow<T, CT, CE>::stats(z + S.from(), S.size(R.C), threadIdx.x), lds);
    if (threadIdx.x == 0) {
        S.st[(int64_t)blockIdx.y * S.chunks + blockIdx.x] = st;
        if (blockIdx.x == 0) S.za[blockIdx.y] = (float)z[a];
    }
}
template <class T>
__device__ __forceinline__ void part_gradient(const Rows &R, const Parts &S, int64_t r, RowStats st, float slope) {
    const T *z = (const T *)R.logits + r * R.ld + S.from();
    T *g = (T *)R.grad + r * R.gld + S.from();
    if (slope == 0.f) store_zeros<T, CT>(g, S.size(R.C), threadIdx.x);
    else StreamedRow<T, CT, CE>::store(z, g, S.size(R.C), threadIdx.x, st, slope, (int)R.actions[r] - S.from(), S.za[blockIdx.y]);
}

template <class T>
__global__ __launch_bounds__(CT) void k_policy_part_stats(Rows R, Policy P, Parts S) {
    __shared__ RowStats lds[CT / 64];
    const int64_t r = blockIdx.y;
    if ((P.weight ? P.weight[r] : P.even_weight) != 0.f) part_stats<T>(R, S, r, lds);
}
template <class T>
__global__ __launch_bounds__(CT) void k_policy_parts(Rows R, Policy P, Parts S) {
    const int64_t r = blockIdx.y, a = R.actions[r];
    const float w = P.weight ? P.weight[r] : P.even_weight;
    RowStats st{-INFINITY, 0.0};
    float loss = 0.f, kl = 0.f, logp = 0.f, slope = 0.f;
    if (w != 0.f && a >= 0 && a < R.C) st = S.joined(r);
    if (st.s != 0.0) {
        const double lp = row_logp(st, S.za[r]);
        logp = (float)lp;
        slope = policy_row(P, lp, P.old_logp[r], P.ref_logp ? P.ref_logp[r] : 0.f, P.advantage[r], w, &loss, &kl);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (P.loss) P.loss[r] = loss;
        if (P.logp) P.logp[r] = logp;
        if (P.kl) P.kl[r] = kl;
    }
    if (R.grad) part_gradient<T>(R, S, r, st, slope);
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
    RowStats st{-INFINITY, 0.0};
    float za = 0.f;
    if (a >= 0 && a < R.C) {
        za = (float)z[a];
        st = StreamedRow<T, LANES, E>::stats(z, R.C, lane);
        if constexpr (LANES > 64) { st = join_waves<LANES>(st, lds); __syncthreads(); }
        else st = join_lanes<LANES>(st);
    }
    const double logp = st.s != 0.0 ? row_logp(st, za) : 0.0;
    if (lane == 0) {
        const float2 bits = __builtin_bit_cast(float2, logp);
        Q.work[r] = {st.m, (float)st.s, bits.x, bits.y};
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
        const auto side = [&](double k, double x) { return k == 0.0 ? 0.0 : k * (soft + fmax(x, 0.0)); };       // (the margin may be infinite)
        if (Q.margin) Q.margin[p] = (float)h;
        if (Q.loss) Q.loss[p] = w == 0.0 ? 0.f : (float)(w * (side(1.0 - e, -h) + side(e, h)));
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

// The same as three launches, for pairs too few or too long for a workgroup each: all rows, all pairs, all rows again.  (Workgroups
// that stay and loop over rows are up to 7 % slower: 30 x 2 x 500 x 10000 bfloat16 345 us, 320.)
template <class T, int THREADS, int LANES, int E>
__global__ __launch_bounds__(THREADS) void k_preference_rows(Rows R, Pairs Q) {
    __shared__ RowStats lds[LANES > 64 ? THREADS / 64 : 1];
    constexpr int TEAMS = THREADS / LANES;
    const int64_t first = seq_at(Q, 0, R.n), last = seq_at(Q, 2 * Q.n, R.n);
    const int64_t r = first + R.first + (int64_t)blockIdx.x * TEAMS + (LANES > 64 ? 0 : threadIdx.x / LANES);
    if (r < last) preference_row<T, LANES, E>(R, Q, r, threadIdx.x % LANES, lds);
}

constexpr int PT = 256;
// (S.chunks > 0: the rows come in parts, a thread joins those of a row)
__global__ __launch_bounds__(PT) void k_preference_pairs(Rows R, Pairs Q, Parts S) {
    __shared__ double lds[PT / 64];
    const int64_t first = seq_at(Q, 0, R.n);
    for (int64_t p = blockIdx.x; p < Q.n; p += gridDim.x) {
        const PairRows P(Q, p, R.n);
        double gap = 0.0;
        for (int64_t i = threadIdx.x; i < P.n; i += PT) {
            const int64_t r = P.row(i);
            double logp;
            if (S.chunks) {
                const int64_t a = R.actions[r], y = r - first;
                RowStats st{-INFINITY, 0.0};
                if (a >= 0 && a < R.C && y >= 0) st = S.joined_alone(y);
                logp = st.s != 0.0 ? row_logp(st, S.za[y]) : 0.0;
                Q.work[r] = {st.m, (float)st.s, 0.f, 0.f};
                if (Q.row_logp) Q.row_logp[r] = (float)logp;
            } else {
                const float4 k = Q.work[r];
                logp = __builtin_bit_cast(double, make_float2(k.z, k.w));
            }
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
    const int64_t r = last - 1 - R.first - (int64_t)blockIdx.x * TEAMS - (LANES > 64 ? 0 : threadIdx.x / LANES);
    if (r >= first) {
        const float4 k = Q.work[r];
        preference_row_grad<T, LANES, E>(R, r, lane, {k.x, k.y}, k.z);
    }
}

template <class T>
__global__ __launch_bounds__(CT) void k_preference_part_stats(Rows R, Pairs Q, Parts S) {
    __shared__ RowStats lds[CT / 64];
    const int64_t r = seq_at(Q, 0, R.n) + blockIdx.y;
    if (r < seq_at(Q, 2 * Q.n, R.n)) part_stats<T>(R, S, r, lds);
}
template <class T>
__global__ __launch_bounds__(CT) void k_preference_parts(Rows R, Pairs Q, Parts S) {
    const int64_t r = seq_at(Q, 0, R.n) + blockIdx.y;
    if (r >= seq_at(Q, 2 * Q.n, R.n)) return;
    const float4 k = Q.work[r];
    part_gradient<T>(R, S, r, {k.x, k.y}, k.z);
}

constexpr int64_t MOST_WORKGROUPS = 1 << 21;        // of a launch, which has less than 2^32 threads

unsigned row_grid(int64_t n, int teams, int64_t most) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(most, gs_ceil_div(n, teams))); }

template <int N> struct Int { static constexpr int value = N; };

// calls f(threads, lanes, elements a lane, way) with the constants of the form
template <class T, class F>
void with_form(int form, F f) {
    const auto go = [&](auto threads, auto lanes, auto e) { f(threads, lanes, e, Int<HELD>{}); };
    switch (form) {
        case ROW_16x8: go(Int<256>{}, Int<16>{}, Int<8>{}); break;
        case ROW_16x16: go(Int<256>{}, Int<16>{}, Int<16>{}); break;
        case ROW_16x32: go(Int<256>{}, Int<16>{}, Int<32>{}); break;
        case ROW_64x16: go(Int<256>{}, Int<64>{}, Int<16>{}); break;
        case ROW_256x32: go(Int<256>{}, Int<256>{}, Int<32>{}); break;
        case ROW_256x64: go(Int<256>{}, Int<256>{}, Int<64>{}); break;
        case ROW_512x64: go(Int<512>{}, Int<512>{}, Int<64>{}); break;
        case ROW_1024x96: go(Int<1024>{}, Int<1024>{}, Int<96>{}); break;
        case ROW_STREAMED: f(Int<1024>{}, Int<1024>{}, Int<32>{}, Int<STREAMED>{}); break;
        default:
            if constexpr (sizeof(T) == 4) {
                if (form == ROW_256x8) go(Int<256>{}, Int<256>{}, Int<8>{});
                else go(Int<1024>{}, Int<1024>{}, Int<64>{});
            } else {
                if (form == ROW_64x32) go(Int<256>{}, Int<64>{}, Int<32>{});
                else if (form == ROW_1024x64) go(Int<1024>{}, Int<1024>{}, Int<64>{});
                else if (form == ROW_512x128_RAW) f(Int<512>{}, Int<512>{}, Int<128>{}, Int<RAW>{});
                else f(Int<1024>{}, Int<1024>{}, Int<128>{}, Int<RAW>{});
            }
    }
}

// the same for kernels that stream rows: lanes a row, elements a lane has in flight
template <class F>
void with_part(int dtype, int lanes, F f) {
    const auto typed = [&](auto type) {
        if (lanes == 16) f(type, Int<16>{}, Int<16>{});
        else if (lanes == 64) f(type, Int<64>{}, Int<32>{});
        else f(type, Int<256>{}, Int<32>{});
    };
    if (dtype == GSPLIT_F32) typed(float{});
    else typed(bf16{});
}

Parts parts_of(const gsplit_ctx *ctx, int64_t n_rows, int C) {
    const int chunks = row_chunks(n_rows, C, ctx->n_cu);
    const int len = (int)gs_ceil_div(gs_ceil_div(C, chunks), 8) * 8;
    return {(RowStats *)ctx->row_part, (float *)((RowStats *)ctx->row_part + GS_ROW_PARTS), (int)gs_ceil_div(C, len), len};
}

template <class T>
void launch_policy(gsplit_ctx *ctx, Rows R, const Policy &P, hipStream_t st) {
    if (policy_in_parts(R.n, R.C, PIECE<T>, ctx->n_cu)) {
        const Parts S = parts_of(ctx, R.n, R.C);
        const dim3 grid(S.chunks, (unsigned)R.n);
        {
            GsTimeScope ts(ctx, "policy_part_stats", -1, st);
            hipLaunchKernelGGL(k_policy_part_stats<T>, grid, dim3(CT), 0, st, R, P, S);
        }
        GsTimeScope ts(ctx, "policy_loss", -1, st);
        hipLaunchKernelGGL(k_policy_parts<T>, grid, dim3(CT), 0, st, R, P, S);
        return;
    }
    with_form<T>(row_form(R.n, R.C, PIECE<T>, ctx->n_cu), [&](auto threads, auto lanes, auto e, auto way) {
        constexpr int TH = decltype(threads)::value, LA = decltype(lanes)::value, E = decltype(e)::value;
        for (; R.first < R.n; R.first += MOST_WORKGROUPS * (TH / LA)) {
            GsTimeScope ts(ctx, "policy_loss", -1, st);
            hipLaunchKernelGGL((k_policy_rows<T, TH, LA, E, decltype(way)::value>), dim3(row_grid(R.n - R.first, TH / LA, MOST_WORKGROUPS)), dim3(TH), 0, st, R, P);
        }
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
        if (c->dtype == GSPLIT_F32) launch_policy<float>(ctx, R, P, st);
        else launch_policy<bf16>(ctx, R, P, st);
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
        Rows R{d_logits, logits_stride, d_grad_logits, grad_stride, d_actions, n_rows, n_classes};
        const Pairs Q{d_seq_ptr, n_pairs, d_ref_logp, d_pair_weight, d_row_logp, d_pair_loss, d_pair_margin,
                      (float4 *)d_row_work, c->beta, c->label_smoothing, (float)(1.0 / (double)n_pairs)};
        const int whole = n_rows > 0 ? preference_whole(n_rows, n_pairs, n_classes, ctx->n_cu) : 0;
        if (whole) {
            GsTimeScope ts(ctx, "preference_loss", -1, st);
            with_part(c->dtype, row_part(n_classes), [&](auto type, auto lanes, auto e) {
                using T = decltype(type);
                constexpr int LA = decltype(lanes)::value, E = decltype(e)::value;
                const auto go = [&](auto threads) {
                    constexpr int TH = decltype(threads)::value;
                    hipLaunchKernelGGL((k_preference_whole<T, TH, LA, E>), dim3((unsigned)n_pairs), dim3(TH), 0, st, R, Q);
                };
                if constexpr (LA == 256) go(Int<256>{});
                else if (whole == 64) go(Int<64>{});
                else if (whole == 256) go(Int<256>{});
                else go(Int<1024>{});
            });
            return GSPLIT_OK;
        }
        const bool grad = n_rows > 0 && d_grad_logits, f32 = c->dtype == GSPLIT_F32;
        const Parts S = n_rows > 0 && preference_in_parts(n_rows, n_classes, ctx->n_cu) ? parts_of(ctx, n_rows, n_classes) : Parts{};
        const dim3 parts(S.chunks, (unsigned)n_rows);
        // launches of a pass over all rows
        const auto over_rows = [&](const char *label, auto part, auto whole_rows) {
            if (S.chunks) {
                GsTimeScope ts(ctx, label, -1, st);
                f32 ? part(float{}) : part(bf16{});
                return;
            }
            with_part(c->dtype, row_part(n_classes), [&](auto type, auto lanes, auto e) {
                constexpr int TEAMS = PT / decltype(lanes)::value;
                for (R.first = 0; R.first < n_rows; R.first += MOST_WORKGROUPS * TEAMS) {
                    GsTimeScope ts(ctx, label, -1, st);
                    whole_rows(type, lanes, e, dim3(row_grid(n_rows - R.first, TEAMS, MOST_WORKGROUPS)));
                }
            });
        };
        if (n_rows > 0)
            over_rows("preference_rows",
                      [&](auto type) { hipLaunchKernelGGL((k_preference_part_stats<decltype(type)>), parts, dim3(CT), 0, st, R, Q, S); },
                      [&](auto type, auto lanes, auto e, dim3 grid) {
                          hipLaunchKernelGGL((k_preference_rows<decltype(type), PT, decltype(lanes)::value, decltype(e)::value>), grid, dim3(PT), 0, st, R, Q);
                      });
        {
            GsTimeScope ts(ctx, "preference_pairs", -1, st);
            hipLaunchKernelGGL(k_preference_pairs, dim3(row_grid(n_pairs, 1, (int64_t)ctx->n_cu * 32)), dim3(PT), 0, st, R, Q, S);
        }
        if (grad)
            over_rows("preference_grad",
                      [&](auto type) { hipLaunchKernelGGL((k_preference_parts<decltype(type)>), parts, dim3(CT), 0, st, R, Q, S); },
                      [&](auto type, auto lanes, auto e, dim3 grid) {
                          hipLaunchKernelGGL((k_preference_grad<decltype(type), PT, decltype(lanes)::value, decltype(e)::value>), grid, dim3(PT), 0, st, R, Q);
                      });
        return GSPLIT_OK;
    });
}
