// Rows of logits in registers: how a team of lanes reads a row, forms its statistics and writes its gradient.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace {

typedef __bf16 bf16;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float floatx2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
// a row starts where the one before it and the padding end: a piece of 16 bytes is aligned to its elements only, which the
// vector loads and stores of the chip take
typedef u32x4 u32x4_any __attribute__((aligned(2)));

template <class T> constexpr int PIECE = 16 / (int)sizeof(T);       // elements of a piece

// load_piece: for what is read once; load_kept: read again soon
__device__ __forceinline__ u32x4 load_piece(const void *p) { return __builtin_nontemporal_load((const u32x4_any *)p); }
__device__ __forceinline__ u32x4 load_kept(const void *p) { return *(const u32x4_any *)p; }
__device__ __forceinline__ void store_kept(void *p, u32x4 q) { *(u32x4_any *)p = q; }
__device__ __forceinline__ void store_piece(void *p, u32x4 q) { __builtin_nontemporal_store(q, (u32x4_any *)p); }

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2_t){lo, hi}, bf16x2_t));
}
template <class T>
__device__ __forceinline__ void unpack(u32x4 q, float *x) {
    if constexpr (sizeof(T) == 4) {
        for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(q[k]);
    } else {
        for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(q[k] << 16); x[2 * k + 1] = __uint_as_float(q[k] & 0xffff0000u); }
    }
}
template <class T>
__device__ __forceinline__ u32x4 pack(const float *x) {
    u32x4 q;
    if constexpr (sizeof(T) == 4) {
        for (int k = 0; k < 4; ++k) q[k] = __float_as_uint(x[k]);
    } else {
        for (int k = 0; k < 4; ++k) q[k] = bf16_pair(x[2 * k], x[2 * k + 1]);
    }
    return q;
}
template <class T> constexpr uint32_t MINUS_INF = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;

// e^x for x <= 0.  The float next to log2(e) alone is low by 1.3e-8 of it, which puts the sum of a row's exponentials 1.5e-8 (47
// classes) to 5e-8 (32768) above what it is, in every row: the margin of a preference over 300 rows came out 2.4e-6 off.  The small
// part goes into the product before that is rounded (added to a rounded one it is lost).
constexpr float LOG2E = 1.44269504f, LOG2E_REST = 1.92596299e-8f;
__device__ __forceinline__ float exp_fine(float x) { return __builtin_amdgcn_exp2f(fmaf(x, LOG2E, x * LOG2E_REST)); }
__device__ __forceinline__ float exp_plain(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

// Statistics of (a part of) a row: maximum m and sum s of exp(z - base(m)).  base(-inf) = 0: a row of -inf alone has the sum 0.
// fmaxf drops a NaN, the sum keeps it.  A lane adds up floats, sums of lanes are joined in double: the lanes' roundings average
// out, those of joining them in float did not (log p off by 4.5e-8 on average, and with it a KL term of 0.005 by 1e-6 of it).
struct RowStats { float m; double s; };
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// what the sums of a part with maximum m count in one with the base b >= m
__device__ __forceinline__ float share(float m, float b) { return m == -INFINITY ? 0.f : exp_fine(m - b); }
__device__ __forceinline__ RowStats join(RowStats a, RowStats b) {
    const float m = fmaxf(a.m, b.m), base = base_of(m);
    return {m, a.s * (double)share(a.m, base) + b.s * (double)share(b.m, base)};
}

// over the LANES (<= 64, a power of two) lanes of a team inside a wave
template <int LANES>
__device__ __forceinline__ RowStats join_lanes(RowStats a) {
    float m = a.m;
    for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    double s = a.s * (double)share(a.m, base_of(m));
    for (int o = LANES / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
    return {m, s};
}
// over a workgroup of LANES threads, for its first wave (all sixteen joining took 0.4 us of one row's 8.5); one barrier, and
// another one has to come before `lds` [LANES / 64] is written again
template <int LANES>
__device__ __forceinline__ RowStats join_waves(RowStats a, RowStats *lds) {
    a = join_lanes<64>(a);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    if (threadIdx.x < 64) a = join_lanes<LANES / 64>(lds[threadIdx.x % (LANES / 64)]);
    return a;
}

// A row of C elements held by LANES lanes, E each: pieces lane, lane + LANES, ..., and of the elements behind the last whole
// piece one in each of the first lanes.  After stats() x holds the exponentials above the lane's own maximum.
template <class T, int LANES, int E>
struct HeldRow {
    static constexpr int V = PIECE<T>, NV = E / V;
    float x[E], rest;
    float m;
    int nv;             // whole pieces of the row; those a shorter row leaves without any are skipped by the whole team

    template <bool AGAIN = false>
    __device__ __forceinline__ void load(const T *z, int C, int lane) {
        nv = C / V;
        u32x4 q[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES < nv) {
                q[i] = MINUS_INF<T>;
                if (lane + i * LANES < nv) q[i] = AGAIN ? load_kept(z + (lane + i * LANES) * V) : load_piece(z + (lane + i * LANES) * V);
            }
        rest = -INFINITY;
        if (lane < C - nv * V) rest = (float)z[nv * V + lane];
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES < nv) unpack<T>(q[i], x + i * V);
    }
    __device__ __forceinline__ RowStats stats() {
        m = rest;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES < nv)
#pragma unroll
                for (int k = 0; k < V; ++k) m = fmaxf(m, x[i * V + k]);
        const float b = base_of(m);
        rest = exp_fine(rest - b);
        float s = rest;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES < nv) {
                float piece = 0.f;      // (a piece by itself first: fewer roundings than one after the other into s)
#pragma unroll
                for (int k = 0; k < V; ++k) { x[i * V + k] = exp_fine(x[i * V + k] - b); piece += x[i * V + k]; }
                s += piece;
            }
        return {m, (double)s};
    }
    // g = -scale * exp(z - base(all.m)), and slope more for class a
    __device__ __forceinline__ void store(T *g, int C, int lane, RowStats all, float slope, int a, float za) const {
        const float b = base_of(all.m), scale = -slope / (float)all.s, mine = scale * share(m, b);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES < nv) {
                float y[V];
#pragma unroll
                for (int k = 0; k < V; ++k) y[k] = mine * x[i * V + k];
                if (lane + i * LANES < nv) store_piece(g + (lane + i * LANES) * V, pack<T>(y));
            }
        if (lane < C - nv * V) g[nv * V + lane] = (T)(mine * rest);
        // by the lane that wrote the action's class, so that this store comes second
        if (lane == (a < nv * V ? a / V % LANES : a - nv * V)) g[a] = (T)(slope + scale * exp_plain(za - b));
    }
};

// Keeps the compiler from holding on to what it has unpacked from q: it would take the registers twice over
__device__ __forceinline__ void anew(u32x4 &q) { asm volatile("" : "+v"(q)); }

// The same for bfloat16 rows as they are, half the registers: exponentials are formed twice
template <class T, int LANES, int E>
struct RawRow {
    static constexpr int V = PIECE<T>, NV = E / V;
    u32x4 q[NV];
    float rest;
    int nv;

    __device__ __forceinline__ void load(const T *z, int C, int lane) {
        nv = C / V;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES < nv) {
                q[i] = MINUS_INF<T>;
                if (lane + i * LANES < nv) q[i] = load_piece(z + (lane + i * LANES) * V);
            }
        rest = -INFINITY;
        if (lane < C - nv * V) rest = (float)z[nv * V + lane];
    }
    __device__ __forceinline__ RowStats stats() {
        float m = rest;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES < nv) {
                float x[V];
                unpack<T>(q[i], x);
#pragma unroll
                for (int k = 0; k < V; ++k) m = fmaxf(m, x[k]);
            }
        const float b = base_of(m);
        float s = exp_fine(rest - b);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES < nv) {
                float x[V];
                anew(q[i]);
                unpack<T>(q[i], x);
                float piece = 0.f;
#pragma unroll
                for (int k = 0; k < V; ++k) piece += exp_fine(x[k] - b);
                s += piece;
            }
        return {m, (double)s};
    }
    __device__ __forceinline__ void store(T *g, int C, int lane, RowStats all, float slope, int a, float za) {
        const float b = base_of(all.m), scale = -slope / (float)all.s;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES < nv) {
                float y[V];
                anew(q[i]);
                unpack<T>(q[i], y);
#pragma unroll
                for (int k = 0; k < V; ++k) y[k] = scale * exp_plain(y[k] - b);
                if (lane + i * LANES < nv) store_piece(g + (lane + i * LANES) * V, pack<T>(y));
            }
        if (lane < C - nv * V) g[nv * V + lane] = (T)(scale * exp_plain(rest - b));
        if (lane == (a < nv * V ? a / V % LANES : a - nv * V)) g[a] = (T)(slope + scale * exp_plain(za - b));
    }
};

template <class T, int LANES>
__device__ __forceinline__ void store_zeros(T *g, int C, int lane) {
    constexpr int V = PIECE<T>;
    const int nv = C / V;
    for (int i = lane; i < nv; i += LANES) store_piece(g + (int64_t)i * V, u32x4{0, 0, 0, 0});
    if (lane < C - nv * V) g[nv * V + lane] = (T)0.f;
}

// The same of a row, or of a part of one, that the registers do not hold: read for the statistics, read again for the gradient.
// E: elements a lane has in flight.
template <class T, int LANES, int E>
struct StreamedRow {
    static constexpr int V = PIECE<T>;
    using Held = HeldRow<T, LANES, E>;
    static constexpr int STEP = LANES * E;

    __device__ __forceinline__ static RowStats stats(const T *z, int C, int lane) {
        RowStats all{-INFINITY, 0.0};
        for (int c = 0; c < C; c += STEP) {
            Held h;
            h.template load<true>(z + c, min(STEP, C - c), lane);
            all = join(all, h.stats());
        }
        return all;
    }
    // (a: the action's class counted from this part's start, outside [0, C) if it lies in another)
    __device__ __forceinline__ static void store(const T *z, T *g, int C, int lane, RowStats all, float slope, int a, float za) {
        const float b = base_of(all.m), scale = -slope / (float)all.s;
        for (int c = 0; c < C; c += STEP) {
            Held h;
            const int n = min(STEP, C - c), nv = n / V;
            h.load(z + c, n, lane);
            T *to = g + c;
#pragma unroll
            for (int i = 0; i < Held::NV; ++i)
                if (i * LANES < nv) {
                    float y[V];
#pragma unroll
                    for (int k = 0; k < V; ++k) y[k] = scale * exp_plain(h.x[i * V + k] - b);
                    if (lane + i * LANES < nv) store_piece(to + (lane + i * LANES) * V, pack<T>(y));
                }
            if (lane < n - nv * V) to[nv * V + lane] = (T)(scale * exp_plain(h.rest - b));
            const int at = a - c;
            if (at >= 0 && at < n && lane == (at < nv * V ? at / V % LANES : at - nv * V)) to[at] = (T)(slope + scale * exp_plain(za - b));
        }
    }
};

}  // namespace
