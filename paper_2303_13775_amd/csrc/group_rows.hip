// Rows sorted by their group: a counting sort that keeps the order of a group's rows.
//
// A wave takes a run of rows, 64 at a time: ballots over the bits of the group say which lanes share one, so a lane's place is the
// number of lanes in front of it in its own group, and one lane adds to a counter for all of them (as many atomics as rows would
// meet at few addresses).  Small calls are one workgroup's, larger ones two launches: the counters of every workgroup's rows, and
// the places, for which each workgroup adds up the counters of those in front of it.
//
// Latency bounds it: 8 MB are 1.6 us of a 5.05 TB/s copy, a million rows of 64 groups take 4.0 + 10.0 us, 1024 rows of 4 groups 3.7 in one
// launch.  The groups of a wave's first 256 rows and their matches stay in registers over both of its passes, the counters come
// eight loads at a time (one after the other, and rows read again: 14.4 us).  No faster: rows put in order in LDS so that threads
// side by side write side by side (11.2), two workgroups a compute unit (5.2 + 15.8, twice the counters for everybody), one every
// two (5.9 + 12.0), sixteen loads at a time (10.2).
#include "group_rules.h"
#include "gsplit_internal.h"
#include "op_checks.h"
#include "row_rules.h"

namespace {

constexpr int GT = 64 * GROUP_WAVES;

struct Rows {
    const int32_t *group;
    int64_t n, a_wave;          // rows; of a wave's run
    int32_t G, bits;
    int32_t *ptr, *rows, *count;        // count [workgroups x G]
};

// DEEP rounds of 64 rows of a wave: every lane's group (-1: none) and the lanes of the same group
constexpr int DEEP = 4;
struct Rounds { int32_t g[DEEP]; uint64_t same[DEEP]; };
__device__ __forceinline__ void load_rounds(const Rows &R, int64_t at, int64_t hi, Rounds &v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 0; d < DEEP; ++d) v.g[d] = -1;
    if (at >= hi) return;                       // (nothing can be read where there are no rows)
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
        const int64_t r = at + 64 * d + lane;
        v.g[d] = R.group[min(r, R.n - 1)];
        if (r >= hi || (uint32_t)v.g[d] >= (uint32_t)R.G) v.g[d] = -1;
    }
}
__device__ __forceinline__ void match_rounds(const Rows &R, Rounds &v) {
#pragma unroll
    for (int d = 0; d < DEEP; ++d) v.same[d] = __ballot(v.g[d] >= 0);
    for (int b = 0; b < R.bits; ++b)
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const uint64_t set = __ballot(v.g[d] >> b & 1);
            v.same[d] &= v.g[d] >> b & 1 ? set : ~set;
        }
}
// the rows lo .. hi - 1 of a wave, of which the first rounds are there: f(first row of the round, group, lanes of the same group)
template <class F>
__device__ __forceinline__ void rounds(const Rows &R, int64_t lo, int64_t hi, const Rounds &first, F &&f) {
    Rounds v = first;
    for (int64_t at = lo; at < hi; at += 64 * DEEP) {
        if (at > lo) {
            load_rounds(R, at, hi, v);
            match_rounds(R, v);
        }
#pragma unroll
        for (int d = 0; d < DEEP; ++d) f(at + 64 * d, v.g[d], v.same[d]);
    }
}
__device__ __forceinline__ int before_me(uint64_t same) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
}
// Counters in LDS pass from lane to lane: what a round reads and writes stays between its neighbours' (LDS does a wave's instructions in
// their order; the compiler is told to keep it)
__device__ __forceinline__ void settle() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ void run_of(const Rows &R, int64_t &lo, int64_t &hi) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    lo = min((blockIdx.x * (int64_t)GROUP_WAVES + wave) * R.a_wave, R.n);
    hi = min(lo + R.a_wave, R.n);
}

__global__ __launch_bounds__(GT) void k_group_count(Rows R) {
    extern __shared__ int32_t s_count[];       // [G]
    int64_t lo, hi;
    run_of(R, lo, hi);
    Rounds first;
    load_rounds(R, lo, hi, first);
    for (int g = threadIdx.x; g < R.G; g += GT) s_count[g] = 0;
    __syncthreads();
    match_rounds(R, first);
    rounds(R, lo, hi, first, [&](int64_t, int32_t g, uint64_t same) {
        if (g >= 0 && before_me(same) == 0) atomicAdd(&s_count[g], __popcll(same));
    });
    __syncthreads();
    for (int g = threadIdx.x; g < R.G; g += GT) R.count[(int64_t)blockIdx.x * R.G + g] = s_count[g];
}

// exclusive sums over the workgroup's threads
__device__ __forceinline__ int32_t sum_before(int32_t x, int32_t *s_wave) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t y = x;
    for (int o = 1; o < 64; o <<= 1) {
        const int32_t z = __shfl_up(y, o);
        if (lane >= o) y += z;
    }
    if (lane == 63) s_wave[wave] = y;
    __syncthreads();
    int32_t base = 0;
    for (int w = 0; w < GROUP_WAVES; ++w) base += w < wave ? s_wave[w] : 0;
    return base + y - x;
}

// WHOLE: the only workgroup, which needs nobody's counters
template <bool WHOLE>
__global__ __launch_bounds__(GT) void k_group_place(Rows R) {
    extern __shared__ int32_t lds[];           // [waves x G] where a wave's next row of a group goes, then [2 x GT]
    __shared__ int32_t s_wave[GROUP_WAVES];
    int32_t *s_next = lds, *s_part = lds + GROUP_WAVES * R.G;
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    int64_t lo, hi;
    run_of(R, lo, hi);
    Rounds first;
    load_rounds(R, lo, hi, first);
    for (int i = t; i < GROUP_WAVES * R.G; i += GT) s_next[i] = 0;
    int32_t in_front = 0, all = 0;              // rows of group t in the workgroups in front; in all
    if (!WHOLE) {
        const int parts = GT / R.G;             // threads that share a group's counters
        const int g = t % R.G, part = t / R.G;
        if (part < parts)
            for (int b = part; b < (int)gridDim.x; b += 8 * parts) {
                int32_t c[8];                   // (eight loads in flight)
#pragma unroll
                for (int u = 0; u < 8; ++u) c[u] = R.count[(int64_t)min(b + u * parts, (int)gridDim.x - 1) * R.G + g];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    all += b + u * parts < (int)gridDim.x ? c[u] : 0;
                    in_front += b + u * parts < (int)blockIdx.x ? c[u] : 0;
                }
            }
        s_part[t] = in_front; s_part[GT + t] = all;
        __syncthreads();
        in_front = all = 0;
        if (t < R.G)
            for (int p = 0; p < parts; ++p) { in_front += s_part[p * R.G + t]; all += s_part[GT + p * R.G + t]; }
    }
    match_rounds(R, first);
    __syncthreads();
    rounds(R, lo, hi, first, [&](int64_t, int32_t g, uint64_t same) {
        if (g >= 0 && before_me(same) == 0) s_next[wave * R.G + g] += __popcll(same);
        settle();
    });
    __syncthreads();
    if (WHOLE && t < R.G)
        for (int w = 0; w < GROUP_WAVES; ++w) all += s_next[w * R.G + t];
    const int32_t start = sum_before(t < R.G ? all : 0, s_wave);
    if (t < R.G) {
        int32_t next = start + in_front;
        for (int w = 0; w < GROUP_WAVES; ++w) {
            const int32_t c = s_next[w * R.G + t];
            s_next[w * R.G + t] = next;
            next += c;
        }
        if (blockIdx.x == 0) {
            R.ptr[t] = start;
            if (t == R.G - 1) R.ptr[R.G] = start + all;
        }
    }
    __syncthreads();
    rounds(R, lo, hi, first, [&](int64_t at, int32_t g, uint64_t same) {
        const int before = before_me(same);
        int32_t next = 0;
        if (g >= 0) {
            next = s_next[wave * R.G + g];
            R.rows[next + before] = (int32_t)(at + (threadIdx.x & 63));
        }
        settle();
        if (g >= 0 && before == 0) s_next[wave * R.G + g] = next + __popcll(same);
        settle();
    });
}

}  // namespace

extern "C" int gsplit_group_rows(gsplit_ctx *ctx, const int32_t *d_group, int64_t n_rows, int32_t n_groups, int32_t *d_group_ptr,
                                 int32_t *d_rows, void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        const char *e = op_check_group_rows(d_group, n_rows, n_groups, d_group_ptr, d_rows);
        if (!e) e = op_apart_group_rows(d_group, n_rows, n_groups, d_group_ptr, d_rows);
        if (e)
            return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_group_rows: ") + e);
        const GroupRuns runs = group_runs(n_rows, n_groups, GS_ROW_PARTS * GS_ROW_PART_BYTES / 4, ctx->n_cu);
        int bits = 0;
        while (1 << bits < n_groups) ++bits;
        const Rows R{d_group, n_rows, runs.rows_a_wave, n_groups, bits, d_group_ptr, d_rows, (int32_t *)ctx->row_part};
        const size_t lds = sizeof(int32_t) * ((size_t)GROUP_WAVES * n_groups + 2 * GT);
        if (runs.workgroups > 1) {
            GsTimeScope ts(ctx, "group_count", -1, st);
            hipLaunchKernelGGL(k_group_count, dim3(runs.workgroups), dim3(GT), sizeof(int32_t) * n_groups, st, R);
        }
        GsTimeScope ts(ctx, "group_place", -1, st);
        hipLaunchKernelGGL(runs.workgroups > 1 ? k_group_place<false> : k_group_place<true>, dim3(runs.workgroups), dim3(GT), lds, st, R);
        return GSPLIT_OK;
    });
}
