// Matrices orthogonalised by Newton-Schulz steps, and their update by orthogonalised momentum.
//
//     X = G / (|G| + eps);   A = X X^T,   B = a I + b A + c A^2,   X <- B X      for X with no more rows than columns
//
// (a tall matrix' transpose: (X X^T) X = X (X^T X)).  A and B are symmetric: only the tiles of their lower triangles are formed.
// The last product's X is read transposed on its way out of LDS (tile_core.h), so X is kept one way only.
//
// The steps start from singular values far below 1 and raise the small ones by a at most each, 485 in all: what the products round
// off small directions is raised with them, so a step's products have to be as good as float's.  Float matrix instructions reach a
// sixteenth of the half-precision ones.  All values here are below 2 (X), 4 (A) and 15 (B), so one power of two for each keeps them in
// the range of a half, and a value is held as two halves, v = hi + lo: hi = half(v), lo = half(v - hi), 22 bits and the sign of lo, as good as
// a float's 24 to a factor of 1 to 2.  A product is hi hi' + hi lo' + lo hi', three instructions; lo lo' is below 2^-24 of it.  Sums are float.
// A row keeps 32 hi and the 32 lo of the same columns side by side: a tile of 32 columns is one line of 128 bytes.
//
// What bounds them.  Large matrices: the way from the L2s into LDS, and power (16 of 2048 x 1024: A 164 us, B 81, X 214, 963 TFLOP/s
// with the matrix unit busy for 48 % at 1.9 GHz; a half-precision library product of 8192^3 reaches 1096).  Tiles of 128 x 128: with 256 x 256 X
// took 226 and A and B, triangles of few tiles, more.  Small ones: a chain of two launches and three a step, 5 to 7.5 us each,
// which matrices of at most 64 x 384 escape in one workgroup's LDS (2 x 64 x 64 and 2 x 64 x 16: 82 us by launches, 18 so).
#include <algorithm>
#include <cmath>

#include "gsplit_internal.h"
#include "newton_rules.h"
#include "op_checks.h"

namespace {

#include "tile_core.h"

typedef floatx16_t floatx16;
typedef _Float16 half;
typedef half halfx4 __attribute__((ext_vector_type(4)));
typedef half halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16;
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
// matrices start at any multiple of their elements' size
typedef floatx4 floatx4_any __attribute__((aligned(4)));
typedef bf16x4 bf16x4_any __attribute__((aligned(2)));

constexpr int NT = 256;
constexpr float SCALE_X = 0x1p14f, SCALE_A = 0x1p13f, SCALE_B = 0x1p12f;

struct Stack {
    const void *g;              // gradients, or the matrices
    float *mom;                 // momenta, or NULL
    void *out;                  // results, or the parameters
    float *master;              // bfloat16 parameters: their float copy
    int64_t at;                 // word of the working memory where the stack's starts
    int32_t count, rows, cols, m, n, mp, np;
    float scale;                // of the update
    int8_t half_g, half_out, tall;
    __host__ __device__ NewtonSize size() const { return {count, rows, cols, m, n, mp, np}; }
};
struct Call {
    Stack s[NEWTON_STACKS];
    int32_t first[NEWTON_STACKS + 1];           // first workgroup of a stack in this launch
    int32_t n;
    uint4 *work;
    // words of matrix i of the stack
    __device__ __forceinline__ uint4 *x(const Stack &s, int i, int which) const {
        return work + s.at + ((int64_t)which * s.count + i) * ((int64_t)s.mp * s.np / 4);
    }       // (a step reads one and writes the other)
    __device__ __forceinline__ uint4 *a(const Stack &s, int i, int which) const {
        return work + s.at + s.count * ((int64_t)s.mp * s.np / 2) + ((int64_t)which * s.count + i) * ((int64_t)s.mp * s.mp / 4);
    }       // 0: A, 1: B
    __device__ __forceinline__ double *sums(const Stack &s) const {
        return (double *)(work + s.at + s.count * ((int64_t)s.mp * s.np / 2 + (int64_t)s.mp * s.mp / 2));
    }
};
static_assert(sizeof(Call) <= 4096 - 256, "kernel arguments");

__device__ __forceinline__ int stack_of(const Call &C, int block) {      // (a lane a stack: a loop would wait for each)
    const int lane = threadIdx.x & 63;
    const bool before = lane + 1 < C.n && C.first[min(lane + 1, NEWTON_STACKS)] <= block;
    return __builtin_amdgcn_readfirstlane((int)__popcll(__ballot(before)));
}

// -- the matrix to be orthogonalised ------------------------------------------------------------

struct Momentum { float keep, take; int32_t nesterov; };        // m = keep m + take g

__device__ __forceinline__ float mixed(const Momentum &M, float m, float g) { return M.nesterov ? M.keep * m + M.take * g : m; }

template <class T> __device__ __forceinline__ float value(const void *p, int64_t i) { return (float)((const T *)p)[i]; }
__device__ __forceinline__ float value(const void *p, int64_t i, bool half_type) { return half_type ? value<bf16>(p, i) : value<float>(p, i); }

__device__ __forceinline__ void load4(const Stack &s, int64_t at, float (&g)[4]) {
    if (s.half_g) {
        const bf16x4 q = *(const bf16x4_any *)((const bf16 *)s.g + at);
#pragma unroll
        for (int k = 0; k < 4; ++k) g[k] = (float)q[k];
    } else {
        const floatx4 q = *(const floatx4_any *)((const float *)s.g + at);
#pragma unroll
        for (int k = 0; k < 4; ++k) g[k] = q[k];
    }
}

// momenta, and a chunk's sum of squares of what is to be orthogonalised (double: any float's square, in a fixed order)
template <bool MOMENTUM>
__global__ __launch_bounds__(NT) void k_newton_sums(Call C, Momentum M) {
    __shared__ double s_sum[NT / 64];
    const int k = stack_of(C, blockIdx.x);
    const Stack &s = C.s[k];
    const int64_t size = (int64_t)s.rows * s.cols, chunk = newton_chunk(size), slots = (size + chunk - 1) / chunk;
    const int item = blockIdx.x - C.first[k];
    const int64_t lo = item % slots * chunk, hi = min(lo + chunk, size), base = item / slots * size;
    double sum = 0.0;
    constexpr int DEEP = 4;             // pieces of four that a thread has in flight
    for (int64_t at = lo + threadIdx.x * 4; at < hi; at += NT * 4 * DEEP) {
        float g[DEEP][4] = {}, m[DEEP][4] = {};
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const int64_t i = at + d * NT * 4;
            const int n = (int)min<int64_t>(4, hi - i);
            if (n >= 4) {
                load4(s, base + i, g[d]);
                if (MOMENTUM) {
                    const floatx4 q = *(const floatx4_any *)(s.mom + base + i);
#pragma unroll
                    for (int x = 0; x < 4; ++x) m[d][x] = q[x];
                }
            } else {
                for (int x = 0; x < n; ++x) {
                    g[d][x] = value(s.g, base + i + x, s.half_g);
                    if (MOMENTUM) m[d][x] = s.mom[base + i + x];
                }
            }
        }
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const int64_t i = at + d * NT * 4;
            const int n = (int)min<int64_t>(4, hi - i);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if (MOMENTUM) m[d][x] = M.keep * m[d][x] + M.take * g[d][x];
                const double u = MOMENTUM ? mixed(M, m[d][x], g[d][x]) : g[d][x];
                sum = fma(u, u, sum);
            }
            if (!MOMENTUM) continue;
            if (n >= 4) *(floatx4_any *)(s.mom + base + i) = floatx4{m[d][0], m[d][1], m[d][2], m[d][3]};
            else
                for (int x = 0; x < n; ++x) s.mom[base + i + x] = m[d][x];
        }
    }
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) C.sums(s)[item] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

__device__ __forceinline__ floatx16 mfma_half(const halfx8 &a, const halfx8 &b, const floatx16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 zero16() {
    floatx16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}

// where column c of a row of `ld` columns lies, in halves; its lo part 32 further on
__device__ __forceinline__ int64_t place(int64_t row, int ld, int c) { return row * 2 * ld + (c >> 5) * 64 + (c & 31); }
__device__ __forceinline__ void split4(const float (&v)[4], halfx4 &hi, halfx4 &lo) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        hi[k] = (half)v[k];
        lo[k] = (half)(v[k] - (float)hi[k]);
    }
}
// four values side by side (c a multiple of 4)
__device__ __forceinline__ void put4(half *p, const float (&v)[4]) {
    halfx4 hi, lo;
    split4(v, hi, lo);
    *(halfx4 *)p = hi;
    *(halfx4 *)(p + 32) = lo;
}

// What a matrix is scaled by.  One of zeros stays one, also where an eps below 2^14 / the largest double is all of the norm; of a norm
// that is not finite nothing is left
__device__ __forceinline__ double newton_factor(double norm) {
    return norm < INFINITY ? norm > 0.0 ? fmin((double)SCALE_X / norm, 1e300) : 0.0 : NAN;
}

// X = u / (|u| + eps): a workgroup a tile of 64 x 64 of the padded matrix
template <bool MOMENTUM>
__global__ __launch_bounds__(NT) void k_newton_start(Call C, Momentum M, double eps) {
    __shared__ float s_x[64][65];
    __shared__ double s_sum[NT / 64];
    const int k = stack_of(C, blockIdx.x);
    const Stack &s = C.s[k];
    const int64_t size = (int64_t)s.rows * s.cols;
    const int rp = s.tall ? s.np : s.mp, cp = s.tall ? s.mp : s.np;
    const int tiles = rp / 64 * (cp / 64), item = blockIdx.x - C.first[k], i = item / tiles, tile = item % tiles;
    const int r0 = tile / (cp / 64) * 64, c0 = tile % (cp / 64) * 64;
    const int64_t chunk = newton_chunk(size);
    const int slots = (int)((size + chunk - 1) / chunk);
    double sum = 0.0;
    for (int j = threadIdx.x; j < slots; j += NT) sum += C.sums(s)[(int64_t)i * slots + j];
    const int c = threadIdx.x % 16 * 4, n = min(max(s.cols - c0 - c, 0), 4);
    float u[4][4] = {}, m[4][4] = {};
    if (r0 + 64 <= s.rows && c0 + 64 <= s.cols) {           // (no branch around a load in the tiles that lie inside: each would be waited for)
#pragma unroll
        for (int x = 0; x < 4; ++x) load4(s, i * size + (int64_t)(r0 + (int)threadIdx.x / 16 + 16 * x) * s.cols + c0 + c, u[x]);
        if (MOMENTUM)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const floatx4 q = *(const floatx4_any *)(s.mom + i * size + (int64_t)(r0 + (int)threadIdx.x / 16 + 16 * x) * s.cols + c0 + c);
#pragma unroll
                for (int k = 0; k < 4; ++k) m[x][k] = q[k];
            }
    } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int r = r0 + (int)threadIdx.x / 16 + 16 * x;
            const int64_t at = i * size + (int64_t)r * s.cols + c0 + c;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (r < s.rows && k < n) {
                    u[x][k] = value(s.g, at + k, s.half_g);
                    if (MOMENTUM) m[x][k] = s.mom[at + k];
                }
        }
    }
    if (MOMENTUM)
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int k = 0; k < 4; ++k) u[x][k] = mixed(M, m[x][k], u[x][k]);
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    const double norm = sqrt((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3])) + eps;
    const double factor = newton_factor(norm);
    half *const out = (half *)C.x(s, i, 0);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int r = (int)threadIdx.x / 16 + 16 * x;
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = (float)(u[x][q] * factor);
        if (s.tall) {
#pragma unroll
            for (int q = 0; q < 4; ++q) s_x[r][c + q] = v[q];
        } else {
            put4(out + place(r0 + r, cp, c0 + c), v);
        }
    }
    if (!s.tall) return;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int r = (int)threadIdx.x / 16 + 16 * x;
        const float v[4] = {s_x[c][r], s_x[c + 1][r], s_x[c + 2][r], s_x[c + 3][r]};
        put4(out + place(c0 + r, rp, r0 + c), v);
    }
}

// -- the products -----------------------------------------------------------------------------

// what a product is for: A, B, the next X, the last one
enum : int { FORM_A, FORM_B, FORM_X, FORM_LAST };
struct Step {
    float a, b, c;
    int32_t from;               // which X (0 or 1)
    float lr, keep, decay;      // the update: p = keep p - lr scale x, keep = 1 - lr decay
    const float *d_lr;
    int32_t update;
};

// 4 x 4 values across four lanes: lane i holds column i of what they held as rows
__device__ __forceinline__ float across(float x, int by) {       // the value of the lane whose number differs by the bits of `by`
    return by == 1 ? __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, true))
                   : __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, true));
}
__device__ __forceinline__ void transpose4(float (&v)[4]) {
    const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
#pragma unroll
    for (int p = 0; p < 4; p += 2) {
        const float give = odd ? v[p] : v[p + 1], got = across(give, 1);
        if (odd) v[p] = got; else v[p + 1] = got;
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const float give = high ? v[p] : v[p + 2], got = across(give, 2);
        if (high) v[p] = got; else v[p + 2] = got;
    }
}

// p[0 .. n - 1] (n <= 4) = keep p - rate v (UPDATE), or v
__device__ __forceinline__ void write_result(const Stack &s, int64_t at, const float (&v)[4], int n, bool update, float keep, float rate) {
    float y[4] = {v[0], v[1], v[2], v[3]};
    float *full = s.half_out ? s.master : (float *)s.out;
    if (n >= 4) {
        if (update) {
            const floatx4 p = *(const floatx4_any *)(full + at);
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = keep * p[k] - rate * v[k];
        }
        if (full) *(floatx4_any *)(full + at) = floatx4{y[0], y[1], y[2], y[3]};
        if (s.half_out) *(bf16x4_any *)((bf16 *)s.out + at) = bf16x4{(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
    } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (k < n) {
                if (update) y[k] = keep * full[at + k] - rate * v[k];
                if (full) full[at + k] = y[k];
                if (s.half_out) ((bf16 *)s.out)[at + k] = (bf16)y[k];
            }
    }
}

// What of C = P Q^T a workgroup forms
struct Part { int stack, i, ti, tj; };
template <int TILE, int FORM>
__device__ __forceinline__ Part part_of(const Call &C) {
    Part p;
    p.stack = stack_of(C, blockIdx.x);
    const Stack &s = C.s[p.stack];
    const int tm = s.mp / TILE, tn = s.np / TILE;
    const int tiles = FORM <= FORM_B ? tm * (tm + 1) / 2 : tm * tn;
    // consecutive tiles belong into one XCD's L2; workgroups are dealt round-robin to the eight
    int item = blockIdx.x - C.first[p.stack];
    const int of = C.first[p.stack + 1] - C.first[p.stack], whole = of / 8 * 8;
    if (item < whole) item = (item & 7) * (of / 8) + (item >> 3);
    p.i = item / tiles;
    const int tile = item % tiles;
    if (FORM <= FORM_B) {
        p.ti = (int)((sqrtf(8.f * (float)tile + 1.f) - 1.f) * 0.5f);
        while (p.ti * (p.ti + 1) / 2 > tile) --p.ti;
        while ((p.ti + 1) * (p.ti + 2) / 2 <= tile) ++p.ti;
        p.tj = tile - p.ti * (p.ti + 1) / 2;
    } else {
        p.ti = tile % tm; p.tj = tile / tm;
    }
    return p;
}
struct Factors { const uint4 *p, *q; int k; };
template <int FORM>
__device__ __forceinline__ Factors factors_of(const Call &C, const Stack &s, int i, const Step &S) {
    const uint4 *p = FORM == FORM_A ? C.x(s, i, S.from) : C.a(s, i, FORM == FORM_B ? 0 : 1);
    return {p, FORM <= FORM_B ? p : C.x(s, i, S.from), FORM == FORM_A ? s.np : s.mp};
}

// the learning rate and what a step keeps of a parameter
__device__ __forceinline__ void rates(const Step &S, float &keep, float &lr) {
    lr = S.lr; keep = S.keep;
    if (S.d_lr) {
        lr = *S.d_lr;
        keep = (float)(1.0 - (double)lr * S.decay);
    }
}

// What becomes of a wave's block of MI x MI times 32 x 32 sums at (row0, col0).  A lane has four columns side by side of one row, sixteen
// times; in `lds` (the wave's own) rows are put together, or columns where the transpose is asked for, and go out as they lie in memory.
// `mirror`: the block lies below the diagonal of a symmetric matrix and fills its mirror image too.
template <int MI, int FORM>
__device__ __forceinline__ void finish(const Call &C, const Stack &s, int i, const Step &S, const floatx16 (&acc)[MI][MI], core_u32x4 *lds, int row0, int col0,
                                       bool mirror) {
    constexpr int SIDE = 32 * MI, ROW = 8 * MI;         // rows of a block, granules of one
    const int lane = threadIdx.x & 63, l32 = lane & 31, half_ = lane >> 5;
    const auto granule = [&](int r, int g) __attribute__((always_inline)) { return lds + r * ROW + (g ^ (r & (ROW - 1))); };
    // rows of the block, four values side by side: a block's 32 columns are 4 granules of hi and 4 of lo, or 8 of floats
    const auto pair_at = [&](int r, int c, int lo) __attribute__((always_inline)) { return (halfx4 *)granule(r, c / 32 * 8 + lo * 4 + c % 32 / 8) + (c / 4 & 1); };
    const auto put_pair = [&](int r, int c, const float (&v)[4]) __attribute__((always_inline)) {
        halfx4 hi, lo;
        split4(v, hi, lo);
        *pair_at(r, c, 0) = hi;
        *pair_at(r, c, 1) = lo;
    };
    // lanes read what others have written, and write what others have read (LDS does a wave's instructions in their order)
    const auto settle = [] __attribute__((always_inline)) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    // granules of the block and of its place in memory: f(row, granule, where it lies in LDS)
    const auto granules = [&](auto f) __attribute__((always_inline)) {
        settle();
#pragma unroll
        for (int j = 0; j < SIDE * ROW / 64; ++j) {
            const int x = j * 64 + lane, r = x / ROW, g = x % ROW;
            f(r, g, granule(r, g));
        }
        settle();
    };
    // each(row, column, four values) of the block; turned: transposed
    const auto each = [&](bool turned, auto value_of, auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int a = 0; a < MI; ++a)
#pragma unroll
            for (int b = 0; b < MI; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int r = 32 * a + l32, c = 32 * b + 8 * q + 4 * half_;
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = acc[a][b][4 * q + j];
                    value_of(r, c, v);
                    if (turned) transpose4(v);
                    if (turned) f(c + (lane & 3), r & ~3, v);
                    else f(r, c, v);
                }
    };
    // rows of granules of a matrix of pairs
    const auto pairs = [&](uint4 *m, int ld, int r0, int c0) __attribute__((always_inline)) {
        return [=](int r, int g) __attribute__((always_inline)) { return (core_u32x4 *)m + (int64_t)(r0 + r) * (ld / 4) + c0 / 4 + g; };
    };
    if constexpr (FORM == FORM_LAST) {
        float keep, lr;
        rates(S, keep, lr);
        const auto scaled = [&](int, int, float (&v)[4]) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] *= 1.f / (SCALE_B * SCALE_X);
        };
        each(s.tall, scaled, [&](int r, int c, const float (&v)[4]) __attribute__((always_inline)) {
            *(floatx4 *)granule(r, c / 4) = floatx4{v[0], v[1], v[2], v[3]};
        });
        const int64_t base = (int64_t)i * s.rows * s.cols;
        const int first_r = s.tall ? col0 : row0, first_c = s.tall ? row0 : col0;
        granules([&](int r, int g, const core_u32x4 *from) __attribute__((always_inline)) {
            const int row = first_r + r, col = first_c + 4 * g;
            const floatx4 q = *(const floatx4 *)from;
            const float v[4] = {q[0], q[1], q[2], q[3]};
            if (row < s.rows && col < s.cols) write_result(s, base + (int64_t)row * s.cols + col, v, s.cols - col, S.update, keep, lr * s.scale);
        });
    } else {
        if constexpr (FORM == FORM_B) {         // A's block
            const auto at = pairs(C.a(s, i, 0), s.mp, row0, col0);
            core_u32x4 q[SIDE * ROW / 64];
            int n = 0;
            granules([&](int r, int g, core_u32x4 *) __attribute__((always_inline)) { q[n++] = *at(r, g); });
            n = 0;
            granules([&](int, int, core_u32x4 *to) __attribute__((always_inline)) { *to = q[n++]; });
        }
        const auto scaled = [&](int r, int c, float (&v)[4]) __attribute__((always_inline)) {
            if constexpr (FORM == FORM_B) {
                const halfx4 hi = *pair_at(r, c, 0), lo = *pair_at(r, c, 1);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v[j] = S.c * (SCALE_B / (SCALE_A * SCALE_A)) * v[j] + S.b * (SCALE_B / SCALE_A) * ((float)hi[j] + (float)lo[j])
                           + (row0 + r == col0 + c + j ? S.a * SCALE_B : 0.f);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] *= FORM == FORM_A ? SCALE_A / (SCALE_X * SCALE_X) : 1.f / SCALE_B;
            }
        };
        uint4 *out = FORM == FORM_X ? C.x(s, i, S.from ^ 1) : C.a(s, i, FORM == FORM_A ? 0 : 1);
        const int ld = FORM == FORM_X ? s.np : s.mp;
        const auto at = pairs(out, ld, row0, col0);
        floatx16 kept[FORM == FORM_B ? MI : 1][FORM == FORM_B ? MI : 1];         // (A's block in LDS makes room for the result)
        if constexpr (FORM == FORM_B) {
#pragma unroll
            for (int a = 0; a < MI; ++a)
#pragma unroll
                for (int b = 0; b < MI; ++b)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = acc[a][b][4 * q + j];
                        scaled(32 * a + l32, 32 * b + 8 * q + 4 * half_, v);
#pragma unroll
                        for (int j = 0; j < 4; ++j) kept[a][b][4 * q + j] = v[j];
                    }
            settle();
        }
        const auto final = [&](int r, int c, float (&v)[4]) __attribute__((always_inline)) {
            if constexpr (FORM == FORM_B) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = kept[r / 32][c / 32][c % 32 / 8 * 4 + j];
            } else {
                scaled(r, c, v);
            }
        };
        each(false, final, put_pair);
        granules([&](int r, int g, const core_u32x4 *from) __attribute__((always_inline)) { *at(r, g) = *from; });
        if (FORM != FORM_X && mirror) {
            each(true, final, put_pair);
            const auto image = pairs(out, ld, col0, row0);
            granules([&](int r, int g, const core_u32x4 *from) __attribute__((always_inline)) { *image(r, g) = *from; });
        }
    }
}

// A tile of 64 x 64 a workgroup of four waves, 64 of the contraction a stage.  The stage behind the one in work is fetched straight into
// LDS, after the one in work has been read into registers.  Contractions are short here and so are the sums: lo lo' is summed too, and
// what is small has a sum of its own (with three products and one sum, matrices of 3 x 6 were 30 times 2^-24 off).
template <int FORM>
__global__ __launch_bounds__(NT, 2) void k_newton_small(Call C, Step S) {
    constexpr int TILE = 64, SUB = 2, HALF = TILE * 8 * SUB;            // granules of a stage of one factor
    constexpr bool ACROSS = FORM >= FORM_X;
    __shared__ __attribute__((aligned(16))) core_u32x4 lds[2][2 * HALF];
    const Part part = part_of<TILE, FORM>(C);
    const Stack &s = C.s[part.stack];
    const Factors F = factors_of<FORM>(C, s, part.i, S);
    const int m0 = part.ti * TILE, n0 = part.tj * TILE, lane = threadIdx.x & 63, wave = core_wave();
    const uint32_t ld = (uint32_t)F.k * 4u, ldx = (uint32_t)s.np * 4u;          // bytes of a row
    const auto fetch = [&](int t, core_u32x4 *to) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < HALF / NT; ++j) {
            const int x = j * 4 + wave, sub = x / (TILE / 8), row = x % (TILE / 8) * 8;
            const uint32_t off = (uint32_t)along_row(lane) * ld + along_granule(x, lane) * 16;
            core_fetch((const char *)F.p + (int64_t)(m0 + row) * ld + (int64_t)(t * SUB + sub) * 128 + off, to + x * 64);
            if constexpr (ACROSS) {             // four rows of 256 bytes an instruction
                const int r = 4 * x + (lane >> 4);
                core_fetch((const char *)F.q + (int64_t)(t * SUB * 32 + r) * ldx + (int64_t)n0 * 4 + ((lane & 15) ^ (4 * (r & 3))) * 16, to + HALF + x * 64);
            } else {
                core_fetch((const char *)F.q + (int64_t)(n0 + row) * ld + (int64_t)(t * SUB + sub) * 128 + off, to + HALF + x * 64);
            }
        }
    };
    const int half_ = lane >> 5, l32 = lane & 31, wm = (wave & 1) * 32, wn = (wave >> 1) * 32;
    floatx16 acc[1][1], low = zero16();
    acc[0][0] = zero16();
    const int T = F.k / (32 * SUB), base_q = across_base<16>(HALF, wn / 4);
    fetch(0, lds[0]);
    for (int t = 0; t < T; ++t) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const core_u32x4 *now = lds[t & 1];
        halfx8 fp[SUB][2][2], fq[SUB][2][2];            // [sub-tile][16 of it][hi, lo]
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int g = 4 * q + 2 * h + half_;
                    fp[u][h][q] = __builtin_bit_cast(halfx8, now[u * TILE * 8 + along_at(wm + l32, g)]);
                    if constexpr (ACROSS) fq[u][h][q] = __builtin_bit_cast(halfx8, across_fragment<16>(now, base_q, 2 * u + h, 4 * q));
                    else fq[u][h][q] = __builtin_bit_cast(halfx8, now[HALF + u * TILE * 8 + along_at(wn + l32, g)]);
                }
        if (t + 1 < T) fetch(t + 1, lds[(t + 1) & 1]);
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                low = mfma_half(fq[u][h][1], fp[u][h][1], low);
                acc[0][0] = mfma_half(fq[u][h][0], fp[u][h][0], acc[0][0]);
                low = mfma_half(fq[u][h][1], fp[u][h][0], low);
                low = mfma_half(fq[u][h][0], fp[u][h][1], low);
            }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][0][r] += low[r];
    __syncthreads();
    finish<1, FORM>(C, s, part.i, S, acc, &lds[0][0] + wave * 32 * 8, m0 + wm, n0 + wn, part.ti != part.tj);
}

// A tile of 128 x 128 a workgroup of four waves, 64 x 64 each (tile_core.h), two workgroups a compute unit.  What is small of a product
// is summed first.
template <int FORM>
__global__ __launch_bounds__(NT, 2) void k_newton_large(Call C, Step S) {
    constexpr int TILE = NEWTON_TILE, MI = 2, WAVES = NT / 64, HALF = TILE * 8;
    constexpr bool ACROSS = FORM >= FORM_X;
    __shared__ __attribute__((aligned(16))) core_u32x4 lds[2][2 * HALF];
    const Part part = part_of<TILE, FORM>(C);
    const Stack &s = C.s[part.stack];
    const Factors F = factors_of<FORM>(C, s, part.i, S);
    const int m0 = part.ti * TILE, n0 = part.tj * TILE, lane = threadIdx.x & 63, wave = core_wave();
    const uint32_t ld = (uint32_t)F.k * 4u, ldx = (uint32_t)s.np * 4u;          // bytes of a row
    // (a lane's part of the address is the same in all of a wave's instructions: they are a multiple of sixteen rows apart)
    const uint32_t off = (uint32_t)along_row(lane) * ld + (uint32_t)along_granule(wave, lane) * 16u;
    const uint32_t off_q = ACROSS ? (uint32_t)(lane >> 5) * ldx + (uint32_t)((lane & 31) ^ (4 * ((2 * wave + (lane >> 5)) & 3))) * 16u : off;
    const char *const p0 = (const char *)F.p + (int64_t)(m0 + 8 * wave) * ld;
    const char *const q0 = (const char *)F.q + (ACROSS ? (int64_t)(2 * wave) * ldx + (int64_t)n0 * 4 : (int64_t)(n0 + 8 * wave) * ld);
    const auto fetch = [&](int t, core_u32x4 *to) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < HALF / NT; ++j) {
            core_fetch(p0 + (int64_t)(8 * WAVES * j) * ld + (int64_t)t * 128 + off, to + (WAVES * j + wave) * 64);
            const char *q = ACROSS ? q0 + (int64_t)(32 * t + 2 * WAVES * j) * ldx : q0 + (int64_t)(8 * WAVES * j) * ld + (int64_t)t * 128;
            core_fetch(q + off_q, to + HALF + (WAVES * j + wave) * 64);
        }
    };
    const int half_ = lane >> 5, l32 = lane & 31, wm = (wave & 1) * (TILE / 2), wn = (wave >> 1) * (TILE / 2);
    floatx16 acc[MI][MI];
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
        for (int b = 0; b < MI; ++b) acc[a][b] = zero16();
    struct Frag { halfx8 p[MI][2], q[MI][2]; };
    const int base_p = along_base(0, wm), base_q = ACROSS ? across_base<32>(HALF, wn / 4) : along_base(HALF, wn);
    core_contract<2, Frag>(F.k / 32, lds, fetch,
        [&](Frag &f, const core_u32x4 *now, int h) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                // (the lo of a row's 32 columns: four granules behind the hi)
#pragma unroll
                for (int a = 0; a < MI; ++a) f.p[a][q] = __builtin_bit_cast(halfx8, along_fragment(now, base_p, 2 * q + h, a));
#pragma unroll
                for (int b = 0; b < MI; ++b) {
                    if constexpr (ACROSS) f.q[b][q] = __builtin_bit_cast(halfx8, across_fragment<32>(now, base_q, h, 8 * b + 4 * q));
                    else f.q[b][q] = __builtin_bit_cast(halfx8, along_fragment(now, base_q, 2 * q + h, b));
                }
            }
        },
        [&](const Frag &f) __attribute__((always_inline)) {
#pragma unroll
            for (int x = 0; x < 3; ++x)         // hi lo', lo hi', hi hi'
#pragma unroll
                for (int a = 0; a < MI; ++a)
#pragma unroll
                    for (int b = 0; b < MI; ++b) acc[a][b] = mfma_half(f.q[b][x == 0], f.p[a][x == 1], acc[a][b]);
        });
    __syncthreads();
    finish<MI, FORM>(C, s, part.i, S, acc, &lds[0][0] + wave * 64 * 16, m0 + wm, n0 + wn, part.ti != part.tj);
}

// -- small matrices: all steps of one by one workgroup --------------------------------------------

// Sixteen waves form a block of 16 x 16 of A and of B each, and up to ONE_BLOCKS of X; what bounds this is the way through LDS and the
// barriers, about 1 us a product (with four waves 27.7 us for what takes 17.6).
// The matrices lie in LDS, rows of granules: 32 columns are 4 granules of hi and 4 of lo.  Granule p of row r holds granule
// p ^ (4 (r % 4) + r / 4 % 4): sixteen rows of one granule column lie in sixteen groups of banks, and so do the four rows of four
// granules that are read transposed.
constexpr int ONE_ROWS = 64, ONE_NT = 1024, ONE_BLOCKS = NEWTON_ONE_N / 64;
__device__ __forceinline__ int one_turn(int r) { return 4 * (r & 3) + (r >> 2 & 3); }
typedef float floatx4m __attribute__((ext_vector_type(4)));
// 16 rows of p from m0 on times 16 columns from n0 on: rows of q, or columns (ACROSS).  A lane gets four columns of one row.
template <bool ACROSS>
__device__ __forceinline__ floatx4m one_block(const core_u32x4 *p, const core_u32x4 *q, int row_p, int row_q, int m0, int n0, int k) {
    const int lane = threadIdx.x & 63, quarter = lane >> 4, rp = m0 + (lane & 15), rq = n0 + (lane & 15);
    floatx4m acc{0.f, 0.f, 0.f, 0.f}, low = acc;
#pragma unroll 2
    for (int h = 0; h < k / 32; ++h) {          // 32 columns of p: four granules of hi, four of lo
        halfx8 fp[2], fq[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int g = h * 8 + 4 * x + quarter;
            fp[x] = __builtin_bit_cast(halfx8, p[rp * row_p + (g ^ one_turn(rp))]);
            if constexpr (ACROSS) {
                // eight rows of 16 columns, one a lane (see across_fragment)
                const int r = 32 * h + 8 * quarter + ((lane & 15) >> 2), c = n0 / 32 * 8 + n0 / 16 % 2 * 2 + 4 * x + (lane >> 1 & 1);
                typedef __attribute__((address_space(3))) core_s16x4 *P;
                const auto at = [&](int row) { return (P)((__attribute__((address_space(3))) const core_u32x2 *)q + 2 * (row * row_q + (c ^ one_turn(row))) + (lane & 1)); };
                const core_u32x2 a = __builtin_bit_cast(core_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(r)));
                const core_u32x2 b = __builtin_bit_cast(core_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(r + 4)));
                fq[x] = __builtin_bit_cast(halfx8, core_u32x4{a[0], a[1], b[0], b[1]});
            } else {
                fq[x] = __builtin_bit_cast(halfx8, q[rq * row_q + (g ^ one_turn(rq))]);
            }
        }
        low = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[1], fp[1], low, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[0], fp[0], acc, 0, 0, 0);
        low = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[1], fp[0], low, 0, 0, 0);
        low = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[0], fp[1], low, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] += low[j];
    return acc;
}
__device__ __forceinline__ halfx4 *one_pair(core_u32x4 *m, int row, int r, int c, int lo) {
    return (halfx4 *)(m + r * row + ((c / 32 * 8 + lo * 4 + c % 32 / 8) ^ one_turn(r))) + (c / 4 & 1);
}

// A matrix of at most 64 x NEWTON_ONE_N (or its transpose): momentum, norm, steps and result; as above otherwise
template <bool MOMENTUM>
__global__ __launch_bounds__(ONE_NT) void k_newton_one(Call C, Momentum M, double eps, Step S, int steps) {
    extern __shared__ __attribute__((aligned(16))) core_u32x4 one_lds[];          // X [64 x np], A and B [64 x 64]
    __shared__ double s_sum[ONE_NT / 64];
    const int k = stack_of(C, blockIdx.x);
    const Stack &s = C.s[k];
    const int i = blockIdx.x - C.first[k], lane = threadIdx.x & 63, wave = core_wave();
    const int row_x = s.np / 4, row_a = ONE_ROWS / 4;
    core_u32x4 *const X = one_lds, *const A = X + ONE_ROWS * row_x, *const B = A + ONE_ROWS * row_a;
    const int64_t base = (int64_t)i * s.rows * s.cols;
    // four of the matrix' own columns a thread
    const int quads = (s.cols + 3) / 4, items = s.rows * quads;
    const auto load = [&](int x, bool update, int &r, int &c, float (&u)[4]) __attribute__((always_inline)) {
        r = x / quads; c = x % quads * 4;
        const int n = min(4, s.cols - c);
        const int64_t at = base + (int64_t)r * s.cols + c;
        float m[4] = {};
#pragma unroll
        for (int q = 0; q < 4; ++q) u[q] = 0.f;
        if (n == 4) {
            load4(s, at, u);
            if (MOMENTUM) {
                floatx4 f = *(const floatx4_any *)(s.mom + at);
                if (update) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) f[q] = M.keep * f[q] + M.take * u[q];
                    *(floatx4_any *)(s.mom + at) = f;
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) m[q] = f[q];
            }
        } else {
            for (int q = 0; q < n; ++q) {
                u[q] = value(s.g, at + q, s.half_g);
                if (MOMENTUM) {
                    m[q] = s.mom[at + q];
                    if (update) s.mom[at + q] = m[q] = M.keep * m[q] + M.take * u[q];
                }
            }
        }
        if (MOMENTUM)
#pragma unroll
            for (int q = 0; q < 4; ++q) u[q] = mixed(M, m[q], u[q]);
    };
    constexpr int KEPT = 4;             // items that a thread keeps; more are read again
    float kept[KEPT][4];
    double sum = 0.0;
    const auto add = [&](const float (&u)[4]) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 4; ++q) sum = fma((double)u[q], (double)u[q], sum);
    };
#pragma unroll
    for (int j = 0; j < KEPT; ++j) {
        int r, c;
#pragma unroll
        for (int q = 0; q < 4; ++q) kept[j][q] = 0.f;
        if (j * ONE_NT + (int)threadIdx.x < items) load(j * ONE_NT + threadIdx.x, true, r, c, kept[j]);
        add(kept[j]);
    }
    for (int x = KEPT * ONE_NT + threadIdx.x; x < items; x += ONE_NT) {
        int r, c;
        float u[4];
        load(x, true, r, c, u);
        add(u);
    }
    for (int x = threadIdx.x; x < ONE_ROWS * row_x; x += ONE_NT) X[x] = core_u32x4{0u, 0u, 0u, 0u};
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    sum = s_sum[0];
    for (int w = 1; w < ONE_NT / 64; ++w) sum += s_sum[w];
    const double norm = sqrt(sum) + eps;
    const double factor = newton_factor(norm);
    const auto place_x = [&](int r, int c, const float (&u)[4]) __attribute__((always_inline)) {
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = (float)(u[q] * factor);
        if (!s.tall) {
            halfx4 hi, lo;
            split4(v, hi, lo);
            *one_pair(X, row_x, r, c, 0) = hi;
            *one_pair(X, row_x, r, c, 1) = lo;
        } else {                        // the transpose: a value by itself
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (c + q >= s.cols) continue;
                const half hi = (half)v[q];
                ((half *)one_pair(X, row_x, c + q, r & ~3, 0))[r & 3] = hi;
                ((half *)one_pair(X, row_x, c + q, r & ~3, 1))[r & 3] = (half)(v[q] - (float)hi);
            }
        }
    };
#pragma unroll
    for (int j = 0; j < KEPT; ++j) {
        const int x = j * ONE_NT + threadIdx.x;
        if (x < items) place_x(x / quads, x % quads * 4, kept[j]);
    }
    for (int x = KEPT * ONE_NT + threadIdx.x; x < items; x += ONE_NT) {
        int r, c;
        float u[4];
        load(x, false, r, c, u);
        place_x(r, c, u);
    }
    __syncthreads();
    float keep = 0.f, lr = 0.f;
    rates(S, keep, lr);
    const int m0 = (wave & 3) * 16, n0 = (wave >> 2) * 16, r = lane & 15, c = 4 * (lane >> 4);
    const auto put = [&](core_u32x4 *m, int row, int r, int c, const float (&v)[4]) __attribute__((always_inline)) {
        halfx4 hi, lo;
        split4(v, hi, lo);
        *one_pair(m, row, r, c, 0) = hi;
        *one_pair(m, row, r, c, 1) = lo;
    };
    for (int step = 0; step < steps; ++step) {
        floatx4m acc = one_block<false>(X, X, row_x, row_x, m0, n0, s.np);
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = acc[j] * (SCALE_A / (SCALE_X * SCALE_X));
        put(A, row_a, m0 + r, n0 + c, v);
        __syncthreads();
        acc = one_block<false>(A, A, row_a, row_a, m0, n0, ONE_ROWS);
        const halfx4 hi = *one_pair(A, row_a, m0 + r, n0 + c, 0), lo = *one_pair(A, row_a, m0 + r, n0 + c, 1);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = S.c * (SCALE_B / (SCALE_A * SCALE_A)) * acc[j] + S.b * (SCALE_B / SCALE_A) * ((float)hi[j] + (float)lo[j])
                   + (m0 + r == n0 + c + j ? S.a * SCALE_B : 0.f);
        put(B, row_a, m0 + r, n0 + c, v);
        __syncthreads();
        // columns n0, n0 + 64 .. of X, which stay in registers until all waves have read theirs
        floatx4m next[ONE_BLOCKS];
#pragma unroll
        for (int b = 0; b < ONE_BLOCKS; ++b)
            if (64 * b < s.np) next[b] = one_block<true>(B, X, row_a, row_x, m0, n0 + 64 * b, ONE_ROWS);
        __syncthreads();
#pragma unroll
        for (int b = 0; b < ONE_BLOCKS; ++b) {
            if (64 * b >= s.np) break;
            int row = m0 + r, col = n0 + 64 * b + c;
            if (step + 1 < steps) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = next[b][j] * (1.f / SCALE_B);
                put(X, row_x, row, col, v);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = next[b][j] * (1.f / (SCALE_B * SCALE_X));
                if (s.tall) {
                    transpose4(v);
                    const int t = row & ~3;
                    row = col + (lane & 3); col = t;
                }
                if (row < s.rows && col < s.cols) write_result(s, base + (int64_t)row * s.cols + col, v, s.cols - col, S.update, keep, lr * s.scale);
            }
        }
        __syncthreads();
    }
}

// -- launches ---------------------------------------------------------------------------------

struct Settings {
    int32_t steps;
    float a, b, c;
    double eps;
    Momentum mom;
    float lr, keep, decay;
    const float *d_lr;
    bool update;
};

template <class Count>
int deal(Call &C, Count count) {
    C.first[0] = 0;
    for (int k = 0; k < C.n; ++k) C.first[k + 1] = C.first[k] + (int32_t)count(C.s[k].size());
    return C.first[C.n];
}

void steps(gsplit_ctx *ctx, Call &C, const Settings &S, int tile, hipStream_t st) {
    const auto launch = [&](const char *name, auto large, auto small, const Step &step) {
        GsTimeScope ts(ctx, name, -1, st);
        if (tile == NEWTON_TILE) hipLaunchKernelGGL(large, dim3(C.first[C.n]), dim3(NT), 0, st, C, step);
        else hipLaunchKernelGGL(small, dim3(C.first[C.n]), dim3(NT), 0, st, C, step);
    };
    const auto lower = [&](const NewtonSize &z) { return z.count * newton_tiles_a(z, tile); };
    const auto all = [&](const NewtonSize &z) { return z.count * newton_tiles_x(z, tile); };
    for (int k = 0; k < S.steps; ++k) {
        const Step step{S.a, S.b, S.c, k & 1, S.lr, S.keep, S.decay, S.d_lr, S.update};
        deal(C, lower);
        launch("newton_a", k_newton_large<FORM_A>, k_newton_small<FORM_A>, step);
        launch("newton_b", k_newton_large<FORM_B>, k_newton_small<FORM_B>, step);
        deal(C, all);
        if (k + 1 < S.steps) launch("newton_x", k_newton_large<FORM_X>, k_newton_small<FORM_X>, step);
        else launch("newton_last", k_newton_large<FORM_LAST>, k_newton_small<FORM_LAST>, step);
    }
}

// fill(stack, tensor, element where its matrices start)
template <class Size, class Fill>
void run_newton(gsplit_ctx *ctx, int64_t n_tensors, const Settings &S, void *work, Size size, Fill fill, hipStream_t st) {
    newton_groups(n_tensors, size, [&](const NewtonStack *in, int n, int tile) {
        Call C{};
        C.n = n;
        C.work = (uint4 *)work;
        int64_t at = 0;
        for (int k = 0; k < n; ++k) {
            const NewtonSize &z = in[k].size;
            Stack &s = C.s[k];
            s.at = at;
            s.count = (int32_t)z.count; s.rows = z.rows; s.cols = z.cols; s.m = z.m; s.n = z.n; s.mp = z.mp; s.np = z.np;
            s.tall = z.rows > z.cols;
            fill(s, in[k].tensor, in[k].first * z.rows * z.cols);
            at += newton_words(z, tile);
        }
        if (tile == NEWTON_ONE) {
            int np = 0;
            for (int k = 0; k < n; ++k) np = std::max(np, C.s[k].np);
            deal(C, [](const NewtonSize &z) { return z.count; });
            const Step step{S.a, S.b, S.c, 0, S.lr, S.keep, S.decay, S.d_lr, S.update};
            GsTimeScope ts(ctx, "newton_one", -1, st);
            hipLaunchKernelGGL(S.update ? k_newton_one<true> : k_newton_one<false>, dim3(C.first[n]), dim3(ONE_NT), (np + 2 * 64) * 64 * 4, st, C, S.mom,
                               S.eps, step, S.steps);
            return;
        }
        deal(C, [](const NewtonSize &z) { return z.count * newton_slots(z); });
        {
            GsTimeScope ts(ctx, "newton_sums", -1, st);
            hipLaunchKernelGGL(S.update ? k_newton_sums<true> : k_newton_sums<false>, dim3(C.first[n]), dim3(NT), 0, st, C, S.mom);
        }
        deal(C, [](const NewtonSize &z) { return z.count * newton_tiles_x(z, 64); });
        {
            GsTimeScope ts(ctx, "newton_start", -1, st);
            hipLaunchKernelGGL(S.update ? k_newton_start<true> : k_newton_start<false>, dim3(C.first[n]), dim3(NT), 0, st, C, S.mom, S.eps);
        }
        steps(ctx, C, S, tile, st);
    });
}

struct Shape { int64_t count; int32_t rows, cols; };
template <class Tensor> Shape shape_of(const Tensor &t) { return {t.count, t.rows, t.cols}; }

template <class Tensor>
int64_t work_bytes(const Tensor *t, int64_t n_tensors) {
    int64_t most = 0;
    newton_groups(n_tensors, [&](int64_t i) { return shape_of(t[i]); }, [&](const NewtonStack *in, int n, int tile) {
        int64_t words = 0;
        for (int k = 0; k < n; ++k) words += newton_words(in[k].size, tile);
        most = std::max(most, words);
    });
    return most * 16;
}

template <class T> void *moved(T *p, int64_t elements, int32_t dtype) {
    return p ? (char *)p + elements * (dtype == GSPLIT_BF16 ? 2 : 4) : nullptr;
}

}  // namespace

extern "C" int64_t gsplit_orthogonalize_work(const gsplit_matrix_tensor *t, int64_t n_tensors) {
    return op_check_matrices(t, n_tensors) ? GSPLIT_EINVAL : work_bytes(t, n_tensors);
}

extern "C" int gsplit_orthogonalize(gsplit_ctx *ctx, const gsplit_newton_config *c, const gsplit_matrix_tensor *t, int64_t n_tensors,
                                    void *d_work, void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        const char *e = op_check_newton(c);
        if (!e) e = op_check_matrices(t, n_tensors);
        if (!e) e = op_check_work(d_work, work_bytes(t, n_tensors));
        if (e) return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_orthogonalize: ") + e);
        Settings S{};
        S.steps = c->steps; S.a = (float)c->a; S.b = (float)c->b; S.c = (float)c->c; S.eps = c->eps;
        run_newton(ctx, n_tensors, S, d_work, [&](int64_t i) { return shape_of(t[i]); }, [&](Stack &s, int64_t i, int64_t first) {
            s.g = moved((char *)t[i].d_in, first, t[i].in_dtype);
            s.out = moved((char *)t[i].d_out, first, t[i].out_dtype);
            s.half_g = t[i].in_dtype == GSPLIT_BF16; s.half_out = t[i].out_dtype == GSPLIT_BF16;
        }, st);
        return (int)GSPLIT_OK;
    });
}

extern "C" int64_t gsplit_muon_work(const gsplit_muon_tensor *t, int64_t n_tensors) {
    return op_check_muon_tensors(t, n_tensors) ? GSPLIT_EINVAL : work_bytes(t, n_tensors);
}

extern "C" int gsplit_muon_step(gsplit_ctx *ctx, const gsplit_muon_config *c, const gsplit_muon_tensor *t, int64_t n_tensors,
                                void *d_work, void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        const char *e = op_check_muon(c);
        if (!e) e = op_check_muon_tensors(t, n_tensors);
        if (!e) e = op_check_work(d_work, work_bytes(t, n_tensors));
        if (e) return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_muon_step: ") + e);
        Settings S{};
        S.steps = c->newton.steps; S.a = (float)c->newton.a; S.b = (float)c->newton.b; S.c = (float)c->newton.c; S.eps = c->newton.eps;
        S.mom = {(float)c->momentum, (float)(1.0 - c->momentum), c->nesterov != 0};
        S.lr = (float)c->lr; S.keep = (float)(1.0 - c->lr * c->weight_decay); S.decay = (float)c->weight_decay; S.d_lr = c->d_lr;
        S.update = true;
        run_newton(ctx, n_tensors, S, d_work, [&](int64_t i) { return shape_of(t[i]); }, [&](Stack &s, int64_t i, int64_t first) {
            s.g = moved((char *)t[i].d_grad, first, t[i].grad_dtype);
            s.mom = t[i].d_momentum + first;
            s.out = moved((char *)t[i].d_param, first, t[i].param_dtype);
            s.master = t[i].d_master ? t[i].d_master + first : nullptr;
            s.half_g = t[i].grad_dtype == GSPLIT_BF16; s.half_out = t[i].param_dtype == GSPLIT_BF16;
            const double r = t[i].rows, q = t[i].cols;
            s.scale = (float)(c->scaling == GSPLIT_MUON_SHAPE ? std::sqrt(std::max(1.0, q / r))
                              : c->scaling == GSPLIT_MUON_RMS ? 0.2 * std::sqrt(std::max(r, q)) : 1.0);
        }, st);
        return (int)GSPLIT_OK;
    });
}
