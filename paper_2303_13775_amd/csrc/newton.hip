// Matrices orthogonalised by Newton-Schulz steps, and their update by orthogonalised momentum.
//
//     X = G / (|G| + eps);   A = X X^T,   B = a I + b A + c A^2,   X <- B X      for X with no more rows than columns
//
// (a tall matrix' transpose: (X X^T) X = X (X^T X)).  A and B are symmetric: only the tiles of their lower triangles are formed.
// All three products have both factors' contraction along the rows: X is kept with its transpose beside it.
//
// The steps start from singular values far below 1 and raise the small ones by a at most each, 485 in all: what the products round
// off small directions is raised with them, so a step's products have to be as good as float's.  Float matrix instructions reach a
// sixteenth of the half-precision ones.  All values here are below 2 (X), 4 (A) and 15 (B), so one power of two for each keeps them in
// the range of a half, and a value is held as two halves, v = hi + lo: hi = half(v), lo = half(v - hi), 22 bits and the sign of lo, as good as
// a float's 24 to a factor of 1 to 2.  A product is hi hi' + hi lo' + lo hi', three instructions; lo lo' is below 2^-24 of it.  Sums are float.
// A row keeps 32 hi and the 32 lo of the same columns side by side: a tile of 32 columns is one line of 128 bytes.
#include <algorithm>
#include <cmath>

#include "gsplit_internal.h"
#include "newton_rules.h"
#include "op_checks.h"

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
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
    }       // which: 0, 1 X and its transpose, 2, 3 the other pair
    __device__ __forceinline__ uint4 *a(const Stack &s, int i, int which) const {
        return work + s.at + s.count * (int64_t)s.mp * s.np + ((int64_t)which * s.count + i) * ((int64_t)s.mp * s.mp / 4);
    }
    __device__ __forceinline__ double *sums(const Stack &s) const { return (double *)(work + s.at + s.count * ((int64_t)s.mp * s.np + (int64_t)s.mp * s.mp / 2)); }
};
static_assert(sizeof(Call) <= 4096 - 256, "kernel arguments");

__device__ __forceinline__ int stack_of(const Call &C, int block) {
    int k = 0;
    while (k + 1 < C.n && C.first[k + 1] <= block) ++k;
    return k;
}

// -- the matrix to be orthogonalised ------------------------------------------------------------

struct Momentum { float keep, take; int32_t nesterov; };        // m = keep m + take g

__device__ __forceinline__ float mixed(const Momentum &M, float m, float g) { return M.nesterov ? M.keep * m + M.take * g : m; }

template <class T> __device__ __forceinline__ float value(const void *p, int64_t i) { return (float)((const T *)p)[i]; }
__device__ __forceinline__ float value(const void *p, int64_t i, bool half_type) { return half_type ? value<bf16>(p, i) : value<float>(p, i); }

// momenta, and a chunk's sum of squares of what is to be orthogonalised (double: any float's square, in a fixed order)
template <bool MOMENTUM>
__global__ __launch_bounds__(NT) void k_newton_sums(Call C, Momentum M) {
    __shared__ double s_sum[NT / 64];
    const Stack &s = C.s[stack_of(C, blockIdx.x)];
    const int64_t size = (int64_t)s.rows * s.cols, slots = (size + NEWTON_CHUNK - 1) / NEWTON_CHUNK;
    const int64_t item = blockIdx.x - C.first[stack_of(C, blockIdx.x)];
    const int64_t lo = item % slots * NEWTON_CHUNK, hi = min(lo + NEWTON_CHUNK, size), base = item / slots * size;
    double sum = 0.0;
    for (int64_t i = lo + threadIdx.x * 4; i < hi; i += NT * 4) {
        float g[4] = {}, m[4] = {};
        const int n = (int)min<int64_t>(4, hi - i);
        if (n == 4) {
            if (s.half_g) {
                const bf16x4 q = *(const bf16x4_any *)((const bf16 *)s.g + base + i);
                for (int k = 0; k < 4; ++k) g[k] = (float)q[k];
            } else {
                const floatx4 q = *(const floatx4_any *)((const float *)s.g + base + i);
                for (int k = 0; k < 4; ++k) g[k] = q[k];
            }
            if (MOMENTUM) {
                floatx4 q = *(const floatx4_any *)(s.mom + base + i);
                for (int k = 0; k < 4; ++k) q[k] = m[k] = M.keep * q[k] + M.take * g[k];
                *(floatx4_any *)(s.mom + base + i) = q;
            }
        } else {
            for (int k = 0; k < n; ++k) {
                g[k] = value(s.g, base + i + k, s.half_g);
                if (MOMENTUM) s.mom[base + i + k] = m[k] = M.keep * s.mom[base + i + k] + M.take * g[k];
            }
        }
        for (int k = 0; k < 4; ++k) {
            const double u = MOMENTUM ? mixed(M, m[k], g[k]) : g[k];
            sum = fma(u, u, sum);
        }
    }
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) C.sums(s)[item] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

__device__ __forceinline__ void split(float v, half &hi, half &lo) {
    hi = (half)v;
    lo = (half)(v - (float)hi);
}
// where column c of a row of `ld` columns lies, in halves; its lo part 32 further on
__device__ __forceinline__ int64_t place(int64_t row, int ld, int c) { return row * 2 * ld + (c >> 5) * 64 + (c & 31); }
// four values side by side (c a multiple of 4)
__device__ __forceinline__ void put4(half *p, const float (&v)[4]) {
    halfx4 hi, lo;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        half h, l;
        split(v[k], h, l);
        hi[k] = h; lo[k] = l;
    }
    *(halfx4 *)p = hi;
    *(halfx4 *)(p + 32) = lo;
}

// X = u / (|u| + eps), and its transpose: a workgroup a tile of 64 x 64 of the padded matrix
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
    const int slots = (int)((size + NEWTON_CHUNK - 1) / NEWTON_CHUNK);
    double sum = 0.0;
    for (int j = threadIdx.x; j < slots; j += NT) sum += C.sums(s)[(int64_t)i * slots + j];
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    const double norm = sqrt((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3])) + eps;
    // a matrix of zeros stays one; of a norm that is not finite nothing is left
    const double factor = norm < INFINITY ? norm > 0.0 ? (double)SCALE_X / norm : 0.0 : NAN;
    const int c = threadIdx.x % 16 * 4;
    for (int r = threadIdx.x / 16; r < 64; r += NT / 16) {
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float u = 0.f;
            if (r0 + r < s.rows && c0 + c + q < s.cols) {
                const int64_t at = i * size + (int64_t)(r0 + r) * s.cols + c0 + c + q;
                u = value(s.g, at, s.half_g);
                if (MOMENTUM) u = mixed(M, s.mom[at], u);
            }
            s_x[r][c + q] = v[q] = (float)(u * factor);
        }
        put4((half *)C.x(s, i, s.tall ? 1 : 0) + place(r0 + r, cp, c0 + c), v);
    }
    __syncthreads();
    for (int r = threadIdx.x / 16; r < 64; r += NT / 16) {
        const float v[4] = {s_x[c][r], s_x[c + 1][r], s_x[c + 2][r], s_x[c + 3][r]};
        put4((half *)C.x(s, i, s.tall ? 0 : 1) + place(c0 + r, rp, r0 + c), v);
    }
}

// -- the products -----------------------------------------------------------------------------

// what a product is for: A, B, the next X, the last one
enum : int { FORM_A, FORM_B, FORM_X, FORM_LAST };
struct Step {
    float a, b, c;
    int32_t from;               // which pair of X (0 or 2)
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

// C = P Q^T of padded matrices, a tile of TILE x TILE a workgroup of four waves, SUB x 32 of the contraction a stage.  The stage
// behind the one in work is fetched straight into LDS, after the one in work has been read into registers.
template <int TILE, int SUB, int FORM>
__global__ __launch_bounds__(NT, 2) void k_newton(Call C, Step S) {
    constexpr int MI = TILE / 64, STAGE = 2 * TILE * 8 * SUB, LOADS = STAGE / NT;
    __shared__ __attribute__((aligned(16))) uint4 lds[2][STAGE];
    const int block = blockIdx.x, k = stack_of(C, block);
    const Stack &s = C.s[k];
    const int tm = s.mp / TILE, tn = s.np / TILE;
    const int tiles = FORM <= FORM_B ? tm * (tm + 1) / 2 : tm * tn;
    // consecutive tiles belong into one XCD's L2; workgroups are dealt round-robin to the eight
    int item = block - C.first[k];
    const int of = C.first[k + 1] - C.first[k], whole = of / 8 * 8;
    if (item < whole) item = (item & 7) * (of / 8) + (item >> 3);
    const int i = item / tiles, tile = item % tiles;
    int ti, tj;
    if (FORM <= FORM_B) {
        ti = (int)((sqrtf(8.f * (float)tile + 1.f) - 1.f) * 0.5f);
        while (ti * (ti + 1) / 2 > tile) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
        tj = tile - ti * (ti + 1) / 2;
    } else {
        ti = tile % tm; tj = tile / tm;
    }
    const int m0 = ti * TILE, n0 = tj * TILE;
    const uint4 *P = FORM == FORM_A ? C.x(s, i, S.from) : C.a(s, i, FORM == FORM_B ? 0 : 1);
    const uint4 *Q = FORM == FORM_A ? P : FORM == FORM_B ? P : C.x(s, i, S.from + 1);
    const int K = FORM == FORM_A ? s.np : s.mp;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    // granule p of row r of LDS holds granule p ^ (r / 2) % 8 of the row: 16 rows of one granule column lie in 16 bank groups
    const auto turn = [](int row) __attribute__((always_inline)) { return (row >> 1) & 7; };
    // a wave's instruction fetches eight rows of 128 bytes, a granule a lane
    const uint32_t ld = (uint32_t)K * 4u;               // bytes of a row
    const auto fetch = [&](int t, int stage) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int x = j * (NT / 64) + wave;         // eight rows of one sub-tile
            const int sub = x / (2 * TILE / 8), row = x % (2 * TILE / 8) * 8;
            const char *base = (const char *)(row < TILE ? P : Q) + (int64_t)(row < TILE ? m0 + row : n0 + row - TILE) * ld
                               + (int64_t)(t * SUB + sub) * 128;
            const uint32_t off = (uint32_t)(lane >> 3) * ld + (uint32_t)(((lane & 7) ^ turn((row & 8) + (lane >> 3))) * 16);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + off),
                                             (__attribute__((address_space(3))) void *)&lds[stage][x * 64], 16, 0, 0);
        }
    };
    const int half_ = lane >> 5, l32 = lane & 31, wm = (wave & 1) * (TILE / 2), wn = (wave >> 1) * (TILE / 2);
    floatx16 acc[MI][MI];
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
        for (int b = 0; b < MI; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;
    const int T = K / (32 * SUB);
    fetch(0, 0);
    for (int t = 0; t < T; ++t) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const uint4 *now = lds[t & 1];
        halfx8 fp[SUB][2][MI][2], fq[SUB][2][MI][2];            // [sub-tile][16 of it][block][hi, lo]
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int a = 0; a < MI; ++a)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int rp = wm + 32 * a + l32, rq = wn + 32 * a + l32, g = 4 * q + 2 * h + half_;
                        fp[u][h][a][q] = __builtin_bit_cast(halfx8, now[(u * 2 * TILE + rp) * 8 + (g ^ turn(rp))]);
                        fq[u][h][a][q] = __builtin_bit_cast(halfx8, now[(u * 2 * TILE + TILE + rq) * 8 + (g ^ turn(rq))]);
                    }
        if (t + 1 < T) fetch(t + 1, (t + 1) & 1);
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < 3; ++q)
#pragma unroll
                    for (int a = 0; a < MI; ++a)
#pragma unroll
                        for (int b = 0; b < MI; ++b)
                            acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fq[u][h][b][q == 1], fp[u][h][a][q == 2], acc[a][b], 0, 0, 0);
    }

    float lr = S.lr, keep = S.keep;
    if (FORM == FORM_LAST && S.d_lr) {
        lr = *S.d_lr;
        keep = (float)(1.0 - (double)lr * S.decay);
    }
    // a lane has four columns side by side of one row, sixteen of a block
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
        for (int b = 0; b < MI; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int row = m0 + wm + 32 * a + l32, col = n0 + wn + 32 * b + 8 * q + 4 * half_;
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = acc[a][b][4 * q + j];
                // what the transposed place gets: four rows side by side of one column, lane % 4 of the four
                const int trow = row & ~3, tcol = col + (lane & 3);
                if (FORM == FORM_A || FORM == FORM_B) {
                    half *out = (half *)C.a(s, i, FORM == FORM_A ? 0 : 1);
                    if (FORM == FORM_A) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] *= SCALE_A / (SCALE_X * SCALE_X);
                    } else {
                        const half *A = (const half *)P + place(row, s.mp, col);
                        const halfx4 hi = *(const halfx4 *)A, lo = *(const halfx4 *)(A + 32);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            v[j] = S.c * (SCALE_B / (SCALE_A * SCALE_A)) * v[j] + S.b * (SCALE_B / SCALE_A) * ((float)hi[j] + (float)lo[j])
                                   + (row == col + j ? S.a * SCALE_B : 0.f);
                    }
                    put4(out + place(row, s.mp, col), v);
                    if (ti != tj) {
                        transpose4(v);
                        put4(out + place(tcol, s.mp, trow), v);
                    }
                } else if (FORM == FORM_X) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] *= 1.f / SCALE_B;
                    put4((half *)C.x(s, i, S.from ^ 2) + place(row, s.np, col), v);
                    transpose4(v);
                    put4((half *)C.x(s, i, (S.from ^ 2) + 1) + place(tcol, s.mp, trow), v);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] *= 1.f / (SCALE_B * SCALE_X);
                    const int64_t base = (int64_t)i * s.rows * s.cols;
                    if (s.tall) {
                        transpose4(v);
                        if (tcol < s.n && trow < s.m) write_result(s, base + (int64_t)tcol * s.cols + trow, v, s.m - trow, S.update, keep, lr * s.scale);
                    } else if (row < s.m && col < s.n) {
                        write_result(s, base + (int64_t)row * s.cols + col, v, s.n - col, S.update, keep, lr * s.scale);
                    }
                }
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

template <int TILE, int SUB>
void steps(gsplit_ctx *ctx, Call &C, const Settings &S, hipStream_t st) {
    const auto launch = [&](const char *name, auto kernel, const Step &step) {
        GsTimeScope ts(ctx, name, -1, st);
        hipLaunchKernelGGL(kernel, dim3(C.first[C.n]), dim3(NT), 0, st, C, step);
    };
    const auto lower = [](const NewtonSize &z) { return z.count * newton_tiles_a(z, TILE); };
    const auto all = [](const NewtonSize &z) { return z.count * newton_tiles_x(z, TILE); };
    for (int k = 0; k < S.steps; ++k) {
        const Step step{S.a, S.b, S.c, 2 * (k & 1), S.lr, S.keep, S.decay, S.d_lr, S.update};
        deal(C, lower);
        launch("newton_a", k_newton<TILE, SUB, FORM_A>, step);
        launch("newton_b", k_newton<TILE, SUB, FORM_B>, step);
        deal(C, all);
        if (k + 1 < S.steps) launch("newton_x", k_newton<TILE, SUB, FORM_X>, step);
        else launch("newton_last", k_newton<TILE, SUB, FORM_LAST>, step);
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
            at += newton_words(z);
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
        if (tile == 128) steps<128, 1>(ctx, C, S, st);
        else steps<64, 2>(ctx, C, S, st);
    });
}

struct Shape { int64_t count; int32_t rows, cols; };
template <class Tensor> Shape shape_of(const Tensor &t) { return {t.count, t.rows, t.cols}; }

template <class Tensor>
int64_t work_bytes(const Tensor *t, int64_t n_tensors) {
    int64_t most = 0;
    newton_groups(n_tensors, [&](int64_t i) { return shape_of(t[i]); }, [&](const NewtonStack *in, int n, int) {
        int64_t words = 0;
        for (int k = 0; k < n; ++k) words += newton_words(in[k].size);
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
