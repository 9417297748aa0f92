// The grouped products of bfloat16 rows that start at multiples of 16 bytes, in tiles of 256 x 256 (included by grouped.hip inside its
// anonymous namespace): operands go straight into LDS (tile_core.h), eight waves of 128 x 64, one workgroup a compute unit.  Tiles of
// this size because of the L2s: a tile of 128 x 128 asks them for 64 bytes a clock and compute unit while the matrix unit works, which is
// all they have; this one for 32.  65536 rows of 64 groups 2048 x 2048: 650 us, matrix unit busy for 43 % at 2.0 GHz (tiles of 128 x 128 through
// registers 1008; a ring of four stages of 32 instead of two of 64 790 against 735 then: rows of 64 bytes).
#pragma once

constexpr int CT = 512, CORE_TILE = 256, CORE_HALF = CORE_TILE * 8;        // threads; granules of a stage of one operand

__device__ const core_u32x4 core_zeros = {0u, 0u, 0u, 0u};         // what lies past an operand's edge

struct CoreFrag { core_u32x4 p[4], q[2]; };
struct CoreSums {
    floatx16 s[4][2];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b) s[a][b] = zero16();
    }
    __device__ __forceinline__ void multiply(const CoreFrag &f) {
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                s[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, f.q[b]), __builtin_bit_cast(bf16x8_t, f.p[a]), s[a][b], 0, 0, 0);
    }
};
// a wave's part of the tile: the two waves of a SIMD lie in different halves of the rows, so that a tile of few rows takes half the time
__device__ __forceinline__ int core_wm() { return (core_wave() >> 2) * 128; }
__device__ __forceinline__ int core_wn() { return (core_wave() & 3) * 64; }
// lanes read what others have written, and write what others have read (LDS does a wave's instructions in their order)
__device__ __forceinline__ void core_settle() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// c[r] = a[r] W[g] (+ bias), W as K x N, or as N x K (TRANSPOSED)
template <bool TRANSPOSED>
__global__ __launch_bounds__(CT) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_grouped_rows_core(RowsArgs A) {
    constexpr int T = CORE_TILE;
    __shared__ __attribute__((aligned(16))) core_u32x4 lds[2][2 * CORE_HALF];
    __shared__ int s_row[T];
    __shared__ __attribute__((aligned(16))) float s_bias[T];
    const int lane = threadIdx.x & 63, wave = core_wave(), half = lane >> 5, l32 = lane & 31, wm = core_wm(), wn = core_wn();
    const int64_t room = (A.tiles_m * A.tiles_n + 7) / 8 * 8;
    for (int64_t block = blockIdx.x; block < room; block += gridDim.x) {
        Spot s;
        if (!find_spot<false>(A.ptr, A.G, A.list.n, T, block, A.tiles_n, s)) continue;
        const int n0 = s.side * T;
        if (threadIdx.x < T) {
            const int t = threadIdx.x;
            s_row[t] = t < s.rows ? A.list.at(s.first + t) : -1;
            s_bias[t] = A.bias && n0 + t < A.N ? A.bias[(int64_t)s.g * A.N + n0 + t] : 0.f;
        }
        __syncthreads();
        const char *w = (const char *)A.w + (int64_t)s.g * A.K * A.N * 2;
        const char *pa[4];
        const int ga = along_granule(wave, lane) * 8;           // its first column of the contraction in a stage
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = 8 * (8 * j + wave) + along_row(lane);
            pa[j] = (const char *)A.a + row_at(max(s_row[i < s.rows ? i : 0], 0), A.lda) * 2 + ga * 2;
        }
        // W: rows of 256 columns, two an instruction; or eight rows of 64 of the contraction
        const int gb = TRANSPOSED ? ga : ((lane & 31) ^ (4 * ((2 * wave + half) & 3))) * 8;
        const uint32_t off = (uint32_t)(TRANSPOSED ? along_row(lane) : half) * A.ldw * 2 + gb * 2;
        const bool cut = n0 + T > A.N;
        const auto fetch = [&](int t, core_u32x4 *to) __attribute__((always_inline)) {
            const char *const w0 = TRANSPOSED ? w + (int64_t)n0 * A.ldw * 2 + (int64_t)t * 128 : w + (int64_t)t * 64 * A.ldw * 2 + (int64_t)n0 * 2;
            constexpr int ROWS = TRANSPOSED ? 8 : 2;        // of W, an instruction
            if (!cut && (t + 1) * 64 <= A.K) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    core_fetch(pa[j] + (int64_t)t * 128, to + (8 * j + wave) * 64);
                    core_fetch(w0 + (int64_t)(ROWS * (8 * j + wave)) * A.ldw * 2 + off, to + CORE_HALF + (8 * j + wave) * 64);
                }
            } else {            // zeros past the edges; rows of W past its last one: that one
                const char *const zeros = (const char *)&core_zeros;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int row = ROWS * (8 * j + wave);
                    core_fetch(t * 64 + ga < A.K ? pa[j] + (int64_t)t * 128 : zeros, to + (8 * j + wave) * 64);
                    const char *q = w0 + (int64_t)row * A.ldw * 2 + off;
                    if constexpr (TRANSPOSED) {
                        q = w0 + (int64_t)(min(n0 + row + along_row(lane), A.N - 1) - n0) * A.ldw * 2 + gb * 2;
                        q = t * 64 + gb < A.K ? q : zeros;
                    } else {
                        q = n0 + gb < A.N && t * 64 + row + half < A.K ? q : zeros;
                    }
                    core_fetch(q, to + CORE_HALF + (8 * j + wave) * 64);
                }
            }
        };
        CoreSums sums;
        sums.clear();
        const bool live = wm < s.rows && wn < A.N - n0;
        const int base_p = along_base(0, wm), base_q = TRANSPOSED ? along_base(CORE_HALF, wn) : across_base<32>(CORE_HALF, wn / 8);
        const int stages = (A.K + 63) / 64;
        if (live)
            core_contract<4, CoreFrag>(stages, lds, fetch,
                [&](CoreFrag &f, const core_u32x4 *now, int h) __attribute__((always_inline)) {
#pragma unroll
                    for (int a = 0; a < 4; ++a) f.p[a] = along_fragment(now, base_p, h, a);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        if constexpr (TRANSPOSED) f.q[b] = along_fragment(now, base_q, h, b);
                        else f.q[b] = across_fragment<32>(now, base_q, h, 4 * b);
                    }
                },
                [&](const CoreFrag &f) __attribute__((always_inline)) { sums.multiply(f); });
        else
            core_idle(stages, lds, fetch);
        __syncthreads();
        if (live) {
            // the wave's rows of 64 columns are put together in LDS and go out whole, 128 bytes each
            // (the lane made opaque, or what follows from it is worked out in front of the contraction and kept there)
            int lane = threadIdx.x & 63;
            asm volatile("" : "+v"(lane));
            const int half = lane >> 5, l32 = lane & 31;
            core_u32x4 *const own = &lds[0][0] + wave * 1024;
            const auto granule = [&](int r, int g) __attribute__((always_inline)) { return own + r * 8 + (g ^ (r & 7)); };
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = 32 * b + 8 * q + 4 * half;
                        const float4 v = *(const float4 *)&s_bias[wn + c];
                        const floatx16 &y = sums.s[a][b];
                        ((core_u32x2 *)granule(32 * a + l32, c / 8))[half] =
                            core_u32x2{cvt2bf(y[4 * q] + v.x, y[4 * q + 1] + v.y), cvt2bf(y[4 * q + 2] + v.z, y[4 * q + 3] + v.w)};
                    }
            core_settle();
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int r = 8 * j + (lane >> 3), g = lane & 7, to = s_row[wm + r], n = n0 + wn + 8 * g;
                if (to >= 0 && n < A.N) *(core_u32x4 *)((char *)A.c + (row_at(to, A.ldc) + n) * 2) = *granule(r, g);
            }
        }
        __syncthreads();        // s_row and LDS are the next tile's
    }
}

// dW[g] = sum of x[r]^T dy[r], db[g] = sum of dy[r]: of a chunk of a group's rows
__global__ __launch_bounds__(CT) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_grouped_weights_core(WeightArgs A) {
    constexpr int T = CORE_TILE;
    __shared__ __attribute__((aligned(16))) core_u32x4 lds[2][2 * CORE_HALF];
    const int lane = threadIdx.x & 63, wave = core_wave(), half = lane >> 5, l32 = lane & 31, wm = core_wm(), wn = core_wn();
    const int64_t tiles = (int64_t)A.tiles_m * A.tiles_n;
    for (int64_t block = blockIdx.x; block < A.room; block += gridDim.x) {
        Spot s;
        if (!find_spot<true>(A.ptr, A.G, A.list.n, A.per, block, tiles, s, A.pieces)) continue;
        const bool whole = s.chunks == 1;
        if (!whole && (uint64_t)s.slab >= (uint64_t)A.slabs) continue;          // (offsets that make no sense)
        const int m0 = s.side / A.tiles_n * T, n0 = s.side % A.tiles_n * T;
        // a lane holds the number of a row of the next stage (held inside the rows at once: the stage's fetches wait for the list's load)
        int next = 0;
        const auto look_up = [&](int t) __attribute__((always_inline)) {
            const int r = A.list.at(s.first + min(t * 64 + lane, s.rows - 1));
            next = max(r, 0);
        };
        // two rows of 256 columns an instruction
        const int g = ((lane & 31) ^ (4 * ((2 * wave + half) & 3))) * 8;
        // past the last column: zeros, in every row
        const bool in_x = m0 + g < A.K, in_dy = n0 + g < A.N;
        const char *const zeros = (const char *)&core_zeros;
        const char *const x0 = in_x ? (const char *)A.x + (m0 + g) * 2 : zeros, *const dy0 = in_dy ? (const char *)A.dy + (n0 + g) * 2 : zeros;
        const uint32_t ldx = in_x ? A.ldx : 0, lddy = in_dy ? A.lddy : 0;
        const auto fetch = [&](int t, core_u32x4 *to) __attribute__((always_inline)) {
            int r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = __shfl(next, 2 * (8 * j + wave) + half);
            look_up(t + 1);
            if ((t + 1) * 64 <= s.rows) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    core_fetch(x0 + row_at(r[j], ldx) * 2, to + (8 * j + wave) * 64);
                    core_fetch(dy0 + row_at(r[j], lddy) * 2, to + CORE_HALF + (8 * j + wave) * 64);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool in = t * 64 + 2 * (8 * j + wave) + half < s.rows;
                    core_fetch(in ? x0 + row_at(r[j], ldx) * 2 : zeros, to + (8 * j + wave) * 64);
                    core_fetch(in ? dy0 + row_at(r[j], lddy) * 2 : zeros, to + CORE_HALF + (8 * j + wave) * 64);
                }
            }
        };
        CoreSums sums;
        sums.clear();
        floatx16 col[2] = {zero16(), zero16()};
        const bool live = wm < A.K - m0 && wn < A.N - n0, bias = A.db && live && m0 == 0 && wm == 0;
        const int base_p = across_base<32>(0, wm / 8), base_q = across_base<32>(CORE_HALF, wn / 8);
        const core_u32x4 one{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
        if (s.rows > 0) {
            look_up(0);
            const int stages = (s.rows + 63) / 64;
            const auto read = [&](CoreFrag &f, const core_u32x4 *now, int h) __attribute__((always_inline)) {
#pragma unroll
                for (int a = 0; a < 4; ++a) f.p[a] = across_fragment<32>(now, base_p, h, 4 * a);
#pragma unroll
                for (int b = 0; b < 2; ++b) f.q[b] = across_fragment<32>(now, base_q, h, 4 * b);
            };
            if (bias)           // a column's sum is its product with ones, in float over the chunk as dW is (the other forms' are double: here a lane has no column by itself)
                core_contract<4, CoreFrag>(stages, lds, fetch, read, [&](const CoreFrag &f) __attribute__((always_inline)) {
                    sums.multiply(f);
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        col[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, f.q[b]), __builtin_bit_cast(bf16x8_t, one), col[b], 0, 0, 0);
                });
            else if (live)
                core_contract<4, CoreFrag>(stages, lds, fetch, read, [&](const CoreFrag &f) __attribute__((always_inline)) { sums.multiply(f); });
            else
                core_idle(stages, lds, fetch);
        }
        __syncthreads();
        const int64_t words = (int64_t)A.K * A.N;
        float *out = whole ? A.dw + s.g * words : A.slab + s.slab * (words + A.N);
        if (live) {
            int lane = threadIdx.x & 63;
            asm volatile("" : "+v"(lane));
            const int half = lane >> 5, l32 = lane & 31;
            core_u32x4 *const own = &lds[0][0] + wave * 1024;
            const auto granule = [&](int r, int q) __attribute__((always_inline)) { return own + r * 16 + (q ^ (r & 15)); };
#pragma unroll
            for (int part = 0; part < 2; ++part) {           // 64 rows of 64 floats at a time
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const floatx16 &y = sums.s[2 * part + a][b];
                            *(float4 *)granule(32 * a + l32, 8 * b + 2 * q + half) = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
                        }
                core_settle();
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int r = 4 * j + (lane >> 4), q = lane & 15, m = m0 + wm + 64 * part + r, n = n0 + wn + 4 * q;
                    if (m < A.K && n < A.N) *(core_u32x4 *)(out + (int64_t)m * A.N + n) = *granule(r, q);
                }
                core_settle();
            }
        }
        if (bias && l32 == 0) {
            float *const db = whole ? A.db + (int64_t)s.g * A.N : out + words;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = n0 + wn + 32 * b + 8 * q + 4 * half;
                    if (n < A.N) *(core_u32x4 *)(db + n) = __builtin_bit_cast(core_u32x4, make_float4(col[b][4 * q], col[b][4 * q + 1], col[b][4 * q + 2], col[b][4 * q + 3]));
                }
        }
        __syncthreads();
    }
}
