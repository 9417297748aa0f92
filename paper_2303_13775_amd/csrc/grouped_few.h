// The grouped products of few rows (included by grouped.hip inside its anonymous namespace): latency is all of them, and a tile's loop of
// fetch, barrier and multiplication is a chain of round trips to memory.  Here a workgroup forms 32 x 32 of the result; its four waves
// take every fourth step of 16 of the contraction, four steps ahead and straight into registers, without a barrier, and their sums
// meet in LDS, added in a fixed order.  33 rows of 8 groups 256 x 47 5.9 us (tiles of 64: 11.9), dW of 1024 rows of 4 groups 7.8 (13.4).
#pragma once

constexpr int FEW_AHEAD = 4;

// eight contraction indices of one row or column of an operand, as a lane feeds them
template <class T> struct FewItem { T v[8]; };
template <class T>
__device__ __forceinline__ void few_split(const FewItem<T> &x, uint4 (&p)[Kind<T>::PLANES]) {
    if constexpr (sizeof(T) == 4) {
        float s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = x.v[j] * SPLIT_SCALE;
        split8(s, p);
    } else {
        p[0] = make_uint4(x.v[0] | (uint32_t)x.v[1] << 16, x.v[2] | (uint32_t)x.v[3] << 16, x.v[4] | (uint32_t)x.v[5] << 16, x.v[6] | (uint32_t)x.v[7] << 16);
    }
}
// from a row's contraction indices k0 .. k0 + 7, whatever is there from K on.  (One branch for a whole wave: around single loads each
// would be waited for.)
template <class T>
__device__ __forceinline__ void few_along(FewItem<T> &x, const T *row, int k0, int K) {
    if (__ballot(k0 + 8 > K) == 0ull) {
        if constexpr (sizeof(T) == 4) {
            const u32x4 a = *(const u32x4_any *)(row + k0), b = *(const u32x4_any *)(row + k0 + 4);
            __builtin_memcpy(x.v, &a, 16);
            __builtin_memcpy(x.v + 4, &b, 16);
        } else {
            const u32x4 a = *(const u32x4_any *)(row + k0);
            __builtin_memcpy(x.v, &a, 16);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x.v[j] = row[min(k0 + j, K - 1)];
    }
}

template <class T>
struct FewSums {
    floatx16 hi, lo;
    __device__ __forceinline__ void multiply(const FewItem<T> &a, const FewItem<T> &b) {        // rows of the result, its columns
        uint4 p[Kind<T>::PLANES], q[Kind<T>::PLANES];
        few_split(a, p);
        few_split(b, q);
        hi = mfma_bf(q[0], p[0], hi);
        if constexpr (sizeof(T) == 4) {
            lo = mfma_bf(q[0], p[2], lo);
            lo = mfma_bf(q[0], p[1], lo);
            lo = mfma_bf(q[1], p[0], lo);
            lo = mfma_bf(q[1], p[1], lo);
            lo = mfma_bf(q[2], p[0], lo);
        }
    }
};
// The waves' sums joined: a lane gets row lane % 32 and the columns 8 wave + 4 (lane / 32) .. + 3 (zero past the contraction, see Sums::finish)
template <class T, class GetA, class GetB>
__device__ __forceinline__ void few_join(const FewSums<T> &sums, float (&lds)[4][16][64], int K, const GetA &a, const GetB &b, float (&v)[4]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 16; ++r) lds[wave][r][lane] = sizeof(T) == 4 ? sums.hi[r] + sums.lo[r] : sums.hi[r];
    __syncthreads();
    bool ok = sizeof(T) != 4 || K >= SPLIT_MIN_K;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = 4 * wave + j;
        v[j] = (lds[0][r][lane] + lds[1][r][lane]) + (lds[2][r][lane] + lds[3][r][lane]);
        if constexpr (sizeof(T) == 4) {
            v[j] *= SPLIT_UNSCALE;
            ok = ok && fabsf(v[j]) < INFINITY;
        }
    }
    if (sizeof(T) == 4 && __ballot(!ok) != 0ull) {
        const floatx16 e = exact_sum(0, K, lane >> 5, [&](int k) { return b(lane & 31, k); }, [&](int k) { return a(lane & 31, k); });
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (r >> 2 == wave) v[r & 3] = e[r];
    }
}

template <class T, bool TRANSPOSED>
__global__ __launch_bounds__(NT, 3) void k_grouped_rows_few(RowsArgs A) {
    __shared__ float lds[4][16][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    const int64_t room = (A.tiles_m * A.tiles_n + 7) / 8 * 8;
    for (int64_t block = blockIdx.x; block < room; block += gridDim.x) {
        Spot s;
        if (!find_spot<false>(A.ptr, A.G, A.list.n, 32, block, A.tiles_n, s)) continue;
        const int n0 = s.side * 32, n = min(n0 + l32, A.N - 1), K = A.K;
        const int row = A.list.at(s.first + min(l32, s.rows - 1));
        const T *const a = (const T *)A.a + row_at(max(row, 0), A.lda), *const w = (const T *)A.w + (int64_t)s.g * A.K * A.N;
        const T *const b = TRANSPOSED ? w + row_at(n, A.ldw) : w + n;
        FewSums<T> sums{zero16(), zero16()};
        FewItem<T> fa[FEW_AHEAD], fb[FEW_AHEAD];
        const int steps = (K + 15) / 16;
        for (int u0 = wave; u0 < steps; u0 += 4 * FEW_AHEAD) {
#pragma unroll
            for (int u = 0; u < FEW_AHEAD; ++u) {
                if (u0 + 4 * u >= steps) break;
                const int k0 = (u0 + 4 * u) * 16 + 8 * half;
                few_along(fa[u], a, k0, K);
                if (TRANSPOSED) {
                    few_along(fb[u], b, k0, K);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) fb[u].v[j] = b[row_at(min(k0 + j, K - 1), A.ldw)];
                }
            }
#pragma unroll
            for (int u = 0; u < FEW_AHEAD; ++u) {
                const int k0 = (u0 + 4 * u) * 16 + 8 * half;
                if (u0 + 4 * u >= steps) break;
                if (k0 + 8 > K) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (k0 + j >= K) fa[u].v[j] = fb[u].v[j] = 0;
                }
                sums.multiply(fa[u], fb[u]);
            }
        }
        float v[4];
        few_join(sums, lds, K, [&](int, int k) { return k < K ? as_float(a[k]) : 0.f; },
                 [&](int, int k) { return k < K ? as_float(TRANSPOSED ? b[k] : b[row_at(k, A.ldw)]) : 0.f; }, v);
        const int c = n0 + 8 * wave + 4 * half;
        if (row >= 0 && l32 < s.rows && c < A.N) {
            if (A.bias) {
                const float *bias = A.bias + (int64_t)s.g * A.N;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += bias[min(c + j, A.N - 1)];
            }
            store4((T *)A.c + row_at(row, A.ldc) + c, v, A.N - c);
        }
    }
}

template <class T>
__global__ __launch_bounds__(NT, 2) void k_grouped_weights_few(WeightArgs A) {
    __shared__ float lds[4][16][64];
    __shared__ double s_sum[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    const int64_t tiles = (int64_t)A.tiles_m * A.tiles_n;
    for (int64_t block = blockIdx.x; block < A.room; block += gridDim.x) {
        Spot s;
        if (!find_spot<true>(A.ptr, A.G, A.list.n, A.per, block, tiles, s, A.pieces)) continue;
        const bool whole = s.chunks == 1;
        if (!whole && (uint64_t)s.slab >= (uint64_t)A.slabs) continue;          // (offsets that make no sense)
        const int m0 = s.side / A.tiles_n * 32, n0 = s.side % A.tiles_n * 32;
        const T *const x = (const T *)A.x + min(m0 + l32, A.K - 1), *const dy = (const T *)A.dy + min(n0 + l32, A.N - 1);
        const auto row = [&](int k) { return max(A.list.at(s.first + k), 0); };
        FewSums<T> sums{zero16(), zero16()};
        FewItem<T> fa[FEW_AHEAD], fb[FEW_AHEAD];
        double col = 0.0;
        const bool bias = A.db && m0 == 0;
        const int steps = (s.rows + 15) / 16;
        for (int u0 = wave; u0 < steps; u0 += 4 * FEW_AHEAD) {
            int r[FEW_AHEAD][8];
#pragma unroll
            for (int u = 0; u < FEW_AHEAD; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) r[u][j] = s.first + min((u0 + 4 * u) * 16 + 8 * half + j, s.rows - 1);
            if (A.list.rows) {
#pragma unroll
                for (int u = 0; u < FEW_AHEAD; ++u)
#pragma unroll
                    for (int j = 0; j < 8; ++j) r[u][j] = A.list.rows[r[u][j]];
            }
#pragma unroll
            for (int u = 0; u < FEW_AHEAD; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int q = (uint32_t)r[u][j] < (uint32_t)A.list.n ? r[u][j] : 0;
                    fa[u].v[j] = x[row_at(q, A.ldx)];
                    fb[u].v[j] = dy[row_at(q, A.lddy)];
                }
#pragma unroll
            for (int u = 0; u < FEW_AHEAD; ++u) {
                const int k0 = (u0 + 4 * u) * 16 + 8 * half;
                if (u0 + 4 * u >= steps) break;
                if (k0 + 8 > s.rows) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (k0 + j >= s.rows) fa[u].v[j] = fb[u].v[j] = 0;
                }
                if (bias) {
                    float f = 0.f, h = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; j += 2) { f += as_float(fb[u].v[j]); h += as_float(fb[u].v[j + 1]); }
                    col += (double)f + (double)h;
                }
                sums.multiply(fa[u], fb[u]);
            }
        }
        float v[4];
        few_join(sums, lds, s.rows, [&](int, int k) { return k < s.rows ? as_float(x[row_at(row(k), A.ldx)]) : 0.f; },
                 [&](int, int k) { return k < s.rows ? as_float(dy[row_at(row(k), A.lddy)]) : 0.f; }, v);
        const int64_t words = (int64_t)A.K * A.N;
        float *const out = whole ? A.dw + s.g * words : A.slab + s.slab * (words + A.N);
        const int m = m0 + l32, c = n0 + 8 * wave + 4 * half;
        if (m < A.K && c < A.N) store4(out + (int64_t)m * A.N + c, v, A.N - c);
        if (bias) {
            s_sum[wave][lane] = col;
            __syncthreads();
            if (threadIdx.x < 32 && n0 + l32 < A.N) {
                double sum = 0.0;
                for (int w = 0; w < 4; ++w) sum += s_sum[w][l32] + s_sum[w][32 + l32];
                (whole ? A.db + (int64_t)s.g * A.N : out + words)[n0 + l32] = (float)sum;
            }
            __syncthreads();
        }
    }
}
