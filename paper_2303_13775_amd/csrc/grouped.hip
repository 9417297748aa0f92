// Products grouped by row: y[r] = x[r] W[g] + b[g] for the rows r of every group g, and the gradients of x, W and b.
//
// One tile product serves all three.  A tile of BM rows x BN columns of the result goes to a workgroup of four waves, a quarter of it
// each; the contraction is taken KT at a time: operands are fetched into registers while the matrix unit works on the tile in
// front, and laid out in LDS as granules of eight contraction indices, the way a lane feeds the matrix unit.  An operand lies in
// memory with the contraction along its rows (`Along`: x and dy as rows, W of the input gradient) or across them (`Across`: W of the
// forward product, x and dy of the weight gradient); there a thread fetches the same columns of eight rows and transposes them in
// its registers.
// Floats go through the bfloat16 matrix unit as three parts and six products (split_parts.h); products of bfloat16 are exact there.
// Sums are float.
// The columns of the result run along the matrix unit's rows: a lane then holds four consecutive columns of one row.
//
// What bounds them.  Float: the six products and the splitting in front of them (60000 rows of 8 groups 512 x 512 219 us, matrix unit
// busy for 41 %).  bfloat16 rows of whole granules have tiles of their own (grouped_core.h); at other addresses one tile's loads in
// flight (20011 rows of 24 groups 1000 x 1021: dx 95 us, dW 150).  Few rows: latency (4096 x 256 x 172 of 16 groups 12.8; fewer, grouped_few.h).
// Tiles of 128 x 128 where they fill the chip, else 64 x 64 (group_rules.h): a quarter of 128 x 128 is 64 registers of sums
// a lane, and the most that leaves room for a tile in flight and two workgroups a compute unit.
#include <algorithm>
#include <type_traits>

#include "group_rules.h"
#include "gsplit_internal.h"
#include "op_checks.h"

namespace {

#include "gemm_common.h"
#include "split_parts.h"
#include "tile_core.h"

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// rows start at any multiple of their elements' size, which the vector loads and stores of the chip take
typedef uint32_t u32_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

constexpr int NT = 256;

template <class T> struct Kind;
template <> struct Kind<float> {
    static constexpr int PLANES = 3, KT = 32, KG = 4;       // parts of an operand, contraction of a tile, its granules
    // contraction index j of granule g: four threads that fetch a row's granules read 64 bytes side by side
    static __device__ __forceinline__ int k_of(int g, int j) { return granule_k(g, j); }
    static __device__ __forceinline__ int turn(int row) { return (row >> 2) & 3; }
};
template <> struct Kind<uint16_t> {
    static constexpr int PLANES = 1, KT = 64, KG = 8;
    static __device__ __forceinline__ int k_of(int g, int j) { return 8 * g + j; }
    static __device__ __forceinline__ int turn(int row) { return ((row >> 1) ^ (row >> 4)) & 7; }
};
// where granule g of a row lies: rows that are read or written side by side fall into different banks
template <class T> __device__ __forceinline__ int slot(int row, int g) { return row * Kind<T>::KG + (g ^ Kind<T>::turn(row)); }

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(uint16_t x) { return bf2f(x); }

// eight values of a granule -> LDS, as `planes` parts
template <class T, int ROWS>
__device__ __forceinline__ void land(uint4 *lds, int at, const float (&v)[8]) {
    uint4 p[3];
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = v[j] * SPLIT_SCALE;
    split8(s, p);
#pragma unroll
    for (int q = 0; q < 3; ++q) lds[q * ROWS * Kind<T>::KG + at] = p[q];
}

// An operand with the contraction along its rows: element (i, k) at row(i)[k]
template <class T, int ROWS>
struct Along {
    static constexpr int KG = Kind<T>::KG, KT = Kind<T>::KT, N = ROWS * KG / NT;
    static_assert(N * NT == ROWS * KG, "whole items");
    const T *p[N];
    int K;
    typedef typename std::conditional<sizeof(T) == 4, float[8], uint4>::type Item;
    Item r[N];

    template <class Row>
    __device__ __forceinline__ void init(int k_len, const Row &row) {
        K = k_len;
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = row(((int)threadIdx.x + i * NT) / KG);
    }
    // No branch: where it meets the other way again, what is in flight would be waited for.  Past the row's end: its last eight (float: four)
    // elements once more, from which `cut` takes what there is.
    __device__ __forceinline__ void load(int t) {
        const int g = threadIdx.x % KG, k0 = t * KT;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (sizeof(T) == 4) {
                const u32x4 a = *(const u32x4_any *)(p[i] + min(k0 + 4 * g, K - 4)), b = *(const u32x4_any *)(p[i] + min(k0 + 16 + 4 * g, K - 4));
#pragma unroll
                for (int j = 0; j < 4; ++j) { r[i][j] = __uint_as_float(a[j]); r[i][4 + j] = __uint_as_float(b[j]); }
            } else {
                const u32x4 a = *(const u32x4_any *)(p[i] + min(k0 + 8 * g, K - 8));
                r[i] = make_uint4(a[0], a[1], a[2], a[3]);
            }
        }
    }
    // zeros past the end of the contraction, in its tile t
    __device__ __forceinline__ void cut(int t) {
        if ((t + 1) * KT <= K) return;
        const int g = threadIdx.x % KG, k0 = t * KT;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                const int past = max(k0 + 4 * h + 4 * g - (K - 4), 0);         // elements in front of the first that is wanted
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float v = 0.f;
#pragma unroll
                        for (int q = j; q < 4; ++q) v = q == j + past ? r[i][h + q] : v;
                        r[i][h + j] = v;
                    }
            }
        } else {
            const int past = max(k0 + 8 * g - (K - 8), 0);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t w[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
                uint32_t v[5] = {};
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int q = j; q < 4; ++q) v[j] = q == j + past / 2 ? w[q] : v[j];
                const uint32_t by = past & 1 ? 16 : 0;
                r[i] = make_uint4(__builtin_amdgcn_alignbit(v[1], v[0], by), __builtin_amdgcn_alignbit(v[2], v[1], by),
                                  __builtin_amdgcn_alignbit(v[3], v[2], by), __builtin_amdgcn_alignbit(v[4], v[3], by));
            }
        }
    }
    __device__ __forceinline__ void store(uint4 *lds) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int x = (int)threadIdx.x + i * NT, at = slot<T>(x / KG, x % KG);
            if constexpr (sizeof(T) == 4) land<T, ROWS>(lds, at, r[i]);
            else lds[at] = r[i];
        }
    }
};

// An operand with the contraction across its rows: element (i, k) at row(k)[i], i < cols; of these the ones from `first` on.  A thread
// takes W columns of the eight rows of a granule; THREADS of them fetch the operand.
template <class T, int ROWS, int THREADS = NT>
struct Across {
    static constexpr int KG = Kind<T>::KG, KT = Kind<T>::KT, W = ROWS * KG / THREADS, WORDS = W * (int)sizeof(T) / 4;
    static_assert(W * THREADS == ROWS * KG && (WORDS == 1 || WORDS == 2 || WORDS == 4), "one item a thread");
    int cols, col, base;            // this thread's first column; LDS row of it
    uint32_t r[8][WORDS];

    static __device__ __forceinline__ int granule() { return (int)threadIdx.x % THREADS / (ROWS / W); }
    __device__ __forceinline__ void init(int n_cols, int first) {
        cols = n_cols;
        const int want = first + (int)threadIdx.x % (ROWS / W) * W;
        // past the last column: the last ones once more, whose granules are then written twice, with the same values
        col = max(0, min(want, cols - W));
        base = col - first;
    }
    // from row(j), the row of the granule's contraction index j.  (No branch around a single load: each would wait for the one before.)
    template <class Row>
    __device__ __forceinline__ void load(const Row &row) {
        // (tiles of 128 are for more columns, but without this way the weight gradients' take 256 registers, not 239, and 166 us, not 159: 20011 rows of 24
        // groups 1000 x 1021 bf16)
        if ((ROWS == 64 || THREADS < NT) && W > 1 && cols < W) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const T *p = row(j);
                T v[W];
#pragma unroll
                for (int c = 0; c < W; ++c) v[c] = p[min(c, cols - 1)];
                __builtin_memcpy(r[j], v, sizeof(v));
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const T *p = row(j) + col;
                if constexpr (WORDS == 1) {
                    r[j][0] = *(const u32_any *)p;
                } else if constexpr (WORDS == 4) {
                    const u32x4 a = *(const u32x4_any *)p;
#pragma unroll
                    for (int w = 0; w < 4; ++w) r[j][w] = a[w];
                } else {
                    const u32x2 a = *(const u32x2_any *)p;
                    r[j][0] = a[0]; r[j][1] = a[1];
                }
            }
        }
    }
    // zeros past the end of the contraction of K, in its tile t
    __device__ __forceinline__ void cut(int t, int K) {
        if ((t + 1) * KT <= K) return;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (t * KT + Kind<T>::k_of(granule(), j) >= K)
#pragma unroll
                for (int w = 0; w < WORDS; ++w) r[j][w] = 0u;
    }
    __device__ __forceinline__ float at(int j, int c) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(r[j][c]);
        else return __uint_as_float(c & 1 ? r[j][c / 2] & 0xFFFF0000u : r[j][c / 2] << 16);
    }
    __device__ __forceinline__ void store(uint4 *lds) const {
#pragma unroll
        for (int c = 0; c < W; ++c) {
            const int row = base + c;
            if (row < 0 || row >= ROWS) continue;
            const int to = slot<T>(row, granule());
            if constexpr (sizeof(T) == 4) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = at(j, c);
                land<T, ROWS>(lds, to, v);
            } else {
                // the low or the high halves of two rows' words side by side
                const uint32_t pick = c & 1 ? 0x07060302u : 0x05040100u;
                uint32_t w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) w[q] = __builtin_amdgcn_perm(r[2 * q + 1][c / 2], r[2 * q][c / 2], pick);
                lds[to] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
};

// Rows of LDS that an `Across` of a tile's last columns leaves unwritten: zeros, or what was there would decide whether the tile's
// sums look finite.
template <class T, int ROWS>
__device__ __forceinline__ void clear_rows(uint4 *lds) {
    for (int i = threadIdx.x; i < ROWS * Kind<T>::KG * Kind<T>::PLANES; i += NT) lds[i] = make_uint4(0u, 0u, 0u, 0u);
}

// A workgroup's tile of the result: BM rows x BN columns, waves 2 x 2
template <int BM_, int BN_> struct Tile {
    static constexpr int BM = BM_, BN = BN_, MI = BM / 64, NI = BN / 64;       // blocks of 32 x 32 of a wave
};

template <class T, class TL>
struct Sums {
    floatx16 hi[TL::NI][TL::MI], lo[sizeof(T) == 4 ? TL::NI : 1][sizeof(T) == 4 ? TL::MI : 1];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < TL::NI; ++n)
#pragma unroll
            for (int m = 0; m < TL::MI; ++m) {
                hi[n][m] = zero16();
                if constexpr (sizeof(T) == 4) lo[n][m] = zero16();
            }
    }
    // one tile of the contraction: rows (the result's) in a, columns in b
    __device__ __forceinline__ void multiply(const uint4 *a, const uint4 *b) {
        constexpr int KG = Kind<T>::KG, P = Kind<T>::PLANES;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, l32 = lane & 31;
        const int wm = (wave & 1) * (TL::BM / 2), wn = (wave >> 1) * (TL::BN / 2);
#pragma unroll
        for (int s = 0; s < KG / 2; ++s) {
            uint4 fa[TL::MI][P], fb[TL::NI][P];
#pragma unroll
            for (int q = 0; q < P; ++q) {
#pragma unroll
                for (int m = 0; m < TL::MI; ++m) fa[m][q] = a[q * TL::BM * KG + slot<T>(wm + 32 * m + l32, 2 * s + half)];
#pragma unroll
                for (int n = 0; n < TL::NI; ++n) fb[n][q] = b[q * TL::BN * KG + slot<T>(wn + 32 * n + l32, 2 * s + half)];
            }
#pragma unroll
            for (int n = 0; n < TL::NI; ++n)
#pragma unroll
                for (int m = 0; m < TL::MI; ++m) {
                    hi[n][m] = mfma_bf(fb[n][0], fa[m][0], hi[n][m]);
                    if constexpr (P == 3) {
                        lo[n][m] = mfma_bf(fb[n][0], fa[m][2], lo[n][m]);
                        lo[n][m] = mfma_bf(fb[n][0], fa[m][1], lo[n][m]);
                        lo[n][m] = mfma_bf(fb[n][1], fa[m][0], lo[n][m]);
                        lo[n][m] = mfma_bf(fb[n][1], fa[m][1], lo[n][m]);
                        lo[n][m] = mfma_bf(fb[n][2], fa[m][0], lo[n][m]);
                    }
                }
        }
    }
    // Calls f(row of the tile, first of four consecutive columns, their values) for all of them.  Values that the parts of floats
    // cannot carry (infinities, NaN, very large ones) have made a sum that is not finite: a wave that finds one, and contractions
    // of one or two products, are formed again with the float matrix instructions, block by block.
    // a(i, k), b(i, k): element of row / column i of the tile, 0 past the contraction's end
    template <class GetA, class GetB, class F>
    __device__ __forceinline__ void finish(int K, const GetA &a, const GetB &b, const F &f) {
        int lane = threadIdx.x & 63;
        const int wave = threadIdx.x >> 6, wm = (wave & 1) * (TL::BM / 2), wn = (wave >> 1) * (TL::BN / 2);
        const auto block = [&](int m, int n, const floatx16 &x) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v[4] = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
                f(wm + 32 * m + (lane & 31), wn + 32 * n + 8 * q + 4 * (lane >> 5), v);
            }
        };
        bool ok = K >= SPLIT_MIN_K || sizeof(T) != 4;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int n = 0; n < TL::NI; ++n)
#pragma unroll
                for (int m = 0; m < TL::MI; ++m) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) hi[n][m][r] = (hi[n][m][r] + lo[n][m][r]) * SPLIT_UNSCALE;
                    ok = ok && finite16(hi[n][m]);
                }
        }
        if (sizeof(T) != 4 || __ballot(!ok) == 0ull) {
#pragma unroll
            for (int m = 0; m < TL::MI; ++m)
#pragma unroll
                for (int n = 0; n < TL::NI; ++n) block(m, n, hi[n][m]);
        } else {
            // (the lane made opaque, or what follows from it is worked out in front of the contraction and kept there)
            asm volatile("" : "+v"(lane));
#pragma unroll 1
            for (int x = 0; x < TL::MI * TL::NI; ++x) {
                const int m = x / TL::NI, n = x % TL::NI;
                block(m, n, exact_sum(0, K, lane >> 5, [&](int k) { return b(wn + 32 * n + (lane & 31), k); },
                                      [&](int k) { return a(wm + 32 * m + (lane & 31), k); }));
            }
        }
    }
};

// Which rows a tile takes: its group, the place of its first row among the sorted ones, how many.  Tiles of rows are numbered group by
// group, `across` of them side by side; every wave works it out for itself, 64 groups at a time.  Offsets that make no sense are held
// inside 0 .. n_rows.
struct Spot { int g, first, rows, chunks, slab, side; };
template <bool EMPTY_TOO>
__device__ __forceinline__ bool find_spot(const int32_t *__restrict__ ptr, int G, int n_rows, int per, int64_t block, int64_t across, Spot &s, int pieces = 1) {
    const int lane = threadIdx.x & 63;
    int lo, hi, tiles, sum, own_slabs, slabs;
    const auto scan = [&](int base) __attribute__((always_inline)) {
        const int g = base + lane;
        lo = min(max(ptr[min(g, G)], 0), n_rows); hi = min(max(ptr[min(g + 1, G)], lo), n_rows);
        tiles = (int)(((int64_t)(hi - lo) + per - 1) / per);
        if (EMPTY_TOO) tiles = max(tiles, 1);
        if (g >= G) tiles = 0;
        sum = tiles;
        slabs = own_slabs = tiles > 1 ? tiles : 0;
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(sum, o), up2 = EMPTY_TOO ? __shfl_up(slabs, o) : 0;
            if (lane >= o) { sum += up; slabs += up2; }
        }
    };
    int all = 0;
    for (int base = (G - 1) / 64 * 64; base >= 0; base -= 64) {         // (the first groups last: they are what the search begins with)
        scan(base);
        all += __builtin_amdgcn_readlane(sum, 63);
    }
    // Workgroups are dealt round-robin to the eight XCDs: consecutive tiles (the same rows, the same matrix) go to one of them, for its
    // L2, an eighth of the tiles there are each (not of those there may be, or the last XCDs have less to do)
    int j, slab = 0;
    if (EMPTY_TOO && all >= 16) {
        // (chunks of rows are of all lengths, and the long ones lie side by side: pieces of their tiles, each in turn to another XCD)
        const int each = (int)((across + pieces - 1) / pieces), q = (int)((block >> 3) / each);
        const int64_t piece = (int64_t)q * 8 + (block & 7);
        j = (int)(piece / pieces);
        s.side = (int)(piece - (int64_t)j * pieces) * each + (int)((block >> 3) - (int64_t)q * each);
        if (j >= all || s.side >= across) return false;
    } else {
        const int64_t total = all * across, each = (total + 7) / 8, x = (block & 7) * each + (block >> 3);
        if (block >> 3 >= each || x >= total) return false;
        j = (int)(x / across);
        s.side = (int)(x - j * across);
    }
    for (int base = 0;;) {
        const int n = __builtin_amdgcn_readlane(sum, 63);
        if (j < n) {
            const uint64_t past = __ballot(sum > j);
            const int l = past ? __builtin_ctzll(past) : 0;
            const int c = j - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(tiles, l));
            s.g = base + l;
            s.chunks = __builtin_amdgcn_readlane(tiles, l);
            if (c < 0 || c >= s.chunks) return false;       // (offsets that make no sense may make sums that do not fit)
            s.first = __builtin_amdgcn_readlane(lo, l) + c * per;
            s.rows = min(per, __builtin_amdgcn_readlane(hi, l) - s.first);
            s.slab = slab + __builtin_amdgcn_readlane(slabs, l) - __builtin_amdgcn_readlane(own_slabs, l) + c;
            return true;
        }
        j -= n;
        slab += __builtin_amdgcn_readlane(slabs, 63);
        base += 64;
        if (base >= G) return false;
        scan(base);
    }
}

// The list of rows; a number outside the rows reads row 0 and is not written
struct RowList {
    const int32_t *rows;
    int32_t n;
    __device__ __forceinline__ int at(int place) const {
        const int r = rows ? rows[place] : place;
        return (uint32_t)r < (uint32_t)n ? r : -1;
    }
};

// where row r of a matrix starts: one multiplication (strides are below 2^31)
__device__ __forceinline__ uint64_t row_at(int r, uint32_t ld) { return (uint64_t)(uint32_t)r * ld; }

struct RowsArgs {
    const void *a, *w;
    const float *bias;
    void *c;
    uint32_t lda, ldc, ldw;
    int32_t K, N, G;
    const int32_t *ptr;
    RowList list;
    int64_t tiles_m;
    int32_t tiles_n;
};

template <class T>
__device__ __forceinline__ void store4(T *p, const float (&v)[4], int n) {
    if (n >= 4) {
        if constexpr (sizeof(T) == 4) *(u32x4_any *)p = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        else *(u32x2_any *)p = u32x2{cvt2bf(v[0], v[1]), cvt2bf(v[2], v[3])};
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) {
                if constexpr (sizeof(T) == 4) p[j] = v[j];
                else p[j] = f2bf(v[j]);
            }
    }
}

// c[r] = a[r] W[g] (+ bias), W as K x N, or as N x K (TRANSPOSED)
template <class T, class TL, bool TRANSPOSED>
__global__ __launch_bounds__(NT, 2) void k_grouped_rows(RowsArgs A) {
    constexpr int BM = TL::BM, BN = TL::BN, KG = Kind<T>::KG, P = Kind<T>::PLANES;
    __shared__ __attribute__((aligned(16))) uint4 s_a[P * BM * KG], s_b[P * BN * KG];
    __shared__ int s_row[BM];
    __shared__ __attribute__((aligned(16))) float s_bias[BN];
    const int64_t room = (A.tiles_m * A.tiles_n + 7) / 8 * 8;
    for (int64_t block = blockIdx.x; block < room; block += gridDim.x) {
        Spot s;
        if (!find_spot<false>(A.ptr, A.G, A.list.n, BM, block, A.tiles_n, s)) continue;
        const int n0 = s.side * BN;
        if (threadIdx.x < BM) s_row[threadIdx.x] = (int)threadIdx.x < s.rows ? A.list.at(s.first + threadIdx.x) : -1;
        if (threadIdx.x < BN) s_bias[threadIdx.x] = A.bias && n0 + (int)threadIdx.x < A.N ? A.bias[(int64_t)s.g * A.N + n0 + threadIdx.x] : 0.f;
        if (!TRANSPOSED && n0 + BN > A.N) clear_rows<T, BN>(s_b);
        __syncthreads();
        const T *a = (const T *)A.a, *w = (const T *)A.w + (int64_t)s.g * A.K * A.N;
        const auto a_row = [&](int i) { return a + row_at(max(s_row[i < s.rows ? i : 0], 0), A.lda); };
        Along<T, BM> la;
        la.init(A.K, a_row);
        typename std::conditional<TRANSPOSED, Along<T, BN>, Across<T, BN>>::type lb;
        const auto w_row = [&](int k) { return w + row_at(k, A.ldw); };
        const auto w_col = [&](int i) { return w + row_at(min(n0 + i, A.N - 1), A.ldw); };
        if constexpr (TRANSPOSED) lb.init(A.K, w_col);
        else lb.init(A.N, n0);
        const auto load = [&](int t) __attribute__((always_inline)) {
            la.load(t);
            if constexpr (TRANSPOSED) lb.load(t);
            else lb.load([&](int j) { return w_row(min(t * Kind<T>::KT + Kind<T>::k_of(lb.granule(), j), A.K - 1)); });
        };
        Sums<T, TL> sums;
        sums.clear();
        const int KT = (A.K + Kind<T>::KT - 1) / Kind<T>::KT;
        load(0);
        for (int t = 0; t < KT; ++t) {
            la.cut(t);
            if constexpr (TRANSPOSED) lb.cut(t);
            else lb.cut(t, A.K);
            la.store(s_a);
            lb.store(s_b);
            __syncthreads();
            if (t + 1 < KT) load(t + 1);
            sums.multiply(s_a, s_b);
            __syncthreads();
        }
        sums.finish(A.K, [&](int i, int k) { return k < A.K ? as_float(a_row(i)[k]) : 0.f; },
                    [&](int i, int k) {
                        if (k >= A.K) return 0.f;
                        if constexpr (TRANSPOSED) return as_float(w_col(i)[k]);
                        else return as_float(w_row(k)[min(n0 + i, A.N - 1)]);
                    },
                    [&](int i, int j, const float (&v)[4]) {
            const int r = s_row[i], n = n0 + j, left = A.N - n;
            if (r < 0 || left <= 0) return;
            const float4 b = *(const float4 *)&s_bias[j];
            const float y[4] = {v[0] + b.x, v[1] + b.y, v[2] + b.z, v[3] + b.w};
            store4((T *)A.c + row_at(r, A.ldc) + n, y, left);
        });
        __syncthreads();        // s_row is the next tile's
    }
}

struct WeightArgs {
    const void *x, *dy;
    uint32_t ldx, lddy;
    int32_t K, N, G;            // rows and columns of a gradient
    const int32_t *ptr;
    RowList list;
    int32_t per;                // rows of a chunk
    int64_t room;               // workgroups that have a piece of a chunk's tiles, at most
    int32_t pieces;
    int32_t tiles_m, tiles_n;
    float *dw, *db;
    float *slab;                // [slabs x (K + 1) x N]: the chunks' gradients of W, then of b
    int64_t slabs;
};

// dW[g] = sum of x[r]^T dy[r], db[g] = sum of dy[r]: of a chunk of a group's rows, into the slab of the chunk where a group has several
template <class T, class TL>
__global__ __launch_bounds__(NT, 2) void k_grouped_weights(WeightArgs A) {
    constexpr int BM = TL::BM, BN = TL::BN, KG = Kind<T>::KG, P = Kind<T>::PLANES;
    __shared__ __attribute__((aligned(16))) uint4 s_a[P * BM * KG], s_b[P * BN * KG];
    __shared__ double s_sum[KG][BN];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t tiles = (int64_t)A.tiles_m * A.tiles_n;
    for (int64_t block = blockIdx.x; block < A.room; block += gridDim.x) {
        Spot s;
        if (!find_spot<true>(A.ptr, A.G, A.list.n, A.per, block, tiles, s, A.pieces)) continue;
        const bool whole = s.chunks == 1;
        if (!whole && (uint64_t)s.slab >= (uint64_t)A.slabs) continue;          // (offsets that make no sense)
        const int m0 = s.side / A.tiles_n * BM, n0 = s.side % A.tiles_n * BN;
        const T *xs = (const T *)A.x, *dys = (const T *)A.dy;
        const auto x_row = [&](int k) { return xs + row_at(max(A.list.at(s.first + k), 0), A.ldx); };
        const auto dy_row = [&](int k) { return dys + row_at(max(A.list.at(s.first + k), 0), A.lddy); };
        // two waves fetch x, two dy: sixteen bytes a load
        static_assert(BM == BN, "one operand is like the other");
        typedef Across<T, BM, NT / 2> Half;
        Half l;
        const bool is_dy = wave >= 2;
        l.init(is_dy ? A.N : A.K, is_dy ? n0 : m0);
        const T *const from = is_dy ? dys : xs;
        const uint32_t ld = is_dy ? A.lddy : A.ldx;
        uint4 *const to = is_dy ? s_b : s_a;
        // the rows of the next tile are looked up a tile ahead: their loads would wait for the list's
        int next[8];
        const auto look_up = [&](int t) __attribute__((always_inline)) {
            int place[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) place[j] = s.first + min(t * Kind<T>::KT + Kind<T>::k_of(l.granule(), j), s.rows - 1);
            if (A.list.rows) {
#pragma unroll
                for (int j = 0; j < 8; ++j) next[j] = A.list.rows[place[j]];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) next[j] = place[j];
            }
        };
        const auto load = [&](int t) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) next[j] = (uint32_t)next[j] < (uint32_t)A.list.n ? next[j] : 0;
            l.load([&](int j) { return from + row_at(next[j], ld); });
            look_up(t + 1);
        };
        Sums<T, TL> sums;
        sums.clear();
        double col[Half::W] = {};
        const bool bias = A.db && m0 == 0;
        if (m0 + BM > A.K) clear_rows<T, BM>(s_a);
        if (n0 + BN > A.N) clear_rows<T, BN>(s_b);
        __syncthreads();
        const int KT = (s.rows + Kind<T>::KT - 1) / Kind<T>::KT;
        if (KT > 0) { look_up(0); load(0); }
        for (int t = 0; t < KT; ++t) {
            l.cut(t, s.rows);
            l.store(to);
            if (bias && is_dy) {
#pragma unroll
                for (int c = 0; c < Half::W; ++c) {
                    float f = 0.f, h = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; j += 2) { f += l.at(j, c); h += l.at(j + 1, c); }
                    col[c] += (double)f + (double)h;
                }
            }
            __syncthreads();
            if (t + 1 < KT) load(t + 1);
            sums.multiply(s_a, s_b);
            __syncthreads();
        }
        const int64_t words = (int64_t)A.K * A.N;
        float *out = whole ? A.dw + s.g * words : A.slab + s.slab * (words + A.N);
        sums.finish(s.rows, [&](int i, int k) { return k < s.rows ? as_float(x_row(k)[min(m0 + i, A.K - 1)]) : 0.f; },
                    [&](int i, int k) { return k < s.rows ? as_float(dy_row(k)[min(n0 + i, A.N - 1)]) : 0.f; },
                    [&](int i, int j, const float (&v)[4]) {
            const int m = m0 + i, n = n0 + j;
            if (m < A.K && n < A.N) store4(out + (int64_t)m * A.N + n, v, A.N - n);
        });
        if (bias) {
            if (is_dy) {
#pragma unroll
                for (int c = 0; c < Half::W; ++c)
                    if (l.base + c >= 0 && l.base + c < BN) s_sum[l.granule()][l.base + c] = col[c];
            }
            __syncthreads();
            for (int j = threadIdx.x; j < BN && n0 + j < A.N; j += NT) {
                double sum = 0.0;
                for (int q = 0; q < KG; ++q) sum += s_sum[q][j];
                (whole ? A.db + (int64_t)s.g * A.N : out + words)[n0 + j] = (float)sum;
            }
            __syncthreads();
        }
    }
}

// the slabs of every group that has several, added up in their order: blockIdx.y counts those groups
__global__ __launch_bounds__(NT) void k_grouped_weights_sum(WeightArgs A) {
    const int64_t words = (int64_t)A.K * A.N, all = words + (A.db ? A.N : 0), each = words + A.N;
    // the blockIdx.y-th group of several chunks, a lane a group
    const int lane = threadIdx.x & 63;
    int g = -1, slab = 0, chunks = 0, left = blockIdx.y;
    for (int base = 0; base < A.G && g < 0; base += 64) {
        const int x = base + lane;
        const int lo = min(max(A.ptr[min(x, A.G)], 0), A.list.n), hi = min(max(A.ptr[min(x + 1, A.G)], lo), A.list.n);
        const int n = x < A.G ? (int)(((int64_t)(hi - lo) + A.per - 1) / A.per) : 0, own = n > 1 ? n : 0;
        int sum = own;
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(sum, o);
            if (lane >= o) sum += up;
        }
        uint64_t several = __ballot(own > 0);
        const int found = __popcll(several);
        if (left < found) {
            for (; left > 0; --left) several &= several - 1;
            const int l = __builtin_ctzll(several);
            g = base + l;
            chunks = __builtin_amdgcn_readlane(own, l);
            slab += __builtin_amdgcn_readlane(sum, l) - chunks;
        } else {
            left -= found;
            slab += __builtin_amdgcn_readlane(sum, 63);
        }
    }
    if (g < 0 || slab < 0 || (int64_t)slab + chunks > A.slabs) return;
    const float *part = A.slab + slab * each;
    float *const dw = A.dw + g * words, *const db = A.db ? A.db + (int64_t)g * A.N : nullptr;
    // four words a thread (the last ones, and those of rows that are no multiple of four, by themselves)
    const int64_t quads = words / 4, items = quads + (all - quads * 4);
    for (int64_t x = blockIdx.x * (int64_t)NT + threadIdx.x; x < items; x += (int64_t)gridDim.x * NT) {
        if (x < quads) {
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
            const auto add = [&](const u32x4 &q) {
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] += __uint_as_float(q[k]);
            };
            int c = 0;
            for (; c + 4 <= chunks; c += 4) {
                u32x4 q[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) q[k] = *(const u32x4_any *)(part + (c + k) * each + 4 * x);
#pragma unroll
                for (int k = 0; k < 4; ++k) add(q[k]);
            }
            for (; c < chunks; ++c) add(*(const u32x4_any *)(part + c * each + 4 * x));
            store4(dw + 4 * x, sum, 4);
        } else {
            const int64_t i = quads * 4 + (x - quads);
            double sum = 0.0;           // (a bias gradient's, as within most chunks; and the last words of dW)
            for (int c = 0; c < chunks; ++c) sum += (double)part[c * each + i];
            (i < words ? dw + i : db + (i - words))[0] = (float)sum;
        }
    }
}

#include "grouped_core.h"
#include "grouped_few.h"

// -- launches ---------------------------------------------------------------------------------

constexpr int64_t MOST_BLOCKS = 1 << 22;        // (a launch has less than 2^32 threads; workgroups go round)
inline unsigned blocks(int64_t total) { return (unsigned)std::min<int64_t>((total + 7) / 8 * 8, MOST_BLOCKS); }

// rows that start at multiples of 16 bytes, and are a whole number of them
bool in_granules(std::initializer_list<const void *> p, std::initializer_list<int64_t> widths) {
    for (const void *x : p)
        if (!aligned16(x)) return false;
    for (int64_t n : widths)
        if (n % 8) return false;
    return true;
}
template <class T, bool TRANSPOSED>
void launch_rows(const gsplit_ctx *ctx, RowsArgs A, hipStream_t st) {
    const auto launch = [&](auto kernel, int rows, int cols, int threads) {
        A.tiles_m = group_row_tiles(A.list.n, A.G, rows);
        A.tiles_n = (int32_t)group_ceil(A.N, cols);
        hipLaunchKernelGGL(kernel, dim3(blocks(A.tiles_m * A.tiles_n)), dim3(threads), 0, st, A);
    };
    constexpr bool FLOAT = sizeof(T) == 4;
    switch (group_rows_form(A.list.n, A.G, A.K, A.N, FLOAT, TRANSPOSED, !FLOAT && in_granules({A.a, A.w, A.c}, {A.K, A.N, A.lda, A.ldc}), ctx->n_cu)) {
    case GROUP_CORE: return launch(k_grouped_rows_core<TRANSPOSED>, CORE_TILE, CORE_TILE, CT);
    case GROUP_FEW: return launch(k_grouped_rows_few<T, TRANSPOSED>, 32, 32, NT);
    case GROUP_128: return launch(k_grouped_rows<T, Tile<128, 128>, TRANSPOSED>, 128, 128, NT);
    case GROUP_64: return launch(k_grouped_rows<T, Tile<64, 64>, TRANSPOSED>, 64, 64, NT);
    }
}
template <bool TRANSPOSED>
void launch_rows(const gsplit_ctx *ctx, int32_t dtype, const RowsArgs &A, hipStream_t st) {
    if (dtype == GSPLIT_F32) launch_rows<float, TRANSPOSED>(ctx, A, st);
    else launch_rows<uint16_t, TRANSPOSED>(ctx, A, st);
}
template <class T>
auto weights_kernel(GroupForm form) {
    if constexpr (sizeof(T) == 2)
        if (form == GROUP_CORE) return k_grouped_weights_core;
    return form == GROUP_FEW ? k_grouped_weights_few<T> : form == GROUP_128 ? k_grouped_weights<T, Tile<128, 128>> : k_grouped_weights<T, Tile<64, 64>>;
}

}  // namespace

extern "C" int gsplit_grouped_linear_fwd(gsplit_ctx *ctx, const gsplit_grouped_config *c, const void *d_x, int64_t n_rows, int64_t x_stride,
                                         const int32_t *d_group_ptr, const int32_t *d_rows, const void *d_w, const float *d_bias,
                                         void *d_y, int64_t y_stride, void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        const char *e = op_check_grouped_fwd(c, d_x, n_rows, x_stride, d_group_ptr, d_rows, d_w, d_bias, d_y, y_stride);
        if (!e) e = op_apart_grouped_fwd(c, d_x, n_rows, x_stride, d_group_ptr, d_rows, d_w, d_bias, d_y, y_stride);
        if (e)
            return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_grouped_linear_fwd: ") + e);
        if (n_rows == 0) return (int)GSPLIT_OK;
        GsTimeScope ts(ctx, "grouped_fwd", -1, st);
        launch_rows<false>(ctx, c->dtype, RowsArgs{d_x, d_w, d_bias, d_y, (uint32_t)x_stride, (uint32_t)y_stride, (uint32_t)c->n_out, c->n_in, c->n_out, c->n_groups,
                                                   d_group_ptr, {d_rows, (int32_t)n_rows}, 0, 0}, st);
        return (int)GSPLIT_OK;
    });
}

extern "C" int64_t gsplit_grouped_linear_work(gsplit_ctx *ctx, const gsplit_grouped_config *c, int64_t n_rows) {
    if (!ctx) return GSPLIT_EINVAL;
    if (const char *e = op_check_grouped(c, n_rows)) {
        try { return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_grouped_linear_work: ") + e); } catch (...) { return GSPLIT_ENOMEM; }
    }
    const int64_t slabs = group_most_slabs(n_rows, c->n_groups, c->n_in, c->n_out, c->dtype == GSPLIT_F32, ctx->n_cu);
    return slabs * ((int64_t)c->n_in + 1) * c->n_out * (int64_t)sizeof(float);
}

extern "C" int gsplit_grouped_linear_bwd(gsplit_ctx *ctx, const gsplit_grouped_config *c, const void *d_x, int64_t n_rows, int64_t x_stride,
                                         const int32_t *d_group_ptr, const int32_t *d_rows, const void *d_w, const void *d_dy,
                                         int64_t dy_stride, void *d_dx, int64_t dx_stride, float *d_dw, float *d_dbias, void *d_work,
                                         void *stream) {
    if (!ctx) return GSPLIT_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    return gs_call(ctx, st, [&] {
        const char *e = op_check_grouped_bwd(c, d_x, n_rows, x_stride, d_group_ptr, d_rows, d_w, d_dy, dy_stride, d_dx, dx_stride, d_dw,
                                             d_dbias, d_work);
        GroupWeights f{};
        if (!e && d_dw) {
            f = group_weights_form(n_rows, c->n_groups, c->n_in, c->n_out, c->dtype == GSPLIT_F32,
                                   in_granules({d_x, d_dy, d_dw, d_dbias}, {c->n_in, c->n_out, x_stride, dy_stride}), ctx->n_cu);
            if (f.slabs && !d_work) e = "NULL d_work";
        }
        if (!e) e = op_apart_grouped_bwd(c, d_x, n_rows, x_stride, d_group_ptr, d_rows, d_w, d_dy, dy_stride, d_dx, dx_stride, d_dw, d_dbias,
                                         d_work, f.slabs * ((int64_t)c->n_in + 1) * c->n_out * (int64_t)sizeof(float));
        if (e) return gs_fail(ctx, GSPLIT_EINVAL, std::string("gsplit_grouped_linear_bwd: ") + e);
        const RowList list{d_rows, (int32_t)n_rows};
        if (d_dx && n_rows > 0) {
            GsTimeScope ts(ctx, "grouped_dx", -1, st);
            launch_rows<true>(ctx, c->dtype, RowsArgs{d_dy, d_w, nullptr, d_dx, (uint32_t)dy_stride, (uint32_t)dx_stride, (uint32_t)c->n_out, c->n_out, c->n_in,
                                                      c->n_groups, d_group_ptr, list, 0, 0}, st);
        }
        if (d_dw) {
            const int64_t tiles_m = group_ceil(c->n_in, f.tile), tiles_n = group_ceil(c->n_out, f.tile);
            const int pieces = group_pieces(tiles_m * tiles_n);
            const int64_t chunks = group_ceil(n_rows / f.chunk + c->n_groups, 8) * 8;          // (at most)
            WeightArgs A{d_x, d_dy, (uint32_t)x_stride, (uint32_t)dy_stride, c->n_in, c->n_out, c->n_groups, d_group_ptr, list, (int32_t)f.chunk,
                         chunks * pieces * group_ceil(tiles_m * tiles_n, pieces), pieces, (int32_t)tiles_m, (int32_t)tiles_n, d_dw, d_dbias, (float *)d_work, f.slabs};
            const dim3 grid(blocks(A.room));
            {
                GsTimeScope ts(ctx, "grouped_dw", -1, st);
                hipLaunchKernelGGL(c->dtype == GSPLIT_F32 ? weights_kernel<float>(f.form) : weights_kernel<uint16_t>(f.form), grid,
                                   dim3(f.form == GROUP_CORE ? CT : NT), 0, st, A);
            }
            if (f.slabs) {
                GsTimeScope ts(ctx, "grouped_dw_sum", -1, st);
                const int64_t quads = (int64_t)c->n_in * c->n_out / 4 + c->n_out + 4;
                hipLaunchKernelGGL(k_grouped_weights_sum, dim3((unsigned)std::min<int64_t>(group_ceil(quads, NT), 1024),
                                                               (unsigned)std::min<int64_t>(c->n_groups, n_rows / f.chunk)), dim3(NT), 0, st, A);
            }
        }
        return (int)GSPLIT_OK;
    });
}
