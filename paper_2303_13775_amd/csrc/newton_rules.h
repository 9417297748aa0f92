// How matrices are grouped into launches for their Newton-Schulz steps and where their working memory lies: rules on sizes alone
// (host programs include this header too).
#pragma once

#include <algorithm>
#include <cstdint>

constexpr int NEWTON_TILE = 128;                // the large tile; the small one is 64
constexpr int NEWTON_ONE = 1;                   // (not a tile:) the kernel that takes a matrix in LDS, at most 64 x NEWTON_ONE_N, padded to 64
constexpr int64_t NEWTON_ONE_N = 384;
constexpr int NEWTON_STACKS = 24;               // of a launch: they travel in its arguments

// A stack of `count` matrices rows x cols, or a run of one's matrices.  The steps work on m x n with m <= n (the transpose of a tall
// matrix), padded with zeros to multiples of the tile.
struct NewtonSize {
    int64_t count;
    int32_t rows, cols, m, n, mp, np;
};
inline int32_t newton_pad(int64_t x, int tile) { return (int32_t)((x + tile - 1) / tile * tile); }
inline NewtonSize newton_size(int64_t count, int32_t rows, int32_t cols, int tile) {
    const int32_t m = std::min(rows, cols), n = std::max(rows, cols);
    const int pad = tile == NEWTON_ONE ? 64 : tile;
    return {count, rows, cols, m, n, newton_pad(m, pad), newton_pad(n, pad)};
}
// 16-byte words of the working memory: X, twice; A and B; the sums of squares.  A value is two halves.
inline int64_t newton_words_x(const NewtonSize &s) { return (int64_t)s.mp * s.np / 4; }         // of one X
inline int64_t newton_words_a(const NewtonSize &s) { return (int64_t)s.mp * s.mp / 4; }         // of one A
// elements whose squares a workgroup adds up: a thread's four pieces of four, or a 1024th of the matrix
#ifdef __HIPCC__
__host__ __device__
#endif
inline int64_t newton_chunk(int64_t size) { return size <= 4096 * 1024 ? 4096 : (size / 1024 + 4095) / 4096 * 4096; }
inline int64_t newton_slots(const NewtonSize &s) {
    const int64_t size = (int64_t)s.rows * s.cols, chunk = newton_chunk(size);
    return (size + chunk - 1) / chunk;
}
inline int64_t newton_words(const NewtonSize &s, int tile) {
    if (tile == NEWTON_ONE) return 0;
    return s.count * (2 * newton_words_x(s) + 2 * newton_words_a(s) + (newton_slots(s) + 1) / 2);
}
// tiles of X, of the lower triangle of A
inline int64_t newton_tiles_x(const NewtonSize &s, int tile) { return (int64_t)(s.mp / tile) * (s.np / tile); }
inline int64_t newton_tiles_a(const NewtonSize &s, int tile) { const int64_t t = s.mp / tile; return t * (t + 1) / 2; }

// The tile of a call's matrices of more than 64 rows, by the tiles of 128 x 128 that all their A have (us of five steps, large / small):
// four of 1024 x 1024 (144) 470 / 580, one of 2048 x 2048 (136) 799 / 1023; 32 of 200 x 200 (96) 193 / 144, two of 1024 x 4096 (72) 893 / 884,
// one of 1024 x 1024 (36) 420 / 244, 16 of 128 x 2048 (16) 339 / 216.
inline bool newton_large(int64_t tiles_of_a) { return tiles_of_a >= 128; }
// A launch takes stacks up to this many padded elements, so that working memory stays in proportion; a matrix of more is one by itself
constexpr int64_t NEWTON_LAUNCH = 1 << 27;

// Matrices that one workgroup each takes through all steps (one launch).  By itself a small matrix is done sooner that way; in front of
// launches for larger ones few of them would only add theirs (us, by themselves / in the launches; 64 of 64 x 64 18 / 70, 1024 73 / 167, one of
// 64 x 384 50 / 81, 1024 233 / 428; beside one of 256 x 256: 64 of 64 x 64 124 / 109, 256 128 / 127, 1024 180 / 231, 64 of 64 x 384 155 / 120, 256
// 169 / 181, 1024 331 / 485).
inline bool newton_one(int64_t rows, int64_t cols) { return std::min(rows, cols) <= 64 && std::max(rows, cols) <= NEWTON_ONE_N; }
inline bool newton_ones(int64_t small, int64_t others) { return others == 0 || small >= 256; }

// Deals the stacks to launches: group(stacks, n, tile) for each.  size(i): (count, rows, cols) of stack i
struct NewtonStack { int64_t tensor, first; NewtonSize size; };         // matrices first .. first + size.count - 1 of a tensor
template <class Size, class Group>
void newton_groups(int64_t n_tensors, Size size, Group group) {
    int64_t tiles = 0, small = 0, others = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const auto s = size(i);
        if (s.count == 0 || s.rows == 0 || s.cols == 0) continue;
        if (std::min(s.rows, s.cols) > 64) {
            const int64_t t = newton_pad(std::min(s.rows, s.cols), 128) / 128;
            tiles += s.count * (t * (t + 1) / 2);
        }
        (newton_one(s.rows, s.cols) ? small : others) += s.count;
    }
    const bool large = newton_large(tiles), ones = newton_ones(small, others);
    const auto tile_of = [&](int32_t rows, int32_t cols) {
        return ones && newton_one(rows, cols) ? NEWTON_ONE : large && std::min(rows, cols) > 64 ? NEWTON_TILE : 64;
    };
    for (const int tile : {NEWTON_TILE, 64, NEWTON_ONE}) {
        NewtonStack in[NEWTON_STACKS];
        int n = 0;
        int64_t room = NEWTON_LAUNCH;
        for (int64_t i = 0; i < n_tensors; ++i) {
            const auto s = size(i);
            if (s.rows == 0 || s.cols == 0 || tile_of(s.rows, s.cols) != tile) continue;
            for (int64_t first = 0; first < s.count;) {
                NewtonSize one = newton_size(1, s.rows, s.cols, tile);
                const int64_t each = (int64_t)one.mp * one.np;
                int64_t take = std::min<int64_t>(s.count - first, room / each);
                if (n == NEWTON_STACKS || (take <= 0 && n > 0)) {           // (below 0: behind a matrix of more than a launch takes)
                    group(in, n, tile);
                    n = 0; room = NEWTON_LAUNCH;
                    continue;
                }
                take = std::max<int64_t>(take, 1);
                one.count = take;
                in[n++] = {i, first, one};
                room -= take * each;
                first += take;
            }
        }
        if (n) group(in, n, tile);
    }
}
