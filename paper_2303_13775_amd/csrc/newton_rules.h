// How matrices are grouped into launches for their Newton-Schulz steps and where their working memory lies: rules on sizes alone
// (host programs include this header too).
#pragma once

#include <algorithm>
#include <cstdint>

constexpr int NEWTON_TILE = 128;                // the large tile; the small one is 64
constexpr int NEWTON_STACKS = 24;               // of a launch: they travel in its arguments
constexpr int64_t NEWTON_CHUNK = 16384;         // elements whose squares a workgroup adds up

// A stack of `count` matrices rows x cols, or a run of one's matrices.  The steps work on m x n with m <= n (the transpose of a tall
// matrix), padded with zeros to multiples of the tile.
struct NewtonSize {
    int64_t count;
    int32_t rows, cols, m, n, mp, np;
};
inline int32_t newton_pad(int64_t x, int tile) { return (int32_t)((x + tile - 1) / tile * tile); }
inline NewtonSize newton_size(int64_t count, int32_t rows, int32_t cols, int tile) {
    const int32_t m = std::min(rows, cols), n = std::max(rows, cols);
    return {count, rows, cols, m, n, newton_pad(m, tile), newton_pad(n, tile)};
}
// 16-byte words of the working memory: X, twice; A and B; the sums of squares.  A value is two halves.
inline int64_t newton_words_x(const NewtonSize &s) { return (int64_t)s.mp * s.np / 4; }         // of one X
inline int64_t newton_words_a(const NewtonSize &s) { return (int64_t)s.mp * s.mp / 4; }         // of one A
inline int64_t newton_slots(const NewtonSize &s) { return ((int64_t)s.rows * s.cols + NEWTON_CHUNK - 1) / NEWTON_CHUNK; }
inline int64_t newton_words(const NewtonSize &s) {
    return s.count * (2 * newton_words_x(s) + 2 * newton_words_a(s) + (newton_slots(s) + 1) / 2);
}
// tiles of X, of the lower triangle of A
inline int64_t newton_tiles_x(const NewtonSize &s, int tile) { return (int64_t)(s.mp / tile) * (s.np / tile); }
inline int64_t newton_tiles_a(const NewtonSize &s, int tile) { const int64_t t = s.mp / tile; return t * (t + 1) / 2; }

// The tile of a call's matrices: the large one where its tiles of A fill the chip.
inline bool newton_large(int64_t tiles_of_a) { return tiles_of_a >= 256; }
// A launch takes stacks up to this many padded elements, so that working memory stays in proportion
constexpr int64_t NEWTON_LAUNCH = 1 << 27;

// Deals the stacks to launches: group(stacks, n) for each.  size(i): (count, rows, cols) of stack i
struct NewtonStack { int64_t tensor, first; NewtonSize size; };         // matrices first .. first + size.count - 1 of a tensor
template <class Size, class Group>
void newton_groups(int64_t n_tensors, Size size, Group group) {
    int64_t tiles = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const auto s = size(i);
        if (std::min(s.rows, s.cols) > 64) tiles += s.count * newton_tiles_a(newton_size(s.count, s.rows, s.cols, NEWTON_TILE), NEWTON_TILE);
    }
    const bool large = newton_large(tiles);
    for (int pass = 0; pass < 2; ++pass) {              // those of the large tile, then the others
        const int tile = pass == 0 ? NEWTON_TILE : 64;
        if (pass == 0 && !large) continue;
        NewtonStack in[NEWTON_STACKS];
        int n = 0;
        int64_t room = NEWTON_LAUNCH;
        for (int64_t i = 0; i < n_tensors; ++i) {
            const auto s = size(i);
            if ((large && std::min(s.rows, s.cols) > 64) != (tile == NEWTON_TILE)) continue;
            for (int64_t first = 0; first < s.count;) {
                NewtonSize one = newton_size(1, s.rows, s.cols, tile);
                if (one.m == 0) break;
                const int64_t each = (int64_t)one.mp * one.np;
                int64_t take = std::min<int64_t>(s.count - first, room / each);
                if (n == NEWTON_STACKS || (take == 0 && n > 0)) {
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
