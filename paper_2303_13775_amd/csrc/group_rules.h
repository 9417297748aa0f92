// How rows sorted by group and the products by group are dealt to workgroups: rules on sizes alone (host programs include this
// header too).
#pragma once

#include <algorithm>
#include <cstdint>

// -- sorting rows by their group: workgroups of sixteen waves, a run of rows a wave --
constexpr int GROUP_WAVES = 16;
struct GroupRuns { int workgroups; int64_t rows_a_wave; };
// `counters`: how many the scratch memory holds; a workgroup has one for every group
// One workgroup up to 4096 rows (us of one launch / two: 2048 rows of 64 groups 5.2 / 8.5, 4096 of 4, 64, 512 groups 4.8 / 9.5, 6.1 / 8.8,
// 7.3 / 11.1; 6000 6.7 / 9.7, 9.4 / 9.0, 11.7 / 11.3; 16384 of 64 18.4 / 9.7).
inline GroupRuns group_runs(int64_t n_rows, int n_groups, int64_t counters, int n_cu) {
    const int64_t rounds = (n_rows + 63) / 64;
    int64_t most = std::min<int64_t>(n_cu, counters / n_groups);
    if (rounds <= 4 * GROUP_WAVES) most = 1;        // one launch, not two
    const int64_t a_wave = std::max<int64_t>(1, (rounds + most * GROUP_WAVES - 1) / (most * GROUP_WAVES));
    return {(int)std::max<int64_t>(1, (rounds + a_wave * GROUP_WAVES - 1) / (a_wave * GROUP_WAVES)), a_wave * 64};
}

// -- the products: tiles of `rows` x `cols` --
inline int64_t group_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }
// tiles of rows of all groups, at most: every group that has rows leaves one of its tiles short
inline int64_t group_row_tiles(int64_t n_rows, int n_groups, int rows) { return n_rows / rows + std::min<int64_t>(n_groups, n_rows); }

// bfloat16 rows of whole granules (16 bytes): tiles of 256 x 256 that go straight into LDS, against tiles of 128 or 64 through registers
// (us, y / dx / dW).  16384 rows of 16 groups 512 x 512 22 / 22 / 37 and 31 / 26 / 53; 8192 of 8 1024 x 1024 34 / 34 / 53 and 50 / 42 / 79; 4096 of 2
// 2048 x 2048 56 / 55 / 81 and 85 / 69 / 108; 32768 of 128 512 x 512 41 / 41 / 76 and 50 / 43 / 97; but 8192 of 8 512 x 512 21 / 20 / 33 and
// 19 / 18 / 37, 65536 of 8 128 x 128 21 / 21 / 34 and 18 / 17 / 41.
inline bool group_core_rows(int64_t n_rows, int n_groups, int64_t k, int64_t n, int n_cu) {
    return k >= 128 && n > 128 && n_rows >= 64 * (int64_t)n_groups && group_ceil(n_rows, 256) * group_ceil(n, 256) >= n_cu / 2;
}
inline bool group_core_weights(int64_t n_rows, int n_groups, int64_t n_in, int64_t n_out, int n_cu) {
    return n_in >= 128 && n_out >= 128 && n_rows >= 64 * (int64_t)n_groups &&
           group_ceil(n_in, 256) * group_ceil(n_out, 256) * group_ceil(n_rows, 256) >= n_cu / 2;
}

// Few rows: workgroups of 32 x 32 without a loop of barriers, against tiles of 64 (us, y / dx, few / tiles).  Where groups have few rows
// (float 64 rows of 8 groups, 2048 x 2048: 31 / 73, 30 / 52; 2048 of 64, 512 x 512: 29 / 48, 33 / 43; 512 of 8, 1024 x 1024: 27 / 41,
// 31 / 29; bfloat16 64 of 8: 17 / 24, 16 / 21; 2048 of 64: 15 / 16, 16 / 15; 512 of 8: 14 / 13.5, 14 / 10), and forward where few tiles
// leave compute units to the longer way (float 1024 x 256 x 172 of 16 5.9 / 9.7, 4096 of 16 10.5 / 10.1, 8192 of 16 22 / 16).
inline bool group_few_rows(int64_t n_rows, int n_groups, int64_t n, bool is_float, bool transposed, int n_cu) {
    const int64_t a_group = n_rows / std::max<int64_t>(1, std::min<int64_t>(n_groups, n_rows));
    return a_group <= (is_float ? 48 : 32) || (is_float && !transposed && group_row_tiles(n_rows, n_groups, 32) * group_ceil(n, 32) <= 3 * n_cu);
}
// The weight gradients of few rows: a group's rows in one go, as long as that is short
inline bool group_few_weights(int64_t n_rows, int n_groups, int64_t n_in, int64_t n_out, int n_cu) {
    return n_rows <= 4096 && n_rows <= 512 * (int64_t)n_groups && n_groups * group_ceil(n_in, 32) * group_ceil(n_out, 32) <= 4 * n_cu;
}

// -- weight gradients: tiles of 128 or of 64 --
inline bool group_weights_large(int64_t n_in, int64_t n_out) { return n_in > 64 && n_out > 64 && n_in * n_out >= 1 << 18; }

// The rows of a group are taken in chunks where one group's tiles do not fill the chip: as many chunks of all rows as give `workgroups`.
// Short chunks even out groups of all sizes, and cost the sum over them.  Tiles of 128 and 64, four workgroups a compute unit (three, two):
// 20011 rows of 24 groups 1000 x 1021 bf16 157 us (165, 184), float, before chunks went in pieces, 400 (422, 489), 65536 of 8 512 x 512 float 300 (279, 349).  Tiles of 256, one
// every two compute units (one, two): 65536 of 8 512 x 512 82 us (97, 123), 20011 of 24 1000 x 1024 115 (112, 160).
inline int64_t group_chunk(int64_t n_rows, int64_t tiles_of_a_group, int64_t workgroups) {
    const int64_t want = group_ceil(workgroups, tiles_of_a_group);
    if (want <= 1) return std::max<int64_t>(n_rows, 1);
    return std::max<int64_t>(256, group_ceil(group_ceil(n_rows, want), 64) * 64);
}
// Pieces of a chunk's tiles, which go to the XCDs in turn: more of them are dealt more evenly and share less in an XCD's L2 (whole chunks,
// 2, 4, 8 pieces: 65536 rows of 64 groups 2048 x 2048 bf16 1360, 1010, 962, 1055 us; 20011 of 24 1000 x 1024 113, 102, 103, 105, float
// 1000 x 1021 388, 365, 341, 353; 65536 of 8 512 x 512 float 294, 294, 260, 274).
inline int group_pieces(int64_t tiles) { return tiles >= 16 ? 4 : 1; }
// slabs: the chunks of those groups that have more than one
inline int64_t group_slabs(int64_t n_rows, int64_t chunk) { return n_rows > chunk ? 2 * (n_rows / chunk) : 0; }

// Which kernel forms y or dx [n_rows x n] of a contraction of k, and which the weight gradients; granules: rows of whole 16 bytes.  (The tiles
// through registers fetch eight elements of a row at once.)
// Tiles of 128 where they fill the chip and are not mostly empty columns (us forward, 128 / 64: 65536 rows of 8 groups float 100 x 64 37 / 20,
// 256 x 100 56 / 51, 256 x 172 83 / 74, 100 x 256 57 / 56, 32768 of 16 512 x 300 102 / 108, 60000 of 8 512 x 511 228 / 289; bf16 100 x 64 15.5 / 11.0,
// 256 x 172 31 / 28, 512 x 300 32 / 35, 512 x 511 78 / 102; dx of 256 x 100 float 49 / 56).
enum GroupForm { GROUP_CORE, GROUP_FEW, GROUP_128, GROUP_64 };
inline GroupForm group_rows_form(int64_t n_rows, int n_groups, int64_t k, int64_t n, bool is_float, bool transposed, bool granules, int n_cu) {
    if (!is_float && granules && group_core_rows(n_rows, n_groups, k, n, n_cu)) return GROUP_CORE;
    if (k < 8 || group_few_rows(n_rows, n_groups, n, is_float, transposed, n_cu)) return GROUP_FEW;
    return n > 192 && group_row_tiles(n_rows, n_groups, 128) * group_ceil(n, 128) >= n_cu ? GROUP_128 : GROUP_64;
}
struct GroupWeights { GroupForm form; int tile; int64_t chunk, slabs; };
inline GroupWeights group_weights_form(int64_t n_rows, int n_groups, int64_t n_in, int64_t n_out, bool is_float, bool granules, int n_cu) {
    GroupWeights f{};
    f.form = !is_float && granules && group_core_weights(n_rows, n_groups, n_in, n_out, n_cu) ? GROUP_CORE
             : group_few_weights(n_rows, n_groups, n_in, n_out, n_cu) ? GROUP_FEW : group_weights_large(n_in, n_out) ? GROUP_128 : GROUP_64;
    f.tile = f.form == GROUP_CORE ? 256 : f.form == GROUP_FEW ? 32 : f.form == GROUP_128 ? 128 : 64;
    f.chunk = f.form == GROUP_FEW ? std::max<int64_t>(n_rows, 1)
                                  : group_chunk(n_rows, group_ceil(n_in, f.tile) * group_ceil(n_out, f.tile), f.form == GROUP_CORE ? n_cu / 2 : 4 * n_cu);
    f.slabs = group_slabs(n_rows, f.chunk);
    return f;
}
// slabs that a call may need, whatever its addresses
inline int64_t group_most_slabs(int64_t n_rows, int n_groups, int64_t n_in, int64_t n_out, bool is_float, int n_cu) {
    const bool granules = n_in % 8 == 0 && n_out % 8 == 0;
    return std::max(group_weights_form(n_rows, n_groups, n_in, n_out, is_float, granules, n_cu).slabs,
                    group_weights_form(n_rows, n_groups, n_in, n_out, is_float, false, n_cu).slabs);
}
