// How rows sorted by group and the products by group are dealt to workgroups: rules on sizes alone (host programs include this
// header too).
#pragma once

#include <algorithm>
#include <cstdint>

// -- sorting rows by their group: workgroups of sixteen waves, a run of rows a wave --
constexpr int GROUP_WAVES = 16;
struct GroupRuns { int workgroups; int64_t rows_a_wave; };
// `counters`: how many the scratch memory holds; a workgroup has one for every group
inline GroupRuns group_runs(int64_t n_rows, int n_groups, int64_t counters, int n_cu) {
    const int64_t rounds = (n_rows + 63) / 64;
    int64_t most = std::min<int64_t>(n_cu, counters / n_groups);
    if (rounds <= 4 * GROUP_WAVES) most = 1;        // (one launch instead of two)
    const int64_t a_wave = std::max<int64_t>(1, (rounds + most * GROUP_WAVES - 1) / (most * GROUP_WAVES));
    return {(int)std::max<int64_t>(1, (rounds + a_wave * GROUP_WAVES - 1) / (a_wave * GROUP_WAVES)), a_wave * 64};
}

// -- the products: tiles of `rows` x `cols` --
struct GroupTile { int rows, cols; };
inline int64_t group_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }
// tiles of rows of all groups, at most: every group that has rows leaves one of its tiles short
inline int64_t group_row_tiles(int64_t n_rows, int n_groups, int rows) { return n_rows / rows + std::min<int64_t>(n_groups, n_rows); }

// -- weight gradients: the rows of a group are taken in chunks where one group's tiles do not fill the chip --
inline int64_t group_chunk(int64_t n_rows, int64_t tiles_of_a_group, int n_cu) {
    if (tiles_of_a_group >= n_cu) return std::max<int64_t>(n_rows, 1);
    const int64_t want = group_ceil(2 * n_cu, tiles_of_a_group);        // chunks of all rows
    return std::max<int64_t>(256, group_ceil(group_ceil(n_rows, want), 64) * 64);
}
// slabs: the chunks of those groups that have more than one
inline int64_t group_slabs(int64_t n_rows, int64_t chunk) { return 2 * (n_rows / chunk); }
