// Which form a kernel over rows of logits takes: rules on sizes alone (host programs include this header too).
#pragma once

#include <cstdint>

// lanes a row x elements a lane holds; then rows that are read twice
enum : int { ROW_16x8, ROW_16x16, ROW_64x8, ROW_64x16, ROW_256x8, ROW_256x16, ROW_256x32, ROW_512x32, ROW_512x64, ROW_1024x64, ROW_STREAMED };

// the first form whose registers hold a row of C elements, `piece` elements in 16 bytes
inline int row_form(int C, int piece) {
    const int held[] = {16 * 8, 16 * 16, 64 * 8, 64 * 16, 256 * 8, 256 * 16, 256 * 32, 512 * 32, 512 * 64, 1024 * 64};
    for (int f = 0; f < ROW_STREAMED; ++f)
        if (C / piece * piece <= held[f]) return f;
    return ROW_STREAMED;
}

// lanes a row of the kernels that stream rows
inline int row_part(int C) { return C <= 256 ? 16 : C <= 1024 ? 64 : 256; }

// Threads of the workgroup that takes a pair of the preference loss from its rows to their gradient (0: three launches over all
// rows, all pairs and all rows)
inline int preference_whole(int64_t n_rows, int64_t n_pairs, int64_t row_bytes, int n_cu) {
    if (n_pairs >= (1 << 24)) return 0;         // (a launch has less than 2^32 threads)
    const int64_t pair_bytes = n_rows * row_bytes / n_pairs;
    if (pair_bytes > (64 << 10) && n_pairs < 2 * n_cu) return 0;
    return n_rows <= 4 * n_pairs ? 64 : 256;
}
