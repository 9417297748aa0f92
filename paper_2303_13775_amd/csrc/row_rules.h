// Which form a kernel over rows of logits takes: rules on sizes alone (host programs include this header too).
#pragma once

#include <cstdint>

// lanes a row x elements a lane holds
enum : int {
    ROW_16x8, ROW_16x16, ROW_16x32, ROW_64x16, ROW_64x32, ROW_256x8, ROW_256x32, ROW_256x64, ROW_512x64, ROW_1024x64, ROW_1024x96,
    ROW_512x128_RAW, ROW_1024x128_RAW, ROW_STREAMED
};

// The form of n_rows rows of C elements, `piece` of them in 16 bytes (4: float, 8: bfloat16): the fewest lanes whose registers hold
// the row, as long as the lanes of a wave hide the memory's latency.  Policy loss, us (taken / the next form up or down):
//   lanes: 32768 x 172 float 16 10.5 / 64 22.2, 32768 x 512 bf16 16 13.8 / 64 23.7 (a row's double arithmetic is a wave's, whatever
//     number of rows the wave has); 32768 x 1024 float 64 43.6 / 256 59.8; 32768 x 2048 bf16 64 45.0 / 256 60.6, float 64 91 / 256 84.7
//   elements a lane: 32768 x 128 float 8 8.1 / 16 8.6; 32768 x 256 16 11.9 / 32 13.7; 32768 x 1024 16 43.6 / 32 44.9; 32768 x 4096
//     float, 256 lanes, 32 172 / 64 168 / 16 172, bf16 32 87.7 / 64 110 / 16 87.6; 8192 x 16384 float 256 x 64 183 / 512 x 32 195
//   bfloat16 rows as they are, exponentials formed twice, in half the registers, where a compute unit then holds two rows instead
//     of one: 2048 x 65536 94.6 / 100, 2048 x 50001 92.7 / 102; no more rows than compute units: 1 x 65536 9.2 / 7.4.  Narrower ones
//     gain nothing: 4096 x 32768 95.1 / 91.9, 16384 x 8192 87.2 / 84.7
//   rows in all registers of a compute unit, against reading them twice: 1024 x 70000 float 96 a lane 107 / 127, bf16 61.6 / 64.6 (as
//     they are), 1024 x 98304 147 / 169, 80.5 / 85.4; 1024 x 131072 bf16 as they are 107 / 118.
inline int row_form(int64_t n_rows, int C, int piece, int n_cu) {
    const int n = C / piece * piece;        // (what is behind the last whole piece has registers of its own)
    if (n <= 16 * 8) return ROW_16x8;
    if (n <= 16 * 16) return ROW_16x16;
    if (n <= 16 * 32) return ROW_16x32;
    if (n <= 64 * 16) return ROW_64x16;
    if (n <= 64 * 32) return piece == 4 ? ROW_256x8 : ROW_64x32;
    if (n <= 256 * 32) return ROW_256x32;
    if (n <= 256 * 64) return ROW_256x64;
    if (n <= 512 * 64) return ROW_512x64;
    if (n <= 1024 * 64) return piece == 4 || n_rows <= n_cu ? ROW_1024x64 : ROW_512x128_RAW;
    if (n <= 1024 * 96) return ROW_1024x96;
    return piece == 8 && n <= 1024 * 128 ? ROW_1024x128_RAW : ROW_STREAMED;
}

// Lanes a row of the preference loss, which streams rows.  16 x 500 x 2 rows of 2048 float, three launches: 64 lanes 69 us, 256 89.
inline int row_part(int C) { return C <= 256 ? 16 : C <= 4096 ? 64 : 256; }

// Threads of the workgroup that takes a pair of the preference loss from its rows to their gradient; 0: three launches, over all
// rows, all pairs and all rows.  A row a team up to what fills the chip with all pairs (in us, 1024 / 256 threads: 512 pairs of
// 2 x 32 rows of 172 17.4 / 20.9, 2048 of 2 x 16 40 / 26.6).  The call takes as long as its longest pair at least, and the host
// knows their mean alone: a workgroup pays where its teams go round once for a mean pair, and a few times more where there are pairs
// enough for the long ones to come out even.  In us, float, lengths all alike / uniform from 0 / exponential / one pair of eight times the
// others' (three launches, whatever the lengths):
//   once        256 pairs of 32 x 172 7.7 / 8.3 / 12 / 19 (14.7), 512 of 64 x 172 18 / 21 / 28 / 37 (25), 512 of 16 x 2048 31 / 34 / 47 / 63
//               (40), 64 of 16 x 2048 10.5 / 15 / 29 / 47 (14)
//   twice       256 of 32 x 2048 34 / 36 / 64 / 107 (40), 128 of 32 x 2048 19 / 28 / 60 / 100 (25): launches; 1024 of 32 x 172 16 / 19 / 30 / 45
//               (25), 2048 of 32 x 172 27 / 32 / 40 / 54 (43), 4096 of 8 x 2048 109 / 115 / 130 / 125 (138): workgroups
//   four times  16 of 64 x 2048 29 / 43 / 83 / 137 (15), 1024 of 64 x 172 30 / 38 / 58 / 98 (40): launches; 8192 of 16 x 172 56 / 64 / 84 / 104
//               (85), 16384 of 16 x 172 102 / 113 / 137 / 136 (157): workgroups
//   eight       1024 of 32 x 2048 125 / 135 / 200 / 326 (130), 8192 of 32 x 47 68 / 88 / 129 / 165 (86): launches
// Where the team is the whole workgroup its rows come one after the other: 512 pairs of 8 x 65536 547 / 757 / 1096 / 1957 (549), of 2 x
// 65536 123 / 149 / 269 / 430 (134).  So those pairs have a row a sequence (as many rows as sequences, and pairs for the chip: 2 x 65536
// above, alike; or narrow ones, 100 of 2 x 8000 12 / 20 / 40 / 64 (15)), or are very many (4096 of 2 x 20000 288 / 297 / 324 / 319 (345)).
inline int preference_whole(int64_t n_rows, int64_t n_pairs, int C, int n_cu) {
    if (n_pairs >= (1 << 24)) return 0;         // (a launch has less than 2^32 threads)
    const int lanes = row_part(C);
    const int64_t rows = (n_rows + n_pairs - 1) / n_pairs;      // of a pair, on average
    if (lanes == 256) {
        const bool one_each = n_rows == 2 * n_pairs || n_rows <= 2;
        return (one_each && (n_pairs >= 2 * n_cu || C <= 8192)) || (rows <= 2 && n_pairs >= 16 * n_cu) ? 256 : 0;
    }
    const int64_t room = (int64_t)n_cu * 2048 / n_pairs, want = rows * lanes < room ? rows * lanes : room;
    const int threads = want <= 64 ? 64 : want <= 256 || room < 1024 ? 256 : 1024;
    const int quarters = n_pairs < 4 * n_cu ? 5 : n_pairs < 32 * n_cu ? 8 : 16;         // of a round
    return 4 * rows * lanes <= quarters * threads ? threads : 0;
}

// Parts of a row where there are few rows: two workgroups a compute unit, parts of at least 4096 elements, at most 64 of them.
// Policy loss, parts / whole rows: 1 x 131072 float 9.4 / 21.6, bf16 9.6 / 16.7, 1 x 70000 9.1 / 10.4, 9.1 / 8.9, 64 x 131072 16.3 /
// 23.1, 11.7 / 17.2, 64 x 70000 12.5 / 12.9, 11.0 / 10.4; 100 x 131072 32.0 / 31.8, 19.2 / 18.5, 100 x 70000 16.3 / 14.5, 12.9 / 10.5.
// Preference loss: 1 pair of 65536 12.4 / 28, 120 pairs 39 / 47.
constexpr int GS_ROW_PARTS = 8192;      // (row, part) pairs the context's scratch holds
constexpr int GS_ROW_PART_BYTES = 20;   // of each
inline int row_chunks(int64_t n_rows, int C, int n_cu) {
    int64_t chunks = (2 * n_cu + n_rows - 1) / n_rows;
    if (chunks > C / 4096) chunks = C / 4096;
    if (chunks > GS_ROW_PARTS / n_rows) chunks = GS_ROW_PARTS / n_rows;
    return chunks < 1 ? 1 : chunks > 64 ? 64 : (int)chunks;
}
inline bool policy_in_parts(int64_t n_rows, int C, int piece, int n_cu) { return C / piece * piece > 1024 * 64 && n_rows <= n_cu / 4; }
inline bool preference_in_parts(int64_t n_rows, int C, int n_cu) { return C > 8192 && n_rows < n_cu; }
