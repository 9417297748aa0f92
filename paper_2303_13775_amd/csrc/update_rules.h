// How the norm and the update deal their elements to workgroups: rules on sizes alone (host programs include this header too).
#pragma once

#include <cstdint>

// Elements of a chunk, which a workgroup takes at a time: four workgroups of 256 threads a compute unit while that leaves each thread
// at least four elements, then up to 16384 (250 M elements of the update 1735 us, with 4096 1715, with 65536 1782; 387 gradients of
// 400 M elements clipped 680, 694, 720).
inline int update_chunk(int64_t total, int n_cu) {
    int64_t chunk = 1024;
    while (chunk < 16384 && chunk * 4 * n_cu < total) chunk *= 2;
    while (total / chunk > (1 << 30)) chunk *= 2;
    return (int)chunk;
}

// Norm and clipping in one launch of one workgroup of 1024 threads, against two launches: 10 k elements 5.4 us / 8.6, 20 k 6.6 / 8.7,
// 40 k 8.4 / 8.7, 65 k 11.4 / 8.7.
constexpr int UPDATE_CLIP_SMALL = 32768;
inline bool update_clip_small(int64_t total) { return total <= UPDATE_CLIP_SMALL; }
// The norm formed by every workgroup (of 1024 threads) of the update, against a launch of its own: 10 k elements 5.8 / 7.7, 20 k 6.4 /
// 7.7, 40 k 7.5 / 7.7, 65 k 8.6 / 7.7.
inline bool update_norm_here(int64_t total) { return total <= 32768; }
