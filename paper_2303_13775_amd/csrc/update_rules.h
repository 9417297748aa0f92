// How the norm and the update deal their elements to workgroups: rules on sizes alone (host programs include this header too).
#pragma once

#include <cstdint>

// Elements of a chunk, which a workgroup of 256 takes at a time: four workgroups a compute unit while that leaves each thread
// at least four elements, then up to 16384.
inline int update_chunk(int64_t total, int n_cu) {
    int64_t chunk = 1024;
    while (chunk < 16384 && chunk * 4 * n_cu < total) chunk *= 2;
    while (total / chunk > (1 << 30)) chunk *= 2;
    return (int)chunk;
}

// Norm and clipping in one launch of one workgroup
constexpr int UPDATE_CLIP_SMALL = 32768;
inline bool update_clip_small(int64_t total) { return total <= UPDATE_CLIP_SMALL; }
// the norm formed by every workgroup of the update
inline bool update_norm_here(int64_t total) { return total <= 32768; }
