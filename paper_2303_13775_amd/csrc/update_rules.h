// How the norm and the update deal their elements to workgroups: rules on sizes alone (host programs include this header too).
#pragma once

#include <cstdint>

// Elements of a chunk of the norm, which workgroups of 256 threads that stay, four a compute unit, take one after the other: from four
// elements a thread up to 8192 a chunk.
inline int norm_chunk(int64_t total, int n_cu) {
    int64_t chunk = 1024;
    while (chunk < 8192 && chunk * 4 * n_cu < total) chunk *= 2;
    while (total / chunk > (1 << 30)) chunk *= 2;
    return (int)chunk;
}
// Elements of a chunk of the passes that write, a workgroup of 256 threads each: as many as give a compute unit four, up to `most`: 4096
// for clipping (400 M gradients 605 us; 2048 648, 8192 620), 2048 for the update (250 M elements 1355 us; 1024 1363, 4096 1445).
// Workgroups that stay, four a compute unit, are slower (679; 1629).
inline int update_chunk(int64_t total, int most, int n_cu) {
    int64_t chunk = 1024;
    while (chunk < most && chunk * 4 * n_cu < total) chunk *= 2;
    while (total / chunk > (1 << 23)) chunk *= 2;       // (a launch has less than 2^32 threads)
    return (int)chunk;
}
// An update whose parameters, moments and gradients (16 bytes an element) outgrow the 256 MB cache says that what it moves is not read
// again (32 M elements 161 us, 195 without; 250 M 1441 and 1472; but 16 M 87 and 85), and its workgroups ask for LDS that they do not
// use, so that three are on a compute unit and not eight: the memory does better with fewer places at once in each of the eight
// streams (250 M 1355 us; eight workgroups 1410, five 1381, four 1380, two 1379).
inline bool update_large(int64_t total) { return total > 16 << 20; }
constexpr int UPDATE_LARGE_LDS = 52 << 10;
// A pass of many workgroups reads the norm from one slot, which a launch of its own forms, instead of all of them (400 M gradients
// clipped 612 us, 636).
inline bool norm_in_one_slot(int64_t workgroups, int n_cu) { return workgroups > 8 * n_cu; }

// Norm and clipping in one launch of one workgroup of 1024 threads, against two launches.  Its sixteen waves take a chunk each (1024
// elements of a tensor, of which every tensor has one at least) and go round for the norm and again for clipping.  One tensor of
// 10 k elements 5.2 us / 9.4, of 20 k 5.7 / 9.4, of 32 k 6.8 / 9.4; 16 tensors of 50 5.5 / 9.4, 32 7.7 / 9.3, 48 9.5 to 10.0 / 9.6, 72 13.7 / 9.9,
// 144 26.4 / 10.2.  (total / 1024 + tensors: not less than the chunks)
constexpr int UPDATE_CLIP_SMALL = 32768, UPDATE_CLIP_SMALL_CHUNKS = 48;
inline bool update_clip_small(int64_t total, int64_t tensors = 1) {
    return total <= UPDATE_CLIP_SMALL && total / 1024 + tensors <= UPDATE_CLIP_SMALL_CHUNKS;
}
// The norm formed by every workgroup (of 1024 threads) of the update, against a launch of its own: one tensor of 10 k elements 5.8 / 9.7,
// of 20 k 5.9 / 9.9, of 32 k 6.3 / 9.9, of 65 k 8.6 / 7.7 on another card; 32 tensors of 50 7.5 / 10.0, 72 (which a launch takes) 10.5 / 10.6.
inline bool update_norm_here(int64_t total) { return total <= 32768; }
