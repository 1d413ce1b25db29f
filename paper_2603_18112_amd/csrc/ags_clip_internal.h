// Internal declarations of gradient clipping (include/ags_clip.h), shared by
// its host code and its kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ags_clip.h"

namespace ags {

// A block's share: `count` consecutive elements of one segment.
struct ClipPiece {
    int64_t in_off, out_off;  // elements from the tensors' starts
    int32_t count;
    int32_t in_base, out_base;
    int32_t group;
    int32_t in_dt, out_dt;
};

constexpr int kClipBlock = 256;

// Pieces are at least this many elements (a segment's last one aside), and as
// long as kClipPieces of them cover a large set: the block that finishes last
// adds up one partial per piece.
constexpr int64_t kClipMinPiece = 8192;
constexpr int64_t kClipPieces = 4096;

// A set this small goes through one block in one launch.
constexpr int64_t kClipSmallElems = 32768;
constexpr int kClipSmallPieces = 128;

// Blocks count themselves in on kClipCounters counters, each in a line of its
// own, and the last on each of those on a root: with all blocks on one counter
// the additions, some 14 ns each, took longer than the reads (MI355X, 25.6
// million bf16 in 3251 pieces: 46.7 us).
constexpr int kClipCounters = 64, kClipCounterStride = 64;  // dwords
constexpr size_t kClipCounterBytes = (kClipCounters + 1) * kClipCounterStride * sizeof(unsigned);

// Device pointers that travel in a kernel's arguments (a kernel takes at
// most 4 KiB of them); larger sets go through a table in the workspace.
constexpr int kClipArgPtrs = 440;

struct ClipArgs {
    const void* ptr[kClipArgPtrs];  // inputs, then outputs
    const void* const* table;       // the same in device memory, or NULL
    const ClipPiece* pieces;
    const int32_t* group_begin;  // [n_groups + 1] piece ranges
    double* partials;            // [n_pieces]
    float2* coef;                // [n_groups] c_g as a product
    unsigned* done;              // finished pieces' counters, 0 between calls
    float* norms;                // [n_groups], the caller's
    double max_norm, eps;
    int32_t n_in, n_groups, n_pieces;
    int32_t in_place;
};
static_assert(sizeof(ClipArgs) <= 4096, "kernel arguments");

struct ClipTableArgs {
    const void* ptr[kClipArgPtrs];
    const void** table;
    int32_t first, count;
};

// The launchers live with the kernels.  They are weak so that a library of
// the host code alone (a sanitizer build) links; a launch there is an error.
__attribute__((weak)) hipError_t launch_clip_table(const ClipTableArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_clip_norm(const ClipArgs&, int kind, hipStream_t);
__attribute__((weak)) hipError_t launch_clip_small(const ClipArgs&, int kind, bool scale, hipStream_t);
__attribute__((weak)) hipError_t launch_clip_scale(const ClipArgs&, hipStream_t);

}  // namespace ags
