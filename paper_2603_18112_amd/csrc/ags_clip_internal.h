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

// Pieces are at least kClipMinPiece elements (a segment's last one aside), and
// as long as clip_pieces() of them cover a large set: so many that blocks of
// uneven length even out, but for few segments, whose pieces are nearly all of
// one length, no more than fit the card at once; the block that finishes last
// adds up one partial per piece.  MI355X, 1024 pieces against 4096, norm / norm
// and scaling into another tensor: 1 segment of 25.5M bf16 14.4 / 32.7 us against
// 17.8 / 34.4, 138M fp32 87 / 280 against 92 / 285; 16 segments of 1M bf16 12.9 /
// 24.7 against 15.0 / 27.1, of 25.5M 130 / 456 against 131 / 441; 1288 segments
// of 2 to 2.4M fp32 138 / 390 against 127 / 350, 32 tensors of 138M fp32 in all
// 89.2 against 87.2.  At least 32768 elements against 8192: 9.5 / 15.5 against
// 7.1 / 11.1 (1M fp32); 16384: 9.1 / 17.8 against 9.4 / 16.4 (5M fp32).
constexpr int64_t kClipMinPiece = 8192;
constexpr int64_t clip_pieces(int64_t segments) { return segments <= 16 ? 1024 : 4096; }

// The norm's pass leaves the end of a large set in the caches for the scaling
// pass, which starts there: pieces further from the end than this many bytes
// are read past the caches in both passes, and scaled gradients are written
// past them.  MI355X, 128 MiB kept against all by way of the caches: norm of
// 8 x 25.5M fp32 125 us against 142, with the rows scaled to bf16 351 against
// 397 (some 20 of these by the writes); 16 x 25.5M bf16 131 / 442 against 148 /
// 498, and a kernel that reads the rows afterwards loses nothing (573 against
// 649 in all).  64, 96 or 192 MiB: 1 to 3% slower than 128.
constexpr int64_t kClipKept = (int64_t)128 << 20;

// A set this small goes through one block in one launch, cut into a piece for
// each of its kClipSmallWaves waves.  MI355X, one launch against two, clipping
// 65536 fp32: 6.9 us against 10.6 from the caches (both bound by the host), 12.8
// against 11.4 from memory into another tensor; 32768: 7.1 / 8.7 against 10.5 /
// 11.3; 131072: 7.3 / 21.9 against 10.4 / 11.2.
constexpr int64_t kClipSmallElems = 65536;
constexpr int kClipSmallWaves = 16;
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
    int32_t streamed;  // pieces at the front that are read past the caches
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
