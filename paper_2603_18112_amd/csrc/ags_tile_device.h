// Device functions of the kernels that go through an output in tiles whose
// operands are staged through LDS: the order of the tiles, loads, waits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ags {
namespace tile {

constexpr int kXcds = 8;

// Consecutive blocks go to the 8 XCDs in turn.  Each XCD takes a run of
// consecutive tiles, and tiles are numbered in bands of BAND rows, so the
// blocks that share an XCD's L2 read few rows and few columns.
template <unsigned BAND>
__device__ __forceinline__ void tile_of_block(unsigned block, unsigned tm, unsigned tn, unsigned& i, unsigned& j) {
    const unsigned total = tm * tn, xcd = block % kXcds, at = block / kXcds;
    const unsigned base = total / kXcds, rest = total % kXcds;
    const unsigned t = xcd * base + min(xcd, rest) + at;
    const unsigned band = t / (BAND * tn), first = band * BAND, h = min(BAND, tm - first);
    const unsigned in = t - band * BAND * tn;
    i = first + in % h;
    j = in / h;
}

// Loads from memory straight into LDS: 64 lanes of 16 (or 4) bytes, lane after
// lane from LDS byte `to`.  Written out because the compiler would wait for
// all of them before the next LDS read; wait_loads() does so once a stage.
// (m0 is reserved: the compiler sets it anew where it needs it itself.)
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t r, unsigned to, unsigned lane_off, unsigned off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(lane_off),
                 "s"(r), "s"(off)
                 : "memory");
}
__device__ __forceinline__ void load_lds4(__amdgpu_buffer_rsrc_t r, unsigned to, unsigned lane_off, unsigned off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(to), "v"(lane_off),
                 "s"(r), "s"(off)
                 : "memory");
}

// Waits until at most N of this wave's loads are under way.
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void block_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace tile
}  // namespace ags
