// gfx950 kernels of gradient clipping (include/ags_clip.h).
//
// clip_norm_kernel   one block per piece: the piece's sum (or maximum) in
//                    fp64; the block that finishes last adds the partials of
//                    each group in index order and writes N_g and c_g.
// clip_scale_kernel  one block per piece: out = x c_g.  In place, blocks of a
//                    group with c_g = 1 exit at once.
// clip_small_kernel  both of them in one block, for few elements.
//
// All stream from HBM (about one flop per byte; fp64 sums cost nothing: with
// fp32 sums the norm takes as long) and use no matrix cores.  c_g is known only
// when all has been read, so a set larger than the caches is read twice.
// MI355X: norm of 138M fp32 88 us (6.3 TB/s; a kernel that only reads reaches
// 7.1), of 138M bf16 48 us; scaling passes 8 x 25.5M fp32 to bf16 some 225 us
// (5.4 TB/s read and written; a copy reaches 4.7); 25.5M bf16 into a row 32 us in
// all; 2000 to 65536 elements 7, which is the host's time for the call.
#include <math.h>

#include "ags_clip_internal.h"

namespace ags {
namespace {

constexpr int kWaves = kClipBlock / 64;

__device__ __forceinline__ float bf16_value(unsigned short b) {
    return __uint_as_float((unsigned)b << 16);
}

// Round to nearest even; a NaN keeps its sign and stays a NaN.
__device__ __forceinline__ unsigned short bf16_round(float x) {
    const unsigned u = __float_as_uint(x);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (unsigned short)((u >> 16) | 0x40u);
    return (unsigned short)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

template <int KIND>
__device__ __forceinline__ double accumulate(double acc, float x) {
    if (KIND == AGS_CLIP_L2) return fma((double)x, (double)x, acc);
    if (KIND == AGS_CLIP_L1) return acc + fabs((double)x);
    const double a = fabs((double)x);
    return a > acc || a != a ? a : acc;  // a NaN replaces and is never replaced
}

template <int KIND>
__device__ __forceinline__ double combine(double a, double b) {
    if (KIND != AGS_CLIP_MAX) return a + b;
    return b > a || b != b ? b : a;
}

template <int KIND>
__device__ __forceinline__ double wave_reduce(double v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = combine<KIND>(v, __shfl_xor(v, off, 64));
    return v;
}

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const unsigned short* p) { return bf16_value(*p); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(unsigned short* p, float x) { *p = bf16_round(x); }

// N elements of T side by side, as fp32.  An access is of at most 16 bytes a
// lane and side by side over the lanes (8 fp32 elements a lane, in two accesses
// half a line apart, read 138M elements with streaming at 5.1 TB/s; 4 do at
// 6.0).  Any alignment of the element will do.
template <typename T, int N>
struct Access {
    static_assert(N * sizeof(T) <= 16, "one access");
    typedef unsigned V __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T))));

    // STREAM: past the caches.
    template <bool STREAM>
    static __device__ __forceinline__ void load(const T* p, float* x) {
        const V* q = reinterpret_cast<const V*>(p);
        const V v = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(v[i]);
            else x[i] = __uint_as_float(i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
        }
    }
    template <bool STREAM>
    static __device__ __forceinline__ void store(T* p, const float* x) {
        V v;
#pragma unroll
        for (unsigned i = 0; i < N * sizeof(T) / 4; ++i) {
            if constexpr (sizeof(T) == 4) v[i] = __float_as_uint(x[i]);
            else v[i] = bf16_round(x[2 * i]) | ((unsigned)bf16_round(x[2 * i + 1]) << 16);
        }
        V* q = reinterpret_cast<V*>(p);
        if (STREAM) __builtin_nontemporal_store(v, q);
        else *q = v;
    }
};

__device__ __forceinline__ const void* base_of(const ClipArgs& a, int i) {
    return a.table ? a.table[i] : a.ptr[i];
}

// The sum over n elements by NT threads, this one's share.  Which elements a
// thread takes depends on n alone, not on the address, so that equal gradients
// have equal norms wherever they lie.  Against a share that starts at the first
// 16-byte boundary, 138M elements one element past it: fp32 85.7 us against 86.9,
// bf16, whose accesses then start inside a dword, 52.9 against 44.7.
template <int KIND, int NT, bool STREAM, typename T>
__device__ __forceinline__ double piece_sum(const T* p, int n, int tid) {
    constexpr int N = 16 / sizeof(T), U = 32 / N;  // an access, and those in flight
    typedef Access<T, N> A;
    double acc = 0.0, acc2 = 0.0;
    const int groups = n / N;
    int i = tid;
    for (; i + (U - 1) * NT < groups; i += U * NT) {
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) A::template load<STREAM>(p + (size_t)(i + u * NT) * N, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                acc = accumulate<KIND>(acc, x[u][j]);
                acc2 = accumulate<KIND>(acc2, x[u][j + 1]);
            }
    }
    for (; i < groups; i += NT) {
        float x[N];
        A::template load<STREAM>(p + (size_t)i * N, x);
#pragma unroll
        for (int j = 0; j < N; ++j) acc = accumulate<KIND>(acc, x[j]);
    }
    const int tail = groups * N + tid;
    if (tail < n) acc = accumulate<KIND>(acc, load1(p + tail));
    return combine<KIND>(acc, acc2);
}

template <int KIND, int NT, bool STREAM>
__device__ __forceinline__ double sum_of(const ClipArgs& a, const ClipPiece& pc, int tid) {
    const void* base = base_of(a, pc.in_base);
    return pc.in_dt == AGS_F32
               ? piece_sum<KIND, NT, STREAM>(static_cast<const float*>(base) + pc.in_off, pc.count, tid)
               : piece_sum<KIND, NT, STREAM>(static_cast<const unsigned short*>(base) + pc.in_off, pc.count, tid);
}

template <int KIND>
__device__ __forceinline__ void write_group(const ClipArgs& a, int g, double sum) {
    const double norm = KIND == AGS_CLIP_L2 ? sqrt(sum) : sum;
    a.norms[g] = (float)norm;
    const double r = a.max_norm / (norm + a.eps);
    // c_g in two factors, so that one too small for a normal fp32 value keeps
    // its 24 bits (fp32 gradients of a norm above 1e38); a NaN stays one.
    const bool tiny = r < 0x1p-100;
    a.coef[g] = r >= 1.0 ? make_float2(1.0f, 1.0f)
                         : make_float2((float)(tiny ? r * 0x1p100 : r), tiny ? 0x1p-100f : 1.0f);
}

// Counts this thread's block in and returns the count before it.  The order
// between a block's partial and the count, and between the count and what the
// last block loads, needs no fences (which write back and invalidate an XCD's
// L2) on gfx950: agent-scope stores write through, and vmcnt reaches 0 once
// they have reached the level every XCD reads them from; the loads come after
// a branch on the count, so after the atomic's reply, and go past the L2.
#if defined(__HIP_DEVICE_COMPILE__) && !defined(__gfx950__)
#error "the order that count_in relies on is argued for gfx950 only"
#endif
__device__ __forceinline__ unsigned count_in(unsigned* p) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const unsigned before = __hip_atomic_fetch_add(p, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("" ::: "memory");
    return before;
}

template <int KIND>
__global__ __launch_bounds__(kClipBlock) void clip_norm_kernel(ClipArgs a) {
    __shared__ double sh[kWaves];
    __shared__ int sh_last;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const ClipPiece pc = a.pieces[blockIdx.x];
    double v = (int)blockIdx.x < a.streamed ? sum_of<KIND, kClipBlock, true>(a, pc, tid)
                                            : sum_of<KIND, kClipBlock, false>(a, pc, tid);
    v = wave_reduce<KIND>(v);
    if (lane == 0) sh[wave] = v;
    __syncthreads();
    if (tid == 0) {
        v = sh[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v = combine<KIND>(v, sh[w]);
        __hip_atomic_store(&a.partials[blockIdx.x], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const unsigned n = (unsigned)a.n_pieces, c = blockIdx.x % kClipCounters;
        const unsigned mine = (n - c + kClipCounters - 1) / kClipCounters;  // blocks on this counter
        sh_last = count_in(a.done + (c + 1) * kClipCounterStride) + 1 == mine &&
                  count_in(a.done) + 1 == min(n, (unsigned)kClipCounters);
    }
    __syncthreads();
    if (!sh_last) return;
    // The last block.  Few groups take the whole block one after the other; of
    // more, those of few pieces take a lane each, those of some more 16 lanes and
    // the others a wave.  MI355X, norms of 1000 groups of three pieces 191 us with
    // a wave for each and 20 so, 64 groups of 49 pieces 31.7 and 24.7; one group
    // of 4000 pieces 25.6 with the block against 36.2 with a wave.
    auto load = [&](int i) { return __hip_atomic_load(&a.partials[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    if (a.n_groups < kWaves) {
        for (int g = 0; g < a.n_groups; ++g) {
            double s = 0.0;
            for (int i = a.group_begin[g] + tid; i < a.group_begin[g + 1]; i += kClipBlock) s = combine<KIND>(s, load(i));
            s = wave_reduce<KIND>(s);
            __syncthreads();
            if (lane == 0) sh[wave] = s;
            __syncthreads();
            if (tid == 0) {
                for (int w = 1; w < kWaves; ++w) s = combine<KIND>(s, sh[w]);
                write_group<KIND>(a, g, s);
            }
        }
    } else {
        // Lane l of wave w looks after group base + l kWaves + w.
        for (int base = wave; base < a.n_groups; base += 64 * kWaves) {
            const int g = base + lane * kWaves;
            const int b = g < a.n_groups ? a.group_begin[g] : 0, e = g < a.n_groups ? a.group_begin[g + 1] : 0;
            if (g < a.n_groups && e - b <= 8) {
                double s = 0.0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (b + i < e) s = combine<KIND>(s, load(b + i));
                write_group<KIND>(a, g, s);
            }
            for (int wide = 0; wide < 2; ++wide) {
                const int width = wide ? 64 : 16;
                uint64_t todo = __ballot(wide ? e - b > 256 : e - b > 8 && e - b <= 256);
                while (todo) {
                    int mine = -1;  // the lane whose group this lane works on
                    for (int k = 0; k < 64 / width && todo; ++k) {
                        if (lane / width == k) mine = __ffsll((unsigned long long)todo) - 1;
                        todo &= todo - 1;
                    }
                    const int from = __shfl(b, mine < 0 ? 0 : mine, 64), to = __shfl(e, mine < 0 ? 0 : mine, 64);
                    double s = 0.0;
                    if (mine >= 0)
                        for (int i = from + lane % width; i < to; i += width) s = combine<KIND>(s, load(i));
                    for (int off = width / 2; off >= 1; off >>= 1) s = combine<KIND>(s, __shfl_xor(s, off, 64));
                    if (mine >= 0 && lane % width == 0) write_group<KIND>(a, base + mine * kWaves, s);
                }
            }
        }
    }
    if (tid <= kClipCounters) a.done[tid * kClipCounterStride] = 0u;
}

// Elements before p's next 16-byte boundary, at most n.
template <typename T>
__device__ __forceinline__ int head_elems(const T* p, int n) {
    const int h = (int)((16u - ((unsigned)reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / (int)sizeof(T);
    return min(h, n);
}

// The product is rounded to fp32 before it is rounded to bf16: the formula in
// fp32 arithmetic, off by 2^-24 more than one rounding at most.
// IN, OUT: past the caches.
template <int NT, bool IN, bool OUT, typename TI, typename TO>
__device__ __forceinline__ void piece_scale(const TI* in, TO* out, int n, float2 c, int tid) {
    constexpr int N = sizeof(TI) + sizeof(TO) == 4 ? 8 : 4, U = 32 / N;
    const int head = head_elems(in, n);
    if (tid < head) store1(out + tid, load1(in + tid) * c.x * c.y);
    in += head;
    out += head;
    n -= head;
    const int groups = n / N;
    int i = tid;
    for (; i + (U - 1) * NT < groups; i += U * NT) {
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) Access<TI, N>::template load<IN>(in + (size_t)(i + u * NT) * N, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int j = 0; j < N; ++j) x[u][j] = x[u][j] * c.x * c.y;
            Access<TO, N>::template store<OUT>(out + (size_t)(i + u * NT) * N, x[u]);
        }
    }
    for (; i < groups; i += NT) {
        float x[N];
        Access<TI, N>::template load<IN>(in + (size_t)i * N, x);
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = x[j] * c.x * c.y;
        Access<TO, N>::template store<OUT>(out + (size_t)i * N, x);
    }
    const int tail = groups * N + tid;
    if (tail < n) store1(out + tail, load1(in + tail) * c.x * c.y);
}

template <int NT, bool IN, bool OUT>
__device__ __forceinline__ void scale_piece(const ClipArgs& a, const ClipPiece& pc, float2 c, int tid) {
    if (a.in_place && c.x == 1.0f && c.y == 1.0f) return;
    const void* in = base_of(a, pc.in_base);
    void* out = const_cast<void*>(a.in_place ? in : base_of(a, a.n_in + pc.out_base));
    const int64_t oo = a.in_place ? pc.in_off : pc.out_off;
    const int odt = a.in_place ? pc.in_dt : pc.out_dt;
    if (pc.in_dt == AGS_F32) {
        const float* p = static_cast<const float*>(in) + pc.in_off;
        if (odt == AGS_F32) piece_scale<NT, IN, OUT>(p, static_cast<float*>(out) + oo, pc.count, c, tid);
        else piece_scale<NT, IN, OUT>(p, static_cast<unsigned short*>(out) + oo, pc.count, c, tid);
    } else {
        const unsigned short* p = static_cast<const unsigned short*>(in) + pc.in_off;
        if (odt == AGS_F32) piece_scale<NT, IN, OUT>(p, static_cast<float*>(out) + oo, pc.count, c, tid);
        else piece_scale<NT, IN, OUT>(p, static_cast<unsigned short*>(out) + oo, pc.count, c, tid);
    }
}

__global__ __launch_bounds__(kClipBlock) void clip_scale_kernel(ClipArgs a) {
    // Backwards: the norm's pass left its last pieces in the caches.
    const int i = a.n_pieces - 1 - (int)blockIdx.x;
    const ClipPiece pc = a.pieces[i];
    const float2 c = a.coef[pc.group];
    if (i < a.streamed) scale_piece<kClipBlock, true, true>(a, pc, c, threadIdx.x);
    else scale_piece<kClipBlock, false, true>(a, pc, c, threadIdx.x);
}

// Both passes over a small set in one block, a wave to a piece.
template <int KIND>
__global__ __launch_bounds__(kClipSmallWaves * 64) void clip_small_kernel(ClipArgs a, int scale) {
    __shared__ double sums[kClipSmallPieces];
    constexpr int kW = kClipSmallWaves;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int i = wave; i < a.n_pieces; i += kW) {
        const double v = wave_reduce<KIND>(sum_of<KIND, 64, false>(a, a.pieces[i], lane));
        if (lane == 0) sums[i] = v;
    }
    __syncthreads();
    for (int g = wave; g < a.n_groups; g += kW) {
        double s = 0.0;
        for (int i = a.group_begin[g] + lane; i < a.group_begin[g + 1]; i += 64) s = combine<KIND>(s, sums[i]);
        s = wave_reduce<KIND>(s);
        if (lane == 0) write_group<KIND>(a, g, s);
    }
    if (!scale) return;
    __syncthreads();
    for (int i = wave; i < a.n_pieces; i += kW) {
        const ClipPiece pc = a.pieces[i];
        scale_piece<64, false, false>(a, pc, a.coef[pc.group], lane);
    }
}

__global__ void clip_table_kernel(ClipTableArgs a) {
    for (int i = threadIdx.x; i < a.count; i += blockDim.x) a.table[a.first + i] = a.ptr[i];
}

}  // namespace

hipError_t launch_clip_table(const ClipTableArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(clip_table_kernel, dim3(1), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_clip_norm(const ClipArgs& a, int kind, hipStream_t s) {
    const dim3 grid(a.n_pieces), block(kClipBlock);
    switch (kind) {
        case AGS_CLIP_L2: hipLaunchKernelGGL(clip_norm_kernel<AGS_CLIP_L2>, grid, block, 0, s, a); break;
        case AGS_CLIP_L1: hipLaunchKernelGGL(clip_norm_kernel<AGS_CLIP_L1>, grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL(clip_norm_kernel<AGS_CLIP_MAX>, grid, block, 0, s, a); break;
    }
    return hipGetLastError();
}

hipError_t launch_clip_small(const ClipArgs& a, int kind, bool scale, hipStream_t s) {
    const dim3 grid(1), block(kClipSmallWaves * 64);
    const int sc = scale ? 1 : 0;
    switch (kind) {
        case AGS_CLIP_L2: hipLaunchKernelGGL(clip_small_kernel<AGS_CLIP_L2>, grid, block, 0, s, a, sc); break;
        case AGS_CLIP_L1: hipLaunchKernelGGL(clip_small_kernel<AGS_CLIP_L1>, grid, block, 0, s, a, sc); break;
        default: hipLaunchKernelGGL(clip_small_kernel<AGS_CLIP_MAX>, grid, block, 0, s, a, sc); break;
    }
    return hipGetLastError();
}

hipError_t launch_clip_scale(const ClipArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(clip_scale_kernel, dim3(a.n_pieces), dim3(kClipBlock), 0, s, a);
    return hipGetLastError();
}

}  // namespace ags
