// Device- and host-side helpers of the microscaled 4-bit kernels: types of real-valued tensors, containers, ragged segments.
#pragma once
#include "hq_device.h"

typedef int v2i __attribute__((ext_vector_type(2)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef int HqUnaligned16 __attribute__((ext_vector_type(4), aligned(2)));           // 16 bytes of a tensor at any element

constexpr int MX_CHUNK = HQ_MX4_CHUNK, MX_CODES = HQ_MX4_CHUNK / 2, MX_SCALES = HQ_MX4_CHUNK / HQ_MX4_BLOCK;   // values, bytes, bytes
constexpr long MX_MOST = 0x7fffffffL - MX_CHUNK;                          // rows, columns, products' sizes

inline bool hq_mx4_type_ok(int type) { return type == HQ_FP32 || type == HQ_BF16 || type == HQ_FP16; }
inline size_t hq_mx4_type_bytes(int type) { return type == HQ_FP32 ? 4 : 2; }

// `blocks` workgroups of `threads` each, in as many launches as they need: HIP takes fewer than 2^32 threads in one.  launch(first, count): those from
// number `first` on.  (Runs of a multiple of 8: a workgroup's number modulo 8 stays that of its XCD.)
template <typename Launch> inline int hq_mx4_launch(unsigned blocks, unsigned threads, const Launch &launch)
{
    const unsigned most = 0xffffffffu / threads;
    for (unsigned first = 0; first < blocks;) {
        const unsigned left = blocks - first, count = left <= most ? left : most & ~7u;
        launch(first, count);
        if (hipGetLastError() != hipSuccess) return HQ_E_HIP;
        first += count;
    }
    return HQ_OK;
}

// ---- real values -------------------------------------------------------------------------------
// Rounded to nearest even where the type is narrower than fp32 (half a step at most: bf16 2^-8, fp16 2^-11 relative).
template <int TYPE> struct HqReal;
template <> struct HqReal<HQ_FP32> {
    typedef float T;
    static __device__ inline float load(T v) { return v; }
    static __device__ inline T store(float v) { return v; }
};
template <> struct HqReal<HQ_BF16> {
    typedef unsigned short T;
    static __device__ inline float load(T v) { return __uint_as_float((unsigned)v << 16); }
    static __device__ inline T store(float v) { return __builtin_bit_cast(unsigned short, (__bf16)v); }
};
template <> struct HqReal<HQ_FP16> {
    typedef unsigned short T;
    static __device__ inline float load(T v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ inline T store(float v) { return __builtin_bit_cast(unsigned short, (_Float16)v); }
};

// ---- ragged segments ---------------------------------------------------------------------------
// Offsets are the caller's device data: clamped to 0 .. n, a descending pair is an empty segment, so that nothing is read or
// written outside the tensors whatever they hold.
struct HqSegment {
    int e;                         // segment; -1: none has this unit
    int unit;                      // unit within the segment
    int first, end;                // its rows
};

__device__ inline int hq_segment_bound(const int *offs, int e, int n) { return min(max(offs[e], 0), n); }

// The inclusive sum over the lanes below and the lane itself.
__device__ inline int hq_wave_scan(int v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int u = __shfl_up(v, d);
        v += lane >= d ? u : 0;
    }
    return v;
}

// Which segment has unit `index`, every segment being cut into units of `size` rows of its own (segment behind segment).  Called by
// whole wavefronts with the same index; 64 segments a step.
template <int SIZE> __device__ inline HqSegment hq_segment_of(const int *offs, int segments, int n, int index)
{
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < segments; base += 64) {
        const int e = base + lane;
        int lo = 0, hi = 0;
        if (e < segments) { lo = hq_segment_bound(offs, e, n); hi = max(lo, hq_segment_bound(offs, e + 1, n)); }
        const int units = (int)(((unsigned)(hi - lo) + SIZE - 1) / SIZE);
        const int upto = before + hq_wave_scan(units), mine = upto - units;
        const unsigned long long hit = __builtin_amdgcn_ballot_w64((unsigned)(index - mine) < (unsigned)units);
        if (hit) {
            const int src = __builtin_ctzll(hit);
            return HqSegment{base + src, index - __builtin_amdgcn_readlane(mine, src), __builtin_amdgcn_readlane(lo, src),
                             __builtin_amdgcn_readlane(hi, src)};
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return HqSegment{-1, 0, 0, 0};
}

// The first unit of segment e, and its rows.  Called by whole wavefronts with the same e.
template <int SIZE> __device__ inline HqSegment hq_segment_start(const int *offs, int n, int e)
{
    const int lane = threadIdx.x & 63;
    int units = 0;
    for (int k = lane; k < e; k += 64) {
        const int lo = hq_segment_bound(offs, k, n), hi = max(lo, hq_segment_bound(offs, k + 1, n));
        units += (int)(((unsigned)(hi - lo) + SIZE - 1) / SIZE);
    }
    units = __builtin_amdgcn_readlane(hq_wave_scan(units), 63);
    const int lo = hq_segment_bound(offs, e, n);
    return HqSegment{e, units, __builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(max(lo, hq_segment_bound(offs, e + 1, n)))};
}
