// Wavefront and workgroup helpers of the kernels on rows (gfx950: 64 lanes).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace qsv {

// Workgroups are numbered over two grid dimensions (one holds less than 2^32 threads); the last ones may have no work.
constexpr unsigned long long kGridX = 1 << 20;
__device__ __forceinline__ unsigned long long grid_block() { return (unsigned long long)blockIdx.y * kGridX + blockIdx.x; }
inline dim3 grid_of(unsigned long long blocks) {
    return dim3((unsigned)std::min(blocks, kGridX), (unsigned)((blocks + kGridX - 1) / kGridX));
}

// A lane's value from the one that the data-parallel primitives name, 0 where there is none.
template <int CTRL, int ROWS> __device__ __forceinline__ unsigned moved(unsigned v) {
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS> __device__ __forceinline__ unsigned long long moved(unsigned long long v) {
    return ((unsigned long long)moved<CTRL, ROWS>((unsigned)(v >> 32)) << 32) | moved<CTRL, ROWS>((unsigned)v);
}
template <int CTRL, int ROWS> __device__ __forceinline__ double moved(double v) {
    return __longlong_as_double((long long)moved<CTRL, ROWS>((unsigned long long)__double_as_longlong(v)));
}

// Sums of the lanes up to and with each one: within rows of 16 lanes, then the rows' sums into those behind them.
template <class T> __device__ __forceinline__ T wave_scan(T v) {
    v += moved<0x111, 0xf>(v);      // one lane up, then two, four, eight
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);      // lane 15 of a row to the next, rows 1 and 3
    v += moved<0x143, 0xc>(v);      // lane 31 to rows 2 and 3
    return v;
}

// The same value in all lanes, as one that the compiler knows to be: in scalar registers.
__device__ __forceinline__ unsigned uniform(unsigned v) { return (unsigned)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }
__device__ __forceinline__ unsigned long long uniform(unsigned long long v) {
    return ((unsigned long long)uniform((unsigned)(v >> 32)) << 32) | uniform((unsigned)v);
}
__device__ __forceinline__ double uniform(double v) { return __longlong_as_double((long long)uniform((unsigned long long)__double_as_longlong(v))); }

// Pointers whose memory is known: through a struct or a lambda the compiler loses it, and a flat access waits for both kinds.
template <class T> using in_global = const __attribute__((address_space(1))) T;
template <class T> using in_lds = const __attribute__((address_space(3))) T;

template <class T> __device__ __forceinline__ T lds_add(T* p, T v) {
    return __hip_atomic_fetch_add((__attribute__((address_space(3))) T*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

template <class T> __device__ __forceinline__ T last_lane(T v);
template <> __device__ __forceinline__ unsigned last_lane(unsigned v) { return (unsigned)__builtin_amdgcn_readlane((int)v, 63); }
template <> __device__ __forceinline__ unsigned long long last_lane(unsigned long long v) {
    return ((unsigned long long)last_lane((unsigned)(v >> 32)) << 32) | last_lane((unsigned)v);
}
template <> __device__ __forceinline__ double last_lane(double v) {
    return __longlong_as_double((long long)last_lane((unsigned long long)__double_as_longlong(v)));
}
template <class T> __device__ __forceinline__ T wave_sum(T v) { return last_lane(wave_scan(v)); }

__device__ __forceinline__ unsigned lane_of(unsigned v, unsigned lane) { return (unsigned)__builtin_amdgcn_readlane((int)v, (int)lane); }
__device__ __forceinline__ unsigned long long lane_of(unsigned long long v, unsigned lane) {
    return ((unsigned long long)lane_of((unsigned)(v >> 32), lane) << 32) | lane_of((unsigned)v, lane);
}

}  // namespace qsv
