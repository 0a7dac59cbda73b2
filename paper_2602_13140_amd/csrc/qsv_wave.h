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

template <class T> __device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

template <class T> __device__ __forceinline__ T wave_scan(T v, int lane) {      // inclusive
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T up = __shfl_up(v, o, 64);
        if (lane >= o) v += up;
    }
    return v;
}

// The same value in all lanes, as one that the compiler knows to be: in scalar registers.
__device__ __forceinline__ unsigned uniform(unsigned v) { return (unsigned)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }
__device__ __forceinline__ unsigned long long uniform(unsigned long long v) {
    return ((unsigned long long)uniform((unsigned)(v >> 32)) << 32) | uniform((unsigned)v);
}
__device__ __forceinline__ double uniform(double v) { return __longlong_as_double((long long)uniform((unsigned long long)__double_as_longlong(v))); }

}  // namespace qsv
