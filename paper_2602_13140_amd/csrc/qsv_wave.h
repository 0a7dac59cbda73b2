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

}  // namespace qsv
