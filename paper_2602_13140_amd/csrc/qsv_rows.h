// Values of rows in memory, one at a time and by vectors of 16 bytes (gfx950).
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "qsv_scores.h"

namespace qsv {

template <int KIND> constexpr int kPer = KIND == kScoreF32 ? 4 : 8;      // values of a vector
template <int KIND> constexpr int kSize = KIND == kScoreF32 ? 4 : 2;

// Rows start anywhere an element may: vectors of 16 bytes at the element's alignment, which the memory pipeline takes.
typedef unsigned vec __attribute__((ext_vector_type(4)));
typedef unsigned vec_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned vec_at4 __attribute__((ext_vector_type(4), aligned(4)));

template <int KIND> __device__ __forceinline__ float value_at(const char* row, unsigned k) {
    if (KIND == kScoreF32) return ((const float*)row)[k];
    if (KIND == kScoreF16) return __half2float(((const __half*)row)[k]);
    return __uint_as_float((unsigned)((const unsigned short*)row)[k] << 16);
}

template <int KIND> __device__ __forceinline__ void store_one(char* row, unsigned k, float v) {
    if (KIND == kScoreF32) ((float*)row)[k] = v;
    else if (KIND == kScoreF16) ((__half*)row)[k] = __float2half_rn(v);
    else ((__bf16*)row)[k] = (__bf16)v;
}

template <int KIND> __device__ __forceinline__ float part(const vec& x, int i) {
    if (KIND == kScoreF32) return __uint_as_float(x[i]);
    const unsigned two = x[i >> 1];
    if (KIND == kScoreBF16) return __uint_as_float((i & 1) ? two & 0xffff0000u : two << 16);
    return __half2float(__ushort_as_half((unsigned short)((i & 1) ? two >> 16 : two)));
}

// A float64 on its way to a row, as a float32 that is rounded to the type later: to the nearest where that is float32, otherwise to one
// whose last bit tells that something was cut off, so that the second rounding is that of the value itself (the types of 16 bits
// have 13 bits less).
template <int KIND> __device__ __forceinline__ float narrowed(double v) {
    const float f = (float)v;
    if (KIND == kScoreF32) return f;
    unsigned u = __float_as_uint(f);
    if ((double)f != v && v == v) u = (u - (fabs((double)f) > fabs(v) ? 1u : 0u)) | 1u;
    return __uint_as_float(u);
}

// A vector of values, each rounded once.
template <int KIND> __device__ __forceinline__ vec packed(const float (&g)[kPer<KIND>]) {
    constexpr int W = kPer<KIND>;
    vec x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (KIND == kScoreF32) {
            x[i] = __float_as_uint(g[i]);
        } else if (KIND == kScoreBF16) {
            typedef __bf16 two __attribute__((ext_vector_type(2)));
            const two b = {(__bf16)g[(2 * i) % W], (__bf16)g[(2 * i + 1) % W]};
            x[i] = __builtin_bit_cast(unsigned, b);
        } else {
            x[i] = (unsigned)__half_as_ushort(__float2half_rn(g[(2 * i) % W])) | (unsigned)__half_as_ushort(__float2half_rn(g[(2 * i + 1) % W])) << 16;
        }
    }
    return x;
}

// PAST: past the caches.
template <int KIND, bool PAST = false> __device__ __forceinline__ vec vec_at(const char* p) {
    if (KIND == kScoreF32) return PAST ? __builtin_nontemporal_load((const vec_at4*)p) : *(const vec_at4*)p;
    return PAST ? (vec)__builtin_nontemporal_load((const vec_at2*)p) : (vec)*(const vec_at2*)p;
}

template <int KIND, bool PAST> __device__ __forceinline__ void put_vec(char* p, const vec& x) {
    if (KIND == kScoreF32) {
        if (PAST) __builtin_nontemporal_store(x, (vec_at4*)p);
        else *(vec_at4*)p = x;
    } else {
        if (PAST) __builtin_nontemporal_store(x, (vec_at2*)p);
        else *(vec_at2*)p = x;
    }
}

}  // namespace qsv
