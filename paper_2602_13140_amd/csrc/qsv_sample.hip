// Outcomes drawn from rows of scores, probabilities or amplitudes after temperature, min-p, top-k and top-p.
//
// All filters cut one order: value descending, ties by the lowest index first.  So what is left of a row is known by a
// cut (value, index): everything above the value, and what equals it up to that index.  No row is sorted:
//   top-k   Every thread knows the highest of its own values.  The k-th of those is a bound that k outcomes reach and few
//           more; they go into a list, and the list is sorted in LDS (32768 scores, k = 50: some 55 entries).
//   top-p   Needs the weight of the whole row: one scan adds every weight to a histogram over its distance from the
//           highest value; what lies above the bin that the cut falls into is kept, what lies in it is sorted.
//   else    (k large, a bin of nearly equal values, a row in parts) histograms over the bits of the values in the bin, 11
//           at a time, until the bin is one value.
// The draw finds the 1024 values that the running sum passes the shot in by sums over such chunks, and then the value.
//
// Weights are whole numbers, rint(e 2^S) with e in 64 bits: their sums are the same in any order, so a call's results do
// not depend on how its work was split or in which order atomics arrived.
//
// A row of up to 262144 outcomes is one workgroup's, which reads it two or three times: bound by memory for top-k (256 x
// 131072 f32, k = 50: 52 us, two scans of 134 MB at 5.2 TB/s), by vector issue for top-p (105 us; a weight
// takes 19 instructions, and the slowest of 256 rows has half of its outcomes left).  Few rows are bound by latency (1 x
// 32768 bf16: 11 us).  64-bit atomics, weights and the search of a cut in 64 bits cost nothing here that 32 bits would
// save: double precision issues at the rate of single.
#include "qsv_scores.h"
#include "qsv_wave.h"

#include <hip/hip_fp16.h>

namespace qsv {
namespace {

typedef unsigned long long u64;
typedef unsigned u32;

constexpr float kInf = __builtin_inff();
constexpr u32 kAll = 0xffffffffu;      // of a cut: every outcome that equals its key

template <int KIND> constexpr bool kLogs = KIND <= kScoreBF16;          // scores; else probabilities
template <int KIND> constexpr bool kKeys16 = KIND == kScoreF16 || KIND == kScoreBF16;
// the lowest key an outcome can have; masked ones have lower ones
template <int KIND> constexpr u32 kLowest = KIND == kScoreF32 ? 0x00800000u : KIND == kScoreBF16 ? 0x0080u : KIND == kScoreF16 ? 0x0400u : 1u;

template <int KIND> constexpr float kMasked = kLogs<KIND> ? -kInf : 0.f;

// Values are compared as they are: a masked one (NaN, -inf; of probabilities all that are not positive) is never as high as a
// value that a row's filters name, and -0 equals 0.  Their keys: of masked values below the lowest, of -0 that of 0.
template <int KIND> __device__ __forceinline__ u32 key_of(float v) {
    v = kLogs<KIND> ? (v > -kInf ? v + 0.f : -kInf) : (v > 0.f ? v : 0.f);
    if (!kLogs<KIND>) return __float_as_uint(v);
    if (KIND == kScoreF16) {
        const u32 b = __half_as_ushort(__float2half_rn(v));
        return (b & 0x8000u) ? b ^ 0xffffu : b | 0x8000u;
    }
    const u32 b = __float_as_uint(v);
    const u32 k = b ^ ((u32)((int)b >> 31) | 0x80000000u);
    return KIND == kScoreBF16 ? k >> 16 : k;
}

template <int KIND> __device__ __forceinline__ float value_of(u32 k) {
    if (!kLogs<KIND>) return __uint_as_float(k);
    if (KIND == kScoreF16) {
        const u32 b = (k & 0x8000u) ? k ^ 0x8000u : k ^ 0xffffu;
        return __half2float(__ushort_as_half((unsigned short)b));
    }
    const u32 f = KIND == kScoreBF16 ? k << 16 : k;
    if (f & 0x80000000u) return __uint_as_float(f ^ 0x80000000u);
    return __uint_as_float(KIND == kScoreBF16 ? (f ^ 0xffff0000u) : ~f);
}

// The lowest key of a value that is not below x.  (16 bits: x itself may lie between two, and its key then be the lower one's.)
template <int KIND> __device__ __forceinline__ u32 key_from(float x) {
    const u32 k = key_of<KIND>(x);
    return kKeys16<KIND> && value_of<KIND>(k) < x ? k + 1u : k;
}

// ---- rows ------------------------------------------------------------------------------------------------------------
// A row is read four values a lane in aligned vectors: vector j holds the values 4 j - skew .. 4 j - skew + 3, where skew
// values lie between the last aligned address and the row's start.  Vectors that reach over an end are read value by value.
struct Row {
    in_global<char>* base;     // where vector 0 would start
    u32 cols, skew, vecs;
    u32 first, whole;          // the first whole vector, and how many there are
};

template <int KIND> __device__ __forceinline__ Row row_of(const SampleArgs& a, u64 r) {
    constexpr int size = KIND == kScoreState ? 8 : kKeys16<KIND> ? 2 : 4;
    Row w;
    const char* p = (const char*)a.scores + r * (u64)a.stride * size;
    w.cols = a.cols;
    w.skew = KIND == kScoreState ? 0u : (u32)(((uintptr_t)p / size) & 3u);
    w.base = (in_global<char>*)(p - w.skew * size);
    w.vecs = (w.cols + w.skew + 3u) >> 2;
    w.first = w.skew ? 1u : 0u;
    w.whole = (w.cols + w.skew) / 4u > w.first ? (w.cols + w.skew) / 4u - w.first : 0u;
    return w;
}

// Value number k behind the row's vector 0.
template <int KIND> __device__ __forceinline__ float one_value(const Row& w, u32 k) {
    if constexpr (KIND == kScoreState) {
        in_global<float>* z = (in_global<float>*)w.base + 2ull * k;
        return __builtin_fmaf(z[1], z[1], z[0] * z[0]);     // the probability as every measurement has it
    } else if constexpr (kKeys16<KIND>) {
        const unsigned short b = ((in_global<unsigned short>*)w.base)[k];
        return KIND == kScoreF16 ? __half2float(__ushort_as_half(b)) : __uint_as_float((u32)b << 16);
    } else {
        return ((in_global<float>*)w.base)[k];
    }
}

// Vector j, which lies in the row whole.
template <int KIND> __device__ __forceinline__ void load_whole(const Row& w, u32 j, float (&v)[4]) {
    typedef float f4 __attribute__((ext_vector_type(4)));
    typedef u32 u2 __attribute__((ext_vector_type(2)));
    if constexpr (KIND == kScoreState) {
        in_global<f4>* q = (in_global<f4>*)w.base + 2ull * j;
        const f4 x = q[0], y = q[1];
        v[0] = __builtin_fmaf(x[1], x[1], x[0] * x[0]);
        v[1] = __builtin_fmaf(x[3], x[3], x[2] * x[2]);
        v[2] = __builtin_fmaf(y[1], y[1], y[0] * y[0]);
        v[3] = __builtin_fmaf(y[3], y[3], y[2] * y[2]);
    } else if constexpr (kKeys16<KIND>) {
        const u2 x = ((in_global<u2>*)w.base)[j];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32 two = x[i >> 1];
            if (KIND == kScoreBF16) v[i] = __uint_as_float((i & 1) ? two & 0xffff0000u : two << 16);
            else v[i] = __half2float(__ushort_as_half((unsigned short)((i & 1) ? two >> 16 : two)));
        }
    } else {
        const f4 x = ((in_global<f4>*)w.base)[j];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = x[i];
    }
}

// Any vector: masked values where it reaches over the row's ends.
template <int KIND> __device__ __forceinline__ void load4(const Row& w, u32 j, float (&v)[4]) {
    if (j - w.first < w.whole) return load_whole<KIND>(w, j, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = kMasked<KIND>;
    if (j >= w.vecs) return;
#pragma unroll
    for (u32 i = 0; i < 4; ++i)
        if (4 * j + i >= w.skew && 4 * j + i - w.skew < w.cols) v[i] = one_value<KIND>(w, 4 * j + i);
}

// f(values, j) for every vector from j0 to j1 (or the row's end), a thread each, UN of a thread on their way at once.
template <int KIND, int NT, int UN, class F> __device__ __forceinline__ void walk(const Row& w, u32 j0, u32 j1, F f) {
    if (j0 == 0 && w.first) {
        if (threadIdx.x == 0) {
            float v[4];
            load4<KIND>(w, 0, v);
            f(v, 0u);
        }
        j0 = 1;
    }
    const u32 end = min(j1, w.first + w.whole);
    for (; j0 + NT * UN <= end; j0 += NT * UN) {
        float v[UN][4];
#pragma unroll
        for (int u = 0; u < UN; ++u) load_whole<KIND>(w, j0 + u * NT + threadIdx.x, v[u]);
#pragma unroll
        for (int u = 0; u < UN; ++u) f(v[u], j0 + u * NT + threadIdx.x);
    }
    for (u32 j = j0 + threadIdx.x; j < min(j1, w.vecs); j += NT) {
        float v[4];
        load4<KIND>(w, j, v);
        f(v, j);
    }
}

// The vectors j0 + lane, j0 + 64 + lane, ... of a wavefront's chunk.
template <int KIND, int STEPS> __device__ __forceinline__ void load_chunk(const Row& w, u32 j0, u32 lane, float (&v)[STEPS][4]) {
    if (j0 >= w.first && j0 + 64 * STEPS <= w.first + w.whole) {
#pragma unroll
        for (int it = 0; it < STEPS; ++it) load_whole<KIND>(w, j0 + it * 64u + lane, v[it]);
    } else {
#pragma unroll
        for (int it = 0; it < STEPS; ++it) load4<KIND>(w, j0 + it * 64u + lane, v[it]);
    }
}

// ---- weights ---------------------------------------------------------------------------------------------------------
// 2^x for x <= 0, relative error below 2^-51; below 2^-200 that (nothing differs there: weights end at 2^-52).
__device__ __forceinline__ double exp2_neg(double x) {
    x = fmax(x, -200.0);
    const double n = __builtin_rint(x);
    const double f = (x - n) * 0.69314718055994530942;     // |f| <= 0.347: the series to f^13 / 13!
    double s = 1.0 / 6227020800.0;
    s = fma(s, f, 1.0 / 479001600.0);
    s = fma(s, f, 1.0 / 39916800.0);
    s = fma(s, f, 1.0 / 3628800.0);
    s = fma(s, f, 1.0 / 362880.0);
    s = fma(s, f, 1.0 / 40320.0);
    s = fma(s, f, 1.0 / 5040.0);
    s = fma(s, f, 1.0 / 720.0);
    s = fma(s, f, 1.0 / 120.0);
    s = fma(s, f, 1.0 / 24.0);
    s = fma(s, f, 1.0 / 6.0);
    s = fma(s, f, 0.5);
    s = fma(s, f, 1.0);
    s = fma(s, f, 1.0);
    return __builtin_ldexp(s, (int)n);
}

// How a row's values become weights.
struct Scale {
    float m;           // the highest value
    float top;         // m, or the highest finite float
    double md;
    double mq, rm;     // for quotients: m and 1 / m, or 1 and 0 where m is infinite
    double log_m;      // probabilities: log2 m
    double c0, c;      // scores: log2(e) / T; probabilities: 1 / T; and that NP times
    double one;        // 2^S
    float per_bin;     // scores: bins for a distance of 1 below m
    float low_w;       // the lowest value whose weight may differ from 0
    bool t_one;
    u32 kmax;
};

// The lowest float that is not below x.
__device__ __forceinline__ float float_from(double x) {
    const float f = (float)x;
    if ((double)f >= x) return f;
    return f < 0.f ? __uint_as_float(__float_as_uint(f) - 1u) : __uint_as_float(__float_as_uint(f) + 1u);
}

template <int KIND> __device__ __forceinline__ double weight64(const Scale& s, float v) {
    if (v == s.m) return 1.0;
    if (!(s.m < kInf)) return 0.0;
    if (kLogs<KIND>) return exp2_neg(((double)v - s.md) * s.c0);
    const double q = (double)v / s.md;
    return s.t_one ? q : exp2_neg(log2(q) * s.c0);
}

// log2 of a positive float in 64 bits, for probabilities at another temperature than 1: v = 2^k f, f in 1..2, its upper 8 bits
// name a factor c near 1 / f; log2 v = k - log2 c + log2(1 + r), r = f c - 1, |r| < 2^-8: the series to r^7.  16 instructions;
// the library's log2 takes some sixty.
struct Logs { double c[256], log2_c[256]; };
template <int NT> __device__ __forceinline__ void fill_logs(Logs* l) {
    for (int i = threadIdx.x; i < 256; i += NT) {
        const double c = (double)(float)(512.0 / (513.0 + 2 * i));     // (24 bits: f c - 1 is exact)
        l->c[i] = c;
        l->log2_c[i] = log2(c);
    }
}
__device__ __forceinline__ double log2_of(const Logs* l, float v) {
    const u64 b = (u64)__double_as_longlong((double)v);
    const int k = (int)(b >> 52) - 1023, i = (int)(b >> 44) & 255;
    const double f = __longlong_as_double((long long)((b & 0xfffffffffffffull) | 0x3ff0000000000000ull));
    const double r = fma(f, ((in_lds<double>*)l->c)[i], -1.0);
    double s = 1.0 / 7.0;
    s = fma(s, -r, 1.0 / 6.0);
    s = fma(s, -r, 1.0 / 5.0);
    s = fma(s, -r, 1.0 / 4.0);
    s = fma(s, -r, 1.0 / 3.0);
    s = fma(s, -r, 1.0 / 2.0);
    s = fma(s, -r, 1.0);
    return ((double)k - ((in_lds<double>*)l->log2_c)[i]) + s * r * 1.4426950408889634074;
}

// What weights are looked up in: a kernel's tables in LDS.
// 2^(S - 63) 2^(i / NP): 1024 of them save a term of the series, 256 are filled sooner.
template <int KIND, int NP> struct Tables { double powers[NP]; };
template <int NP> struct Tables<kScoreProbs, NP> { double powers[NP]; Logs logs; };
template <int NP> struct Tables<kScoreState, NP> { double powers[NP]; Logs logs; };
template <int NT> constexpr int kPowers = NT > 256 ? 1024 : 256;

template <int KIND, int NB, int NP> __device__ __forceinline__ Scale scale_of(const Tables<KIND, NP>* tables, u32 kmax, float t, int bits) {
    Scale s;
    s.kmax = kmax;
    s.m = value_of<KIND>(kmax);
    s.top = fminf(s.m, 3.402823466e38f);
    s.md = (double)s.top;
    s.mq = s.m < kInf ? s.md : 1.0;
    s.rm = s.m < kInf ? 1.0 / s.md : 0.0;
    s.c0 = (kLogs<KIND> ? 1.4426950408889634074 : 1.0) / (double)t;
    s.c = s.c0 * NP;
    s.log_m = 0.0;
    if constexpr (!kLogs<KIND>) s.log_m = log2_of(&tables->logs, s.top);
    s.one = __builtin_ldexp(1.0, bits);
    s.t_one = t == 1.f;
    s.per_bin = (float)s.c0 * ((float)NB / (float)(bits + 2));
    // weights end below 2^-(S + 2)
    if (!(s.m < kInf)) s.low_w = s.m;
    else if (kLogs<KIND>) s.low_w = float_from(s.md - (double)(bits + 2) * (0.69314718055994530942 * (double)t));
    else s.low_w = fmaxf(float_from(s.md * exp2(-(double)(bits + 2) * (double)t)), __uint_as_float(1u));
    return s;
}

// rint(e 2^S), the whole number that adding 2^52 leaves in the low bits.  2^x as a power from the table, its exponent raised by
// whole steps, times a series of three terms (NP = 256: four; the next is below 2^-50): half the arithmetic of exp2_neg.
// For values from s.low_w on; lower ones weigh nothing.  step: NP times the distance from m, in factors of two, below 63 NP.
// (Of its instructions those that the compiler would spend moves or a 64-bit addition on are named.)
template <int NP> constexpr u32 kTopStep = 63 * NP;
__device__ __forceinline__ double fma3(double a, double b, double c) {
    double d;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}
__device__ __forceinline__ u64 whole(double x) { return (u64)__double_as_longlong(x) & 0xfffffffffffffull; }
template <int KIND, int NP> __device__ __forceinline__ u64 weight_of(const Scale& s, const Tables<KIND, NP>* tables, float v, u32* step) {
    if (!kLogs<KIND> && s.t_one) {
        const double q = (double)v * s.rm;
        const double e = fma(fma(-q, s.mq, (double)v), s.rm, q);      // v / m
        *step = kTopStep<NP> - ((s.kmax - __float_as_uint(v)) >> 18) * (NP / 32);
        return whole(fma(v == s.m ? 1.0 : e, s.one, 4503599627370496.0));
    }
    double x;
    if constexpr (kLogs<KIND>) x = ((double)fminf(v, s.top) - s.md) * s.c;
    else x = (log2_of(&tables->logs, fminf(v, s.top)) - s.log_m) * s.c;
    constexpr double magic = 6755399441055744.0 + kTopStep<NP>;       // 1.5 2^52: the nearest whole number in the low bits
    const double y = x + magic;
    const u32 n = (u32)__double_as_longlong(y);
    *step = n;
    const double r = x - (y - magic);
    constexpr double l = 0.69314718055994530942 / NP;
    double p = NP > 256 ? l * l * l / 6.0 : fma3(l * l * l * l / 24.0, r, l * l * l / 6.0);
    p = fma3(p, r, l * l / 2.0);
    p = fma3(p, r, l);
    p = fma(p, r, 1.0);
    constexpr int bits = NP > 256 ? 10 : 8;
    const u64 t = (u64)__double_as_longlong(((in_lds<double>*)tables->powers)[n & (NP - 1)]);
    u32 high;
    asm("v_lshl_add_u32 %0, %1, %2, %3" : "=v"(high) : "v"(n & ~(u32)(NP - 1)), "n"(20 - bits), "v"((u32)(t >> 32)));
    return whole(fma(__longlong_as_double((long long)((u64)high << 32 | (u32)t)), p, 4503599627370496.0));
}

template <int KIND, int NP> __device__ __forceinline__ u64 weight(const Scale& s, const Tables<KIND, NP>* tables, float v) {
    u32 steps;
    const u64 w = weight_of<KIND, NP>(s, tables, v, &steps);
    return v >= s.low_w ? w : 0;
}

// Filled by a kernel's threads before their next barrier; not at all where a row will not look anything up.
template <int KIND, int NT, int NP> __device__ __forceinline__ void fill_tables(Tables<KIND, NP>* tables, int bits, bool t_one) {
    if (!kLogs<KIND> && t_one) return;
    const double two = __builtin_ldexp(2.0, bits - 63);        // (steps start at 63 factors of two)
    for (int i = threadIdx.x; i < NP; i += NT) tables->powers[i] = two * exp2_neg((double)i / NP - 1.0);
    if constexpr (!kLogs<KIND>) fill_logs<NT>(&tables->logs);
}

// Bin of the first histogram: not decreasing in the distance from the highest value.  Scores: linear in it over the S + 2
// factors of two in which weights are not 0; probabilities: 32 bins a factor of two.
template <int KIND, int NB> __device__ __forceinline__ u32 bin_of(const Scale& s, float v) {
    if (kLogs<KIND>) return v == s.m ? 0u : (u32)fminf((s.m - v) * s.per_bin, (float)(NB - 1));
    constexpr int shift = NB >= 2048 ? 18 : NB >= 1024 ? 19 : 21;
    return min((s.kmax - __float_as_uint(v)) >> shift, (u32)(NB - 1));
}

// ---- wavefronts and workgroups ---------------------------------------------------------------------------------------
// Sums over the workgroup before each thread's own, and the whole sum.  sm: NT / 64 entries that nothing else uses.
template <int NT> __device__ __forceinline__ u64 block_scan(u64 v, u64* sm, u64* total) {
    constexpr int NW = NT / 64;
    const u32 lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const u64 incl = wave_scan(v);
    if (NW == 1) {
        *total = last_lane(incl);
        return incl - v;
    }
    __syncthreads();
    if (lane == 63) sm[wave] = incl;
    __syncthreads();
    const u64 waves = wave_scan(lane < NW ? sm[lane & (NW - 1)] : 0ull);
    *total = last_lane(waves);
    return (wave ? lane_of(waves, wave - 1) : 0) + incl - v;
}

template <int NT> __device__ __forceinline__ u32 block_max(u32 v, u64* sm) {
    constexpr int NW = NT / 64;
    const u32 lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, (u32)__shfl_xor((int)v, o, 64));
    if (NW == 1) return uniform(v);
    __syncthreads();
    if (lane == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (u32)sm[lane & (NW - 1)];
#pragma unroll
    for (int o = NW / 2; o > 0; o >>= 1) v = max(v, (u32)__shfl_xor((int)v, o, 64));
    return uniform(v);
}

// The lowest key of lo .. hi for which `is` holds; it holds for hi and, with a key, for all above.  64 probes at a time.
template <class F> __device__ __forceinline__ u32 first_key(u32 lo, u32 hi, F is) {
    const u32 lane = threadIdx.x & 63;
    while (lo < hi) {
        const u32 step = (hi - lo + 63u) >> 6;
        const u32 probe = min(lo + lane * step, hi);
        const u64 hit = __ballot(is(probe));
        if (hit == 0) { lo += 63u * step + 1u; continue; }     // (lane 63's probe lies below hi then)
        const u32 f = (u32)__ffsll((long long)hit) - 1u;
        const u32 top = min(lo + f * step, hi);
        if (f > 0) lo = lo + (f - 1u) * step + 1u;
        hi = top;
    }
    return hi;
}

// ---- the search for a cut --------------------------------------------------------------------------------------------
struct Cut { float v; u32 idx; };     // kept: values above, and of what equals v the indices up to idx

struct Find {
    u32 klo, khi;        // the keys the cut is among
    u32 done;            // the cut is known: (klo, ne)
    u32 ne;
    u64 target;          // outcomes, or (top-p) weights
    u64 count, weight;   // of what lies above khi
};

// ceil(P W / 2^31), the weights that top-p keeps of W; at least 1, which the first outcome alone exceeds.
__device__ __forceinline__ u64 mass_of(float top_p, u64 w) {
    const u64 part = (u64)__builtin_rint((double)top_p * 2147483648.0);
    const u64 low = part * (w & 0x7fffffffull);
    const u64 h = part * (w >> 31) + (low >> 31) + ((low & 0x7fffffffull) != 0);
    return h > 0 ? h : 1;
}

// The bin in which the running sum (of counts, or of weights) over cnt / wt reaches target, and what lies before it.  false: it
// never does.  total: target holds top_p's bits, which the whole weight turns into the target.  Ends with a barrier.
struct Hit { u32 bin; u64 count, weight, own; };        // own: outcomes in the bin
// MIRROR: weights in bins that rise with the value; the bin's number counts from the last one.
template <int NT, int NB, bool BYW, bool MIRROR = false> __device__ __forceinline__ bool select_bin(const u32* cnt, const u64* weights, u64 target, u64* sm, Hit* hit, Hit* at, u64* total = nullptr) {
    constexpr int per = NB / NT > 0 ? NB / NT : 1;
    const int b0 = threadIdx.x * per;
    struct { const u64* p; __device__ u64 operator[](int b) const { return p[MIRROR ? NB - 1 - b : b]; } __device__ operator bool() const { return p; } } const wt{weights};
    u64 c = 0, w = 0;
    if (b0 < NB) {
#pragma unroll
        for (int i = 0; i < per; ++i) { if (cnt) c += cnt[b0 + i]; if (wt) w += wt[b0 + i]; }
    }
    u64 ct = 0, wtot = 0, cb = 0, wb = 0;
    if (cnt) cb = block_scan<NT>(c, sm, &ct);
    if (wt) wb = block_scan<NT>(w, sm, &wtot);
    if (total) { *total = wtot; target = mass_of(__uint_as_float((u32)target), wtot); }
    const u64 before = BYW ? wb : cb, mine = BYW ? w : c;
    if (before < target && before + mine >= target) {
        u32 b = b0;
        u64 run = before, own = 0;
        for (int i = 0; i < per; ++i) {
            const u64 x = BYW ? wt[b0 + i] : (u64)cnt[b0 + i];
            own = cnt ? cnt[b0 + i] : 0;
            if (run + x >= target) { b = b0 + i; break; }
            run += x;
            if (cnt) cb += cnt[b0 + i];
            if (wt) wb += wt[b0 + i];
        }
        *hit = Hit{b, cb, wb, own};
    }
    __syncthreads();
    *at = *hit;
    __syncthreads();
    return (BYW ? wtot : ct) >= target;
}

// The keys of bin b of the first histogram, from `lowest` on.
template <int KIND, int NB> __device__ __forceinline__ void keys_of_bin(const Scale& s, u32 b, u32 lowest, u32* klo, u32* khi) {
    auto bin = [&](u32 k) { return bin_of<KIND, NB>(s, value_of<KIND>(k)); };
    *klo = first_key(lowest, s.kmax, [&](u32 k) { return bin(k) <= b; });
    // the first key of a lower bin, if there is one, ends the bin
    *khi = b == 0 ? s.kmax : first_key(*klo, s.kmax, [&](u32 k) { return bin(k) < b; }) - 1u;
}

template <int NB> __device__ __forceinline__ int key_shift(u32 range) {
    constexpr int bits = NB >= 2048 ? 11 : NB >= 1024 ? 10 : 8;
    const int have = range ? 32 - __clz((int)range) : 0;
    return have > bits ? have - bits : 0;
}

// What is known of the cut once its bin is: the next keys to look at, or the cut itself.
template <int KIND, bool BYW, int NP> __device__ __forceinline__ void settle(const Scale& s, const Tables<KIND, NP>* tables, Find& f) {
    if (f.klo < f.khi) return;
    f.done = 1;
    if (BYW) {
        const u64 w = weight(s, tables, value_of<KIND>(f.klo));
        f.ne = (u32)((f.target - f.weight + w - 1) / (w ? w : 1));
    } else {
        f.ne = (u32)(f.target - f.count);
    }
}

// A row's parameters; ok = false: one of them is out of its range, and no outcome is drawn.
struct Params {
    float t, top_p, min_p;
    int top_k;
    bool ok;
};

__device__ __forceinline__ Params params_of(const SampleArgs& a, u64 r) {
    Params p;
    p.t = a.temperature ? a.temperature[r] : 1.f;
    p.top_k = a.top_k ? a.top_k[r] : 0;
    p.top_p = a.top_p ? a.top_p[r] : 1.f;
    p.min_p = a.min_p ? a.min_p[r] : 0.f;
    p.ok = p.t >= 0.f && p.t < kInf && p.top_k >= 0 && p.top_p >= 0.f && p.top_p < kInf && p.min_p >= 0.f && p.min_p <= 1.f;
    return p;
}

__device__ __forceinline__ u64 draw_at(double u, u64 w) {           // floor(floor(u 2^53) w / 2^53)
    const u64 r = (u64)(u * 9007199254740992.0);
    return (__umul64hi(r, w) << 11) | ((r * w) >> 53);
}

__device__ __forceinline__ void write_shot(const SampleArgs& a, u64 at, long long k, u64 w, u64 total) {
    a.out[at] = k;
    if (a.logp) a.logp[at] = k < 0 ? -kInf : (float)log((double)w / (double)total);
}

template <int NT> __device__ __forceinline__ void write_none(const SampleArgs& a, u64 row, u64 first, u64 last) {
    for (u64 i = first + threadIdx.x; i < last; i += NT) write_shot(a, row * a.shots + i, -1, 0, 1);
}

// ---- a row's chunks --------------------------------------------------------------------------------------------------
__device__ __forceinline__ bool keeps(const Cut& cut, float v, u32 idx) { return v > cut.v || (v == cut.v && idx <= cut.idx); }

// One chunk's numbers and (WEIGHTS) weights of what is kept.
template <int KIND, int STEPS, bool WEIGHTS, int NP> __device__ __forceinline__ void chunk_sums(const Row& row, const Scale& s, const Tables<KIND, NP>* tables, const Cut& cut, u32 j0, u32 lane, u64* w, u32* n) {
    float v[STEPS][4];
    load_chunk<KIND, STEPS>(row, j0, lane, v);
    u64 sum = 0;
    u32 num = 0;
#pragma unroll
    for (int it = 0; it < STEPS; ++it)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool keep = keeps(cut, v[it][i], 4 * (j0 + it * 64u + lane) - row.skew + i);
            num += keep;
            if (WEIGHTS) {
                const u64 x = weight(s, tables, v[it][i]);
                sum += keep ? x : 0;
            }
        }
    *n = wave_sum(num);
    *w = WEIGHTS ? wave_sum(sum) : 0;
}

// The index of a chunk's ne-th value that equals `value`; the whole wavefront asks.
template <int KIND, int STEPS> __device__ __forceinline__ u32 nth_equal(const Row& row, float value, u32 ne, u32 j0, u32 lane) {
    u32 run = 0, found = kAll;
    for (int it = 0; it < STEPS; ++it) {
        float v[4];
        const u32 j = j0 + it * 64u + lane;
        load4<KIND>(row, j, v);
        u32 n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) n += v[i] == value;
        const u32 incl = wave_scan(n);
        u32 rank = run + incl - n, mine = kAll;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (v[i] == value && ++rank == ne) mine = 4 * j - row.skew + i;
        const u64 who = __ballot(mine != kAll);
        if (who) { found = lane_of(mine, (u32)__ffsll((long long)who) - 1u); break; }
        run += last_lane(incl);
    }
    return found;
}

// The outcome of a chunk at which the running sum of kept weights, `base` before the chunk, exceeds t.  Whole wavefront.
template <int KIND, int STEPS, int NP> __device__ __forceinline__ long long find_in_chunk(const Row& row, const Scale& s, const Tables<KIND, NP>* tables, const Cut& cut, u32 j0, u64 base, u64 t, u32 lane, u64* w_at) {
    for (int it = 0; it < STEPS; ++it) {
        const u32 j = j0 + it * 64u + lane;
        float v[4];
        load4<KIND>(row, j, v);
        u64 w[4], four = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = 0;
            if (keeps(cut, v[i], 4 * j - row.skew + i)) w[i] = weight(s, tables, v[i]);
            four += w[i];
        }
        const u64 incl = wave_scan(four);
        const u64 hit = __ballot(base + incl > t);
        if (hit) {
            const u32 who = (u32)__ffsll((long long)hit) - 1u;
            u64 run = base + incl - four, wk = 0;
            u32 at = 4;
#pragma unroll
            for (u32 i = 0; i < 4; ++i) { run += w[i]; if (at == 4 && run > t) { at = i; wk = w[i]; } }
            *w_at = lane_of(wk, who);
            return (long long)lane_of(4 * j - row.skew + at, who);
        }
        base += last_lane(incl);
    }
    *w_at = 0;
    return -1;
}

// ---- sorting in LDS --------------------------------------------------------------------------------------------------
// Ascending, n distinct entries in room for a power of two of them, 256 or more.  Up to 256: each one's rank is the number of
// entries below it (1 x 32768 bf16, some 55 entries: sorting and drawing 1.7 us, by exchanges 5.2).  Else by exchanges, entries
// behind the n-th up to a power of two at the highest number.
template <int NT> __device__ __forceinline__ void sort_lds(u64* a, u32 n) {
    if (n <= 256) {
        constexpr int per = NT < 256 ? 256 / NT : 1;
        u64 mine[per];
        u32 rank[per];
        const u32 pad = (n + 3) & ~3u;
        if (threadIdx.x < pad - n) a[n + threadIdx.x] = ~0ull;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < per; ++k) {
            rank[k] = 0;
            mine[k] = threadIdx.x + k * NT < n ? a[threadIdx.x + k * NT] : 0;
        }
        if (threadIdx.x < n)
            for (u32 i = 0; i < pad; i += 4) {
                const u64 x = a[i], y = a[i + 1], z = a[i + 2], w = a[i + 3];
#pragma unroll
                for (int k = 0; k < per; ++k) rank[k] += (x < mine[k]) + (y < mine[k]) + (z < mine[k]) + (w < mine[k]);
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < per; ++k)
            if (threadIdx.x + k * NT < n) a[rank[k]] = mine[k];
        __syncthreads();
        return;
    }
    u32 size = 512;
    while (size < n) size <<= 1;
    for (u32 i = n + threadIdx.x; i < size; i += NT) a[i] = ~0ull;
    __syncthreads();
    for (u32 k = 2; k <= size; k <<= 1)
        for (u32 j = k >> 1; j > 0; j >>= 1) {
            for (u32 i = threadIdx.x; i < size / 2; i += NT) {
                const u32 lo = 2 * i - (i & (j - 1)), hi = lo + j;
                const u64 x = a[lo], y = a[hi];
                if ((x > y) == ((lo & k) == 0)) { a[lo] = y; a[hi] = x; }
            }
            __syncthreads();
        }
}

// What was worked out for all four is there before any of it is used: the compiler would move each one's work behind its test.
__device__ __forceinline__ void side_by_side(u64 (&w)[4]) {
    asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
}

// Four values of a lane into a histogram (counts, weights) of those with keys in klo .. khi: over distances (first: khi is the
// highest there is), or over keys down from khi.  The weights of all four are worked out side by side, then what is in the
// range is added; over keys few are, and only theirs are worked out.  (Over keys it is keys that are compared: a range may end
// between those of -0 and 0, which are equal as values.)
template <int KIND, int NB, int NP> __device__ __forceinline__ void add4(const Scale& s, const Tables<KIND, NP>* tables, const float (&v)[4], bool first, bool counts, bool weights, float low, u32 klo, u32 khi, int shift, u64* wt, u32* cnt) {
    u64 w[4] = {0, 0, 0, 0};
    u32 b[4];
    if (weights && first) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = weight(s, tables, v[i]);
        side_by_side(w);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = first ? bin_of<KIND, NB>(s, v[i]) : khi - key_of<KIND>(v[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (first ? v[i] >= low : b[i] <= khi - klo) {
            const u32 at = first ? b[i] : b[i] >> shift;
            if (counts) lds_add(cnt + at, 1u);
            if (weights) lds_add(wt + at, first ? w[i] : weight(s, tables, v[i]));
        }
}

// ---- one workgroup a row ---------------------------------------------------------------------------------------------
template <int NT> struct Shape;
// Bins of a histogram (and entries of a list to be sorted), chunks, vectors of a lane in a chunk; the most outcomes of a row that
// are given as many threads.  bf16, T, top-k and top-p of every row, in us by the fewer / the more threads: 64 or 256 threads 1 x 512
// 9.7 / 9.5, 1024 x 512 11.4 / 12.4, 8192 x 512 28.6 / 64; 256 or 1024 (more than 256 rows: 512) 1 x 1000 9.1 / 10.0, 1 x 8000
// 13.6 / 11.6, 512 x 8000 16.1 / 16.6, 4096 x 8000 59 / 106.  Top-p alone 1 x 8000 19.2 / 15.7, 4096 x 8000 95 / 149.
template <> struct Shape<64> { static constexpr int bins = 256, chunks = 4, steps = 1; static constexpr u32 most = 512; };
template <> struct Shape<256> { static constexpr int bins = 1024, chunks = 36, steps = 1; static constexpr u32 most = 8192; };
template <> struct Shape<512> { static constexpr int bins = 2048, chunks = 264, steps = 4; static constexpr u32 most = 262144; };
template <> struct Shape<1024> { static constexpr int bins = 2048, chunks = 264, steps = 4; static constexpr u32 most = 262144; };

// A row whose shots a later launch draws, all over the chip: what is kept of it (ok = 0: they are drawn already), and its kept
// weights up to the end of every chunk.
struct RowDraw { u32 ok, kmax; Cut cut; };
struct Later {
    RowDraw* rows;         // [rows], or NULL: nothing is left for later
    u64* chunk_w;          // [rows][Shape<1024>::chunks]
};

template <int KIND, int NT>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(4))) void k_sample_row(const SampleArgs a, const Later later) {
    constexpr int NB = Shape<NT>::bins, NC = Shape<NT>::chunks, STEPS = Shape<NT>::steps, LIST = 2 * NB;
    static_assert(NB >= 256 && (NB & (NB - 1)) == 0 && NB % NT == 0, "lists of up to NB entries are sorted in place, NB / NT of a thread");
    constexpr int UN = NT == 1024 ? 4 : 2;  // vectors of a thread on their way at once
    // two histograms; or: a list to be sorted, its entries and their weights, or values on their way; or: a list to be searched
    __shared__ struct { u64 wt[2 * NB]; u32 cnt[2 * NB]; } lds;
    u64* const wt = lds.wt;
    u32* const cnt = lds.cnt;
    constexpr int NP = kPowers<NT>;
    __shared__ Tables<KIND, NP> lds_tables;
    const Tables<KIND, NP>* const tables = &lds_tables;
    __shared__ u64 sm[16];
    __shared__ Hit hit;
    __shared__ u32 list_n, found;
    __shared__ u64 chunk_w[NC];             // kept weights of chunks, later of those up to each
    __shared__ u32 chunk_n[NC];

    const u32 lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const u64 r = grid_block();
    if (r >= (u64)a.rows) return;
    const Row row = row_of<KIND>(a, r);
    const Params p = params_of(a, r);
    const u32 nchunks = (row.vecs + 64 * STEPS - 1) / (64 * STEPS);
    if (later.rows && threadIdx.x == 0) later.rows[r] = RowDraw{0, 0, {0.f, 0}};

    // the first shots' uniforms are on their way while the row is read: a thread's, and a wavefront's
    const double* const uniforms = a.uniforms + r * a.shots;
    const double u_thread = threadIdx.x < (u64)a.shots ? uniforms[threadIdx.x] : 0.0;
    const double u_wave = wave < (u64)a.shots ? uniforms[wave] : 0.0;
    float high = kMasked<KIND>;             // of the thread's values
    walk<KIND, NT, UN>(row, 0, row.vecs, [&high](const float (&v)[4], u32) { high = fmaxf(fmaxf(high, fmaxf(v[0], v[1])), fmaxf(v[2], v[3])); });
    fill_tables<KIND, NT>(&lds_tables, a.bits, p.t == 1.f);
    if (threadIdx.x == 0) list_n = 0;
    const u32 kmax = block_max<NT>(key_of<KIND>(high), sm);
    __syncthreads();
    if (!p.ok || kmax < kLowest<KIND>) {
        write_none<NT>(a, r, 0, a.shots);
        if (threadIdx.x == 0 && a.kept) a.kept[r] = 0;
        return;
    }
    if (p.t == 0.f) {
        u32 first = 0;                      // the complement of the lowest index
        const float top = value_of<KIND>(kmax);
        walk<KIND, NT, UN>(row, 0, row.vecs, [&first, top, skew = row.skew](const float (&v)[4], u32 j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) if (v[i] == top) first = max(first, ~(4 * j - skew + i));
        });
        first = ~block_max<NT>(first, sm);
        for (u64 i = threadIdx.x; i < (u64)a.shots; i += NT) {
            const double u = i < NT ? u_thread : uniforms[i];
            write_shot(a, r * a.shots + i, u >= 0.0 && u < 1.0 ? (long long)first : -1, 1, 1);
        }
        if (threadIdx.x == 0 && a.kept) a.kept[r] = 1;
        return;
    }
    const Scale s = scale_of<KIND, NB, NP>(tables, kmax, p.t, a.bits);
    u32 lowest = kLowest<KIND>;
    if (p.min_p > 0.f)
        lowest = first_key(lowest, kmax, [&](u32 k) { return weight64<KIND>(s, value_of<KIND>(k)) >= (double)p.min_p; });
    u64* const le = wt;                     // of a list to be sorted: entries, and weights
    u64* const lw = wt + NB;

    // the list in order, its entries' weights; the sum of the weights before each thread's entries
    constexpr int per = NB / NT;
    auto ordered = [&](u32 n, u64 (&w)[per]) -> u64 {
        sort_lds<NT>(le, n);
        u64 sum = 0;
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const u32 at = threadIdx.x * per + i;
            w[i] = at < n ? weight(s, tables, value_of<KIND>(~(u32)(le[at] >> 32))) : 0;
            sum += w[i];
        }
        u64 all;
        return block_scan<NT>(sum, sm, &all);
    };
    // how many of the first n entries it takes for `before` and their weights to reach target (all of them at most)
    auto reach = [&](const u64 (&w)[per], u64 sum, u32 n, u64 before, u64 target) -> u32 {
        if (threadIdx.x == 0) found = n;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const u32 at = threadIdx.x * per + i;
            if (at < n && before + sum < target && before + sum + w[i] >= target) found = at + 1;
            sum += w[i];
        }
        __syncthreads();
        return uniform(found);
    };

    const float low = value_of<KIND>(lowest);
    bool by_k = p.top_k > 0 && (u32)p.top_k < row.cols, by_p = p.top_p < 1.f, summed = false, slow = false, listed = false;
    Cut cut{low, kAll};
    Hit at;
    // the outcomes from the distance's bin b up as a list; false: they are more than it holds
    auto collect = [&](u32 b) -> bool {
        u32* const slots = &list_n;
        walk<KIND, NT, UN>(row, 0, row.vecs, [s, low, b, slots, le, skew = row.skew](const float (&v)[4], u32 j) {
            const float top = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
            if (!(top >= low) || bin_of<KIND, NB>(s, top) > b) return;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!(v[i] >= low) || bin_of<KIND, NB>(s, v[i]) > b) continue;
                const u32 slot = lds_add(slots, 1u);
                if (slot < NB) le[slot] = (u64)~key_of<KIND>(v[i]) << 32 | (4 * j - skew + i);
            }
        });
        __syncthreads();
        const bool fits = list_n <= NB;
        if (!fits) {
            __syncthreads();
            if (threadIdx.x == 0) list_n = 0;
            __syncthreads();
        }
        return fits;
    };
    if (by_k) {
        // The k-th highest of the threads' own highest values has k values at or above it, and not many more: of 1024
        // threads' values the 50 highest come from about 49 threads.  From k near the number of threads on the lowest of these
        // maxima bounds little, and the scan is lost (with it / without, us: 256 x 131072 f32 k = 50 51 / 68, 640 81 / 93, 900
        // 115 / 94; 64 x 50021 300 35 / 39, 640 49 / 47).
        if (p.top_k <= NT * 5 / 8) {
            for (int i = threadIdx.x; i < NB; i += NT) cnt[i] = 0;
            __syncthreads();
            if (high >= low) lds_add(cnt + bin_of<KIND, NB>(s, high), 1u);
            __syncthreads();
            listed = select_bin<NT, NB, false>(cnt, nullptr, (u64)p.top_k, sm, &hit, &at) && collect(at.bin);
        }
        if (!listed) {
            for (int i = threadIdx.x; i < NB; i += NT) cnt[i] = 0;
            __syncthreads();
            walk<KIND, NT, UN>(row, 0, row.vecs, [s, low, cnt](const float (&v)[4], u32) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (v[i] >= low) lds_add(cnt + bin_of<KIND, NB>(s, v[i]), 1u);
            });
            __syncthreads();
            by_k = select_bin<NT, NB, false>(cnt, nullptr, (u64)p.top_k, sm, &hit, &at);
            listed = by_k && at.count + at.own <= NB && collect(at.bin);
            slow = by_k && (by_p || at.own > NB);
        }
    }
    if (listed) {
        // few outcomes down to the bin: in order they give the cut, and by index the draw
        u32 n = min(list_n, (u32)NB);      // (more only if the row was written to meanwhile)
        u64 total;
        if (n <= 64) {
            // a wavefront's registers hold them: ranks by reading every lane, no barriers (32768 scores, 22 left: 0.7 us less of a call)
            if (wave == 0) {
                u64 e = lane < n ? le[lane] : ~0ull;
                u32 rank = 0;
                for (u32 i = 0; i < n; ++i) rank += lane_of(e, i) < e;
                if (lane < n) le[rank] = e;
                __threadfence_block();
                e = lane < n ? le[lane] : ~0ull;
                n = min(n, (u32)p.top_k);
                u64 w = lane < n ? weight(s, tables, value_of<KIND>(~(u32)(e >> 32))) : 0;
                if (by_p) {
                    const u64 incl = wave_scan(w);
                    const u64 border = mass_of(p.top_p, last_lane(incl));
                    n = (u32)__popcll(__ballot(lane < n && (lane == 0 || incl - w < border)));
                }
                const u32 idx = (u32)e;
                rank = 0;
                for (u32 i = 0; i < n; ++i) rank += lane_of(idx, i) < idx;
                if (lane < n) {
                    le[rank] = (u64)idx << 32;
                    lw[rank] = w;
                }
                __threadfence_block();
                w = wave_scan(lane < n ? lw[lane] : 0ull);
                if (lane < n) lw[lane] = w;
                if (lane == 0) found = n;
            }
            __syncthreads();
            n = uniform(found);
            total = lw[n - 1];
        } else {
            u64 w[per];
            const u64 before = ordered(n, w);
            n = min(n, (u32)p.top_k);
            if (by_p) {
                u64 mass = 0;
#pragma unroll
                for (int i = 0; i < per; ++i) if (threadIdx.x * per + i < n) mass += w[i];
                u64 all;
                (void)block_scan<NT>(mass, sm, &all);
                n = reach(w, before, n, 0, mass_of(p.top_p, all));
            }
            u64 e[per];
#pragma unroll
            for (int i = 0; i < per; ++i) {
                const u32 k = threadIdx.x * per + i;
                lw[k] = w[i];
                e[i] = k < n ? (le[k] & 0xffffffffull) << 32 | k : 0;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < per; ++i) if (threadIdx.x * per + i < n) le[threadIdx.x * per + i] = e[i];
            __syncthreads();
            sort_lds<NT>(le, n);
            u64 sum = 0;
#pragma unroll
            for (int i = 0; i < per; ++i) {
                const u32 k = threadIdx.x * per + i;
                w[i] = k < n ? lw[(u32)le[k]] : 0;
                sum += w[i];
            }
            u64 run = block_scan<NT>(sum, sm, &total);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < per; ++i) { run += w[i]; lw[threadIdx.x * per + i] = run; }
            __syncthreads();
        }
        if (threadIdx.x == 0 && a.kept) a.kept[r] = (int)n;
        for (u64 i = threadIdx.x; i < (u64)a.shots; i += NT) {
            const double u = i < NT ? u_thread : uniforms[i];
            if (!(u >= 0.0 && u < 1.0)) { write_shot(a, r * a.shots + i, -1, 0, 1); continue; }
            const u64 t = draw_at(u, total);
            u32 lo = 0, len = n;                           // the first with a sum above t is in lo .. lo + len - 1
            while (len > 1) {
                const u32 half = len >> 1;
                if (lw[lo + half - 1] > t) len = half;
                else { lo += half; len -= half; }
            }
            write_shot(a, r * a.shots + i, (long long)(le[lo] >> 32), lw[lo] - (lo ? lw[lo - 1] : 0), total);
        }
        return;
    }
    u64 mass = 0;
    u32 klo = 0, khi = 0;                   // the keys of the bin that the cut falls into
    if (by_k && !slow) {
        keys_of_bin<KIND, NB>(s, at.bin, lowest, &klo, &khi);
    } else if (!by_k && by_p) {
        // a histogram of weights over the steps that they were worked out from, 32 to a factor of two (of small ones 16, 4)
        constexpr int shift = (NP > 256 ? 10 : 8) - (NB >= 2048 ? 5 : NB >= 1024 ? 4 : 2);
        static_assert((kTopStep<NP> >> shift) < NB, "");
        const float from = fmaxf(low, s.low_w);
        for (int i = threadIdx.x; i < NB; i += NT) wt[i] = 0;
        __syncthreads();
        walk<KIND, NT, UN>(row, 0, row.vecs, [s, tables, from, wt](const float (&v)[4], u32) {
            u64 w[4];
            u32 n[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = weight_of(s, tables, v[i], &n[i]);
            side_by_side(w);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[i] >= from) lds_add(wt + (n[i] >> shift), w[i]);
        });
        __syncthreads();
        (void)select_bin<NT, NB, true, true>(nullptr, wt, (u64)__float_as_uint(p.top_p), sm, &hit, &at, &mass);
        const u32 b = NB - 1 - at.bin;
        auto bin = [&](u32 k) -> u32 {
            u32 n;
            (void)weight_of(s, tables, value_of<KIND>(k), &n);
            return n >> shift;
        };
        // (the steps of values below s.low_w may pass 0 and come out as high ones: 63 factors of two are few spacings of 16 bits at
        // a low temperature)
        const u32 lowest_w = uniform(key_from<KIND>(from));
        klo = first_key(lowest_w, kmax, [&](u32 k) { return bin(k) >= b; });
        khi = bin(kmax) == b ? kmax : first_key(klo, kmax, [&](u32 k) { return bin(k) > b; }) - 1u;
    }
    if ((by_k || by_p) && !slow) {
        // what lies above the bin is kept, what lies in it decides: the chunks' sums of the ones, a list of the others
        const float from = value_of<KIND>(klo), to = value_of<KIND>(khi);
        // a wavefront's kept values are gathered in the lower histogram's place: their weights take fewer rounds then
        constexpr u32 room = 4 * NB / (NT / 64);
        static_assert(room >= 512, "a step's values fit behind another's");
        float* const kept_v = (float*)lw + wave * room;
        for (u32 c = wave; c < nchunks; c += NT / 64) {
            float v[STEPS][4];
            load_chunk<KIND, STEPS>(row, c * 64 * STEPS, lane, v);
            u32 num = 0, kept = 0;
            u64 sum = 0;
#pragma unroll
            for (int it = 0; it < STEPS; ++it) {
                const float top = fmaxf(fmaxf(v[it][0], v[it][1]), fmaxf(v[it][2], v[it][3]));
                if (__ballot(top >= from) == 0) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u64 above = __ballot(v[it][i] > to);
                    if (v[it][i] > to) kept_v[num + __popcll(above & ((1ull << lane) - 1))] = v[it][i];
                    num += (u32)__popcll(above);
                    if (v[it][i] >= from && v[it][i] <= to) {
                        const u32 slot = lds_add(&list_n, 1u);
                        if (slot < NB) le[slot] = (u64)~key_of<KIND>(v[it][i]) << 32 | (4 * (c * 64 * STEPS + it * 64u + lane) - row.skew + i);
                    }
                }
                if (it + 1 < STEPS && num <= room - 256) continue;
                __threadfence_block();
                for (u32 k = lane; k < num; k += 64) sum += weight(s, tables, kept_v[k]);
                __threadfence_block();
                kept += num;
                num = 0;
            }
            if (num > 0) {                  // (the last steps had nothing to add)
                __threadfence_block();
                for (u32 k = lane; k < num; k += 64) sum += weight(s, tables, kept_v[k]);
                __threadfence_block();
                kept += num;
            }
            sum = wave_sum(sum);
            if (lane == 0) { chunk_n[c] = kept; chunk_w[c] = sum; }
        }
        __syncthreads();
        u32 n = list_n;
        if (n <= NB) {
            u64 w[per];
            const u64 before = ordered(n, w);
            n = by_k ? min(n, (u32)((u64)p.top_k - at.count)) : reach(w, before, n, at.weight, mass_of(p.top_p, mass));
            // (an empty list: the row was written to while it was read)
            const u64 last = n > 0 ? le[n - 1] : (u64)~khi << 32 | kAll;
            cut = Cut{value_of<KIND>(~(u32)(last >> 32)), (u32)last};
#pragma unroll
            for (int i = 0; i < per; ++i) {
                const u32 k = threadIdx.x * per + i;
                if (k >= n) continue;
                const u32 c = ((u32)le[k] + row.skew) / (256 * STEPS);
                lds_add(chunk_n + c, 1u);
                lds_add(chunk_w + c, w[i]);
            }
            summed = true;
        } else {
            slow = true;                   // a bin of (nearly) equal values
        }
        __syncthreads();
    }
    if (slow) {
        // bins of keys, narrower each time, down to the cut's own: for top-k by counts, then for top-p by weights
        u32 ne = kAll;
        bool have_mass = false;
        auto count = [=](u32 h, bool first, u32 lo, u32 hi) {
            for (int i = threadIdx.x; i < NB; i += NT) { cnt[h + i] = 0; wt[h + i] = 0; }
            __syncthreads();
            const int shift = key_shift<NB>(hi - lo);
            const float from = value_of<KIND>(lo);
            walk<KIND, NT, 1>(row, 0, row.vecs, [=](const float (&v)[4], u32) {
                add4<KIND, NB>(s, tables, v, first, true, by_p, from, lo, hi, shift, wt + h, cnt + h);
            });
            __syncthreads();
        };
        count(0, true, lowest, kmax);
        for (int stage = by_k ? 0 : 1; stage < (by_p ? 2 : 1); ++stage) {
            u64 target = (u64)p.top_k;
            if (stage == 1) {
                if (!have_mass) {
                    u64 sum = 0;
                    for (int i = threadIdx.x; i < NB; i += NT) sum += wt[i];
                    (void)block_scan<NT>(sum, sm, &mass);
                }
                target = mass_of(p.top_p, mass);
            }
            Find f{};
            f.target = target;
            for (u32 h = 0;; h = NB) {
                Hit in;
                const u64* const w = by_p ? wt + h : nullptr;
                if (!(stage == 0 ? select_bin<NT, NB, false>(cnt + h, w, target - f.count, sm, &hit, &in)
                                 : select_bin<NT, NB, true>(cnt + h, w, target - f.weight, sm, &hit, &in)))
                    break;                 // (the row was written to while it was read)
                if (h == 0) {
                    keys_of_bin<KIND, NB>(s, in.bin, lowest, &f.klo, &f.khi);
                } else {
                    const int shift = key_shift<NB>(f.khi - f.klo);
                    const u32 top = f.khi - (in.bin << shift);
                    f.klo = top - f.klo < (1u << shift) ? f.klo : top - (1u << shift) + 1u;
                    f.khi = top;
                }
                f.count += in.count;
                f.weight += in.weight;
                if (stage == 0) settle<KIND, false>(s, tables, f);
                else settle<KIND, true>(s, tables, f);
                if (f.done) break;
                count(NB, false, f.klo, f.khi);
            }
            if (!f.done) continue;
            cut.v = value_of<KIND>(f.klo);
            ne = f.ne;
            if (stage == 0 && by_p) {
                mass = f.weight + (u64)f.ne * weight(s, tables, cut.v);
                have_mass = true;
            }
        }
        // the index of the last that stays of what equals the key
        for (u32 c = wave; c < nchunks; c += NT / 64) {
            u32 n = 0;
            for (int it = 0; it < STEPS; ++it) {
                float v[4];
                load4<KIND>(row, c * 64 * STEPS + it * 64u + lane, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) n += v[i] == cut.v;
            }
            n = wave_sum(n);
            if (lane == 0) chunk_n[c] = n;
        }
        if (threadIdx.x == 0) found = kAll;
        __syncthreads();
        static_assert(NC <= NT || NT == 64, "a thread has a chunk");
        const u32 mine = threadIdx.x < nchunks ? chunk_n[threadIdx.x] : 0;
        u64 all;
        const u64 before = block_scan<NT>((u64)mine, sm, &all);
        if (before < ne && before + mine >= ne) { found = threadIdx.x; list_n = (u32)(ne - before); }
        __syncthreads();
        if (found != kAll) cut.idx = nth_equal<KIND, STEPS>(row, cut.v, list_n, found * 64 * STEPS, lane);
        __syncthreads();
    }
    // several shots a wavefront: what is left goes into a list, if there is room
    const bool many = a.shots > NT / 64;
    if (!summed) {
        const bool count = many && row.cols <= (u32)LIST;
        for (u32 c = wave; c < nchunks; c += NT / 64) {
            u64 w;
            u32 n;
            if (count) chunk_sums<KIND, STEPS, false>(row, s, tables, cut, c * 64 * STEPS, lane, &w, &n);
            else chunk_sums<KIND, STEPS, true>(row, s, tables, cut, c * 64 * STEPS, lane, &w, &n);
            if (lane == 0) { chunk_w[c] = w; chunk_n[c] = n; }
        }
        __syncthreads();
    }
    u64 total, n_kept;
    {
        const bool mine = threadIdx.x < nchunks;
        const u32 n = mine ? chunk_n[threadIdx.x] : 0u;
        const u64 w = mine ? chunk_w[threadIdx.x] : 0u;
        const u64 n_before = block_scan<NT>((u64)n, sm, &n_kept);
        const u64 w_before = block_scan<NT>(w, sm, &total);
        if (mine) {
            chunk_n[threadIdx.x] = (u32)n_before | (n ? 0x80000000u : 0u);     // (2^18 outcomes at most)
            chunk_w[threadIdx.x] = w_before + w;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && a.kept) a.kept[r] = (int)n_kept;
    if (n_kept <= LIST && many) {
        // by index, a thread for every shot
        u64* lw = wt;
        u32* lk = cnt;
        for (u32 c = wave; c < nchunks; c += NT / 64) {
            const u32 packed = chunk_n[c];
            if (!(packed >> 31)) continue;
            u32 pos = packed & 0x7fffffffu;
            for (int it = 0; it < STEPS; ++it) {
                const u32 j = c * 64 * STEPS + it * 64u + lane;
                float v[4];
                load4<KIND>(row, j, v);
                u32 keep = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) keep |= (u32)keeps(cut, v[i], 4 * j - row.skew + i) << i;
                const u32 n = __popc(keep), incl = wave_scan(n);
                u32 to = pos + incl - n;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if ((keep >> i) & 1u) { lw[to] = key_of<KIND>(v[i]); lk[to] = 4u * j - row.skew + i; ++to; }
                pos += last_lane(incl);
            }
        }
        __syncthreads();
        constexpr int own = LIST / NT;
        u64 w[own], sum = 0;
        const u32 first = threadIdx.x * own;
#pragma unroll
        for (int i = 0; i < own; ++i) {
            w[i] = first + i < n_kept ? weight(s, tables, value_of<KIND>((u32)lw[first + i])) : 0;
            sum += w[i];
        }
        u64 run = block_scan<NT>(sum, sm, &total);
#pragma unroll
        for (int i = 0; i < own; ++i) {
            run += w[i];
            if (first + i < n_kept) lw[first + i] = run;
        }
        __syncthreads();
        for (u64 i = threadIdx.x; i < (u64)a.shots; i += NT) {
            const double u = i < NT ? u_thread : uniforms[i];
            if (!(u >= 0.0 && u < 1.0)) { write_shot(a, r * a.shots + i, -1, 0, 1); continue; }
            const u64 t = draw_at(u, total);
            u32 lo = 0, len = (u32)n_kept;
            while (len > 1) {
                const u32 half = len >> 1;
                if (lw[lo + half - 1] > t) len = half;
                else { lo += half; len -= half; }
            }
            write_shot(a, r * a.shots + i, (long long)lk[lo], lw[lo] - (lo ? lw[lo - 1] : 0), total);
        }
        return;
    }
    if (later.rows) {
        if (threadIdx.x < nchunks) later.chunk_w[r * NC + threadIdx.x] = chunk_w[threadIdx.x];
        if (threadIdx.x == 0) later.rows[r] = RowDraw{1, kmax, cut};
        return;
    }
    for (u64 i = wave; i < (u64)a.shots; i += NT / 64) {
        const double u = i < NT / 64 ? u_wave : uniforms[i];
        long long k = -1;
        u64 w = 0;
        if (u >= 0.0 && u < 1.0) {
            const u64 t = draw_at(u, total);
            u32 c = 0;
            for (u32 c0 = 0; c0 < nchunks; c0 += 64) {
                const u64 above = __ballot(c0 + lane < nchunks && chunk_w[min(c0 + lane, nchunks - 1)] > t);
                if (above) { c = c0 + (u32)__ffsll((long long)above) - 1u; break; }
            }
            k = find_in_chunk<KIND, STEPS>(row, s, tables, cut, c * 64 * STEPS, c ? chunk_w[c - 1] : 0, t, lane, &w);
        }
        if (lane == 0) write_shot(a, r * a.shots + i, k, w, total);
    }
}

// The shots that were left for later, a wavefront each.
template <int KIND> __global__ __launch_bounds__(256) void k_row_draw(const SampleArgs a, const Later later) {
    constexpr int NC = Shape<1024>::chunks, STEPS = Shape<1024>::steps, NP = kPowers<1024>;
    __shared__ Tables<KIND, NP> lds_tables;
    const Tables<KIND, NP>* const tables = &lds_tables;
    fill_tables<KIND, 256>(&lds_tables, a.bits, false);
    __syncthreads();
    const u64 at = grid_block() * 4 + (threadIdx.x >> 6);
    if (at >= (u64)a.rows * a.shots) return;
    const u64 r = at / a.shots;
    const RowDraw d = later.rows[r];
    if (!d.ok) return;
    const u32 lane = threadIdx.x & 63;
    const Row row = row_of<KIND>(a, r);
    const Params p = params_of(a, r);
    const Scale s = scale_of<KIND, Shape<1024>::bins, NP>(tables, d.kmax, p.t, a.bits);
    const u32 nchunks = (row.vecs + 64 * STEPS - 1) / (64 * STEPS);
    const u64* cw = later.chunk_w + r * NC;
    const u64 total = cw[nchunks - 1];
    const double u = a.uniforms[at];
    long long k = -1;
    u64 w = 0;
    if (u >= 0.0 && u < 1.0) {
        const u64 t = draw_at(u, total);
        u32 c = 0;
        for (u32 c0 = 0; c0 < nchunks; c0 += 64) {
            const u64 above = __ballot(c0 + lane < nchunks && cw[min(c0 + lane, nchunks - 1)] > t);
            if (above) { c = c0 + (u32)__ffsll((long long)above) - 1u; break; }
        }
        k = find_in_chunk<KIND, STEPS>(row, s, tables, d.cut, c * 64 * STEPS, c ? cw[c - 1] : 0, t, lane, &w);
    }
    if (lane == 0) write_shot(a, at, k, w, total);
}

// ---- long rows: their parts by workgroups of their own ---------------------------------------------------------------
// Bound by memory, a scan after the other (24 qubits, 128 MiB of state a scan: highest value 24 us, 5.6 TB/s; distances 37; keys
// 32 and 25, the third level ends at once; sums 26; running sums 12; 4096 shots 13).  The same steps, a launch each; what a step finds out about a row goes to the next one through the workspace: the parts'
// highest keys, histograms that all parts add to, the state of the search.  Every workgroup of a step works the state out
// again from the one before and its histogram; the row's first one writes it down.  Steps whose cut is known already end
// at once.
constexpr int kLongBins = 2048, kLongThreads = 1024, kLongSteps = 4, kLongChunk = 64 * kLongSteps * 4;
template <int KIND> using LongTables = Tables<KIND, 1024>;
constexpr int kKeySteps = 3;                       // 11 bits of a key each
constexpr int kLevels = 1 + 2 * kKeySteps;         // distances; keys for top-k; keys for top-p

struct LongState {
    u32 ok, kmax, lowest, stage;       // stage 0: no search under way; 1: top-k; 2: top-p
    Find f;
    Cut cut;
    u32 ne;              // how many of what equals the cut's key stay
    u32 have_mass;
    u64 mass;
};

struct Long {
    u32 parts, chunks, chunks_per_part, levels;
    u32* pmax;             // [rows][parts]
    u64* wt;               // [rows][kLevels][kLongBins]
    u32* cnt;              // [rows][kLevels][kLongBins]
    LongState* state;      // [rows][kLevels]
    u64* chunk_w;          // [rows][chunks]: weights above the cut's value
    u32* chunk_n;          // [rows][chunks]: numbers above it (low half) and of those that equal it
    u64* part_w;           // [rows][parts]: weights above the cut's value; then kept ones up to the part's end
    u64* part_n;           // [rows][parts]: numbers, halves of 32 bits; then equals before the part
};

__host__ __device__ inline u64 long_chunks(int64_t cols) { return ((u64)cols + 3 + kLongChunk - 1) / kLongChunk; }

// Parts of a chunk for each wavefront or more, and a workgroup or two a CU: every part adds its histogram to the row's, a
// few hundred bins at the same addresses (24 qubits: 1024 parts of 256 threads 47 us, 256 of 1024 threads 37).
__host__ inline u32 long_parts(int64_t rows, int64_t cols) {
    const u64 want = (long_chunks(cols) + kLongThreads / 64 - 1) / (kLongThreads / 64), most = std::max<u64>(1, 512 / (u64)rows);
    return (u32)std::min(std::min(want, most), (u64)256);
}

struct LongSizes { size_t pmax, wt, cnt, state, chunk_w, chunk_n, part, all; };
__host__ inline LongSizes long_sizes(int64_t rows, int64_t cols) {
    auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
    LongSizes s;
    const size_t n = (size_t)rows, chunks = (size_t)long_chunks(cols);
    s.pmax = up(n * long_parts(rows, cols) * 4);
    s.wt = up(n * kLevels * kLongBins * 8);
    s.cnt = up(n * kLevels * kLongBins * 4);
    s.state = up(n * kLevels * sizeof(LongState));
    s.chunk_w = up(n * chunks * 8);
    s.chunk_n = up(n * chunks * 4);
    s.part = up(n * long_parts(rows, cols) * 8);
    s.all = s.pmax + s.wt + s.cnt + s.state + s.chunk_w + s.chunk_n + 2 * s.part;
    return s;
}

template <int KIND> __device__ __forceinline__ void part_of(const Row& row, const Long& g, u32 part, u32* j0, u32* j1) {
    const u64 per = (u64)g.chunks_per_part * 64 * kLongSteps;
    *j0 = (u32)min((u64)part * per, (u64)row.vecs);
    *j1 = (u32)min((u64)(part + 1) * per, (u64)row.vecs);
}

template <int KIND> __global__ __launch_bounds__(kLongThreads) void k_long_max(const SampleArgs a, const Long g) {
    __shared__ u64 sm[kLongThreads / 64];
    const u64 r = grid_block() / g.parts;
    const u32 part = (u32)(grid_block() % g.parts);
    if (r >= (u64)a.rows) return;
    const Row row = row_of<KIND>(a, r);
    u32 j0, j1;
    float high = kMasked<KIND>;
    part_of<KIND>(row, g, part, &j0, &j1);
    walk<KIND, kLongThreads, 4>(row, j0, j1, [&high](const float (&v)[4], u32) { high = fmaxf(fmaxf(high, fmaxf(v[0], v[1])), fmaxf(v[2], v[3])); });
    const u32 kmax = block_max<kLongThreads>(key_of<KIND>(high), sm);
    if (threadIdx.x == 0) g.pmax[r * g.parts + part] = kmax;
    // the row's histograms start at zero
    const u32 bins = g.levels ? kLevels * kLongBins : 0;
    for (u32 i = part * kLongThreads + threadIdx.x; i < bins; i += g.parts * kLongThreads) {
        g.wt[r * (kLevels * kLongBins) + i] = 0;
        g.cnt[r * (kLevels * kLongBins) + i] = 0;
    }
}

__device__ __forceinline__ bool by_top_k(const SampleArgs& a, const Params& p) { return p.t > 0.f && p.top_k > 0 && (u32)p.top_k < a.cols; }
__device__ __forceinline__ bool by_top_p(const Params& p) { return p.t > 0.f && p.top_p < 1.f; }

// The histogram of the values of vectors j0 .. j1 with keys in klo .. khi, added to the row's.
template <int KIND> __device__ __forceinline__ void long_histogram(const Row& row, const Scale& s, u32 j0, u32 j1, bool first, bool counts, bool weights, u32 klo, u32 khi, const LongTables<KIND>* tables, u64* wt, u32* cnt, u64* gw, u32* gc) {
    for (int i = threadIdx.x; i < kLongBins; i += kLongThreads) { cnt[i] = 0; wt[i] = 0; }
    __syncthreads();
    const int shift = key_shift<kLongBins>(khi - klo);
    const float low = value_of<KIND>(klo);
    walk<KIND, kLongThreads, 4>(row, j0, j1, [=](const float (&v)[4], u32) {
        add4<KIND, kLongBins>(s, tables, v, first, counts, weights, low, klo, khi, shift, wt, cnt);
    });
    __syncthreads();
    for (int i = threadIdx.x; i < kLongBins; i += kLongThreads) {
        if (counts && cnt[i]) atomicAdd(&gc[i], cnt[i]);
        if (weights && wt[i]) atomicAdd(&gw[i], wt[i]);
    }
}

template <int KIND> __global__ __launch_bounds__(kLongThreads) void k_long_first(const SampleArgs a, const Long g) {
    __shared__ u64 sm[kLongThreads / 64], wt[kLongBins];
    __shared__ u32 cnt[kLongBins];
    __shared__ LongTables<KIND> lds_tables;
    const LongTables<KIND>* const tables = &lds_tables;
    fill_tables<KIND, kLongThreads>(&lds_tables, a.bits, false);
    __syncthreads();
    const u64 r = grid_block() / g.parts;
    const u32 part = (u32)(grid_block() % g.parts);
    if (r >= (u64)a.rows) return;
    const Row row = row_of<KIND>(a, r);
    const Params p = params_of(a, r);
    u32 kmax = 0;
    for (u32 i = threadIdx.x; i < g.parts; i += kLongThreads) kmax = max(kmax, g.pmax[r * g.parts + i]);
    kmax = block_max<kLongThreads>(kmax, sm);
    LongState st{};
    st.ok = p.ok && kmax >= kLowest<KIND>;
    st.kmax = kmax;
    st.lowest = kLowest<KIND>;
    if (st.ok) {
        const Scale s = scale_of<KIND, kLongBins, 1024>(tables, kmax, p.t > 0.f ? p.t : 1.f, a.bits);
        if (p.min_p > 0.f && p.t > 0.f)
            st.lowest = first_key(st.lowest, kmax, [&](u32 k) { return weight64<KIND>(s, value_of<KIND>(k)) >= (double)p.min_p; });
        st.cut = Cut{value_of<KIND>(p.t > 0.f ? st.lowest : kmax), kAll};
        st.ne = p.t > 0.f ? kAll : 1;
        if (by_top_k(a, p) || by_top_p(p)) {
            u32 j0, j1;
            part_of<KIND>(row, g, part, &j0, &j1);
            long_histogram<KIND>(row, s, j0, j1, true, by_top_k(a, p), by_top_p(p), st.lowest, kmax, tables, wt, cnt, g.wt + r * (kLevels * kLongBins), g.cnt + r * (kLevels * kLongBins));
        }
    }
    if (part == 0 && threadIdx.x == 0) g.state[r * kLevels] = st;
}

// The search after the histogram of level `prev`.
template <int KIND, int NT = kLongThreads> __device__ __forceinline__ void long_advance(const SampleArgs& a, const Params& p, const Scale& s, const LongTables<KIND>* tables, const Long& g, u64 r, int prev, u64* sm, Hit* hit, LongState* st) {
    if (!st->stage) return;
    Find& f = st->f;
    const u64* wt = g.wt + (r * kLevels + prev) * kLongBins;
    const u32* cnt = g.cnt + (r * kLevels + prev) * kLongBins;
    if (!f.done) {
        Hit at;
        const bool found = st->stage == 1 ? select_bin<NT, kLongBins, false>(cnt, by_top_p(p) ? wt : nullptr, f.target - f.count, sm, hit, &at)
                                          : select_bin<NT, kLongBins, true>(cnt, wt, f.target - f.weight, sm, hit, &at);
        if (!found) { st->stage = 0; return; }             // (the row was written to while it was read)
        const int shift = key_shift<kLongBins>(f.khi - f.klo);
        const u32 top = f.khi - (at.bin << shift);
        f.klo = top - f.klo < (1u << shift) ? f.klo : top - (1u << shift) + 1u;
        f.khi = top;
        f.count += at.count;
        f.weight += at.weight;
        if (st->stage == 1) settle<KIND, false>(s, tables, f);
        else settle<KIND, true>(s, tables, f);
    }
    if (!f.done) return;
    st->cut = Cut{value_of<KIND>(f.klo), kAll};
    st->ne = f.ne;
    if (st->stage == 1 && by_top_p(p)) {
        st->mass = f.weight + (u64)f.ne * weight(s, tables, value_of<KIND>(f.klo));
        st->have_mass = 1;
    }
    st->stage = 0;
}

template <int KIND> __device__ __forceinline__ void long_begin(const SampleArgs& a, const Params& p, const Scale& s, const LongTables<KIND>* tables, const Long& g, u64 r, u32 stage, u64* sm, Hit* hit, LongState* st) {
    const u64* wt = g.wt + r * kLevels * kLongBins;
    const u32* cnt = g.cnt + r * kLevels * kLongBins;
    Hit at;
    u64 target;
    if (stage == 1) {
        target = (u64)p.top_k;
        if (!select_bin<kLongThreads, kLongBins, false>(cnt, by_top_p(p) ? wt : nullptr, target, sm, hit, &at)) return;
    } else {
        u64 mass = st->mass;
        if (!st->have_mass) {
            u64 part = 0;
            for (int i = threadIdx.x; i < kLongBins; i += kLongThreads) part += wt[i];
            (void)block_scan<kLongThreads>(part, sm, &mass);
        }
        target = mass_of(p.top_p, mass);
        if (!select_bin<kLongThreads, kLongBins, true>(cnt, wt, target, sm, hit, &at)) return;
    }
    Find f;
    keys_of_bin<KIND, kLongBins>(s, at.bin, st->lowest, &f.klo, &f.khi);
    f.done = 0;
    f.ne = 0;
    f.target = target;
    f.count = at.count;
    f.weight = at.weight;
    if (stage == 1) settle<KIND, false>(s, tables, f);
    else settle<KIND, true>(s, tables, f);
    st->f = f;
    st->stage = stage;
    if (f.done) long_advance<KIND>(a, p, s, tables, g, r, 0, sm, hit, st);
}

// Level `level` after level `prev`: the first level of top-k is 1, that of top-p 1 + kKeySteps.
template <int KIND> __global__ __launch_bounds__(kLongThreads) void k_long_keys(const SampleArgs a, const Long g, int level, int prev) {
    __shared__ u64 sm[kLongThreads / 64], wt[kLongBins];
    __shared__ u32 cnt[kLongBins];
    __shared__ LongTables<KIND> lds_tables;
    const LongTables<KIND>* const tables = &lds_tables;
    fill_tables<KIND, kLongThreads>(&lds_tables, a.bits, false);
    __syncthreads();
    __shared__ Hit hit;
    const u64 r = grid_block() / g.parts;
    const u32 part = (u32)(grid_block() % g.parts);
    if (r >= (u64)a.rows) return;
    const Row row = row_of<KIND>(a, r);
    const Params p = params_of(a, r);
    LongState st = g.state[r * kLevels + prev];
    if (st.ok) {
        const Scale s = scale_of<KIND, kLongBins, 1024>(tables, st.kmax, p.t > 0.f ? p.t : 1.f, a.bits);
        long_advance<KIND>(a, p, s, tables, g, r, prev, sm, &hit, &st);
        if (level == 1 && by_top_k(a, p)) long_begin<KIND>(a, p, s, tables, g, r, 1, sm, &hit, &st);
        if (level == 1 + kKeySteps && by_top_p(p)) long_begin<KIND>(a, p, s, tables, g, r, 2, sm, &hit, &st);
        if (st.stage) {
            u32 j0, j1;
            part_of<KIND>(row, g, part, &j0, &j1);
            const size_t at = (r * kLevels + level) * kLongBins;
            long_histogram<KIND>(row, s, j0, j1, false, st.stage == 1, by_top_p(p), st.f.klo, st.f.khi, tables, wt, cnt, g.wt + at, g.cnt + at);
        }
    }
    if (part == 0 && threadIdx.x == 0) g.state[r * kLevels + level] = st;
}

// The chunks' weights and numbers above the cut's key, and how many equal it.
template <int KIND> __global__ __launch_bounds__(kLongThreads) void k_long_sums(const SampleArgs a, const Long g, int prev) {
    __shared__ u64 sm[kLongThreads / 64];
    __shared__ Hit hit;
    __shared__ LongTables<KIND> lds_tables;
    const LongTables<KIND>* const tables = &lds_tables;
    fill_tables<KIND, kLongThreads>(&lds_tables, a.bits, false);
    __syncthreads();
    const u64 r = grid_block() / g.parts;
    const u32 part = (u32)(grid_block() % g.parts);
    if (r >= (u64)a.rows) return;
    const Row row = row_of<KIND>(a, r);
    const Params p = params_of(a, r);
    LongState st = g.state[r * kLevels + prev];
    if (!st.ok) return;
    const Scale s = scale_of<KIND, kLongBins, 1024>(tables, st.kmax, p.t > 0.f ? p.t : 1.f, a.bits);
    long_advance<KIND>(a, p, s, tables, g, r, prev, sm, &hit, &st);
    const u32 lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const u32 c1 = min((part + 1) * g.chunks_per_part, g.chunks);
    u64 part_w = 0, part_n = 0;
    for (u32 c = part * g.chunks_per_part + wave; c < c1; c += kLongThreads / 64) {
        float v[kLongSteps][4];
        load_chunk<KIND, kLongSteps>(row, c * 64 * kLongSteps, lane, v);
        u64 w = 0;
        u32 n = 0;
#pragma unroll
        for (int it = 0; it < kLongSteps; ++it)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                n += (v[it][i] > st.cut.v) + ((u32)(v[it][i] == st.cut.v) << 16);
                const u64 x = weight(s, tables, v[it][i]);
                w += v[it][i] > st.cut.v ? x : 0;
            }
        n = wave_sum(n);
        w = wave_sum(w);
        part_w += w;
        part_n += (u64)(n >> 16) << 32 | (n & 0xffffu);
        if (lane == 0) {
            g.chunk_w[r * g.chunks + c] = w;
            g.chunk_n[r * g.chunks + c] = n;
        }
    }
    u64 sum_w, sum_n;
    (void)block_scan<kLongThreads>(lane == 0 ? part_w : 0, sm, &sum_w);
    (void)block_scan<kLongThreads>(lane == 0 ? part_n : 0, sm, &sum_n);
    if (threadIdx.x == 0) {
        g.part_w[r * g.parts + part] = sum_w;
        g.part_n[r * g.parts + part] = sum_n;
    }
}

// A wavefront's search of the row's shot number `at`: its part by the parts' sums, its chunk by those of the part's.
template <int KIND> __device__ __forceinline__ void long_shot(const SampleArgs& a, const Row& row, const Scale& s, const LongTables<KIND>* tables, const LongState& st, const Long& g, u64 r, u64 w_cut, u64 at, u32 lane) {
    const u64* pw = g.part_w + r * g.parts;
    const double u = a.uniforms[at];
    const u64 total = pw[g.parts - 1];
    long long k = -1;
    u64 w = 0;
    if (u >= 0.0 && u < 1.0) {
        const u64 t = draw_at(u, total);
        u32 lo = 0, len = g.parts;                 // the first part with a sum above t is in lo .. lo + len - 1
        while (len > 1) {
            const u32 stride = (len + 63) >> 6;
            const u32 probe = min((lane + 1) * stride, len) - 1;
            const u64 above = __ballot(pw[lo + probe] > t);
            const u32 f = above ? (u32)__ffsll((long long)above) - 1u : 63u;
            const u32 off = min(f * stride, len - 1);
            lo += off;
            len = min(stride, len - off);
        }
        u64 base = lo ? pw[lo - 1] : 0, eq = g.part_n[r * g.parts + lo];
        const u32 c1 = min((lo + 1) * g.chunks_per_part, g.chunks);
        for (u32 c0 = lo * g.chunks_per_part; c0 < c1; c0 += 64) {
            const u32 c = c0 + lane;
            const u32 n = c < c1 ? g.chunk_n[r * g.chunks + c] >> 16 : 0;
            const u64 before = eq + wave_scan((u64)n) - n;
            const u64 take = before >= st.ne ? 0 : min((u64)n, (u64)st.ne - before);
            const u64 own = (c < c1 ? g.chunk_w[r * g.chunks + c] : 0) + take * w_cut;
            const u64 incl = wave_scan(own);
            const u64 above = __ballot(base + incl > t);
            if (above) {
                const u32 f = (u32)__ffsll((long long)above) - 1u;
                base += lane_of(incl - own, f);
                k = find_in_chunk<KIND, kLongSteps>(row, s, tables, st.cut, (c0 + f) * 64 * kLongSteps, base, t, lane, &w);
                break;
            }
            base += last_lane(incl);
            eq = last_lane(before + n);
        }
    }
    if (lane == 0) write_shot(a, at, k, w, total);
}

// One workgroup a row: running sums over its parts, the last index that stays of what equals the cut's value, and (draw) its
// shots.
template <int KIND> __global__ __launch_bounds__(1024) void k_long_scan(const SampleArgs a, const Long g, int prev, int draw) {
    __shared__ u64 sm[16];
    __shared__ Hit hit;
    __shared__ LongTables<KIND> lds_tables;
    const LongTables<KIND>* const tables = &lds_tables;
    __shared__ u32 found, rank;
    fill_tables<KIND, 1024>(&lds_tables, a.bits, false);
    if (threadIdx.x == 0) found = kAll;
    __syncthreads();
    const u64 r = grid_block();
    if (r >= (u64)a.rows) return;
    const Row row = row_of<KIND>(a, r);
    const Params p = params_of(a, r);
    LongState st = g.state[r * kLevels + prev];
    __syncthreads();                               // (the state that is written may be the one that was read)
    if (!st.ok) {
        if (draw) write_none<1024>(a, r, 0, a.shots);
        if (threadIdx.x == 0 && a.kept) a.kept[r] = 0;
        if (threadIdx.x == 0) g.state[r * kLevels + kLevels - 1] = st;
        return;
    }
    const Scale s = scale_of<KIND, kLongBins, 1024>(tables, st.kmax, p.t > 0.f ? p.t : 1.f, a.bits);
    long_advance<KIND, 1024>(a, p, s, tables, g, r, prev, sm, &hit, &st);
    const u64 w_cut = weight(s, tables, st.cut.v);
    const bool mine = threadIdx.x < g.parts;       // (256 parts at most)
    const u64 n = mine ? g.part_n[r * g.parts + threadIdx.x] : 0;
    const u64 eq = n >> 32;
    u64 eq_all, n_kept, total;
    const u64 eq_before = block_scan<1024>(eq, sm, &eq_all);
    const u64 take = eq_before >= st.ne ? 0 : min(eq, (u64)st.ne - eq_before);
    (void)block_scan<1024>((n & 0xffffffffull) + take, sm, &n_kept);
    const u64 own = (mine ? g.part_w[r * g.parts + threadIdx.x] : 0) + take * w_cut;
    const u64 w_before = block_scan<1024>(own, sm, &total);
    if (mine) {
        g.part_w[r * g.parts + threadIdx.x] = w_before + own;
        g.part_n[r * g.parts + threadIdx.x] = eq_before;
    }
    // the ne-th of the equals: the thread that has its part looks through the part's chunks
    if (eq_before < st.ne && eq_before + eq >= st.ne) {
        u32 left = (u32)(st.ne - eq_before);
        u32 c = threadIdx.x * g.chunks_per_part;
        const u32 c1 = min(c + g.chunks_per_part, g.chunks);
        for (; c + 1 < c1; ++c) {
            const u32 k = g.chunk_n[r * g.chunks + c] >> 16;
            if (k >= left) break;
            left -= k;
        }
        found = c;
        rank = left;
    }
    __syncthreads();
    const u32 lane = threadIdx.x & 63;
    if (found != kAll) st.cut.idx = nth_equal<KIND, kLongSteps>(row, st.cut.v, rank, found * 64 * kLongSteps, lane);
    if (threadIdx.x == 0) {
        if (a.kept) a.kept[r] = (int)n_kept;
        g.state[r * kLevels + kLevels - 1] = st;
    }
    if (!draw) return;
    __threadfence_block();
    __syncthreads();
    for (u64 i = threadIdx.x >> 6; i < (u64)a.shots; i += 16)
        long_shot<KIND>(a, row, s, tables, st, g, r, w_cut, r * a.shots + i, lane);
}

template <int KIND> __global__ __launch_bounds__(256) void k_long_draw(const SampleArgs a, const Long g) {
    __shared__ LongTables<KIND> lds_tables;
    const LongTables<KIND>* const tables = &lds_tables;
    fill_tables<KIND, 256>(&lds_tables, a.bits, false);
    __syncthreads();
    const u64 at = grid_block() * 4 + (threadIdx.x >> 6);
    if (at >= (u64)a.rows * a.shots) return;
    const u64 r = at / a.shots;
    const LongState st = g.state[r * kLevels + kLevels - 1];
    const u32 lane = threadIdx.x & 63;
    if (!st.ok) {
        if (lane == 0) write_shot(a, at, -1, 0, 1);
        return;
    }
    const Row row = row_of<KIND>(a, r);
    const Params p = params_of(a, r);
    const Scale s = scale_of<KIND, kLongBins, 1024>(tables, st.kmax, p.t > 0.f ? p.t : 1.f, a.bits);
    long_shot<KIND>(a, row, s, tables, st, g, r, weight(s, tables, st.cut.v), at, lane);
}

}  // namespace

// Rows of more outcomes than one workgroup takes.  (Shorter ones are not split however few there are: a split row takes 4
// launches, 3 more for each of top-k and top-p, and one for many shots, 6 us each where it has nothing to do; 24 x 50021 f16
// take 31 us in one.)
static bool takes_parts(int64_t cols) { return cols > (int64_t)Shape<1024>::most; }

// More shots of a row than two for each of its wavefronts are drawn by another launch (6 x 66088 f32, 564 shots, wide nuclei:
// 209 -> 56 us; for a shot or two the launch costs more).
static bool drawn_later(int64_t shots) { return shots > 32; }

size_t sample_scratch_bytes(int64_t rows, int64_t cols, int64_t shots) {
    if (rows < 1 || cols <= (int64_t)Shape<256>::most) return 0;
    if (takes_parts(cols)) return long_sizes(rows, cols).all;
    if (!drawn_later(shots)) return 0;
    return (size_t)rows * (Shape<1024>::chunks * sizeof(u64) + sizeof(RowDraw));
}

template <int KIND> static hipError_t launch_long(const SampleArgs& a, char* scratch, hipStream_t st) {
    const LongSizes z = long_sizes(a.rows, a.cols);
    Long g;
    g.chunks = (u32)long_chunks(a.cols);
    g.parts = long_parts(a.rows, a.cols);
    g.chunks_per_part = (g.chunks + g.parts - 1) / g.parts;
    g.levels = a.top_k || a.top_p;
    g.wt = (u64*)scratch; scratch += z.wt;
    g.chunk_w = (u64*)scratch; scratch += z.chunk_w;
    g.part_w = (u64*)scratch; scratch += z.part;
    g.part_n = (u64*)scratch; scratch += z.part;
    g.state = (LongState*)scratch; scratch += z.state;
    g.pmax = (u32*)scratch; scratch += z.pmax;
    g.cnt = (u32*)scratch; scratch += z.cnt;
    g.chunk_n = (u32*)scratch;
    const dim3 grid = grid_of((u64)a.rows * g.parts), block(kLongThreads);
    hipLaunchKernelGGL(k_long_max<KIND>, grid, block, 0, st, a, g);
    hipLaunchKernelGGL(k_long_first<KIND>, grid, block, 0, st, a, g);
    int prev = 0;
    for (int stage = 0; stage < 2; ++stage) {
        if (!(stage == 0 ? (const void*)a.top_k : (const void*)a.top_p)) continue;
        for (int i = 1; i <= kKeySteps; ++i) {
            const int level = stage * kKeySteps + i;
            hipLaunchKernelGGL(k_long_keys<KIND>, grid, block, 0, st, a, g, level, prev);
            prev = level;
        }
    }
    hipLaunchKernelGGL(k_long_sums<KIND>, grid, block, 0, st, a, g, prev);
    const int here = a.shots <= 16;
    hipLaunchKernelGGL(k_long_scan<KIND>, grid_of((u64)a.rows), dim3(1024), 0, st, a, g, prev, here);
    if (!here)
        hipLaunchKernelGGL(k_long_draw<KIND>, grid_of(((u64)a.rows * a.shots + 3) / 4), dim3(256), 0, st, a, g);
    return hipGetLastError();
}

template <int KIND> static hipError_t launch_kind(const SampleArgs& a, void* scratch, hipStream_t st) {
    if (takes_parts(a.cols)) return launch_long<KIND>(a, (char*)scratch, st);
    const dim3 grid = grid_of((u64)a.rows);
    Later later{nullptr, nullptr};
    if (a.cols <= Shape<64>::most) {
        hipLaunchKernelGGL((k_sample_row<KIND, 64>), grid, dim3(64), 0, st, a, later);
        return hipGetLastError();
    }
    if (a.cols <= Shape<256>::most) {
        hipLaunchKernelGGL((k_sample_row<KIND, 256>), grid, dim3(256), 0, st, a, later);
        return hipGetLastError();
    }
    if (drawn_later(a.shots)) {
        later.chunk_w = (u64*)scratch;
        later.rows = (RowDraw*)(later.chunk_w + (u64)a.rows * Shape<1024>::chunks);
    }
    // A row for every CU or fewer: all of its threads for the row.  Two workgroups of half of them, which fill each other's
    // waits, where there are more rows (top-p, one / two: 256 x 13885 f16 25.1 / 25.7 us, 300 41.6 / 29.0, 512 46.2 / 31.6; 256 x
    // 131072 f32 105 / 127, 300 164 / 161, 512 195 / 185).
    if (a.rows <= 256) hipLaunchKernelGGL((k_sample_row<KIND, 1024>), grid, dim3(1024), 0, st, a, later);
    else hipLaunchKernelGGL((k_sample_row<KIND, 512>), grid, dim3(512), 0, st, a, later);
    if (later.rows)
        hipLaunchKernelGGL(k_row_draw<KIND>, grid_of(((u64)a.rows * a.shots + 3) / 4), dim3(256), 0, st, a, later);
    return hipGetLastError();
}

hipError_t launch_sample_scores(int kind, const SampleArgs& a, void* scratch, hipStream_t st) {
    switch (kind) {
        case kScoreF32: return launch_kind<kScoreF32>(a, scratch, st);
        case kScoreF16: return launch_kind<kScoreF16>(a, scratch, st);
        case kScoreBF16: return launch_kind<kScoreBF16>(a, scratch, st);
        case kScoreProbs: return launch_kind<kScoreProbs>(a, scratch, st);
        case kScoreState: return launch_kind<kScoreState>(a, scratch, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace qsv
