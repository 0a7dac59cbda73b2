// Penalties for repeated outcomes, biases and masks on rows of scores, and the backward pass of it.
//
//   v = z;  s_k: v = v > 0 ? v / R : v R;  v -= F c_k + A [c_k > 0];  v += b_k + sum_{j: i_j = k} e_j;  masked: v = -inf
//   s_k: outcome k is among the row's earlier ones, c_k: how often behind its prompt
//
// Bound by memory, or over the scores themselves by latency: only the places that change are written then.  A workgroup takes
// a part of a row's columns.  It counts the row's earlier outcomes that lie in its part in a table in LDS, a word a column:
//   bit 31 in the prompt | bits 21-30 one more than the place (among the part's entries) of the first that names it | bits 0-20 c_k
// and marks the columns with such a word in a bitmap, so that a vector of the row asks one byte for whether any of its columns
// has one.  Counts are whole numbers, and a column's entries are added by one thread in their order: no result depends on the
// order of atomics.
//
// Places with a word are worked out in 64 bits and rounded to the type once; the others, a score plus a shared bias, in 32 bits, which is
// half a step of the type and 2^-24 for types of 16.
#include "qsv_rows.h"
#include "qsv_scores.h"
#include "qsv_wave.h"

namespace qsv {
namespace {

typedef unsigned long long u64;
typedef unsigned u32;
constexpr float kInf = __builtin_inff();
constexpr u32 kPrompt = 1u << 31, kCount = (1u << 21) - 1;
constexpr int kEntryBit = 21, kEntryMost = 1023;

// What row r is adjusted by.
struct Row {
    float by, each, once;      // R, F, A
    int len, prompt;
    const u32* mask;           // NULL: all are allowed
    bool good;                 // its parameters are in their ranges
};

// (Absent parameters are read from here: loads without branches between them wait for memory once.)
__device__ const float kOff[4] = {0.f, 1.f, 0.f, 0.f};
__device__ const int kNone = 0;
template <class T> __device__ __forceinline__ T row_value(const T* p, u64 r, const T* off) { return *(p ? (in_global<T>*)p + r : (in_global<T>*)off); }

__device__ __forceinline__ Row row_of(const AdjustArgs& a, u64 r) {
    const float by = row_value(a.repetition, r, kOff + 1), each = row_value(a.frequency, r, kOff), once = row_value(a.presence, r, kOff);
    const int len = row_value(a.prior_len, r, &kNone), prompt = row_value(a.prompt_len, r, &kNone), at = row_value(a.mask_of, r, &kNone);
    Row f;
    f.by = by;
    f.each = each;
    f.once = once;
    f.len = a.prior_len ? len : a.n_prior;
    f.prompt = prompt;
    f.good = by > 0.f && by < kInf && fabsf(each) < kInf && fabsf(once) < kInf && f.prompt >= 0 && f.prompt <= f.len && f.len <= a.n_prior;
    f.mask = nullptr;
    if (a.masks) {
        const int64_t mask = a.mask_of ? (int64_t)at : a.mask_each ? (int64_t)r : 0;
        if (mask < -1 || mask >= a.n_masks) f.good = false;
        else if (mask >= 0) f.mask = a.masks + (u64)mask * (u64)a.mask_stride;
    }
    return f;
}

// The part's table in LDS: nothing of it is there where no row can have a history or entries.
struct Part {
    double* sum;       // by place among the part's entries: of all that name its column, at the first of them
    u32* word;         // by column
    u32* bits;
    int* column;       // by place among the part's entries, in their order
    float* bias;
    u32* entries;      // how many they are
};

__host__ __device__ inline int entry_room(int n) { return (n + 3) & ~3; }
__device__ __forceinline__ Part part_of(char* lds, int n_entries, u32 width) {
    Part p;
    const int room = entry_room(n_entries);
    p.sum = (double*)lds;
    p.word = (u32*)(p.sum + room);
    p.bits = p.word + width;
    p.column = (int*)(p.bits + width / 32);
    p.bias = (float*)(p.column + room);
    p.entries = (u32*)(p.bias + room);
    return p;
}
// Columns that the table has room for: of rows shorter than a part no more than theirs.
__host__ __device__ inline u32 part_room(u32 width, u32 cols) { return width < cols ? width : (cols + 127) & ~127u; }
inline size_t part_bytes(int n_entries, u32 width) { return (size_t)entry_room(n_entries) * 16 + (size_t)width * 4 + width / 8 + 16; }

__device__ __forceinline__ void mark(const Part& p, u32 k) { atomicOr(&p.bits[k / 32], 1u << (k & 31)); }

// 4 N of the row's earlier outcomes a thread: four at a time from place i0 on, -1 behind the last of len.
typedef int four __attribute__((ext_vector_type(4)));
typedef int four_at4 __attribute__((ext_vector_type(4), aligned(4)));
template <int NT, int N> __device__ __forceinline__ void prior_load(const int* prior, int len, int i0, four (&t)[N]) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int i = i0 + (u * NT + (int)threadIdx.x) * 4;
        t[u] = four{-1, -1, -1, -1};
        if (i0 + u * NT * 4 >= len) continue;
        if (i + 4 <= len) {
            t[u] = *(const four_at4*)(prior + i);
        } else {
            if (i < len) t[u][0] = prior[i];
            if (i + 1 < len) t[u][1] = prior[i + 1];
            if (i + 2 < len) t[u][2] = prior[i + 2];
        }
    }
}
// Those behind a row's own last one become -1.
template <int NT, int N> __device__ __forceinline__ void prior_cut(int len, four (&t)[N]) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int left = len - (u * NT + (int)threadIdx.x) * 4;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            if (w >= left) t[u][w] = -1;
    }
}

// Counts an outcome at column k of the part.
__device__ __forceinline__ void prior_add(const Part& p, u32 k, bool prompt) {
    if (prompt) atomicOr(&p.word[k], kPrompt);
    else atomicAdd(&p.word[k], 1u);
    mark(p, k);
}
// ... and is true for the first that names the column.
__device__ __forceinline__ bool prior_count(const Part& p, u32 k, bool prompt) {
    const u32 was = prompt ? atomicOr(&p.word[k], kPrompt) : atomicAdd(&p.word[k], 1u);
    if (was) return false;
    mark(p, k);
    return true;
}

// The part's entries in their order, gathered by the first wavefront.  ZERO: their columns' words start at 0.
template <bool ZERO> __device__ __forceinline__ void gather_entries(const AdjustArgs& a, u64 r, const Part& p, u32 c0, u32 n) {
    const u32 lane = threadIdx.x;
    const int* idx = a.entry_idx + r * (u64)a.n_entries;
    const float* bias = a.entry_bias + r * (u64)a.n_entries;
    u32 m = 0;
    for (int j0 = 0; j0 < a.n_entries; j0 += 256) {
        u32 k[4];
        float b[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = min(j0 + u * 64 + (int)lane, a.n_entries - 1);      // (loads without branches between them)
            k[u] = (u32)idx[j];
            b[u] = bias[j];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) k[u] = j0 + u * 64 + (int)lane < a.n_entries ? k[u] - c0 : ~0u;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const u64 in = __ballot(k[u] < n);
            const u32 at = m + __popcll(in & ((1ull << lane) - 1));
            if (k[u] < n) {
                p.column[at] = (int)k[u];
                p.bias[at] = b[u];
                if (ZERO) p.word[k[u]] = 0;
            }
            m += (u32)__popcll(in);
        }
    }
    if (lane < ((m + 3) & ~3u) - m) p.column[m + lane] = -1;
    if (lane == 0) *p.entries = m;
}

// A column's entries by the thread of the first of them; put(column, the place of that one).
template <int NT, class F> __device__ __forceinline__ void add_entries(const Part& p, F&& put) {
    const u32 m = *p.entries;
    for (u32 j = threadIdx.x; j < m; j += NT) {
        const int k = p.column[j];
        bool first = true;
        double sum = 0.0;
#pragma unroll 4
        for (u32 i = 0; i < m; i += 4) {
            const four x = *(const four*)(p.column + i);
            if (x[0] != k && x[1] != k && x[2] != k && x[3] != k) continue;
#pragma unroll
            for (u32 u = 0; u < 4; ++u)
                if (x[u] == k) {
                    if (i + u < j) first = false;
                    sum += (double)p.bias[i + u];
                }
        }
        if (!first) continue;
        p.sum[j] = sum;
        put((u32)k, j);
    }
}

// A value as it lies in memory: turned into a float where it is used, so that nothing waits for it before.
template <int KIND> __device__ __forceinline__ u32 raw_at(const char* row, u32 k) { return KIND == kScoreF32 ? ((const u32*)row)[k] : ((const unsigned short*)row)[k]; }
template <int KIND> __device__ __forceinline__ float from_raw(u32 v) {
    asm volatile("" : "+v"(v));       // here, and not where the load is
    if (KIND == kScoreF32) return __uint_as_float(v);
    if (KIND == kScoreF16) return __half2float(__ushort_as_half((unsigned short)v));
    return __uint_as_float(v << 16);
}

__device__ __forceinline__ bool seen(u32 word) { return (word & (kPrompt | kCount)) != 0; }

// A place whose column has a word.  inverse: 1 / R.
template <int KIND> __device__ __forceinline__ float adjusted(const Row& f, double inverse, const Part& p, u32 word, float z, float bias) {
    double v = (double)z;
    if (seen(word)) {
        v *= v > 0.0 ? inverse : (double)f.by;
        const u32 c = word & kCount;
        if (c) v -= (double)f.each * (double)c + (double)f.once;
    }
    v += (double)bias;
    const u32 e = (word >> kEntryBit) & kEntryMost;
    if (e) v += p.sum[e - 1];
    return narrowed<KIND>(v);
}

// ... and its gradient.
template <int KIND> __device__ __forceinline__ float taken_back(const Row& f, double inverse, u32 word, float z, float g) {
    return seen(word) ? narrowed<KIND>((double)g * (z > 0.f ? inverse : (double)f.by)) : g;
}

// The table of the part's n columns, a word turned into its place's result in 32 bits at once.  Histories that the threads keep (t, 8 NT)
// fetch the values at their columns first, and the first that counts at a column works it out; only words of theirs start at 0.  Longer ones
// have the bitmap looked through.  result(word, column, its value, (BACK) its score, 1 / R).
constexpr int kKept = 2;
constexpr int kTableNone = 0, kTableKept = 1, kTableLong = 2;
template <int KIND, int NT, bool BACK, bool KEPT, class G>
__device__ __forceinline__ void fill_part(const AdjustArgs& a, u64 r, const Row& f, const Part& p, const char* in, const char* scores, u32 c0, u32 n, four (&t)[kKept], G&& result) {
    const bool entries = !BACK && a.n_entries;
    u32 z[kKept][4], of[kKept][4];
    for (u32 i = threadIdx.x; i < (n + 31) / 32; i += NT) p.bits[i] = 0;
    if (KEPT) {
        prior_cut<NT>(f.len, t);
#pragma unroll
        for (int u = 0; u < kKept; ++u) {
            if (u * 4 * NT >= f.len) break;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if ((u32)t[u][w] - c0 < n) {
                    z[u][w] = raw_at<KIND>(in, (u32)t[u][w]);
                    if (BACK) of[u][w] = raw_at<KIND>(scores, (u32)t[u][w]);
                    p.word[(u32)t[u][w] - c0] = 0;
                }
        }
    } else {
        for (u32 i = threadIdx.x; i < (n + 3) / 4; i += NT) ((four*)p.word)[i] = four{0, 0, 0, 0};
    }
    if (entries && threadIdx.x < 64) gather_entries<true>(a, r, p, c0, n);
    __syncthreads();
    u32 mine = 0, mine_entries = 0;
    if (KEPT) {
#pragma unroll
        for (int u = 0; u < kKept; ++u) {
            if (u * 4 * NT >= f.len) break;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const u32 k = (u32)t[u][w] - c0;
                if (k < n && prior_count(p, k, (u * NT + (int)threadIdx.x) * 4 + w < f.prompt)) mine |= 1u << (u * 4 + w);
            }
        }
    } else {
        const int* prior = a.prior + r * (u64)a.prior_stride;
        constexpr int N = 8;
        for (int i0 = 0; i0 < f.len; i0 += 4 * N * NT) {
            four q[N];
            prior_load<NT>(prior, f.len, i0, q);
#pragma unroll
            for (int u = 0; u < N; ++u)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const u32 k = (u32)q[u][w] - c0;
                    if (k < n) prior_add(p, k, i0 + (u * NT + (int)threadIdx.x) * 4 + w < f.prompt);
                }
        }
    }
    if (entries)
        add_entries<NT>(p, [&](u32 k, u32 j) {
            if (atomicOr(&p.word[k], (j + 1) << kEntryBit)) return;
            mark(p, k);
            mine_entries |= 1u << (j / NT);
        });
    __syncthreads();
    if (KEPT) {
        if (mine | mine_entries) {
            const double inverse = 1.0 / (double)f.by;
#pragma unroll
            for (int u = 0; u < kKept; ++u) {
                if (!(mine >> (u * 4) & 15)) continue;
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    if (mine >> (u * 4 + w) & 1) {
                        u32* to = p.word + ((u32)t[u][w] - c0);
                        *to = __float_as_uint(result(*to, (u32)t[u][w], from_raw<KIND>(z[u][w]), BACK ? from_raw<KIND>(of[u][w]) : 0.f, inverse));
                    }
            }
            for (u32 left = mine_entries; left; left &= left - 1) {
                const u32 k = (u32)p.column[__builtin_ctz(left) * NT + threadIdx.x];
                p.word[k] = __float_as_uint(result(p.word[k], c0 + k, value_at<KIND>(in, c0 + k), 0.f, inverse));
            }
        }
    } else {
        const double inverse = 1.0 / (double)f.by;
        for (u32 k0 = threadIdx.x; k0 < n; k0 += 4 * NT) {          // four values under way
            u32 x[4], of[4], there = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const u32 k = k0 + u * NT;
                if (k < n && (p.bits[k / 32] >> (k & 31) & 1)) {
                    there |= 1u << u;
                    x[u] = raw_at<KIND>(in, c0 + k);
                    if (BACK) of[u] = raw_at<KIND>(scores, c0 + k);
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (there >> u & 1) p.word[k0 + u * NT] = __float_as_uint(result(p.word[k0 + u * NT], c0 + k0 + u * NT, from_raw<KIND>(x[u]), BACK ? from_raw<KIND>(of[u]) : 0.f, inverse));
        }
    }
    __syncthreads();
}

__device__ __forceinline__ u32 allowed_at(const u32* mask, u32 k) { return mask ? mask[k >> 5] >> (k & 31) : ~0u; }

// The gradients of a row's own biases at the columns c0 .. c1 - 1 (the first part's: of those that name no column, too).
template <int KIND, int NT> __device__ __forceinline__ void entry_gradients(const AdjustArgs& a, u64 r, const Row& f, const char* in, u32 c0, u32 c1) {
    const int* idx = a.entry_idx + r * (u64)a.n_entries;
    float* to = a.grad_entry + r * (u64)a.n_entries;
    for (int j = threadIdx.x; j < a.n_entries; j += NT) {
        const u32 k = (u32)idx[j];
        if (!f.good) { if (c0 == 0) to[j] = __builtin_nanf(""); }
        else if (k >= a.cols) { if (c0 == 0) to[j] = 0.f; }
        else if (k >= c0 && k < c1) to[j] = allowed_at(f.mask, k) & 1 ? value_at<KIND>(in, k) : 0.f;
    }
}

template <int KIND> constexpr u32 kBits = (1u << kPer<KIND>) - 1;     // of a vector's columns

// The bits of the vector of columns from k on.
template <int KIND> __device__ __forceinline__ u32 vector_bits(const u32* bits, u32 k) {
    return (((const unsigned char*)bits)[k / 8] >> (k & 7)) & kBits<KIND>;
}

template <int KIND> constexpr u32 kMasked = KIND == kScoreF32 ? 0xff800000u : KIND == kScoreBF16 ? 0xff80ff80u : 0xfc00fc00u;   // -inf

// The values of x where their bit is set, those of y elsewhere, as they lie in memory.
template <int KIND> __device__ __forceinline__ vec chosen(u32 bits, const vec& x, const vec& y) {
    auto all = [&](int i) { return (u32)((int)(bits << (31 - i)) >> 31); };
    vec r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u32 m = KIND == kScoreF32 ? all(i) : (all(2 * i) & 0xffffu) | (all(2 * i + 1) & 0xffff0000u);
        r[i] = (x[i] & m) | (y[i] & ~m);
    }
    return r;
}

template <int KIND> __device__ __forceinline__ vec global_vec(const in_global<char>* p) {
    if (KIND == kScoreF32) return *(const in_global<vec_at4>*)p;
    return *(const in_global<vec_at2>*)p;
}

// Columns c0 .. c0 + NT NV W - 1 of row r, all of them written.  BACK: the gradient.  A thread's vectors of the row are under way
// while the table is filled.  64 registers a thread: with the loads under way of eight wavefronts a SIMD 512 x 131072 bf16, 1024 earlier
// outcomes, a bias and masks, takes 66 us (4.1 TB/s; 290 vector instructions a wavefront keep the SIMDs busy half of it), with seven 74;
// without a table 256 x 131072 f32 48 us (5.5 TB/s, the rate of a large copy); one row of 32768 bf16, 700 earlier outcomes, 4.7.
template <int KIND, bool BACK, int NT, int NV, int TABLE> __global__ __launch_bounds__(NT, 8) void k_adjust(const AdjustArgs a, const u32 parts) {
    constexpr u32 W = kPer<KIND>, width = NT * NV * W;
    extern __shared__ __align__(16) char lds[];
    const u32 block = (u32)grid_block(), r32 = block / parts, c0 = (block - r32 * parts) * width;
    const u64 r = r32;
    if (r >= (u64)a.rows) return;
    const u32 n = min(width, a.cols - c0), whole = n / W;
    const char* scores = (const char*)a.scores + (a.scores ? r * (u64)a.stride * kSize<KIND> : 0);
    const char* in = BACK ? (const char*)a.grad_out + r * (u64)a.grad_out_stride * kSize<KIND> : scores;
    char* out = BACK ? (char*)a.grad + r * (u64)a.grad_stride * kSize<KIND> : (char*)a.out + r * (u64)a.out_stride * kSize<KIND>;
    const Part p = part_of(lds, BACK ? 0 : a.n_entries, part_room(width, a.cols));
    const float none = BACK ? 0.f : -kInf;
    four t[kKept];
    if (TABLE == kTableKept) prior_load<NT>(a.prior + r * (u64)a.prior_stride, a.n_prior, 0, t);
    vec x[NV];
    // Threads without a vector take the row's last one, and a row without any something else: loads without branches between them, whose
    // number is known, so that waiting for the ones before them is not waiting for them.
    const bool tiny = a.cols < W;
    const in_global<char>* in0 = tiny ? (const in_global<char>*)kOff : (const in_global<char>*)in;
    u32 at[NV];
#pragma unroll
    for (u32 v = 0; v < NV; ++v) {
        at[v] = tiny ? 0 : min(c0 + (v * NT + threadIdx.x) * W, a.cols - W);
        x[v] = global_vec<KIND>(in0 + at[v] * (u32)kSize<KIND>);
    }
    const Row f = row_of(a, r);
    if (BACK && a.grad_entry) entry_gradients<KIND, NT>(a, r, f, in, c0, c0 + n);
    if (!f.good) {
        for (u32 k = c0 + threadIdx.x; k < c0 + n; k += NT) store_one<KIND>(out, k, __builtin_nanf(""));
        return;
    }
    unsigned char allowed[NV];       // of the vectors' bytes; (without a mask, something)
    const in_global<unsigned char>* mask0 = f.mask ? (const in_global<unsigned char>*)f.mask : (const in_global<unsigned char>*)in0;
#pragma unroll
    for (u32 v = 0; v < NV; ++v) allowed[v] = mask0[at[v] / 8];
    if (TABLE)
        fill_part<KIND, NT, BACK, TABLE == kTableKept>(a, r, f, p, in, scores, c0, n, t, [&](u32 word, u32 k, float z, float of, double inverse) {
            return BACK ? taken_back<KIND>(f, inverse, word, of, z) : adjusted<KIND>(f, inverse, p, word, z, a.bias ? a.bias[k] : 0.f);
        });
    char* out0 = out + (u64)c0 * kSize<KIND>;
    const char* bias0 = (const char*)a.bias + (u64)c0 * 4;
#pragma unroll
    for (u32 v = 0; v < NV; ++v) {
        const u32 j = v * NT + threadIdx.x;
        if (j >= whole) continue;
        vec y = x[v];
        if (!BACK && a.bias) {
            float z[W];
#pragma unroll
            for (u32 i = 0; i < W; i += 4) {
                const vec q = *(const vec_at4*)(bias0 + (j * W + i) * 4u);
#pragma unroll
                for (u32 u = 0; u < 4; ++u) z[i + u] = part<KIND>(x[v], i + u) + __uint_as_float(q[u]);
            }
            y = packed<KIND>(z);
        }
        if (TABLE) {
            const u32 hit = vector_bits<KIND>(p.bits, j * W);
            if (hit) {
                float got[W];
#pragma unroll
                for (u32 i = 0; i < W; i += 4) {
                    const four q = *(const four*)(p.word + j * W + i);
#pragma unroll
                    for (u32 u = 0; u < 4; ++u) got[i + u] = __uint_as_float((u32)q[u]);
                }
                y = chosen<KIND>(hit, packed<KIND>(got), y);
            }
        }
        if (f.mask) y = chosen<KIND>((u32)allowed[v] >> (j * W & 7), y, BACK ? vec{0, 0, 0, 0} : vec{kMasked<KIND>, kMasked<KIND>, kMasked<KIND>, kMasked<KIND>});
        put_vec<KIND, false>(out0 + j * 16u, y);
    }
    const u32 k = c0 + whole * W + threadIdx.x;
    if (k < c0 + n) {
        const float z = value_at<KIND>(in, k);
        float y = !BACK && a.bias ? z + a.bias[k] : z;
        if (TABLE && (p.bits[(k - c0) / 32] >> (k & 31) & 1)) y = __uint_as_float(p.word[k - c0]);
        store_one<KIND>(out, k, allowed_at(f.mask, k) & 1 ? y : none);
    }
}

// ---- over the scores (BACK: over the gradient): only the places that change ------------------------------------------
// A row's masked places: 64 words of the mask a wavefront, a store for 64 columns by those lanes whose column is masked.  256 x 131072 f32:
// 23 us with nothing allowed (5.8 TB/s written); 45 with 5 %, since memory reads a line that is written in part (four of five are).
template <int KIND, int NT> __device__ __forceinline__ void fill_masked(const u32* mask, char* out, u32 c0, u32 c1, float none) {
    const u32 lane = threadIdx.x & 63;
    for (u32 k0 = c0 + (threadIdx.x >> 6) * 2048; k0 < c1; k0 += NT * 32) {
        const u32 at = k0 / 32 + lane, word = at * 32 < c1 ? mask[at] : ~0u;
#pragma unroll 4
        for (u32 i = 0; i < 32; ++i) {
            const u64 on = (u64)lane_of(word, 2 * i + 1) << 32 | lane_of(word, 2 * i);
            const u32 k = k0 + i * 64 + lane;
            if (!(on >> lane & 1) && k < c1) store_one<KIND>(out, k, none);
        }
    }
}

template <int KIND> __device__ __forceinline__ void fill_nan(char* out, u32 c0, u32 c1) {
    for (u32 k = c0 + threadIdx.x; k < c1; k += blockDim.x) store_one<KIND>(out, k, __builtin_nanf(""));
}

// Sums of blocks of rows (see k_adjust_columns) added up, 64 columns a workgroup, every fourth block a wavefront.
struct Join {
    const double* sums;      // [blocks][cols]
    u32 blocks, cols;
    float* out;
};
__device__ __forceinline__ void join(const Join& j, u64 at) {      // by the first 256 threads
    __shared__ double part[256];
    const u32 t = threadIdx.x;
    const u64 k = at * 64 + (t & 63);
    if (t < 256) {
        double v = 0.0;
        if (k < j.cols) {
#pragma unroll 8
            for (u32 b = t >> 6; b < j.blocks; b += 4) v += j.sums[(u64)b * j.cols + k];
        }
        part[t] = v;
    }
    __syncthreads();
    if (t < 64 && k < j.cols) j.out[k] = (float)(((part[t] + part[t + 64]) + part[t + 128]) + part[t + 192]);
}
__global__ __launch_bounds__(256) void k_adjust_join(const Join j) { join(j, grid_block()); }
inline u32 join_groups(const Join& j) { return j.out ? (j.cols + 63) / 64 : 0; }

// A row's earlier outcomes by their columns where they are few: a table of twice as many places and more, found by a product's upper
// bits and the next free place.
struct Hash {
    u32 *key, *word;      // by place; key: the column, ~0: free
    u32 shift;            // 32 - log2 of the places
    __device__ __forceinline__ u32 place(u32 k) const {
        const u32 last = (1u << (32 - shift)) - 1;
        for (u32 at = k * 2654435769u >> shift;; at = (at + 1) & last) {       // 2^32 over the golden ratio; there is a free place
            const u32 was = atomicCAS(&key[at], ~0u, k);
            if (was == ~0u || was == k) return at;
        }
    }
};
constexpr int kHashMost = 8192;          // earlier outcomes and entries: up to 16 of them a thread are kept
inline int hash_bits(int n) {
    int bits = 8;
    while (1 << bits < 2 * n) ++bits;
    return bits;
}
inline size_t hash_bytes(int n_entries, int bits) { return (size_t)entry_room(n_entries) * 16 + ((size_t)8 << bits) + 16; }

// A workgroup a row for its history and entries (`table`; bound by latency: parameters and tokens, the table, values and mask, stores: 256 rows of
// 131072 with 1000 earlier outcomes 8.9 us), and `parts` of `width` columns each for its masked places.  bits: log2 of the
// table's places, 0: nothing but the entries' gradients.  nan: rows with parameters out of range are written.  Workgroups behind the
// rows' add up sums of a shared bias, which are in nobody's way (513 x 50021 f16: a launch less, 49 -> 46 us).
template <int KIND, bool BACK, int NT> __global__ __launch_bounds__(NT) void k_adjust_over(const AdjustArgs a, const u32 parts, const u32 width, const int table, const int bits, const int nan, const Join sums) {
    extern __shared__ __align__(16) char lds[];
    const u32 block = (u32)grid_block(), r32 = block / (parts + table), at = block - r32 * (parts + table);
    const u64 r = r32;
    if (r >= (u64)a.rows) {
        if (sums.out) join(sums, block - (u32)a.rows * (parts + table));
        return;
    }
    const bool fills = at < parts;
    four t[4];
    if (!fills && bits) prior_load<NT>(a.prior + r * (u64)a.prior_stride, a.n_prior, 0, t);      // with the row's parameters under way
    const Row f = row_of(a, r);
    char* out = BACK ? (char*)a.grad + (a.grad ? r * (u64)a.grad_stride * kSize<KIND> : 0) : (char*)a.out + r * (u64)a.out_stride * kSize<KIND>;
    if (fills) {
        const u32 c0 = at * width, c1 = c0 + min(width, a.cols - c0);
        if (!f.good) fill_nan<KIND>(out, c0, c1);
        else if (f.mask) fill_masked<KIND, NT>(f.mask, out, c0, c1, BACK ? 0.f : -kInf);
        return;
    }
    const char* scores = (const char*)a.scores + (a.scores ? r * (u64)a.stride * kSize<KIND> : 0);
    if (BACK && a.grad_entry) {
        entry_gradients<KIND, NT>(a, r, f, (const char*)a.grad_out + r * (u64)a.grad_out_stride * kSize<KIND>, 0, a.cols);
        __syncthreads();       // read before the places are written
    }
    if (BACK && !a.grad) return;
    if (!f.good) {
        if (nan && !parts) fill_nan<KIND>(out, 0, a.cols);
        return;
    }
    if (!bits || (BACK && f.by == 1.f)) return;
    prior_cut<NT>(f.len, t);
    const double inverse = 1.0 / (double)f.by;
    const int room = entry_room(BACK ? 0 : a.n_entries);
    Hash h;
    Part p;                    // of the entries alone
    p.sum = (double*)lds;
    h.key = (u32*)(p.sum + room);
    h.word = h.key + (1u << bits);
    h.shift = 32 - bits;
    p.column = (int*)(h.word + (1u << bits));
    p.bias = (float*)(p.column + room);
    p.entries = (u32*)(p.bias + room);
    for (u32 i = threadIdx.x; i < (1u << bits) / 4; i += NT) {
        ((four*)h.key)[i] = four{-1, -1, -1, -1};
        ((four*)h.word)[i] = four{0, 0, 0, 0};
    }
    const bool entries = !BACK && a.n_entries;
    if (entries && threadIdx.x < 64) gather_entries<false>(a, r, p, 0, a.cols);
    __syncthreads();
    u32 place[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (u * 4 * NT >= f.len) continue;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            place[u][w] = ~0u;
            if ((u32)t[u][w] >= a.cols) continue;
            const u32 e = h.place((u32)t[u][w]);
            if (u * 4 * NT + (int)threadIdx.x * 4 + w < f.prompt) atomicOr(&h.word[e], kPrompt);
            else atomicAdd(&h.word[e], 1u);
            place[u][w] = e;
        }
    }
    if (entries) add_entries<NT>(p, [&](u32 k, u32 j) { atomicOr(&h.word[h.place(k)], (j + 1) << kEntryBit); });
    __syncthreads();
    // whoever takes a column's word first writes its place
    auto change = [&](u32 word, u32 k, float x, float z) {
        store_one<KIND>(out, k, BACK ? taken_back<KIND>(f, inverse, word, z, x) : adjusted<KIND>(f, inverse, p, word, x, 0.f));
    };
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (u * 4 * NT >= f.len) continue;
        u32 word[4], x[4], z[4], mask[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            word[w] = place[u][w] != ~0u ? atomicExch(&h.word[place[u][w]], 0u) : 0;
            if (!word[w]) continue;
            x[w] = raw_at<KIND>(out, (u32)t[u][w]);
            if (BACK) z[w] = raw_at<KIND>(scores, (u32)t[u][w]);
            mask[w] = f.mask ? f.mask[(u32)t[u][w] >> 5] : ~0u;
        }
#pragma unroll
        for (int w = 0; w < 4; ++w)
            if (word[w] && (mask[w] >> ((u32)t[u][w] & 31) & 1)) change(word[w], (u32)t[u][w], from_raw<KIND>(x[w]), BACK ? from_raw<KIND>(z[w]) : 0.f);
    }
    if (entries) {
        for (u32 j = threadIdx.x; j < *p.entries; j += NT) {
            const u32 k = (u32)p.column[j], word = atomicExch(&h.word[h.place(k)], 0u);
            if (word && (allowed_at(f.mask, k) & 1)) change(word, k, value_at<KIND>(out, k), 0.f);
        }
    }
}

// The same for long histories, by parts of a row with a table of their columns each (256 x 131072 bf16, 20000 earlier outcomes: 66 us).
template <int KIND, bool BACK, bool KEPT> __global__ __launch_bounds__(1024) void k_adjust_over_parts(const AdjustArgs a, const u32 parts, const u32 width, const int nan) {
    constexpr int NT = 1024;
    extern __shared__ __align__(16) char lds[];
    const u32 block = (u32)grid_block(), r32 = block / parts, c0 = (block - r32 * parts) * width;
    const u64 r = r32;
    if (r >= (u64)a.rows) return;
    const Row f = row_of(a, r);
    const u32 c1 = c0 + min(width, a.cols - c0);
    const char* scores = (const char*)a.scores + (a.scores ? r * (u64)a.stride * kSize<KIND> : 0);
    char* out = BACK ? (char*)a.grad + (a.grad ? r * (u64)a.grad_stride * kSize<KIND> : 0) : (char*)a.out + r * (u64)a.out_stride * kSize<KIND>;
    const Part p = part_of(lds, BACK ? 0 : a.n_entries, part_room(width, a.cols));
    if (BACK && a.grad_entry) {
        entry_gradients<KIND, NT>(a, r, f, (const char*)a.grad_out + r * (u64)a.grad_out_stride * kSize<KIND>, c0, c1);
        __syncthreads();       // read before the places are written
    }
    if (!f.good) {
        if (nan) fill_nan<KIND>(out, c0, c1);
        return;
    }
    if (BACK && f.by == 1.f) return;
    four t[kKept];
    if (KEPT) prior_load<NT>(a.prior + r * (u64)a.prior_stride, a.n_prior, 0, t);
    fill_part<KIND, NT, BACK, KEPT>(a, r, f, p, out, scores, c0, c1 - c0, t, [&](u32 word, u32, float x, float of, double inverse) {
        return BACK ? taken_back<KIND>(f, inverse, word, of, x) : adjusted<KIND>(f, inverse, p, word, x, 0.f);
    });
    for (u32 k = c0 + threadIdx.x; k < c1; k += NT)
        if ((p.bits[(k - c0) / 32] >> (k & 31) & 1) && (allowed_at(f.mask, k) & 1)) store_one<KIND>(out, k, __uint_as_float(p.word[k - c0]));
}

// ---- a bias that all rows share --------------------------------------------------------------------------------------
// Sums over a block of rows of a tile of columns, a vector of them a lane, and the gradient of the scores on the way (grad, or NULL).
// A workgroup's wavefronts take every fourth row each and add their sums in order at the end.  OVER: grad lies over
// grad_out, and vectors without a masked place are left.  Sums are in 64 bits: they cost the kernel nothing.  4096 x 32768 bf16: 105 us, 5.1
// TB/s, and 7 for the join.  Results beside grad_out go past the caches: with it / without, us, 513 x 50021 f16 with histories 38 / 46,
// 4096 x 32768 bf16 103 / 108 and with the gradient read once more 155 / 165, 256 x 32768 bf16 12.8 / 14.2 and 21.7 / 22.4, f32 16.1 /
// 20.8 and 32.1 / 31.5; over grad_out there is no difference.
constexpr u32 kSumThreads = 256, kSumGroups = 4, kMostSumRows = 256;

template <int KIND, bool OVER> __global__ __launch_bounds__(kSumThreads) void k_adjust_columns(const AdjustArgs a, const u32 tiles, const u32 block_rows, double* sums, float* out_sums) {
    constexpr u32 W = kPer<KIND>, GROUPS = kSumGroups, LANES = kSumThreads / GROUPS;
    constexpr u32 N = 4;                    // rows under way
    __shared__ const u32* masks[kMostSumRows];
    __shared__ int good[kMostSumRows];
    __shared__ double joined[(GROUPS - 1) * LANES * W];
    const u32 block = (u32)grid_block(), b32 = block / tiles, group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const u32 k = (block - b32 * tiles) * (LANES * W) + lane * W;
    const u64 b = b32;
    if (b * block_rows >= (u64)a.rows) return;
    const u64 r0 = b * block_rows;
    const u32 rows = (u32)min((u64)block_rows, (u64)a.rows - r0);
    if (threadIdx.x < rows) {
        const Row f = row_of(a, r0 + threadIdx.x);
        masks[threadIdx.x] = f.mask;
        good[threadIdx.x] = f.good;
    }
    __syncthreads();
    const u32 n = k < a.cols ? min(W, a.cols - k) : 0;
    const char* in = (const char*)a.grad_out + (r0 * (u64)a.grad_out_stride + k) * kSize<KIND>;
    char* out = (char*)a.grad + (a.grad ? (r0 * (u64)a.grad_stride + k) * kSize<KIND> : 0);
    double sum[W] = {};
    auto some = [&](u32 i0, u32 count) {
        vec x[N];
        u32 allowed[N];
#pragma unroll
        for (u32 u = 0; u < N; ++u) {
            if (u >= count) continue;
            const u32 row = i0 + u * GROUPS;
            const char* p = in + (u64)row * (u64)a.grad_out_stride * kSize<KIND>;
            if (n == W) {
                x[u] = vec_at<KIND>(p);
            } else {
                float v[W] = {};
#pragma unroll
                for (u32 i = 0; i < W; ++i)
                    if (i < n) v[i] = value_at<KIND>(p, i);
                x[u] = packed<KIND>(v);
            }
            const u32* mask = masks[row];
            allowed[u] = mask && n ? vector_bits<KIND>(mask, k) : kBits<KIND>;
        }
#pragma unroll
        for (u32 u = 0; u < N; ++u) {
            if (u >= count) continue;
            const u32 row = i0 + u * GROUPS;
            const bool ok = good[row];
            float v[W];
#pragma unroll
            for (u32 i = 0; i < W; ++i) {
                v[i] = !ok ? __builtin_nanf("") : allowed[u] >> i & 1 ? part<KIND>(x[u], i) : 0.f;
                sum[i] += (double)v[i];
            }
            if (!a.grad || (OVER && ok && allowed[u] == kBits<KIND>)) continue;
            char* p = out + (u64)row * (u64)a.grad_stride * kSize<KIND>;
            if (n == W) {
                put_vec<KIND, !OVER>(p, packed<KIND>(v));
            } else {
#pragma unroll
                for (u32 i = 0; i < W; ++i)
                    if (i < n) store_one<KIND>(p, i, v[i]);
            }
        }
    };
    u32 i = group;
    for (; i + (N - 1) * GROUPS < rows; i += N * GROUPS) some(i, N);
    if (i < rows) some(i, (rows - i + GROUPS - 1) / GROUPS);
    if (group) {
#pragma unroll
        for (u32 i = 0; i < W; ++i) joined[((group - 1) * W + i) * LANES + lane] = sum[i];
    }
    __syncthreads();
    if (group) return;
#pragma unroll
    for (u32 g = 0; g + 1 < GROUPS; ++g)
#pragma unroll
        for (u32 i = 0; i < W; ++i) sum[i] += joined[(g * W + i) * LANES + lane];
#pragma unroll
    for (u32 i = 0; i < W; ++i)
        if (i < n) {
            if (out_sums) out_sums[k + i] = (float)sum[i];
            else sums[b * a.cols + k + i] = sum[i];
        }
}

// Rows of a block, and few enough blocks to add up.  16 / 32 / 64 / 128 rows, us: 4096 x 32768 bf16 130 / 114 / 114 / 116, 4096 x 5000 38 / 31 /
// 33 / 46, 100 x 1000 10 / 11 / 17 / 22, 1024 x 32768 f32 62 / 63 / 72 / 62.  (One wavefront after the other instead of four rows side
// by side: 4096 x 32768 bf16 138, 16 x 1000 f32 17.3 against 13.9 with all that goes with it.)
u32 sum_rows(int64_t rows) { return (u32)std::max((int64_t)32, std::min((int64_t)kMostSumRows, rows / 128)); }

// ---- launches --------------------------------------------------------------------------------------------------------
// A kernel is asked for before it takes more than 64 KiB of LDS.
hipError_t room_for(const void* kernel, size_t lds) {
    return lds > 65536 ? hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) : hipSuccess;
}

template <int KIND, bool BACK, int NT, int NV, int TABLE> hipError_t launch_all(const AdjustArgs& a, hipStream_t st) {
    constexpr u32 width = NT * NV * kPer<KIND>;
    const u32 parts = (a.cols + width - 1) / width;
    if ((u64)a.rows * parts >> 32) return hipErrorInvalidValue;
    const size_t lds = TABLE != kTableNone ? part_bytes(BACK ? 0 : a.n_entries, part_room(width, a.cols)) : 0;
    if (const hipError_t e = room_for((const void*)&k_adjust<KIND, BACK, NT, NV, TABLE>, lds)) return e;
    hipLaunchKernelGGL((k_adjust<KIND, BACK, NT, NV, TABLE>), grid_of((u64)a.rows * parts), dim3(NT), lds, st, a, parts);
    return hipGetLastError();
}
template <int KIND, bool BACK, int NT, int NV> hipError_t launch_table(const AdjustArgs& a, hipStream_t st) {
    return a.n_prior <= 4 * kKept * NT ? launch_all<KIND, BACK, NT, NV, kTableKept>(a, st) : launch_all<KIND, BACK, NT, NV, kTableLong>(a, st);
}

// Threads and vectors a thread by row length, history and how many workgroups that makes, us:
//   no table     256 x 1 / 256 x 2 / 512 x 2: 256 x 131072 bf16 26.9 / 27.1 / 27.6, f32 46.4 / 48.2 / 48.1; with a bias 29.4 / 29.1 / 29.0
//   up to 128 vectors  64 x 1 / 256 x 1 / 1024 x 1: 8 x 500 f32, 50 earlier outcomes 4.0 / 4.0 / 4.7, 300 4.9 / 3.9 / 4.7, 4000 7.8 / 5.5 / 5.4, 32768
//                40 / 19.1 / 18.6; 4096 x 500 f32, 50 8.8 / 10.8 / 32, 300 10.7 / 10.9 / 32, 1000 19.3 / 12.4 / 32, 4000 56 / 31 / 41; 1024 x 70 f16,
//                50 4.8 / 5.4 / 10.6, 1000 7.3 / 5.7 / 10.8, 4000 17.1 / 17.1 / 11.9
//   short rows   64 x 1 / 256 x 1 / 256 x 2: 4096 x 500 f32, 50 earlier outcomes 8.8 / 11.0 / 11.2; 256 x 1 / 256 x 2 / 512 x 2: 4096 x 1500 f32
//                18.1 / 13.0 / 18.1, 1024 x 5000 bf16 9.8 / 8.5 / 8.3
//   many parts   256 x 1 / 256 x 2 / 512 x 2 / 1024 x 2: 512 x 131072 bf16, 1024 earlier ones 88 / 71 / 66 / 68; 256 x 131072 f32, 300 of them 57.5 /
//                47.9 / 47.3 / 48.1, 3000 94 / 67 / 55 / 57, bf16 60 / 52 / 33 / 33; 128 x 131072 bf16, 16000 50 / 41 / 34.9 / 35.7
//   few parts    256 x 1 / 512 x 1 / 1024 x 1: 8 x 200003 f16, 32768 earlier ones 16.7 / 12.8 / 11.5
template <int KIND, bool BACK> hipError_t launch_all(const AdjustArgs& a, hipStream_t st) {
    const bool table = BACK ? a.n_prior && a.repetition : a.n_prior || a.n_entries;
    const u32 vecs = (a.cols + kPer<KIND> - 1) / kPer<KIND>;
    const bool few = (u64)a.rows * ((vecs + 1023) / 1024) < 512;
    if (!table) return few ? launch_all<KIND, BACK, 256, 1, kTableNone>(a, st) : launch_all<KIND, BACK, 256, 2, kTableNone>(a, st);
    if (vecs <= 128 && a.n_prior <= 4 * 64) return launch_table<KIND, BACK, 64, 1>(a, st);
    if (few) return a.n_prior > 8 * 256 ? launch_table<KIND, BACK, 1024, 1>(a, st) : launch_table<KIND, BACK, 256, 1>(a, st);
    if (vecs <= 128) return launch_table<KIND, BACK, 256, 1>(a, st);
    if (a.n_prior > 8 * 256) return launch_table<KIND, BACK, 1024, 2>(a, st);
    if (vecs <= 256) return launch_table<KIND, BACK, 256, 1>(a, st);
    return vecs <= 512 ? launch_table<KIND, BACK, 256, 2>(a, st) : launch_table<KIND, BACK, 512, 2>(a, st);
}

// In place, 131072 columns: 256 / 1024 threads a row, us: 256 rows, 1000 earlier outcomes 8.9 / 9.3, 2000 13.8 / 11.8, 4000 22.5 / 17.3.  By rows / by
// parts: 1 row, 6000 9.5 / 7.9, 8000 10.6 / 7.9; 64 rows with masks, 8000 26 / 31.  Parts of 8192 / 16384 / 32768 columns: 256 rows, 20000
// 82 / 66 / 82, 32 rows 14.4 / 15.7 / 21.9.
// fill: masked places and rows with parameters out of range are written too.
template <int KIND, bool BACK, int NT> hipError_t launch_over(const AdjustArgs& a, u32 filled, int table, int bits, bool fill, hipStream_t st, const Join& sums) {
    const size_t lds = bits ? hash_bytes(BACK ? 0 : a.n_entries, bits) : 0;
    if (const hipError_t e = room_for((const void*)&k_adjust_over<KIND, BACK, NT>, lds)) return e;
    hipLaunchKernelGGL((k_adjust_over<KIND, BACK, NT>), grid_of((u64)a.rows * (filled + table) + join_groups(sums)), dim3(NT), lds, st, a, filled, NT * 32, table, bits, fill, sums);
    return hipGetLastError();
}

template <int KIND, bool BACK, bool KEPT> hipError_t launch_over_parts(const AdjustArgs& a, u32 width, bool nan, hipStream_t st) {
    const u32 parts = (a.cols + width - 1) / width;
    const size_t lds = part_bytes(BACK ? 0 : a.n_entries, part_room(width, a.cols));
    if (const hipError_t e = room_for((const void*)&k_adjust_over_parts<KIND, BACK, KEPT>, lds)) return e;
    hipLaunchKernelGGL((k_adjust_over_parts<KIND, BACK, KEPT>), grid_of((u64)a.rows * parts), dim3(1024), lds, st, a, parts, width, nan);
    return hipGetLastError();
}

template <int KIND, bool BACK> hipError_t launch_over(const AdjustArgs& a, bool fill, hipStream_t st, const Join& sums = Join{nullptr, 0, 0, nullptr}) {
    const bool values = !BACK || a.grad, changes = values && (BACK ? a.n_prior && a.repetition : a.n_prior || a.n_entries);
    const int entries = BACK ? 0 : a.n_entries, n = changes ? a.n_prior + entries : 0;
    const u64 eights = (u64)a.rows * ((a.cols + 8191) / 8192);
    const bool by_parts = n > kHashMost || (n > 4096 && eights <= 256), wide = !by_parts && n > 1024;
    if ((2 * eights + (u64)a.rows + join_groups(sums)) >> 32) return hipErrorInvalidValue;
    // a row's masked places, or all of it where its parameters are out of range
    const bool ranges = a.repetition || a.frequency || a.presence || a.prior_len || a.prompt_len;
    const u32 fill_width = wide ? 1024 * 32 : 256 * 32;
    const u32 filled = fill && values && (a.masks || (ranges && !changes)) ? (a.cols + fill_width - 1) / fill_width : 0;
    const int table = !by_parts && (changes || a.grad_entry) ? 1 : 0, bits = table && changes ? hash_bits(n) : 0;
    hipError_t e = hipSuccess;
    if (filled + table) e = wide ? launch_over<KIND, BACK, 1024>(a, filled, table, bits, fill, st, sums) : launch_over<KIND, BACK, 256>(a, filled, table, bits, fill, st, sums);
    else if (sums.out) hipLaunchKernelGGL(k_adjust_join, grid_of(join_groups(sums)), dim3(256), 0, st, sums);
    if (e != hipSuccess || !by_parts) return e != hipSuccess ? e : hipGetLastError();
    return a.n_prior <= 4 * kKept * 1024 ? launch_over_parts<KIND, BACK, true>(a, eights > 512 ? 16384 : 8192, fill && !filled, st)
                                         : launch_over_parts<KIND, BACK, false>(a, eights > 512 ? 16384 : 8192, fill && !filled, st);
}

template <int KIND> hipError_t launch_forward(const AdjustArgs& a, hipStream_t st) {
    return a.out == a.scores && !a.bias ? launch_over<KIND, false>(a, true, st) : launch_all<KIND, false>(a, st);
}

template <int KIND, bool OVER> bool launch_columns(const AdjustArgs& a, u32 rows, u32 blocks, void* scratch, float* direct, hipStream_t st) {
    const u32 tile = kSumThreads / kSumGroups * kPer<KIND>, tiles = (a.cols + tile - 1) / tile;
    if ((u64)tiles * blocks >> 32) return false;
    hipLaunchKernelGGL((k_adjust_columns<KIND, OVER>), grid_of((u64)tiles * blocks), dim3(kSumThreads), 0, st, a, tiles, rows, (double*)scratch, direct);
    return true;
}

template <int KIND> hipError_t launch_back(const AdjustArgs& a, void* scratch, hipStream_t st) {
    const bool over = a.grad == a.grad_out;
    if (!a.grad_bias) return over || !a.grad ? launch_over<KIND, true>(a, true, st) : launch_all<KIND, true>(a, st);
    const u32 rows = sum_rows(a.rows), blocks = (u32)((a.rows + rows - 1) / rows);
    float* direct = blocks == 1 ? a.grad_bias : nullptr;
    if (blocks) {
        const bool ok = over ? launch_columns<KIND, true>(a, rows, blocks, scratch, direct, st) : launch_columns<KIND, false>(a, rows, blocks, scratch, direct, st);
        if (!ok) return hipErrorInvalidValue;
    }
    const Join sums{(const double*)scratch, blocks, a.cols, direct ? nullptr : a.grad_bias};
    if (blocks && ((a.n_prior && a.repetition && a.grad) || a.grad_entry)) return launch_over<KIND, true>(a, false, st, sums);
    if (!direct) hipLaunchKernelGGL(k_adjust_join, grid_of(join_groups(sums)), dim3(256), 0, st, sums);
    return hipGetLastError();
}

}  // namespace

size_t adjust_grad_scratch_bytes(int64_t rows, int64_t cols) {
    const int64_t block = sum_rows(rows), blocks = (rows + block - 1) / block;
    return blocks > 1 ? (size_t)blocks * (size_t)cols * 8 : 0;
}

hipError_t launch_adjust(int kind, const AdjustArgs& a, hipStream_t st) {
    switch (kind) {
        case kScoreF32: return launch_forward<kScoreF32>(a, st);
        case kScoreF16: return launch_forward<kScoreF16>(a, st);
        case kScoreBF16: return launch_forward<kScoreBF16>(a, st);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_adjust_grad(int kind, const AdjustArgs& a, void* scratch, hipStream_t st) {
    switch (kind) {
        case kScoreF32: return launch_back<kScoreF32>(a, scratch, st);
        case kScoreF16: return launch_back<kScoreF16>(a, scratch, st);
        case kScoreBF16: return launch_back<kScoreBF16>(a, scratch, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace qsv
