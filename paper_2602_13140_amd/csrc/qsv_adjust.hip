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
// Places with a word are worked out in 64 bits and rounded to 32 and to the type; the others, a score plus a shared bias, in 32.
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
    double by, inverse, each, once;     // R, 1 / R, F, A
    int len, prompt;
    const u32* mask;                    // NULL: all are allowed
    bool good;                          // its parameters are in their ranges
};

__device__ __forceinline__ Row row_of(const AdjustArgs& a, u64 r) {
    Row f;
    const float by = a.repetition ? a.repetition[r] : 1.f, each = a.frequency ? a.frequency[r] : 0.f, once = a.presence ? a.presence[r] : 0.f;
    f.len = a.n_prior;
    f.prompt = 0;
    if (a.n_prior) {
        if (a.prior_len) f.len = a.prior_len[r];
        if (a.prompt_len) f.prompt = a.prompt_len[r];
    }
    f.good = by > 0.f && by < kInf && fabsf(each) < kInf && fabsf(once) < kInf && f.prompt >= 0 && f.prompt <= f.len && f.len <= a.n_prior;
    f.by = (double)by;
    f.inverse = 1.0 / f.by;
    f.each = (double)each;
    f.once = (double)once;
    f.mask = nullptr;
    if (a.masks) {
        const int64_t at = a.mask_of ? (int64_t)a.mask_of[r] : a.mask_each ? (int64_t)r : 0;
        if (at < -1 || at >= a.n_masks) f.good = false;
        else if (at >= 0) f.mask = a.masks + (u64)at * (u64)a.mask_stride;
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
inline size_t part_bytes(int n_entries, u32 width) { return (size_t)entry_room(n_entries) * 16 + (size_t)width * 4 + width / 8 + 16; }

__device__ __forceinline__ void mark(const Part& p, u32 k) { atomicOr(&p.bits[k / 32], 1u << (k & 31)); }

// 16 of the row's earlier outcomes a thread: four at a time from place i on, -1 behind the last.
typedef int four __attribute__((ext_vector_type(4)));
typedef int four_at4 __attribute__((ext_vector_type(4), aligned(4)));
template <int NT> __device__ __forceinline__ void prior_load(const int* prior, int len, int i0, four (&t)[4]) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int i = i0 + (u * NT + (int)threadIdx.x) * 4;
        t[u] = four{-1, -1, -1, -1};
        if (i + 4 <= len) {
            t[u] = *(const four_at4*)(prior + i);
        } else {
            if (i < len) t[u][0] = prior[i];
            if (i + 1 < len) t[u][1] = prior[i + 1];
            if (i + 2 < len) t[u][2] = prior[i + 2];
        }
    }
}
template <int NT> __device__ __forceinline__ void prior_count(const Row& f, const Part& p, u32 c0, u32 n, int i0, const four (&t)[4]) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const u32 k = (u32)t[u][w] - c0;
            if (k >= n) continue;
            if (i0 + (u * NT + (int)threadIdx.x) * 4 + w < f.prompt) atomicOr(&p.word[k], kPrompt);
            else atomicAdd(&p.word[k], 1u);
            mark(p, k);
        }
}

// The part's entries in their order, gathered by the first wavefront.
__device__ __forceinline__ void gather_entries(const AdjustArgs& a, u64 r, const Part& p, u32 c0, u32 n) {
    const u32 lane = threadIdx.x;
    const int* idx = a.entry_idx + r * (u64)a.n_entries;
    const float* bias = a.entry_bias + r * (u64)a.n_entries;
    u32 m = 0;
    for (int j0 = 0; j0 < a.n_entries; j0 += 256) {
        u32 k[4];
        float b[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = j0 + u * 64 + (int)lane;
            k[u] = j < a.n_entries ? (u32)idx[j] - c0 : ~0u;
            b[u] = j < a.n_entries ? bias[j] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const u64 in = __ballot(k[u] < n);
            const u32 at = m + __popcll(in & ((1ull << lane) - 1));
            if (k[u] < n) { p.column[at] = (int)k[u]; p.bias[at] = b[u]; }
            m += (u32)__popcll(in);
        }
    }
    if (lane < ((m + 3) & ~3u) - m) p.column[m + lane] = -1;
    if (lane == 0) *p.entries = m;
}

// A column's entries by the thread of the first of them.
template <int NT> __device__ __forceinline__ void add_entries(const Part& p) {
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
        atomicOr(&p.word[k], (j + 1) << kEntryBit);
        mark(p, (u32)k);
    }
}

// The table of the part's n columns.  between: what is to be under way meanwhile.
template <int NT, bool ENTRIES, class F> __device__ __forceinline__ void fill_part(const AdjustArgs& a, u64 r, const Row& f, const Part& p, u32 c0, u32 n, u32 width, F&& between) {
    const int* prior = a.prior + r * (u64)a.prior_stride;
    four t[4];
    prior_load<NT>(prior, f.len, 0, t);
    between();
    for (u32 i = threadIdx.x; i < (width + width / 32) / 4; i += NT) ((four*)p.word)[i] = four{0, 0, 0, 0};    // bits lie behind the words
    if (ENTRIES && a.n_entries && threadIdx.x < 64) gather_entries(a, r, p, c0, n);
    __syncthreads();
    prior_count<NT>(f, p, c0, n, 0, t);
    for (int i0 = 16 * NT; i0 < f.len; i0 += 16 * NT) {
        prior_load<NT>(prior, f.len, i0, t);
        prior_count<NT>(f, p, c0, n, i0, t);
    }
    if (ENTRIES && a.n_entries) add_entries<NT>(p);
    __syncthreads();
}

__device__ __forceinline__ bool seen(u32 word) { return (word & (kPrompt | kCount)) != 0; }

// A place whose column has a word.
__device__ __forceinline__ float adjusted(const Row& f, const Part& p, u32 word, float z, float bias) {
    double v = (double)z;
    if (seen(word)) {
        v *= v > 0.0 ? f.inverse : f.by;
        const u32 c = word & kCount;
        if (c) v -= f.each * (double)c + f.once;
    }
    v += (double)bias;
    const u32 e = (word >> kEntryBit) & kEntryMost;
    if (e) v += p.sum[e - 1];
    return (float)v;
}

// ... and its gradient.
__device__ __forceinline__ float taken_back(const Row& f, u32 word, float z, float g) {
    return seen(word) ? (float)((double)g * (z > 0.f ? f.inverse : f.by)) : g;
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

// Columns c0 .. c0 + NT NV W - 1 of row r, all of them written.  BACK: the gradient.  A thread's vectors of the row are under way
// while the table is filled.
template <int KIND, bool BACK, int NT, int NV, bool TABLE> __global__ __launch_bounds__(NT) void k_adjust(const AdjustArgs a, const u32 parts) {
    constexpr u32 W = kPer<KIND>, width = NT * NV * W;
    extern __shared__ __align__(16) char lds[];
    const u64 r = grid_block() / parts;
    const u32 c0 = (u32)(grid_block() % parts) * width;
    if (r >= (u64)a.rows) return;
    const Row f = row_of(a, r);
    const u32 n = min(width, a.cols - c0), whole = n / W;
    const char* scores = (const char*)a.scores + (a.scores ? r * (u64)a.stride * kSize<KIND> : 0);
    const char* in = BACK ? (const char*)a.grad_out + r * (u64)a.grad_out_stride * kSize<KIND> : scores;
    char* out = BACK ? (char*)a.grad + r * (u64)a.grad_stride * kSize<KIND> : (char*)a.out + r * (u64)a.out_stride * kSize<KIND>;
    const Part p = part_of(lds, BACK ? 0 : a.n_entries, width);
    const float none = BACK ? 0.f : -kInf;
    if (BACK && a.grad_entry) entry_gradients<KIND, NT>(a, r, f, in, c0, c0 + n);
    if (!f.good) {
        for (u32 k = c0 + threadIdx.x; k < c0 + n; k += NT) store_one<KIND>(out, k, __builtin_nanf(""));
        return;
    }
    vec x[NV];
    u32 allowed[NV];
    auto load = [&]() {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const u32 j = v * NT + threadIdx.x, k = c0 + j * W;
            if (j < whole) x[v] = vec_at<KIND>(in + (u64)k * kSize<KIND>);
            allowed[v] = f.mask && j < whole ? vector_bits<KIND>(f.mask, k) : kBits<KIND>;
        }
    };
    if (TABLE) fill_part<NT, !BACK>(a, r, f, p, c0, n, width, load);
    else load();
    auto place = [&](u32 k, float z) {              // a column that has a word
        const u32 word = p.word[k - c0];
        return BACK ? taken_back(f, word, value_at<KIND>(scores, k), z) : adjusted(f, p, word, z, a.bias ? a.bias[k] : 0.f);
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const u32 j = v * NT + threadIdx.x, k = c0 + j * W;
        if (j >= whole) continue;
        float y[W];
        float b[W] = {};
        if (!BACK && a.bias) {
#pragma unroll
            for (u32 i = 0; i < W; i += 4) {
                const vec q = *(const vec_at4*)(a.bias + k + i);
#pragma unroll
                for (u32 u = 0; u < 4; ++u) b[i + u] = __uint_as_float(q[u]);
            }
        }
#pragma unroll
        for (u32 i = 0; i < W; ++i) y[i] = !BACK && a.bias ? part<KIND>(x[v], i) + b[i] : part<KIND>(x[v], i);
        if (TABLE) {
            const u32 hit = vector_bits<KIND>(p.bits, k - c0);
            if (hit) {
                // the results take the words' places, from where every column is fetched: registers know no index
                for (u32 left = hit; left; left &= left - 1) {
                    const u32 i = __builtin_ctz(left);
                    p.word[k - c0 + i] = __float_as_uint(place(k + i, value_at<KIND>(in, k + i)));
                }
                u32 got[W];
#pragma unroll
                for (u32 i = 0; i < W; i += 4) {
                    const four q = *(const four*)(p.word + (k - c0) + i);
#pragma unroll
                    for (u32 u = 0; u < 4; ++u) got[i + u] = (u32)q[u];
                }
#pragma unroll
                for (u32 i = 0; i < W; ++i)
                    if (hit >> i & 1) y[i] = __uint_as_float(got[i]);
            }
        }
#pragma unroll
        for (u32 i = 0; i < W; ++i)
            if (!(allowed[v] >> i & 1)) y[i] = none;
        put_vec<KIND, false>(out + (u64)k * kSize<KIND>, packed<KIND>(y));
    }
    const u32 k = c0 + whole * W + threadIdx.x;
    if (k < c0 + n) {
        const float z = value_at<KIND>(in, k);
        float y = !BACK && a.bias ? z + a.bias[k] : z;
        if (TABLE && p.word[k - c0]) y = place(k, z);
        store_one<KIND>(out, k, allowed_at(f.mask, k) & 1 ? y : none);
    }
}

// The same over the scores (BACK: over the gradient): only the places that change.  fill: the masked ones too.
template <int KIND, bool BACK, int NT> __global__ __launch_bounds__(NT) void k_adjust_over(const AdjustArgs a, const u32 parts, const u32 width, const int table, const int fill) {
    extern __shared__ __align__(16) char lds[];
    const u64 r = grid_block() / parts;
    const u32 c0 = (u32)(grid_block() % parts) * width;
    if (r >= (u64)a.rows) return;
    const Row f = row_of(a, r);
    const u32 c1 = c0 + min(width, a.cols - c0);
    const char* scores = (const char*)a.scores + (a.scores ? r * (u64)a.stride * kSize<KIND> : 0);
    char* out = BACK ? (char*)a.grad + (a.grad ? r * (u64)a.grad_stride * kSize<KIND> : 0) : (char*)a.out + r * (u64)a.out_stride * kSize<KIND>;
    const Part p = part_of(lds, BACK ? 0 : a.n_entries, width);
    const float none = BACK ? 0.f : -kInf;
    if (BACK && a.grad_entry) {
        entry_gradients<KIND, NT>(a, r, f, (const char*)a.grad_out + r * (u64)a.grad_out_stride * kSize<KIND>, c0, c1);
        __syncthreads();       // read before the places are written
    }
    if (BACK && !a.grad) return;
    if (!f.good) {
        if (fill)
            for (u32 k = c0 + threadIdx.x; k < c1; k += NT) store_one<KIND>(out, k, __builtin_nanf(""));
        return;
    }
    if (table) {
        fill_part<NT, !BACK>(a, r, f, p, c0, c1 - c0, width, [] {});
        for (u32 k = c0 + threadIdx.x; k < c1; k += NT) {
            const u32 word = p.word[k - c0];
            if (!word || !(allowed_at(f.mask, k) & 1)) continue;
            const float x = value_at<KIND>(out, k);
            store_one<KIND>(out, k, BACK ? taken_back(f, word, value_at<KIND>(scores, k), x) : adjusted(f, p, word, x, 0.f));
        }
    }
    if (!f.mask || !fill) return;
    // 64 words of the mask a wavefront: a store for 64 columns, by those lanes whose column is masked
    const u32 lane = threadIdx.x & 63;
    for (u32 k0 = c0 + (threadIdx.x >> 6) * 2048; k0 < c1; k0 += NT * 32) {
        const u32 at = k0 / 32 + lane, word = at * 32 < c1 ? f.mask[at] : ~0u;
#pragma unroll 4
        for (u32 i = 0; i < 32; ++i) {
            const u64 on = (u64)lane_of(word, 2 * i + 1) << 32 | lane_of(word, 2 * i);
            const u32 k = k0 + i * 64 + lane;
            if (!(on >> lane & 1) && k < c1) store_one<KIND>(out, k, none);
        }
    }
}

// ---- a bias that all rows share --------------------------------------------------------------------------------------
// Sums over a block of rows of a tile of columns, a vector of them a thread; the gradient of the scores on the way (grad, or NULL).
// OVER: it lies over grad_out, and vectors without a masked place are left.  Sums are in 64 bits: they cost the kernel nothing.
constexpr int kSumThreads = 256, kMostSumRows = 256;

template <int KIND, bool OVER> __global__ __launch_bounds__(kSumThreads) void k_adjust_columns(const AdjustArgs a, const u32 tiles, const u32 block_rows, double* sums, float* out_sums) {
    constexpr u32 W = kPer<KIND>;
    constexpr int N = 4;                    // rows under way
    __shared__ const u32* masks[kMostSumRows];
    __shared__ int good[kMostSumRows];
    const u64 b = grid_block() / tiles;
    const u32 k = (u32)(grid_block() % tiles) * (kSumThreads * W) + threadIdx.x * W;
    if (b * block_rows >= (u64)a.rows) return;
    const u64 r0 = b * block_rows;
    const u32 rows = (u32)min((u64)block_rows, (u64)a.rows - r0);
    if (threadIdx.x < rows) {
        const Row f = row_of(a, r0 + threadIdx.x);
        masks[threadIdx.x] = f.mask;
        good[threadIdx.x] = f.good;
    }
    __syncthreads();
    if (k >= a.cols) return;
    const u32 n = min(W, a.cols - k);
    const char* in = (const char*)a.grad_out + (r0 * (u64)a.grad_out_stride + k) * kSize<KIND>;
    char* out = (char*)a.grad + (a.grad ? (r0 * (u64)a.grad_stride + k) * kSize<KIND> : 0);
    double sum[W] = {};
    auto some = [&](u32 i0, u32 count) {
        vec x[N];
        u32 allowed[N];
#pragma unroll
        for (u32 u = 0; u < (u32)N; ++u) {
            if (u >= count) continue;
            const char* p = in + (u64)(i0 + u) * (u64)a.grad_out_stride * kSize<KIND>;
            if (n == W) {
                x[u] = vec_at<KIND>(p);
            } else {
                float v[W] = {};
#pragma unroll
                for (u32 i = 0; i < W; ++i)
                    if (i < n) v[i] = value_at<KIND>(p, i);
                x[u] = packed<KIND>(v);
            }
            const u32* mask = masks[i0 + u];
            allowed[u] = mask ? vector_bits<KIND>(mask, k) : kBits<KIND>;
        }
#pragma unroll
        for (u32 u = 0; u < (u32)N; ++u) {
            if (u >= count) continue;
            const bool ok = good[i0 + u];
            float v[W];
#pragma unroll
            for (u32 i = 0; i < W; ++i) {
                v[i] = !ok ? __builtin_nanf("") : allowed[u] >> i & 1 ? part<KIND>(x[u], i) : 0.f;
                sum[i] += (double)v[i];
            }
            if (!a.grad || (OVER && ok && allowed[u] == kBits<KIND>)) continue;
            char* p = out + (u64)(i0 + u) * (u64)a.grad_stride * kSize<KIND>;
            if (n == W) {
                put_vec<KIND, false>(p, packed<KIND>(v));
            } else {
#pragma unroll
                for (u32 i = 0; i < W; ++i)
                    if (i < n) store_one<KIND>(p, i, v[i]);
            }
        }
    };
    u32 i = 0;
    for (; i + N <= rows; i += N) some(i, N);
    if (i < rows) some(i, rows - i);
#pragma unroll
    for (u32 i = 0; i < W; ++i)
        if (i < n) {
            if (out_sums) out_sums[k + i] = (float)sum[i];
            else sums[b * a.cols + k + i] = sum[i];
        }
}

__global__ __launch_bounds__(256) void k_adjust_join(const double* sums, const u32 blocks, const u32 cols, float* out) {
    const u64 k = grid_block() * 256 + threadIdx.x;
    if (k >= cols) return;
    double v = 0.0;
#pragma unroll 8
    for (u32 b = 0; b < blocks; ++b) v += sums[(u64)b * cols + k];
    out[k] = (float)v;
}

// Rows of a block: as many as leave some thousand workgroups.
u32 sum_rows(int64_t rows, int64_t cols) {
    const int64_t tiles = (cols + 2047) / 2048, want = rows * tiles / 1024;
    return (u32)std::max((int64_t)16, std::min((int64_t)kMostSumRows, want));
}

// ---- launches --------------------------------------------------------------------------------------------------------
template <int KIND, bool BACK, int NT, int NV> hipError_t launch_all(const AdjustArgs& a, bool table, hipStream_t st) {
    constexpr u32 width = NT * NV * kPer<KIND>;
    const u32 parts = (a.cols + width - 1) / width;
    const dim3 grid = grid_of((u64)a.rows * parts), block(NT);
    if (table) hipLaunchKernelGGL((k_adjust<KIND, BACK, NT, NV, true>), grid, block, part_bytes(BACK ? 0 : a.n_entries, width), st, a, parts);
    else hipLaunchKernelGGL((k_adjust<KIND, BACK, NT, NV, false>), grid, block, 0, st, a, parts);
    return hipGetLastError();
}

template <int KIND, bool BACK> hipError_t launch_all(const AdjustArgs& a, hipStream_t st) {
    const bool table = BACK ? a.n_prior && a.repetition : a.n_prior || a.n_entries;
    const u32 width = 256 * 4 * kPer<KIND>;
    if (table && a.n_prior > 4096) return launch_all<KIND, BACK, 1024, 1>(a, table, st);
    if ((u64)a.rows * ((a.cols + width - 1) / width) < 512) return launch_all<KIND, BACK, 256, 1>(a, table, st);
    return launch_all<KIND, BACK, 256, 4>(a, table, st);
}

template <int KIND, bool BACK> hipError_t launch_over(const AdjustArgs& a, int fill, hipStream_t st) {
    const int table = a.grad || !BACK ? (BACK ? a.n_prior && a.repetition : a.n_prior || a.n_entries) : 0;
    const u32 width = 8192, parts = (a.cols + width - 1) / width;
    const size_t lds = table ? part_bytes(BACK ? 0 : a.n_entries, width) : 0;
    if (table && a.n_prior > 4096) hipLaunchKernelGGL((k_adjust_over<KIND, BACK, 1024>), grid_of((u64)a.rows * parts), dim3(1024), lds, st, a, parts, width, table, fill);
    else hipLaunchKernelGGL((k_adjust_over<KIND, BACK, 256>), grid_of((u64)a.rows * parts), dim3(256), lds, st, a, parts, width, table, fill);
    return hipGetLastError();
}

template <int KIND> hipError_t launch_forward(const AdjustArgs& a, hipStream_t st) {
    return a.out == a.scores && !a.bias ? launch_over<KIND, false>(a, 1, st) : launch_all<KIND, false>(a, st);
}

template <int KIND> hipError_t launch_back(const AdjustArgs& a, void* scratch, hipStream_t st) {
    const bool over = a.grad == a.grad_out;
    if (!a.grad_bias) return over || !a.grad ? launch_over<KIND, true>(a, 1, st) : launch_all<KIND, true>(a, st);
    const u32 tile = kSumThreads * kPer<KIND>, tiles = (a.cols + tile - 1) / tile, rows = sum_rows(a.rows, a.cols), blocks = (u32)((a.rows + rows - 1) / rows);
    float* direct = blocks == 1 ? a.grad_bias : nullptr;
    if (blocks) {
        const dim3 grid = grid_of((u64)tiles * blocks);
        if (over) hipLaunchKernelGGL((k_adjust_columns<KIND, true>), grid, dim3(kSumThreads), 0, st, a, tiles, rows, (double*)scratch, direct);
        else hipLaunchKernelGGL((k_adjust_columns<KIND, false>), grid, dim3(kSumThreads), 0, st, a, tiles, rows, (double*)scratch, direct);
    }
    if (!direct) hipLaunchKernelGGL(k_adjust_join, grid_of(((u64)a.cols + 255) / 256), dim3(256), 0, st, (const double*)scratch, blocks, a.cols, a.grad_bias);
    if (blocks && ((a.n_prior && a.repetition && a.grad) || a.grad_entry)) return launch_over<KIND, true>(a, 0, st);
    return hipGetLastError();
}

}  // namespace

size_t adjust_grad_scratch_bytes(int64_t rows, int64_t cols) {
    const int64_t block = sum_rows(rows, cols), blocks = (rows + block - 1) / block;
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
