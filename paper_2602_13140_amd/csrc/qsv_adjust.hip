// Penalties for repeated outcomes, biases and masks on rows of scores, and the backward pass of it.
//
//   v = z;  s_k: v = v > 0 ? v / R : v R;  v -= F c_k + A [c_k > 0];  v += b_k + sum_{j: i_j = k} e_j;  masked: v = -inf
//   s_k: outcome k is among the row's earlier ones, c_k: how often behind its prompt
//
// Bound by memory, or over the scores themselves by latency: only the places that change are written then.  A workgroup takes
// a part of a row's columns.  It counts the row's earlier outcomes that lie in its part in a table in LDS, a word a column:
//   bit 31 in the prompt | bits 21-30 one more than the first entry (of the row's own biases) that names it | bits 0-20 c_k
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
    double by, each, once;     // R, F, A
    int len, prompt;
    const u32* mask;           // NULL: all are allowed
    bool good;                 // its parameters are in their ranges
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

// The part's table in LDS: nothing of it is there where the row can have neither history nor entries.
struct Part {
    double* sum;       // by entry: of all entries of its column, at the first of them
    u32* word;         // by column
    u32* bits;
    int* idx;          // by entry: its column in the part, or -1
};

__host__ __device__ inline int entry_room(int n) { return (n + 3) & ~3; }
inline size_t part_bytes(const AdjustArgs& a, u32 width) {
    return a.n_prior || a.n_entries ? (size_t)entry_room(a.n_entries) * 12 + (size_t)width * 4 + width / 8 : 0;
}
__device__ __forceinline__ Part part_of(char* lds, int n_entries, u32 width) {
    Part p;
    const int room = entry_room(n_entries);
    p.sum = (double*)lds;
    p.word = (u32*)(p.sum + room);
    p.bits = p.word + width;
    p.idx = (int*)(p.bits + width / 32);
    return p;
}

template <int NT> __device__ __forceinline__ void fill_part(const AdjustArgs& a, u64 r, const Row& f, const Part& p, u32 c0, u32 width) {
    typedef u32 four __attribute__((ext_vector_type(4)));
    for (u32 i = threadIdx.x; i < (width + width / 32) / 4; i += NT) ((four*)p.word)[i] = four{0, 0, 0, 0};    // bits lie behind the words
    if (a.n_entries) {
        const int* idx = a.entry_idx + r * (u64)a.n_entries;
        for (int j = threadIdx.x; j < entry_room(a.n_entries); j += NT) {
            const u32 k = j < a.n_entries ? (u32)idx[j] : ~0u;
            p.idx[j] = k < a.cols && k - c0 < width ? (int)(k - c0) : -1;
        }
    }
    __syncthreads();
    const int* prior = a.prior + r * (u64)a.prior_stride;
    for (int i = threadIdx.x; i < f.len; i += NT) {
        const u32 k = (u32)prior[i];
        if (k >= a.cols || k - c0 >= width) continue;
        if (i < f.prompt) atomicOr(&p.word[k - c0], kPrompt);
        else atomicAdd(&p.word[k - c0], 1u);
        atomicOr(&p.bits[(k - c0) / 32], 1u << (k & 31));
    }
    for (int j = threadIdx.x; j < a.n_entries; j += NT) {
        const int k = p.idx[j];
        if (k < 0) continue;
        bool first = true;
        double sum = 0.0;
        for (int i = 0; i < a.n_entries; ++i)
            if (p.idx[i] == k) {
                if (i < j) { first = false; break; }
                if (a.entry_bias) sum += (double)a.entry_bias[r * (u64)a.n_entries + i];
            }
        if (!first) continue;
        p.sum[j] = sum;
        atomicOr(&p.word[k], (u32)(j + 1) << kEntryBit);
        atomicOr(&p.bits[k / 32], 1u << (k & 31));
    }
    __syncthreads();
}

__device__ __forceinline__ bool seen(u32 word) { return (word & (kPrompt | kCount)) != 0; }

// A place whose column has a word.
__device__ __forceinline__ float adjusted(const Row& f, const Part& p, u32 word, float z, float bias) {
    double v = (double)z;
    if (seen(word)) {
        v = v > 0.0 ? v / f.by : v * f.by;
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
    if (!seen(word)) return g;
    return (float)(z > 0.f ? (double)g / f.by : (double)g * f.by);
}

__device__ __forceinline__ u32 allowed_at(const u32* mask, u32 k) { return mask ? mask[k >> 5] >> (k & 31) : ~0u; }

// Columns c0 .. c0 + width - 1 of row r.  BACK: the gradient.  OVER: out is the source, only the places that change are written.
// fill: (OVER) the masked places too.
template <int KIND, bool BACK, bool OVER, int NT> __global__ __launch_bounds__(NT) void k_adjust(const AdjustArgs a, const u32 width, const u32 parts, const int fill) {
    constexpr int W = kPer<KIND>;
    extern __shared__ char lds[];
    const u64 r = grid_block() / parts;
    const u32 c0 = (u32)(grid_block() % parts) * width;
    if (r >= (u64)a.rows) return;
    const Row f = row_of(a, r);
    const u32 c1 = a.cols - c0 < width ? a.cols : c0 + width;
    const char* scores = (const char*)a.scores + (a.scores ? r * (u64)a.stride * kSize<KIND> : 0);
    const char* in = BACK ? (const char*)a.grad_out + r * (u64)a.grad_out_stride * kSize<KIND> : scores;
    char* out = BACK ? (char*)a.grad + (a.grad ? r * (u64)a.grad_stride * kSize<KIND> : 0) : (char*)a.out + r * (u64)a.out_stride * kSize<KIND>;
    const bool table = a.n_prior || a.n_entries;
    const Part p = part_of(lds, a.n_entries, width);
    const float none = BACK ? 0.f : -kInf, nan = __builtin_nanf("");
    if (f.good && table) fill_part<NT>(a, r, f, p, c0, width);
    if (BACK && a.grad_entry) {
        const int* idx = a.entry_idx + r * (u64)a.n_entries;
        for (int j = threadIdx.x; j < a.n_entries; j += NT) {
            const u32 k = (u32)idx[j];
            float* to = a.grad_entry + r * (u64)a.n_entries + j;
            if (!f.good) { if (c0 == 0) *to = nan; }
            else if (k >= a.cols) { if (c0 == 0) *to = 0.f; }
            else if (k >= c0 && k < c1) *to = allowed_at(f.mask, k) & 1 ? value_at<KIND>(in, k) : 0.f;
        }
        if (OVER) __syncthreads();       // read before the places are written
    }
    if (BACK && !a.grad) return;
    if (!f.good) {
        if (!OVER || fill)
            for (u32 k = c0 + threadIdx.x; k < c1; k += NT) store_one<KIND>(out, k, nan);
        return;
    }
    if (OVER) {
        if (table)
            for (u32 k = c0 + threadIdx.x; k < c1; k += NT) {
                const u32 word = p.word[k - c0];
                if (!word || !(allowed_at(f.mask, k) & 1)) continue;
                const float x = value_at<KIND>(out, k);
                if (!BACK) store_one<KIND>(out, k, adjusted(f, p, word, x, 0.f));
                else if (seen(word) && f.by != 1.0) store_one<KIND>(out, k, taken_back(f, word, value_at<KIND>(scores, k), x));
            }
        if (f.mask && fill)
            for (u32 k = c0 + threadIdx.x; k < c1; k += NT)
                if (!(allowed_at(f.mask, k) & 1)) store_one<KIND>(out, k, none);
        return;
    }
    auto value = [&](u32 k, float x) {
        float v = x;
        const u32 word = table ? p.word[k - c0] : 0;
        if (!BACK) {
            const float b = a.bias ? a.bias[k] : 0.f;
            v = word ? adjusted(f, p, word, x, b) : a.bias ? x + b : x;
        } else if (word && f.by != 1.0) {
            v = taken_back(f, word, value_at<KIND>(scores, k), x);
        }
        return allowed_at(f.mask, k) & 1 ? v : none;
    };
    const u32 whole = (c1 - c0) / W;
    for (u32 j = threadIdx.x; j < whole; j += NT) {
        const u32 k = c0 + j * W;
        const vec x = vec_at<KIND>(in + (u64)k * kSize<KIND>);
        float v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = value(k + i, part<KIND>(x, i));
        put_vec<KIND, false>(out + (u64)k * kSize<KIND>, packed<KIND>(v));
    }
    const u32 k = c0 + whole * W + threadIdx.x;
    if (k < c1) store_one<KIND>(out, k, value(k, value_at<KIND>(in, k)));
}

// ---- a bias that all rows share --------------------------------------------------------------------------------------
// Sums over rows r0 .. of a tile of columns, a vector of them a thread, in 32 bits over kSumRows rows at most; the gradient of the
// scores on the way (grad, or NULL).  OVER: it lies over grad_out.
constexpr int kSumRows = 256, kSumThreads = 256;

template <int KIND, bool OVER> __global__ __launch_bounds__(kSumThreads) void k_adjust_columns(const AdjustArgs a, const u32 tiles, float* sums) {
    constexpr int W = kPer<KIND>;
    const u64 b = grid_block() / tiles;
    const u32 k = (u32)(grid_block() % tiles) * (kSumThreads * W) + threadIdx.x * W;
    if (b * kSumRows >= (u64)a.rows || k >= a.cols) return;
    const u64 r1 = min((u64)a.rows, (b + 1) * kSumRows);
    const int n = (int)min((u32)W, a.cols - k);
    float sum[W] = {};
    for (u64 r = b * kSumRows; r < r1; ++r) {
        const Row f = row_of(a, r);
        const char* in = (const char*)a.grad_out + r * (u64)a.grad_out_stride * kSize<KIND>;
        char* out = (char*)a.grad + (a.grad ? r * (u64)a.grad_stride * kSize<KIND> : 0);
        const u32 allowed = allowed_at(f.mask, k);
        float v[W];
        if (n == W) {
            const vec x = vec_at<KIND>(in + (u64)k * kSize<KIND>);
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = part<KIND>(x, i);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = i < n ? value_at<KIND>(in, k + i) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if (!f.good) v[i] = __builtin_nanf("");
            else if (!(allowed >> i & 1)) v[i] = 0.f;
            sum[i] += v[i];
        }
        if (!a.grad) continue;
        if (n == W) {
            put_vec<KIND, false>(out + (u64)k * kSize<KIND>, packed<KIND>(v));
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (i < n) store_one<KIND>(out, k + i, v[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < W; ++i)
        if (i < n) sums[b * a.cols + k + i] = sum[i];
}

__global__ __launch_bounds__(256) void k_adjust_join(const float* sums, const u32 blocks, const u32 cols, float* out) {
    const u64 k = grid_block() * 256 + threadIdx.x;
    if (k >= cols) return;
    double v = 0.0;
    for (u32 b = 0; b < blocks; ++b) v += (double)sums[(u64)b * cols + k];
    out[k] = (float)v;
}

// ---- launches --------------------------------------------------------------------------------------------------------
template <int KIND, bool BACK, bool OVER> hipError_t launch_parts(const AdjustArgs& a, int fill, hipStream_t st) {
    const u32 width = 8192, parts = (a.cols + width - 1) / width;
    hipLaunchKernelGGL((k_adjust<KIND, BACK, OVER, 256>), grid_of((u64)a.rows * parts), dim3(256), part_bytes(a, width), st, a, width, parts, fill);
    return hipGetLastError();
}

template <int KIND> hipError_t launch_forward(const AdjustArgs& a, hipStream_t st) {
    return a.out == a.scores && !a.bias ? launch_parts<KIND, false, true>(a, 1, st) : launch_parts<KIND, false, false>(a, 1, st);
}

template <int KIND> hipError_t launch_back(const AdjustArgs& a, void* scratch, hipStream_t st) {
    const bool over = a.grad == a.grad_out;
    if (!a.grad_bias) return over || !a.grad ? launch_parts<KIND, true, true>(a, 1, st) : launch_parts<KIND, true, false>(a, 1, st);
    const u32 tile = kSumThreads * kPer<KIND>, tiles = (a.cols + tile - 1) / tile, blocks = (u32)((a.rows + kSumRows - 1) / kSumRows);
    if (!blocks) {}
    else if (over) hipLaunchKernelGGL((k_adjust_columns<KIND, true>), grid_of((u64)tiles * blocks), dim3(kSumThreads), 0, st, a, tiles, (float*)scratch);
    else hipLaunchKernelGGL((k_adjust_columns<KIND, false>), grid_of((u64)tiles * blocks), dim3(kSumThreads), 0, st, a, tiles, (float*)scratch);
    hipLaunchKernelGGL(k_adjust_join, grid_of(((u64)a.cols + 255) / 256), dim3(256), 0, st, (const float*)scratch, blocks, a.cols, a.grad_bias);
    if (blocks && ((a.n_prior && a.repetition && a.grad) || a.grad_entry)) return launch_parts<KIND, true, true>(a, 0, st);
    return hipGetLastError();
}

}  // namespace

size_t adjust_grad_scratch_bytes(int64_t rows, int64_t cols) { return (size_t)((rows + kSumRows - 1) / kSumRows) * (size_t)cols * 4; }

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
