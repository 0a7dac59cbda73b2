// The norm of many tensors' gradients together, gradients scaled to a highest norm, and Adam's step with that on the way.
//
//   N = sqrt(sum g^2),  f = N > M ? M / N : 1;  out = f g
//   m = b1 m + (1 - b1) f g,  v = b2 v + (1 - b2) (f g)^2,  p -= lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// Bound by memory: every gradient is read for the norm and once more for what is made of it.  Tensors are cut into pieces of
// 256 to 4096 values (whole rows where they are shorter), numbered through a list that comes with the launch's arguments; a
// wavefront takes every so many-th piece, and a workgroup leaves one sum.  The next launch's workgroups each add all of these in
// the same order, so results depend on nothing but the list, and take the pieces from the last to the first, which the first
// launch has read last.  Squares and their sums are in 64 bits, where no float32 value overflows or vanishes.
#include "qsv_rows.h"
#include "qsv_tensors.h"
#include "qsv_wave.h"

#include <cmath>

namespace qsv {
namespace {

typedef unsigned long long u64;
typedef unsigned u32;

constexpr int kThreads = 256;
constexpr u32 kSums = 2048;           // sums of all launches together; rounded up for each of them
constexpr int kKindBit = 56;

// Lists within 4 KiB of arguments: tensors of any rows; rows without a gap, which are one, to be
// summed up and to be scaled; Adam's.  (Fewer launches: 192 tensors' squares by one instead of two, Adam's step of them 552 -> 542 us.)
struct Seg {
    const char* src;
    char* dst;                        // where the scaled gradient goes
    u64 rows, cols;
    u64 src_stride, dst_stride;       // bytes
    u32 row_pieces;                   // pieces of a row; 0: rows_piece rows are a piece
    u32 rows_piece;
    u32 kind;
};
constexpr int kSegs = 58, kSummed = 200, kFlats = 140, kAdams = 90;
struct SegList {
    static constexpr int kRoom = kSegs;
    u32 n, pieces, piece;
    u32 first[kSegs];                 // a tensor's first piece's number
    Seg seg[kSegs];
};
struct SumList {
    static constexpr int kRoom = kSummed;
    u32 n, pieces, piece;
    u32 first[kSummed];
    u64 count[kSummed];               // | kind << kKindBit
    const char* src[kSummed];
};
struct FlatList {
    static constexpr int kRoom = kFlats;
    u32 n, pieces, piece;
    u32 first[kFlats];
    u64 count[kFlats];                // | kind << kKindBit
    const char* src[kFlats];
    char* dst[kFlats];
};
struct AdamList {
    static constexpr int kRoom = kAdams;
    u32 n, pieces, piece;
    u32 first[kAdams];
    u64 count[kAdams];
    float* p[kAdams];
    const char* g[kAdams];
    float* m[kAdams];
    float* v[kAdams];
};
static_assert(sizeof(SegList) <= 4032 && sizeof(SumList) <= 4032 && sizeof(FlatList) <= 4032 && sizeof(AdamList) <= 4032, "a launch's arguments");
constexpr int kMostLists = kMostTensors / kSegs + 1 + kMostTensors / kSummed + 1;  // a call's, of those that are summed up

// The place in the list of a piece's tensor: a lane asks for some of them.
template <class L> struct Places {
    static constexpr int N = (L::kRoom + 63) / 64;
    u32 first[N];
    __device__ __forceinline__ explicit Places(const L& list) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const u32 at = i * 64 + (threadIdx.x & 63);
            first[i] = at < list.n ? list.first[at] : ~0u;
        }
    }
    __device__ __forceinline__ u32 of(u32 piece) const {
        u32 n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += (u32)__popcll(__ballot(first[i] <= piece));
        return uniform(n - 1);
    }
};

// A sum over the workgroup, the same in all threads.
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double sm[16];
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (u32 w = 0; w < blockDim.x / 64; ++w) v += sm[w];
    return v;
}

// n values next to each other, by a wavefront: whole vectors (with the place their results go to), and single values.
template <int KIND, class F> __device__ __forceinline__ void visit(const char* src, char* dst, u32 n, const F& f) {
    constexpr u32 W = kPer<KIND>, N = 4;
    const u32 lane = threadIdx.x & 63, whole = n / W;
    u32 j = lane;
    for (; j - lane + N * 64 <= whole; j += N * 64) {
        vec x[N];
#pragma unroll
        for (u32 i = 0; i < N; ++i) x[i] = vec_at<KIND, F::kPast>(src + (j + i * 64) * 16);
#pragma unroll
        for (u32 i = 0; i < N; ++i) f.whole(x[i], dst + (j + i * 64) * 16);
    }
    for (; j < whole; j += 64) f.whole(vec_at<KIND, F::kPast>(src + j * 16), dst + j * 16);
    const u32 k = whole * W + lane;
    if (k < n) f.one(value_at<KIND>(src, k), dst, k);
}

template <int KIND, class F> __device__ __forceinline__ void visit(const Seg& s, u32 q, u32 piece, const F& f) {
    constexpr u32 W = kPer<KIND>, S = kSize<KIND>;
    if (s.row_pieces) {
        const u64 row = q / s.row_pieces, c0 = (u64)(q % s.row_pieces) * piece;
        visit<KIND>(s.src + row * s.src_stride + c0 * S, s.dst + row * s.dst_stride + c0 * S, (u32)min((u64)piece, s.cols - c0), f);
        return;
    }
    const u64 row = (u64)q * s.rows_piece;
    const u32 lane = threadIdx.x & 63, cols = (u32)s.cols, units = (cols + W - 1) / W, n = (u32)min((u64)s.rows_piece, s.rows - row) * units;
    const u32 dr = 64 / units, du = 64 % units;
    u32 r = lane / units, u = lane % units;
    for (u32 i = lane; i < n; i += 64) {
        const char* src = s.src + (row + r) * s.src_stride;
        char* dst = s.dst + (row + r) * s.dst_stride;
        if (u * W + W <= cols) f.whole(vec_at<KIND, F::kPast>(src + u * 16), dst + u * 16);
        else
            for (u32 k = u * W; k < cols; ++k) f.one(value_at<KIND>(src, k), dst, k);
        r += dr;
        u += du;
        if (u >= units) { u -= units; ++r; }
    }
}

// F<KIND> made by `make` sees every value of a piece.
template <class M> __device__ __forceinline__ void visit(const SegList& l, u32 at, u32 piece, M&& make) {
    const Seg& s = l.seg[at];
    const u32 q = piece - l.first[at];
    if (s.kind == kScoreF32) visit<kScoreF32>(s, q, l.piece, make.template of<kScoreF32>());
    else if (s.kind == kScoreF16) visit<kScoreF16>(s, q, l.piece, make.template of<kScoreF16>());
    else visit<kScoreBF16>(s, q, l.piece, make.template of<kScoreBF16>());
}
template <class L, class M> __device__ __forceinline__ void visit_flat(const L& l, const char* src, char* dst, u32 at, u32 piece, M&& make) {
    const u64 c0 = (u64)(piece - l.first[at]) * l.piece, count = l.count[at];
    const u32 kind = (u32)(count >> kKindBit), n = (u32)min((u64)l.piece, (count & ((1ull << kKindBit) - 1)) - c0);
    const u64 off = c0 * (kind == kScoreF32 ? 4 : 2);
    if (kind == kScoreF32) visit<kScoreF32>(src + off, dst + off, n, make.template of<kScoreF32>());
    else if (kind == kScoreF16) visit<kScoreF16>(src + off, dst + off, n, make.template of<kScoreF16>());
    else visit<kScoreBF16>(src + off, dst + off, n, make.template of<kScoreBF16>());
}
template <class M> __device__ __forceinline__ void visit(const FlatList& l, u32 at, u32 piece, M&& make) { visit_flat(l, l.src[at], l.dst[at], at, piece, make); }
template <class M> __device__ __forceinline__ void visit(const SumList& l, u32 at, u32 piece, M&& make) { visit_flat(l, l.src[at], (char*)nullptr, at, piece, make); }
template <class M> __device__ __forceinline__ void visit(const AdamList& l, u32 at, u32 piece, M&& make) { visit_flat(l, l.g[at], (char*)nullptr, at, piece, make); }

struct Squares {
    double sum = 0.0;
    template <int KIND> struct Of {
        static constexpr bool kPast = false;
        double& sum;
        __device__ __forceinline__ void whole(const vec& x, char*) const {
#pragma unroll
            for (int i = 0; i < kPer<KIND>; ++i) one(part<KIND>(x, i), nullptr, 0);
        }
        __device__ __forceinline__ void one(float x, char*, u32) const { sum = fma((double)x, (double)x, sum); }
    };
    template <int KIND> __device__ __forceinline__ Of<KIND> of() { return Of<KIND>{sum}; }
};

// The workgroup's sum of squares; (pieces that it takes: its wavefronts' numbers, and so on by all wavefronts').
template <class L> __device__ __forceinline__ double squares(const L& list, const Places<L>& places) {
    const u32 waves = blockDim.x / 64;
    Squares f;
    for (u32 piece = uniform(blockIdx.x * waves + threadIdx.x / 64); piece < list.pieces; piece += gridDim.x * waves) visit(list, places.of(piece), piece, f);
    return block_sum(f.sum);
}

// (160 million bf16 values of padded rows: 56 us, 5.7 TB/s.)
template <class L> __global__ __launch_bounds__(kThreads) void k_squares(const L list, double* sums) {
    const double sum = squares(list, Places<L>(list));
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

// The norm, and the factor.  (A NaN makes the factor NaN, an infinite norm makes it 0.)
struct Norm { double norm, factor; };
__device__ __forceinline__ Norm norm_of(double sum, double most) {
    Norm r;
    r.norm = sqrt(sum);
    r.factor = r.norm <= most || most == __builtin_inf() ? 1.0 : most / r.norm;
    return r;
}
// ... from all sums, the same in every workgroup.
__device__ __forceinline__ Norm norm_of(const double* sums, u32 n, double most) {
    double v = 0.0;
    for (u32 i = threadIdx.x; i < n; i += kThreads) v += sums[i];
    return norm_of(block_sum(v), most);
}

__global__ __launch_bounds__(kThreads) void k_norm(const double* sums, u32 n, float* norm) {
    const Norm r = norm_of(sums, n, __builtin_inf());
    if (threadIdx.x == 0) *norm = (float)r.norm;
}

// PAST: results go past the caches, and the gradients' second reading leaves nothing there.
template <bool PAST> struct Scaled {
    double factor;
    template <int KIND> struct Of {
        static constexpr bool kPast = PAST;
        double factor;
        // (kept from being rounded to 16 bits in one go where the compiler would: every place of a tensor by the same steps)
        __device__ __forceinline__ float of(float x) const {
            float v = (float)((double)x * factor);
            asm("" : "+v"(v));
            return v;
        }
        __device__ __forceinline__ void whole(const vec& x, char* to) const {
            float v[kPer<KIND>];
#pragma unroll
            for (int i = 0; i < kPer<KIND>; ++i) v[i] = of(part<KIND>(x, i));
            put_vec<KIND, PAST>(to, packed<KIND>(v));
        }
        __device__ __forceinline__ void one(float x, char* dst, u32 k) const { store_one<KIND>(dst, k, of(x)); }
    };
    template <int KIND> __device__ __forceinline__ Of<KIND> of() { return Of<KIND>{factor}; }
};

template <bool PAST, class L> __device__ __forceinline__ void scale(const L& list, const Places<L>& places, double factor) {
    const u32 waves = blockDim.x / 64;
    Scaled<PAST> f{factor};
    for (u32 piece = uniform(blockIdx.x * waves + threadIdx.x / 64); piece < list.pieces; piece += gridDim.x * waves) {
        const u32 back = list.pieces - 1 - piece;
        visit(list, places.of(back), back, f);
    }
}

// (... 104 us for 305 MiB read, most of it out of the memory-side cache, and as much written.)
template <class L, bool PAST> __global__ __launch_bounds__(kThreads) void k_scale(const L list, const double* sums, u32 n_sums, double most, int over, float* norm) {
    const Places<L> places(list);
    const Norm r = norm_of(sums, n_sums, most);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)r.norm;
    if (over && r.factor == 1.0) return;
    scale<PAST>(list, places, r.factor);
}

// All of it by one workgroup.
template <class L> __global__ __launch_bounds__(1024) void k_clip_few(const L list, double most, int over, float* norm) {
    const Places<L> places(list);
    const Norm r = norm_of(squares(list, places), most);
    if (norm && threadIdx.x == 0) *norm = (float)r.norm;
    if (over && r.factor == 1.0) return;
    scale<false>(list, places, r.factor);
}

// As qsv_adam_step, of the scaled gradient, its fused products included: their order shows in float32 where 0.9 m + 0.1 g lies in the
// middle between two of its numbers, one value in two hundred.
struct Adam {
    AdamRates by;
    double factor;
    __device__ __forceinline__ void operator()(float& p, float g, float& m, float& v) const {
        const double gi = (double)g * factor;
        const double mi = fma(1.0 - by.b1, gi, by.b1 * (double)m);
        const double vi = fma((1.0 - by.b2) * gi, gi, by.b2 * (double)v);
        p = (float)((double)p - by.lr * (mi / by.c1) / (sqrt(vi / by.c2) + by.eps));
        m = (float)mi;
        v = (float)vi;
    }
};

// Four gradients from k on.
template <int KIND, bool PAST> __device__ __forceinline__ void gradients_at(const char* g, u32 k, float (&x)[4]) {
    if (KIND == kScoreF32) {
        const vec q = vec_at<KIND, PAST>(g + (u64)k * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(q[i]);
    } else {
        typedef u32 two_at2 __attribute__((ext_vector_type(2), aligned(2)));
        const two_at2* from = (const two_at2*)(g + (u64)k * 2);
        const two_at2 q = PAST ? __builtin_nontemporal_load(from) : *from;
        const vec y = {q[0], q[1], 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = part<KIND>(y, i);
    }
}

// PAST: of what nobody reads again before the caches have seen other things.
template <bool PAST> __device__ __forceinline__ void four_at(const float* p, float (&x)[4]) {
    const vec q = PAST ? __builtin_nontemporal_load((const vec_at4*)p) : *(const vec_at4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(q[i]);
}
template <bool PAST> __device__ __forceinline__ void put_four(float* p, const float (&x)[4]) { put_vec<kScoreF32, PAST>((char*)p, packed<kScoreF32>(x)); }

template <int KIND, bool PAST> __device__ __forceinline__ void adam_values(float* p, const char* g, float* m, float* v, u32 n, const Adam& step) {
    const u32 lane = threadIdx.x & 63, whole = n / 4 * 4;
    for (u32 k = lane * 4; k < whole; k += 256) {
        float x[4], a[4], b[4], c[4];
        gradients_at<KIND, PAST>(g, k, x);
        four_at<PAST>(p + k, a);
        four_at<PAST>(m + k, b);
        four_at<PAST>(v + k, c);
#pragma unroll
        for (int i = 0; i < 4; ++i) step(a[i], x[i], b[i], c[i]);
        put_four<PAST>(p + k, a);
        put_four<PAST>(m + k, b);
        put_four<PAST>(v + k, c);
    }
    const u32 k = whole + lane;
    if (k < n) {
        float a = p[k], b = m[k], c = v[k];
        step(a, value_at<KIND>(g, k), b, c);
        p[k] = a;
        m[k] = b;
        v[k] = c;
    }
}

template <bool PAST> __device__ __forceinline__ void adam(const AdamList& l, const Places<AdamList>& places, const Adam& step) {
    const u32 waves = blockDim.x / 64;
    for (u32 i = uniform(blockIdx.x * waves + threadIdx.x / 64); i < l.pieces; i += gridDim.x * waves) {
        const u32 piece = l.pieces - 1 - i, at = places.of(piece);
        const u64 c0 = (u64)(piece - l.first[at]) * l.piece, count = l.count[at];
        const u32 kind = (u32)(count >> kKindBit), n = (u32)min((u64)l.piece, (count & ((1ull << kKindBit) - 1)) - c0);
        const char* g = l.g[at] + c0 * (kind == kScoreF32 ? 4 : 2);
        if (kind == kScoreF32) adam_values<kScoreF32, PAST>(l.p[at] + c0, g, l.m[at] + c0, l.v[at] + c0, n, step);
        else if (kind == kScoreF16) adam_values<kScoreF16, PAST>(l.p[at] + c0, g, l.m[at] + c0, l.v[at] + c0, n, step);
        else adam_values<kScoreBF16, PAST>(l.p[at] + c0, g, l.m[at] + c0, l.v[at] + c0, n, step);
    }
}

// A norm that is no number or infinite, as it is reported in float32: everything is left as it is.  (90 tensors of 49 million values with bf16 gradients: 250 us, 5.1 TB/s; the
// arithmetic of some 75 64-bit instructions a value would take half of that.)
template <bool PAST> __global__ __launch_bounds__(kThreads) void k_adam_list(const AdamList list, const double* sums, u32 n_sums, double most, const AdamRates by, float* norm) {
    const Places<AdamList> places(list);
    const Norm r = norm_of(sums, n_sums, most);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)r.norm;
    if (!((float)r.norm < __builtin_inff())) return;
    adam<PAST>(list, places, Adam{by, r.factor});
}

__global__ __launch_bounds__(1024) void k_adam_few(const AdamList list, double most, const AdamRates by, float* norm) {
    const Places<AdamList> places(list);
    const Norm r = norm_of(squares(list, places), most);
    if (norm && threadIdx.x == 0) *norm = (float)r.norm;
    if (!((float)r.norm < __builtin_inff())) return;
    adam<false>(list, places, Adam{by, r.factor});
}

// ---- lists -----------------------------------------------------------------------------------------------------------
u64 size_of(int kind) { return kind == kScoreF32 ? 4 : 2; }
u64 packed_count(u64 count, int kind) { return count | (u64)kind << kKindBit; }

// Few values in all are cut finer: more wavefronts share them, and a step's 64-bit arithmetic most of all.  Us: clipping by 1024 / 2048 /
// 4096 values 2 x 500000 f32 8.6 / 9.0 / 10.5, 2 x 2000000 14.1 / 13.0 / 13.2, the padded
// rows of 160 million bf16 values - / 176 / 167; Adam by 256 / 512 / 1024 2 x 8000
// 8.7 / 8.9 / 10.1, 2 x 256000 9.8 / 10.1 / 11.7, by 1024 / 2048 / 4096 2 x 500000 13.2 / 16.6 / 24.0, 2 x 1000000 17.4 / 17.9 / 24.8,
// 2 x 32000000 333 / 333 / 353.
u32 clip_piece(u64 values) { return values < 1ull << 21 ? 1024 : values < 1ull << 26 ? 2048 : 4096; }
u32 step_piece(u64 values) { return values < 3ull << 18 ? 256 : values < 1ull << 21 ? 1024 : 2048; }

// Up to so many pieces are one workgroup's, in one launch.  One launch / two, us: clipping 16000 f32 5.7 / 8.7, 32000 7.0 / 8.7, 4 x 8000 bf16
// 8.9 / 8.8, 64000 f32 10.8 / 8.7; Adam 2 x 2000 5.9 / 8.8, 2 x 4000 9.1 / 8.8, 2 x 8000 15.4 / 8.7.
constexpr u32 kFewPieces = 24;

// From so many bytes of results on they go past the caches, which the gradients' second reading has for itself then.  With / without,
// us: clipping 2 x 4000000 f32 19.6 / 19.3, 2 x 16000000 67 / 80, 2 x 64000000 266 / 292; Adam 2 x 2000000 28.8 / 26.5, 2 x 8000000 95 /
// 103, 2 x 64000000 746 / 821.  (Clipped gradients of less are read by the step that follows out of the cache.)  That second reading goes
// past them as well: clipping 2 x 64000000 f32 252 / 268, 160 million bf16 values of padded rows 157 / 163, Adam over 104 million parameters with
// bf16 gradients 534 / 546; the first reading too: 178 and 572.  Over the gradients (three lists in turn, each above the highest norm at every
// call) the two together, with / without: 2 x 8000000 f32 41 / 35, 2 x 17500000 73 / 86, 2 x 32000000 125 / 149, 2 x 64000000 254 / 305; and with the
// results read behind it 343 / 378.
constexpr u64 kPastClip = 128ull << 20, kPastStep = 64ull << 20;

struct Clip {
    const qsv_tensor *src, *dst;
    int64_t n;
    u32 piece;
    bool all_segs;                    // one list has room for all of them
    u64 values(int64_t i) const { return (u64)src[i].rows * (u64)src[i].cols; }
    bool flat(int64_t i) const {
        const qsv_tensor &a = src[i], &b = dst[i];
        return a.rows == 1 || (a.row_stride == a.cols && b.row_stride == b.cols);
    }
    // Whether tensor i goes to lists of this kind, and there.
    bool takes(const SegList&, int64_t i) const { return values(i) && (all_segs || !flat(i)); }
    bool takes(const FlatList&, int64_t i) const { return values(i) && !all_segs && flat(i); }
    bool takes(const SumList&, int64_t i) const { return values(i) && !all_segs && flat(i); }
    void put(SegList& l, int64_t i) const {
        const qsv_tensor &a = src[i], &b = dst[i];
        const bool one = flat(i);
        Seg& s = l.seg[l.n];
        s.src = (const char*)a.data_dev;
        s.dst = (char*)b.data_dev;
        s.rows = one ? 1 : (u64)a.rows;
        s.cols = one ? values(i) : (u64)a.cols;
        s.src_stride = (u64)a.row_stride * size_of(a.kind);
        s.dst_stride = (u64)b.row_stride * size_of(a.kind);
        s.kind = (u32)a.kind;
        const bool parts = s.rows == 1 || s.cols > piece / 2;
        s.row_pieces = parts ? (u32)((s.cols + piece - 1) / piece) : 0;
        s.rows_piece = parts ? 1 : (u32)(piece / s.cols);
        l.pieces += parts ? (u32)s.rows * s.row_pieces : (u32)((s.rows + s.rows_piece - 1) / s.rows_piece);
    }
    void put(SumList& l, int64_t i) const {
        l.src[l.n] = (const char*)src[i].data_dev;
        l.count[l.n] = packed_count(values(i), src[i].kind);
        l.pieces += (u32)((values(i) + piece - 1) / piece);
    }
    void put(FlatList& l, int64_t i) const {
        l.src[l.n] = (const char*)src[i].data_dev;
        l.dst[l.n] = (char*)dst[i].data_dev;
        l.count[l.n] = packed_count(values(i), src[i].kind);
        l.pieces += (u32)((values(i) + piece - 1) / piece);
    }
};

struct Step {
    const qsv_adam_tensor* t;
    int64_t n;
    u32 piece;
    bool takes(const SumList&, int64_t i) const { return t[i].count > 0; }
    bool takes(const AdamList&, int64_t i) const { return t[i].count > 0; }
    void put(SumList& l, int64_t i) const {
        l.src[l.n] = (const char*)t[i].grad_dev;
        l.count[l.n] = packed_count((u64)t[i].count, t[i].kind);
        l.pieces += (u32)(((u64)t[i].count + piece - 1) / piece);
    }
    void put(AdamList& l, int64_t i) const {
        l.p[l.n] = t[i].param_dev;
        l.g[l.n] = (const char*)t[i].grad_dev;
        l.m[l.n] = t[i].m_dev;
        l.v[l.n] = t[i].v_dev;
        l.count[l.n] = packed_count((u64)t[i].count, t[i].kind);
        l.pieces += (u32)(((u64)t[i].count + piece - 1) / piece);
    }
};

// The tensors from i on, to the end or as many as a list has room for.
template <class L, class S> void next_list(const S& s, int64_t* i, L& l) {
    l.n = l.pieces = 0;
    l.piece = s.piece;
    for (; *i < s.n && l.n < (u32)L::kRoom; ++*i) {
        if (!s.takes(l, *i)) continue;
        l.first[l.n] = l.pieces;
        s.put(l, *i);
        ++l.n;
    }
}

// One launch of the sums a list; `all` pieces share kSums of them.
template <class L, class S> void launch_squares(const S& s, u64 all, double* sums, u32* done, hipStream_t st) {
    L l;
    for (int64_t i = 0; i < s.n;) {
        next_list(s, &i, l);
        if (!l.pieces) continue;
        const u64 blocks = (l.pieces + kThreads / 64 - 1) / (kThreads / 64);
        const u32 grid = (u32)std::min(blocks, 1 + (u64)l.pieces * (kSums - 1) / all);
        hipLaunchKernelGGL(k_squares<L>, dim3(grid), dim3(kThreads), 0, st, l, sums + *done);
        *done += grid;
    }
}

u32 grid_for(u32 pieces) { return std::min((pieces + kThreads / 64 - 1) / (kThreads / 64), kSums); }

template <class L, bool PAST> void launch_scale(const Clip& s, const double* sums, u32 done, double max_norm, int over, float** norm, hipStream_t st) {
    L l;
    for (int64_t i = 0; i < s.n;) {
        next_list(s, &i, l);
        if (!l.pieces) continue;
        hipLaunchKernelGGL((k_scale<L, PAST>), dim3(grid_for(l.pieces)), dim3(kThreads), 0, st, l, sums, done, max_norm, over, *norm);
        *norm = nullptr;
    }
}

template <class L, class S> u64 all_pieces(const S& s) {
    L l;
    u64 all = 0;
    for (int64_t i = 0; i < s.n;) { next_list(s, &i, l); all += l.pieces; }
    return all;
}

}  // namespace

size_t norm_scratch_bytes() { return (kSums + kMostLists) * sizeof(double); }

hipError_t launch_clip(const qsv_tensor* grads, const qsv_tensor* outs, int64_t n, double max_norm, float* norm, void* scratch, hipStream_t st) {
    double* sums = (double*)scratch;
    Clip s{grads, outs ? outs : grads, n, 0, n <= kSegs};
    u64 values = 0, bytes = 0;
    for (int64_t i = 0; i < n; ++i) {
        values += s.values(i);
        bytes += s.values(i) * size_of(grads[i].kind);
    }
    s.piece = clip_piece(values);
    const int over = outs ? 0 : 1;
    if (s.all_segs) {
        SegList l;
        int64_t i = 0;
        next_list(s, &i, l);
        if (l.pieces <= kFewPieces) {
            hipLaunchKernelGGL(k_clip_few<SegList>, dim3(1), dim3(1024), 0, st, l, max_norm, over, norm);
            return hipGetLastError();
        }
    }
    const u64 all = all_pieces<SegList>(s) + all_pieces<SumList>(s);
    u32 done = 0;
    launch_squares<SegList>(s, all, sums, &done, st);
    launch_squares<SumList>(s, all, sums, &done, st);
    if (!done || (over && max_norm == HUGE_VAL)) {
        if (norm) hipLaunchKernelGGL(k_norm, dim3(1), dim3(kThreads), 0, st, sums, done, norm);
        return hipGetLastError();
    }
    if (bytes >= kPastClip) {
        launch_scale<FlatList, true>(s, sums, done, max_norm, over, &norm, st);
        launch_scale<SegList, true>(s, sums, done, max_norm, over, &norm, st);
    } else {
        launch_scale<FlatList, false>(s, sums, done, max_norm, over, &norm, st);
        launch_scale<SegList, false>(s, sums, done, max_norm, over, &norm, st);
    }
    return hipGetLastError();
}

hipError_t launch_adam_clipped(const qsv_adam_tensor* t, int64_t n, double max_norm, const AdamRates& by, float* norm, void* scratch, hipStream_t st) {
    double* sums = (double*)scratch;
    Step s{t, n, 0};
    u64 values = 0;
    for (int64_t i = 0; i < n; ++i) values += (u64)t[i].count;
    s.piece = step_piece(values);
    AdamList l;
    int64_t i = 0;
    next_list(s, &i, l);
    if (i == n && l.pieces <= kFewPieces) {
        hipLaunchKernelGGL(k_adam_few, dim3(1), dim3(1024), 0, st, l, max_norm, by, norm);
        return hipGetLastError();
    }
    u32 done = 0;
    launch_squares<SumList>(s, all_pieces<SumList>(s), sums, &done, st);
    for (i = 0; i < n;) {
        next_list(s, &i, l);
        if (!l.pieces) continue;
        if (12 * values >= kPastStep) hipLaunchKernelGGL(k_adam_list<true>, dim3(grid_for(l.pieces)), dim3(kThreads), 0, st, l, sums, done, max_norm, by, norm);
        else hipLaunchKernelGGL(k_adam_list<false>, dim3(grid_for(l.pieces)), dim3(kThreads), 0, st, l, sums, done, max_norm, by, norm);
        norm = nullptr;
    }
    return hipGetLastError();
}

}  // namespace qsv
