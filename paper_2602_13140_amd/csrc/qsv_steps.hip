// The norm of many tensors' gradients together, gradients scaled to a highest norm, and Adam's step with that on the way.
//
//   N = sqrt(sum g^2),  f = N > M ? M / N : 1;  out = f g
//   m = b1 m + (1 - b1) f g,  v = b2 v + (1 - b2) (f g)^2,  p -= lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// Bound by memory: every gradient is read for the norm and once more for what is made of it.  Tensors are cut into pieces of
// kPiece values (whole rows where they are shorter), numbered through a list of up to kList tensors that comes with the launch's
// arguments; a workgroup takes every so many-th piece and leaves one sum.  The next launch's workgroups each add all of these
// in the same order, so results depend on nothing but the list.  Squares and their sums are in 64 bits, where no float32 value
// overflows or vanishes.
#include "qsv_rows.h"
#include "qsv_tensors.h"
#include "qsv_wave.h"

#include <cmath>

namespace qsv {
namespace {

typedef unsigned long long u64;
typedef unsigned u32;

constexpr int kList = 60;             // tensors of a launch: 64 bytes each, within 4 KiB of arguments; no more than lanes
constexpr int kThreads = 256;
constexpr u32 kPiece = 8192;
constexpr u32 kSums = 2048;           // sums of all launches together; rounded up for each of them
constexpr int kMostLists = (kMostTensors + kList - 1) / kList;

struct Seg {
    const char* src;
    char* dst;                        // where the scaled gradient goes
    u64 rows, cols;
    u64 src_stride, dst_stride;       // bytes
    u32 first;                        // its first piece's number
    u32 row_pieces;                   // pieces of a row; 0: rows_piece rows are a piece
    u32 rows_piece;
    u32 kind;
};
struct Segs {
    u32 n, pieces;
    Seg seg[kList];
};

struct AdamSeg {
    float* p;
    const char* g;
    float* m;
    float* v;
    u64 count;
    u32 first, kind;
};
struct AdamSegs {
    u32 n, pieces;
    AdamSeg seg[kList];
};

// The place in the list of a piece's tensor: a lane asks for each of them.
template <class L> __device__ __forceinline__ u32 firsts(const L& list) {
    const u32 lane = threadIdx.x & 63;
    return lane < list.n ? list.seg[lane].first : ~0u;
}
__device__ __forceinline__ u32 place_of(u32 piece, u32 first) { return (u32)__popcll(__ballot(first <= piece)) - 1; }

__device__ __forceinline__ double block_sum(double v, double* sm) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) v += sm[w];
    return v;
}

// Every value of a piece: whole vectors (with the place their results go to), and single values.
template <int KIND, class F> __device__ __forceinline__ void visit(const Seg& s, u32 q, F&& f) {
    constexpr u32 W = kPer<KIND>, S = kSize<KIND>;
    if (s.row_pieces) {
        const u64 row = q / s.row_pieces, c0 = (u64)(q % s.row_pieces) * kPiece;
        const u32 n = (u32)min((u64)kPiece, s.cols - c0), whole = n / W;
        const char* src = s.src + row * s.src_stride + c0 * S;
        char* dst = s.dst + row * s.dst_stride + c0 * S;
        for (u32 j = threadIdx.x; j < whole; j += kThreads) f.whole(vec_at<KIND>(src + j * 16), dst + j * 16);
        const u32 k = whole * W + threadIdx.x;
        if (k < n) f.one(value_at<KIND>(src, k), dst, k);
        return;
    }
    const u64 row = (u64)q * s.rows_piece;
    const u32 cols = (u32)s.cols, units = (cols + W - 1) / W, n = (u32)min((u64)s.rows_piece, s.rows - row) * units;
    const u32 dr = kThreads / units, du = kThreads % units;
    u32 r = threadIdx.x / units, u = threadIdx.x % units;
    for (u32 i = threadIdx.x; i < n; i += kThreads) {
        const char* src = s.src + (row + r) * s.src_stride;
        char* dst = s.dst + (row + r) * s.dst_stride;
        if (u * W + W <= cols) f.whole(vec_at<KIND>(src + u * 16), dst + u * 16);
        else
            for (u32 k = u * W; k < cols; ++k) f.one(value_at<KIND>(src, k), dst, k);
        r += dr;
        u += du;
        if (u >= units) { u -= units; ++r; }
    }
}

template <int KIND> struct Squares {
    double sum = 0.0;
    __device__ __forceinline__ void whole(const vec& x, char*) {
#pragma unroll
        for (int i = 0; i < kPer<KIND>; ++i) one(part<KIND>(x, i), nullptr, 0);
    }
    __device__ __forceinline__ void one(float x, char*, u32) { sum = fma((double)x, (double)x, sum); }
};

__global__ __launch_bounds__(kThreads) void k_squares(const Segs list, double* sums) {
    __shared__ double sm[kThreads / 64];
    const u32 first = firsts(list);
    double sum = 0.0;
    for (u32 piece = blockIdx.x; piece < list.pieces; piece += gridDim.x) {
        const Seg& s = list.seg[uniform(place_of(piece, first))];
        if (s.kind == kScoreF32) {
            Squares<kScoreF32> f;
            visit<kScoreF32>(s, piece - s.first, f);
            sum += f.sum;
        } else if (s.kind == kScoreF16) {
            Squares<kScoreF16> f;
            visit<kScoreF16>(s, piece - s.first, f);
            sum += f.sum;
        } else {
            Squares<kScoreBF16> f;
            visit<kScoreBF16>(s, piece - s.first, f);
            sum += f.sum;
        }
    }
    sum = block_sum(sum, sm);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

// The norm from all sums, the same in every workgroup, and the factor.  (A NaN makes the factor NaN, an infinite norm makes it 0.)
struct Norm { double norm, factor; };
__device__ __forceinline__ Norm norm_of(const double* sums, u32 n, double most) {
    __shared__ double sm[kThreads / 64];
    double v = 0.0;
    for (u32 i = threadIdx.x; i < n; i += kThreads) v += sums[i];
    Norm r;
    r.norm = sqrt(block_sum(v, sm));
    r.factor = r.norm <= most || most == __builtin_inf() ? 1.0 : most / r.norm;
    return r;
}

__global__ __launch_bounds__(kThreads) void k_norm(const double* sums, u32 n, float* norm) {
    const Norm r = norm_of(sums, n, __builtin_inf());
    if (threadIdx.x == 0) *norm = (float)r.norm;
}

template <int KIND> struct Scaled {
    double factor;
    __device__ __forceinline__ float of(float x) const { return (float)((double)x * factor); }
    __device__ __forceinline__ void whole(const vec& x, char* to) {
        float v[kPer<KIND>];
#pragma unroll
        for (int i = 0; i < kPer<KIND>; ++i) v[i] = of(part<KIND>(x, i));
        put_vec<KIND, false>(to, packed<KIND>(v));
    }
    __device__ __forceinline__ void one(float x, char* dst, u32 k) { store_one<KIND>(dst, k, of(x)); }
};

__global__ __launch_bounds__(kThreads) void k_scale(const Segs list, const double* sums, u32 n_sums, double most, int over, float* norm) {
    const Norm r = norm_of(sums, n_sums, most);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)r.norm;
    if (over && r.factor == 1.0) return;
    const u32 first = firsts(list);
    for (u32 piece = blockIdx.x; piece < list.pieces; piece += gridDim.x) {
        const Seg& s = list.seg[uniform(place_of(piece, first))];
        if (s.kind == kScoreF32) visit<kScoreF32>(s, piece - s.first, Scaled<kScoreF32>{r.factor});
        else if (s.kind == kScoreF16) visit<kScoreF16>(s, piece - s.first, Scaled<kScoreF16>{r.factor});
        else visit<kScoreBF16>(s, piece - s.first, Scaled<kScoreBF16>{r.factor});
    }
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

template <int KIND> __device__ __forceinline__ void adam_piece(const AdamSeg& s, u32 q, const Adam& step) {
    const u64 c0 = (u64)q * kPiece;
    const u32 n = (u32)min((u64)kPiece, s.count - c0);
    for (u32 k = threadIdx.x; k < n; k += kThreads) {
        float p = s.p[c0 + k], m = s.m[c0 + k], v = s.v[c0 + k];
        step(p, value_at<KIND>(s.g + c0 * kSize<KIND>, k), m, v);
        s.p[c0 + k] = p;
        s.m[c0 + k] = m;
        s.v[c0 + k] = v;
    }
}

// A norm that is no number or infinite: everything is left as it is.
__global__ __launch_bounds__(kThreads) void k_adam_list(const AdamSegs list, const double* sums, u32 n_sums, double most, const AdamRates by, float* norm) {
    const Norm r = norm_of(sums, n_sums, most);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)r.norm;
    if (!(r.norm < __builtin_inf())) return;
    const Adam step{by, r.factor};
    const u32 first = firsts(list);
    for (u32 piece = blockIdx.x; piece < list.pieces; piece += gridDim.x) {
        const AdamSeg& s = list.seg[uniform(place_of(piece, first))];
        if (s.kind == kScoreF32) adam_piece<kScoreF32>(s, piece - s.first, step);
        else if (s.kind == kScoreF16) adam_piece<kScoreF16>(s, piece - s.first, step);
        else adam_piece<kScoreBF16>(s, piece - s.first, step);
    }
}

// ---- lists -----------------------------------------------------------------------------------------------------------
u64 size_of(int kind) { return kind == kScoreF32 ? 4 : 2; }

// Adds a tensor of rows x cols values; rows without a gap are one.
void add(Segs& l, int kind, const void* src, void* dst, u64 rows, u64 cols, u64 src_stride, u64 dst_stride) {
    if (rows > 1 && src_stride == cols && dst_stride == cols) { cols *= rows; rows = 1; }
    Seg& s = l.seg[l.n++];
    s.src = (const char*)src;
    s.dst = (char*)dst;
    s.rows = rows;
    s.cols = cols;
    s.src_stride = src_stride * size_of(kind);
    s.dst_stride = dst_stride * size_of(kind);
    s.first = l.pieces;
    s.kind = (u32)kind;
    if (rows == 1 || cols > kPiece / 2) {
        s.row_pieces = (u32)((cols + kPiece - 1) / kPiece);
        s.rows_piece = 1;
        l.pieces += (u32)rows * s.row_pieces;
    } else {
        s.row_pieces = 0;
        s.rows_piece = (u32)(kPiece / cols);
        l.pieces += (u32)((rows + s.rows_piece - 1) / s.rows_piece);
    }
}

bool empty(const qsv_tensor& t) { return t.rows < 1 || t.cols < 1; }

// Tensors from `at` on, up to a launch's room.
void next_list(const qsv_tensor* src, const qsv_tensor* dst, int64_t n, int64_t* at, Segs& l) {
    l.n = l.pieces = 0;
    for (; *at < n && l.n < (u32)kList; ++*at) {
        const qsv_tensor &a = src[*at], &b = (dst ? dst : src)[*at];
        if (!empty(a)) add(l, a.kind, a.data_dev, b.data_dev, (u64)a.rows, (u64)a.cols, (u64)a.row_stride, (u64)b.row_stride);
    }
}
void next_list(const qsv_adam_tensor* t, int64_t n, int64_t* at, Segs& l) {
    l.n = l.pieces = 0;
    for (; *at < n && l.n < (u32)kList; ++*at)
        if (t[*at].count > 0) add(l, t[*at].kind, t[*at].grad_dev, nullptr, 1, (u64)t[*at].count, 0, 0);
}
void next_list(const qsv_adam_tensor* t, int64_t n, int64_t* at, AdamSegs& l) {
    l.n = l.pieces = 0;
    for (; *at < n && l.n < (u32)kList; ++*at) {
        if (t[*at].count < 1) continue;
        l.seg[l.n++] = AdamSeg{t[*at].param_dev, (const char*)t[*at].grad_dev, t[*at].m_dev, t[*at].v_dev, (u64)t[*at].count, l.pieces, (u32)t[*at].kind};
        l.pieces += (u32)(((u64)t[*at].count + kPiece - 1) / kPiece);
    }
}

// One launch of the sums a list; the number of sums left.  NEXT fills the list from a place on.
template <class NEXT> u32 launch_squares(int64_t n, NEXT&& next, double* sums, hipStream_t st) {
    Segs l;
    u64 all = 0;
    u32 lists = 0, done = 0;
    for (int64_t at = 0; at < n;) { next(&at, l); all += l.pieces; lists += l.pieces ? 1 : 0; }
    for (int64_t at = 0; at < n;) {
        next(&at, l);
        if (!l.pieces) continue;
        const u64 share = lists == 1 ? kSums : 1 + (u64)l.pieces * kSums / all;
        const u32 grid = (u32)std::min((u64)l.pieces, share);
        hipLaunchKernelGGL(k_squares, dim3(grid), dim3(kThreads), 0, st, l, sums + done);
        done += grid;
    }
    return done;
}

}  // namespace

size_t norm_scratch_bytes() { return (kSums + kMostLists) * sizeof(double); }

hipError_t launch_clip(const qsv_tensor* grads, const qsv_tensor* outs, int64_t n, double max_norm, float* norm, void* scratch, hipStream_t st) {
    double* sums = (double*)scratch;
    const u32 done = launch_squares(n, [&](int64_t* at, Segs& l) { next_list(grads, outs, n, at, l); }, sums, st);
    if (max_norm == HUGE_VAL && !outs) {
        if (norm) hipLaunchKernelGGL(k_norm, dim3(1), dim3(kThreads), 0, st, sums, done, norm);
        return hipGetLastError();
    }
    if (!done && norm) hipLaunchKernelGGL(k_norm, dim3(1), dim3(kThreads), 0, st, sums, done, norm);
    Segs l;
    for (int64_t at = 0; at < n;) {
        next_list(grads, outs, n, &at, l);
        if (!l.pieces) continue;
        hipLaunchKernelGGL(k_scale, dim3(std::min(l.pieces, kSums)), dim3(kThreads), 0, st, l, sums, done, max_norm, outs ? 0 : 1, norm);
        norm = nullptr;
    }
    return hipGetLastError();
}

hipError_t launch_adam_clipped(const qsv_adam_tensor* t, int64_t n, double max_norm, const AdamRates& by, float* norm, void* scratch, hipStream_t st) {
    double* sums = (double*)scratch;
    const u32 done = launch_squares(n, [&](int64_t* at, Segs& l) { next_list(t, n, at, l); }, sums, st);
    if (!done && norm) hipLaunchKernelGGL(k_norm, dim3(1), dim3(kThreads), 0, st, sums, done, norm);
    AdamSegs l;
    for (int64_t at = 0; at < n;) {
        next_list(t, n, &at, l);
        if (!l.pieces) continue;
        hipLaunchKernelGGL(k_adam_list, dim3(std::min(l.pieces, kSums)), dim3(kThreads), 0, st, l, sums, done, max_norm, by, norm);
        norm = nullptr;
    }
    return hipGetLastError();
}

}  // namespace qsv
