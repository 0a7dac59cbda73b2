// Loss of rows of scores against a teacher known by its top logits, and its gradient.
//
//   q_j = exp(t_j / T - norm) over the teacher's entries, Q = sum q;  p = softmax(z / T)
//   L = sum_j q_j (ln q_j - ln p_{i_j}) = sum_j q_j (t_j / T - norm) - sum_j q_j (z_{i_j} - m) / T + Q ln s
//   dL/dz_k = (Q e_k / s - sum_{j: i_j = k} q_j) / T,  e_k = exp((z_k - m) / T), m = max z, s = sum e
//
// Bound by memory: a row is read once and its gradient written once.  A workgroup keeps its row in registers between the
// maximum, the sum and the gradient (16 vectors of 16 bytes a thread: up to 131072 values of 16 bits, 65536 of 32); longer
// rows are read again for the gradient.  The gradient is written as if no entry of the teacher were there, and the few
// places of the entries are written once more after a barrier.
//
// Exponentials and the values they are taken of are in 32 bits, sums over a thread's values too; sums over threads, the
// teacher's weights and the loss, a small difference of large numbers, in 64.
#include "qsv_rows.h"
#include "qsv_scores.h"
#include "qsv_wave.h"

namespace qsv {
namespace {

typedef unsigned long long u64;
typedef unsigned u32;
constexpr float kInf = __builtin_inff();

template <int KIND> constexpr u32 kNone = KIND == kScoreF32 ? 0xff800000u : KIND == kScoreBF16 ? 0xff80ff80u : 0xfc00fc00u;   // -inf

// Vector j of a row's whole vectors; -inf behind them.  (Offsets of 32 bits to a uniform address: a row has 4 GiB at most.)
template <int KIND> __device__ __forceinline__ vec load_vec(const char* row, u32 whole, u32 j) {
    vec x = {kNone<KIND>, kNone<KIND>, kNone<KIND>, kNone<KIND>};
    if (j < whole) x = vec_at<KIND>(row + j * 16u);
    return x;
}

// The values behind a row's whole vectors, one a lane; -inf in the others.
template <int KIND> __device__ __forceinline__ float load_rest(const char* row, u32 cols, u32 lane) {
    const u32 k = cols / kPer<KIND> * kPer<KIND> + lane;
    return lane < kPer<KIND> && k < cols ? value_at<KIND>(row, k) : -kInf;
}

// PAST: past the caches.
template <int KIND, bool PAST> __device__ __forceinline__ void store_vec(char* row, u32 whole, u32 j, const float (&g)[kPer<KIND>]) {
    if (j < whole) put_vec<KIND, PAST>(row + j * 16u, packed<KIND>(g));
}

template <int KIND> __device__ __forceinline__ void store_rest(char* row, u32 cols, u32 lane, float g) {
    const u32 k = cols / kPer<KIND> * kPer<KIND> + lane;
    if (lane < kPer<KIND> && k < cols) store_one<KIND>(row, k, g);
}

// The compiler keeps nothing that it worked out of the vectors: unpacked values of one phase, kept for the next, would take
// twice the registers of the vectors themselves.
template <int N> __device__ __forceinline__ void forget(vec (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// ---- workgroups ------------------------------------------------------------------------------------------------------
// A wavefront's result a lane, then over the lanes: a loop over the wavefronts' results would hold all of them in registers.
template <int NT> __device__ __forceinline__ float block_max(float v, double* sm) {
    constexpr int NW = NT / 64;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    if (NW == 1) return uniform(v);
    __syncthreads();
    if (lane == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (float)sm[lane & (NW - 1)];
#pragma unroll
    for (int o = NW / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return uniform(v);
}

template <int NT, int N> __device__ __forceinline__ void block_sums(double (&v)[N], double* sm) {     // sm: 16 N entries
    constexpr int NW = NT / 64;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
    if (NW > 1) {
        __syncthreads();
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) sm[k * 16 + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = sm[k * 16 + (lane & (NW - 1))];
#pragma unroll
            for (int o = NW / 2; o > 0; o >>= 1) v[k] += __shfl_xor(v[k], o, 64);
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = uniform(v[k]);
}

// A row's teacher: idx, q and z of its entries in LDS, and their sums.
struct Taught { double q, qx; };      // sum q, sum q (t / T - norm)
struct TeacherLds { double* q; int* idx; float* z; };

__device__ __forceinline__ TeacherLds teacher_lds(char* lds, int top) {
    const int room = (top + 3) & ~3;
    TeacherLds t;
    t.q = (double*)lds;
    t.idx = (int*)(t.q + room);
    t.z = (float*)(t.idx + room);
    return t;
}

inline size_t teacher_bytes(int top) { return (size_t)((top + 3) & ~3) * 16; }

// LISTED: `row` holds the scores at the entries, in their order.
template <int KIND, int NT, bool LISTED = false> __device__ __forceinline__ Taught teach(const TeacherArgs& a, u64 r, const char* row, u32 cols, const TeacherLds& l, double* sm) {
    const int* idx = a.idx + r * a.top;
    const float* logits = a.logits + r * a.top;
    float high = -kInf;
    if (threadIdx.x < ((a.top + 3) & ~3) - a.top) l.idx[a.top + threadIdx.x] = -1;
    for (int j = threadIdx.x; j < a.top; j += NT) {
        const int i = idx[j];
        const bool real = i >= 0 && (u32)i < cols;
        const float t = logits[j];
        l.idx[j] = real ? i : -1;
        l.z[j] = real ? value_at<KIND>(row, LISTED ? (u32)j : (u32)i) : 0.f;
        l.q[j] = (double)t;
        if (real) high = fmaxf(high, t);
    }
    double norm;
    if (a.lse) {
        norm = (double)a.lse[r];
    } else {
        high = block_max<NT>(high, sm);
        const double top = high > -kInf ? (double)high * a.inv_t : 0.0;
        double s[1] = {0.0};
        for (int j = threadIdx.x; j < a.top; j += NT)
            if (l.idx[j] >= 0) s[0] += exp(l.q[j] * a.inv_t - top);
        block_sums<NT, 1>(s, sm);
        norm = top + log(s[0]);              // no entry: -inf, and every q below 0
    }
    double v[2] = {0.0, 0.0};
    for (int j = threadIdx.x; j < a.top; j += NT) {
        const double x = l.q[j] * a.inv_t - norm;
        const double q = l.idx[j] >= 0 && l.q[j] != -(double)kInf ? exp(x) : 0.0;
        if (q != 0.0) {
            v[0] += q;
            v[1] += q * x;
        }
        l.q[j] = q;
    }
    block_sums<NT, 2>(v, sm);
    return Taught{v[0], v[1]};
}

// The thread's part of sum q (z - m) / T: differences first, scores may be large.
template <int NT> __device__ __forceinline__ double below_top(const TeacherLds& l, int top, float m, double inv_t) {
    double v = 0.0;
    for (int j = threadIdx.x; j < top; j += NT)
        if (l.q[j] != 0.0) v += l.z[j] == -kInf ? -(double)kInf : l.q[j] * (((double)l.z[j] - (double)m) * inv_t);
    return v;
}

// A row's loss from its statistics.  below: the sum over all threads.
__device__ __forceinline__ float loss_of(const Taught& t, double below, double s) {
    if (t.q == 0.0) return 0.f;
    if (below == -(double)kInf && s == s) return kInf;         // an entry that the student excludes
    return (float)(t.qx - below + t.q * log(s));
}

struct Gradient { float m, c, scale, of_q; };      // scale: of e; of_q: of q

// e_k times scale is the gradient where the teacher has no entry.
__device__ __forceinline__ Gradient gradient_of(const Taught& t, float m, double s, double inv_t, float grad_loss) {
    Gradient g;
    g.m = m > -kInf ? m : 0.f;
    g.c = (float)(1.4426950408889634074 * inv_t);
    const double by = t.q != 0.0 ? (double)grad_loss * inv_t : 0.0;
    g.scale = s > 0.0 || s != s ? (float)(by * t.q / s) : 0.f;
    g.of_q = (float)by;
    return g;
}

__device__ __forceinline__ float e_of(const Gradient& g, float z) { return __builtin_amdgcn_exp2f((z - g.m) * g.c); }

// The places of the teacher's entries between k0 and k1, once each, whichever entries name them.  The others are looked
// through four at a time: an entry twice is rare, and the search bound by the latency of LDS.
template <int KIND, int NT> __device__ __forceinline__ void write_entries(const TeacherLds& l, int top, const Gradient& g, char* grad, u32 k0, u32 k1) {
    typedef int four __attribute__((ext_vector_type(4)));
    for (int j = threadIdx.x; j < top; j += NT) {
        const int k = l.idx[j];
        if (k < 0 || (u32)k < k0 || (u32)k >= k1) continue;
        double q = l.q[j];
        bool first = true;
#pragma unroll 4
        for (int i = 0; i < top; i += 4) {
            const four x = *(const four*)(l.idx + i);
            if (x[0] != k && x[1] != k && x[2] != k && x[3] != k) continue;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (x[u] == k && i + u != j) {
                    if (i + u < j) first = false;
                    q += l.q[i + u];
                }
        }
        if (first) store_one<KIND>(grad, (u32)k, (float)((double)(e_of(g, l.z[j]) * g.scale) - q * (double)g.of_q));
    }
}

// ---- one workgroup a row ---------------------------------------------------------------------------------------------
// Loss and gradient, 64 entries, 4096 x 32768 bf16: 124 us, 4.3 TB/s (a copy of 4 GiB: 4.8); 4096 x 131072 bf16, 128 entries: 519
// us, 4.1 TB/s: such a row takes a CU's registers, and its loads wait for the stores of the one before.  A loss alone, 513 x
// 50021 f16: 16.4 us.  Short rows are bound by latency (16 x 1000 f32: 6.4 us).
template <int KIND, int NT, bool KEPT, bool PAST>
__global__ __launch_bounds__(NT) void k_distill_row(const DistillArgs a) {
    constexpr int W = kPer<KIND>, NV = 16;
    extern __shared__ char lds[];
    __shared__ double sm[48];
    const u64 r = grid_block();
    if (r >= (u64)a.rows) return;
    const char* row = (const char*)a.scores + r * (u64)a.stride * kSize<KIND>;
    const TeacherLds l = teacher_lds(lds, a.teacher.top);
    const u32 whole = a.cols / W;
    const float c = (float)(1.4426950408889634074 * a.teacher.inv_t);
    vec x[KEPT ? NV : 1];
    if (KEPT) {
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = load_vec<KIND>(row, whole, (u32)i * NT + threadIdx.x);
    }
    const float rest = load_rest<KIND>(row, a.cols, threadIdx.x);
    float m = rest, sum;
    const Taught t = teach<KIND, NT>(a.teacher, r, row, a.cols, l, sm);
    if (KEPT) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < W; ++k) m = fmaxf(m, part<KIND>(x[i], k));
        m = block_max<NT>(m, sm);
        forget(x);
        const float base = m > -kInf ? m : 0.f;
        sum = __builtin_amdgcn_exp2f((rest - base) * c);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float some = 0.f;
#pragma unroll
            for (int k = 0; k < W; ++k) some += __builtin_amdgcn_exp2f((part<KIND>(x[i], k) - base) * c);
            sum += some;
        }
    } else {
        // the thread's own maximum so far, and the sum relative to it: of one value 1, or 0 where that is -inf, or NaN (of +inf too)
        sum = __builtin_amdgcn_exp2f((rest - (m > -kInf ? m : 0.f)) * c);
        for (u32 j = threadIdx.x; j < whole; j += 4 * NT) {
            vec y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = load_vec<KIND>(row, whole, j + i * NT);
            float high = m;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int k = 0; k < W; ++k) high = fmaxf(high, part<KIND>(y[i], k));
            forget(y);
            const float base = high > -kInf ? high : 0.f;
            sum *= high > m ? __builtin_amdgcn_exp2f((m - high) * c) : 1.f;
            m = high;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float some = 0.f;
#pragma unroll
                for (int k = 0; k < W; ++k) some += __builtin_amdgcn_exp2f((part<KIND>(y[i], k) - base) * c);
                sum += some;
            }
        }
        const float own = m;
        m = block_max<NT>(m, sm);
        if (own < m) sum *= __builtin_amdgcn_exp2f((own - m) * c);
    }
    double s[2] = {(double)sum, a.loss ? below_top<NT>(l, a.teacher.top, m, a.teacher.inv_t) : 0.0};
    block_sums<NT, 2>(s, sm);
    if (threadIdx.x == 0) {
        if (a.loss) a.loss[r] = loss_of(t, s[1], s[0]);
        if (a.stats) { a.stats[2 * r] = m; a.stats[2 * r + 1] = (float)s[0]; }
    }
    if (!a.grad) return;
    char* grad = (char*)a.grad + r * (u64)a.grad_stride * kSize<KIND>;
    const Gradient g = gradient_of(t, m, s[0], a.teacher.inv_t, a.grad_loss ? a.grad_loss[r] : 1.f);
    const bool zero = t.q == 0.0;
    auto write = [&](u32 j, const vec& y) {
        float o[W];
#pragma unroll
        for (int k = 0; k < W; ++k) o[k] = zero ? 0.f : e_of(g, part<KIND>(y, k)) * g.scale;
        store_vec<KIND, PAST>(grad, whole, j, o);
    };
    if (KEPT) {
        forget(x);
#pragma unroll
        for (int i = 0; i < NV; ++i) write((u32)i * NT + threadIdx.x, x[i]);
    } else {
        for (u32 j = threadIdx.x; j < whole; j += NT) write(j, load_vec<KIND>(row, whole, j));
    }
    store_rest<KIND>(grad, a.cols, threadIdx.x, zero ? 0.f : e_of(g, rest) * g.scale);
    if (zero) return;
    __syncthreads();       // the entries' places are written a second time
    write_entries<KIND, NT>(l, a.teacher.top, g, grad, 0, a.cols);
}

// ---- few rows, or a gradient from kept statistics: parts of rows by workgroups of their own -------------------------
// A part: PV vectors a thread.  Few rows take 2, which spreads them over four times the CUs; long ones, which fill the chip
// anyway, 8, and so does a gradient from kept statistics, since every part works its row's teacher out again.
constexpr int kPartThreads = 256;

struct Parts {
    u32 parts;
    double* taught;       // [rows][2]: sum q, sum q (t / T - norm)
    double* part;         // [rows][parts][2]: maximum, sum relative to it
    double* q;            // [rows][top]: of the teacher's entries
    float* z;             // [rows][top]: the scores there
    double* joined;       // [rows][2]: the whole row's maximum and sum, or NULL: every part joins the parts' by itself
};

// A row's parts, and one workgroup more for its teacher (its scores are read here: the gradient may be written over them).
template <int KIND, int PV> __global__ __launch_bounds__(kPartThreads) void k_distill_stats(const DistillArgs a, const Parts p) {
    constexpr int W = kPer<KIND>;
    extern __shared__ char lds[];
    __shared__ double sm[48];
    const u64 r = grid_block() / (p.parts + 1);
    const u32 at = (u32)(grid_block() % (p.parts + 1));
    if (r >= (u64)a.rows) return;
    const char* row = (const char*)a.scores + r * (u64)a.stride * kSize<KIND>;
    if (at == p.parts) {
        const int top = a.teacher.top;
        const TeacherLds l = teacher_lds(lds, top);
        const Taught t = teach<KIND, kPartThreads>(a.teacher, r, row, a.cols, l, sm);
        for (int j = threadIdx.x; j < top; j += kPartThreads) {
            p.q[r * top + j] = l.q[j];
            p.z[r * top + j] = l.z[j];
        }
        if (threadIdx.x == 0) {
            p.taught[2 * r] = t.q;
            p.taught[2 * r + 1] = t.qx;
        }
        return;
    }
    const u32 j0 = at * (kPartThreads * PV) + threadIdx.x;
    const float c = (float)(1.4426950408889634074 * a.teacher.inv_t);
    const u32 whole = a.cols / W;
    vec x[PV];
#pragma unroll
    for (int i = 0; i < PV; ++i) x[i] = load_vec<KIND>(row, whole, j0 + (u32)i * kPartThreads);
    const float rest = at + 1 == p.parts ? load_rest<KIND>(row, a.cols, threadIdx.x) : -kInf;
    float m = rest;
#pragma unroll
    for (int i = 0; i < PV; ++i)
#pragma unroll
        for (int k = 0; k < W; ++k) m = fmaxf(m, part<KIND>(x[i], k));
    m = block_max<kPartThreads>(m, sm);
    forget(x);
    const float base = m > -kInf ? m : 0.f;
    float sum = __builtin_amdgcn_exp2f((rest - base) * c);
#pragma unroll
    for (int i = 0; i < PV; ++i)
#pragma unroll
        for (int k = 0; k < W; ++k) sum += __builtin_amdgcn_exp2f((part<KIND>(x[i], k) - base) * c);
    double s[1] = {(double)sum};
    block_sums<kPartThreads, 1>(s, sm);
    if (threadIdx.x == 0) {
        p.part[(r * p.parts + at) * 2] = (double)m;
        p.part[(r * p.parts + at) * 2 + 1] = s[0];
    }
}

// The parts' maxima and sums joined, a workgroup a row.
__global__ __launch_bounds__(1024) void k_distill_join(const DistillArgs a, const Parts p) {
    __shared__ double sm[16];
    const u64 r = grid_block();
    if (r >= (u64)a.rows) return;
    const double* part = p.part + r * p.parts * 2;
    float m = -kInf;
    for (u32 i = threadIdx.x; i < p.parts; i += 1024) m = fmaxf(m, (float)part[2 * i]);
    m = block_max<1024>(m, sm);
    double s[1] = {0.0};
    for (u32 i = threadIdx.x; i < p.parts; i += 1024)
        if (part[2 * i + 1] != 0.0) s[0] += part[2 * i + 1] * exp((part[2 * i] - (double)m) * a.teacher.inv_t);
    block_sums<1024, 1>(s, sm);
    if (threadIdx.x == 0) { p.joined[2 * r] = (double)m; p.joined[2 * r + 1] = s[0]; }
}

template <int KIND, int PV, bool PAST> __global__ __launch_bounds__(kPartThreads) void k_distill_apply(const DistillArgs a, const Parts p, u32 blocks) {
    constexpr int W = kPer<KIND>;
    extern __shared__ char lds[];
    __shared__ double sm[48];
    const u64 r = grid_block() / blocks;
    const u32 at = (u32)(grid_block() % blocks);
    if (r >= (u64)a.rows) return;
    const char* row = (const char*)a.scores + r * (u64)a.stride * kSize<KIND>;
    const TeacherLds l = teacher_lds(lds, a.teacher.top);
    const u32 j0 = at * (kPartThreads * PV) + threadIdx.x;
    const u32 whole = a.cols / W;
    vec x[PV];
    float rest = -kInf;
    if (a.grad) {
#pragma unroll
        for (int i = 0; i < PV; ++i) x[i] = load_vec<KIND>(row, whole, j0 + (u32)i * kPartThreads);
        if (at + 1 == blocks) rest = load_rest<KIND>(row, a.cols, threadIdx.x);
    }
    const int top = a.teacher.top;
    Taught t;
    float m = -kInf;
    double s[2] = {0.0, 0.0};
    if (a.have_stats) {
        t = teach<KIND, kPartThreads>(a.teacher, r, row, a.cols, l, sm);
        m = a.stats[2 * r];
        s[0] = (double)a.stats[2 * r + 1];
    } else {
        const double* part = p.part + r * p.parts * 2;
        t = Taught{p.taught[2 * r], p.taught[2 * r + 1]};
        if (threadIdx.x < ((top + 3) & ~3) - top) l.idx[top + threadIdx.x] = -1;
        for (int j = threadIdx.x; j < top; j += kPartThreads) {
            const int i = a.teacher.idx[r * top + j];
            l.idx[j] = i >= 0 && (u32)i < a.cols ? i : -1;
            l.q[j] = p.q[r * top + j];
            l.z[j] = p.z[r * top + j];
        }
        if (p.joined) {
            m = (float)p.joined[2 * r];
            s[0] = p.joined[2 * r + 1];
        } else {                           // few: each wavefront for itself
            const u32 lane = threadIdx.x & 63;
            for (u32 i = lane; i < p.parts; i += 64) m = fmaxf(m, (float)part[2 * i]);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
            m = uniform(m);
            for (u32 i = lane; i < p.parts; i += 64)
                if (part[2 * i + 1] != 0.0) s[0] += part[2 * i + 1] * exp((part[2 * i] - (double)m) * a.teacher.inv_t);
            s[0] = uniform(wave_sum(s[0]));
        }
        __syncthreads();
        if (a.loss && at == 0) {
            s[1] = below_top<kPartThreads>(l, top, m, a.teacher.inv_t);
            double v[1] = {s[1]};
            block_sums<kPartThreads, 1>(v, sm);
            s[1] = v[0];
        }
    }
    if (at == 0 && threadIdx.x == 0) {
        if (a.loss) a.loss[r] = loss_of(t, s[1], s[0]);
        if (a.stats && !a.have_stats) { a.stats[2 * r] = m; a.stats[2 * r + 1] = (float)s[0]; }
    }
    if (!a.grad) return;
    char* grad = (char*)a.grad + r * (u64)a.grad_stride * kSize<KIND>;
    const Gradient g = gradient_of(t, m, s[0], a.teacher.inv_t, a.grad_loss ? a.grad_loss[r] : 1.f);
    const bool zero = t.q == 0.0;
#pragma unroll
    for (int i = 0; i < PV; ++i) {
        float o[W];
#pragma unroll
        for (int k = 0; k < W; ++k) o[k] = zero ? 0.f : e_of(g, part<KIND>(x[i], k)) * g.scale;
        store_vec<KIND, PAST>(grad, whole, j0 + (u32)i * kPartThreads, o);
    }
    if (at + 1 == blocks) store_rest<KIND>(grad, a.cols, threadIdx.x, zero ? 0.f : e_of(g, rest) * g.scale);
    if (zero) return;
    __syncthreads();
    const u64 k0 = (u64)at * (kPartThreads * PV * W);
    write_entries<KIND, kPartThreads>(l, a.teacher.top, g, grad, (u32)k0, (u32)min(k0 + kPartThreads * PV * W, (u64)a.cols));
}

// ---- a circuit's own outcomes ----------------------------------------------------------------------------------------
// The loss of rows of amplitudes a against the teacher, with p_k = |a_k|^2, and lambda_k = dL/dp_k a_k = -q_k a_k / p_k at
// the entries, which reverse mode takes back.  (The derivative of the rows' norm is left out: no gate changes it.)  A row's
// entries are few: a workgroup each, bound by the latency of gathering them.
// lambda: NULL, or rows of 2^n that are zero, `per` rows apart, the first one `first` rows on.
// res: what the rounded scalars of a table's groups have made of a row's length; as a factor m of every p_k it would make the loss
// wrong by -Q ln m, some 3e-8 a group, and is taken out (14 qubits, 40 layers of rotations: 4.0e-7 from 64 bits with it, 1.0e-7
// without).  In lambda, which goes as 1 / a, it meets the inverse of itself in psi.
__global__ __launch_bounds__(256) void k_distill_state(const float2* A, int n, TeacherArgs te, u64 rows, double* f, u64 f_stride, float2* lambda, int per, int first, Residues res, int rowdep) {
    extern __shared__ char lds[];
    __shared__ double sm[48];
    const u64 r = grid_block();
    if (r >= rows) return;
    const float2* a = A + (r << n);
    const u32 cols = 1u << n;
    const TeacherLds l = teacher_lds(lds, te.top);
    const Taught t = teach<kScoreF32, 256, true>(te, r, (const char*)(te.logits + r * te.top), cols, l, sm);
    double loss[1] = {0.0};
    for (int j = threadIdx.x; j < te.top; j += 256) {
        const int k = l.idx[j];
        if (k < 0 || l.q[j] == 0.0) continue;
        const float2 z = a[k];
        const double pk = (double)z.x * z.x + (double)z.y * z.y;
        loss[0] -= l.q[j] * log(pk);
        if (!lambda) continue;
        double q = 0.0;
        bool once = true;
        for (int i = 0; i < te.top; ++i)
            if (l.idx[i] == k) {
                if (i < j && l.q[i] != 0.0) { once = false; break; }
                q += l.q[i];
            }
        if (once) {
            const double by = pk >= 0x1p-252 ? -q / pk : 0.0;      // (lambda of lower amplitudes would leave the range of 32 bits)
            lambda[((r * (u64)per + (u64)first) << n) + (u64)k] = make_float2((float)(by * z.x), (float)(by * z.y));
        }
    }
    block_sums<256, 1>(loss, sm);
    double m = 1.0;
    if (f && res.count) {
        const double* e = res.table + ((rowdep ? r * (u64)res.stride : 0) + (u64)res.first) * 2;
        for (int k = threadIdx.x & 63; k < res.count; k += 64) m *= e[2 * k] * e[2 * k] + e[2 * k + 1] * e[2 * k + 1];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m *= __shfl_xor(m, o, 64);
    }
    if (threadIdx.x == 0 && f) f[r * f_stride] = t.q == 0.0 ? 0.0 : t.qx + loss[0] + t.q * log(m);
}

// lambda's rows at zero, and (paired) psi beside them: rows 2r, 2r + 1.
__global__ __launch_bounds__(256) void k_distill_zero(const float2* A, int n, u64 total, float2* S, int paired) {
    const u64 e = grid_block() * 256 + threadIdx.x;
    if (e >= total) return;
    if (!paired) { S[e] = make_float2(0.f, 0.f); return; }
    const u64 r = e >> n, k = e & ((1ull << n) - 1);
    S[((2 * r) << n) | k] = A[e];
    S[((2 * r + 1) << n) | k] = make_float2(0.f, 0.f);
}

}  // namespace

static u64 parts_of(int kind, int64_t cols, int vecs) {
    const u64 values = (u64)kPartThreads * vecs * (kind == kScoreF32 ? 4 : 8);
    return ((u64)cols + values - 1) / values;
}
constexpr int kFewVecs = 2, kBackVecs = 8;

// Rows that would leave half of the chip idle, and are long enough to be split.  Loss and gradient, whole / split, us: 96 x 50021
// bf16 19.3 / 16.1, 127 19.7 / 17.9, 192 20.6 / 22.7, 512 31 / 41; 32 x 131072 f32 28.5 / 17.7, 127 39.5 / 39.7, 512 159 / 171; a loss
// alone 96 x 262144 bf16 24 / 17, 192 24.5 / 24.4, 256 26 / 30.
static bool takes_parts(int kind, int64_t rows, int64_t cols) { return rows < 128 && parts_of(kind, cols, kBackVecs) > 2; }

size_t distill_scratch_bytes(int64_t rows, int64_t cols) {
    if (rows < 1 || !takes_parts(kScoreF32, rows, cols)) return 0;
    return (size_t)rows * (32 + parts_of(kScoreF32, cols, kFewVecs) * 16 + 1024 * (8 + 4));
}

// Gradients of this size and more are written past the caches, which would not hold them for the next reader either (256 MiB:
// 124 us through the caches, 126 past them; 512 MiB 196 / 183; 1 GiB 553 / 515).
constexpr u64 kPastBytes = (u64)384 << 20;

// Rows of more parts than this take larger ones, and a launch that joins them; by themselves they would read all parts' results
// once a part (1 x 2^24 f32: 425 us, joined 38; 1 x 2^22 bf16 22 and 15; 1 x 2^20 f32, 512 small parts, 13.4 and 12.8).
constexpr u64 kFewParts = 256;

template <int KIND, int PV, bool PAST> static hipError_t launch_parts(const DistillArgs& a, void* scratch, hipStream_t st) {
    const size_t lds = teacher_bytes(a.teacher.top);
    const dim3 block(kPartThreads);
    Parts p{};
    p.parts = (u32)parts_of(KIND, a.cols, PV);
    const u32 blocks = a.grad ? p.parts : 1;
    p.taught = (double*)scratch;
    double* const joined = p.taught + 2 * (u64)a.rows;
    if (PV != kFewVecs) p.joined = joined;
    p.q = joined + 2 * (u64)a.rows;
    p.part = p.q + (u64)a.rows * a.teacher.top;
    p.z = (float*)(p.part + (u64)a.rows * p.parts * 2);
    hipLaunchKernelGGL((k_distill_stats<KIND, PV>), grid_of((u64)a.rows * (p.parts + 1)), block, lds, st, a, p);
    if (p.joined) hipLaunchKernelGGL(k_distill_join, grid_of((u64)a.rows), dim3(1024), 0, st, a, p);
    hipLaunchKernelGGL((k_distill_apply<KIND, PV, PAST>), grid_of((u64)a.rows * blocks), block, lds, st, a, p, blocks);
    return hipGetLastError();
}

template <int KIND, bool PAST> static hipError_t launch_kind(const DistillArgs& a, void* scratch, hipStream_t st) {
    const size_t lds = teacher_bytes(a.teacher.top);
    const dim3 block(kPartThreads);
    if (a.have_stats) {
        const u32 blocks = (u32)parts_of(KIND, a.cols, kBackVecs);
        hipLaunchKernelGGL((k_distill_apply<KIND, kBackVecs, PAST>), grid_of((u64)a.rows * blocks), block, lds, st, a, Parts{}, blocks);
        return hipGetLastError();
    }
    if (takes_parts(KIND, a.rows, a.cols))
        return parts_of(KIND, a.cols, kFewVecs) <= kFewParts ? launch_parts<KIND, kFewVecs, PAST>(a, scratch, st)
                                                             : launch_parts<KIND, kBackVecs, PAST>(a, scratch, st);
    const u64 vecs = ((u64)a.cols + kPer<KIND> - 1) / kPer<KIND>;
    const dim3 grid = grid_of((u64)a.rows);
    if (!a.grad && vecs > 64 * 16) {
        // A loss alone needs nothing kept: half the registers and twice the rows on a CU (513 x 50021 f16: 20.8 -> 16.4 us; 2048 x
        // 30000 bf16 30.5 -> 25.8).  Rows that one wavefront's registers hold are kept all the same (4096 x 4000 f32 17 us, streamed
        // 21).  By 256 threads / 512: 300 x 16000 f32 8.8 / 9.4, 2048 x 30000 bf16 25.6 / 30.6.
        if (vecs <= 256 * 16) hipLaunchKernelGGL((k_distill_row<KIND, 256, false, false>), grid, dim3(256), lds, st, a);
        else hipLaunchKernelGGL((k_distill_row<KIND, 512, false, false>), grid, dim3(512), lds, st, a);
        return hipGetLastError();
    }
    // The fewest threads whose registers hold the row: barriers of fewer wavefronts, more rows on a CU.  The fewer / the more, us: 64 or 256
    // threads 16 x 1000 f32, 64 entries 9.7 / 10.7, 4096 x 1000 19 / 42, 4096 x 4000 29 / 47; 256 or 512 2048 x 16000 66 / 75; 512 or 1024 2048
    // x 32000 116 / 159.  Hundreds of entries are weighed and looked through by one wavefront then, which few rows do not cover:
    // 300 x 4000 f32, 256 entries 40 / 18, 1024 rows 44 / 26, 4096 72 / 76.
    if (vecs <= 64 * 16) hipLaunchKernelGGL((k_distill_row<KIND, 64, true, PAST>), grid, dim3(64), lds, st, a);
    else if (vecs <= 256 * 16) hipLaunchKernelGGL((k_distill_row<KIND, 256, true, PAST>), grid, dim3(256), lds, st, a);
    else if (vecs <= 512 * 16) hipLaunchKernelGGL((k_distill_row<KIND, 512, true, PAST>), grid, dim3(512), lds, st, a);
    else if (vecs <= 1024 * 16) hipLaunchKernelGGL((k_distill_row<KIND, 1024, true, PAST>), grid, dim3(1024), lds, st, a);
    else hipLaunchKernelGGL((k_distill_row<KIND, 1024, false, PAST>), grid, dim3(1024), lds, st, a);
    return hipGetLastError();
}

template <int KIND> static hipError_t launch_kind(const DistillArgs& a, void* scratch, hipStream_t st) {
    const bool past = a.grad && (u64)a.rows * a.cols * kSize<KIND> >= kPastBytes;
    return past ? launch_kind<KIND, true>(a, scratch, st) : launch_kind<KIND, false>(a, scratch, st);
}

hipError_t launch_distill(int kind, const DistillArgs& a, void* scratch, hipStream_t st) {
    switch (kind) {
        case kScoreF32: return launch_kind<kScoreF32>(a, scratch, st);
        case kScoreF16: return launch_kind<kScoreF16>(a, scratch, st);
        case kScoreBF16: return launch_kind<kScoreBF16>(a, scratch, st);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_distill_state(const float2* A, int n, const TeacherArgs& te, int64_t rows, double* f, int64_t f_stride, float2* S, int paired, hipStream_t st,
                                const Residues* res, int rowdep) {
    if (S) hipLaunchKernelGGL(k_distill_zero, grid_of((((u64)rows << n) + 255) / 256), dim3(256), 0, st, A, n, (u64)rows << n, S, paired);
    hipLaunchKernelGGL(k_distill_state, grid_of((u64)rows), dim3(256), teacher_bytes(te.top), st, A, n, te, (u64)rows, f, (u64)f_stride, S,
                       paired ? 2 : 1, paired ? 1 : 0, res ? *res : Residues{nullptr, 0, 0, 0}, rowdep);
    return hipGetLastError();
}

}  // namespace qsv
