// Checks of the requests on rows of scores and on lists of tensors: host only, no device is asked.
#pragma once
#include <algorithm>
#include <cstdint>
#include <memory>
#include <new>
#include <numeric>

#include "qsv.h"

namespace qsv {

constexpr int64_t kMostRows = (int64_t)1 << 24, kMostCols = (int64_t)1 << 30, kMostShots = (int64_t)1 << 32,
                  kMostStride = (int64_t)1 << 36;

inline int score_bytes(int kind) { return kind == QSV_S_STATE ? 8 : kind == QSV_S_F16 || kind == QSV_S_BF16 ? 2 : 4; }

// Rows of scores in memory: what is wrong with them, or NULL.
inline const char* check_rows(int kind, const void* scores, int64_t rows, int64_t cols, int64_t stride) {
    if (rows < 0 || rows > kMostRows) return "rows must be in 0..2^24";
    if (cols < 1 || cols > kMostCols) return "cols must be in 1..2^30";
    if (rows == 0) return nullptr;
    if (!scores) return "scores_dev is NULL";
    if ((uintptr_t)scores % score_bytes(kind)) return "scores_dev must be aligned to its element";
    if (rows > 1 && (stride < cols || stride > kMostStride)) return "row_stride must be in cols..2^36";
    return nullptr;
}

// What is wrong with a request of qsv_sample on a context of batch samples of n qubits, or NULL.
inline const char* check_sample(const qsv_sample_req* q, int n, int64_t batch) {
    if (!q) return "req is NULL";
    if (q->reserved != 0) return "reserved must be 0";
    if (q->kind < QSV_S_F32 || q->kind > QSV_S_STATE) return "unknown kind of scores";
    if (q->kind == QSV_S_STATE) {
        if (q->scores_dev) return "scores_dev must be NULL for the context's state";
        if (q->rows != batch || q->cols != ((int64_t)1 << n)) return "the context's state has batch rows of 2^n outcomes";
    } else if (const char* why = check_rows(q->kind, q->scores_dev, q->rows, q->cols, q->row_stride)) {
        return why;
    }
    if (q->shots < 0 || q->shots > kMostShots || q->rows * q->shots > kMostShots)
        return "shots must be >= 0 with rows * shots <= 2^32";
    if (q->rows > 0 && q->shots > 0 && (!q->uniforms_dev || !q->out_dev)) return "uniforms_dev or out_dev is NULL";
    return nullptr;
}

// What is wrong with a teacher, or NULL.
inline const char* check_teacher(const qsv_teacher* t) {
    if (!t) return "teacher is NULL";
    if (t->reserved != 0) return "reserved must be 0";
    if (t->n_top < 1 || t->n_top > 1024) return "n_top must be in 1..1024";
    if (!t->top_idx_dev || !t->top_logits_dev) return "top_idx_dev or top_logits_dev is NULL";
    // further out the scores' factor 1 / T would leave the range of 32 bits, and 0 times infinity make rows NaN
    if (!(t->temperature >= 0x1p-100) || !(t->temperature <= 0x1p100)) return "temperature must be in 2^-100..2^100";
    return nullptr;
}

// The bytes from the first row's start to the last row's end.
inline uint64_t span_bytes(int kind, int64_t rows, int64_t cols, int64_t stride) {
    return ((uint64_t)(rows - 1) * (rows > 1 ? (uint64_t)stride : 0) + (uint64_t)cols) * (uint64_t)score_bytes(kind);
}

// What is wrong with a request of qsv_distill, or NULL.
inline const char* check_distill(const qsv_distill_req* q, const qsv_teacher* t) {
    if (!q) return "req is NULL";
    if (q->kind != QSV_S_F32 && q->kind != QSV_S_F16 && q->kind != QSV_S_BF16) return "kind must be one of the three types of scores";
    if (q->have_stats != 0 && q->have_stats != 1) return "have_stats must be 0 or 1";
    if (const char* why = check_rows(q->kind, q->scores_dev, q->rows, q->cols, q->row_stride)) return why;
    if (q->rows == 0) return nullptr;
    if (const char* why = check_teacher(t)) return why;
    if (q->have_stats && (!q->stats_dev || q->loss_dev)) return "have_stats = 1 needs stats_dev, and no loss_dev";
    if (q->grad_dev) {
        if ((uintptr_t)q->grad_dev % score_bytes(q->kind)) return "grad_dev must be aligned to its element";
        if (q->rows > 1 && (q->grad_stride < q->cols || q->grad_stride > kMostStride)) return "grad_stride must be in cols..2^36";
        const uint64_t s = (uintptr_t)q->scores_dev, g = (uintptr_t)q->grad_dev;
        const bool over = s < g + span_bytes(q->kind, q->rows, q->cols, q->grad_stride) && g < s + span_bytes(q->kind, q->rows, q->cols, q->row_stride);
        if (over && (s != g || (q->rows > 1 && q->row_stride != q->grad_stride)))
            return "grad_dev must be the scores themselves or not overlap them";
    }
    return nullptr;
}

// Rows that results go to, beside rows that are read: what is wrong with them, or NULL.  same: they may be those rows.
inline const char* check_apart(int kind, int64_t rows, int64_t cols, const void* from, int64_t from_stride, const void* to, int64_t to_stride, bool same) {
    const uint64_t s = (uintptr_t)from, g = (uintptr_t)to;
    if (!from || s >= g + span_bytes(kind, rows, cols, to_stride) || g >= s + span_bytes(kind, rows, cols, from_stride)) return nullptr;
    if (same && s == g && (rows == 1 || from_stride == to_stride)) return nullptr;
    return same ? "the result must be the rows themselves or not overlap them" : "the gradient must not overlap the scores";
}

inline const char* check_out(int kind, int64_t rows, int64_t cols, const void* out, int64_t stride) {
    if (!out) return "the result's address is NULL";
    if ((uintptr_t)out % score_bytes(kind)) return "results must be aligned to their element";
    if (rows > 1 && (stride < cols || stride > kMostStride)) return "the stride of results must be in cols..2^36";
    return nullptr;
}

constexpr int64_t kMostPrior = (int64_t)1 << 20, kMostEntries = 1023, kMostMasks = (int64_t)1 << 24;

// What a request of qsv_adjust says about history, entries and masks, with at least one row.
inline const char* check_adjust_lists(const qsv_adjust_req* q, bool back) {
    if (q->n_prior < 0 || q->n_prior > kMostPrior) return "n_prior must be in 0..2^20";
    if (q->n_prior > 0) {
        if (!q->prior_dev) return "prior_dev is NULL";
        if (q->rows > 1 && (q->prior_stride < q->n_prior || q->prior_stride > kMostStride)) return "prior_stride must be in n_prior..2^36";
    }
    if (q->n_entries < 0 || q->n_entries > kMostEntries) return "n_entries must be in 0..1023";
    if (q->n_entries > 0 && (!q->entry_idx_dev || (!back && !q->entry_bias_dev))) return "entry_idx_dev or entry_bias_dev is NULL";
    if (q->masks_dev) {
        if (q->n_masks < 1 || q->n_masks > kMostMasks) return "n_masks must be in 1..2^24";
        if (q->n_masks > 1 && (q->mask_stride < (q->cols + 31) / 32 || q->mask_stride > kMostStride)) return "mask_stride must be in ceil(cols / 32)..2^36";
        if (!q->mask_of_dev && q->n_masks != 1 && q->n_masks != q->rows) return "without mask_of_dev there must be one mask, or one for each row";
    }
    return nullptr;
}

inline bool score_kind(int kind) { return kind == QSV_S_F32 || kind == QSV_S_F16 || kind == QSV_S_BF16; }

// What is wrong with a request of qsv_adjust, or NULL.
inline const char* check_adjust(const qsv_adjust_req* q) {
    if (!q) return "req is NULL";
    if (!score_kind(q->kind)) return "kind must be one of the three types of scores";
    if (const char* why = check_rows(q->kind, q->scores_dev, q->rows, q->cols, q->row_stride)) return why;
    if (q->rows == 0) return nullptr;
    if (const char* why = check_out(q->kind, q->rows, q->cols, q->out_dev, q->out_stride)) return why;
    if (const char* why = check_apart(q->kind, q->rows, q->cols, q->scores_dev, q->row_stride, q->out_dev, q->out_stride, true)) return why;
    return check_adjust_lists(q, false);
}

// What is wrong with a request of qsv_adjust_grad, or NULL.
inline const char* check_adjust_grad(const qsv_adjust_req* q, const qsv_adjust_grad_req* g) {
    if (!q || !g) return "req or grad is NULL";
    if (!score_kind(q->kind)) return "kind must be one of the three types of scores";
    const bool scores = g->grad_dev && q->repetition_dev && q->n_prior > 0;      // they are read
    if (const char* why = check_rows(q->kind, scores ? q->scores_dev : g->grad_out_dev, q->rows, q->cols, scores ? q->row_stride : g->grad_out_stride)) return why;
    if (q->rows == 0) return nullptr;
    if (const char* why = check_adjust_lists(q, true)) return why;
    if (!g->grad_out_dev) return "grad_out_dev is NULL";
    if ((uintptr_t)g->grad_out_dev % score_bytes(q->kind)) return "grad_out_dev must be aligned to its element";
    if (q->rows > 1 && (g->grad_out_stride < q->cols || g->grad_out_stride > kMostStride)) return "grad_out_stride must be in cols..2^36";
    if (g->grad_entry_dev && q->n_entries == 0) return "grad_entry_dev without entries";
    if (!g->grad_dev) return nullptr;
    if (const char* why = check_out(q->kind, q->rows, q->cols, g->grad_dev, g->grad_stride)) return why;
    if (const char* why = check_apart(q->kind, q->rows, q->cols, g->grad_out_dev, g->grad_out_stride, g->grad_dev, g->grad_stride, true)) return why;
    return scores ? check_apart(q->kind, q->rows, q->cols, q->scores_dev, q->row_stride, g->grad_dev, g->grad_stride, false) : nullptr;
}

// ---- lists of tensors ------------------------------------------------------------------------------------------------
constexpr int64_t kMostTensors = 4096, kMostValues = (int64_t)1 << 38, kMostReach = (int64_t)1 << 56;

struct Span {                 // bytes; rows of `width` at `stride`
    uint64_t from, to, width, stride;
    bool written;
};

// Rows that lie between each other's, as columns of one buffer do: told apart by where they lie in a period that both strides are multiples
// of.  (A single row has the other's.  Exact where no two strides of several rows differ: extents that overlap have rows of both in one period.)
inline bool columns_apart(const Span& a, const Span& b) {      // a.from <= b.from
    const uint64_t period = std::gcd(a.stride, b.stride);
    if (period == 0) return false;
    const uint64_t behind = (b.from - a.from) % period;
    return behind >= a.width && behind + b.width <= period;
}

// Bytes from .. to - 1; the lowest bit of `from`, an even address, says that they are written.
struct Flat { uint64_t from, to; };

// Whether something that is written meets something else.  Lists at[k] .. end[k] - 1 are sorted where they are not (those of a program
// mostly are) and gone through side by side.  (48 tensors of a step 1.2 us, by one sort of all 4.4: as long as a launch.)
template <int LISTS> bool flats_meet(Flat* (&at)[LISTS], Flat* (&end)[LISTS]) {
    auto less = [](const Flat& a, const Flat& b) { return a.from < b.from; };
    for (int k = 0; k < LISTS; ++k)
        if (!std::is_sorted(at[k], end[k], less)) std::sort(at[k], end[k], less);
    uint64_t any = 0, written = 0;      // where what came so far ends
    for (;;) {
        int next = -1;
        for (int k = 0; k < LISTS; ++k)
            if (at[k] < end[k] && (next < 0 || at[k]->from < at[next]->from)) next = k;
        if (next < 0) return false;
        const Flat now = *at[next]++;
        const uint64_t from = now.from & ~(uint64_t)1;
        if (from < written || ((now.from & 1) && from < any)) return true;
        any = std::max(any, now.to);
        if (now.from & 1) written = std::max(written, now.to);
    }
}

// Whether rows whose extents overlap, sorted by their first bytes, meet where some of them are written: all against all in a common period
// of their strides, and pair by pair where that says so.
inline bool rows_meet(const Span* s, int64_t n, Span* open, Flat* room) {
    uint64_t period = 0;
    for (int64_t i = 0; i < n; ++i) period = std::gcd(period, s[i].stride);
    Flat* at[1] = {room};
    Flat* end[1] = {room};
    bool fits = period > 0;
    for (int64_t i = 0; fits && i < n; ++i) {
        const uint64_t from = (s[i].from - s[0].from) % period, to = from + s[i].width, bit = s[i].written ? 1u : 0u;
        fits = s[i].width <= period;
        *end[0]++ = Flat{from | bit, std::min(to, period)};
        if (to > period) *end[0]++ = Flat{bit, to - period};
    }
    if (fits && !flats_meet(at, end)) return false;
    int64_t before = 0;          // those that may reach over the one that is looked at
    for (int64_t i = 0; i < n; ++i) {
        int64_t left = 0;
        for (int64_t j = 0; j < before; ++j) {
            if (open[j].to <= s[i].from) continue;
            open[left++] = open[j];
            if ((open[j].written || s[i].written) && !columns_apart(open[j], s[i])) return true;
        }
        open[left++] = s[i];
        before = left;
    }
    return false;
}

// Whether something that is written meets something else; `open` has room for n, `room` for 2 n.  (Columns of one buffer, ms of the host, by one
// period / pair by pair: 512 tensors 0.011 / 0.48, 4096 0.10 / 30.)
inline bool spans_meet(Span* s, int64_t n, Span* open, Flat* room) {
    std::sort(s, s + n, [](const Span& a, const Span& b) { return a.from < b.from; });
    for (int64_t i = 0, j = 0; i < n; i = j) {
        uint64_t to = s[i].to;
        for (j = i + 1; j < n && s[j].from < to; ++j) to = std::max(to, s[j].to);
        if (j - i > 1 && rows_meet(s + i, j - i, open, room)) return true;
    }
    return false;
}

inline Span span_of(const qsv_tensor& t, bool written) {
    const uint64_t size = (uint64_t)score_bytes(t.kind), from = (uintptr_t)t.data_dev;
    const uint64_t stride = t.rows > 1 ? (uint64_t)t.row_stride : 0;
    return Span{from, from + ((uint64_t)(t.rows - 1) * stride + (uint64_t)t.cols) * size, (uint64_t)t.cols * size, stride * size, written};
}

// A gradient and where it goes, the same rows.
inline bool same_rows(const Span& a, const Span& b) { return a.from == b.from && a.to == b.to && a.stride == b.stride; }

// Whether the norm's four bytes meet the rows of a tensor.
inline bool norm_meets(const Span& s, const float* norm) {
    const uint64_t at = (uintptr_t)norm;
    if (!norm || at + 4 <= s.from || at >= s.to) return false;
    if (at < s.from || s.stride == 0) return true;
    const uint64_t behind = (at - s.from) % s.stride;
    return behind < s.width || behind + 4 > s.stride;
}

inline const char* check_tensor(const qsv_tensor& t) {
    if (t.reserved != 0) return "reserved must be 0";
    if (!score_kind(t.kind)) return "kind must be one of the three types of scores";
    int64_t values = 0;
    if (t.rows < 0 || t.cols < 0 || t.rows > kMostValues || t.cols > kMostValues || __builtin_mul_overflow(t.rows, t.cols, &values) || values > kMostValues)
        return "a tensor has rows and cols >= 0, and 2^38 values at most";
    if (t.rows == 0 || t.cols == 0) return nullptr;
    if (!t.data_dev) return "data_dev is NULL";
    if ((uintptr_t)t.data_dev & (score_bytes(t.kind) - 1)) return "data_dev must be aligned to its element";
    if (t.rows > 1 && (t.row_stride < t.cols || t.row_stride > kMostValues)) return "row_stride must be in cols..2^38";
    int64_t last = 0;      // so that addresses and extents do not wrap around
    if (t.rows > 1 && (__builtin_mul_overflow(t.rows - 1, t.row_stride, &last) || last > kMostReach)) return "a tensor's last row must start within 2^56 elements";
    return nullptr;
}

// What is wrong with a request of qsv_clip_grads, or NULL.
inline const char* check_clip(const qsv_tensor* grads, const qsv_tensor* outs, int64_t n, double max_norm, const float* norm = nullptr) {
    if (n < 0 || n > kMostTensors) return "a list has 0..4096 tensors";
    if (n > 0 && !grads) return "grads is NULL";
    if (!(max_norm >= 0.0)) return "max_norm must be >= 0";
    int64_t values = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (const char* why = check_tensor(grads[i])) return why;
        if ((values += grads[i].rows * grads[i].cols) > kMostValues) return "a list has 2^38 values at most";
        if (grads[i].rows && grads[i].cols && norm_meets(span_of(grads[i], false), norm)) return "norm_dev lies in a tensor";
        if (!outs) continue;
        if (const char* why = check_tensor(outs[i])) return why;
        if (outs[i].kind != grads[i].kind || outs[i].rows != grads[i].rows || outs[i].cols != grads[i].cols)
            return "outs must have the kinds and shapes of the gradients";
        if (outs[i].rows && outs[i].cols && norm_meets(span_of(outs[i], true), norm)) return "norm_dev lies in a tensor";
    }
    if (!outs && max_norm > 1.7976931348623157e308) return nullptr;      // nothing is written
    // from first byte to last, as most lists are apart already
    std::unique_ptr<Flat[]> flats(new (std::nothrow) Flat[(size_t)(2 * n) + 1]);
    if (!flats) return "out of host memory";
    Flat *at[2] = {flats.get(), flats.get() + n}, *end[2] = {at[0], at[1]};
    for (int64_t i = 0; i < n; ++i) {
        if (grads[i].rows == 0 || grads[i].cols == 0) continue;
        const Span g = span_of(grads[i], false);
        if (!outs) {
            *end[0]++ = Flat{g.from | 1u, g.to};
            continue;
        }
        const Span o = span_of(outs[i], true);
        *end[1]++ = Flat{o.from | 1u, o.to};
        if (!same_rows(g, o)) *end[0]++ = Flat{g.from, g.to};
    }
    if (!flats_meet(at, end)) return nullptr;
    // row by row
    std::unique_ptr<Span[]> spans(new (std::nothrow) Span[(size_t)(4 * n) + 1]);
    std::unique_ptr<Flat[]> room(new (std::nothrow) Flat[(size_t)(4 * n) + 1]);
    if (!spans || !room) return "out of host memory";
    int64_t m = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (grads[i].rows == 0 || grads[i].cols == 0) continue;
        const Span g = span_of(grads[i], !outs), o = outs ? span_of(outs[i], true) : g;
        spans[m++] = o;
        if (!same_rows(g, o)) spans[m++] = g;
    }
    return spans_meet(spans.get(), m, spans.get() + 2 * n, room.get()) ? "a tensor that is written overlaps another one" : nullptr;
}

// What is wrong with a request of qsv_adam_clipped, or NULL.
inline const char* check_adam_list(const qsv_adam_tensor* tensors, int64_t n, double max_norm, const float* norm = nullptr) {
    if (n < 0 || n > kMostTensors) return "a list has 0..4096 tensors";
    if (n > 0 && !tensors) return "tensors is NULL";
    if (!(max_norm >= 0.0)) return "max_norm must be >= 0";
    std::unique_ptr<Flat[]> flats(new (std::nothrow) Flat[(size_t)(4 * n) + 1]);
    if (!flats) return "out of host memory";
    int64_t m = 0, values = 0;
    const uint64_t place = (uintptr_t)norm;
    for (int64_t i = 0; i < n; ++i) m += tensors[i].count > 0;
    int64_t l = 0;
    for (int64_t i = 0; i < n; ++i) {
        const qsv_adam_tensor& t = tensors[i];
        if (t.reserved != 0) return "reserved must be 0";
        if (!score_kind(t.kind)) return "kind must be one of the three types of scores";
        if (t.count < 0 || t.count > kMostValues) return "count must be in 0..2^38";
        if ((values += t.count) > kMostValues) return "a list has 2^38 values at most";
        if (t.count == 0) continue;
        if (!t.param_dev || !t.grad_dev || !t.m_dev || !t.v_dev) return "param_dev, grad_dev, m_dev or v_dev is NULL";
        if (((uintptr_t)t.param_dev | (uintptr_t)t.m_dev | (uintptr_t)t.v_dev) % 4 || ((uintptr_t)t.grad_dev & (score_bytes(t.kind) - 1)))
            return "tensors must be aligned to their element";
        const void* at[4] = {t.param_dev, t.m_dev, t.v_dev, t.grad_dev};
        for (int k = 0; k < 4; ++k) {
            const uint64_t from = (uintptr_t)at[k], to = from + (uint64_t)t.count * (k < 3 ? 4 : score_bytes(t.kind));
            if (norm && place + 4 > from && place < to) return "norm_dev lies in a tensor";
            flats[k * m + l] = Flat{from | (k < 3 ? 1u : 0u), to};
        }
        ++l;
    }
    Flat *at[4], *end[4];
    for (int k = 0; k < 4; ++k) {
        at[k] = flats.get() + k * m;
        end[k] = at[k] + m;
    }
    return flats_meet(at, end) ? "a tensor that is written overlaps another one" : nullptr;
}

}  // namespace qsv
