// Checks of the requests on rows of scores: host only, no device is asked.
#pragma once
#include <cstdint>

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

}  // namespace qsv
