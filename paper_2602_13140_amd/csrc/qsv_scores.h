// Launch interface of the kernels on rows of scores, probabilities or amplitudes (gfx950 only): sampling after filters,
// distillation from a teacher's top logits, penalties, biases and masks.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "qsv_kernels.h"

namespace qsv {

// What a row holds (the values of qsv_scores_kind).
enum ScoreKind { kScoreF32 = 1, kScoreF16 = 2, kScoreBF16 = 3, kScoreProbs = 4, kScoreState = 5 };

struct SampleArgs {
    const void* scores;          // row r starts r * stride elements further
    int64_t rows, stride;
    uint32_t cols;
    int bits;                    // S: a weight of 1 is 2^S
    const float* temperature;    // [rows], or NULL: off, as the next three
    const int* top_k;
    const float* top_p;
    const float* min_p;
    const double* uniforms;      // [rows][shots]
    int64_t shots;
    long long* out;              // [rows][shots]
    float* logp;                 // [rows][shots] or NULL
    int* kept;                   // [rows] or NULL
};

// Bytes of workspace that launch_sample_scores needs for such rows (0: none).
size_t sample_scratch_bytes(int64_t rows, int64_t cols, int64_t shots);
hipError_t launch_sample_scores(int kind, const SampleArgs& a, void* scratch, hipStream_t st);

// A teacher's top logits of a row, and what they make of it.
struct TeacherArgs {
    const int* idx;              // [rows][top]
    const float* logits;         // [rows][top]
    const float* lse;            // [rows], or NULL: normalised over the entries given
    int top;
    double inv_t;                // 1 / T
};

struct DistillArgs {
    const void* scores;
    int64_t rows, stride;
    uint32_t cols;
    TeacherArgs teacher;
    float* loss;                 // [rows] or NULL
    float* stats;                // [rows][2] or NULL
    int have_stats;              // stats are an input
    const float* grad_loss;      // [rows] or NULL: 1
    void* grad;                  // of the scores' type, or NULL
    int64_t grad_stride;
};

size_t distill_scratch_bytes(int64_t rows, int64_t cols);
hipError_t launch_distill(int kind, const DistillArgs& a, void* scratch, hipStream_t st);

// Rows of 2^n amplitudes against a teacher (its arrays start at the first of them): the loss of row r to f[r * f_stride]
// (f may be NULL), and, where S is not NULL, lambda to S: row r, or (paired) psi to row 2r and lambda to row 2r + 1.
// res, rowdep: see launch_expz_finish.
hipError_t launch_distill_state(const float2* A, int n, const TeacherArgs& te, int64_t rows, double* f, int64_t f_stride,
                                float2* S, int paired, hipStream_t st, const Residues* res = nullptr, int rowdep = 0);

// Rows of scores after penalties, biases and masks; the backward pass has the gradients behind them.
struct AdjustArgs {
    const void* scores;          // row r starts r * stride elements further
    void* out;
    int64_t rows, stride, out_stride;
    uint32_t cols;
    int n_prior;                 // earlier outcomes of a row: at most so many
    const int* prior;            // row r starts r * prior_stride further
    int64_t prior_stride;
    const int* prior_len;        // [rows] or NULL: n_prior
    const int* prompt_len;       // [rows] or NULL: 0
    const float* repetition;     // [rows], or NULL: off, as the next two
    const float* frequency;
    const float* presence;
    const float* bias;           // [cols] or NULL
    int n_entries;               // a row's own biases
    const int* entry_idx;        // [rows][n_entries]
    const float* entry_bias;     // [rows][n_entries], or NULL in the backward pass
    const unsigned* masks;       // [n_masks] rows of mask_stride words, or NULL
    int64_t n_masks, mask_stride;
    const int* mask_of;          // [rows] or NULL
    int mask_each;               // mask_of NULL: row r takes mask r, or (0) all take the one
    const void* grad_out;
    void* grad;                  // or NULL
    int64_t grad_out_stride, grad_stride;
    float* grad_bias;            // [cols] or NULL
    float* grad_entry;           // [rows][n_entries] or NULL
};

hipError_t launch_adjust(int kind, const AdjustArgs& a, hipStream_t st);
// Bytes of workspace for grad_bias.
size_t adjust_grad_scratch_bytes(int64_t rows, int64_t cols);
hipError_t launch_adjust_grad(int kind, const AdjustArgs& a, void* scratch, hipStream_t st);

}  // namespace qsv
