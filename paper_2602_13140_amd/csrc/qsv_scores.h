// Launch interface of the kernels on rows of scores, probabilities or amplitudes (gfx950 only): sampling after filters,
// distillation from a teacher's top logits.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

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

// Bytes of workspace that launch_sample needs for such rows (0: none).
size_t sample_scratch_bytes(int64_t rows, int64_t cols);
hipError_t launch_sample_scores(int kind, const SampleArgs& a, void* scratch, hipStream_t st);

}  // namespace qsv
