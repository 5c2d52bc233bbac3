// The operators of a classifier's head on caller buffers: dropout (k_dropout.hip), log probabilities of logits
// (k_log_probs.hip) and of features through a classifier (k_classifier.hip).  Launchers only queue work on `st`; arguments
// are checked by the C boundary (operators.cpp).
#pragma once
#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>

namespace edl {

// ---- dropout ----------------------------------------------------------------
// y[r][c] = kept(r, c) ? x[r][c] / (1 - rate) : 0, rows ldx / ldy elements apart; y may be x.  Whether an element is kept
// follows from key and its place (first_row + r, c) alone.
void launch_dropout(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, float rate, uint64_t key,
                    uint64_t first_row, hipStream_t st);
// The key of one layer's masks in one step of a job.
uint64_t dropout_key(uint64_t seed, int64_t step, int layer);

}  // namespace edl
