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

// ---- log probabilities --------------------------------------------------------
constexpr int kMaxTop = 64;        // one lane of a wave each
struct LogProbsPlan { int parts; int64_t part; size_t sums_bytes, bytes; };      // parts of a row; bytes of workspace
LogProbsPlan plan_log_probs(int64_t rows, int64_t classes, int k);
struct LogProbsOut { float *log_prob, *entropy, *lse, *top_value; int32_t* top_class; };
void launch_log_probs(int dtype, const void* logits, int64_t ld, int64_t rows, int64_t classes, const int32_t* targets, int k,
                      const LogProbsOut& out, void* work, hipStream_t st);
void launch_log_probs_grad(int dtype, const void* logits, int64_t ld, int64_t rows, int64_t classes, const int32_t* targets, const float* lse,
                           const float* entropy, const float* dlog_prob, const float* dentropy, void* dlogits, int64_t ldd, hipStream_t st);

// ---- classifier ------------------------------------------------------------------
struct ClassifierCall {
    int dtype;
    const void* x;             // [rows][dim]
    int64_t ldx;
    const void* w;             // [classes][dim]
    int64_t ldw;
    const float* bias;         // [classes] or null
    int64_t rows, dim, classes;
    const int32_t* targets;
    void* work;
};
struct ClassifierOut { float *log_prob, *entropy, *lse; };
struct ClassifierGrads {
    const float *lse, *entropy, *dlog_prob, *dentropy;
    void* dx;                  // [rows][dim]
    int64_t lddx;
    float* dw;                 // [classes][dim]
    int64_t lddw;
    float* dbias;              // [classes] or null
};
// for operands that lie as x and w do; null ones: however they lie
size_t classifier_work_bytes(const ClassifierCall& c, bool backward);
void launch_classifier(const ClassifierCall& c, const ClassifierOut& out, hipStream_t st);
void launch_classifier_grads(const ClassifierCall& c, const ClassifierGrads& d, hipStream_t st);

}  // namespace edl
