// C boundary of the operators on caller buffers that make up a classifier's head: checks of arguments, then one launcher.
// See include/edl.h for the contract of every call.
#include <hip/hip_runtime.h>

#include <initializer_list>

#include "graph.h"
#include "operators.h"

using namespace edl;

namespace {

// A launch has fewer than 2^32 work items: element-wise ones have one for up to four pieces of eight elements, others a
// block of 256 for a row.  kMaxTiles is counted in tiles of 128x128; a block of the classifier's products has 512 threads, but so many
// tiles are 256x256 ones, a quarter as many, unless one side is at most 1,792 long (longer ones fill them to three quarters): 14 tiles by at most 2^17.
constexpr int64_t kMaxPieces = 1ll << 33, kMaxRows = 1ll << 23, kMaxDim = 1 << 16, kMaxClasses = 1 << 24, kMaxTiles = 1 << 23;

int launched() {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return EDL_OK;
    set_error("launch failed: %s", hipGetErrorString(e));
    return EDL_EHIP;
}

bool known_dtype(int32_t dtype) {
    if (dtype == EDL_DTYPE_F32 || dtype == EDL_DTYPE_BF16) return true;
    set_error("unknown dtype %d", dtype);
    return false;
}

bool element_aligned(int32_t dtype, const void* p) { return (uintptr_t)p % (dtype == EDL_DTYPE_BF16 ? 2 : 4) == 0; }

// rows of `cols` elements, ld elements apart
bool rows_ok(const char* what, int32_t dtype, const void* p, int64_t rows, int64_t cols, int64_t ld) {
    if (!p) { set_error("%s is NULL", what); return false; }
    if (!element_aligned(dtype, p)) { set_error("%s is not aligned to its elements", what); return false; }
    if (rows > 1 && ld < cols) { set_error("rows of %s overlap: %lld elements, %lld apart", what, (long long)cols, (long long)ld); return false; }
    if (ld < 0 || ld > INT32_MAX) { set_error("rows of %s are %lld elements apart", what, (long long)ld); return false; }
    return true;
}

}  // namespace

extern "C" {

int32_t edl_dropout_key(uint64_t seed, int64_t step, int32_t layer, uint64_t* out_key) {
    if (!out_key) { set_error("null argument"); return EDL_EINVAL; }
    if (step < 0 || layer < 0) { set_error("negative step or layer"); return EDL_EINVAL; }
    *out_key = dropout_key(seed, step, layer);
    return EDL_OK;
}

int32_t edl_dropout(int32_t dtype, const void* dev_x, int64_t ldx, void* dev_y, int64_t ldy, int64_t rows, int64_t cols, float rate,
                    uint64_t key, int64_t first_row, void* hip_stream) {
    if (!known_dtype(dtype)) return EDL_EINVAL;
    if (rows < 0 || cols < 0 || first_row < 0) { set_error("negative rows, cols or first_row"); return EDL_EINVAL; }
    if (!(rate >= 0.f && rate < 1.f)) { set_error("the rate must lie in [0, 1)"); return EDL_EINVAL; }
    if (rows == 0 || cols == 0) return EDL_OK;
    if (!rows_ok("x", dtype, dev_x, rows, cols, ldx) || !rows_ok("y", dtype, dev_y, rows, cols, ldy)) return EDL_EINVAL;
    if (dev_x == dev_y && rows > 1 && ldx != ldy) { set_error("in place, x and y need the same ld"); return EDL_EINVAL; }
    if (cols > INT32_MAX || rows > kMaxPieces / ((cols + 7) / 8)) { set_error("%lld x %lld elements are too many", (long long)rows, (long long)cols); return EDL_ERANGE; }
    launch_dropout(dtype, dev_x, ldx, dev_y, ldy, rows, cols, rate, key, (uint64_t)first_row, (hipStream_t)hip_stream);
    return launched();
}

// what the calls over rows of logits have in common; EDL_OK if there is something to do
static int32_t check_logits(int32_t dtype, int64_t rows, int64_t classes) {
    if (!known_dtype(dtype)) return EDL_EINVAL;
    if (rows < 0 || classes <= 0) { set_error("rows must not be negative, classes positive"); return EDL_EINVAL; }
    if (classes > INT32_MAX || rows > kMaxRows || rows * ((classes + 7) / 8) > kMaxPieces) { set_error("%lld x %lld logits are too many", (long long)rows, (long long)classes); return EDL_ERANGE; }
    return EDL_OK;
}

static bool vectors_aligned(std::initializer_list<const void*> v) {
    for (const void* p : v)
        if ((uintptr_t)p % 4) { set_error("a vector is not aligned to its elements"); return false; }
    return true;
}

int32_t edl_log_probs_workspace(int64_t rows, int64_t classes, int32_t k, int64_t* out_bytes) {
    if (!out_bytes) { set_error("null argument"); return EDL_EINVAL; }
    const int32_t rc = check_logits(EDL_DTYPE_F32, rows, classes);
    if (rc) return rc;
    if (k < 0 || k > kMaxTop || k > classes) { set_error("k=%d outside [0, min(%d, classes)]", k, kMaxTop); return EDL_EINVAL; }
    *out_bytes = (int64_t)plan_log_probs(rows, classes, k).bytes;
    return EDL_OK;
}

int32_t edl_log_probs(int32_t dtype, const void* dev_logits, int64_t ld, int64_t rows, int64_t classes, const int32_t* dev_targets, int32_t k,
                      float* dev_log_prob, float* dev_entropy, float* dev_lse, float* dev_top_log_prob, int32_t* dev_top_class,
                      void* dev_work, size_t work_bytes, void* hip_stream) {
    const int32_t rc = check_logits(dtype, rows, classes);
    if (rc) return rc;
    if (k < 0 || k > kMaxTop || k > classes) { set_error("k=%d outside [0, min(%d, classes)]", k, kMaxTop); return EDL_EINVAL; }
    if (rows == 0) return EDL_OK;
    if (!rows_ok("logits", dtype, dev_logits, rows, classes, ld)) return EDL_EINVAL;
    if (!dev_entropy || !dev_lse || (dev_targets && !dev_log_prob) || (k > 0 && (!dev_top_log_prob || !dev_top_class))) { set_error("null argument"); return EDL_EINVAL; }
    if (!vectors_aligned({dev_targets, dev_log_prob, dev_entropy, dev_lse, dev_top_log_prob, dev_top_class})) return EDL_EINVAL;
    const LogProbsPlan p = plan_log_probs(rows, classes, k);
    if (work_bytes < p.bytes) { set_error("workspace of %zu bytes is smaller than the %zu needed", work_bytes, p.bytes); return EDL_ENOMEM; }
    if (p.bytes > 0 && (!dev_work || (uintptr_t)dev_work % 16)) { set_error("the workspace must be 16-byte aligned"); return EDL_EINVAL; }
    launch_log_probs(dtype, dev_logits, ld, rows, classes, dev_targets, k, LogProbsOut{dev_log_prob, dev_entropy, dev_lse, dev_top_log_prob, dev_top_class},
                     dev_work, (hipStream_t)hip_stream);
    return launched();
}

int32_t edl_log_probs_backward(int32_t dtype, const void* dev_logits, int64_t ld, int64_t rows, int64_t classes, const int32_t* dev_targets,
                               const float* dev_lse, const float* dev_entropy, const float* dev_dlog_prob, const float* dev_dentropy,
                               void* dev_dlogits, int64_t ldd, void* hip_stream) {
    const int32_t rc = check_logits(dtype, rows, classes);
    if (rc) return rc;
    if (rows == 0) return EDL_OK;
    if (!rows_ok("logits", dtype, dev_logits, rows, classes, ld) || !rows_ok("dlogits", dtype, dev_dlogits, rows, classes, ldd)) return EDL_EINVAL;
    if (dev_logits == dev_dlogits && rows > 1 && ld != ldd) { set_error("in place, logits and dlogits need the same ld"); return EDL_EINVAL; }
    if (!dev_lse || (dev_dentropy && !dev_entropy) || (dev_dlog_prob && !dev_targets)) { set_error("null argument"); return EDL_EINVAL; }
    if (!vectors_aligned({dev_targets, dev_lse, dev_entropy, dev_dlog_prob, dev_dentropy})) return EDL_EINVAL;
    launch_log_probs_grad(dtype, dev_logits, ld, rows, classes, dev_targets, dev_lse, dev_entropy, dev_dlog_prob, dev_dentropy, dev_dlogits, ldd,
                          (hipStream_t)hip_stream);
    return launched();
}

// what the calls over features and classifier weights have in common
static int32_t check_classifier(int32_t dtype, int64_t rows, int64_t dim, int64_t classes) {
    if (!known_dtype(dtype)) return EDL_EINVAL;
    if (rows < 0 || dim <= 0 || classes <= 0) { set_error("rows must not be negative, dim and classes positive"); return EDL_EINVAL; }
    if (rows > kMaxRows || dim > kMaxDim || classes > kMaxClasses || rows * dim > (1ll << 29) || classes * dim > (1ll << 33) ||
        ((rows + 127) / 128) * ((classes + 127) / 128) > kMaxTiles) {
        set_error("%lld rows of %lld features for %lld classes are too many", (long long)rows, (long long)dim, (long long)classes);
        return EDL_ERANGE;
    }
    return EDL_OK;
}

// (of a single row, ld means nothing)
static ClassifierCall classifier_call(int32_t dtype, const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias, int64_t rows, int64_t dim,
                                      int64_t classes, const int32_t* targets, void* work) {
    return ClassifierCall{dtype, x, rows == 1 ? dim : ldx, w, classes == 1 ? dim : ldw, bias, rows, dim, classes, targets, work};
}

static int32_t check_work(const ClassifierCall& c, bool backward, size_t work_bytes) {
    const size_t need = classifier_work_bytes(c, backward);
    if (work_bytes < need) { set_error("workspace of %zu bytes is smaller than the %zu needed", work_bytes, need); return EDL_ENOMEM; }
    if (need > 0 && (!c.work || (uintptr_t)c.work % 256)) { set_error("the workspace must be 256-byte aligned"); return EDL_EINVAL; }
    return EDL_OK;
}

int32_t edl_classifier_workspace(int32_t dtype, const void* dev_x, int64_t ldx, const void* dev_w, int64_t ldw, int64_t rows, int64_t dim,
                                 int64_t classes, int32_t backward, int64_t* out_bytes) {
    if (!out_bytes) { set_error("null argument"); return EDL_EINVAL; }
    const int32_t rc = check_classifier(dtype, rows, dim, classes);
    if (rc) return rc;
    const ClassifierCall c = classifier_call(dtype, dev_x, ldx, dev_w, ldw, nullptr, rows, dim, classes, nullptr, nullptr);
    *out_bytes = rows == 0 ? 0 : (int64_t)classifier_work_bytes(c, backward != 0);
    return EDL_OK;
}

int32_t edl_classifier_log_probs(int32_t dtype, const void* dev_x, int64_t ldx, const void* dev_w, int64_t ldw, const float* dev_bias, int64_t rows,
                                 int64_t dim, int64_t classes, const int32_t* dev_targets, float* dev_log_prob, float* dev_entropy, float* dev_lse,
                                 void* dev_work, size_t work_bytes, void* hip_stream) {
    int32_t rc = check_classifier(dtype, rows, dim, classes);
    if (rc) return rc;
    if (rows == 0) return EDL_OK;
    if (!rows_ok("x", dtype, dev_x, rows, dim, ldx) || !rows_ok("w", dtype, dev_w, classes, dim, ldw)) return EDL_EINVAL;
    if (!dev_entropy || !dev_lse || (dev_targets && !dev_log_prob)) { set_error("null argument"); return EDL_EINVAL; }
    if (!vectors_aligned({dev_bias, dev_targets, dev_log_prob, dev_entropy, dev_lse})) return EDL_EINVAL;
    const ClassifierCall c = classifier_call(dtype, dev_x, ldx, dev_w, ldw, dev_bias, rows, dim, classes, dev_targets, dev_work);
    rc = check_work(c, false, work_bytes);
    if (rc) return rc;
    launch_classifier(c, ClassifierOut{dev_log_prob, dev_entropy, dev_lse}, (hipStream_t)hip_stream);
    return launched();
}

int32_t edl_classifier_log_probs_backward(int32_t dtype, const void* dev_x, int64_t ldx, const void* dev_w, int64_t ldw, const float* dev_bias,
                                          int64_t rows, int64_t dim, int64_t classes, const int32_t* dev_targets, const float* dev_lse,
                                          const float* dev_entropy, const float* dev_dlog_prob, const float* dev_dentropy, void* dev_dx, int64_t lddx,
                                          float* dev_dw, int64_t lddw, float* dev_dbias, void* dev_work, size_t work_bytes, void* hip_stream) {
    int32_t rc = check_classifier(dtype, rows, dim, classes);
    if (rc) return rc;
    if (!rows_ok("dw", EDL_DTYPE_F32, dev_dw, classes, dim, lddw)) return EDL_EINVAL;
    if (rows > 0) {
        if (!rows_ok("x", dtype, dev_x, rows, dim, ldx) || !rows_ok("w", dtype, dev_w, classes, dim, ldw) || !rows_ok("dx", dtype, dev_dx, rows, dim, lddx))
            return EDL_EINVAL;
        if (!dev_lse || (dev_dentropy && !dev_entropy) || (dev_dlog_prob && !dev_targets)) { set_error("null argument"); return EDL_EINVAL; }
    }
    if (!vectors_aligned({dev_bias, dev_targets, dev_lse, dev_entropy, dev_dlog_prob, dev_dentropy, dev_dbias})) return EDL_EINVAL;
    if (rows > 0 && (dev_dx == dev_x || dev_dx == dev_w || (const void*)dev_dw == dev_w || (const void*)dev_dw == dev_x)) {
        set_error("gradients cannot take the place of what they are computed from");
        return EDL_EINVAL;
    }
    const ClassifierCall c = classifier_call(dtype, dev_x, ldx, dev_w, ldw, dev_bias, rows, dim, classes, dev_targets, dev_work);
    if (rows > 0) {
        rc = check_work(c, true, work_bytes);
        if (rc) return rc;
    }
    launch_classifier_grads(c, ClassifierGrads{dev_lse, dev_entropy, dev_dlog_prob, dev_dentropy, dev_dx, lddx, dev_dw, lddw, dev_dbias}, (hipStream_t)hip_stream);
    return launched();
}

}  // extern "C"
