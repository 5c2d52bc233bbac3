// C boundary of the operators on caller buffers that make up a classifier's head: checks of arguments, then one launcher.
// See include/edl.h for the contract of every call.
#include <hip/hip_runtime.h>

#include <cmath>

#include "graph.h"
#include "operators.h"

using namespace edl;

namespace {

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
    if (cols > INT32_MAX || rows > (1ll << 39) / ((cols + 7) / 8)) { set_error("%lld x %lld elements are too many", (long long)rows, (long long)cols); return EDL_ERANGE; }
    launch_dropout(dtype, dev_x, ldx, dev_y, ldy, rows, cols, rate, key, (uint64_t)first_row, (hipStream_t)hip_stream);
    return launched();
}

}  // extern "C"
