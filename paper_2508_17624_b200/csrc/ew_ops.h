// Shared host side of the stand-alone operators (grouped products, 4-bit matrix-vector products, SwiGLU): what they
// need to know of a device, argument checks, tensor maps.  These operators take no pool: everything they work on is
// passed in, and they keep nothing between calls but the constants of a device.
#pragma once
#include <cuda.h>
#include <cuda_runtime_api.h>

#include <cstdint>
#include <string>

#include "ew_internal.h"

namespace ew {
namespace ops {

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Bits of the operators' device error word (one per device): 2 = a bounded wait expired, 4 = an index that the call
// was given (an offset, a slot) lies outside its range and was clamped or skipped.
constexpr int kErrBadIndex = 4;

struct Device {
    int sm_count = 0;
    int *err = nullptr;              // device address of the error word
    EncodeTiled encode = nullptr;
};

// The device's constants, resolved on first use (thread-safe).  The caller has made the device current.
ew_status_t device_state(int device, const Device **out);

// Waits for the device and takes one status' bits out of its error word.
ew_status_t take_error(const Device &d, int *bits);

// Per-file attributes of the operators' kernels, set once per device by device_state().
int grouped_setup();
int quant_setup();
int swiglu_setup();

inline bool is_16bit(int dtype) { return dtype == EW_BF16 || dtype == EW_FP16; }
inline int elem_bytes(int dtype) { return dtype == EW_FP32 ? 4 : 2; }
inline CUtensorMapDataType map_type(int dtype) {
    return dtype == EW_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
}

// Whether `count` row-major matrices [rows, width] keep their rows apart: they lie one behind the other, or take turns row by row
// (as the middle dimension of a [rows, count, width] tensor).
inline bool rows_apart(int64_t count, int64_t stride, int64_t rows, int64_t ld, int64_t width) {
    return count < 2 || stride >= (__int128)(rows - 1) * ld + width || (stride >= width && ld >= (__int128)(count - 1) * stride + width);
}

inline ew_status_t refuse(const char *why) {
    set_last_error(why);
    return EW_ERR_INVALID_ARG;
}

// Tiled descriptor; dims and box innermost first, strides in bytes for dimensions 1 and up.
inline ew_status_t encode_map(const Device &d, CUtensorMap *out, CUtensorMapDataType type, const void *base, int rank,
                              const uint64_t *dims, const uint64_t *strides, const uint32_t *box, CUtensorMapSwizzle swizzle) {
    cuuint64_t gdim[5], gstride[5];
    cuuint32_t bx[5], estr[5];
    for (int i = 0; i < rank; ++i) {
        gdim[i] = dims[i];
        bx[i] = box[i];
        estr[i] = 1;
        if (i) gstride[i - 1] = strides[i - 1];
    }
    const CUresult r = d.encode(out, type, (cuuint32_t)rank, const_cast<void *>(base), gdim, gstride, bx, estr,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r == CUDA_SUCCESS) return EW_OK;
    set_last_error("cuTensorMapEncodeTiled failed with code " + std::to_string((int)r));
    return EW_ERR_CUDA;
}

inline ew_status_t launched(int rc, const char *what) {
    if (rc == 0) return EW_OK;
    (void)cudaGetLastError();                            // reported here: not once more by the thread's next call that asks
    set_last_error(std::string(what) + ": " + cudaGetErrorString((cudaError_t)rc));
    return EW_ERR_CUDA;
}

}  // namespace ops
}  // namespace ew
