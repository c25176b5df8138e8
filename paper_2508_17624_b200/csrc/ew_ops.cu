// What the stand-alone operators keep per device: its size, the tensor-map encoder and one error word.
#include "ew_ops.h"

#include <atomic>
#include <mutex>

namespace ew {
namespace ops {
namespace {

constexpr int kMaxDevices = 64;
__device__ int g_operator_error[2];                  // the error word; what the last reader took from it

// Takes what one status can report out of the error word: an expired wait, or else the index.  What is not reported stays, and
// so does a bit that a kernel sets meanwhile.
__global__ void take_error_kernel(int *err) {
    const int seen = *(volatile int *)err, report = (seen & 2) ? 2 : seen;
    err[1] = atomicAnd(err, ~report) & report;
}

std::mutex g_mutex;
Device g_devices[kMaxDevices];
std::atomic<bool> g_ready[kMaxDevices];

ew_status_t resolve(Device *d, int device) {
    void *fn = nullptr, *err = nullptr;
    cudaDriverEntryPointQueryResult q;
    cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
    if (e == cudaSuccess && !fn) e = cudaErrorUnknown;
    if (e == cudaSuccess) e = cudaGetSymbolAddress(&err, g_operator_error);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&d->sm_count, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return launched((int)e, "operator set-up");
    d->encode = reinterpret_cast<EncodeTiled>(fn);
    d->err = static_cast<int *>(err);
    cudaFuncAttributes fa;
    return launched((int)cudaFuncGetAttributes(&fa, take_error_kernel) | grouped_setup() | quant_setup() | swiglu_setup() | blocks_setup() |
                    norm_setup(d) | scaled_setup(), "operator set-up");
}

}  // namespace

ew_status_t take_error(const Device &d, int *bits) {
    std::lock_guard<std::mutex> lock(g_mutex);       // (readers take turns at the second word)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = cfg.blockDim = dim3(1);
    ew_status_t s = launched((int)cudaDeviceSynchronize(), "cudaDeviceSynchronize");
    if (s == EW_OK) s = launched((int)cudaLaunchKernelEx(&cfg, take_error_kernel, d.err), "operator error");
    if (s == EW_OK) s = launched((int)cudaMemcpy(bits, d.err + 1, 4, cudaMemcpyDeviceToHost), "cudaMemcpy");
    return s;
}

ew_status_t device_state(int device, const Device **out) {
    if (device >= kMaxDevices) return refuse("device ordinal out of range");
    if (!g_ready[device].load(std::memory_order_acquire)) {
        std::lock_guard<std::mutex> lock(g_mutex);
        if (!g_ready[device].load(std::memory_order_relaxed)) {
            const ew_status_t s = resolve(&g_devices[device], device);
            if (s != EW_OK) return s;
            g_ready[device].store(true, std::memory_order_release);
        }
    }
    *out = &g_devices[device];
    return EW_OK;
}

}  // namespace ops
}  // namespace ew

using namespace ew;

extern "C" ew_status_t ew_last_operator_error(int32_t device, int32_t *code) {
    if (!code) return EW_ERR_INVALID_ARG;
    if (device < 0) return EW_ERR_NO_DEVICE;
    DeviceGuard guard;
    ew_status_t s = ops::launched((int)guard.enter(device), "cudaSetDevice");
    const ops::Device *d = nullptr;
    if (s == EW_OK) s = ops::device_state(device, &d);
    int v = 0;
    if (s == EW_OK) s = ops::take_error(*d, &v);
    if (s == EW_OK) *code = (v & 2) ? EW_ERR_TIMEOUT : (v & ops::kErrBadIndex) ? EW_ERR_INVALID_ARG : EW_OK;
    return s;
}
