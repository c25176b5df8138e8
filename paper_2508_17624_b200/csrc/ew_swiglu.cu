// SwiGLU between an expert's two linears, with the routing weight of a row folded in, and its gradient.
//
//   act[r, i] = p_r silu(g) u                        g = h[r, i], u = h[r, I + i], s = 1 / (1 + e^-g), silu(g) = g s
//   dg = p da u s (1 + g (1 - s)),   du = p da g s,   dp_r = sum_i da g s u
//
// s is 1 / (1 + e^-g) by the fast exponential and division: 2 + 1.2 |g| steps of 2^-23, and 0 for g below -87.3, where 1 + e^-g passes
// 2^126 (silu is above -1.1e-36 there).  The weight p_r commutes with the down projection that follows, so with it folded in here the combine step is a plain
// sum over a token's rows, and its gradient falls out of the pass that reads da and h anyway.
// Bound by HBM: 6 bytes an element forward, 10 backward, each read or written once.  Measured at 1408 columns: forward 66 us
// for 49152 rows = 6.29 TB/s (96 % of the measured copy bandwidth), backward 58 us for 24582 = 5.97 TB/s (91 %).  A row is a
// warp's: four steps of its loop are unrolled, so that a lane has eight (twelve) 16-byte loads on their way (two steps: 71 and
// 65 us; six: 91 and 79), and the rows are dealt by the hardware, a CTA per eight rows (a grid that fills the GPU once and
// strides: 81 and 63, its last round is a fifth full).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ew_ops.h"
#include "ew_tc.cuh"

namespace ew {
namespace ops {
namespace {

constexpr int kThreads = 256;

template <class T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

template <class T, int V> struct alignas(sizeof(T) * V) Vec { T v[V]; };

struct Args {
    const void *h, *da;
    const float *p;
    void *out;              // act, or dh
    float *dp;
    long long ldh, ldda, ldo, rows;
    int inter;
};

// W warps share a row.  One warp a row streams a large batch; a batch too small to fill the GPU that way gives a row to
// the whole CTA.
template <class T, int V, int W, bool GRAD>
__global__ void __launch_bounds__(kThreads, GRAD ? 4 : 6) swiglu_kernel(const Args a) {
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    constexpr int kRows = kThreads / 32 / W;                                 // rows a CTA works on at a time
    const int team = (threadIdx.x >> 5) / W, t = threadIdx.x - team * W * 32;
    for (long long r = (long long)blockIdx.x * kRows + team; r < a.rows; r += (long long)gridDim.x * kRows) {
        const T *g_row = reinterpret_cast<const T *>(a.h) + r * a.ldh, *u_row = g_row + a.inter;
        T *o_row = reinterpret_cast<T *>(a.out) + r * a.ldo;
        const T *d_row = GRAD ? reinterpret_cast<const T *>(a.da) + r * a.ldda : nullptr;
        const float p = a.p ? a.p[r] : 1.f;
        float dp = 0.f;
#pragma unroll 4
        for (int i = t * V; i < a.inter; i += W * 32 * V) {
            const Vec<T, V> g = *reinterpret_cast<const Vec<T, V> *>(g_row + i), u = *reinterpret_cast<const Vec<T, V> *>(u_row + i);
            Vec<T, V> d, o0, o1;
            if (GRAD) d = *reinterpret_cast<const Vec<T, V> *>(d_row + i);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float gf = to_f(g.v[j]), uf = to_f(u.v[j]);
                const float s = __fdividef(1.f, 1.f + __expf(-gf)), silu = gf * s;
                if (!GRAD) {
                    o0.v[j] = from_f<T>(silu * uf * p);
                } else {
                    const float df = to_f(d.v[j]), dfp = df * p;
                    o0.v[j] = from_f<T>(dfp * uf * (s * (1.f + gf * (1.f - s))));
                    o1.v[j] = from_f<T>(dfp * silu);
                    dp += df * silu * uf;
                }
            }
            *reinterpret_cast<Vec<T, V> *>(o_row + i) = o0;
            if (GRAD) *reinterpret_cast<Vec<T, V> *>(o_row + a.inter + i) = o1;
        }
        if (GRAD && a.dp) {                                                  // summed in a fixed order
#pragma unroll
            for (int m = 16; m; m >>= 1) dp += __shfl_xor_sync(0xffffffffu, dp, m);
            if (W == 1) {
                if (t == 0) a.dp[r] = dp;
            } else {
                __shared__ float part[kThreads / 32];
                if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = dp;
                __syncthreads();
                if (threadIdx.x == 0) {
                    float sum = 0.f;
                    for (int w = 0; w < W; ++w) sum += part[w];
                    a.dp[r] = sum;
                }
                __syncthreads();
            }
        }
    }
}

template <class T, int V, bool GRAD>
ew_status_t launch(const Device &d, const Args &a, cudaStream_t st) {
    constexpr int kWarps = kThreads / 32;
    // Measured (replayed graphs; a CTA a row against a warp a row), 1408 columns: forward 148 rows 2.1 and 3.8 us, 1184: 3.1 and 4.1, 2368: 4.6
    // both, 4736: 7.4 and 6.4; gradient 148: 2.3 and 4.4, 1184: 4.9 and 4.6, 4736: 13.8 and 9.0; 264 columns, forward 592: 2.1 and 2.3,
    // 2368: 3.6 and 2.6.  (So for narrow rows and the gradient the change could come earlier, by a few microseconds.)
    const bool wide = a.rows < (long long)d.sm_count * kWarps * 4;
    const long long ctas = wide ? a.rows : (a.rows + kWarps - 1) / kWarps, most = 0x7fffffff;
    const dim3 grid((unsigned)(ctas < most ? ctas : most));
    const int rc = wide ? launch_pdl(swiglu_kernel<T, V, kWarps, GRAD>, grid, dim3(kThreads), 0, st, a)
                        : launch_pdl(swiglu_kernel<T, V, 1, GRAD>, grid, dim3(kThreads), 0, st, a);
    return launched(rc, "SwiGLU");
}

ew_status_t swiglu(bool grad, int32_t device, int32_t dtype, const void *da, int64_t ldda, const void *h, int64_t ldh, const float *p, int32_t rows,
                   int32_t inter, void *out, int64_t ldo, float *dp, void *stream) {
    if (!is_16bit(dtype)) return refuse("SwiGLU: bf16 or fp16");
    if (rows < 0 || inter < 1 || inter > 0x3fffffff) return refuse("SwiGLU: size out of range");
    if (ldh < 2ll * inter || ldo < (grad ? 2ll : 1ll) * inter || (grad && ldda < inter)) return refuse("SwiGLU: rows overlap");
    if (rows > 0 && (!h || !out || (grad && !da) || (dp && !p) || (((uintptr_t)h | (uintptr_t)out | (uintptr_t)da) & 1) || (((uintptr_t)p | (uintptr_t)dp) & 3)))
        return refuse("SwiGLU: null or misaligned pointer, or a weight gradient without weights");
    if (device < 0) return EW_ERR_NO_DEVICE;
    if (rows == 0) return EW_OK;
    DeviceGuard guard;
    ew_status_t s = launched((int)guard.enter(device), "cudaSetDevice");
    const Device *d;
    if (s != EW_OK || (s = device_state(device, &d)) != EW_OK) return s;
    const Args a = {h, da, p, out, dp, ldh, grad ? ldda : 0, ldo, rows, inter};
    // eight elements (16 bytes) at a time where every row starts on a 16-byte boundary
    const bool vec = !((((uintptr_t)h | (uintptr_t)out | (uintptr_t)da) & 15) | ((ldh | ldo | a.ldda | inter) & 7));
    cudaStream_t st = (cudaStream_t)stream;
#define EW_PICK(T) (vec ? (grad ? launch<T, 8, true>(*d, a, st) : launch<T, 8, false>(*d, a, st)) : (grad ? launch<T, 1, true>(*d, a, st) : launch<T, 1, false>(*d, a, st)))
    return dtype == EW_BF16 ? EW_PICK(__nv_bfloat16) : EW_PICK(__half);
#undef EW_PICK
}

template <class T, int V>
int load_one() {
    constexpr int kWarps = kThreads / 32;
    cudaFuncAttributes fa;
    return (int)cudaFuncGetAttributes(&fa, swiglu_kernel<T, V, 1, false>) | (int)cudaFuncGetAttributes(&fa, swiglu_kernel<T, V, kWarps, false>) |
           (int)cudaFuncGetAttributes(&fa, swiglu_kernel<T, V, 1, true>) | (int)cudaFuncGetAttributes(&fa, swiglu_kernel<T, V, kWarps, true>);
}

}  // namespace

// Loads the kernels (a first launch inside a graph capture would have to).
int swiglu_setup() {
    return load_one<__nv_bfloat16, 1>() | load_one<__nv_bfloat16, 8>() | load_one<__half, 1>() | load_one<__half, 8>();
}

}  // namespace ops
}  // namespace ew

extern "C" ew_status_t ew_swiglu(int32_t device, int32_t dtype, const void *h, int64_t ldh, const float *row_weights, int32_t rows, int32_t inter, void *act,
                                 int64_t ldact, void *cuda_stream) {
    return ew::ops::swiglu(false, device, dtype, nullptr, 0, h, ldh, row_weights, rows, inter, act, ldact, nullptr, cuda_stream);
}

extern "C" ew_status_t ew_swiglu_grad(int32_t device, int32_t dtype, const void *dact, int64_t lddact, const void *h, int64_t ldh, const float *row_weights,
                                      int32_t rows, int32_t inter, void *dh, int64_t lddh, float *drow_weights, void *cuda_stream) {
    return ew::ops::swiglu(true, device, dtype, dact, lddact, h, ldh, row_weights, rows, inter, dh, lddh, drow_weights, cuda_stream);
}
