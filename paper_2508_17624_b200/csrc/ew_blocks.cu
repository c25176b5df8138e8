// Rows, SwiGLU's result and weights as 8-bit floating point in blocks of 128 (see ew_blocks.cuh for the form).
//
//   rows     q s = x[r, :]                       a scale for 128 values of a row
//   SwiGLU   q s = p_r silu(h[r, :I]) h[r, I:]   the same (silu as in the 16-bit operator)
//   weights  q s = w[g, :, :]                    a scale for 128 x 128 values
//
// Bound by HBM: 3, 5 and 3 bytes a value, each read or written once.  A block's values stay in the registers of half a warp
// (rows) or a CTA (weights) between the search for the largest and the rounding.  Measured: rows 24582 x 2048 25 us = 6.1 TB/s
// (93 % of the measured copy bandwidth), SwiGLU 49152 x 1408 57 us = 6.1 TB/s, 63 to 67 in long runs at the power limit, weights
// 64 x 2816 x 2048 166 us = 6.7 TB/s, 174 to 180 in long runs.
#include "ew_blocks.cuh"
#include "ew_ops.h"
#include "ew_tc.cuh"

namespace ew {
namespace ops {
namespace {
using namespace blocks;

constexpr int kThreads = 256;

struct RowArgs {
    const void *x;                                     // the rows, or h
    const float *p;
    uint8_t *q, *scales;
    long long ldx, ldq, lds, rows;
    int width;                                         // of the result
};

// g / (1 + 2^(-g log2 e)) by the fast power of two and reciprocal: 2 + 1.2 |g| steps of 2^-23, and 0 where the power passes 2^126
__device__ __forceinline__ Two silu(Two g) {
    constexpr float kLog2e = 1.44269504f;
    float2 e = parts_of(mul2(g, two(-kLog2e, -kLog2e)));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
    const Two one = two(1.f, 1.f);
    e = parts_of(fma2(two(e.x, e.y), one, one));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e.y));
    return mul2(g, two(e.x, e.y));
}

// W warps share a row; each asks for kAhead spans before it works on the first.  (SwiGLU of 49152 x 1408 with five CTAs an SM: three spans 57 us,
// two 59, one 62, six, with room for three CTAs, 65; rows of 24582 x 2048: four spans 25 us, two 29, eight 27.)
template <class T, bool ACT, bool E5M2, bool VEC, int W>
__global__ void __launch_bounds__(kThreads, VEC && W == 1 ? 5 : 1) rows_kernel(const RowArgs a) {
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    constexpr int kRows = kThreads / 32 / W, kAhead = W > 1 ? 1 : !VEC ? 2 : ACT ? 3 : 4;
    const int lane = threadIdx.x & 31, w = (threadIdx.x >> 5) % W;
    for (long long r = (long long)blockIdx.x * kRows + (threadIdx.x >> 5) / W; r < a.rows; r += (long long)gridDim.x * kRows) {
        const T *row = reinterpret_cast<const T *>(a.x) + r * a.ldx;
        uint8_t *q = a.q + r * a.ldq, *scales = a.scales + r * a.lds;
        const float p = ACT && a.p ? a.p[r] : 1.f;
        for (int from = w * kSpan; from < a.width; from += W * kSpan * kAhead) {
            Eight<T> g[kAhead], u[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                load_span<T, VEC>(g[k], row, from + k * W * kSpan, lane, a.width);
                if (ACT) load_span<T, VEC>(u[k], row + a.width, from + k * W * kSpan, lane, a.width);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int at = from + k * W * kSpan;
                if (at < a.width) {
                    Two v[4];
                    to_pairs(v, g[k]);
                    if (ACT) {
                        Two up[4];
                        to_pairs(up, u[k]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = mul2(mul2(silu(v[j]), up[j]), two(p, p));
                    }
                    put_span<VEC, E5M2>(v, q, scales, at, lane, a.width);
                }
            }
        }
    }
}

struct WeightArgs {
    const void *w;
    uint8_t *q, *scales;
    long long ldw, w_stride, ldq, q_stride;
    int n, k, nb, kb;
};

// A CTA a block of 128 x 128.  VEC: sixteen lanes a row of the block; otherwise 128.  (Three CTAs an SM 166 us, 179 in long
// runs at the power limit; four 160 and 185; two 201.)
template <class T, bool VEC>
__global__ void __launch_bounds__(kThreads, VEC ? 3 : 2) weights_kernel(const WeightArgs a) {
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    __shared__ float part[kThreads / 32];
    const int t = threadIdx.x, bk = blockIdx.x % a.kb, bn = blockIdx.x / a.kb;
    const T *w = reinterpret_cast<const T *>(a.w) + blockIdx.y * a.w_stride;
    uint8_t *q = a.q + blockIdx.y * a.q_stride;
    // the row and column of a thread's value j of step i
    auto row_of = [&](int i, int j) { return bn * kBlock + (VEC ? i * 16 + (t >> 4) : (i * 8 + j) * 2 + (t >> 7)); };
    auto col_of = [&](int j) { return bk * kBlock + (VEC ? (t & 15) * 8 + j : t & 127); };
    Eight<T> raw[8];                                   // what lies behind an edge reads the block's last values once more, without a branch
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (VEC) {                           // (k is a multiple of eight)
            *reinterpret_cast<uint4 *>(&raw[i]) = *reinterpret_cast<const uint4 *>(w + min(row_of(i, 0), a.n - 1) * a.ldw + min(col_of(0), a.k - 8));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) raw[i].v[j] = w[min(row_of(i, j), a.n - 1) * a.ldw + min(col_of(j), a.k - 1)];
        }
    }
    float most = 0.f;
    auto of_all = [&] {                                // the CTA's largest, in every thread
#pragma unroll
        for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(kAll, most, d));
        if ((t & 31) == 0) part[t >> 5] = most;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i) most = fmaxf(most, part[i]);
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        Two v[4];
        to_pairs(v, raw[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) most = max_abs(most, v[j]);
    }
    of_all();
    if (not_finite(most)) {                            // the same in every thread
        most = 0.f;
#pragma unroll
        for (int i = 0; i < 64; ++i) {
            T &x = raw[i >> 3].v[i & 7];
            if (not_finite(to_f(x))) x = from_f<T>(__int_as_float(0x7fffffff));
            else most = fmaxf(most, fabsf(to_f(x)));
        }
        __syncthreads();
        of_all();
    }
    const uint32_t code = scale_code(most, kTop<false>);
    const Two f = two(inverse_scale(code), inverse_scale(code));
    if (t == 0) a.scales[((long long)blockIdx.y * a.nb + bn) * a.kb + bk] = (uint8_t)code;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        Two v[4];
        to_pairs(v, raw[i]);
        uint32_t pair[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 x = parts_of(mul2(v[j], f));
            pair[j] = two_values<false>(x.x, x.y);
        }
        if constexpr (VEC) {
            if (col_of(0) < a.k && row_of(i, 0) < a.n)
                *reinterpret_cast<uint2 *>(q + row_of(i, 0) * a.ldq + col_of(0)) = make_uint2(pair[0] | pair[1] << 16, pair[2] | pair[3] << 16);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (row_of(i, j) < a.n && col_of(j) < a.k) q[row_of(i, j) * a.ldq + col_of(j)] = (uint8_t)(pair[j >> 1] >> (8 * (j & 1)));
        }
    }
}

template <class T, bool ACT, bool E5M2, bool VEC>
ew_status_t launch_rows(const Device &d, const RowArgs &a, cudaStream_t st) {
    constexpr int kWarps = kThreads / 32;
    // a CTA a row where warps would not fill half of the GPU (SwiGLU of 1408 columns: 2368 rows 4.9 us against 6.7 with a warp a row, 4736
    // rows 10.6 against 9.7; rows of 2048: 3.9 and 4.8, 7.3 and 5.9; of 512, either way in the launch's noise up to 2368 rows: 3.9 and 3.4)
    const bool wide = a.rows < (long long)d.sm_count * kWarps * 2;
    const long long ctas = wide ? a.rows : (a.rows + kWarps - 1) / kWarps, most = 0x7fffffff;
    const dim3 grid((unsigned)(ctas < most ? ctas : most));
    const int rc = wide ? launch_pdl(rows_kernel<T, ACT, E5M2, VEC, kWarps>, grid, dim3(kThreads), 0, st, a)
                        : launch_pdl(rows_kernel<T, ACT, E5M2, VEC, 1>, grid, dim3(kThreads), 0, st, a);
    return launched(rc, "blocks of rows");
}

ew_status_t to_rows(bool act, int32_t device, int32_t dtype, int32_t q_type, const void *x, int64_t ldx, const float *p, int32_t rows, int32_t width, void *q,
                    int64_t ldq, void *scales, int64_t lds, void *stream) {
    if (!is_16bit(dtype)) return refuse("blocks of rows: bf16 or fp16");
    if (!is_8bit(q_type)) return refuse("blocks of rows: e4m3 or e5m2");
    if (rows < 0 || width < 1 || width > 0x3fffffff) return refuse("blocks of rows: size out of range");
    if (ldx < (act ? 2ll : 1ll) * width || ldq < width || lds < (width + kBlock - 1) / kBlock) return refuse("blocks of rows: rows overlap");
    if (rows > 0 && (!x || !q || !scales || ((uintptr_t)x & 1) || ((uintptr_t)p & 3))) return refuse("blocks of rows: null or misaligned pointer");
    if (device < 0) return EW_ERR_NO_DEVICE;
    if (rows == 0) return EW_OK;
    DeviceGuard guard;
    ew_status_t s = launched((int)guard.enter(device), "cudaSetDevice");
    const Device *d;
    if (s != EW_OK || (s = device_state(device, &d)) != EW_OK) return s;
    const RowArgs a = {x, p, (uint8_t *)q, (uint8_t *)scales, ldx, ldq, lds, rows, width};
    const bool vec = !(((uintptr_t)x & 15) | ((uintptr_t)q & 7) | ((ldx | ldq | width) & 7));
    cudaStream_t st = (cudaStream_t)stream;
#define EW_PICK(T, ACT, E5M2) (vec ? launch_rows<T, ACT, E5M2, true>(*d, a, st) : launch_rows<T, ACT, E5M2, false>(*d, a, st))
    if (act) return dtype == EW_BF16 ? EW_PICK(__nv_bfloat16, true, false) : EW_PICK(__half, true, false);
    if (q_type == EW_E4M3) return dtype == EW_BF16 ? EW_PICK(__nv_bfloat16, false, false) : EW_PICK(__half, false, false);
    return dtype == EW_BF16 ? EW_PICK(__nv_bfloat16, false, true) : EW_PICK(__half, false, true);
#undef EW_PICK
}

template <class T, bool VEC>
int load_one() {
    constexpr int kWarps = kThreads / 32;
    cudaFuncAttributes fa;
    return (int)cudaFuncGetAttributes(&fa, rows_kernel<T, true, false, VEC, 1>) | (int)cudaFuncGetAttributes(&fa, rows_kernel<T, true, false, VEC, kWarps>) |
           (int)cudaFuncGetAttributes(&fa, rows_kernel<T, false, false, VEC, 1>) | (int)cudaFuncGetAttributes(&fa, rows_kernel<T, false, false, VEC, kWarps>) |
           (int)cudaFuncGetAttributes(&fa, rows_kernel<T, false, true, VEC, 1>) | (int)cudaFuncGetAttributes(&fa, rows_kernel<T, false, true, VEC, kWarps>) |
           (int)cudaFuncGetAttributes(&fa, weights_kernel<T, VEC>);
}

}  // namespace

// Loads the kernels (a first launch inside a graph capture would have to).
int blocks_setup() {
    return load_one<__nv_bfloat16, false>() | load_one<__nv_bfloat16, true>() | load_one<__half, false>() | load_one<__half, true>();
}

}  // namespace ops
}  // namespace ew

using namespace ew;
using namespace ew::ops;

extern "C" ew_status_t ew_scaled_rows(int32_t device, int32_t dtype, int32_t q_type, const void *x, int64_t ldx, int32_t rows, int32_t width, void *q, int64_t ldq,
                                      void *scales, int64_t ldscales, void *cuda_stream) {
    return to_rows(false, device, dtype, q_type, x, ldx, nullptr, rows, width, q, ldq, scales, ldscales, cuda_stream);
}

extern "C" ew_status_t ew_swiglu_scaled(int32_t device, int32_t dtype, const void *h, int64_t ldh, const float *row_weights, int32_t rows, int32_t inter, void *q,
                                        int64_t ldq, void *scales, int64_t ldscales, void *cuda_stream) {
    return to_rows(true, device, dtype, EW_E4M3, h, ldh, row_weights, rows, inter, q, ldq, scales, ldscales, cuda_stream);
}

extern "C" ew_status_t ew_scaled_pack(int32_t device, int32_t dtype, const void *w, int64_t ldw, int64_t slot_stride, int32_t n_slots, int32_t n, int32_t k, void *q,
                                      int64_t ldq, int64_t q_stride, void *scales, void *cuda_stream) {
    if (!is_16bit(dtype)) return refuse("blocks of weights: bf16 or fp16");
    const int64_t nb = ((int64_t)n + blocks::kBlock - 1) / blocks::kBlock, kb = ((int64_t)k + blocks::kBlock - 1) / blocks::kBlock;
    if (n_slots < 1 || n_slots > kMostSlots || n < 1 || k < 1 || n > 0x7fff0000 || k > 0x7fff0000 || nb * kb > 0x7fffffff) return refuse("blocks of weights: size out of range");
    if (ldw < k || ldq < k || !rows_apart(n_slots, slot_stride, n, ldw, k) || !rows_apart(n_slots, q_stride, n, ldq, k)) return refuse("blocks of weights: rows overlap");
    if (!w || !q || !scales || ((uintptr_t)w & 1)) return refuse("blocks of weights: null or misaligned pointer");
    if (device < 0) return EW_ERR_NO_DEVICE;
    DeviceGuard guard;
    ew_status_t s = launched((int)guard.enter(device), "cudaSetDevice");
    const Device *d;
    if (s != EW_OK || (s = device_state(device, &d)) != EW_OK) return s;
    const WeightArgs a = {w, (uint8_t *)q, (uint8_t *)scales, ldw, n_slots > 1 ? slot_stride : 0, ldq, n_slots > 1 ? q_stride : 0, n, k, (int)nb, (int)kb};
    const bool vec = !(((uintptr_t)w & 15) | ((uintptr_t)q & 7) | ((a.ldw | a.w_stride | a.ldq | a.q_stride | k) & 7));
    const dim3 grid((unsigned)(nb * kb), (unsigned)n_slots);
    cudaStream_t st = (cudaStream_t)cuda_stream;
#define EW_PICK(T) (vec ? launch_pdl(weights_kernel<T, true>, grid, dim3(kThreads), 0, st, a) : launch_pdl(weights_kernel<T, false>, grid, dim3(kThreads), 0, st, a))
    return launched(dtype == EW_BF16 ? EW_PICK(__nv_bfloat16) : EW_PICK(__half), "blocks of weights");
#undef EW_PICK
}
