// 8-bit floating point in blocks of 128: the form that the scaled products read and the operators before them write.
//
// A block is 128 values q in e4m3 or e5m2 and one exponent byte c (e8m0), and stands for q 2^(c - 127).  c is the smallest, from 0
// on, for which the block's largest finite value fits the type (448 or 57344, both 1.75 times a power of two):
//     c = max(0, E - top + [mantissa of the largest above 1.75]),   E its biased exponent, top = 8 or 15
// which is integer arithmetic on its bits.  A scale that is a power of two costs the values nothing but range: q is the value
// rounded once, to nearest even, as if the type had no smallest exponent (but below 2^-9 of the block's largest, where e4m3 runs
// out of exponents).  An infinity or NaN becomes the NaN of the type and takes no part in its block's scale.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cstdint>

#include "../../include/expertweave.h"

namespace ew {
namespace ops {
namespace blocks {

constexpr int kBlock = 128;
constexpr int kSpan = 256;                             // values a warp works on at a time: eight a lane, two blocks
constexpr unsigned kAll = 0xffffffffu;

template <class T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

template <class T> struct alignas(16) Eight { T v[8]; };

template <bool E5M2> constexpr int kTop = E5M2 ? 15 : 8;
__device__ __forceinline__ uint32_t scale_code(float most, int top) {
    return (uint32_t)max((int)((__float_as_uint(most) + 0x1fffffu) >> 23) - top, 0);
}
__device__ __forceinline__ float inverse_scale(uint32_t code) { return __uint_as_float((254u - code) << 23); }      // 2^(127 - code)

template <bool E5M2>
__device__ __forceinline__ uint32_t two_values(float lo, float hi) {
    return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, E5M2 ? __NV_E5M2 : __NV_E4M3);
}
__device__ __forceinline__ bool not_finite(float v) { return !(fabsf(v) <= 3.402823466e38f); }

// Two fp32 numbers in one instruction: kernels that pass over memory at its full rate have some thirty issue slots a value.
struct Two { unsigned long long v; };
__device__ __forceinline__ Two two(float lo, float hi) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 parts_of(Two a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
// max(m, |a.lo|, |a.hi|); a NaN is passed over
__device__ __forceinline__ float max_abs(float m, Two a) {
    const float2 v = parts_of(a);
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(fabsf(v.x)), "f"(fabsf(v.y)), "f"(m));
    return m;
}
template <class T>
__device__ __forceinline__ void to_pairs(Two (&p)[4], const Eight<T> &o) {
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = two(to_f(o.v[2 * j]), to_f(o.v[2 * j + 1]));
}

__device__ __forceinline__ void round_pair(__nv_bfloat16 *to, float2 f) { *reinterpret_cast<__nv_bfloat162 *>(to) = __floats2bfloat162_rn(f.x, f.y); }
__device__ __forceinline__ void round_pair(__half *to, float2 f) { *reinterpret_cast<__half2 *>(to) = __floats2half2_rn(f.x, f.y); }
template <class T>
__device__ __forceinline__ void from_pairs(Eight<T> &o, const Two (&p)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) round_pair(o.v + 2 * j, parts_of(p[j]));
}

// Where a lane's eight values of a span lie.  VEC: side by side, so that they move in one access (rows on 16-byte boundaries, of a
// multiple of eight values); otherwise 32 apart, so that a warp's accesses of single values are whole sectors all the same.
template <bool VEC> __device__ __forceinline__ int place(int lane, int j) { return VEC ? lane * 8 + j : lane + 32 * j; }

// Loading has no branch: a place behind the row's end reads its last values once more.  (With a branch around each access the
// compiler waits for one before it begins the next: the norm of 8192 rows took 90 us, SwiGLU of 49152 206.)  They lie in the
// row's last block or in one that is not written, so its largest is the same; sums have to leave them out.
template <class T, bool VEC>
__device__ __forceinline__ void load_span(Eight<T> &o, const T *row, int at, int lane, int width) {
    if constexpr (VEC) {
        *reinterpret_cast<uint4 *>(&o) = *reinterpret_cast<const uint4 *>(row + min(at + lane * 8, width - 8));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = at + lane + 32 * j;
            o.v[j] = row[min(i, width - 1)];
        }
    }
}
// What lies behind the row's end becomes zeros.
template <class T, bool VEC>
__device__ __forceinline__ void clear_span(Eight<T> &o, int at, int lane, int width) {
    if constexpr (VEC) {
        uint4 &v = *reinterpret_cast<uint4 *>(&o);
        const bool in = at + lane * 8 < width;
        v = make_uint4(in ? v.x : 0, in ? v.y : 0, in ? v.z : 0, in ? v.w : 0);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (at + lane + 32 * j >= width) o.v[j] = from_f<T>(0.f);
    }
}
template <class T, bool VEC>
__device__ __forceinline__ void store_span(const Eight<T> &o, T *row, int at, int lane, int width) {
    if constexpr (VEC) {
        if (at + lane * 8 < width) *reinterpret_cast<Eight<T> *>(row + at + lane * 8) = o;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = at + place<VEC>(lane, j);
            if (i < width) row[i] = o.v[j];
        }
    }
}

// Writes a span as two blocks.  The whole warp calls it.
template <bool VEC, bool E5M2>
__device__ __forceinline__ void put_span(Two (&v)[4], uint8_t *q_row, uint8_t *scale_row, int at, int lane, int width) {
    constexpr int kFirst = VEC ? 4 : 2;                // of the lane's pairs, those of its first block
    float m0, m1;
    auto most = [&] {
        m0 = m1 = 0.f;
#pragma unroll
        for (int j = 0; j < kFirst; ++j) m0 = max_abs(m0, v[j]);
#pragma unroll
        for (int j = kFirst; j < 4; ++j) m1 = max_abs(m1, v[j]);
#pragma unroll
        for (int d = VEC ? 8 : 16; d; d >>= 1) {
            m0 = fmaxf(m0, __shfl_xor_sync(kAll, m0, d));
            if (!VEC) m1 = fmaxf(m1, __shfl_xor_sync(kAll, m1, d));
        }
    };
    most();
    if (__any_sync(kAll, not_finite(m0) || not_finite(m1))) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float2 f = parts_of(v[j]);
            if (not_finite(f.x)) f.x = __int_as_float(0x7fffffff);
            if (not_finite(f.y)) f.y = __int_as_float(0x7fffffff);
            v[j] = two(f.x, f.y);
        }
        most();
    }
    const uint32_t c0 = scale_code(m0, kTop<E5M2>), c1 = VEC ? c0 : scale_code(m1, kTop<E5M2>);
    const float i0 = inverse_scale(c0), i1 = VEC ? i0 : inverse_scale(c1);
    uint32_t pair[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float f = j < kFirst ? i0 : i1;
        const float2 x = parts_of(mul2(v[j], two(f, f)));
        pair[j] = two_values<E5M2>(x.x, x.y);
    }
    if constexpr (VEC) {
        if (at + lane * 8 < width) *reinterpret_cast<uint2 *>(q_row + at + lane * 8) = make_uint2(pair[0] | pair[1] << 16, pair[2] | pair[3] << 16);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = at + place<VEC>(lane, j);
            if (i < width) q_row[i] = (uint8_t)(pair[j >> 1] >> (8 * (j & 1)));
        }
    }
    uint8_t *s = scale_row + at / kBlock;
    if (VEC) {
        if ((lane & 15) == 0 && at + lane * 8 < width) s[lane >> 4] = (uint8_t)c0;
    } else if (lane == 0) {
        s[0] = (uint8_t)c0;
        if (at + kBlock < width) s[1] = (uint8_t)c1;
    }
}

}  // namespace blocks
}  // namespace ops
}  // namespace ew
