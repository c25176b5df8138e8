// Matrix-vector products with 4-bit expert weights and group scales, and the packing of the weights.
//
//   y[p, n] = sum_k x[row(p), k] (q[slot(p), n, k] - 8) scale[slot(p), k / group, n]
//
// for a batch's (token, expert) pairs p, whose slots come straight from the router: nothing is sorted or counted before
// the call, every CTA groups the few hundred pairs itself, so that pairs of one slot share its weights' bytes.
//
// Bound by HBM: half a byte a weight and little else, at 6.5 TB/s 46 weights a cycle and SM.  Turning each into a 16-bit
// number first (and-or, shift, subtract: 22 warp instructions for 512 weights and as many again around them) keeps the SM's
// issue slots busy for longer than the bytes take (measured: 37 us where the bytes need 22), so the weights are used as
// they are: one mask, or a shift and a mask, turns a word into four bytes 0..15, and the 8-bit integer m16n8k32
// instruction multiplies 512 weights with eight pairs (2.1 cycles of an SM measured, what bf16 takes for 256; the 8-bit
// floating-point form is made of 16-bit ones on this machine and slower).  x goes in as fixed-point numbers: a group of x,
// which the scales split off anyway, is scaled by a power of two so that its largest magnitude lies above 4177855, rounded
// to whole numbers and cut into three signed bytes.  That rounding is below 1/8355711 of the group's largest x (or 2^-127, the most
// that the scale's power of two goes down to), and none at all for bf16 values down to a 2^15th of it (two bytes would cost 9 to 13 % less time, but a group with one large value
// would leave its small ones six bits).  The products' sums are exact integers, the offset 8 is their first value
// (-8 sum x); only then come fp32 numbers: group sum times scale, added up over the groups.  A slot with many pairs repays
// the unpacking: there the weights become 16-bit numbers (q - 8, exact) and x stays as it is.
//
// A warp owns 32 weight rows and streams them through a ring of its own with TMA, a line of 256 weights of each row (4 KiB)
// at a time; the products' order within a line is arbitrary as long as both operands agree, so a lane's word of eight
// weights meets the same eight k of x without any shuffling.  A CTA's tiles are contiguous and its lines are dealt to
// its warps evenly; a tile that crosses from one warp to the next is added up in shared memory, in order.
//
// Measured (one B200, copy bandwidth 6551 GB/s), 2816 x 2048 weights unless said: one token's six experts 8.9 us (18 MB; 2.7 us
// of bytes behind a launch, the slots' way from memory and the first line's); 96
// pairs over 96 slots of 2048 x 1408 27 us = 3.4 TB/s; 256 tokens, some sixteen pairs a slot, 114 us = 2.7 TB/s, bound by the
// instructions around the products together with the latencies between them (55 % of the issue slots of the active cycles, 40 % of the
// tensor pipe's; 127 registers leave room for sixteen warps).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ew_ops.h"
#include "ew_tc.cuh"

namespace ew {
namespace ops {
namespace {
using namespace tc;

constexpr int kWarps = 16;
constexpr int kThreads = kWarps * 32;
constexpr int kRows = 32;                      // weight rows of a tile: two tiles of the MMA
constexpr int kLineK = 256;                    // weights of a row in one 128-byte swizzled line
constexpr int kLineBytes = kRows * kLineK / 2; // a stage: 4 KiB
constexpr __host__ __device__ int scale_bytes(int spg) { return 8 / spg * kRows * 2; }           // a stage's scales: up to eight groups x 32 rows
constexpr int kMaxStages = 2;                  // of a warp
constexpr int kMaxPairs = 2048;                // of one launch; a larger batch is split
constexpr int kMaxSlots = 2048;
constexpr int kMaxK = 16384;
constexpr int kSmemLimit = 227 * 1024;

struct Args {
    const uint8_t *x;           // row 0 of this launch
    const int32_t *slots;       // null: every pair uses slot 0
    void *out;
    int *err;
    long long ldx, ldo;         // elements
    int pairs, pair0, share;    // of this launch; its first pair; pairs per row of x
    int lead;                   // pair0 % share
    int n, k, n_slots;
    int tiles;                  // 32-row tiles of a slot
    int out_fp32;
    int job_rows;               // most pairs of a job
    int stages;                 // of a warp's ring
    // shared memory: the rows of x being worked on (capacity, bytes a row, of that the two higher bytes - or x itself - and the
    // lowest byte of its numbers)
    int x_cap, x_bytes, x_wide, x_third;
    int at_x, at_bars, at_red, at_jobs, at_start, at_order, at_row;
};

struct alignas(8) Job { uint16_t slot, first, count, pad; };                // pairs order[first .. first + count) of one slot

__device__ __forceinline__ void mma8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// byte `at` of four numbers, the first one's lowest
__device__ __forceinline__ uint32_t bytes(const uint32_t (&u)[8], int i0, int i1, int i2, int i3, int at) {
    const uint32_t sel = (uint32_t)at | (uint32_t)(4 + at) << 4;
    return __byte_perm(__byte_perm(u[i0], u[i1], sel), __byte_perm(u[i2], u[i3], sel), 0x5410);
}
template <class T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }

template <class T>
__device__ __forceinline__ void put(void *out, size_t at, float v, bool wide) {
    if (wide) reinterpret_cast<float *>(out)[at] = v;
    else reinterpret_cast<T *>(out)[at] = (T)v;
}

template <class T>
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    if constexpr (__is_same(T, __nv_bfloat16)) {
        const __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&r);
    } else {
        const __half2 r = __hsub2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
}
// Eight 4-bit values to q - 8 in four registers, k ascending: a nibble or-ed into the last mantissa bits of 128 (bf16) or
// 1024 (fp16) is that number plus q, from which 136 (1032) is subtracted exactly.
template <class T>
__device__ __forceinline__ void unpack(uint32_t w, uint32_t (&a)[4]) {
    constexpr bool kBf = __is_same(T, __nv_bfloat16);
    constexpr uint32_t kMagic = kBf ? 0x43004300u : 0x64006400u, kBias = kBf ? 0x43084308u : 0x64086408u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t v;
        asm("lop3.b32 %0, %1, 0x000F000F, %2, 0xEA;" : "=r"(v) : "r"(w >> (4 * i)), "r"(kMagic));    // (w & mask) | magic
        a[i] = sub2<T>(v, kBias);
    }
}
template <class T>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, const float (&c)[4]) {
    if constexpr (__is_same(T, __nv_bfloat16))
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

// A whole number i, |i| < 2^22, plus these bits is the float kFloat + i: the sums start there and become floats by one
// subtraction (the conversion instruction runs at an eighth of its rate; |a group's sum of q times a byte| < 2^18).
constexpr int kFloatBits = 0x4B400000;
constexpr float kFloat = 12582912.f;

// A line of a row of x (a lane: eight k) into three bytes a number, highest first; per group of 32 SPG its scale 2^-e and the
// sums' first values -8 sum of each byte (the weights' offset).  A group with an infinity or NaN gets the scale NaN.
template <class T, int SPG>
__device__ __forceinline__ void convert_line(const uint4 raw, int line, bool there, uint8_t *to, const Args &a) {
    const int lane = threadIdx.x & 31, at_k = line * kLineK + lane * 8;
    const T *v = reinterpret_cast<const T *>(&raw);
    float f[8], most = 0.f;
    bool odd = false;                                                        // (fmaxf drops a NaN)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f[i] = to_f<T>(v[i]);
        most = fmaxf(most, fabsf(f[i]));
        odd |= !(fabsf(f[i]) < __int_as_float(0x7f800000));
    }
    if (odd) most = __int_as_float(0x7f800000);
#pragma unroll
    for (int m = 1; m < 4 * SPG; m <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, m));
    // signed bytes reach 127 (1 + 256 + 65536) = 8355711: the largest x goes to [2^22, 2^23), or half of that if it
    // is more, i.e. above 4177855
    constexpr int kTop = 22, kMost = 8355711;
    const int e = __float_as_int(most) >> 23;                                // biased exponent of the largest
    int up = min(254 + kTop - e, 253);                                       // biased exponent of the scale
    if (most * __int_as_float(max(up, 1) << 23) > (float)kMost) --up;
    up = max(up, 1);
    const float scale = __int_as_float(up << 23), back = e == 255 ? __int_as_float(0x7fc00000) : __int_as_float((254 - up) << 23);
    uint32_t u[8], lo[3], hi[3];
    int sums[3];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        // number = sum of (byte_j - 128) 256^j for the bytes of number + 0x808080; the same bytes with their top bit turned are
        // byte_j - 128
        u[i] = (uint32_t)(__float2int_rn(e == 255 ? 0.f : f[i] * scale) + 0x808080) ^ 0x808080u;
#pragma unroll
    for (int j = 0; j < 3; ++j) {                                            // in the order in which a word's nibbles come out
        lo[j] = bytes(u, 0, 4, 1, 5, j);
        hi[j] = bytes(u, 2, 6, 3, 7, j);
        sums[j] = __dp4a((int)lo[j], 0x01010101, __dp4a((int)hi[j], 0x01010101, 0));
    }
    // |a group's sum of a byte| <= 2^14: two of them in one number on their way through the lanes
    int low = sums[0] + sums[1] * 65536;
#pragma unroll
    for (int m = 1; m < 4 * SPG; m <<= 1) {
        low += __shfl_xor_sync(0xffffffffu, low, m);
        sums[2] += __shfl_xor_sync(0xffffffffu, sums[2], m);
    }
    sums[0] = (int)(int16_t)low;
    sums[1] = (low - sums[0]) >> 16;
    if (!there) return;
    *reinterpret_cast<uint4 *>(to + line * 512 + lane * 16) = make_uint4(lo[2], hi[2], lo[1], hi[1]);
    *reinterpret_cast<uint2 *>(to + a.x_wide + line * 256 + lane * 8) = make_uint2(lo[0], hi[0]);
    if (lane % (4 * SPG) == 0)
        *reinterpret_cast<int4 *>(to + a.x_wide + a.x_third + (at_k / (32 * SPG)) * 16) =
            make_int4(__float_as_int(back), kFloatBits - 8 * sums[2], kFloatBits - 8 * sums[1], kFloatBits - 8 * sums[0]);
}

template <int OFFSET>
__device__ __forceinline__ uint32_t lds(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1 + %2];" : "=r"(v) : "r"(at), "n"(OFFSET));
    return v;
}
__device__ __forceinline__ int4 lds4(uint32_t at) {
    int4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}

// One line and one column of eight pairs: acc += scale 2^-e (sum of q x 2^e - 8 sum of x 2^e).  w_at: this lane's word of the
// line's first 32-weight step; 16-byte piece i of row r lies at piece i ^ (r mod 8) of its line, one exclusive-or of the
// address.  xb, xc: this lane's operand bytes of the row's first step (two higher bytes, lowest byte), fac0, fac1: of its
// first group, for the columns 2c and 2c + 1.
template <class T, int SPG>
__device__ __forceinline__ void line_products(float (&acc)[2][1][4], uint32_t xb, uint32_t xc, uint32_t fac0, uint32_t fac1, uint32_t w_at, uint32_t s_at, int line,
                                              int left) {
    // (two groups a pass of the loop and no more: small calls run this code cold, and fetching it is what they wait for; one:
    // 3 to 6 % slower)
#pragma unroll 2
    for (int i0 = 0; i0 < 8 && 32 * i0 < left; i0 += SPG) {
        const uint32_t g16 = (uint32_t)(line * (8 / SPG) + i0 / SPG) * 16;
        const int4 v0 = lds4(fac0 + g16), v1 = lds4(fac1 + g16);
        const float f0 = __int_as_float(v0.x), f1 = __int_as_float(v1.x);
        int sum[3][2][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum[0][m][e] = e & 1 ? v1.y : v0.y;
                sum[1][m][e] = e & 1 ? v1.z : v0.z;
                sum[2][m][e] = e & 1 ? v1.w : v0.w;
            }
#pragma unroll
        for (int j = 0; j < SPG; ++j) {
            const int i = i0 + j;
            uint32_t w[4], lo[4], hi[4], d0, d1;
            const uint32_t piece = w_at ^ (i << 4);
            w[0] = lds<0>(piece);
            w[1] = lds<1024>(piece);
            w[2] = lds<2048>(piece);
            w[3] = lds<2048 + 1024>(piece);
            const int4 b = lds4(xb + line * 512 + i * 64);
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(d0), "=r"(d1) : "r"(xc + line * 256 + i * 32));
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                lo[h] = w[h] & 0x0F0F0F0Fu;
                hi[h] = (w[h] >> 4) & 0x0F0F0F0Fu;
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                mma8(sum[0][m], lo[2 * m], lo[2 * m + 1], hi[2 * m], hi[2 * m + 1], b.x, b.y);
                mma8(sum[1][m], lo[2 * m], lo[2 * m + 1], hi[2 * m], hi[2 * m + 1], b.z, b.w);
                mma8(sum[2][m], lo[2 * m], lo[2 * m + 1], hi[2 * m], hi[2 * m + 1], d0, d1);
            }
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            uint16_t r0, r1;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(r0) : "r"(s_at + ((i0 / SPG) * kRows + m * 16) * 2));
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(r1) : "r"(s_at + ((i0 / SPG) * kRows + m * 16) * 2 + 16));
            const float s0 = to_f<T>(*reinterpret_cast<T *>(&r0)), s1 = to_f<T>(*reinterpret_cast<T *>(&r1));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float v = fmaf(__int_as_float(sum[0][m][e]) - kFloat, 256.f, __int_as_float(sum[1][m][e]) - kFloat);
                v = fmaf(v, 256.f, __int_as_float(sum[2][m][e]) - kFloat);
                acc[m][0][e] += ((e < 2 ? s0 : s1) * (e & 1 ? f1 : f0)) * v;
            }
        }
    }
}

// The same with 16-bit operands: the weights as q - 8, x as it is.
template <class T, int N, int NT, int SPG>
__device__ __forceinline__ void line_products_16(float (&acc)[2][NT][4], const uint32_t (&xb)[NT], uint32_t w_at, uint32_t s_at, int line, int left) {
#pragma unroll
    for (int i0 = 0; i0 < 8; i0 += SPG) {
        if (32 * i0 >= left) break;
        float sum[2][N][4];
#pragma unroll
        for (int j = 0; j < SPG; ++j) {
            const int i = i0 + j;
            uint32_t w[4];
            const uint32_t piece = w_at ^ (i << 4);
            w[0] = lds<0>(piece);
            w[1] = lds<1024>(piece);
            w[2] = lds<2048>(piece);
            w[3] = lds<2048 + 1024>(piece);
            int4 b[N];
#pragma unroll
            for (int t = 0; t < N; ++t) b[t] = lds4(xb[t] + line * 512 + i * 64);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                uint32_t lo[4], hi[4];
                unpack<T>(w[2 * m], lo);
                unpack<T>(w[2 * m + 1], hi);
                const float none[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    if (j == 0) mma16<T>(sum[m][t], lo[0], hi[0], lo[1], hi[1], b[t].x, b[t].y, none);
                    else mma16<T>(sum[m][t], lo[0], hi[0], lo[1], hi[1], b[t].x, b[t].y, sum[m][t]);
                }
#pragma unroll
                for (int t = 0; t < N; ++t) mma16<T>(sum[m][t], lo[2], hi[2], lo[3], hi[3], b[t].z, b[t].w, sum[m][t]);
            }
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            uint16_t r0, r1;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(r0) : "r"(s_at + ((i0 / SPG) * kRows + m * 16) * 2));
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(r1) : "r"(s_at + ((i0 / SPG) * kRows + m * 16) * 2 + 16));
            const float s0 = to_f<T>(*reinterpret_cast<T *>(&r0)), s1 = to_f<T>(*reinterpret_cast<T *>(&r1));
#pragma unroll
            for (int t = 0; t < N; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[m][t][e] += (e < 2 ? s0 : s1) * sum[m][t][e];
        }
    }
}

// All lanes ask once (asleep for a while if need be); only a line that is very late is left to one lane's polling.
__device__ __forceinline__ bool wait_line(uint32_t bar, uint32_t parity, volatile int *abort_flag, int *err) {
    if (__all_sync(0xffffffffu, try_nap<false>(bar, parity))) return true;
    return mbar_wait_warp(bar, parity, abort_flag, err);
}

// T: operand type; NT: columns of eight pairs a warp accumulates at a time, one (x in bytes) or three (x as it is); SPG:
// 32-weight steps in a group
template <class T, int NT, int SPG>
__global__ void __launch_bounds__(kThreads, 1)
quant_mv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_s, const __grid_constant__ Args a) {
    constexpr bool BYTES = NT == 1;
    const bool wide = a.out_fp32;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (smem_base - smem_u32(smem_raw));
    int *start = reinterpret_cast<int *>(smem + a.at_start);
    uint16_t *order = reinterpret_cast<uint16_t *>(smem + a.at_order), *x_row = reinterpret_cast<uint16_t *>(smem + a.at_row);
    Job *jobs = reinterpret_cast<Job *>(smem + a.at_jobs);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + a.at_bars + kWarps * kMaxStages * 8);
    volatile int *n_jobs_at = abort_flag + 1;
    const uint32_t x_bar = smem_base + a.at_bars + kWarps * kMaxStages * 8 + 8;   // the rows of x of a batch that come as they are
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t my_bars = smem_base + a.at_bars + warp * kMaxStages * 8;
    const uint32_t my_ring = smem_base + warp * a.stages * kLineBytes, my_scales = smem_base + kWarps * a.stages * kLineBytes + warp * a.stages * scale_bytes(SPG);

    if (lane == 0) {
        for (int s = 0; s < a.stages; ++s) mbar_init(my_bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        mbar_init(x_bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *abort_flag = 0;
        prefetch_map(&map_q);
        prefetch_map(&map_s);
    }
    // (the table from which the pairs are grouped - per warp and slot the pairs before it - lies where the ring and the rows of x
    // will be)
    uint16_t *before = reinterpret_cast<uint16_t *>(smem);
    const int kinds = a.n_slots + 1;                                         // the last one: pairs without a slot
    const bool few = a.pairs <= 32;
    if (!few)
        for (int g = threadIdx.x; g < kWarps * kinds; g += kThreads) before[g] = 0;
    pdl_launch_dependents();
    __syncthreads();
    pdl_wait();

    // ---------------------------------------------------------------------- pairs by slot
    const int32_t *slots = a.slots;
    auto slot_at = [&](int p, bool there) {
        const int raw = there && slots ? *(const volatile int32_t *)(slots + p) : 0;
        if (raw >= a.n_slots && blockIdx.x == 0) atomicOr(a.err, kErrBadIndex);
        return !there ? -1 : raw < 0 || raw >= a.n_slots ? a.n_slots : raw;
    };
    auto scan = [&](int v) {                                                 // inclusive sum over the lanes
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int w = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v += w;
        }
        return v;
    };
    if (few) {
        // one warp sees all pairs: slots in the order of their first pair, pairs without a slot last
        if (warp == 0) {
            const int s = slot_at(lane, lane < a.pairs);
            const uint32_t same = __match_any_sync(0xffffffffu, s), below = (1u << lane) - 1;
            const bool live = s >= 0 && s < a.n_slots, leads = live && !(same & below);
            const int c = __popc(same), nj = leads ? (c + a.job_rows - 1) / a.job_rows : 0;
            const int to = scan(leads ? c : 0), job_to = scan(nj), live_all = __shfl_sync(0xffffffffu, to, 31);
            const int of_leader = __shfl_sync(0xffffffffu, to - c, __ffs(same) - 1), first = live ? of_leader : live_all;
            if (s >= 0) {
                order[first + __popc(same & below)] = (uint16_t)lane;
                x_row[first + __popc(same & below)] = (uint16_t)((lane + a.lead) / a.share);
            }
            for (int j = 0; j < nj; ++j) jobs[job_to - nj + j] = Job{(uint16_t)s, (uint16_t)(to - c + j * a.job_rows), (uint16_t)min(a.job_rows, c - j * a.job_rows), 0};
            if (lane == 31) *n_jobs_at = job_to;
            if (lane == 0) start[a.n_slots] = live_all;
        }
    } else {
        // a stable counting sort, the same in every CTA: each warp counts its stretch of the pairs in order, the warps'
        // counts are added up per slot, and a pair's position is that sum plus its rank in its warp
        const int stretch = ((a.pairs + kThreads - 1) / kThreads) * 32, p_end = min(a.pairs, (warp + 1) * stretch);
        uint16_t *mine = before + warp * kinds;
        constexpr int kMost = (kMaxPairs + kThreads - 1) / kThreads;
        int s_of[kMost], place[kMost];
#pragma unroll
        for (int j = 0; j < kMost; ++j) s_of[j] = 32 * j < stretch ? slot_at(warp * stretch + 32 * j + lane, warp * stretch + 32 * j + lane < p_end) : -1;
#pragma unroll
        for (int j = 0; j < kMost; ++j) {
            if (32 * j >= stretch) break;
            const int s = s_of[j];
            const uint32_t same = __match_any_sync(0xffffffffu, s);
            const int rank = __popc(same & ((1u << lane) - 1)), prior = s >= 0 ? mine[s] : 0;
            __syncwarp();
            if (s >= 0 && rank == 0) mine[s] = (uint16_t)(prior + __popc(same));
            __syncwarp();
            place[j] = prior + rank;
        }
        __syncthreads();
        for (int g = threadIdx.x; g < kinds; g += kThreads) {
            int sum = 0;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const int v = before[w * kinds + g];
                before[w * kinds + g] = (uint16_t)sum;
                sum += v;
            }
            start[g] = sum;
        }
        __syncthreads();
        if (warp == 0) {
            int seen = 0, jobs_before = 0;
            for (int g0 = 0; g0 < kinds; g0 += 32) {
                const int g = g0 + lane, c = g < kinds ? start[g] : 0, nj = g < a.n_slots ? (c + a.job_rows - 1) / a.job_rows : 0;
                const int both = scan(c | nj << 16);                         // two sums of at most 2048 in one
                const int first = seen + (both & 0xffff) - c, first_job = jobs_before + (both >> 16) - nj;
                if (g < kinds) start[g] = first;
                for (int j = 0; j < nj; ++j) jobs[first_job + j] = Job{(uint16_t)g, (uint16_t)(first + j * a.job_rows), (uint16_t)min(a.job_rows, c - j * a.job_rows), 0};
                const int all = __shfl_sync(0xffffffffu, both, 31);
                seen += all & 0xffff;
                jobs_before += all >> 16;
            }
            if (lane == 0) *n_jobs_at = jobs_before;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kMost; ++j)
            if (s_of[j] >= 0) {
                const int p = warp * stretch + 32 * j + lane, to = start[s_of[j]] + mine[s_of[j]] + place[j];
                order[to] = (uint16_t)p;
                x_row[to] = (uint16_t)((p + a.lead) / a.share);
            }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");         // the ring belongs to the copies from here on
    }
    __syncthreads();

    // ---------------------------------------------------------------------- the stream
    // This CTA's tiles (an item: a job's 32-row tile), in batches whose rows of x fit the shared memory.
    const int n_jobs = *n_jobs_at, n_items = n_jobs * a.tiles, grid = (int)gridDim.x, each = n_items / grid, rest = n_items - each * grid;
    int left_items = each + ((int)blockIdx.x < rest);
    const int first_item = each * (int)blockIdx.x + min((int)blockIdx.x, rest);
    int job0 = first_item / a.tiles, tile0 = first_item - job0 * a.tiles;
    const int k_lines = (a.k + kLineK - 1) / kLineK, groups = a.k / (32 * SPG);
    const int r = lane >> 2, c = lane & 3;
    uint32_t ask_stage = 0, stage = 0, phase = 0, x_phase = 0;                            // of the warp's ring, over all batches
    bool ok = true;
    while (left_items > 0) {
        int job1 = job0, rows = 0, items = -tile0;
        while (job1 < n_jobs && items < left_items && rows + jobs[job1].count <= a.x_cap) {
            rows += jobs[job1++].count;
            items += a.tiles;
        }
        items = min(items, left_items);
        const int lines = items * k_lines, l0 = (int)((long long)lines * warp / kWarps), l1 = (int)((long long)lines * (warp + 1) / kWarps);

        // the line being worked on, and the next one to ask for with its rows in the two tensor maps
        int job = job0, line = l0 % k_lines, tile = tile0 + l0 / k_lines;
        while (tile >= a.tiles) { tile -= a.tiles; ++job; }
        int left_to_ask = l1 - l0, ask_job = job, ask_line = line, ask_tile = tile;
        int ask_slot = left_to_ask > 0 ? jobs[job].slot : 0;
        auto issue = [&]() {
            if (left_to_ask <= 0 || !ok) return;
            if (lane == 0) {
                const uint32_t bar = my_bars + 8 * ask_stage;
                mbar_expect_tx(bar, kLineBytes + scale_bytes(SPG));
                tma_load_2d(my_ring + ask_stage * kLineBytes, &map_q, ask_line * (kLineK / 2), ask_slot * a.n + ask_tile * kRows, bar);
                tma_load_2d(my_scales + ask_stage * scale_bytes(SPG), &map_s, ask_tile * kRows, ask_slot * groups + ask_line * (8 / SPG), bar);
            }
            if (++ask_stage == (uint32_t)a.stages) ask_stage = 0;
            --left_to_ask;
            if (++ask_line == k_lines) {
                ask_line = 0;
                if (++ask_tile == a.tiles) {
                    ask_tile = 0;
                    if (left_to_ask > 0) ask_slot = jobs[++ask_job].slot;
                }
            }
        };
        // The batch's rows of x: contiguous in the order of the pairs.
        const int pair_at = jobs[job0].first;
        if constexpr (!BYTES) {
            // as they are, one copy a row
            if (warp == 0) {
                if (lane == 0) mbar_expect_tx(x_bar, (uint32_t)rows * a.k * 2);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); // (the last batch's rows have been read)
                __syncwarp();
                for (int i = lane; i < rows; i += 32)
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                 ::"r"(smem_base + a.at_x + i * a.x_bytes), "l"(a.x + (size_t)x_row[pair_at + i] * a.ldx * 2), "r"(a.k * 2), "r"(x_bar) : "memory");
            }
#pragma unroll 1
            for (int s = 0; s < a.stages; ++s) issue();
            if (ok) ok = mbar_wait_warp(x_bar, x_phase, abort_flag, a.err);
            x_phase ^= 1;
        } else {
            // a line at a time, a few at once: a line is a chain of a load and a dozen shuffles.  The first ones are asked for
            // before the weights, behind which they would wait, and put in place while those are on their way.
            constexpr int kAtOnce = 2;
            uint4 raw[kAtOnce];
            int rows_of[kAtOnce], lines_of[kAtOnce], next_row = warp / k_lines, next_line = warp - next_row * k_lines;
            auto fetch = [&]() {
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    rows_of[j] = next_row;
                    lines_of[j] = next_line;
                    raw[j] = make_uint4(0, 0, 0, 0);
                    const int at_k = next_line * kLineK + lane * 8;
                    if (next_row < rows && at_k < a.k) raw[j] = *reinterpret_cast<const uint4 *>(a.x + ((size_t)x_row[pair_at + next_row] * a.ldx + at_k) * 2);
                    for (next_line += kWarps; next_line >= k_lines; next_line -= k_lines) ++next_row;
                }
            };
            fetch();
#pragma unroll 1
            for (int s = 0; s < a.stages; ++s) issue();
            while (rows_of[0] < rows) {
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    if (rows_of[j] >= rows) break;
                    convert_line<T, SPG>(raw[j], lines_of[j], lines_of[j] * kLineK + lane * 8 < a.k, smem + a.at_x + rows_of[j] * a.x_bytes, a);
                }
                fetch();
            }
        }
        // (the rows of x are in place, and the last batch's partial tiles have been read)
        __syncthreads();

        float acc[2][NT][4];
        Job jb = {};
        uint32_t xb[NT], xc[NT], fac0[NT], fac1[NT];
        bool mine = false;                       // the tile's first line was this warp's
        int pending = -1;                        // line of a tile that this warp began and others go on with, where it stopped
        float *red = reinterpret_cast<float *>(smem + a.at_red);
        // one pass more than lines: after it all partial tiles are in place, and the pending one is finished
#pragma unroll 1
        for (int l = l0; l <= l1; ++l) {
            bool done = false;
            if (l < l1) {
                if (l == l0 || line == 0) {
                    jb = jobs[job];
                    mine = line == 0;
                    const uint32_t base = smem_base + a.at_x + (jb.first - pair_at) * a.x_bytes, fac = a.x_wide + a.x_third;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        // a column behind the job's last pair repeats that one: an MMA column depends on its own operand
                        // only, and it is not stored
                        const uint32_t own = base + min(t * 8 + r, jb.count - 1) * a.x_bytes;
                        xb[t] = own + c * 16;
                        xc[t] = own + a.x_wide + c * 8;
                        fac0[t] = base + min(t * 8 + 2 * c, jb.count - 1) * a.x_bytes + fac;
                        fac1[t] = base + min(t * 8 + 2 * c + 1, jb.count - 1) * a.x_bytes + fac;
                    }
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int t = 0; t < NT; ++t) acc[m][t][0] = acc[m][t][1] = acc[m][t][2] = acc[m][t][3] = 0.f;
                }
                // (after an expired wait the warp walks on without data: the CTA's barriers still need it)
                if (ok) ok = wait_line(my_bars + 8 * stage, phase, abort_flag, a.err);
                if (ok) {
                    const uint32_t w_at = my_ring + stage * kLineBytes + r * 144 + c * 4, s_at = my_scales + stage * scale_bytes(SPG) + r * 2;
                    const int left = a.k - line * kLineK;
                    if constexpr (BYTES) {
                        line_products<T, SPG>(acc, xb[0], xc[0], fac0[0], fac1[0], w_at, s_at, line, left);
                    } else {
                        if (jb.count <= 8) line_products_16<T, 1, NT, SPG>(acc, xb, w_at, s_at, line, left);
                        else if (jb.count <= 16) line_products_16<T, 2, NT, SPG>(acc, xb, w_at, s_at, line, left);
                        else line_products_16<T, 3, NT, SPG>(acc, xb, w_at, s_at, line, left);
                    }
                    if (++stage == (uint32_t)a.stages) { stage = 0; phase ^= 1; }
                    __syncwarp();                                            // all lanes have read the stage
                    issue();
                }
                const bool last = line == k_lines - 1;
                if (mine) {
                    done = last;
                    if (!last && l == l1 - 1) pending = line;
                } else if (last || l == l1 - 1) {
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) red[((warp * 2 + m) * NT * 4 + t * 4 + e) * 32 + lane] = acc[m][t][e];
                }
            } else {
                __syncthreads();                                             // partial tiles are in place, and the rows of x free
                if (pending < 0) break;
                const int tile_end = l1 - 1 - pending + k_lines;
#pragma unroll 1
                for (int w = warp + 1; w < kWarps; ++w) {
                    const int from = (int)((long long)lines * w / kWarps), to = (int)((long long)lines * (w + 1) / kWarps);
                    if (from >= tile_end) break;
                    if (to > from) {
#pragma unroll
                        for (int m = 0; m < 2; ++m)
#pragma unroll
                            for (int t = 0; t < NT; ++t)
#pragma unroll
                                for (int e = 0; e < 4; ++e) acc[m][t][e] += red[((w * 2 + m) * NT * 4 + t * 4 + e) * 32 + lane];
                    }
                }
                done = true;
            }
            if (done) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int at_pair = t * 8 + 2 * c + e;
                        if (at_pair < jb.count) {
                            const size_t to = (size_t)(a.pair0 + order[jb.first + at_pair]) * a.ldo;
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                const int row = tile * kRows + m * 16 + r;
                                if (row < a.n) put<T>(a.out, to + row, acc[m][t][e], wide);
                                if (row + 8 < a.n) put<T>(a.out, to + row + 8, acc[m][t][2 + e], wide);
                            }
                        }
                    }
            }
            if (l < l1 && ++line == k_lines) {
                line = 0;
                if (++tile == a.tiles) { tile = 0; ++job; }
            }
        }
        left_items -= items;
        job0 = job1;
        tile0 = 0;
    }
    // pairs without a slot: rows of zeros
    for (int i = start[a.n_slots] + blockIdx.x * kWarps + warp; i < a.pairs; i += gridDim.x * kWarps)
        for (int n = lane; n < a.n; n += 32) put<T>(a.out, (size_t)(a.pair0 + order[i]) * a.ldo + n, 0.f, wide);
    if (*abort_flag) {                                                       // let copies in flight land
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000ll) {}
    }
}

template <class T, int NT, int SPG>
ew_status_t launch(const CUtensorMap &mq, const CUtensorMap &ms, const Args &a, int smem, int ctas, cudaStream_t st) {
    return launched(launch_pdl(quant_mv_kernel<T, NT, SPG>, dim3(ctas), dim3(kThreads), (size_t)smem, st, mq, ms, a), "4-bit product");
}
template <class T, int NT>
ew_status_t launch_group(int group, const CUtensorMap &mq, const CUtensorMap &ms, const Args &a, int smem, int ctas, cudaStream_t st) {
    if (group == 32) return launch<T, NT, 1>(mq, ms, a, smem, ctas, st);
    if (group == 64) return launch<T, NT, 2>(mq, ms, a, smem, ctas, st);
    return launch<T, NT, 4>(mq, ms, a, smem, ctas, st);
}
template <class T>
ew_status_t launch_type(int nt, int group, const CUtensorMap &mq, const CUtensorMap &ms, const Args &a, int smem, int ctas, cudaStream_t st) {
    return nt == 1 ? launch_group<T, 1>(group, mq, ms, a, smem, ctas, st) : launch_group<T, 3>(group, mq, ms, a, smem, ctas, st);
}
template <class T, int NT>
int setup_one() {
    return (int)cudaFuncSetAttribute(quant_mv_kernel<T, NT, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) |
           (int)cudaFuncSetAttribute(quant_mv_kernel<T, NT, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) |
           (int)cudaFuncSetAttribute(quant_mv_kernel<T, NT, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
}

// Shared memory of a launch: ring and scales, rows of x, barriers, partial tiles, job and pair tables.  As many
// stages a warp as leave room for the rows of x of a whole job.  Returns the bytes, 0 if not even one row fits.
int lay_out(Args &a, int nt, int group) {
    const int groups = a.k / group;
    // rows of x start 64 bytes apart modulo 128: the two rows that a quarter of a warp reads lie in different banks
    a.x_wide = (a.k * 2 + 127) / 128 * 128 + 64;
    a.x_third = nt == 1 ? (a.k + 127) / 128 * 128 : 0;
    a.x_bytes = nt == 1 ? (a.x_wide + a.x_third + groups * 16 + 127) / 128 * 128 + 64 : a.x_wide;
    const int live = a.pairs < a.n_slots ? a.pairs : a.n_slots;
    for (a.stages = kMaxStages; a.stages >= 1; --a.stages) {
        const int ring = kWarps * a.stages * (kLineBytes + scale_bytes(group / 32)), bars = kWarps * kMaxStages * 8 + 16, red = kWarps * 1024 * nt;
        const int fixed = 1024 + ring + 16 + bars + red + (a.n_slots + 1) * 4 + a.pairs * 4;
        // a row of x, and the jobs (eight bytes each) that jobs of so few rows can make
        a.x_cap = 0;
        int jobs = 0;
        for (int rows = 8 * nt < a.pairs ? 8 * nt : a.pairs; rows >= 1; --rows) {
            jobs = live + a.pairs / rows;
            const int cap = (kSmemLimit - fixed - jobs * 8) / a.x_bytes;
            if (cap < rows) continue;
            a.x_cap = cap < a.pairs ? cap : a.pairs;
            a.job_rows = rows;
            break;
        }
        if (a.x_cap < 1) {
            if (a.stages > 1) continue;
            return 0;
        }
        if (a.stages > 1 && a.job_rows < 8 * nt && a.job_rows < a.pairs) continue;
        int o = ring;
        a.at_x = o; o += a.x_cap * a.x_bytes;
        a.at_bars = o = (o + 15) / 16 * 16; o += bars;
        a.at_red = o; o += red;
        a.at_jobs = o; o += jobs * 8;
        a.at_start = o; o += (a.n_slots + 1) * 4;
        a.at_order = o; o += a.pairs * 2;
        a.at_row = o; o += a.pairs * 2;
        // the grouping table lies where ring and rows of x will be
        if (kWarps * (a.n_slots + 1) * 2 <= a.at_bars) return o + 1024;
    }
    return 0;
}

// Packing: eight weights (one 32-bit word) a thread, a group in group / 8 neighbouring lanes.
template <class T>
__global__ void __launch_bounds__(256) quant_pack_kernel(const T *w, long long ldw, long long group_stride, int n, int k, int lanes, long long words, uint32_t *q,
                                                         T *scales) {
    pdl_launch_dependents();
    pdl_wait();
    const int per_row = k / 8, groups = k / (lanes * 8);
    // whole warps walk on together (a group's lanes talk to one another): words behind the last are computed, not written
    for (long long i0 = ((long long)blockIdx.x * blockDim.x + threadIdx.x) & ~31ll; i0 < words; i0 += (long long)gridDim.x * blockDim.x) {
        const long long i = i0 + (threadIdx.x & 31), j = i < words ? i : words - 1;
        const long long row = j / per_row, slot = row / n;
        const int word = (int)(j - row * per_row), rn = (int)(row - slot * n);
        const T *src = w + slot * group_stride + rn * ldw + word * 8;
        float v[8], most = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = (float)src[e];
            most = fmaxf(most, fabsf(v[e]));
        }
        for (int m = 1; m < lanes; m <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, m));
        const T scale = (T)__fdiv_rn(most, 7.f);
        const float s = (float)scale;
        uint32_t bits = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // s = 0 (a group of zeros, or smaller than the type's smallest step): everything stands for 0
            const int level = s > 0.f ? min(max(__float2int_rn(__fdiv_rn(v[e], s)), -8), 7) + 8 : 8;
            bits |= (uint32_t)level << (4 * ((e >> 1) + 4 * (e & 1)));
        }
        if (i < words) {
            q[i] = bits;
            if (word % lanes == 0) scales[(slot * groups + word / lanes) * n + rn] = scale;
        }
    }
}

}  // namespace

int quant_setup() {
    // (the packing kernels too: everything is loaded before a graph may be captured)
    cudaFuncAttributes fa;
    return setup_one<__nv_bfloat16, 1>() | setup_one<__nv_bfloat16, 3>() | setup_one<__half, 1>() | setup_one<__half, 3>() |
           (int)cudaFuncGetAttributes(&fa, quant_pack_kernel<__nv_bfloat16>) | (int)cudaFuncGetAttributes(&fa, quant_pack_kernel<__half>);
}

}  // namespace ops
}  // namespace ew

using namespace ew;
using namespace ew::ops;

static bool bad_group(int32_t group, int32_t k) { return (group != 32 && group != 64 && group != 128) || k < 1 || k % group; }

extern "C" ew_status_t ew_quant_mv(int32_t device, int32_t dtype, int32_t out_dtype, const void *x, int64_t ldx, const void *q, const void *scales,
                                   const int32_t *slots, int32_t pairs, int32_t pairs_per_row, int32_t n_slots, int32_t n, int32_t k, int32_t group, void *y,
                                   int64_t ldy, void *cuda_stream) {
    if (!is_16bit(dtype) || (out_dtype != dtype && out_dtype != EW_FP32)) return refuse("4-bit product: x is bf16 or fp16, results of the same type or fp32");
    if (bad_group(group, k) || k > kMaxK) return refuse("4-bit product: groups of 32, 64 or 128 weights that divide k, k at most 16384");
    if (pairs < 0 || pairs_per_row < 1 || pairs % pairs_per_row || n_slots < 1 || n_slots > kMaxSlots || n < 8 || n % 8 || (int64_t)n_slots * n > 0x7fffffff || kMaxPairs * (((int64_t)n + kRows - 1) / kRows) > 0x7fffffff)
        return refuse("4-bit product: size out of range (n in multiples of 8, at most 2048 slots)");
    // (a tensor without entries may have no address)
    if (pairs > 0 && !slots && n_slots != 1) return refuse("4-bit product: without slot ids there is one matrix");
    if (ldx < k || (ldx & 7) || ldy < n || !q || !scales || (((uintptr_t)q | (uintptr_t)scales) & 15) || ((uintptr_t)slots & 3) ||
        (pairs > 0 && (!x || ((uintptr_t)x & 15) || !y || ((uintptr_t)y & (elem_bytes(out_dtype) - 1)))))
        return refuse("4-bit product: null or misaligned pointer, or overlapping rows (x, q and scales on 16 bytes, ldx a multiple of 8)");
    if (device < 0) return EW_ERR_NO_DEVICE;
    if (pairs == 0) return EW_OK;
    DeviceGuard guard;
    ew_status_t s = launched((int)guard.enter(device), "cudaSetDevice");
    const Device *d;
    if (s != EW_OK || (s = device_state(device, &d)) != EW_OK) return s;
    CUtensorMap mq, ms;
    const uint64_t qd[2] = {(uint64_t)k / 2, (uint64_t)n_slots * n}, qs[1] = {(uint64_t)k / 2};
    const uint64_t sd[2] = {(uint64_t)n, (uint64_t)n_slots * (k / group)}, ss[1] = {(uint64_t)n * 2};
    const uint32_t qbox[2] = {128, kRows}, sbox[2] = {kRows, (uint32_t)(kLineK / group)};
    if ((s = encode_map(*d, &mq, CU_TENSOR_MAP_DATA_TYPE_UINT8, q, 2, qd, qs, qbox, CU_TENSOR_MAP_SWIZZLE_128B)) != EW_OK) return s;
    if ((s = encode_map(*d, &ms, CU_TENSOR_MAP_DATA_TYPE_UINT16, scales, 2, sd, ss, sbox, CU_TENSOR_MAP_SWIZZLE_NONE)) != EW_OK) return s;
    Args a = {};
    a.err = d->err;
    a.out = y;
    a.ldx = ldx;
    a.ldo = ldy;
    a.share = pairs_per_row;
    a.n = n;
    a.k = k;
    a.n_slots = n_slots;
    a.out_fp32 = out_dtype == EW_FP32;
    a.tiles = (n + kRows - 1) / kRows;
    for (int64_t p0 = 0; p0 < pairs; p0 += kMaxPairs) {                      // (the step behind the last launch may pass 2^31)
        a.pair0 = (int)p0;
        a.pairs = pairs - p0 < kMaxPairs ? (int)(pairs - p0) : kMaxPairs;
        a.x = (const uint8_t *)x + (size_t)(p0 / pairs_per_row) * ldx * 2;
        a.lead = (int)(p0 % pairs_per_row);
        a.slots = slots ? slots + p0 : nullptr;
        // One column of eight pairs with x in bytes, or up to three with x as it is: what a slot has more is another job, which
        // reads its weights again.  The bytes' sums are scaled group by group, so they pay with long groups and few pairs.
        // Measured (64 slots of 2816 x 2048; bytes, then 16 bits): groups of 128 with 2 pairs a slot 42 and 48 us, 4: 52 and 53,
        // 8: 70 and 60; groups of 64 with 1 pair 37.6 and 38.4, 3: 57 and 56, 6: 71 and 62.  The pairs are counted against all slots,
        // since the host does not know which of them the batch uses: over mostly unused slots this takes bytes longer than it should.
        const int nt = a.pairs <= 8 || 24ll * a.pairs <= (long long)n_slots * group ? 1 : 3;
        const int smem = lay_out(a, nt, group);
        if (!smem) return refuse("4-bit product: k is too large for a row of x in shared memory");
        const long long most = ((long long)a.pairs / a.job_rows + (a.pairs < n_slots ? a.pairs : n_slots)) * a.tiles;
        const int grid = (int)(most < d->sm_count ? most : d->sm_count);
        cudaStream_t st = (cudaStream_t)cuda_stream;
        s = dtype == EW_BF16 ? launch_type<__nv_bfloat16>(nt, group, mq, ms, a, smem, grid, st) : launch_type<__half>(nt, group, mq, ms, a, smem, grid, st);
        if (s != EW_OK) return s;
    }
    return EW_OK;
}

extern "C" ew_status_t ew_quant_pack(int32_t device, int32_t dtype, const void *w, int64_t ldw, int64_t slot_stride, int32_t n_slots, int32_t n, int32_t k,
                                     int32_t group, void *q, void *scales, void *cuda_stream) {
    if (!is_16bit(dtype)) return refuse("packing: weights are bf16 or fp16");
    if (bad_group(group, k)) return refuse("packing: groups of 32, 64 or 128 weights that divide k");
    if (n_slots < 1 || n < 8 || n % 8) return refuse("packing: size out of range (n in multiples of 8)");
    if (ldw < k || !rows_apart(n_slots, slot_stride, n, ldw, k) || !w || !q || !scales || ((uintptr_t)w & 1) ||
        (((uintptr_t)q | (uintptr_t)scales) & 15))
        return refuse("packing: null or misaligned pointer, or overlapping rows (q and scales on 16 bytes)");
    if (device < 0) return EW_ERR_NO_DEVICE;
    DeviceGuard guard;
    ew_status_t s = launched((int)guard.enter(device), "cudaSetDevice");
    const Device *d;
    if (s != EW_OK || (s = device_state(device, &d)) != EW_OK) return s;
    const long long words = (long long)n_slots * n * (k / 8), ctas = (words + 255) / 256, most = (long long)d->sm_count * 8;
    const dim3 grid((unsigned)(ctas < most ? ctas : most));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int rc = dtype == EW_BF16 ? launch_pdl(quant_pack_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, (const __nv_bfloat16 *)w, ldw, slot_stride, n, k,
                                                 group / 8, words, (uint32_t *)q, (__nv_bfloat16 *)scales)
                                    : launch_pdl(quant_pack_kernel<__half>, grid, dim3(256), 0, st, (const __half *)w, ldw, slot_stride, n, k, group / 8, words,
                                                 (uint32_t *)q, (__half *)scales);
    return launched(rc, "packing");
}
