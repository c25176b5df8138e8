// RMS norm with the residual's addition, its result in 16 bits, in 8-bit blocks or in both, and its gradient.
//
//   t = x + residual, rounded to their type (the stream as it is kept: the norm and its gradient are of that)
//   y = t r w,   r = 1 / sqrt(mean(t^2) + eps)                                  of a row
//   dt = r (g - u mean(g u)) + dt_in,   g = dy w, u = t r;     dw = sum over the rows of dy u
//
// Bound by HBM: forward 2 to 4 bytes of operands and 1 to 5 of results a value, backward 6 or 8, each read or written once: a row
// stays in the registers of a warp (or of 8 or 16, for wide rows and few) between the sum and its use.  The weight's gradient
// is summed in the registers of the threads that own its columns, over all rows that a CTA meets; a second kernel adds the
// CTAs' sums up, in the same order every time (few rows: one cluster of CTAs, one kernel).  Measured: 8192 x 2048 with a
// residual and both results 25.6 us = 5.9 TB/s (90 % of the measured copy bandwidth); its gradient 27.2 us = 4.9 TB/s, 23 of them the
// first kernel's stream.
#include "ew_blocks.cuh"
#include "ew_ops.h"
#include "ew_tc.cuh"

#include <cstdlib>

namespace ew {
namespace ops {
namespace {
using namespace blocks;

constexpr int kThreads = 256;
constexpr int kMostWidth = 16384;                      // sixteen warps with four spans each
template <int W> constexpr int kThreadsOf = W == 1 ? kThreads : W * 32;     // several warps a row: a CTA a row

struct Args {
    const void *x, *residual, *weight;
    void *sum, *y;
    uint8_t *q, *scales;
    long long ldx, ldr, ldsum, ldy, ldq, lds, rows;
    int width;
    float inv_width, eps;
};

// The sum over the W warps of a row, in every thread of them.  `turn`: of the calls, so that one barrier a call is enough.
template <int W, int N>
__device__ __forceinline__ void add_up(float (&v)[N], int turn) {
#pragma unroll
    for (int d = 16; d; d >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(kAll, v[i], d);
    if (W == 1) return;
    __shared__ __align__(16) float part[2][N][W];
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) part[turn & 1][i][threadIdx.x >> 5] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) v[i] += part[turn & 1][i][w];
    }
}

// W warps a row, NV spans a warp
template <class T, bool VEC, int W, int NV>
__global__ void __launch_bounds__(kThreadsOf<W>) norm_kernel(const Args a) {
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    constexpr int kRows = kThreadsOf<W> / 32 / W;
    const int lane = threadIdx.x & 31, w = (threadIdx.x >> 5) % W;
    int turn = 0;
    for (long long r = (long long)blockIdx.x * kRows + (threadIdx.x >> 5) / W; r < a.rows; r += (long long)gridDim.x * kRows) {
        Eight<T> t[NV];
        {
            Eight<T> more[NV];
            const T *x = reinterpret_cast<const T *>(a.x) + r * a.ldx, *res = a.residual ? reinterpret_cast<const T *>(a.residual) + r * a.ldr : x;
#pragma unroll
            for (int i = 0; i < NV; ++i) load_span<T, VEC>(t[i], x, (i * W + w) * kSpan, lane, a.width);
            if (a.residual) {
#pragma unroll
                for (int i = 0; i < NV; ++i) load_span<T, VEC>(more[i], res, (i * W + w) * kSpan, lane, a.width);
                T *sum = reinterpret_cast<T *>(a.sum) + r * a.ldsum;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    Two xv[4], rv[4];
                    to_pairs(xv, t[i]);
                    to_pairs(rv, more[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) xv[j] = add2(xv[j], rv[j]);
                    from_pairs(t[i], xv);
                    store_span<T, VEC>(t[i], sum, (i * W + w) * kSpan, lane, a.width);
                }
            }
        }
        Two square = two(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Two v[4];
            clear_span<T, VEC>(t[i], (i * W + w) * kSpan, lane, a.width);
            to_pairs(v, t[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) square = fma2(v[j], v[j], square);
        }
        float ss[1] = {parts_of(square).x + parts_of(square).y};
        add_up<W, 1>(ss, turn++);
        const float norm = rsqrtf(ss[0] * a.inv_width + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (i * W + w) * kSpan;
            Eight<T> weight, y;
            load_span<T, VEC>(weight, reinterpret_cast<const T *>(a.weight), at, lane, a.width);
            Two tv[4], wv[4];
            to_pairs(tv, t[i]);
            to_pairs(wv, weight);
#pragma unroll
            for (int j = 0; j < 4; ++j) tv[j] = mul2(mul2(tv[j], two(norm, norm)), wv[j]);
            from_pairs(y, tv);
            if (a.y) store_span<T, VEC>(y, reinterpret_cast<T *>(a.y) + r * a.ldy, at, lane, a.width);
            if (a.q && at < a.width) put_span<VEC, false>(tv, a.q + r * a.ldq, a.scales + r * a.lds, at, lane, a.width);
        }
    }
}

// The gradient's CTAs are counted in SMs of a B200, whatever the device: their sums are the workspace, whose size a caller learns without naming one.
constexpr int kSms = 148;
constexpr int kMostCtas = 3 * kSms;                    // (8192 x 2048: 27 us; two an SM 34, four 31)
constexpr int kMostStages = 3;
// A CTA's rows on their way, at least one of the widest, of three operands; where one CTA has the SM, two (1024 x 16384: 46.8 us, with one 47.8)
template <int W> constexpr int kRingBytes = W == 16 ? 196608 : 98304;
static_assert(kMostWidth * 6 * 2 <= kRingBytes<16>, "room for two rows");

struct GradArgs {
    const void *dy, *t, *weight, *more;
    void *dt;
    float *parts;                                      // [gridDim.x, width]: each CTA's sums for dw
    long long lddy, ldt, ldmore, lddt, rows;
    int *err;
    int width, stages;
    float inv_width, eps;
};

// Teams of W warps (eight teams of one, or one team a CTA), a row a team at a time, its columns' sums in the registers of the threads that own
// them.  BULK: rows come to shared memory by bulk copies, up to kMostStages of them ahead of the one that is worked on; without them a
// team's loads wait for the row before.  Needs rows on 16-byte boundaries of a multiple of eight values.
template <class T, bool BULK, int W, int NV>
__global__ void __launch_bounds__(kThreadsOf<W>, W == 4 && NV <= 2 ? 3 : W == 1 && NV <= 2 ? 2 : 1) grad_kernel(const GradArgs a) {
    tc::pdl_launch_dependents();
    constexpr int kRows = kThreadsOf<W> / 32 / W;
    extern __shared__ __align__(128) uint8_t ring[];   // [teams][stages][t, dy, dt_in][width]; at the end, with several teams, their sums
    __shared__ uint64_t bars[kRows * kMostStages];
    __shared__ int abort_word;
    volatile int *abort_flag = &abort_word;
    const int lane = threadIdx.x & 31, w = (threadIdx.x >> 5) % W, team = (threadIdx.x >> 5) / W;
    const bool fetcher = threadIdx.x % (W * 32) == 0;
    const uint32_t row_bytes = (uint32_t)a.width * 2, stage_bytes = row_bytes * (a.more ? 3 : 2);
    const uint32_t bar = tc::smem_u32(bars + team * kMostStages);
    const uint8_t *stages = ring + team * a.stages * stage_bytes;
    const uint32_t stages_at = tc::smem_u32(stages);
    const long long first = (long long)blockIdx.x * kRows + team, step = (long long)gridDim.x * kRows;
    auto fetch = [&](long long r, int stage) {         // by one thread
        const uint32_t to = stages_at + stage * stage_bytes, full = bar + 8 * stage;
        tc::mbar_expect_tx(full, stage_bytes);
        tc::bulk_load(to, reinterpret_cast<const T *>(a.t) + r * a.ldt, row_bytes, full);
        tc::bulk_load(to + row_bytes, reinterpret_cast<const T *>(a.dy) + r * a.lddy, row_bytes, full);
        if (a.more) tc::bulk_load(to + 2 * row_bytes, reinterpret_cast<const T *>(a.more) + r * a.ldmore, row_bytes, full);
    };
    if (BULK) {
        if (threadIdx.x == 0) {
            for (int i = 0; i < kRows * kMostStages; ++i) tc::mbar_init(tc::smem_u32(bars + i), 1);
            abort_word = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
    }
    tc::pdl_wait();
    if (BULK && fetcher)
        for (int i = 0; i < a.stages; ++i)
            if (first + i * step < a.rows) fetch(first + i * step, i);
    constexpr bool kHold = W * NV < 64;                // the weights in registers; those of the widest rows are read again (4096 x 16384: 123 us, held 128, for what spills; without a third operand 110 and 120)
    Two weight[kHold ? NV : 1][4], dw[NV][4];
    auto weight_of = [&](Two (&v)[4], int i) {
        Eight<T> x;
        load_span<T, BULK>(x, reinterpret_cast<const T *>(a.weight), (i * W + w) * kSpan, lane, a.width);
        to_pairs(v, x);
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (kHold) weight_of(weight[i], i);
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[i][j] = two(0.f, 0.f);
    }
    int turn = 0, stage = 0, phase = 0;
    for (long long r = first; r < a.rows; r += step) {
        Eight<T> dy[NV], t[NV], more[NV];
        const T *t_row, *dy_row, *more_row;
        if (BULK) {
            // Every lane waits for itself: what the copy wrote is visible to the threads that saw its phase end, and to no others.  (Where it
            // gives up, the rest is wrong and reported, but ends.)
            tc::wait_all<false>(bar + 8 * stage, phase, abort_flag, a.err);
            t_row = reinterpret_cast<const T *>(stages + stage * stage_bytes);
            dy_row = t_row + a.width;
            more_row = dy_row + a.width;
        } else {
            t_row = reinterpret_cast<const T *>(a.t) + r * a.ldt;
            dy_row = reinterpret_cast<const T *>(a.dy) + r * a.lddy;
            more_row = reinterpret_cast<const T *>(a.more) + r * a.ldmore;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            load_span<T, BULK>(t[i], t_row, (i * W + w) * kSpan, lane, a.width);
            load_span<T, BULK>(dy[i], dy_row, (i * W + w) * kSpan, lane, a.width);
        }
        if (a.more)
#pragma unroll
            for (int i = 0; i < NV; ++i) load_span<T, BULK>(more[i], more_row, (i * W + w) * kSpan, lane, a.width);
        Two square = two(0.f, 0.f), along2 = square;   // sums of t^2 and of dy w t
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Two tv[4], dv[4];
            clear_span<T, BULK>(t[i], (i * W + w) * kSpan, lane, a.width);
            to_pairs(tv, t[i]);
            to_pairs(dv, dy[i]);
            if (!kHold) weight_of(weight[0], i);
            Two (&wv)[4] = weight[kHold ? i : 0];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                square = fma2(tv[j], tv[j], square);
                along2 = fma2(mul2(dv[j], wv[j]), tv[j], along2);
            }
        }
        float sums[2] = {parts_of(square).x + parts_of(square).y, parts_of(along2).x + parts_of(along2).y};
        add_up<W, 2>(sums, turn++);
        if (BULK) {                                    // every thread of the team has its part of the stage: the next row may come, unless a wait gave up with a copy still on its way
            if (W == 1) {                              // (several warps have met at a barrier)
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            if (fetcher && r + a.stages * step < a.rows && !*abort_flag) fetch(r + a.stages * step, stage);
            if (++stage == a.stages) { stage = 0; phase ^= 1; }
        }
        const float norm = rsqrtf(sums[0] * a.inv_width + a.eps), along = norm * norm * (sums[1] * a.inv_width);      // mean(g u) = norm mean(g t)
        const Two norm2 = two(norm, norm), back = two(-norm * along, -norm * along);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Eight<T> dt;
            Two tv[4], dv[4], mv[4];
            to_pairs(tv, t[i]);
            to_pairs(dv, dy[i]);
            if (!kHold) weight_of(weight[0], i);
            Two (&wv)[4] = weight[kHold ? i : 0];
            if (a.more) to_pairs(mv, more[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Two scaled = mul2(dv[j], norm2);
                dw[i][j] = fma2(scaled, tv[j], dw[i][j]);
                tv[j] = fma2(scaled, wv[j], a.more ? fma2(tv[j], back, mv[j]) : mul2(tv[j], back));
            }
            from_pairs(dt, tv);
            store_span<T, BULK>(dt, reinterpret_cast<T *>(a.dt) + r * a.lddt, (i * W + w) * kSpan, lane, a.width);
        }
    }
    float *part = a.parts + (long long)blockIdx.x * a.width, *mine = kRows > 1 ? reinterpret_cast<float *>(ring) + team * a.width : part;
    if (kRows > 1) __syncthreads();                    // all rows have been read
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = (i * W + w) * kSpan + place<BULK>(lane, j);
            const float2 f = parts_of(dw[i][j >> 1]);
            if (c < a.width) mine[c] = j & 1 ? f.y : f.x;
        }
    if (kRows > 1) {
        __syncthreads();
        for (int c = threadIdx.x; c < a.width; c += kThreadsOf<W>) {
            float v = 0.f;
#pragma unroll
            for (int k = 0; k < kRows; ++k) v += reinterpret_cast<const float *>(ring)[k * a.width + c];
            part[c] = v;
        }
    }
    if (BULK) {
        __syncthreads();
        if (*abort_flag) {                             // let copies in flight land before the CTA's memory is reused
            const long long t0 = clock64();
            while (clock64() - t0 < 2000000ll) {}
        }
    }
}

// The gradient of few rows in one launch: a cluster of sixteen CTAs, four teams of four warps in each, a row a team at a time, the next one
// asked for before this one is worked on.  The teams' and then the CTAs' sums for dw are added up through shared memory, in their
// order.  One launch and no workspace take the host 4 us less, which is what a call of few rows waits for; a replayed graph does not wait for
// it, and there the two kernels above are faster from 130 to 220 rows on.  Replayed and called from Python, us, with the two kernels behind the stroke:
//   2048 columns: 64 rows 5.4, 11.3 / 6.3, 15.0; 220: 8.6, 11.3 / 8.4, 15.1; 333: 10.7, 11.3 / 8.9, 15.1; 384: 11.5, 11.9 / 8.7, 15.1; 512: 13.7, 14.2 / 8.9, 15.1
//   1024 columns: 64 rows 3.8, 11.2 / 6.0, 15.0; 220: 5.6, 11.2 / 5.6, 15.1; 384: 7.3, 11.2 / 6.1, 15.1; 512: 8.6, 11.2 / 5.8, 15.1
//    300 columns: 64 rows 3.8, 11.2 / 4.6, 15.1; 128: 4.8, 11.1 / 4.7, 15.1; 384: 8.6, 11.2 / 5.1, 15.2; 512: 10.4, 11.2 / 5.1, 15.2
// The limit is where a call from Python gains what a replayed one loses, 3 us.  (Clusters of eight: 333 rows of 2048 17.4 us replayed.)
// (A device whose GPCs, or what this process has of them, hold no cluster of sixteen takes one of eight, which all hold.)
constexpr int kMostCluster = 16, kPortableCluster = 8, kTeams = 4, kTeamWarps = 4;
constexpr int kFewRows = 384, kFewWidth = 2048;

__device__ __forceinline__ float peer_value(const float *p, uint32_t rank) {
    float v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}" : "=f"(v) : "r"(tc::smem_u32(p)), "r"(rank) : "memory");
    return v;
}

template <class T, bool VEC, int NV, int CLUSTER>
__global__ void __launch_bounds__(kTeams * kTeamWarps * 32, 1) few_rows_kernel(const GradArgs a) {
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    constexpr int W = kTeamWarps;
    extern __shared__ float columns[];                 // [kTeams][width]
    __shared__ __align__(16) float part[kTeams][2][2][W];
    const int lane = threadIdx.x & 31, w = (threadIdx.x >> 5) % W, team = (threadIdx.x >> 5) / W, step = CLUSTER * kTeams;
    const int rank = (int)tc::cluster_ctarank();
    Eight<T> dy[NV], t[NV], more[NV];
    auto load = [&](int r) {
        r = min(r, (int)a.rows - 1);
        const T *dy_row = reinterpret_cast<const T *>(a.dy) + r * a.lddy, *t_row = reinterpret_cast<const T *>(a.t) + r * a.ldt;
        const T *more_row = a.more ? reinterpret_cast<const T *>(a.more) + r * a.ldmore : t_row;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            load_span<T, VEC>(t[i], t_row, (i * W + w) * kSpan, lane, a.width);
            load_span<T, VEC>(dy[i], dy_row, (i * W + w) * kSpan, lane, a.width);
            load_span<T, VEC>(more[i], more_row, (i * W + w) * kSpan, lane, a.width);
        }
    };
    const int first = rank + CLUSTER * team;          // (one row a CTA before two)
    load(first);
    Two weight[NV][4], dw[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        Eight<T> x;
        load_span<T, VEC>(x, reinterpret_cast<const T *>(a.weight), (i * W + w) * kSpan, lane, a.width);
        to_pairs(weight[i], x);
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[i][j] = two(0.f, 0.f);
    }
    int turn = 0;
    for (int r = first; r < (int)a.rows; r += step, turn ^= 1) {
        Two tv[NV][4], dv[NV][4], mv[NV][4], square = two(0.f, 0.f), along2 = square;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            clear_span<T, VEC>(t[i], (i * W + w) * kSpan, lane, a.width);
            to_pairs(tv[i], t[i]);
            to_pairs(dv[i], dy[i]);
            to_pairs(mv[i], more[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                square = fma2(tv[i][j], tv[i][j], square);
                along2 = fma2(mul2(dv[i][j], weight[i][j]), tv[i][j], along2);
            }
        }
        load(r + step);
        float sums[2] = {parts_of(square).x + parts_of(square).y, parts_of(along2).x + parts_of(along2).y};
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            sums[0] += __shfl_xor_sync(kAll, sums[0], d);
            sums[1] += __shfl_xor_sync(kAll, sums[1], d);
        }
        if (lane == 0) {
            part[team][turn][0][w] = sums[0];
            part[team][turn][1][w] = sums[1];
        }
        asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + team), "n"(W * 32) : "memory");
        sums[0] = sums[1] = 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k) {
            sums[0] += part[team][turn][0][k];
            sums[1] += part[team][turn][1][k];
        }
        const float norm = rsqrtf(sums[0] * a.inv_width + a.eps), along = norm * norm * (sums[1] * a.inv_width);
        const Two norm2 = two(norm, norm), back = two(-norm * along, -norm * along);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Eight<T> dt;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Two scaled = mul2(dv[i][j], norm2);
                Two v = a.more ? fma2(tv[i][j], back, mv[i][j]) : mul2(tv[i][j], back);
                v = fma2(scaled, weight[i][j], v);
                dw[i][j] = fma2(scaled, tv[i][j], dw[i][j]);
                round_pair(dt.v + 2 * j, parts_of(v));
            }
            store_span<T, VEC>(dt, reinterpret_cast<T *>(a.dt) + r * a.lddt, (i * W + w) * kSpan, lane, a.width);
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = (i * W + w) * kSpan + place<VEC>(lane, j);
            const float2 f = parts_of(dw[i][j >> 1]);
            if (c < a.width) columns[team * a.width + c] = j & 1 ? f.y : f.x;
        }
    __syncthreads();
    for (int c = threadIdx.x; c < a.width; c += kTeams * W * 32) {
        float v = columns[c];
#pragma unroll
        for (int k = 1; k < kTeams; ++k) v += columns[k * a.width + c];
        columns[c] = v;
    }
    __syncwarp();                                      // (the cluster's barrier is one of whole warps, and the last turn of such a loop may have had a part of one)
    tc::cluster_sync_all();
    const int share = (a.width + CLUSTER - 1) / CLUSTER, from = rank * share, to = min(from + share, a.width);
    for (int c = from + threadIdx.x; c < to; c += kTeams * W * 32) {
        float x[CLUSTER], v = 0.f;
#pragma unroll
        for (int k = 0; k < CLUSTER; ++k) x[k] = peer_value(columns + c, k);
#pragma unroll
        for (int k = 0; k < CLUSTER; ++k) v += x[k];
        a.parts[c] = v;
    }
    __syncwarp();
    tc::cluster_sync_all();                            // until then the others read this CTA's sums
}

// dw[c] = the sum of parts[:, c]: 32 columns a CTA, 32 threads a column
__global__ void __launch_bounds__(1024) parts_kernel(const float *parts, float *dw, int n_parts, int width) {
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float x[(kMostCtas + 31) / 32], v = 0.f;           // all of a thread's loads are on their way together
#pragma unroll
    for (int i = 0; i < (kMostCtas + 31) / 32; ++i) x[i] = c < width && warp + 32 * i < n_parts ? parts[(long long)(warp + 32 * i) * width + c] : 0.f;
#pragma unroll
    for (int i = 0; i < (kMostCtas + 31) / 32; ++i) v += x[i];
    sums[warp][lane] = v;
    __syncthreads();
    v = sums[lane][warp];
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
    if (lane == 0 && blockIdx.x * 32 + warp < width) dw[blockIdx.x * 32 + warp] = v;
}

template <class T, bool VEC, int W, int NV>
ew_status_t launch(const Args &a, cudaStream_t st) {
    constexpr int kRows = kThreadsOf<W> / 32 / W;
    const long long ctas = (a.rows + kRows - 1) / kRows, most = 0x7fffffff;
    return launched(launch_pdl(norm_kernel<T, VEC, W, NV>, dim3((unsigned)(ctas < most ? ctas : most)), dim3(kThreadsOf<W>), 0, st, a), "RMS norm");
}

// (8192 x 2048: four warps a row 25.7 us, two 28.3, eight 28.8, one 33; one row: 2.0, 2.9, 1.8 us.  65536 x 256: one span a lane 26.1, two
// 33.4; 32768 x 512: one warp 25.3, two 35, four 44; 16384 x 1024: two 25.5, four 27.3; 4096 x 4096: eight 26.3, four 27.2; 2048 x 8192: eight
// 30.4, sixteen 41)
template <class T, bool VEC>
ew_status_t pick(const Args &a, cudaStream_t st) {
    if (a.width <= 256) return launch<T, VEC, 1, 1>(a, st);
    if (a.width <= 512) return launch<T, VEC, 1, 2>(a, st);
    if (a.width <= 1024) return launch<T, VEC, 2, 2>(a, st);
    if (a.width <= 2048) return launch<T, VEC, 4, 2>(a, st);
    if (a.width <= 4096) return launch<T, VEC, 8, 2>(a, st);
    if (a.width <= 8192) return launch<T, VEC, 8, 4>(a, st);
    return launch<T, VEC, 16, 4>(a, st);
}

// Up to here a warp a row, eight rows a CTA, then a CTA a row: with short rows a CTA a row has too few bytes on their way and meets at a
// barrier a row (65536 x 256: 25.8 us against 157; 32768 x 512: 26.8, 81; 16384 x 1024: 26.1, 38; 600 x 1024: 5.3, 6.0; 400 x 512: 5.3, 5.0).
// As many CTAs as stay on the SMs at once (65536 x 256: 444 of them 25.8 us, 296 34.6, 148 58; 32768 x 512: 296 26.8, 148 34.9,
// 444 30.1; 16384 x 1024: 148 26.2, 296 28.9; 4096 x 4096: 296 29.8, 444 33.9; 2048 x 8192: 148 30.1, 296 35, 444 42; 1024 x 16384: 148 47, 444 69).
constexpr int kNarrow = 1024;
int grad_ctas(long long rows, int width) {
    const long long wanted = width <= kNarrow ? (rows + 7) / 8 : rows,
                    most = kSms * (width <= 256 ? 3 : width <= 512 ? 2 : width <= kNarrow ? 1 : width <= 2048 ? 3 : width <= 4096 ? 2 : 1);
    return (int)(wanted < most ? wanted : most);
}
bool few_rows(long long rows, int width) { return rows <= kFewRows && width <= kFewWidth; }

// One cluster of so many CTAs
void few_config(cudaLaunchConfig_t *cfg, cudaLaunchAttribute *attr, int cluster, int width) {
    cfg->gridDim = dim3(cluster);
    cfg->blockDim = dim3(kTeams * kTeamWarps * 32);
    cfg->dynamicSmemBytes = (size_t)kTeams * width * 4;
    attr->id = cudaLaunchAttributeClusterDimension;
    attr->val.clusterDim.x = cluster;
    attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
    cfg->attrs = attr;
    cfg->numAttrs = 1;
}

template <class T, bool VEC, int NV>
ew_status_t launch_few(const Device &d, GradArgs a, float *dw, cudaStream_t st) {
    a.parts = dw;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    few_config(&cfg, attr, d.few_rows_cluster, a.width);
    cfg.stream = st;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    if (pdl_enabled()) cfg.numAttrs = 2;
    return launched((int)(d.few_rows_cluster == kMostCluster ? cudaLaunchKernelEx(&cfg, few_rows_kernel<T, VEC, NV, kMostCluster>, a)
                                                             : cudaLaunchKernelEx(&cfg, few_rows_kernel<T, VEC, NV, kPortableCluster>, a)), "RMS norm gradient");
}

template <class T, bool BULK, int W, int NV>
ew_status_t launch_grad(GradArgs a, float *dw, cudaStream_t st) {
    constexpr int kRows = kThreadsOf<W> / 32 / W;
    const int ctas = grad_ctas(a.rows, a.width), stage_bytes = a.width * 2 * (a.more ? 3 : 2) * kRows, fit = kRingBytes<W> / stage_bytes;
    a.stages = fit < 1 ? 1 : fit < kMostStages ? fit : kMostStages;
    const int sums = kRows > 1 ? kRows * a.width * 4 : 0, ring = BULK ? a.stages * stage_bytes : 0;
    const ew_status_t s = launched(launch_pdl(grad_kernel<T, BULK, W, NV>, dim3((unsigned)ctas), dim3(kThreadsOf<W>), ring > sums ? ring : sums, st, a), "RMS norm gradient");
    if (s != EW_OK) return s;
    return launched(launch_pdl(parts_kernel, dim3((unsigned)((a.width + 31) / 32)), dim3(1024), 0, st, (const float *)a.parts, dw, ctas, a.width), "RMS norm gradient");
}

template <class T, bool BULK>
ew_status_t pick_grad(const Device &d, const GradArgs &a, float *dw, cudaStream_t st) {
    if (few_rows(a.rows, a.width)) return a.width <= 1024 ? launch_few<T, BULK, 1>(d, a, dw, st) : launch_few<T, BULK, 2>(d, a, dw, st);
    if (a.width <= 256) return launch_grad<T, BULK, 1, 1>(a, dw, st);
    if (a.width <= 512) return launch_grad<T, BULK, 1, 2>(a, dw, st);
    if (a.width <= kNarrow) return launch_grad<T, BULK, 1, 4>(a, dw, st);
    if (a.width <= 2048) return launch_grad<T, BULK, 4, 2>(a, dw, st);
    if (a.width <= 4096) return launch_grad<T, BULK, 8, 2>(a, dw, st);
    if (a.width <= 8192) return launch_grad<T, BULK, 16, 2>(a, dw, st);
    return launch_grad<T, BULK, 16, 4>(a, dw, st);
}

template <class T, bool BULK, int W, int NV>
int load_grad() {
    return (int)cudaFuncSetAttribute(grad_kernel<T, BULK, W, NV>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes<W>);
}

template <class T, bool VEC, int NV>
int load_few(int *cluster) {
    const auto kernel = few_rows_kernel<T, VEC, NV, kMostCluster>;
    cudaFuncAttributes fa;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    few_config(&cfg, &attr, kMostCluster, kFewWidth);
    int fit = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess || cudaOccupancyMaxActiveClusters(&fit, kernel, &cfg) != cudaSuccess || fit < 1) {
        cudaGetLastError();                            // (an answer, not an error)
        *cluster = kPortableCluster;
    }
    return (int)cudaFuncGetAttributes(&fa, kernel) | (int)cudaFuncGetAttributes(&fa, few_rows_kernel<T, VEC, NV, kPortableCluster>);
}

template <class T, bool VEC>
int load_one(int *cluster) {
    cudaFuncAttributes fa;
    return (int)cudaFuncGetAttributes(&fa, norm_kernel<T, VEC, 1, 1>) | (int)cudaFuncGetAttributes(&fa, norm_kernel<T, VEC, 1, 2>) |
           (int)cudaFuncGetAttributes(&fa, norm_kernel<T, VEC, 2, 2>) | (int)cudaFuncGetAttributes(&fa, norm_kernel<T, VEC, 4, 2>) | (int)cudaFuncGetAttributes(&fa, norm_kernel<T, VEC, 8, 2>) |
           (int)cudaFuncGetAttributes(&fa, norm_kernel<T, VEC, 8, 4>) | (int)cudaFuncGetAttributes(&fa, norm_kernel<T, VEC, 16, 4>) |
           load_grad<T, VEC, 1, 1>() | load_grad<T, VEC, 1, 2>() | load_grad<T, VEC, 1, 4>() | load_grad<T, VEC, 4, 2>() | load_grad<T, VEC, 8, 2>() | load_grad<T, VEC, 16, 2>() | load_grad<T, VEC, 16, 4>() |
           load_few<T, VEC, 1>(cluster) | load_few<T, VEC, 2>(cluster) | (int)cudaFuncGetAttributes(&fa, parts_kernel);
}

bool bad_eps(float eps) { return !(eps >= 0.f && eps <= 3.402823466e38f); }

}  // namespace

// Loads the kernels (a first launch inside a graph capture would have to) and finds out which cluster the gradient of few rows can have
// (EW_DISABLE_CLUSTER16=1: the portable one).
int norm_setup(Device *d) {
    const char *e = getenv("EW_DISABLE_CLUSTER16");
    int *c = &d->few_rows_cluster;
    *c = e && e[0] == '1' ? kPortableCluster : kMostCluster;
    return load_one<__nv_bfloat16, false>(c) | load_one<__nv_bfloat16, true>(c) | load_one<__half, false>(c) | load_one<__half, true>(c);
}

}  // namespace ops
}  // namespace ew

using namespace ew;
using namespace ew::ops;

extern "C" ew_status_t ew_rms_norm(int32_t device, int32_t dtype, const void *x, int64_t ldx, const void *residual, int64_t ldres, const void *weight, float eps,
                                   int32_t rows, int32_t width, void *sum, int64_t ldsum, void *y, int64_t ldy, void *q, int64_t ldq, void *scales,
                                   int64_t ldscales, void *cuda_stream) {
    if (!is_16bit(dtype)) return refuse("RMS norm: bf16 or fp16");
    if (rows < 0 || width < 1 || width > kMostWidth || bad_eps(eps)) return refuse("RMS norm: size or eps out of range");
    if (!y && !q && rows > 0) return refuse("RMS norm: no result is wanted");
    if (ldx < width || (residual && (ldres < width || ldsum < width)) || (y && ldy < width) || (q && (ldq < width || ldscales < (width + blocks::kBlock - 1) / blocks::kBlock)))
        return refuse("RMS norm: rows overlap");
    if (rows > 0 && (!x || !weight || (residual && !sum) || (q && !scales) || (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)weight | (uintptr_t)sum | (uintptr_t)y) & 1)))
        return refuse("RMS norm: null or misaligned pointer");
    if (device < 0) return EW_ERR_NO_DEVICE;
    if (rows == 0) return EW_OK;
    DeviceGuard guard;
    ew_status_t s = launched((int)guard.enter(device), "cudaSetDevice");
    const Device *d;
    if (s != EW_OK || (s = device_state(device, &d)) != EW_OK) return s;
    const Args a = {x, residual, weight, residual ? sum : nullptr, y, (uint8_t *)q, (uint8_t *)scales, ldx, residual ? ldres : 0, residual ? ldsum : 0, y ? ldy : 0, q ? ldq : 0,
                    q ? ldscales : 0, rows, width, (float)(1.0 / width), eps};
    const bool vec = !((((uintptr_t)x | (uintptr_t)residual | (uintptr_t)weight | (uintptr_t)a.sum | (uintptr_t)y) & 15) | ((uintptr_t)q & 7) |
                       ((a.ldx | a.ldr | a.ldsum | a.ldy | a.ldq | width) & 7));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == EW_BF16) return vec ? pick<__nv_bfloat16, true>(a, st) : pick<__nv_bfloat16, false>(a, st);
    return vec ? pick<__half, true>(a, st) : pick<__half, false>(a, st);
}

extern "C" int32_t ew_rms_norm_grad_parts(int32_t rows, int32_t width) {
    return rows < 1 || few_rows(rows, width) ? 0 : grad_ctas(rows, width);
}

extern "C" ew_status_t ew_rms_norm_grad(int32_t device, int32_t dtype, const void *dy, int64_t lddy, const void *t, int64_t ldt, const void *weight, const void *dt_in,
                                        int64_t lddt_in, float eps, int32_t rows, int32_t width, void *dt, int64_t lddt, float *dweight, float *workspace,
                                        void *cuda_stream) {
    if (!is_16bit(dtype)) return refuse("RMS norm: bf16 or fp16");
    if (rows < 0 || width < 1 || width > kMostWidth || bad_eps(eps)) return refuse("RMS norm: size or eps out of range");
    if (lddy < width || ldt < width || (dt_in && lddt_in < width) || lddt < width) return refuse("RMS norm: rows overlap");
    if (!dweight || ((uintptr_t)dweight & 3) ||
        (rows > 0 && (!dy || !t || !weight || !dt || (!workspace && !few_rows(rows, width)) || ((uintptr_t)workspace & 3) || (((uintptr_t)dy | (uintptr_t)t | (uintptr_t)weight | (uintptr_t)dt_in | (uintptr_t)dt) & 1))))
        return refuse("RMS norm: null or misaligned pointer");
    if (device < 0) return EW_ERR_NO_DEVICE;
    DeviceGuard guard;
    ew_status_t s = launched((int)guard.enter(device), "cudaSetDevice");
    const Device *d;
    if (s != EW_OK || (s = device_state(device, &d)) != EW_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (rows == 0) return launched((int)cudaMemsetAsync(dweight, 0, (size_t)width * 4, st), "cudaMemsetAsync");
    const GradArgs a = {dy, t, weight, dt_in, dt, workspace, lddy, ldt, dt_in ? lddt_in : 0, lddt, rows, d->err, width, 0, (float)(1.0 / width), eps};
    const bool vec = !((((uintptr_t)dy | (uintptr_t)t | (uintptr_t)weight | (uintptr_t)dt_in | (uintptr_t)dt) & 15) | ((a.lddy | a.ldt | a.ldmore | a.lddt | width) & 7));
    if (dtype == EW_BF16) return vec ? pick_grad<__nv_bfloat16, true>(*d, a, dweight, st) : pick_grad<__nv_bfloat16, false>(*d, a, dweight, st);
    return vec ? pick_grad<__half, true>(*d, a, dweight, st) : pick_grad<__half, false>(*d, a, dweight, st);
}
