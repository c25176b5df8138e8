// Matrix-vector products with 4-bit expert weights and group scales, and the packing of the weights.
//
//   y[p, n] = sum_k x[row(p), k] (q[slot(p), n, k] - 8) scale[slot(p), k / group, n]
//
// for a batch's (token, expert) pairs p, whose slots come straight from the router: nothing is sorted or counted before
// the call, every CTA groups the few hundred pairs itself, so that pairs of one slot share its weights' bytes.
//
// Bound by HBM: half a byte a weight and little else.  A stream of 6.5 TB/s is 46 weights a cycle and SM, more than plain
// fp32 arithmetic keeps up with once an expert has several rows, so the products run on the warp-level tensor-core
// instruction m16n8k16: 16 weight rows x 8 pairs (the tcgen05 kernels need 128-row tiles staged as 16-bit values in shared
// memory, i.e. four times the bytes written and read back there).  A warp owns 16 rows and streams them through a ring of
// its own with TMA (2 KiB a stage: 16 rows x 256 weights), no barrier is shared between warps.  Within a 32-weight step a
// lane's word holds eight neighbouring k of one row and its 16 bytes of x the same eight k, so the operands meet without
// any shuffling: the order of k inside an MMA is arbitrary as long as both sides use it.  q - 8 is exact in bf16 and fp16,
// products are summed per group in fp32 and scaled in fp32: no rounding but the result's.
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
constexpr int kStageK = 256;                   // weights of a row in one stage = one 128-byte swizzled line
constexpr int kStageBytes = 16 * kStageK / 2;  // 2 KiB
constexpr int kScaleBytes = 256;               // up to eight groups x 16 rows
constexpr int kStages = 4;
constexpr int kMaxPairs = 2048;                // of one launch; a larger batch is split
constexpr int kMaxSlots = 2048;

struct Args {
    const uint8_t *x;
    const int32_t *slots;       // null: every pair uses slot 0
    void *out;
    int *err;
    long long ldx, ldo;         // elements
    int pairs, pair0, share;    // of this launch; its first pair; pairs per row of x
    int n, k, n_slots;
    int tiles;                  // 16-row tiles of a slot
    int split;                  // warps that share a tile, each with every split-th stage of k
    int out_kind;
};

struct alignas(8) Job { uint16_t slot, first, count, pad; };                // pairs order[first .. first + count) of one slot

__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b, __nv_bfloat16) {
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b, __half) {
    const __half2 r = __hsub2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// Eight 4-bit values to q - 8 in four registers, k ascending: a nibble or-ed into the last mantissa bits of 128 (bf16) or
// 1024 (fp16) is that number plus q, from which 136 (1032) is subtracted exactly.
template <class T>
__device__ __forceinline__ void unpack(uint32_t w, uint32_t (&a)[4]) {
    constexpr bool kBf = sizeof(T) == 2 && __is_same(T, __nv_bfloat16);
    constexpr uint32_t kMagic = kBf ? 0x43004300u : 0x64006400u, kBias = kBf ? 0x43084308u : 0x64086408u;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = sub2(((w >> (4 * i)) & 0x000F000Fu) | kMagic, kBias, T());
}
template <class T>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (__is_same(T, __nv_bfloat16))
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <class T> __device__ __forceinline__ float scale_at(const uint8_t *s, int i);
template <> __device__ __forceinline__ float scale_at<__nv_bfloat16>(const uint8_t *s, int i) { return __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(s)[i]); }
template <> __device__ __forceinline__ float scale_at<__half>(const uint8_t *s, int i) { return __half2float(reinterpret_cast<const __half *>(s)[i]); }

__device__ __forceinline__ void put(void *out, size_t at, float v, int kind) {
    if (kind == EW_FP32) reinterpret_cast<float *>(out)[at] = v;
    else if (kind == EW_BF16) reinterpret_cast<__nv_bfloat16 *>(out)[at] = __float2bfloat16_rn(v);
    else reinterpret_cast<__half *>(out)[at] = __float2half_rn(v);
}

// Shared memory.  The tables from which the pairs are grouped (per warp and slot the pairs before it, per pair its place)
// lie in the ring, which is not in use yet.
struct Layout {
    int scales, bars, red, start, jobs, order, bytes;
    int place, slot_of;                         // in the ring, behind the counters
    __host__ __device__ Layout(int nt, int split, int n_slots, int pairs) {
        int o = kWarps * kStages * kStageBytes;
        scales = o; o += kWarps * kStages * kScaleBytes;
        bars = o; o += kWarps * kStages * 8 + 16;
        red = o; o += split > 1 ? kWarps * 128 * nt * 4 : 0;
        jobs = o; o += pairs * 8;
        start = o; o += (n_slots + 1) * 4;
        order = o; o += pairs * 2;
        bytes = o + 1024;
        place = kWarps * (n_slots + 1) * 2;
        slot_of = place + pairs * 2;
    }
};
static_assert(kWarps * (kMaxSlots + 1) * 2 + kMaxPairs * 4 <= kWarps * kStages * kStageBytes, "the grouping tables fit the ring");
static_assert(kWarps * kStages * (kStageBytes + kScaleBytes + 8) + 16 + kWarps * 128 * 4 * 4 + kMaxPairs * 10 + (kMaxSlots + 1) * 4 + 1024 <= 227 * 1024, "shared memory");

// T: operand type; NT: columns of eight pairs a warp accumulates at a time; SPG: 32-weight steps in a group
template <class T, int NT, int SPG>
__global__ void __launch_bounds__(kThreads, 1)
quant_mv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_s, const __grid_constant__ Args a) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (smem_base - smem_u32(smem_raw));
    const Layout L(NT, a.split, a.n_slots, a.pairs);
    int *start = reinterpret_cast<int *>(smem + L.start);
    uint16_t *order = reinterpret_cast<uint16_t *>(smem + L.order);
    uint16_t *before = reinterpret_cast<uint16_t *>(smem), *place = reinterpret_cast<uint16_t *>(smem + L.place), *slot_of = reinterpret_cast<uint16_t *>(smem + L.slot_of);
    Job *jobs = reinterpret_cast<Job *>(smem + L.jobs);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L.bars + kWarps * kStages * 8);
    volatile int *n_jobs_at = abort_flag + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t my_bars = smem_base + L.bars + warp * kStages * 8;
    const uint32_t my_ring = smem_base + warp * kStages * kStageBytes, my_scales = smem_base + L.scales + warp * kStages * kScaleBytes;

    if (lane == 0) {
        for (int s = 0; s < kStages; ++s) mbar_init(my_bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        prefetch_map(&map_q);
        prefetch_map(&map_s);
    }
    const int kinds = a.n_slots + 1;                                         // the last one: pairs without a slot
    for (int g = threadIdx.x; g < kWarps * kinds; g += kThreads) before[g] = 0;
    pdl_launch_dependents();
    __syncthreads();
    pdl_wait();

    // ---------------------------------------------------------------------- pairs by slot
    // A stable counting sort, the same in every CTA: each warp counts its stretch of the pairs in order, the warps' counts
    // are added up per slot, and a pair's position is that sum plus its rank in its warp.
    const int32_t *slots = a.slots;
    const int stretch = ((a.pairs + kThreads - 1) / kThreads) * 32, p_end = min(a.pairs, (warp + 1) * stretch);
    uint16_t *mine = before + warp * kinds;
    bool bad = false;
    for (int p0 = warp * stretch; p0 < p_end; p0 += 32) {
        const int p = p0 + lane;
        const bool there = p < p_end;
        const int raw = there && slots ? *(const volatile int32_t *)(slots + p) : 0;
        const int s = !there ? -1 : raw < 0 || raw >= a.n_slots ? a.n_slots : raw;
        bad |= raw >= a.n_slots;
        const uint32_t same = __match_any_sync(0xffffffffu, s);
        const int rank = __popc(same & ((1u << lane) - 1)), prior = there ? mine[s] : 0;
        __syncwarp();
        if (there && rank == 0) mine[s] = (uint16_t)(prior + __popc(same));
        __syncwarp();
        if (there) {
            place[p] = (uint16_t)(prior + rank);
            slot_of[p] = (uint16_t)s;
        }
    }
    if (bad && blockIdx.x == 0) atomicOr(a.err, kErrBadIndex);
    __syncthreads();
    for (int g = threadIdx.x; g < kinds; g += kThreads) {
        int sum = 0;
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
            const int g = g0 + lane, c = g < kinds ? start[g] : 0, nj = g < a.n_slots ? (c + 8 * NT - 1) / (8 * NT) : 0;
            int inc = c, jinc = nj;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, inc, d), w = __shfl_up_sync(0xffffffffu, jinc, d);
                if (lane >= d) { inc += v; jinc += w; }
            }
            const int first = seen + inc - c;
            if (g < kinds) start[g] = first;
            for (int j = 0; j < nj; ++j)
                jobs[jobs_before + jinc - nj + j] = Job{(uint16_t)g, (uint16_t)(first + j * 8 * NT), (uint16_t)min(8 * NT, c - j * 8 * NT), 0};
            seen += __shfl_sync(0xffffffffu, inc, 31);
            jobs_before += __shfl_sync(0xffffffffu, jinc, 31);
        }
        if (lane == 0) *n_jobs_at = jobs_before;
    }
    __syncthreads();
    for (int p = threadIdx.x; p < a.pairs; p += kThreads) {
        const int s = slot_of[p];
        order[start[s] + before[(p / stretch) * kinds + s] + place[p]] = (uint16_t)p;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");             // the ring belongs to the copies from here on
    __syncthreads();

    // ---------------------------------------------------------------------- the stream
    const int n_items = *n_jobs_at * a.tiles;
    const int team = warp / a.split, part = warp - team * a.split, teams = kWarps / a.split;
    const int first_item = blockIdx.x * teams + team, step_items = gridDim.x * teams;
    const int k_stages = (a.k + kStageK - 1) / kStageK;
    const int my_stages = k_stages > part ? (k_stages - part + a.split - 1) / a.split : 0;       // of every item
    constexpr uint32_t kTx = kStageBytes + (8 / SPG) * 32;
    const int groups = a.k / (32 * SPG);

    int i_item = first_item, i_stage = 0;                                    // the next stage to ask for
    uint32_t issued = 0, used = 0;
    auto issue = [&]() {
        if (i_item >= n_items || my_stages == 0) return;
        const int job = i_item / a.tiles, tile = i_item - job * a.tiles, kb = part + i_stage * a.split;
        const uint32_t s = issued % kStages, bar = my_bars + 8 * s;
        const int slot = jobs[job].slot;
        if (lane == 0) {
            mbar_expect_tx(bar, kTx);
            tma_load_2d(my_ring + s * kStageBytes, &map_q, kb * (kStageK / 2), slot * a.n + tile * 16, bar);
            tma_load_2d(my_scales + s * kScaleBytes, &map_s, tile * 16, slot * groups + kb * (8 / SPG), bar);
        }
        ++issued;
        if (++i_stage == my_stages) { i_stage = 0; i_item += step_items; }
    };
    for (int s = 0; s < kStages; ++s) issue();

    const int r = lane >> 2, c = lane & 3;
    bool ok = true;
    for (int item = first_item; item < n_items; item += step_items) {
        const int job = item / a.tiles, tile = item - job * a.tiles;
        const Job jb = jobs[job];
        const int n_tiles = (jb.count + 7) >> 3;
        const uint8_t *xp[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int m = t * 8 + r;
            xp[t] = m < jb.count ? a.x + ((size_t)((a.pair0 + order[jb.first + m]) / a.share) * a.ldx + 8 * c) * 2 : nullptr;
        }
        float acc[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.f;
        for (int j = 0; j < my_stages; ++j) {
            const int k0 = (part + j * a.split) * kStageK, steps = min(kStageK, a.k - k0) >> 5;
            const uint32_t s = used % kStages;
            const uint8_t *w_at = smem + (my_ring - smem_base) + s * kStageBytes + r * 128 + c * 4;
            const uint8_t *s_at = smem + (my_scales - smem_base) + s * kScaleBytes;
            // (after an expired wait the warp walks on without data: its team's barriers still need it)
            if (ok) ok = mbar_wait_warp(my_bars + 8 * s, (used / kStages) & 1, abort_flag, a.err);
            if (!ok) continue;
            ++used;
#pragma unroll
            for (int i0 = 0; i0 < 8; i0 += SPG) {
                if (i0 < steps) {
                    float sum[NT][4];
#pragma unroll
                    for (int t = 0; t < NT; ++t) sum[t][0] = sum[t][1] = sum[t][2] = sum[t][3] = 0.f;
#pragma unroll
                    for (int i = i0; i < i0 + SPG; ++i) {
                        uint32_t lo[4], hi[4];
                        const uint8_t *w = w_at + ((i ^ r) << 4);
                        unpack<T>(*reinterpret_cast<const uint32_t *>(w), lo);
                        unpack<T>(*reinterpret_cast<const uint32_t *>(w + 1024), hi);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            if (t < n_tiles) {
                                uint4 b = make_uint4(0, 0, 0, 0);
                                if (xp[t]) b = *reinterpret_cast<const uint4 *>(xp[t] + (size_t)(k0 + 32 * i) * 2);
                                mma<T>(sum[t], lo[0], hi[0], lo[1], hi[1], b.x, b.y);
                                mma<T>(sum[t], lo[2], hi[2], lo[3], hi[3], b.z, b.w);
                            }
                        }
                    }
                    const float s0 = scale_at<T>(s_at, (i0 / SPG) * 16 + r), s1 = scale_at<T>(s_at, (i0 / SPG) * 16 + 8 + r);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        acc[t][0] += s0 * sum[t][0];
                        acc[t][1] += s0 * sum[t][1];
                        acc[t][2] += s1 * sum[t][2];
                        acc[t][3] += s1 * sum[t][3];
                    }
                }
            }
            __syncwarp();                                                    // all lanes have read the stage
            issue();
        }
        if (a.split > 1) {
            // the team's parts meet in shared memory and are added in order
            float *red = reinterpret_cast<float *>(smem + L.red) + (size_t)team * a.split * 128 * NT;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) red[(part * NT * 4 + t * 4 + e) * 32 + lane] = acc[t][e];
            asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(a.split * 32) : "memory");
            if (part == 0) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        for (int q = 1; q < a.split; ++q) acc[t][e] += red[(q * NT * 4 + t * 4 + e) * 32 + lane];
            }
            asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(a.split * 32) : "memory");
            if (part) continue;
        }
        const int row = tile * 16 + r;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int m = t * 8 + 2 * c + e;
                if (m < jb.count) {
                    const size_t at = (size_t)(a.pair0 + order[jb.first + m]) * a.ldo + row;
                    if (row < a.n) put(a.out, at, acc[t][e], a.out_kind);
                    if (row + 8 < a.n) put(a.out, at + 8, acc[t][2 + e], a.out_kind);
                }
            }
    }
    // pairs without a slot: rows of zeros
    for (int i = start[a.n_slots] + blockIdx.x * kWarps + warp; i < a.pairs; i += gridDim.x * kWarps)
        for (int n = lane; n < a.n; n += 32) put(a.out, (size_t)(a.pair0 + order[i]) * a.ldo + n, 0.f, a.out_kind);
    if (*abort_flag) {                                                       // let copies in flight land
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000ll) {}
    }
}

template <class T, int NT, int SPG>
ew_status_t launch(const CUtensorMap &mq, const CUtensorMap &ms, const Args &a, int ctas, cudaStream_t st) {
    const Layout L(NT, a.split, a.n_slots, a.pairs);
    return launched(launch_pdl(quant_mv_kernel<T, NT, SPG>, dim3(ctas), dim3(kThreads), (size_t)L.bytes, st, mq, ms, a), "4-bit product");
}
template <class T, int NT>
ew_status_t launch_group(int group, const CUtensorMap &mq, const CUtensorMap &ms, const Args &a, int ctas, cudaStream_t st) {
    if (group == 32) return launch<T, NT, 1>(mq, ms, a, ctas, st);
    if (group == 64) return launch<T, NT, 2>(mq, ms, a, ctas, st);
    return launch<T, NT, 4>(mq, ms, a, ctas, st);
}
template <class T, int NT>
int setup_one() {
    const int most = 227 * 1024;
    return (int)cudaFuncSetAttribute(quant_mv_kernel<T, NT, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) |
           (int)cudaFuncSetAttribute(quant_mv_kernel<T, NT, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) |
           (int)cudaFuncSetAttribute(quant_mv_kernel<T, NT, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
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
    return setup_one<__nv_bfloat16, 1>() | setup_one<__nv_bfloat16, 4>() | setup_one<__half, 1>() | setup_one<__half, 4>();
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
    if (bad_group(group, k)) return refuse("4-bit product: groups of 32, 64 or 128 weights that divide k");
    if (pairs < 0 || pairs_per_row < 1 || pairs % pairs_per_row || n_slots < 1 || n_slots > kMaxSlots || n < 8 || n % 8 || (int64_t)n_slots * n > 0x7fffffff ||
        (int64_t)n_slots * (k / group) > 0x7fffffff)
        return refuse("4-bit product: size out of range (n in multiples of 8, at most 2048 slots)");
    if (!slots && n_slots != 1) return refuse("4-bit product: without slot ids there is one matrix");
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
    const uint32_t qbox[2] = {128, 16}, sbox[2] = {16, (uint32_t)(kStageK / group)};
    if ((s = encode_map(*d, &mq, CU_TENSOR_MAP_DATA_TYPE_UINT8, q, 2, qd, qs, qbox, CU_TENSOR_MAP_SWIZZLE_128B)) != EW_OK) return s;
    if ((s = encode_map(*d, &ms, CU_TENSOR_MAP_DATA_TYPE_UINT16, scales, 2, sd, ss, sbox, CU_TENSOR_MAP_SWIZZLE_NONE)) != EW_OK) return s;
    Args a = {};
    a.x = (const uint8_t *)x;
    a.out = y;
    a.err = d->err;
    a.ldx = ldx;
    a.ldo = ldy;
    a.share = pairs_per_row;
    a.n = n;
    a.k = k;
    a.n_slots = n_slots;
    a.tiles = (n + 15) / 16;
    a.out_kind = out_dtype;
    const int k_stages = (k + kStageK - 1) / kStageK;
    for (int32_t p0 = 0; p0 < pairs; p0 += kMaxPairs) {
        a.pair0 = p0;
        a.pairs = pairs - p0 < kMaxPairs ? pairs - p0 : kMaxPairs;
        a.slots = slots ? slots + p0 : nullptr;
        // A slot of few pairs needs one column of the MMA, a busy one up to four at a time.
        const bool narrow = a.pairs <= 8 || a.pairs <= 2 * n_slots;
        const long long live = a.pairs < n_slots ? a.pairs : n_slots, items = live * a.tiles;
        // Too few tiles for all warps: several warps share one, each with a part of k.
        a.split = 1;
        while (a.split < kWarps && a.split < k_stages && items * a.split * 2 <= (long long)d->sm_count * kWarps) a.split *= 2;
        const long long most_jobs = a.pairs / (narrow ? 8 : 32) + live, ctas = (most_jobs * a.tiles * a.split + kWarps - 1) / kWarps;
        const int grid = (int)(ctas < d->sm_count ? ctas : d->sm_count);
        cudaStream_t st = (cudaStream_t)cuda_stream;
        if (dtype == EW_BF16)
            s = narrow ? launch_group<__nv_bfloat16, 1>(group, mq, ms, a, grid, st) : launch_group<__nv_bfloat16, 4>(group, mq, ms, a, grid, st);
        else
            s = narrow ? launch_group<__half, 1>(group, mq, ms, a, grid, st) : launch_group<__half, 4>(group, mq, ms, a, grid, st);
        if (s != EW_OK) return s;
    }
    return EW_OK;
}

extern "C" ew_status_t ew_quant_pack(int32_t device, int32_t dtype, const void *w, int64_t ldw, int64_t slot_stride, int32_t n_slots, int32_t n, int32_t k,
                                     int32_t group, void *q, void *scales, void *cuda_stream) {
    if (!is_16bit(dtype)) return refuse("packing: weights are bf16 or fp16");
    if (bad_group(group, k)) return refuse("packing: groups of 32, 64 or 128 weights that divide k");
    if (n_slots < 1 || n < 8 || n % 8) return refuse("packing: size out of range (n in multiples of 8)");
    if (ldw < k || (n_slots > 1 && slot_stride < (int64_t)(n - 1) * ldw + k) || !w || !q || !scales || ((uintptr_t)w & 1) ||
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
