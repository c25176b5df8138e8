// Products of 8-bit floating-point rows and weights with a scale for each block of 128, grouped by expert, and their input
// gradient (tcgen05 block-scaled products + TMEM + TMA).
//
//   product         y [r, n] = sum_k (x[r, k] 2^sx[r, k/128]) (w[g, n, k] 2^sw[g, n/128, k/128])     rows r of group g
//   input gradient  dx[r, k] = sum_n (dy[r, n] 2^sdy[r, n/128]) (w[g, n, k] 2^sw[g, n/128, k/128])
//
// The form is that of the 16-bit grouped products: the output's contiguous axis f is the MMA's M axis, the rows c its N axis, the
// summed axis t is staged 128 bytes at a time, a block's length:
//   D[f, c] = sum_t A[f, t] B[c, t],   out[row(c), f] = D[f, c]
//               f   t    A                            B
//   product     n   k    w[g]  (t contiguous)         x  (t contiguous)
//   dx          k   n    w[g]  (f contiguous)         dy (t contiguous)
//
// The scales are powers of two held as exponents, which the tensor core takes as they are: an instruction multiplies 32 terms and
// scales them by one exponent of A's row and one of B's, read from tensor memory, before it adds them to the fp32 accumulator.
// A column of tensor memory holds four exponents of a row, so the exponents of four k-blocks are brought there at a time: a warp
// gathers them into shared memory in the tensor core's order (row r at 16 (r mod 32) + 4 (r / 32), a byte a k-block), and the MMA
// thread has them copied right before the products that use them.  A tile's 128 f share A's exponent, a block of the weights'
// scales.  There are kSlots such places, in shared and in tensor memory; one is written again after the products that
// read it have finished.
//
// Two tile widths as in the 16-bit products: 128 columns on one CTA, and a CTA pair with 256 f x 224 columns (two accumulator sets of 256
// would leave the exponents no tensor memory).
//
// Measured (one B200; copy bandwidth 6551 GB/s, cuBLAS bf16 1669 TFLOP/s in a burst, 1392 sustained):
//   y,  1536 rows, 96 groups, 2816 x 2048   93 us = 6.1 TB/s, 92 % of the copy bandwidth (bound by the weights' bytes)
//   y, 49152 rows, 64 groups, 2816 x 2048   286 to 313 us sustained = 1.8 to 2.0 PFLOP/s, bound by power (1.04 GHz at 990 W); 235 us in a
//                                           burst of milliseconds, 211 us = 2.7 PFLOP/s for one launch on an idle GPU
//   y, 49152 rows, one group, 2816 x 2048   240 us sustained = 2.4 PFLOP/s (cuBLAS, 8 bits: 238 with a scale for 32 values, 258 with one in all)
//   dx, 24582 rows, 64 groups, 2048 x 1408  90 to 92 us sustained, 75 in a burst, 72 for one launch
//   y, 6 rows of 64 groups, 2816 x 2048     9.9 us: 35 MB, 5.3 us of stream, behind launch, offsets and the first copies
// Without its scales (one kind of product less) the prompt takes the same time.

#include "ew_ops.h"
#include "ew_tc.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace ew {
namespace ops {
namespace {
using namespace tc;

enum Way { kProduct = 0, kInputGrad = 1 };

constexpr int kBlock = 128;                            // values a scale; bytes of a stage's row
constexpr int threads_of(int epilogue_warps) { return (3 + epilogue_warps) * 32; }       // TMA, MMA, epilogue, scales
constexpr int kATile = 128 * kBlock;                   // 16 KiB: 128 f of one stage
constexpr int kSmemLimit = 227 * 1024;
constexpr int kMaxStages = 7;
constexpr int kSlots = 4;                              // places for the exponents of four k-blocks
constexpr int kMaps = 8;                               // row boxes of 16, 32 .. 128 rows
constexpr int kTiles = 2;                              // 16-bit results on their way out: tiles of 64 f x 32 rows of each pair of epilogue warps
// Long sums are made in parts that the epilogue adds up in fp32, as in the 16-bit products and for the same reason: 2048 terms for
// fp32 results, 8192 for fp16, 65536 for bf16.  (Products of 8-bit values have few digits: over terms of one sign and size 1.1e-7 of the result is cut
// off in 1024 of them; with a first block 2^12 times the others up to 7e-6, 1.4e-5 in 2048, 5.5e-5 in 8192.  At most it is what lies below 2^-25 of
// the largest addend's power of two, of 33 addends an instruction, and the sum's 24th bit: 9.25 steps of 2^-23 an instruction, 7.1e-5 in 2048 terms
// (a first term 2^26 times all others: 5.4e-5 measured), 2.8e-4 in 8192, 2.3e-3 in 65536, where the worst order of fp32 additions loses 1.2e-4, 4.9e-4, 3.9e-3.)
constexpr int sum_blocks(int out_dtype) { return (out_dtype == EW_FP32 ? 2048 : out_dtype == EW_FP16 ? 8192 : 65536) / kBlock; }

struct Args {
    const int32_t *offsets;                            // null: one group, all rows
    const uint8_t *row_scales, *w_scales;
    void *out;
    int *err;
    long long ldo, lds;                                // elements between output rows; bytes between the rows' scales
    int rows, groups;
    int f_size, t_size;                                // the output's contiguous axis, the summed axis
    int f_tiles;
    int nb, kb;                                        // blocks of w along n and k
    int out_kind;                                      // ew_dtype_t
    int sum_blocks;
    int e5m2;                                          // type of the rows
    int words;                                         // the rows' scales start on 4-byte boundaries
    int wide;                                          // 16-bit results whose rows lie on 16-byte boundaries, f_size a multiple of eight
    int stages;
};

// CG: CTAs that share one MMA tile (1, or 2 = a pair with 256 f); NT: columns of an accumulator set; EW: epilogue warps, four or
// eight (two to each quarter of the TMEM lanes, taking turns at the columns)
template <int CG, int NT, int EW>
struct Cfg {
    static constexpr int kThreads = (3 + EW) * 32, kScaleWarp = 2 + EW, kStaging = EW / 2 * kTiles * 4096;
    static constexpr int kBRows = NT / CG;             // c staged by each CTA
    static constexpr int kStageBytes = kATile + kBRows * kBlock;
    static constexpr int kTile = 128 * CG;             // f of an item
    static constexpr int kStep = 16 * CG;              // granularity of an MMA's N
    static constexpr int kBChunks = (NT + 127) / 128;  // of 128 rows' exponents: 512 bytes, four columns
    static constexpr int kSlotBytes = 512 * (1 + kBChunks);
    static constexpr int kScaleCol = 2 * NT;           // tensor memory: two accumulator sets, then the exponents
    static constexpr int kSlotCols = 4 * (1 + kBChunks);
    static_assert(kScaleCol + kSlots * kSlotCols <= 512, "fits the tensor memory");
    static_assert(kStageBytes % 1024 == 0, "tiles on their swizzle's boundary");
};

struct RowMaps { CUtensorMap m[kMaps]; };

struct Item {
    int g, f0, row0, cols, kb, chunk;                  // cols: output rows of this item; kb: k-blocks; chunk: k-blocks summed in the tensor core at a time
};

// 128-byte swizzle, MN-major, 8-bit: rows of 128 values along the output, eight to a group of 1 KiB along the summed axis
__device__ __forceinline__ uint64_t desc_mnmajor(uint32_t addr) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3FFFF) >> 4);
    d |= (uint64_t)(16384 >> 4) << 16;                 // the next 128 values along the output: there are none
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// 32 rows of 16 bytes side by side, no swizzle: groups of eight rows 128 bytes apart
__device__ __forceinline__ uint64_t desc_scales(uint32_t addr) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3FFFF) >> 4);
    d |= (uint64_t)(128 >> 4) << 16;
    d |= (uint64_t)(128 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    return d;
}
template <int CG>
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap *m, int x, int y, uint32_t bar) {
    if constexpr (CG == 1) tma_load_2d(dst, m, x, y, bar);
    else tma2_load_2d(dst, m, x, y, bar);
}
template <int CG>
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap *m, int x, int y, int z, uint32_t bar) {
    if constexpr (CG == 1) tma_load_3d(dst, m, x, y, z, bar);
    else tma2_load_3d(dst, m, x, y, z, bar);
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
}
// 512 bytes of exponents to four columns, the same in all four quarters of the lanes; a pair's CTAs each copy their own
template <int CG>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    if constexpr (CG == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
    if constexpr (CG == 1) tc_commit(bar);
    else tc2_commit_both(bar);
}
template <int CG>
__device__ __forceinline__ void arrive_leader(uint32_t bar) {
    if constexpr (CG == 1) mbar_arrive(bar);
    else mbar_arrive_leader(bar);
}

// Columns of the accumulator into `lim` output rows: a warp writes 32 neighbouring f of a row at a time.
template <class T>
__device__ __forceinline__ void store_columns(T *p, long long ldo, const uint32_t (&v)[32], int lim) {
    T *q[8];                                           // eight addresses that do not wait for one another
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = p + j * ldo;
    const long long step = 8 * ldo;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        if (j < lim) *q[j & 7] = (T)__uint_as_float(v[j]);
        q[j & 7] += step;
    }
}
// Pairs of epilogue warps: 2 and 3, 4 and 5 ..., and their barriers
__device__ __forceinline__ uint32_t pair_index() { return (threadIdx.x >> 6) - 1; }
__device__ __forceinline__ uint32_t pair_barrier() { return 1 + pair_index(); }
__device__ __forceinline__ bool both_of_pair(bool ok) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)ok), "r"(pair_barrier()) : "memory");
    return r != 0;
}
// The same for 16-bit results in rows on 16-byte boundaries.  A warp reads its 32 x 32 part of the accumulator in the order of the
// small matrix instructions' results and turns it over on the way to shared memory, where it and its neighbour fill a tile of 32 rows of 64 f
// (128 bytes; pieces of 16 bytes exchanged by the row, the copy's swizzle, so that no bank is met twice).  A bulk copy takes the tile away while the next
// is filled; of rows behind the item's end only the others are stored, 16 bytes a lane.
// (Prompt and input gradient: 242 and 75 us; 32 stores of two bytes a lane 261 and 95, of 16 bytes 258 and 78.)
template <bool BF16>
__device__ __forceinline__ void store_tile(uint32_t taddr, uint8_t *tile, const CUtensorMap *map, int f, int row0, uint16_t *p, long long ldo, int lim, int lane, int odd, int f_left) {
    uint32_t v[2][16];
    tc_ld16x256(taddr, v[0]);
    tc_ld16x256(taddr + (16u << 16), v[1]);
    tc_wait_ld();
    const uint32_t at = smem_u32(tile);
#pragma unroll
    for (int i = 0; i < 4; ++i) {                      // eight columns a time: four 8 x 8 matrices, 8 f each
        uint32_t m[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float lo = __uint_as_float(v[j >> 1][4 * i + 2 * (j & 1)]), hi = __uint_as_float(v[j >> 1][4 * i + 2 * (j & 1) + 1]);
            if (BF16) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
                m[j] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __half2 h = __floats2half2_rn(lo, hi);
                m[j] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
        const int row = 8 * i + (lane & 7), piece = odd * 4 + (lane >> 3);
        asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                     ::"r"(at + row * 128 + ((piece ^ (row & 7)) << 4)), "r"(m[0]), "r"(m[1]), "r"(m[2]), "r"(m[3]) : "memory");
    }
    const bool copier = lane == 0 && !odd;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (copier) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kTiles - 2) : "memory");      // the next tile is free again
    asm volatile("barrier.cta.sync %0, 64;" ::"r"(pair_barrier()) : "memory");
    if (lim >= 32) {
        if (copier)
            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];\n\tcp.async.bulk.commit_group;"
                         ::"l"(map), "r"(at), "r"(f), "r"(row0) : "memory");
    } else {
        const int piece = odd * 4 + (lane & 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 8 * i + (lane >> 2);
            const uint4 x = *reinterpret_cast<const uint4 *>(tile + row * 128 + ((piece ^ (row & 7)) << 4));
            if (row < lim && (lane & 3) * 8 < f_left) *reinterpret_cast<uint4 *>(p + row * ldo + (lane & 3) * 8) = x;
        }
    }
}
__device__ __forceinline__ void add_columns(float *p, long long ldo, const uint32_t (&v)[32], int lim) {
#pragma unroll
    for (int j0 = 0; j0 < 32; j0 += 8) {
        float old[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j0 + j < lim) old[j] = p[j * ldo];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j0 + j < lim) p[j * ldo] = old[j] + __uint_as_float(v[j0 + j]);
        p += 8 * ldo;
    }
}

// LONG: 16-bit results whose sums may have several parts (more than 8192 terms: four epilogue warps)
template <int CG, int NT, int EW, int WAY, bool LONG>
__global__ void __launch_bounds__(threads_of(EW), 1)
scaled_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ RowMaps map_b, const __grid_constant__ CUtensorMap map_out,
                      const __grid_constant__ Args a) {
    using C = Cfg<CG, NT, EW>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem_al = smem_raw + (smem_base - smem_u32(smem_raw));
    // after the ring: 16-bit results on their way out; the exponents; barriers full, empty [kMaxStages] each, exponents full, empty [kSlots] each, tmem full, empty [2]
    // each; TMEM base, abort flag; then the group table: first block of each group, first row, rows
    uint8_t *staging = smem_al + a.stages * C::kStageBytes, *scales = staging + C::kStaging;
    uint64_t *bars = reinterpret_cast<uint64_t *>(scales + kSlots * C::kSlotBytes);
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * kMaxStages, bar_sfull = bar_empty + 8 * kMaxStages, bar_sempty = bar_sfull + 8 * kSlots;
    const uint32_t bar_tfull = bar_sempty + 8 * kSlots, bar_tempty = bar_tfull + 16;
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(bars + 2 * kMaxStages + 2 * kSlots + 4);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    int *t_pre = reinterpret_cast<int *>(tmem_holder + 2), *t_lo = t_pre + a.groups + 1, *t_cnt = t_lo + a.groups;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_ctarank() : 0;
    const int unit = blockIdx.x / CG, units = gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(bar_sfull + 8 * i, CG);
            mbar_init(bar_sempty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_tfull + 8 * i, 1);
            mbar_init(bar_tempty + 8 * i, EW * CG);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&map_a);
    }
    if (warp == 1) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)), "r"(512u) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)), "r"(512u) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
        pdl_launch_dependents();                       // (once the tensor memory is held: a kernel that found room beside this one and took some of it would wait for this one's end)
    }
    pdl_wait();                                        // the operands and the offsets may come from the kernel before
    if (warp == 0) {
        // group table: first row and rows of each group, and the number of row blocks before it.  Offsets are clamped to
        // the matrix and to the largest one before them, so that whatever the call was given the groups lie inside the
        // matrix and apart from one another.
        // The offsets of 128 groups are asked for together.
        auto offset = [&](int g) { return a.offsets ? *(const volatile int32_t *)(a.offsets + g) : g ? a.rows : 0; };
        int before = 0, raw = offset(0), end = min(max(raw, 0), a.rows);
        bool bad = raw != end;
        for (int g0 = 0; g0 < a.groups; g0 += 128) {
            int next[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) next[c] = offset(min(g0 + 32 * c + lane, a.groups - 1) + 1);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int g = g0 + 32 * c + lane;
                int hi = g < a.groups ? min(max(next[c], 0), a.rows) : end;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, hi, d);
                    if (lane >= d) hi = max(hi, v);
                }
                hi = max(hi, end);
                int lo = __shfl_up_sync(0xffffffffu, hi, 1);
                if (lane == 0) lo = end;
                const int nb = g >= a.groups ? 0 : (hi - lo + NT - 1) / NT;
                int inc = nb;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, inc, d);
                    if (lane >= d) inc += v;
                }
                if (g < a.groups) {
                    bad |= next[c] != hi;
                    t_lo[g] = lo;
                    t_cnt[g] = hi - lo;
                    t_pre[g] = before + inc - nb;
                }
                before += __shfl_sync(0xffffffffu, inc, 31);
                end = __shfl_sync(0xffffffffu, hi, 31);
            }
        }
        if (lane == 0) t_pre[a.groups] = before;
        if (bad && blockIdx.x == 0) atomicOr(a.err, kErrBadIndex);
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;
    const int n_items = t_pre[a.groups] * a.f_tiles;
    const int t_blocks = (a.t_size + kBlock - 1) / kBlock;

    auto item_at = [&](int i) -> Item {
        Item it;
        const int block = i / a.f_tiles;
        it.f0 = (i - block * a.f_tiles) * C::kTile;
        int lo = 0, hi = a.groups;                     // the last group whose first block is <= block
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (t_pre[mid] <= block) lo = mid; else hi = mid;
        }
        it.g = lo;
        const int b = block - t_pre[lo], cnt = t_cnt[lo], nb = t_pre[lo + 1] - t_pre[lo];
        // the group's rows in equal blocks, rounded up to the MMA's step
        const int size = ((cnt + nb - 1) / nb + C::kStep - 1) / C::kStep * C::kStep;
        it.row0 = t_lo[lo] + b * size;
        it.cols = min(size, cnt - b * size);
        it.kb = t_blocks;
        const int chunks = (it.kb + a.sum_blocks - 1) / a.sum_blocks;
        it.chunk = chunks > 1 ? (it.kb + chunks - 1) / chunks : it.kb;
        return it;
    };
    // Whether an item's parts are added up in tensor memory: they all use one accumulator set, the running sum is in the other,
    // and the next item begins with the set of the parts, so that its first wait frees both.
    auto sums_here = [&](const Item &it) { return LONG && it.chunk < it.kb; };
    // A role's walk through this unit's items: the warp finds 32 at once, a lane each.
    Item found = {};
    auto next_item = [&](int i, int turn) -> Item {
        if ((turn & 31) == 0) found = item_at(min(i + lane * units, n_items - 1));
        Item it;
        const int from = turn & 31;
        it.g = __shfl_sync(0xffffffffu, found.g, from);
        it.f0 = __shfl_sync(0xffffffffu, found.f0, from);
        it.row0 = __shfl_sync(0xffffffffu, found.row0, from);
        it.cols = __shfl_sync(0xffffffffu, found.cols, from);
        it.kb = __shfl_sync(0xffffffffu, found.kb, from);
        it.chunk = __shfl_sync(0xffffffffu, found.chunk, from);
        return it;
    };

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        for (int i = unit, turn = 0; i < n_items && ok; i += units, ++turn) {
            const Item it = next_item(i, turn);
            const int n_cta = (it.cols + C::kStep - 1) / C::kStep * 16;      // c of this item that each CTA stages
            const int f = it.f0 + (int)rank * 128, c = it.row0 + (int)rank * n_cta;
            const CUtensorMap *mb = &map_b.m[n_cta / 16 - 1];
            const uint32_t bytes = CG * (kATile + n_cta * kBlock);
            for (int kb = 0; kb < it.kb; ++kb) {
                if (!(ok = wait_all<false>(bar_empty + 8 * stage, phase ^ 1, abort_flag, a.err))) break;
                if (elect()) {
                    const uint32_t sa = smem_base + stage * C::kStageBytes, sb = sa + kATile;
                    const uint32_t bar = CG == 2 ? leader_addr(bar_full + 8 * stage) : bar_full + 8 * stage;
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * stage, bytes);
                    const int t = kb * kBlock;
                    if (WAY == kProduct) load_3d<CG>(sa, &map_a, t, f, it.g, bar);
                    else load_3d<CG>(sa, &map_a, f, t, it.g, bar);
                    load_2d<CG>(sb, mb, t, c, bar);
                }
                if (++stage == (uint32_t)a.stages) { stage = 0; phase ^= 1; }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (the leader CTA's)
        if (rank == 0) {
            uint32_t stage = 0, phase = 0, slot = 0, slot_phase = 0, acc = 0, acc_phases = 0;       // (a bit a set)
            const uint32_t base = (a.e5m2 ? 1u << 10 : 0u) | (WAY != kProduct ? 1u << 15 : 0u) | (1u << 23) | ((uint32_t)(C::kTile >> 7) << 27);
            bool ok = true;
            for (int i = unit, turn = 0; i < n_items && ok; i += units, ++turn) {
                const Item it = next_item(i, turn);
                const int n = (it.cols + C::kStep - 1) / C::kStep * C::kStep;
                const uint32_t idesc = base | ((uint32_t)(n >> 3) << 17);
                for (int kb = 0; kb < it.kb && ok;) {
                    if (!(ok = wait_all<CG == 2>(bar_tempty + 8 * acc, (acc_phases >> acc & 1) ^ 1, abort_flag, a.err))) break;
                    tc_fence_after();
                    const uint32_t d = tmem_base + acc * NT;
                    for (const int first = kb, end = min(it.kb, kb + it.chunk); kb < end; ++kb) {
                        const uint32_t t_sa = tmem_base + C::kScaleCol + slot * C::kSlotCols, t_sb = t_sa + 4;
                        if ((kb & 3) == 0) {           // the exponents of the next four k-blocks
                            if (!(ok = wait_all<CG == 2>(bar_sfull + 8 * slot, slot_phase, abort_flag, a.err))) break;
                            tc_fence_after();
                            const uint64_t from = desc_scales(smem_u32(scales) + slot * C::kSlotBytes);
                            if (elect())
#pragma unroll
                                for (int c = 0; c <= C::kBChunks; ++c)
                                    if (c < 2 || n > 128 * (c - 1)) copy_scales<CG>(t_sa + 4 * c, from + c * (512 >> 4));
                        }
                        if (!(ok = wait_all<CG == 2>(bar_full + 8 * stage, phase, abort_flag, a.err))) break;
                        tc_fence_after();
                        const bool last = (kb & 3) == 3 || kb == it.kb - 1;
                        if (elect()) {
                            const uint32_t sa = smem_base + stage * C::kStageBytes, sb = sa + kATile;
                            const uint64_t da = WAY == kProduct ? smem_desc_sw128(sa) : desc_mnmajor(sa), db = smem_desc_sw128(sb);
                            const uint32_t id = idesc | (uint32_t)(kb & 3) << 4 | (uint32_t)(kb & 3) << 29;      // which byte of the exponents
                            // 32 summed values a step: 32 bytes further along a K-major row, 32 rows of 128 bytes in an MN-major tile
                            constexpr int kStepA = WAY == kProduct ? 2 : 256, kStepB = 2;
#pragma unroll
                            for (int ki = 0; ki < kBlock / 32; ++ki) mma<CG>(d, da + kStepA * ki, db + kStepB * ki, id, t_sa, t_sb, (kb != first || ki) ? 1u : 0u);
                            commit<CG>(bar_empty + 8 * stage);
                            if (last) commit<CG>(bar_sempty + 8 * slot);
                        }
                        if (++stage == (uint32_t)a.stages) { stage = 0; phase ^= 1; }
                        if (last && ++slot == kSlots) { slot = 0; slot_phase ^= 1; }
                    }
                    if (!ok) break;
                    if (elect()) commit<CG>(bar_tfull + 8 * acc);
                    acc_phases ^= 1u << acc;
                    if (!sums_here(it)) acc ^= 1;
                }
            }
        }
    } else if (warp == C::kScaleWarp) {
        // ------------------------------------------------------------------ exponents (both CTAs)
        uint32_t slot = 0, phase = 0;
        bool ok = true;
        for (int i = unit, turn = 0; i < n_items && ok; i += units, ++turn) {
            const Item it = next_item(i, turn);
            const int fb = min((it.f0 + (int)rank * 128) / kBlock, (WAY == kProduct ? a.nb : a.kb) - 1);
            const uint8_t *w_scales = a.w_scales + (long long)it.g * a.nb * a.kb + (WAY == kProduct ? (long long)fb * a.kb : fb);
            const int w_step = WAY == kProduct ? 1 : a.kb;
            uint32_t word[4 * C::kBChunks], w_word;
            auto gather = [&](int kb) {                // of the k-blocks kb .. kb + 3
                const int left = min(4, it.kb - kb);
                uint32_t byte = lane < left ? (uint32_t)w_scales[(long long)(kb + lane) * w_step] << (8 * lane) : 0;
                byte |= __shfl_xor_sync(0xffffffffu, byte, 1);
                byte |= __shfl_xor_sync(0xffffffffu, byte, 2);
                w_word = __shfl_sync(0xffffffffu, byte, 0);
#pragma unroll
                for (int j = 0; j < 4 * C::kBChunks; ++j) {
                    const uint8_t *p = a.row_scales + (long long)(it.row0 + min(lane + 32 * j, it.cols - 1)) * a.lds + kb;
                    word[j] = 0;
                    if (32 * j < it.cols) {
                        if (a.words) {                 // (what a row's last word holds behind its end is not used)
                            word[j] = *reinterpret_cast<const uint32_t *>(p);
                        } else {
#pragma unroll
                            for (int b = 0; b < 4; ++b) word[j] |= (uint32_t)p[min(b, left - 1)] << (8 * b);
                        }
                    }
                }
            };
            gather(0);
            for (int kb = 0; kb < it.kb; kb += 4) {
                if (!(ok = wait_all<false>(bar_sempty + 8 * slot, phase ^ 1, abort_flag, a.err))) break;
                uint4 *to = reinterpret_cast<uint4 *>(scales + slot * C::kSlotBytes) + lane;
                to[0] = make_uint4(w_word, w_word, w_word, w_word);
#pragma unroll
                for (int c = 0; c < C::kBChunks; ++c) to[32 * (c + 1)] = make_uint4(word[4 * c], word[4 * c + 1], word[4 * c + 2], word[4 * c + 3]);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) arrive_leader<CG>(bar_sfull + 8 * slot);
                if (++slot == kSlots) { slot = 0; phase ^= 1; }
                if (kb + 4 < it.kb) gather(kb + 4);
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue (both CTAs)
        const int lg = warp & 3, half = (warp - 2) >> 2;     // the TMEM lanes this warp may read; its columns
        int tiles = 0;                                 // stored so far
        uint32_t acc = 0, acc_phases = 0;
        bool ok = true;
        for (int i = unit, turn = 0; i < n_items && ok; i += units, ++turn) {
            const Item it = next_item(i, turn);
            const int f = it.f0 + (int)rank * 128 + lg * 32 + lane;
            const bool f_ok = f < a.f_size;
            const size_t at = (size_t)it.row0 * a.ldo + f;
            for (int kb = 0; kb < it.kb; kb += it.chunk) {
                // (the two warps of a pair meet at barriers below, so they go on or give up together)
                if (!(ok = both_of_pair(wait_all<false>(bar_tfull + 8 * acc, acc_phases >> acc & 1, abort_flag, a.err)))) break;
                tc_fence_after();
                const uint32_t lanes = tmem_base + ((uint32_t)(lg * 32) << 16), t0 = lanes + acc * NT;
                const bool here = sums_here(it);
                int to_store = it.cols;
                if (here) {
                    // the running sum and this part, to where the sum stays, the last time to where the results are stored from
                    const bool last = kb + it.chunk >= it.kb;
                    const uint32_t t_sum = lanes + (acc ^ 1) * NT;
#pragma unroll 1
                    for (int c0 = 32 * half; c0 < it.cols; c0 += 8 * EW) {
                        uint32_t v[32], sum[32];
                        tc_ld32(t0 + c0, v);
                        tc_ld32(t_sum + c0, sum);
                        tc_wait_ld();
                        if (kb > 0)
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(sum[j]) + __uint_as_float(v[j]));
                        tc_st32((last ? t0 : t_sum) + c0, v);
                    }
                    tc_wait_st();
                    if (!last) to_store = 0;
                }
                if (a.wide) {
                    const int f_left = a.f_size - (f - lane), f_pair = f - lane - 32 * (lg & 1);
                    uint16_t *out = reinterpret_cast<uint16_t *>(a.out) + at - lane;
                    if (f_pair < a.f_size)
#pragma unroll 1
                        for (int c0 = 32 * half; c0 < to_store; c0 += 8 * EW) {
                            uint8_t *tile = staging + (pair_index() * kTiles + tiles++ % kTiles) * 4096;
                            if (a.out_kind == EW_BF16)
                                store_tile<true>(t0 + c0, tile, &map_out, f_pair, it.row0 + c0, out + (size_t)c0 * a.ldo, a.ldo, it.cols - c0, lane, lg & 1, f_left);
                            else
                                store_tile<false>(t0 + c0, tile, &map_out, f_pair, it.row0 + c0, out + (size_t)c0 * a.ldo, a.ldo, it.cols - c0, lane, lg & 1, f_left);
                        }
                } else {
#pragma unroll 1
                    for (int c0 = 32 * half; c0 < to_store; c0 += 8 * EW) {
                        uint32_t v[32];
                        tc_ld32(t0 + c0, v);           // columns behind the item's last are in the accumulator set, not stored
                        tc_wait_ld();
                        const int lim = min(32, it.cols - c0);
                        const size_t to = at + (size_t)c0 * a.ldo;
                        if (f_ok) {
                            if (a.out_kind == EW_FP32) {
                                if (kb > 0) add_columns(reinterpret_cast<float *>(a.out) + to, a.ldo, v, lim);
                                else store_columns(reinterpret_cast<float *>(a.out) + to, a.ldo, v, lim);
                            } else if (a.out_kind == EW_BF16) {
                                store_columns(reinterpret_cast<__nv_bfloat16 *>(a.out) + to, a.ldo, v, lim);
                            } else {
                                store_columns(reinterpret_cast<__half *>(a.out) + to, a.ldo, v, lim);
                            }
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_leader<CG>(bar_tempty + 8 * acc);
                acc_phases ^= 1u << acc;
                if (!here) acc ^= 1;
            }
        }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");            // the copies out of shared memory have arrived
    }

    // ---------------------------------------------------------------------- teardown
    if (*abort_flag) {                                 // let copies in flight land before the CTA's memory is reused
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000ll) {}
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync_all();
    tc_fence_after();
    if (warp == 1) {
        if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

constexpr int kBarBytes = (2 * kMaxStages + 2 * kSlots + 4 + 1) * 8;

template <int CG, int NT, int EW, int WAY>
ew_status_t launch(const Device &d, const CUtensorMap &ma, const RowMaps &mb, const CUtensorMap &mo, Args a, cudaStream_t st) {
    using C = Cfg<CG, NT, EW>;
    a.f_tiles = (a.f_size + C::kTile - 1) / C::kTile;
    const long long live = a.groups < a.rows ? a.groups : a.rows;            // groups that can have rows
    const long long max_items = (live + a.rows / NT) * a.f_tiles;
    if (max_items > 0x7fff0000) return refuse("scaled product: too many output tiles");
    const int rest = 1024 + kSlots * C::kSlotBytes + C::kStaging + kBarBytes + (3 * a.groups + 1) * 4, fit = (kSmemLimit - rest) / C::kStageBytes;
    a.stages = fit < kMaxStages ? fit : kMaxStages;
    cudaLaunchConfig_t cfg = {};
    const long long units = d.sm_count / CG;
    cfg.gridDim = dim3((unsigned)(CG * (max_items < units ? max_items : units)));
    cfg.blockDim = dim3(C::kThreads);
    cfg.dynamicSmemBytes = (size_t)a.stages * C::kStageBytes + rest;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    int attrs = 0;
    if (CG > 1) {
        attr[attrs].id = cudaLaunchAttributeClusterDimension;
        attr[attrs].val.clusterDim.x = CG;
        attr[attrs].val.clusterDim.y = attr[attrs].val.clusterDim.z = 1;
        ++attrs;
    }
    if (pdl_enabled()) {
        attr[attrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[attrs].val.programmaticStreamSerializationAllowed = 1;
        ++attrs;
    }
    cfg.attrs = attr;
    cfg.numAttrs = attrs;
    a.sum_blocks = sum_blocks(a.out_kind);
    const bool long_sums = a.out_kind != EW_FP32 && a.t_size > a.sum_blocks * kBlock;
    return launched((int)(EW == 4 && long_sums ? cudaLaunchKernelEx(&cfg, scaled_product_kernel<CG, NT, EW, WAY, EW == 4>, ma, mb, mo, a)
                                    : cudaLaunchKernelEx(&cfg, scaled_product_kernel<CG, NT, EW, WAY, false>, ma, mb, mo, a)), "scaled product");
}

template <int CG, int NT, int EW, int WAY>
int setup_one() {
    return (int)cudaFuncSetAttribute(scaled_product_kernel<CG, NT, EW, WAY, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) |
           (int)cudaFuncSetAttribute(scaled_product_kernel<CG, NT, EW, WAY, EW == 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
}

// A row-major matrix of bytes whose rows keep every TMA copy on a 16-byte boundary
bool bad_matrix(const void *p, long long ld, long long width) {
    return !p || ((uintptr_t)p & 15) || ld < width || (ld & 15) || ld >= (1ll << 39);
}

// The form that a product takes: ew_scaled_mm_form's numbers.
// One CTA with 128 columns against the pair: 64 groups of 2816 x 2048 with 96 rows each 69.4 and 69.8 us, 128 rows 73.0 and 72.7, 144 rows 95.7
// and 75.7; where the pairs' tiles would not fill the GPU (8 groups of 1024 x 512, 160 rows each) 6.7 and 7.5.  (The host
// knows only how many groups there are, not which have rows: over many empty ones the one-CTA form may be taken where the pair would
// be faster.)
// Short sums: the results' way out is what counts, and eight warps walk it (20000 rows, 16 groups, n = 1408; k = 256: 19.6 us
// against 23.8, 512: 22.4 and 25.8, 1024: 31.5 and 32.3); long ones: at the power limit four cost less (2048, 49152 rows: 285 and 289).
enum Form { kOneCta = 0, kPairEight = 1, kPairFour = 2 };
Form form_of(long long rows, long long groups, long long f, long long t, int sm_count) {
    const long long live = groups < rows ? groups : rows, pair_tiles = (live + rows / 224) * ((f + 255) / 256);
    if (rows <= 128 * groups || pair_tiles <= sm_count / 2) return kOneCta;
    return t <= 1024 ? kPairEight : kPairFour;
}

ew_status_t product(bool grad, int32_t device, int32_t row_type, int32_t out_dtype, const void *x, int64_t ldx, const void *x_scales, int64_t lds, const void *w,
                    int64_t ldw, int64_t group_stride, const void *w_scales, const int32_t *offsets, int32_t rows, int32_t groups, int32_t n, int32_t k, void *out,
                    int64_t ldo, void *stream) {
    const int t = grad ? n : k, f = grad ? k : n;
    constexpr int32_t kMostSize = 0x7fff0000;                                // (indexes run a tile past the end)
    if (!is_8bit(row_type) || (!is_16bit(out_dtype) && out_dtype != EW_FP32)) return refuse("scaled product: rows are e4m3 or e5m2, results bf16, fp16 or fp32");
    if (rows < 0 || rows > kMostSize || groups < 1 || groups > kMostSlots || n < 1 || n > kMostSize || k < 1 || k > kMostSize)
        return refuse("scaled product: size out of range");
    if ((!offsets && groups != 1) || ((uintptr_t)offsets & 3) || !w_scales || (rows > 0 && (!out || ((uintptr_t)out & (elem_bytes(out_dtype) - 1)))))
        return refuse("scaled product: null or misaligned pointer (without offsets there is one group)");
    if ((rows > 0 && bad_matrix(x, ldx, t)) || bad_matrix(w, ldw, k) || ldo < f || !rows_apart(groups, group_stride, n, ldw, k) ||
        (groups > 1 && ((group_stride & 15) || group_stride >= (1ll << 39))))
        return refuse("scaled product: operands need 16-byte aligned rows that do not overlap");
    if (rows > 0 && (!x_scales || lds < (t + (int64_t)kBlock - 1) / kBlock)) return refuse("scaled product: the rows' scales are missing or overlap");
    if (device < 0) return EW_ERR_NO_DEVICE;
    if (rows == 0) return EW_OK;
    DeviceGuard guard;
    ew_status_t s = launched((int)guard.enter(device), "cudaSetDevice");
    const Device *d;
    if (s != EW_OK || (s = device_state(device, &d)) != EW_OK) return s;
    CUtensorMap ma, mo;
    RowMaps mb;
    const uint64_t wd[3] = {(uint64_t)k, (uint64_t)n, (uint64_t)groups}, ws[2] = {(uint64_t)ldw, groups > 1 ? (uint64_t)group_stride : (uint64_t)ldw};
    const uint32_t w_box[3] = {kBlock, 128, 1};
    if ((s = encode_map(*d, &ma, CU_TENSOR_MAP_DATA_TYPE_UINT8, w, 3, wd, ws, w_box, CU_TENSOR_MAP_SWIZZLE_128B)) != EW_OK) return s;
    const uint64_t xd[2] = {(uint64_t)t, (uint64_t)rows}, xs[1] = {(uint64_t)ldx};
    for (int i = 0; i < kMaps && 16 * i < rows; ++i) {                       // (an item has no more rows than there are)
        const uint32_t box[2] = {kBlock, 16u * (i + 1)};
        if ((s = encode_map(*d, &mb.m[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, x, 2, xd, xs, box, CU_TENSOR_MAP_SWIZZLE_128B)) != EW_OK) return s;
    }
    Args a = {};
    a.offsets = offsets;
    a.row_scales = (const uint8_t *)x_scales;
    a.w_scales = (const uint8_t *)w_scales;
    a.out = out;
    a.err = d->err;
    a.ldo = ldo;
    a.lds = lds;
    a.rows = rows;
    a.groups = groups;
    a.f_size = f;
    a.t_size = t;
    a.nb = (int)((n + (int64_t)kBlock - 1) / kBlock);
    a.kb = (int)((k + (int64_t)kBlock - 1) / kBlock);
    a.out_kind = out_dtype;
    a.e5m2 = row_type == EW_E5M2;
    a.words = !(((uintptr_t)x_scales | lds) & 3);
    a.wide = out_dtype != EW_FP32 && !(((uintptr_t)out & 15) | ((ldo | f) & 7)) && ldo < (1ll << 38);
    if (a.wide) {
        const uint64_t od[2] = {(uint64_t)f, (uint64_t)rows}, os[1] = {(uint64_t)ldo * 2};
        const uint32_t box[2] = {64, 32};
        if ((s = encode_map(*d, &mo, map_type(out_dtype), out, 2, od, os, box, CU_TENSOR_MAP_SWIZZLE_128B)) != EW_OK) return s;
    }
    cudaStream_t st = (cudaStream_t)stream;
#define EW_LAUNCH(CG, NT, EW) (grad ? launch<CG, NT, EW, kInputGrad>(*d, ma, mb, mo, a, st) : launch<CG, NT, EW, kProduct>(*d, ma, mb, mo, a, st))
    switch (form_of(rows, groups, f, t, d->sm_count)) {
        case kOneCta: return EW_LAUNCH(1, 128, 4);
        case kPairEight: return EW_LAUNCH(2, 224, 8);
        default: return EW_LAUNCH(2, 224, 4);
    }
#undef EW_LAUNCH
}

}  // namespace

int scaled_setup() {
    return setup_one<1, 128, 4, kProduct>() | setup_one<1, 128, 4, kInputGrad>() | setup_one<2, 224, 4, kProduct>() | setup_one<2, 224, 4, kInputGrad>() |
           setup_one<2, 224, 8, kProduct>() | setup_one<2, 224, 8, kInputGrad>();
}

}  // namespace ops
}  // namespace ew

extern "C" ew_status_t ew_scaled_mm(int32_t device, int32_t row_type, int32_t out_dtype, const void *x, int64_t ldx, const void *x_scales, int64_t ldxs, const void *w,
                                    int64_t ldw, int64_t group_stride, const void *w_scales, const int32_t *offsets, int32_t rows, int32_t groups, int32_t n,
                                    int32_t k, void *y, int64_t ldy, void *cuda_stream) {
    return ew::ops::product(false, device, row_type, out_dtype, x, ldx, x_scales, ldxs, w, ldw, group_stride, w_scales, offsets, rows, groups, n, k, y, ldy, cuda_stream);
}

extern "C" ew_status_t ew_scaled_mm_dx(int32_t device, int32_t row_type, int32_t out_dtype, const void *dy, int64_t lddy, const void *dy_scales, int64_t lddys,
                                       const void *w, int64_t ldw, int64_t group_stride, const void *w_scales, const int32_t *offsets, int32_t rows, int32_t groups,
                                       int32_t n, int32_t k, void *dx, int64_t lddx, void *cuda_stream) {
    return ew::ops::product(true, device, row_type, out_dtype, dy, lddy, dy_scales, lddys, w, ldw, group_stride, w_scales, offsets, rows, groups, n, k, dx, lddx, cuda_stream);
}

extern "C" int32_t ew_scaled_mm_form(int32_t input_gradient, int32_t rows, int32_t groups, int32_t n, int32_t k, int32_t sm_count) {
    return ew::ops::form_of(rows, groups, input_gradient ? k : n, input_gradient ? n : k, sm_count);
}
