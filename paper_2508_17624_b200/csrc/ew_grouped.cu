// Matrix products grouped by expert, with ragged groups of rows, and their two gradients (tcgen05 + TMEM + TMA).
//
//   product         y [r, n] = sum_k x[r, k] w[g, n, k]         for the rows r of group g: offsets[g] <= r < offsets[g+1]
//   input gradient  dx[r, k] = sum_n dy[r, n] w[g, n, k]
//   weight gradient dw[g, n, k] (+)= sum_{r in g} dy[r, n] x[r, k]
//
// One kernel for the three.  In all of them the output is row-major with a contiguous axis f (n, k, k), and
//   D[f, c] = sum_t A[f, t] B[c, t],   out[row(c), f] = D[f, c]:
//
//               f   c            t (summed)   A                              B
//   product     n   rows of x    k            w[g]  (t contiguous)           x  (t contiguous)
//   dx          k   rows of dy   n            w[g]  (f contiguous)           dy (t contiguous)
//   dw          k   n            rows of g    x     (f contiguous)           dy (c contiguous)
//
// f is the MMA's M axis (TMEM lanes), so a warp of the epilogue holds 32 neighbouring f of one output row and its store
// instructions write whole sectors, whatever the group's length; c is the MMA's N axis, which an instruction can choose
// in steps of 16: a group of few rows costs few tensor-core cycles and the kernel is then a stream of its weights.  The
// operand whose summed axis is contiguous is staged K-major, the other MN-major: the tensor core transposes, nothing is
// moved for it.
//
// Two tile widths, by the rows a group has on average: up to 128 rows, 128 columns on one CTA (64 columns and nine stages were
// up to 8 % slower from 16 rows a group on, 32 columns and twelve stages 3 % slower for one); beyond, a CTA pair with 256 f x
// 256 columns, every operand byte crossing from L2 once per 256 x 256 tile.
//
// Measured (one B200; copy bandwidth 6551 GB/s, cuBLAS bf16 1655 TFLOP/s in a burst, 1403 sustained):
//   y,  1536 rows, 96 groups, 2816 x 2048   174 to 181 us = 6.2 to 6.4 TB/s, 95 to 98 % of the copy bandwidth (bound by the weights' bytes)
//   y, 49152 rows, 64 groups, 2816 x 2048   490 to 551 us sustained = 1030 to 1160 TFLOP/s (1337 in a burst), bound by the tensor cores at
//                                           the power limit; the MMA thread waits for data 17 % of the time
//   dx, 24582 rows, 64 groups, 2048 x 1408  143 to 174 us: 384 rows a group leave 192-column tiles, and a tile costs 218 ns a
//                                           k-block plus 0.7 ns a column whatever its width
//   dw, 12289 rows, 32 groups, fp32         183 to 222 us = 3.9 to 4.7 TB/s: 738 MB of results, 128 bytes every five cycles of
//                                           an SM while the epilogue stores, which it does 70 % of the time

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ew_ops.h"
#include "ew_tc.cuh"

namespace ew {
namespace ops {
namespace {
using namespace tc;

enum Way { kProduct = 0, kInputGrad = 1, kWeightGrad = 2, kWeightAdd = 3 };      // the last: added to what is there

constexpr int threads_of(int epilogue_warps) { return (3 + epilogue_warps) * 32; }       // TMA, MMA, epilogue, relay (weight gradient)
constexpr int kATile = 128 * kBlockK * 2;              // 16 KiB: 128 f of one stage
constexpr int kMaxGroups = 2048;                       // bounds the group table in shared memory
constexpr int kSmemLimit = 227 * 1024;
constexpr int kMaxStages = 7;                          // of 32 KiB
// The tensor core cuts off, rather than rounds, what a product has below the running sum's last bit.  Over terms of one sign
// that takes 6.4e-9 of the result a term (5.8e-6 at 1024, 4.1e-4 at 65536: measured), over random ones a tenth of it.  Long
// sums are therefore made in parts of so many k-blocks, which the epilogue adds up in fp32: fp32 results 1024 terms at a time
// (in the output, always the same thread's part of it), 16-bit ones when the loss would pass an eighth of half their step: 8192
// terms for fp16, 65536 for bf16.  Their running sum stays in the accumulator set that the parts do not use, which costs such
// an item the overlap of its parts (weight gradient of one group of 40000 rows, 2048 x 1408, fp16: 236 -> 243 us).  No wait is for more than a part, however many rows a group has.
constexpr int sum_blocks(int out_dtype) { return out_dtype == EW_FP32 ? 16 : out_dtype == EW_FP16 ? 128 : 1024; }

struct Args {
    const int32_t *offsets;
    void *out;
    int *err;
    long long ldo;          // elements between output rows
    long long group_out;    // dw: elements between groups
    int rows, groups;
    int f_size;             // length of the output's contiguous axis
    int c_size;             // dw: n
    int t_size;             // product, dx: length of the summed axis
    int f_tiles, c_tiles;
    int out_kind;           // ew_dtype_t
    int sum_blocks;         // most k-blocks that are summed up in the tensor core
    int a_pairs, b_pairs;   // operands with a contiguous f (c): 1 = two 64-wide boxes come in one copy
    int fp16;               // operand type
    int stages;
    int table_bytes;
};

// CG: CTAs that share one MMA tile (1, or 2 = a pair with 256 f); NT: columns of an accumulator set; EW: epilogue warps, four or
// eight (two to each quarter of the TMEM lanes, taking turns at the columns)
template <int CG, int NT>
struct Cfg {
    static constexpr int kBRows = NT / CG;                                   // c staged by each CTA
    static constexpr int kStageBytes = kATile + kBRows * kBlockK * 2;
    static constexpr int kTile = 128 * CG;                                   // f of an item
    static constexpr int kTmemCols = 2 * NT;                                 // two accumulator sets
    static constexpr int kStep = 16 * CG;                                    // granularity of an MMA's N
    static_assert((kSmemLimit - 1024) / kStageBytes <= kMaxStages, "barriers for every stage that fits");
};

// The row operand's tensor maps: boxes of 32, 64, 96 and 128 rows (weight gradient: one map).  A stage's rows come in one
// copy of about their number: several small copies a stage cost up to a fifth of the time of a large product, and a 128-row
// box for 96 rows a third more bytes.
struct RowMaps { CUtensorMap m[4]; };

struct Item {
    int g, f0, row0, cols, kb, tail;      // cols: output rows (c) of this item; kb: k-blocks; tail: live rows of the last one (dw)
    int chunk;                            // k-blocks summed up in the tensor core at a time
};

__device__ __forceinline__ uint64_t desc_kmajor(uint32_t addr) { return smem_desc_sw128(addr); }
// MN-major operand, 128-byte swizzle: blocks of 64 MN-elements x 64 summed rows of 128 bytes (one TMA box, 8 KiB); the
// next 64 MN-elements lie 8 KiB further on (leading offset), the next eight summed rows 1 KiB (stride offset).
__device__ __forceinline__ uint64_t desc_mnmajor(uint32_t addr) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3FFFF) >> 4);
    d |= (uint64_t)(8192 >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
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
__device__ __forceinline__ void load_4d(uint32_t dst, const CUtensorMap *m, int x, int y, int z, int w, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                     ::"r"(dst), "l"(m), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                     ::"r"(dst), "l"(m), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    if constexpr (CG == 1) tc_mma(d, a, b, idesc, acc);
    else tc2_mma(d, a, b, idesc, acc);
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
    // eight addresses that do not wait for one another
    T *q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = p + j * ldo;
    const long long step = 8 * ldo;
    if (lim == 32) {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            *q[j & 7] = (T)__uint_as_float(v[j]);
            q[j & 7] += step;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if (j < lim) *q[j & 7] = (T)__uint_as_float(v[j]);
            q[j & 7] += step;
        }
    }
}
// The same added to what is there, eight rows at a time (their old values are asked for together).
template <class T>
__device__ __forceinline__ void add_columns(T *p, long long ldo, const uint32_t (&v)[32], int lim) {
#pragma unroll
    for (int j0 = 0; j0 < 32; j0 += 8) {
        float old[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j0 + j < lim) old[j] = (float)p[j * ldo];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j0 + j < lim) p[j * ldo] = (T)(old[j] + __uint_as_float(v[j0 + j]));
        p += 8 * ldo;
    }
}
template <class T, bool ADD>
__device__ __forceinline__ void put_columns(void *out, size_t at, long long ldo, const uint32_t (&v)[32], int lim) {
    if (ADD) add_columns(reinterpret_cast<T *>(out) + at, ldo, v, lim);
    else store_columns(reinterpret_cast<T *>(out) + at, ldo, v, lim);
}
__device__ __forceinline__ void store_zero(void *out, size_t at, int kind) {
    if (kind == EW_FP32) reinterpret_cast<float *>(out)[at] = 0.f;
    else reinterpret_cast<uint16_t *>(out)[at] = 0;
}

// LONG: 16-bit results whose sums may have several parts (without that code the others' weight gradients are 1 to 3 % faster)
template <int CG, int NT, int EW, int WAY, bool LONG>
__global__ void __launch_bounds__(threads_of(EW), 1)
grouped_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ RowMaps map_b, const __grid_constant__ Args a) {
    using C = Cfg<CG, NT>;
    constexpr int kRelayWarp = 2 + EW;
    constexpr bool DW = WAY == kWeightGrad || WAY == kWeightAdd;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem_al = smem_raw + (smem_base - smem_u32(smem_raw));
    // after the ring: barriers full, ready, empty [kMaxStages] each, tmem full [2], tmem empty [2], TMEM base, abort
    // flag; then the group table: first block of each group, first row, rows
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem_al + a.stages * C::kStageBytes);
    const uint32_t bar_full = smem_u32(bars), bar_ready = bar_full + 8 * kMaxStages, bar_empty = bar_ready + 8 * kMaxStages;
    const uint32_t bar_tfull = bar_empty + 8 * kMaxStages, bar_tempty = bar_tfull + 16;
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(bars + 3 * kMaxStages + 4);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    int *t_pre = reinterpret_cast<int *>(bars + 3 * kMaxStages + 6), *t_lo = t_pre + a.groups + 1, *t_cnt = t_lo + a.groups;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_ctarank() : 0;
    const int unit = blockIdx.x / CG, units = gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_ready + 8 * s, CG);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_tfull + 8 * i, 1);
            mbar_init(bar_tempty + 8 * i, EW * CG);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&map_a);
        prefetch_map(&map_b.m[DW ? 0 : C::kBRows / 32 - 1]);
    }
    if (warp == 1) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                         "r"((uint32_t)C::kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                         "r"((uint32_t)C::kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    pdl_launch_dependents();
    pdl_wait();                                        // the operands and the offsets may come from the kernel before
    if (warp == 0) {
        // group table: first row and rows of each group, and the number of row blocks before it.  Offsets are clamped to
        // the matrix and to the largest one before them, so that whatever the call was given the groups lie inside the
        // matrix and apart from one another.
        int before = 0, raw = *(const volatile int32_t *)a.offsets, end = min(max(raw, 0), a.rows);
        bool bad = raw != end;
        for (int g0 = 0; g0 < a.groups; g0 += 32) {
            const int g = g0 + lane;
            int hi = end;
            if (g < a.groups) {
                raw = *(const volatile int32_t *)(a.offsets + g + 1);
                hi = min(max(raw, 0), a.rows);
            }
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, hi, d);
                if (lane >= d) hi = max(hi, v);
            }
            hi = max(hi, end);
            int lo = __shfl_up_sync(0xffffffffu, hi, 1);
            if (lane == 0) lo = end;
            const int nb = g >= a.groups ? 0 : DW ? a.c_tiles : (hi - lo + NT - 1) / NT;
            int inc = nb;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, inc, d);
                if (lane >= d) inc += v;
            }
            if (g < a.groups) {
                bad |= raw != hi;
                t_lo[g] = lo;
                t_cnt[g] = hi - lo;
                t_pre[g] = before + inc - nb;
            }
            before += __shfl_sync(0xffffffffu, inc, 31);
            end = __shfl_sync(0xffffffffu, hi, 31);
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
    const int t_blocks = (a.t_size + kBlockK - 1) / kBlockK;

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
        const int b = block - t_pre[lo], cnt = t_cnt[lo];
        if (DW) {
            it.row0 = b * NT;                          // first n of the tile
            it.cols = min(NT, a.c_size - it.row0);
            it.kb = (cnt + kBlockK - 1) / kBlockK;
            it.tail = cnt - (it.kb - 1) * kBlockK;
        } else {
            // the group's rows in equal blocks, rounded up to the MMA's step: 257 rows make 160 + 97 (pair) or 96 + 96 + 65, not
            // 256 + 1 (2049 rows, whose nine equal blocks round up to 256 each, still make eight of 256 and one of 1)
            const int nb = t_pre[lo + 1] - t_pre[lo];
            const int size = ((cnt + nb - 1) / nb + C::kStep - 1) / C::kStep * C::kStep;
            it.row0 = t_lo[lo] + b * size;
            it.cols = min(size, cnt - b * size);
            it.kb = t_blocks;
            it.tail = kBlockK;
        }
        const int chunks = (it.kb + a.sum_blocks - 1) / a.sum_blocks;
        it.chunk = chunks > 1 ? (it.kb + chunks - 1) / chunks : it.kb;
        return it;
    };
    // Whether an item's parts are added up in tensor memory: they all use one accumulator set, the running sum is in the other,
    // and the next item begins with the set of the parts, so that its first wait frees both.
    auto sums_here = [&](const Item &it) { return LONG && it.chunk < it.kb; };
    // A role's walk through this unit's items.  Finding an item takes a few hundred cycles of divisions and look-ups, which for a
    // weight gradient of few rows was most of the copying thread's time: the warp finds 32 items at once, a lane each.
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
        it.tail = __shfl_sync(0xffffffffu, found.tail, from);
        it.chunk = __shfl_sync(0xffffffffu, found.chunk, from);
        return it;
    };

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        for (int i = unit, turn = 0; i < n_items && ok; i += units, ++turn) {
            const Item it = next_item(i, turn);
            if (lane == 0) {
                const int n = (it.cols + C::kStep - 1) / C::kStep * C::kStep;
                const int n_cta = n / CG;                                    // c of this item that each CTA stages
                const int f = it.f0 + (int)rank * 128;
                const int c = it.row0 + (DW ? (int)rank * (NT / CG) : (int)rank * n_cta);
                const int boxes = DW ? 0 : (n_cta + 31) / 32;                // of 32 rows
                const CUtensorMap *mb = &map_b.m[DW ? 0 : boxes - 1];
                const uint32_t b_bytes = DW ? (uint32_t)(NT / CG) * kBlockK * 2 : boxes * kChunkBytes;
                const int first = DW ? t_lo[it.g] : 0;
                for (int kb = 0; kb < it.kb; ++kb) {
                    if (!(ok = wait_on<false>(bar_empty + 8 * stage, phase ^ 1, abort_flag, a.err))) break;
                    const uint32_t sa = smem_base + stage * C::kStageBytes, sb = sa + kATile;
                    // the weight gradient's copies are counted on each CTA's own barrier (its relay warp reads them), the
                    // others' on the leader's
                    const uint32_t bar = (CG == 2 && !DW) ? leader_addr(bar_full + 8 * stage) : bar_full + 8 * stage;
                    if (DW || rank == 0) mbar_expect_tx(bar_full + 8 * stage, DW ? kATile + b_bytes : CG * (kATile + b_bytes));
                    const int t = first + kb * kBlockK;
                    if (WAY == kProduct) {
                        load_3d<CG>(sa, &map_a, t, f, it.g, bar);
                    } else if (WAY == kInputGrad) {
                        if (a.a_pairs) {
                            load_4d<CG>(sa, &map_a, 0, t, f >> 6, it.g, bar);
                        } else {
                            load_3d<CG>(sa, &map_a, f, t, it.g, bar);
                            load_3d<CG>(sa + 8192, &map_a, f + 64, t, it.g, bar);
                        }
                    } else if (a.a_pairs) {
                        tma_load_3d(sa, &map_a, 0, t, f >> 6, bar);
                    } else {
                        tma_load_2d(sa, &map_a, f, t, bar);
                        tma_load_2d(sa + 8192, &map_a, f + 64, t, bar);
                    }
                    if (!DW) {
                        load_2d<CG>(sb, mb, t, c, bar);
                    } else if (a.b_pairs) {
                        tma_load_3d(sb, mb, 0, t, c >> 6, bar);
                    } else {
                        tma_load_2d(sb, mb, c, t, bar);
                        tma_load_2d(sb + 8192, mb, c + 64, t, bar);
                    }
                    if (++stage == (uint32_t)a.stages) { stage = 0; phase ^= 1; }
                }
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (the leader CTA's)
        if (rank == 0) {
            uint32_t stage = 0, phase = 0, acc = 0, acc_phases = 0;          // (a bit a set)
            const uint32_t type = a.fp16 ? 0u : (1u << 7) | (1u << 10);
            const uint32_t base = (1u << 4) | type | (WAY != kProduct ? 1u << 15 : 0u) | (DW ? 1u << 16 : 0u) |
                                  ((uint32_t)(C::kTile >> 4) << 24);
            const uint32_t bar_in = DW ? bar_ready : bar_full;
            bool ok = true;
            for (int i = unit, turn = 0; i < n_items && ok; i += units, ++turn) {
                const Item it = next_item(i, turn);
                if (DW && it.kb == 0) continue;                              // an empty group: the epilogue writes its zeros
                const int n = DW ? NT : (it.cols + C::kStep - 1) / C::kStep * C::kStep;
                const uint32_t idesc = base | ((uint32_t)(n >> 3) << 17);
                for (int kb = 0; lane == 0 && kb < it.kb && ok;) {
                    if (!(ok = wait_on<CG == 2>(bar_tempty + 8 * acc, (acc_phases >> acc & 1) ^ 1, abort_flag, a.err))) break;
                    tc_fence_after();
                    const uint32_t d = tmem_base + acc * NT;
                    for (const int first = kb, end = min(it.kb, kb + it.chunk); kb < end; ++kb) {
                        if (!(ok = wait_on<CG == 2>(bar_in + 8 * stage, phase, abort_flag, a.err))) break;
                        tc_fence_after();
                        const uint32_t sa = smem_base + stage * C::kStageBytes, sb = sa + kATile;
                        const uint64_t da = WAY == kProduct ? desc_kmajor(sa) : desc_mnmajor(sa);
                        const uint64_t db = DW ? desc_mnmajor(sb) : desc_kmajor(sb);
                        // 16 summed elements a step: 32 bytes further along a K-major row, two groups of eight 128-byte
                        // rows (2 KiB) further in an MN-major tile; descriptors count 16 bytes
                        constexpr int kStepA = WAY == kProduct ? 2 : 128, kStepB = DW ? 128 : 2;
                        const int steps = DW && kb == it.kb - 1 ? (it.tail + 15) >> 4 : kBlockK / 16;
#pragma unroll
                        for (int ki = 0; ki < kBlockK / 16; ++ki)
                            if (!DW || ki < steps) mma<CG>(d, da + kStepA * ki, db + kStepB * ki, idesc, (kb != first || ki) ? 1u : 0u);
                        commit<CG>(bar_empty + 8 * stage);
                        if (++stage == (uint32_t)a.stages) { stage = 0; phase ^= 1; }
                    }
                    if (!ok) break;
                    commit<CG>(bar_tfull + 8 * acc);
                    acc_phases ^= 1u << acc;
                    if (!sums_here(it)) acc ^= 1;
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
            }
        }
    } else if (warp == kRelayWarp) {
        // ------------------------------------------------------------------ relay (weight gradient, both CTAs)
        // The last k-block of a group ends inside a tile, and the rows behind it are the next group's: up to the end of
        // the MMA step both operands are set to zero (both: a NaN there would survive a zero on the other side).
        if (DW) {
            uint32_t stage = 0, phase = 0;
            bool ok = true;
            for (int i = unit, turn = 0; i < n_items && ok; i += units, ++turn) {
                const Item it = next_item(i, turn);
                for (int kb = 0; kb < it.kb; ++kb) {
                    if (!(ok = wait_warp(bar_full + 8 * stage, phase, abort_flag, a.err))) break;
                    if (kb == it.kb - 1 && (it.tail & 15)) {
                        const int from = it.tail * 128, to = ((it.tail + 15) & ~15) * 128;
                        uint8_t *tile = smem_al + stage * C::kStageBytes;
                        for (int box = 0; box < C::kStageBytes / 8192; ++box)
                            for (int o = from + lane * 16; o < to; o += 512)
                                *reinterpret_cast<uint4 *>(tile + box * 8192 + o) = make_uint4(0, 0, 0, 0);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    if (lane == 0) arrive_leader<CG>(bar_ready + 8 * stage);
                    if (++stage == (uint32_t)a.stages) { stage = 0; phase ^= 1; }
                }
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue (EW warps of each CTA)
        const int lg = warp & 3, half = (warp - 2) >> 2;                     // the TMEM lanes this warp may read; its columns
        uint32_t acc = 0, acc_phases = 0;
        bool ok = true;
        for (int i = unit, turn = 0; i < n_items && ok; i += units, ++turn) {
            const Item it = next_item(i, turn);
            const int f = it.f0 + (int)rank * 128 + lg * 32 + lane;
            const bool f_ok = f < a.f_size;
            const size_t at = (DW ? (size_t)it.g * a.group_out : 0) + (size_t)it.row0 * a.ldo + f;
            if (DW && it.kb == 0) {
                if (f_ok && WAY == kWeightGrad)
                    for (int j = half; j < it.cols; j += EW / 4) store_zero(a.out, at + (size_t)j * a.ldo, a.out_kind);
                continue;
            }
            for (int kb = 0; kb < it.kb; kb += it.chunk) {
                if (!(ok = wait_warp(bar_tfull + 8 * acc, acc_phases >> acc & 1, abort_flag, a.err))) break;
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
#pragma unroll 1
                for (int c0 = 32 * half; c0 < to_store; c0 += 8 * EW) {
                    uint32_t v[32];
                    tc_ld32(t0 + c0, v);               // columns behind the item's last are in the accumulator set, not stored
                    tc_wait_ld();
                    const int lim = min(32, it.cols - c0);
                    const size_t to = at + (size_t)c0 * a.ldo;
                    if (f_ok) {
                        if (a.out_kind == EW_FP32) {
                            if (WAY == kWeightAdd || kb > 0) add_columns(reinterpret_cast<float *>(a.out) + to, a.ldo, v, lim);
                            else store_columns(reinterpret_cast<float *>(a.out) + to, a.ldo, v, lim);
                        } else if (a.out_kind == EW_BF16) {
                            put_columns<__nv_bfloat16, WAY == kWeightAdd>(a.out, to, a.ldo, v, lim);
                        } else {
                            put_columns<__half, WAY == kWeightAdd>(a.out, to, a.ldo, v, lim);
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
        if constexpr (CG == 1)
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::kTmemCols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::kTmemCols) : "memory");
    }
}

constexpr int kBarBytes = (3 * kMaxStages + 6) * 8;

// terms: of the longest sum there can be
template <int CG, int NT, int EW, int WAY>
ew_status_t launch(const Device &d, const CUtensorMap &ma, const RowMaps &mb, Args a, long long max_items, int terms,
                   cudaStream_t st) {
    using C = Cfg<CG, NT>;
    if (max_items > 0x7fff0000) return refuse("grouped product: too many output tiles");
    a.table_bytes = (3 * a.groups + 1) * 4;
    const int room = kSmemLimit - 1024 - kBarBytes - a.table_bytes;
    a.stages = room / C::kStageBytes;
    cudaLaunchConfig_t cfg = {};
    const long long units = d.sm_count / CG;
    cfg.gridDim = dim3((unsigned)(CG * (max_items < units ? max_items : units)));
    cfg.blockDim = dim3(threads_of(EW));
    cfg.dynamicSmemBytes = (size_t)a.stages * C::kStageBytes + 1024 + kBarBytes + a.table_bytes;
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
    const bool long_sums = a.out_kind != EW_FP32 && terms > a.sum_blocks * kBlockK;
    return launched((int)(long_sums ? cudaLaunchKernelEx(&cfg, grouped_product_kernel<CG, NT, EW, WAY, true>, ma, mb, a)
                                    : cudaLaunchKernelEx(&cfg, grouped_product_kernel<CG, NT, EW, WAY, false>, ma, mb, a)), "grouped product");
}

template <int CG, int NT, int EW, int WAY>
int setup_one() {
    return (int)cudaFuncSetAttribute(grouped_product_kernel<CG, NT, EW, WAY, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) |
           (int)cudaFuncSetAttribute(grouped_product_kernel<CG, NT, EW, WAY, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
}

// A row-major matrix's row stride: multiples of eight elements keep every TMA copy on a 16-byte boundary.
bool bad_matrix(const void *p, long long ld, long long width) {
    return !p || ((uintptr_t)p & 15) || ld < width || (ld & 7) || ld >= (1ll << 38);
}

ew_status_t check_common(int32_t dtype, int32_t out_dtype, const int32_t *offsets, int32_t rows, int32_t groups, int32_t n, int32_t k,
                         const void *out) {
    if (!is_16bit(dtype) || (out_dtype != dtype && out_dtype != EW_FP32)) return refuse("grouped product: operands are bf16 or fp16, results of the same type or fp32");
    constexpr int32_t kMostSize = 0x7fff0000;                                // (indexes run a tile past the end)
    if (rows < 0 || rows > kMostSize || groups < 1 || groups > kMaxGroups || n < 1 || n > kMostSize || k < 1 || k > kMostSize)
        return refuse("grouped product: size out of range");
    if (!offsets || ((uintptr_t)offsets & 3) || !out || ((uintptr_t)out & (elem_bytes(out_dtype) - 1)))
        return refuse("grouped product: null or misaligned pointer");
    return EW_OK;
}

ew_status_t rows_product(bool grad, int32_t device, int32_t dtype, int32_t out_dtype, const void *x, int64_t ldx, const void *w,
                         int64_t ldw, int64_t group_stride, const int32_t *offsets, int32_t rows, int32_t groups, int32_t n, int32_t k,
                         void *out, int64_t ldo, void *stream) {
    const int t = grad ? n : k, f = grad ? k : n;
    // (a tensor without rows may have no address)
    ew_status_t s = check_common(dtype, out_dtype, offsets, rows, groups, n, k, rows == 0 ? w : out);
    if (s != EW_OK) return s;
    if ((rows > 0 && bad_matrix(x, ldx, t)) || bad_matrix(w, ldw, k) || ldo < f || !rows_apart(groups, group_stride, n, ldw, k) || (groups > 1 && ((group_stride & 7) || group_stride >= (1ll << 38))))
        return refuse("grouped product: operands need 16-byte aligned rows (strides in multiples of eight elements) that do not overlap");
    if (device < 0) return EW_ERR_NO_DEVICE;
    if (rows == 0) return EW_OK;
    DeviceGuard guard;
    if ((s = launched((int)guard.enter(device), "cudaSetDevice")) != EW_OK) return s;
    const Device *d;
    if ((s = device_state(device, &d)) != EW_OK) return s;
    CUtensorMap ma;
    RowMaps mb;
    const uint64_t between = groups > 1 ? (uint64_t)group_stride * 2 : (uint64_t)ldw * 2;
    const bool pairs = grad && k % 64 == 0;            // (otherwise a 64-wide block could end behind the last row)
    if (pairs) {
        const uint64_t wd[4] = {64, (uint64_t)n, (uint64_t)k / 64, (uint64_t)groups}, ws[3] = {(uint64_t)ldw * 2, 128, between};
        const uint32_t box[4] = {64, 64, 2, 1};
        s = encode_map(*d, &ma, map_type(dtype), w, 4, wd, ws, box, CU_TENSOR_MAP_SWIZZLE_128B);
    } else {
        const uint64_t wd[3] = {(uint64_t)k, (uint64_t)n, (uint64_t)groups}, ws[2] = {(uint64_t)ldw * 2, between};
        const uint32_t box[3] = {64, grad ? 64u : 128u, 1};
        s = encode_map(*d, &ma, map_type(dtype), w, 3, wd, ws, box, CU_TENSOR_MAP_SWIZZLE_128B);
    }
    if (s != EW_OK) return s;
    const uint64_t xd[2] = {(uint64_t)t, (uint64_t)rows}, xs[1] = {(uint64_t)ldx * 2};
    for (int i = 0; i < 4; ++i) {
        const uint32_t box[2] = {64, 32u * (i + 1)};
        if ((s = encode_map(*d, &mb.m[i], map_type(dtype), x, 2, xd, xs, box, CU_TENSOR_MAP_SWIZZLE_128B)) != EW_OK) return s;
    }
    Args a = {};
    a.offsets = offsets;
    a.out = out;
    a.err = d->err;
    a.ldo = ldo;
    a.rows = rows;
    a.groups = groups;
    a.f_size = f;
    a.t_size = t;
    a.out_kind = out_dtype;
    a.fp16 = dtype == EW_FP16;
    a.a_pairs = pairs;
    cudaStream_t st = (cudaStream_t)stream;
    const long long live = groups < rows ? groups : rows;                    // groups that can have rows
#define EW_LAUNCH(CG, NT)                                                                                                     \
    do {                                                                                                                      \
        a.f_tiles = (f + 128 * CG - 1) / (128 * CG);                                                                          \
        const long long items = (live + rows / NT) * a.f_tiles;                                                               \
        return grad ? launch<CG, NT, 4, kInputGrad>(*d, ma, mb, a, items, t, st) : launch<CG, NT, 4, kProduct>(*d, ma, mb, a, items, t, st); \
    } while (0)
    // (64 groups of 2816 x 2048, one CTA with 128 columns against the pair: 96 rows a group 127.7 and 130.0 us, 128 rows 134.1 and
    // 134.7, 160 rows 214 and 141.  The host knows only how many groups there are, not which have rows: offsets over many empty
    // slots make the groups look shorter than they are, and the one-CTA form may be taken where the pair would be faster)
    if (rows <= 128ll * groups) EW_LAUNCH(1, 128);
    EW_LAUNCH(2, 256);
#undef EW_LAUNCH
}

}  // namespace

int grouped_setup() {
    return setup_one<1, 128, 4, kProduct>() | setup_one<1, 128, 4, kInputGrad>() |
           setup_one<2, 256, 4, kProduct>() | setup_one<2, 256, 4, kInputGrad>() | setup_one<2, 256, 4, kWeightGrad>() | setup_one<2, 256, 8, kWeightGrad>() |
           setup_one<2, 256, 8, kWeightAdd>();
}

}  // namespace ops
}  // namespace ew

using namespace ew;
using namespace ew::ops;

extern "C" ew_status_t ew_grouped_mm(int32_t device, int32_t dtype, int32_t out_dtype, const void *x, int64_t ldx, const void *w,
                                     int64_t ldw, int64_t group_stride, const int32_t *offsets, int32_t rows, int32_t groups, int32_t n,
                                     int32_t k, void *y, int64_t ldy, void *cuda_stream) {
    return rows_product(false, device, dtype, out_dtype, x, ldx, w, ldw, group_stride, offsets, rows, groups, n, k, y, ldy, cuda_stream);
}

extern "C" ew_status_t ew_grouped_mm_dx(int32_t device, int32_t dtype, int32_t out_dtype, const void *dy, int64_t lddy, const void *w,
                                        int64_t ldw, int64_t group_stride, const int32_t *offsets, int32_t rows, int32_t groups, int32_t n,
                                        int32_t k, void *dx, int64_t lddx, void *cuda_stream) {
    return rows_product(true, device, dtype, out_dtype, dy, lddy, w, ldw, group_stride, offsets, rows, groups, n, k, dx, lddx, cuda_stream);
}

extern "C" ew_status_t ew_grouped_mm_dw(int32_t device, int32_t dtype, int32_t out_dtype, const void *dy, int64_t lddy, const void *x,
                                        int64_t ldx, const int32_t *offsets, int32_t rows, int32_t groups, int32_t n, int32_t k,
                                        int32_t accumulate, void *dw, int64_t lddw, int64_t group_stride, void *cuda_stream) {
    ew_status_t s = check_common(dtype, out_dtype, offsets, rows, groups, n, k, dw);
    if (s != EW_OK) return s;
    if (lddw < k || !rows_apart(groups, group_stride, n, lddw, k))
        return refuse("grouped product: the weight gradient's rows overlap");
    if (rows > 0 && (bad_matrix(dy, lddy, n) || bad_matrix(x, ldx, k)))
        return refuse("grouped product: operands need 16-byte aligned rows (strides in multiples of eight elements) that do not overlap");
    if (device < 0) return EW_ERR_NO_DEVICE;
    DeviceGuard guard;
    if ((s = launched((int)guard.enter(device), "cudaSetDevice")) != EW_OK) return s;
    const Device *d;
    if ((s = device_state(device, &d)) != EW_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (rows == 0) {                                                         // no row: every group's gradient is zero
        if (accumulate) return EW_OK;
        const size_t e = elem_bytes(out_dtype);
        for (int g = 0; g < groups; ++g)
            if ((s = launched((int)cudaMemset2DAsync((uint8_t *)dw + (size_t)g * group_stride * e, lddw * e, 0, k * e, n, st), "cudaMemset2DAsync")) != EW_OK)
                return s;
        return EW_OK;
    }
    CUtensorMap ma;
    RowMaps mb;
    // 64 columns x 64 rows, two such blocks side by side in one copy where the row is made of whole ones
    auto columns = [&](CUtensorMap *m, const void *at, int64_t ld, int width) {
        if (width % 64) {
            const uint64_t dim[2] = {(uint64_t)width, (uint64_t)rows}, stride[1] = {(uint64_t)ld * 2};
            const uint32_t box[2] = {64, 64};
            return encode_map(*d, m, map_type(dtype), at, 2, dim, stride, box, CU_TENSOR_MAP_SWIZZLE_128B);
        }
        const uint64_t dim[3] = {64, (uint64_t)rows, (uint64_t)width / 64}, stride[2] = {(uint64_t)ld * 2, 128};
        const uint32_t box[3] = {64, 64, 2};
        return encode_map(*d, m, map_type(dtype), at, 3, dim, stride, box, CU_TENSOR_MAP_SWIZZLE_128B);
    };
    if ((s = columns(&ma, x, ldx, k)) != EW_OK || (s = columns(&mb.m[0], dy, lddy, n)) != EW_OK) return s;
    Args a = {};
    a.offsets = offsets;
    a.out = dw;
    a.err = d->err;
    a.ldo = lddw;
    a.group_out = group_stride;
    a.rows = rows;
    a.groups = groups;
    a.f_size = k;
    a.a_pairs = k % 64 == 0;
    a.b_pairs = n % 64 == 0;
    a.c_size = n;
    a.f_tiles = (k + 255) / 256;
    a.c_tiles = (n + 255) / 256;
    a.out_kind = out_dtype;
    a.fp16 = dtype == EW_FP16;
    const long long items = (long long)groups * a.c_tiles * a.f_tiles;
    if (accumulate) return launch<2, 256, 8, kWeightAdd>(*d, ma, mb, a, items, rows, st);
    // Few rows a group: the results' way out is what counts, and eight warps walk it (192 rows: 80 us against 95); many: the
    // arithmetic does, at the power limit, where four cost less (768 rows: 259 against 270).  Empty groups count as above.
    return rows <= 256ll * groups ? launch<2, 256, 8, kWeightGrad>(*d, ma, mb, a, items, rows, st) : launch<2, 256, 4, kWeightGrad>(*d, ma, mb, a, items, rows, st);
}
