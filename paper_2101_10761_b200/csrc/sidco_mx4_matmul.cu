// Product of two matrices of microscaled 4-bit numbers, C = A B^T (+ C), on the block-scaled tensor-core path of
// sm_100a (E2M1 operands, E8M0 scales per 32 along K, fp32 accumulation).
//
//   C[i, j] = sum_k a[i, k] b[j, k],   a, b the decoded values; one rounding to the type of C.
//
// Codes arrive by tensor copies of 128-byte rows (256 elements), zero-filled behind the matrix; scales are stored in the
// order in which tensor memory takes them, so that those of 128 rows and a stage are 1024 contiguous bytes.
//
//   pair_kernel   large C: tiles of 256 x 256 by pairs of CTAs, persistent
//   split_kernel  everything else: tiles of 128 x (16 .. 128), K split over a cluster of CTAs
//
// Measured: 8192^3 into bf16 216 us alone (5.1 PFLOP/s, 1000 W: the power limit holds the clock at 1.64 GHz), 255 us in a
// long loop; 6000 x 1500 x 700 added to fp32 18 us (75 MB, 0.62 of the copy rate); one token times 6000 x 1500 4.6 us
// inside a graph (4.8 MB: start, one trip to memory, exchange of the sums), times 8192 x 8192 10 us (0.53 of the copy rate).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "../../include/sidco.h"
#include "sidco_internal.h"
#include "sidco_mx4.cuh"
#include "sidco_tc.cuh"

namespace sidco_mx4mm {

using namespace sidco_tc;
using sidco_mx4::blocks_of;
using sidco_mx4::kTileBytes;

constexpr int kStageK = 256;                                          // elements; 128 bytes of codes
constexpr int kRowBytes = 128;
constexpr int kScales = 2 * kTileBytes;                               // of 128 rows and a stage

struct Args {
    int64_t m, n, k;
    int64_t ktiles;                   // scale tiles along K
    void* c;
    int64_t ldc;
    int add;
    int boxes;                        // pair tiles: C is aligned for tensor stores (16 bytes); 2: so is the end of its rows
    int* timeouts;
};

__device__ int g_timeouts;

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half narrow<__half>(float x) { return __float2half_rn(x); }

// 64-wide products of stage k.
__device__ __forceinline__ int quarters_of(const Args& A, int k) {
    return (int)min((int64_t)4, (A.k - (int64_t)k * kStageK + 63) / 64);
}

// ---------------------------------------------------------------------------------------------- pair tiles
//
// Each of the two CTAs holds 128 rows of A and half of the 256 rows of B per stage (a 128 x 128 tile would read twice the
// operand bytes per operation: 8192^3 took 407 us with those, bound by L2).  Two sets of 256 columns of sums and the scales
// of four stages do not fit into the 512 columns of tensor memory, so the sets share 96 columns: those are taken out first,
// and then the next tile's products start.
//   warp 0     feeds the stages        warp 1     issues the products (first CTA)
//   warps 2-9  take the sums out: a quarter of the CTA's 128 rows, two of the four times 64 columns
// Sums leave through shared memory as boxes of 32 rows x 128 bytes: the tensor copies write (or, in fp32, add) them as whole
// lines and leave out what lies behind C.  (Transposed in shared memory and written by single elements they took 33 us per
// tile, twice the products; 6000 x 1500 x 700 added to fp32 29 us instead of 18.)

constexpr int kPairTile = 256;
constexpr int kPairThreads = 320;
constexpr int kPairStages = 5;
constexpr int kPairStageBytes = 2 * 128 * kRowBytes + 3 * kScales;    // 35 KB
constexpr int kPairWarpOut = 32 * 128;                                // a box of C per warp: 32 rows of 128 bytes
constexpr int kPairSmem = kPairStages * kPairStageBytes + 8 * kPairWarpOut + 1024;
constexpr int kSecondSums = 160, kScaleColumns = 416, kScaleColumnsPerStage = 24, kScaleStages = 4;

template <typename T>
__global__ void __launch_bounds__(kPairThreads, 1) __cluster_dims__(2)
    pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
                const __grid_constant__ CUtensorMap map_c, const Args A, int tiles_m, int tiles_n) {
    extern __shared__ uint8_t s_raw[];
    __shared__ uint64_t s_full[kPairStages], s_free[kPairStages], s_sums[2], s_shared;
    __shared__ uint32_t s_tmem;
    __shared__ int s_failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    uint8_t* smem = (uint8_t*)(((uintptr_t)s_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t stage0 = smem_addr(smem);
    if (warp == 1) tmem_alloc_pair(&s_tmem, 512);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairStages; ++i) {
            mbar_init(smem_addr(&s_full[i]), 1);
            mbar_init(smem_addr(&s_free[i]), 1);
        }
        for (int i = 0; i < 2; ++i) mbar_init(smem_addr(&s_sums[i]), 1);
        mbar_init(smem_addr(&s_shared), 16);                          // eight warps of both CTAs
        s_failed = 0;
        mbar_init_fence();
    }
    fence_before_sync();
    __syncthreads();
    cluster_sync();
    fence_after_sync();
    const uint32_t tmem = s_tmem;
    wait_prerequisites();                                             // (the set-up may run under the kernel before)
    launch_dependents();
    const int n_pairs = gridDim.x / 2, first = blockIdx.x / 2, total = tiles_m * tiles_n;
    const int steps = (int)((A.k + kStageK - 1) / kStageK);
    // tiles in bands of eight tile rows, column by column, so that pairs at work at the same time share operands in L2
    const auto place = [&](int i, int& ti, int& tj) {
        const int band = i / (8 * tiles_n), in = i - band * 8 * tiles_n, rows = min(8, tiles_m - band * 8);
        ti = band * 8 + in % rows;
        tj = in / rows;
    };
    if (warp == 0) {
        if (lane == 0) {
            int st = 0;
            uint32_t round = 0;
            bool ok = true;
            for (int i = first; i < total && ok; i += n_pairs) {
                int ti, tj;
                place(i, ti, tj);
                const int row_a = ti * kPairTile + (int)rank * 128, row_b = tj * kPairTile + (int)rank * 128;
                for (int k = 0; k < steps; ++k) {
                    const uint32_t a = stage0 + st * kPairStageBytes, b = a + 128 * kRowBytes, sa = b + 128 * kRowBytes;
                    const uint32_t bar = smem_addr(&s_full[st]);
                    ok = mbar_wait(smem_addr(&s_free[st]), (round & 1) ^ 1, &s_failed);
                    if (!ok) break;
                    if (rank == 0) mbar_expect_tx(bar, 2 * kPairStageBytes);
                    tensor_load_2d_pair(a, &map_a, k * kRowBytes, row_a, bar);
                    tensor_load_2d_pair(b, &map_b, k * kRowBytes, row_b, bar);
                    // (scales as rows of 128 bytes: four per tile; every CTA needs those of all rows of B)
                    tensor_load_2d_pair(sa, &map_sa, 0, (int)((ti * 2 + rank) * A.ktiles + 2 * k) * 4, bar);
                    tensor_load_2d_pair(sa + kScales, &map_sb, 0, (int)(tj * 2 * A.ktiles + 2 * k) * 4, bar);
                    tensor_load_2d_pair(sa + 2 * kScales, &map_sb, 0, (int)((tj * 2 + 1) * A.ktiles + 2 * k) * 4, bar);
                    if (++st == kPairStages) { st = 0; ++round; }
                }
            }
        }
    } else if (warp == 1) {
        // (the whole warp waits, one thread issues)
        if (rank == 0) {
            int st = 0, n = 0, used = 0;
            uint32_t round = 0;
            bool ok = true;
            for (int i = first; i < total && ok; i += n_pairs, ++n) {
                const uint32_t sums = tmem + (n & 1) * kSecondSums;
                if (n) ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&s_shared), (n - 1) & 1, &s_failed));
                for (int k = 0; k < steps && ok; ++k, ++used) {
                    ok = mbar_wait(smem_addr(&s_full[st]), round & 1, &s_failed);
                    // the columns for the scales: free when the products of four stages ago are done
                    if (ok && used >= kScaleStages) {
                        const int back = st >= kScaleStages ? st - kScaleStages : st + kPairStages - kScaleStages;
                        ok = mbar_wait(smem_addr(&s_free[back]), (st >= kScaleStages ? round : round - 1) & 1, &s_failed);
                    }
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    fence_after_sync();
                    const uint32_t a = stage0 + st * kPairStageBytes, b = a + 128 * kRowBytes, sa = b + 128 * kRowBytes;
                    const uint32_t ta = tmem + kScaleColumns + (used & (kScaleStages - 1)) * kScaleColumnsPerStage, tb = ta + 8;
                    const int quarters = quarters_of(A, k);
                    if (elect_one()) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (h * 2 >= quarters) break;
                            copy_scales_pair(ta + h * 4, plain_operand(sa + h * kTileBytes, 16, 128));
                            copy_scales_pair(tb + h * 8, plain_operand(sa + kScales + h * kTileBytes, 16, 128));
                            copy_scales_pair(tb + h * 8 + 4, plain_operand(sa + 2 * kScales + h * kTileBytes, 16, 128));
                        }
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            if (q >= quarters) break;
                            mma_mx4_pair(sums, swizzled_operand(a + q * 32, 16, 1024), swizzled_operand(b + q * 32, 16, 1024),
                                         mx4_shape(kPairTile, kPairTile, (q & 1) * 2, (q & 1) * 2), ta + (q >> 1) * 4,
                                         tb + (q >> 1) * 8, k > 0 || q > 0);
                        }
                        tc_commit_pair(smem_addr(&s_free[st]));
                        if (k + 1 == steps) tc_commit_pair(smem_addr(&s_sums[n & 1]));
                    }
                    __syncwarp();
                    if (++st == kPairStages) { st = 0; ++round; }
                }
            }
        }
    } else {
        const int quarter = warp & 3, odd = (warp - 2) >> 2;
        uint8_t* box = smem + kPairStages * kPairStageBytes + (warp - 2) * kPairWarpOut;
        const uint32_t shared_taken = in_cta(smem_addr(&s_shared), 0);
        T* c = static_cast<T*>(A.c);
        int n = 0;
        for (int i = first; i < total; i += n_pairs, ++n) {
            int ti, tj;
            place(i, ti, tj);
            const int64_t r0 = (int64_t)ti * kPairTile + rank * 128 + quarter * 32;
            const int lines = (int)max((int64_t)0, min((int64_t)32, A.m - r0));
            const uint32_t sums = tmem + (n & 1) * kSecondSums + ((uint32_t)(quarter * 32) << 16);
            // 64 columns at a time, those of the shared columns first: the upper half of the first set, the lower of the second
#pragma unroll 1
            for (int p = 0; p < 2; ++p) {
                const int part = (n & 1 ? p : p ^ 1) * 2 + odd;
                const int64_t col = (int64_t)tj * kPairTile + part * 64;
                const T* mine = c + (r0 + lane) * A.ldc + col;        // this lane's row
                // (a tensor store leaves out 16 bytes at a time: a box over any other end of the rows would write behind it)
                const bool boxes = A.boxes && (col + 64 <= A.n || (A.boxes == 2 && (sizeof(T) == 4 || !A.add)));
                uint4 old[8];                                         // (16-bit types are added here, rounded once)
                if (sizeof(T) == 2 && A.add && boxes && lane < lines) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) old[j] = reinterpret_cast<const uint4*>(mine)[j];
                }
                if (p == 0) {
                    mbar_wait(smem_addr(&s_sums[n & 1]), (n >> 1) & 1, &s_failed);
                    __syncwarp();
                    fence_after_sync();
                }
                uint32_t acc[64];
                tmem_load32(sums + part * 64, *reinterpret_cast<uint32_t(*)[32]>(acc));
                tmem_load32(sums + part * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(acc + 32));
                if (p == 0) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(shared_taken);
                }
                if (__any_sync(0xffffffffu, *(volatile int*)&s_failed)) break;
                if (boxes) {
                    constexpr int kPer = 16 / (int)sizeof(T);         // elements of 16 bytes
#pragma unroll
                    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {    // boxes of 128 bytes
                        if (lane == 0) bulk_store_wait_read();
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            alignas(16) T t[kPer];
#pragma unroll
                            for (int e = 0; e < kPer; ++e) {
                                float v = __uint_as_float(acc[h * 32 + j * kPer + e]);
                                if (sizeof(T) == 2 && A.add)
                                    v += lane < lines ? widen(reinterpret_cast<const T*>(&old[j])[e]) : 0.0f;
                                t[e] = narrow<T>(v);
                            }
                            *reinterpret_cast<uint4*>(box + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                                *reinterpret_cast<const uint4*>(t);
                        }
                        fence_async_shared();
                        __syncwarp();
                        if (lane == 0) {
                            const int x = (int)col + h * 32;
                            if (lines && x < A.n) {
                                if (sizeof(T) == 4 && A.add) tensor_add_2d(&map_c, x, (int)r0, smem_addr(box));
                                else tensor_store_2d(&map_c, x, (int)r0, smem_addr(box));
                            }
                            bulk_store_commit();
                        }
                    }
                    continue;
                }
                // other alignments: eight columns at a time through shared memory, so that a quarter of the warp writes
                // neighbours of a row
                if (lane == 0) bulk_store_wait_read();
                float* s_t = reinterpret_cast<float*>(box);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j) s_t[lane * 9 + j] = __uint_as_float(acc[e * 8 + j]);
                    __syncwarp();
                    const int64_t my_col = col + e * 8 + (lane & 7);
                    if (my_col >= A.n) continue;
                    T* to = c + r0 * A.ldc + my_col;
                    float before[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const int line = r * 4 + (lane >> 3);
                        before[r] = A.add && line < lines ? widen(to[line * A.ldc]) : 0.0f;
                    }
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const int line = r * 4 + (lane >> 3);
                        if (line < lines) to[line * A.ldc] = narrow<T>(s_t[line * 9 + (lane & 7)] + before[r]);
                    }
                }
            }
            if (__any_sync(0xffffffffu, *(volatile int*)&s_failed)) break;
        }
        if (lane == 0) bulk_store_wait();
    }
    __syncwarp();
    fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s_failed) {
        atomicAdd(A.timeouts, 1);
        let_work_end();
    }
    __syncthreads();
    cluster_sync();
    if (warp == 1) tmem_free_pair(tmem, 512);
}

// ---------------------------------------------------------------------------------------------- split tiles
//
// A tile of 128 x N by a cluster of CTAs, each with its part of K: their partial sums are added through distributed shared
// memory in the order of the CTAs, each CTA finishing its share of the tile.  With few rows on one side (a single token, a
// small batch) that side is the N of the product and the other streams through its 128 rows ("swapped": the tile is
// C^T).  Two CTAs per SM; a CTA's stages are all in flight at once.

constexpr int kSplitThreads = 256;
constexpr int kSplitMost = 8;                                         // CTAs per tile
template <int N> constexpr int kSplitStageBytes = (128 + N) * kRowBytes + 2 * kScales;
template <int N> constexpr int kSplitStages = N == 128 ? 3 : N == 64 ? 4 : 5;
template <int N> constexpr int kSplitSmem = kSplitStages<N> * kSplitStageBytes<N> + 1024;

__device__ __forceinline__ float4 remote_load16(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}

template <typename T, int N>
__global__ void __launch_bounds__(kSplitThreads, 2)
    split_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                 const uint8_t* __restrict__ a_scales, const uint8_t* __restrict__ b_scales, const Args A, int tiles_b,
                 int swapped, int vec) {
    constexpr int kStages = kSplitStages<N>, kStageBytes = kSplitStageBytes<N>;
    constexpr uint32_t kColumns = N == 128 ? 256 : 128;               // N of sums, 16 of scales per stage
    extern __shared__ uint8_t s_raw[];
    __shared__ uint64_t s_full[kStages], s_free[kStages], s_done;
    __shared__ uint32_t s_tmem;
    __shared__ int s_failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t ctas;
    asm("mov.u32 %0, %cluster_nctaid.x;" : "=r"(ctas));
    const uint32_t rank = cluster_rank();
    uint8_t* smem = (uint8_t*)(((uintptr_t)s_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t stage0 = smem_addr(smem);
    if (warp == 0) tmem_alloc(&s_tmem, kColumns);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(smem_addr(&s_full[i]), 1);
            mbar_init(smem_addr(&s_free[i]), 1);
        }
        mbar_init(smem_addr(&s_done), 1);
        s_failed = 0;
        mbar_init_fence();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = s_tmem;
    wait_prerequisites();                                             // (the set-up may run under the kernel before)
    launch_dependents();
    const int tile = blockIdx.x / ctas, ti = tile / tiles_b, tj = tile % tiles_b;
    const int steps = (int)((A.k + kStageK - 1) / kStageK);
    const int from = steps * (int)rank / (int)ctas, to = steps * (int)(rank + 1) / (int)ctas;

    if (warp == 0) {
        if (elect_one()) {
            for (int k = from; k < to; ++k) {
                const int i = k - from, st = i % kStages;
                if (i >= kStages && !mbar_wait(smem_addr(&s_free[st]), (i / kStages - 1) & 1, &s_failed)) break;
                const uint32_t a = stage0 + st * kStageBytes, b = a + 128 * kRowBytes, sa = b + N * kRowBytes, sb = sa + kScales;
                const uint32_t bar = smem_addr(&s_full[st]);
                const uint32_t bytes = (uint32_t)min((int64_t)2, A.ktiles - 2 * k) * kTileBytes;
                mbar_expect_tx(bar, (128 + N) * kRowBytes + 2 * bytes);
                tensor_load_2d(a, &map_a, k * kRowBytes, ti * 128, bar);
                tensor_load_2d(b, &map_b, k * kRowBytes, tj * N, bar);
                bulk_load(sa, a_scales + (ti * A.ktiles + 2 * k) * kTileBytes, bytes, bar);
                bulk_load(sb, b_scales + (tj * A.ktiles + 2 * k) * kTileBytes, bytes, bar);
            }
        }
    } else if (warp == 1) {
        for (int k = from; k < to; ++k) {
            const int i = k - from, st = i % kStages;
            if (!__all_sync(0xffffffffu, mbar_wait(smem_addr(&s_full[st]), (i / kStages) & 1, &s_failed))) break;
            fence_after_sync();
            const uint32_t a = stage0 + st * kStageBytes, b = a + 128 * kRowBytes, sa = b + N * kRowBytes, sb = sa + kScales;
            // (every stage has columns of its own: they are free when the stage is)
            const uint32_t ta = tmem + N + st * 16, tb = ta + 8;
            const int quarters = quarters_of(A, k);
            if (elect_one()) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h * 2 >= quarters) break;
                    copy_scales(ta + h * 4, plain_operand(sa + h * kTileBytes, 16, 128));
                    copy_scales(tb + h * 4, plain_operand(sb + h * kTileBytes, 16, 128));
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (q >= quarters) break;
                    mma_mx4(tmem, swizzled_operand(a + q * 32, 16, 1024), swizzled_operand(b + q * 32, 16, 1024),
                            mx4_shape(128, N, (q & 1) * 2, (q & 1) * 2), ta + (q >> 1) * 4, tb + (q >> 1) * 4, i > 0 || q > 0);
                }
                tc_commit(smem_addr(&s_free[st]));
            }
            __syncwarp();
        }
        if (elect_one()) tc_commit(smem_addr(&s_done));
    }
    __syncwarp();
    mbar_wait(smem_addr(&s_done), 0, &s_failed);
    __syncwarp();
    fence_after_sync();

    // the partial sums as rows of C (the stages are free), four words of padding against bank conflicts
    float* s_c = reinterpret_cast<float*>(smem);
    const int row = (warp & 3) * 32 + lane, half = warp >> 2;
    const int len = swapped ? 128 : N, pitch = len + 4;
    for (int q = half; q < (N + 31) / 32; q += 2) {
        uint32_t acc[32];
        tmem_load32(tmem + ((uint32_t)((warp & 3) * 32) << 16) + q * 32, acc);
        if (from == to) {                                             // no part of K
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[j] = 0;
        }
        if (swapped) {
#pragma unroll
            for (int j = 0; j < (N < 32 ? N : 32); ++j) s_c[(q * 32 + j) * pitch + row] = __uint_as_float(acc[j]);
        } else {
#pragma unroll
            for (int j = 0; j < (N < 32 ? N : 32) / 4; ++j)
                *reinterpret_cast<float4*>(s_c + row * pitch + q * 32 + j * 4) =
                    make_float4(__uint_as_float(acc[j * 4]), __uint_as_float(acc[j * 4 + 1]),
                                __uint_as_float(acc[j * 4 + 2]), __uint_as_float(acc[j * 4 + 3]));
        }
    }
    fence_before_sync();
    __syncthreads();
    cluster_sync();
    const int64_t r0 = swapped ? (int64_t)tj * N : (int64_t)ti * 128, c0 = swapped ? (int64_t)ti * 128 : (int64_t)tj * N;
    const int lines = (int)min((int64_t)(swapped ? N : 128), A.m - r0);
    T* c = static_cast<T*>(A.c);
    const int fours = len / 4, mine = lines * fours;                  // four neighbours of a row at a time
    const int shift = swapped ? 5 : N == 128 ? 5 : N == 64 ? 4 : N == 32 ? 3 : 2;
    if (!s_failed)
        for (int i = (int)rank * kSplitThreads + threadIdx.x; i < mine; i += (int)ctas * kSplitThreads) {
            const int r = i >> shift, q4 = (i & (fours - 1)) * 4;
            const int64_t col = c0 + q4;
            if (col >= A.n) continue;
            T* at = c + (r0 + r) * A.ldc + col;
            const uint32_t src = smem_addr(s_c + r * pitch + q4);
            const bool whole = vec && col + 4 <= A.n;
            float old[4] = {};
            if (A.add) {
                if (whole) {
                    T t[4];
                    if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(t) = *reinterpret_cast<const uint4*>(at);
                    else *reinterpret_cast<uint2*>(t) = *reinterpret_cast<const uint2*>(at);
#pragma unroll
                    for (int j = 0; j < 4; ++j) old[j] = widen(t[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) old[j] = col + j < A.n ? widen(at[j]) : 0.0f;
                }
            }
            float4 w[kSplitMost];
#pragma unroll
            for (uint32_t p = 0; p < kSplitMost; ++p)
                if (p < ctas) w[p] = remote_load16(in_cta(src, p));
            float v[4] = {};
#pragma unroll
            for (uint32_t p = 0; p < kSplitMost; ++p)
                if (p < ctas) {
                    v[0] += w[p].x;
                    v[1] += w[p].y;
                    v[2] += w[p].z;
                    v[3] += w[p].w;
                }
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += old[j];
            if (whole) {
                alignas(16) T t[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) t[j] = narrow<T>(v[j]);
                if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(at) = *reinterpret_cast<const uint4*>(t);
                else *reinterpret_cast<uint2*>(at) = *reinterpret_cast<const uint2*>(t);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (col + j < A.n) at[j] = narrow<T>(v[j]);
            }
        }
    if (threadIdx.x == 0 && s_failed) {
        atomicAdd(A.timeouts, 1);
        let_work_end();
    }
    __syncthreads();
    cluster_sync();                                                   // nobody reads this CTA's sums any more
    if (warp == 0) tmem_free(tmem, kColumns);
}

// ---------------------------------------------------------------------------------------------- host side

// Codes: boxes of 128 bytes x `box` rows, swizzled, zeros outside.
static bool code_map(CUtensorMap* map, const uint8_t* codes, int64_t rows, int64_t k, int box) {
    const int64_t pitch = blocks_of(k) * 16;
    return sidco_internal::byte_map(map, codes, pitch, rows, pitch, 128, box, true);
}

// Scales: rows of 128 bytes, boxes of 1024 bytes.
static bool scale_map(CUtensorMap* map, const uint8_t* scales, int64_t rows, int64_t ktiles) {
    return sidco_internal::byte_map(map, scales, 128, (rows + 127) / 128 * ktiles * 4, 128, 128, 8, false);
}

template <typename T> constexpr int type_of() {
    return sizeof(T) == 4 ? SIDCO_T_F32 : std::is_same<T, __half>::value ? SIDCO_T_F16 : SIDCO_T_BF16;
}

struct Operands {
    const uint8_t *a_codes, *a_scales, *b_codes, *b_scales;
};

template <typename T>
static cudaError_t prepare(int* max_pairs) {
    const auto most = cudaFuncAttributeMaxDynamicSharedMemorySize;
    cudaError_t e;
    if ((e = cudaFuncSetAttribute(pair_kernel<T>, most, kPairSmem)) != cudaSuccess ||
        (e = cudaFuncSetAttribute(split_kernel<T, 16>, most, kSplitSmem<16>)) != cudaSuccess ||
        (e = cudaFuncSetAttribute(split_kernel<T, 32>, most, kSplitSmem<32>)) != cudaSuccess ||
        (e = cudaFuncSetAttribute(split_kernel<T, 64>, most, kSplitSmem<64>)) != cudaSuccess ||
        (e = cudaFuncSetAttribute(split_kernel<T, 128>, most, kSplitSmem<128>)) != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = kPairSmem;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(max_pairs, pair_kernel<T>, &cfg);
    return e == cudaSuccess && *max_pairs < 1 ? cudaErrorInvalidConfiguration : e;
}

template <typename T, int N>
static int split(const Operands& o, const Args& a, bool swapped, int max_pairs, cudaStream_t s) {
    const int64_t rows_a = swapped ? a.n : a.m, rows_b = swapped ? a.m : a.n;
    const int64_t tiles_a = (rows_a + 127) / 128, tiles_b = (rows_b + N - 1) / N, steps = (a.k + kStageK - 1) / kStageK;
    if (tiles_a * tiles_b * kSplitMost > 0x7fffffff) return SIDCO_E_SIZE;
    // as many parts of K as the resident CTAs (four per pair of SMs) take at once, two stages each at least
    int ctas = 1;
    while (ctas < kSplitMost && tiles_a * tiles_b * ctas * 2 <= 4 * (int64_t)max_pairs && steps >= 4 * ctas) ctas *= 2;
    CUtensorMap map_a, map_b;
    if (!code_map(&map_a, swapped ? o.b_codes : o.a_codes, rows_a, a.k, 128) ||
        !code_map(&map_b, swapped ? o.a_codes : o.b_codes, rows_b, a.k, N))
        return SIDCO_E_UNSUPPORTED;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles_a * tiles_b * ctas));
    cfg.blockDim = dim3(kSplitThreads);
    cfg.dynamicSmemBytes = kSplitSmem<N>;
    cfg.stream = s;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const int vec = (uintptr_t)a.c % (4 * sizeof(T)) == 0 && a.ldc % 4 == 0;
    return (int)cudaLaunchKernelEx(&cfg, split_kernel<T, N>, map_a, map_b, swapped ? o.b_scales : o.a_scales,
                                   swapped ? o.a_scales : o.b_scales, a, (int)tiles_b, (int)swapped, vec);
}

template <typename T>
static int matmul_typed(const Operands& o, Args a, cudaStream_t s) {
    static std::atomic<int> pairs[64];                                // pairs of CTAs that are resident at once
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return (int)e;
    if (dev < 0 || dev >= 64) return SIDCO_E_SIZE;
    if (!pairs[dev].load()) {                // (setting it twice from two threads is harmless)
        int n = 0;
        if ((e = prepare<T>(&n)) != cudaSuccess) return (int)e;
        pairs[dev].store(n);
    }
    const int max_pairs = pairs[dev].load();
    if ((e = cudaGetSymbolAddress((void**)&a.timeouts, g_timeouts)) != cudaSuccess) return (int)e;
    const int64_t tiles_m = (a.m + kPairTile - 1) / kPairTile, tiles_n = (a.n + kPairTile - 1) / kPairTile;
    int rc;
    // Pairs of CTAs from as many tiles on as there are pairs.  Measured on both sides (us, pairs / split): 40 tiles, K = 256
    // 5.4 / 9.5, K = 8192 19.1 / 22.7; 72 tiles 5.9 / 9.6 and 19.7 / 23.9; 80 tiles (two rounds) 7.4 / 15.3 and 33.7 / 41.2;
    // 150 tiles 9.8 / 24.0 and 48.2 / 61.1.  So the line might lie at 40 tiles or lower; below that it was not measured.
    if (tiles_m * tiles_n >= max_pairs && a.m > 64 && a.n > 64) {
        if (tiles_m * tiles_n > 0x7fffffff / 2) return SIDCO_E_SIZE;
        CUtensorMap map_a, map_b, map_sa, map_sb, map_c{};
        if (!code_map(&map_a, o.a_codes, a.m, a.k, 128) || !code_map(&map_b, o.b_codes, a.n, a.k, 128) ||
            !scale_map(&map_sa, o.a_scales, a.m, a.ktiles) || !scale_map(&map_sb, o.b_scales, a.n, a.ktiles) ||
            (a.boxes && !sidco_internal::out_map(&map_c, a.c, type_of<T>(), a.n, a.m, a.ldc, 128 / (int)sizeof(T), 32)))
            return SIDCO_E_UNSUPPORTED;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(2 * max_pairs);
        cfg.blockDim = dim3(kPairThreads);
        cfg.dynamicSmemBytes = kPairSmem;
        cfg.stream = s;
        cudaLaunchAttribute attr{};
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        rc = (int)cudaLaunchKernelEx(&cfg, pair_kernel<T>, map_a, map_b, map_sa, map_sb, map_c, a, (int)tiles_m, (int)tiles_n);
    } else {
        const int64_t few = std::min(a.m, a.n);
        const bool swapped = few <= 64 && a.m <= a.n;
        rc = few > 64 ? split<T, 128>(o, a, false, max_pairs, s)
             : few > 32 ? split<T, 64>(o, a, swapped, max_pairs, s)
             : few > 16 ? split<T, 32>(o, a, swapped, max_pairs, s)
                        : split<T, 16>(o, a, swapped, max_pairs, s);
    }
    if (rc == 0) sidco_internal::note_launch();
    return rc;
}

}  // namespace sidco_mx4mm

namespace {

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static Encode encoder() {
    static Encode f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (Encode)p;
    }();
    return f;
}

}  // namespace

bool sidco_internal::byte_map(CUtensorMap* map, const void* base, int64_t width, int64_t rows, int64_t pitch, int box_width,
                              int box_rows, bool swizzle) {
    if (!encoder()) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t boxes[2] = {(cuuint32_t)box_width, (cuuint32_t)box_rows}, steps[2] = {1, 1};
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, boxes, steps,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool sidco_internal::out_map(CUtensorMap* map, void* base, int type, int64_t width, int64_t rows, int64_t pitch, int box_width,
                             int box_rows) {
    if (!encoder()) return false;
    const int size = type == SIDCO_T_F32 ? 4 : 2;
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(pitch * size)};
    const cuuint32_t boxes[2] = {(cuuint32_t)box_width, (cuuint32_t)box_rows}, steps[2] = {1, 1};
    return encoder()(map,
                     type == SIDCO_T_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                     : type == SIDCO_T_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                            : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                     2, base, dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sidco_internal::mx4_matmul_timeouts(int* count) {
    return (int)cudaMemcpyFromSymbol(count, sidco_mx4mm::g_timeouts, sizeof(int));
}

extern "C" {

int sidco_mx4_matmul(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales,
                     int64_t m, int64_t n, int64_t k, void* c, int c_type, int64_t ldc, int add, void* stream) {
    using namespace sidco_mx4mm;
    const int64_t most = ((int64_t)1 << 31) - ((int64_t)1 << 16);
    if (m < 0 || n < 0 || k < 0 || m > most || n > most || k > most) return SIDCO_E_SIZE;
    if (c_type < SIDCO_T_F32 || c_type > SIDCO_T_F16) return SIDCO_E_TYPE;
    if (ldc < n) return SIDCO_E_PARAMS;
    if (m == 0 || n == 0) return 0;
    if (!c || (k > 0 && (!a_codes || !a_scales || !b_codes || !b_scales))) return SIDCO_E_NULL;
    const uintptr_t size = c_type == SIDCO_T_F32 ? 4 : 2;
    if (((uintptr_t)a_codes | (uintptr_t)a_scales | (uintptr_t)b_codes | (uintptr_t)b_scales) % 16 || (uintptr_t)c % size)
        return SIDCO_E_ALIGN;
    cudaStream_t s = (cudaStream_t)stream;
    if (k == 0) {                            // an empty sum
        if (add) return 0;
        return (int)cudaMemset2DAsync(c, ldc * size, 0, n * size, m, s);
    }
    const int boxes = (uintptr_t)c % 16 || ldc * size % 16 ? 0 : n * size % 16 ? 1 : 2;
    Args a{m, n, k, (blocks_of(k) + 3) / 4, c, ldc, add != 0, boxes, nullptr};
    const Operands o{a_codes, a_scales, b_codes, b_scales};
    if (c_type == SIDCO_T_F32) return matmul_typed<float>(o, a, s);
    if (c_type == SIDCO_T_BF16) return matmul_typed<__nv_bfloat16>(o, a, s);
    return matmul_typed<__half>(o, a, s);
}

int sidco_wait_timeouts(void) {
    int a = 0, b = 0, rc;
    if ((rc = sidco_internal::orthogonalize_timeouts(&a)) || (rc = sidco_internal::mx4_matmul_timeouts(&b)))
        return rc > 0 ? -rc : rc;
    return a + b;
}

}  // extern "C"
