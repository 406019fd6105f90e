// Product of two matrices of microscaled 4-bit numbers, C = A B^T (+ C), on the block-scaled tensor-core path of
// sm_100a (E2M1 operands, E8M0 scales per 32 along K, fp32 accumulation).
//
//   C[i, j] = sum_k a[i, k] b[j, k],   a, b the decoded values; one rounding to the type of C.
//
// Codes arrive by tensor copies of 128 rows x 128 bytes (256 elements), zero-filled behind the matrix; scales are
// stored in the order in which tensor memory takes them, so a stage's scales are one contiguous copy per 128 rows.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sidco.h"
#include "sidco_internal.h"
#include "sidco_mx4.cuh"
#include "sidco_tc.cuh"

namespace sidco_mx4mm {

using namespace sidco_tc;
using sidco_mx4::blocks_of;
using sidco_mx4::kTileBytes;

constexpr int kTileM = 128, kTileN = 128;
constexpr int kStageK = 256;                                          // elements; 128 bytes of codes
constexpr int kCodesA = kTileM * 128, kCodesB = kTileN * 128;
constexpr int kScales = 2 * kTileBytes;                               // of 128 rows and a stage
constexpr int kStageBytes = kCodesA + kCodesB + 2 * kScales;          // (a multiple of 1024)
constexpr int kStages = 3;
constexpr int kThreads = 128;
constexpr int kSmem = kStages * kStageBytes + 1024;
constexpr int kTmemColumns = 256;                                     // 128 of sums, 16 of scales per stage

struct Args {
    const uint8_t *a_scales, *b_scales;
    int64_t m, n, k;
    int64_t ktiles;                   // scale tiles along K
    void* c;
    int64_t ldc;
    int type, add;
    int tiles_n;
    int* timeouts;
};

__device__ int g_timeouts;

__device__ __forceinline__ float read_c(const void* c, int type, int64_t i) {
    if (type == SIDCO_T_F32) return ((const float*)c)[i];
    if (type == SIDCO_T_BF16) return __bfloat162float(((const __nv_bfloat16*)c)[i]);
    return __half2float(((const __half*)c)[i]);
}

__device__ __forceinline__ void write_c(void* c, int type, int64_t i, float v) {
    if (type == SIDCO_T_F32) ((float*)c)[i] = v;
    else if (type == SIDCO_T_BF16) ((__nv_bfloat16*)c)[i] = __float2bfloat16_rn(v);
    else ((__half*)c)[i] = __float2half_rn(v);
}

__global__ void __launch_bounds__(kThreads, 2) matmul_kernel(const __grid_constant__ CUtensorMap map_a,
                                                             const __grid_constant__ CUtensorMap map_b, const Args A) {
    extern __shared__ uint8_t s_raw[];
    __shared__ uint64_t s_full[kStages], s_free[kStages], s_done;
    __shared__ uint32_t s_tmem;
    __shared__ int s_failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* smem = (uint8_t*)(((uintptr_t)s_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t stage0 = smem_addr(smem);
    if (warp == 0) tmem_alloc(&s_tmem, kTmemColumns);
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
    const int ti = blockIdx.x / A.tiles_n, tj = blockIdx.x % A.tiles_n;
    const int steps = (int)((A.k + kStageK - 1) / kStageK);

    if (threadIdx.x == 0) {
        for (int k = 0; k < steps; ++k) {
            const int st = k % kStages;
            if (k >= kStages && !mbar_wait(smem_addr(&s_free[st]), (k / kStages - 1) & 1, &s_failed)) break;
            const uint32_t a = stage0 + st * kStageBytes, b = a + kCodesA, sa = b + kCodesB, sb = sa + kScales;
            const uint32_t bar = smem_addr(&s_full[st]);
            const uint32_t bytes = (uint32_t)min((int64_t)2, A.ktiles - 2 * k) * kTileBytes;
            mbar_expect_tx(bar, kCodesA + kCodesB + 2 * bytes);
            tensor_load_2d(a, &map_a, k * 128, ti * kTileM, bar);
            tensor_load_2d(b, &map_b, k * 128, tj * kTileN, bar);
            bulk_load(sa, A.a_scales + (ti * A.ktiles + 2 * k) * kTileBytes, bytes, bar);
            bulk_load(sb, A.b_scales + (tj * A.ktiles + 2 * k) * kTileBytes, bytes, bar);
        }
    } else if (threadIdx.x == 32) {
        for (int k = 0; k < steps; ++k) {
            const int st = k % kStages;
            if (!mbar_wait(smem_addr(&s_full[st]), (k / kStages) & 1, &s_failed)) break;
            fence_after_sync();
            const uint32_t a = stage0 + st * kStageBytes, b = a + kCodesA, sa = b + kCodesB, sb = sa + kScales;
            // (every stage has columns of its own: they are free when the stage is)
            const uint32_t ta = tmem + kTileN + st * 16, tb = ta + 8;
            const int quarters = (int)min((int64_t)4, (A.k - (int64_t)k * kStageK + 63) / 64);
            for (int h = 0; h * 2 < quarters; ++h) {
                copy_scales(ta + h * 4, plain_operand(sa + h * kTileBytes, 16, 128));
                copy_scales(tb + h * 4, plain_operand(sb + h * kTileBytes, 16, 128));
            }
            for (int q = 0; q < quarters; ++q)
                mma_mx4(tmem, swizzled_operand(a + q * 32, 16, 1024), swizzled_operand(b + q * 32, 16, 1024),
                        mx4_shape(kTileM, kTileN, (q & 1) * 2, (q & 1) * 2), ta + (q >> 1) * 4, tb + (q >> 1) * 4,
                        k > 0 || q > 0);
            tc_commit(smem_addr(&s_free[st]));
        }
        tc_commit(smem_addr(&s_done));
    }
    __syncwarp();
    mbar_wait(smem_addr(&s_done), 0, &s_failed);
    __syncwarp();
    fence_after_sync();

    // the tile through shared memory (the stages are free), so that a warp writes neighbours of a row
    constexpr int kPad = kTileN + 1;
    float* s_c = reinterpret_cast<float*>(smem);
    const int row = warp * 32 + lane;
#pragma unroll 1
    for (int q = 0; q < kTileN / 32; ++q) {
        uint32_t acc[32];
        tmem_load32(tmem + ((uint32_t)(warp * 32) << 16) + q * 32, acc);
#pragma unroll
        for (int j = 0; j < 32; ++j) s_c[row * kPad + q * 32 + j] = __uint_as_float(acc[j]);
    }
    fence_before_sync();
    __syncthreads();
    if (!s_failed) {
        const int64_t r0 = (int64_t)ti * kTileM, c0 = (int64_t)tj * kTileN;
        for (int r = warp; r < kTileM && r0 + r < A.m; r += kThreads / 32) {
#pragma unroll
            for (int j = 0; j < kTileN / 32; ++j) {
                const int64_t col = c0 + j * 32 + lane;
                if (col >= A.n) continue;
                const int64_t at = (r0 + r) * A.ldc + col;
                float v = s_c[r * kPad + j * 32 + lane];
                if (A.add) v += read_c(A.c, A.type, at);
                write_c(A.c, A.type, at, v);
            }
        }
    }
    if (threadIdx.x == 0 && s_failed) atomicAdd(A.timeouts, 1);
    if (warp == 0) tmem_free(tmem, kTmemColumns);
}

// ---------------------------------------------------------------------------------------------- host side

// Codes: boxes of 128 bytes x `box` rows, swizzled, zeros outside.
static bool code_map(CUtensorMap* map, const uint8_t* codes, int64_t rows, int64_t k, int box) {
    const int64_t pitch = blocks_of(k) * 16;
    return sidco_internal::byte_map(map, codes, pitch, rows, pitch, 128, box, true);
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
    const int64_t tiles_m = (m + kTileM - 1) / kTileM, tiles_n = (n + kTileN - 1) / kTileN;
    if (tiles_m * tiles_n > 0x7fffffff) return SIDCO_E_SIZE;
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e;
    if (k == 0) {                            // an empty sum
        if (add) return 0;
        return (int)cudaMemset2DAsync(c, ldc * size, 0, n * size, m, s);
    }
    static bool ready[64] = {};
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return (int)e;
    if (dev < 0 || dev >= 64) return SIDCO_E_SIZE;
    if (!ready[dev]) {                       // (setting it twice from two threads is harmless)
        if ((e = cudaFuncSetAttribute(matmul_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem)) != cudaSuccess)
            return (int)e;
        ready[dev] = true;
    }
    Args a{a_scales, b_scales, m, n, k, (blocks_of(k) + 3) / 4, c, ldc, c_type, add != 0, (int)tiles_n, nullptr};
    if ((e = cudaGetSymbolAddress((void**)&a.timeouts, g_timeouts)) != cudaSuccess) return (int)e;
    CUtensorMap map_a, map_b;
    if (!code_map(&map_a, a_codes, m, k, kTileM) || !code_map(&map_b, b_codes, n, k, kTileN)) return SIDCO_E_UNSUPPORTED;
    matmul_kernel<<<(unsigned)(tiles_m * tiles_n), kThreads, kSmem, s>>>(map_a, map_b, a);
    if ((e = cudaGetLastError()) != cudaSuccess) return (int)e;
    sidco_internal::note_launch();
    return 0;
}

int sidco_wait_timeouts(void) {
    int a = 0, b = 0, rc;
    if ((rc = sidco_internal::orthogonalize_timeouts(&a)) || (rc = sidco_internal::mx4_matmul_timeouts(&b)))
        return rc > 0 ? -rc : rc;
    return a + b;
}

}  // extern "C"
