// Quantising to microscaled 4-bit blocks and reading them back (formulas and layout: sidco_mx4.cuh), for sm_100a.
//
//   quantize_kernel    matrix -> codes and scales along its rows and / or of its transpose, from one read
//   dequantize_kernel  the values of a quantised matrix
//   compress_kernel    error-compensated quantisation of a flat gradient: acc = g + r, codes of acc, r <- acc - value
//   mean_kernel        dense mean of N workers' gathered codes
//
// A lane holds eight neighbours (its codes are one word), four lanes hold a block; one four-lane maximum and a few
// conversions per eight elements.  Measured (share of the copy rate of 6549 GB/s on the bytes that have to move):
//   compress  25.6 M bf16 gradients: 42 us, 269 MB, 0.98: bound by memory
//   mean      8 x 25.6 M: 38 us, 211 MB, 0.84: four fifths of the issue slots are busy with conversions and sums
//   quantize  10000 x 1500 fp32, both forms: 17 us, 76 MB, 0.68: bound by neither memory nor issue (0.6 of the slots): a CTA
//             loads, then converts both forms, and has no other loads under way meanwhile
//   reading one form of it back to bf16: 9 us, 38 MB, 0.65: three quarters of the issue slots are busy with conversions
// Small calls take 3 to 4 us on the device, less than the host needs to launch them; every kernel may be set up under the
// end of the one before.
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sidco.h"
#include "sidco_internal.h"
#include "sidco_mx4.cuh"
#include "sidco_tc.cuh"

namespace sidco_mx4 {

constexpr unsigned kFull = 0xffffffffu;

// (every kernel is set up under the end of the kernel before it, and waits for that one here)
__device__ __forceinline__ void begin() {
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
}

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half narrow<__half>(float x) { return __float2half_rn(x); }

// Eight neighbours in accesses of W bytes (the widest that the addresses allow: see width_of): 32-byte accesses of fp32
// move whole sectors per lane, two 16-byte ones half a sector each.
template <int W> struct Word;
template <> struct Word<2> { using type = uint16_t; };
template <> struct Word<4> { using type = uint32_t; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<16> { using type = uint4; };

template <typename T, int W>
__device__ __forceinline__ void move_in(const T* p, uint32_t* w) {
    if constexpr (W == 32) {
        asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                     : "l"(p));
    } else {
        using V = typename Word<W>::type;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) * 8 / W; ++i) reinterpret_cast<V*>(w)[i] = reinterpret_cast<const V*>(p)[i];
    }
}

template <typename T, int W>
__device__ __forceinline__ void move_out(T* p, const uint32_t* w) {
    if constexpr (W == 32) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                     "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        using V = typename Word<W>::type;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) * 8 / W; ++i) reinterpret_cast<V*>(p)[i] = reinterpret_cast<const V*>(w)[i];
    }
}

// The first n of eight neighbours, zeros behind them.
template <typename T, int W>
__device__ __forceinline__ void load8(const T* p, int n, float (&x)[8]) {
    if (n >= 8) {
        alignas(16) uint32_t w[2 * sizeof(T)];
        move_in<T, W>(p, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = widen(reinterpret_cast<const T*>(w)[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? widen(p[i]) : 0.0f;
}

template <typename T, int W>
__device__ __forceinline__ void store8(T* p, int n, const float (&x)[8]) {
    if (n >= 8) {
        alignas(16) uint32_t w[2 * sizeof(T)];
#pragma unroll
        for (int i = 0; i < 8; ++i) reinterpret_cast<T*>(w)[i] = narrow<T>(x[i]);
        move_out<T, W>(p, w);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = narrow<T>(x[i]);
}

__device__ __forceinline__ uint32_t max8(const float (&x)[8]) {
    uint32_t m = magnitude_bits(x[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = max(m, magnitude_bits(x[i]));
    return m;
}

// Largest magnitude over the four lanes of a block.
__device__ __forceinline__ uint32_t block_max(uint32_t m) {
    m = max(m, __shfl_xor_sync(kFull, m, 1));
    return max(m, __shfl_xor_sync(kFull, m, 2));
}

__device__ __forceinline__ uint32_t encode(const float (&x)[8], uint32_t byte) {
    const uint32_t c = encode8(x, inverse_scale_of(byte));
    return byte == 255u ? 0u : c;
}

// ------------------------------------------------------------------------------------------------ matrices

constexpr int kQuantThreads = 256;
constexpr int kQuantRows = 64, kQuantCols = 128;      // elements of a CTA: half a tile of scales in either direction
constexpr int kQuantSmem = (kQuantRows * kQuantCols + 16) * (int)sizeof(float);

struct QuantArgs {
    const void* x;
    int64_t rows, cols, ld;
    uint8_t *codes, *scales, *codes_t, *scales_t;
    int64_t pitch, pitch_t;           // bytes of a row of codes
    int64_t ktiles, ktiles_t;         // scale tiles along a row
    int64_t tiles_c;                  // CTA tiles along the columns
};

// Rows are quantised as they are loaded (four lanes of a warp hold a block); for the transpose the tile goes through
// shared memory, where one thread then reads 32 elements of a column.  The second 32 rows start 16 words later, so that
// the lanes of a warp (16 columns x 2 blocks) read from 32 different banks.  (128 x 128 tiles were no faster for large
// matrices and have half the CTAs for small ones.)
template <typename T, int W>
__global__ void __launch_bounds__(kQuantThreads) quantize_kernel(const QuantArgs A) {
    extern __shared__ float s_x[];                                   // [64][128], skewed; only with codes_t
    __shared__ __align__(16) uint8_t s_scale[kQuantRows * 4];
    begin();
    const int64_t r0 = (int64_t)(blockIdx.x / A.tiles_c) * kQuantRows, c0 = (int64_t)(blockIdx.x % A.tiles_c) * kQuantCols;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int oct = lane & 15;                                       // which eight columns
    const int64_t c = c0 + oct * 8;
    const int left = (int)min((int64_t)8, A.cols - c);               // may be <= 0
    float x[4][8];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int64_t r = r0 + p * 16 + warp * 2 + (lane >> 4);
        const bool in = r < A.rows && left > 0;
        load8<T, W>(in ? (const T*)A.x + r * A.ld + c : (const T*)A.x, in ? left : 0, x[p]);
    }
    if (A.codes_t) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            float* at = s_x + (p * 16 + warp * 2 + (lane >> 4)) * kQuantCols + (p >> 1) * 16 + oct * 8;
            // (every other four lanes write their second half first: eight lanes then cover all banks)
            const int swap = (lane >> 2) & 1;
            const float4 lo = make_float4(x[p][0], x[p][1], x[p][2], x[p][3]), hi = make_float4(x[p][4], x[p][5], x[p][6], x[p][7]);
            reinterpret_cast<float4*>(at)[swap] = swap ? hi : lo;
            reinterpret_cast<float4*>(at)[swap ^ 1] = swap ? lo : hi;
        }
    }
    if (A.codes) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int rt = p * 16 + warp * 2 + (lane >> 4);
            const int64_t r = r0 + rt;
            const uint32_t byte = scale_byte(block_max(max8(x[p])));
            // (rows and columns behind the matrix hold zeros, so that the unused bytes of a scale tile become 0)
            if ((lane & 3) == 0) s_scale[rt * 4 + (oct >> 2)] = (uint8_t)byte;
            if (r < A.rows && c - (oct & 3) * 8 < A.cols)            // the last block is written whole
                *reinterpret_cast<uint32_t*>(A.codes + r * A.pitch + (c >> 1)) = encode(x[p], byte);
        }
    }
    __syncthreads();
    if (A.codes && threadIdx.x < kQuantRows)                          // the four blocks of a row
        *reinterpret_cast<uint32_t*>(A.scales + ((r0 / kTileRows) * A.ktiles + c0 / kQuantCols) * kTileBytes +
                                     scale_in_tile((int)(r0 & 64) + threadIdx.x, 0)) =
            *reinterpret_cast<const uint32_t*>(s_scale + threadIdx.x * 4);
    if (!A.codes_t) return;
    const int col = warp * 16 + (lane & 15), g = lane >> 4;          // a column and one of its two blocks
    const float* from = s_x + g * (32 * kQuantCols + 16) + col;
    float y[4][8];
#pragma unroll
    for (int i = 0; i < 32; ++i) y[i >> 3][i & 7] = from[i * kQuantCols];
    const uint32_t byte = scale_byte(max(max(max8(y[0]), max8(y[1])), max(max8(y[2]), max8(y[3]))));
    const uint4 codes = make_uint4(encode(y[0], byte), encode(y[1], byte), encode(y[2], byte), encode(y[3], byte));
    if (c0 + col < A.cols && r0 + g * 32 < A.rows)
        *reinterpret_cast<uint4*>(A.codes_t + (c0 + col) * A.pitch_t + (r0 + g * 32) / 2) = codes;
    const uint32_t other = __shfl_down_sync(kFull, byte, 16);        // the scales of a column's two blocks together
    if (g == 0)
        *reinterpret_cast<uint16_t*>(A.scales_t + ((c0 / kTileRows) * A.ktiles_t + r0 / kTileRows) * kTileBytes +
                                     scale_in_tile(col, (int)(r0 & 64) / kBlock)) = (uint16_t)(byte | other << 8);
}

// A lane reads a word of codes and writes eight values, U times; 2^log2_lanes lanes work on a row, `parts` CTAs along it.
// (Sixteen values per lane halve the instructions for codes and scales, but its two stores then leave gaps between the
// lanes' 16 bytes: 12 to 18 us instead of 9.)
constexpr int kDequantU = 2;

template <typename T, int W>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* codes,
                                                         const uint8_t* scales, int rows, int cols,
                                                         int64_t pitch, int64_t ktiles, T* __restrict__ out, int64_t ld,
                                                         int octs, int log2_lanes, int parts) {
    begin();
    const int lanes = 1 << log2_lanes, group = blockIdx.x / parts, part = blockIdx.x - group * parts;
    const int r = group * (256 >> log2_lanes) + (threadIdx.x >> log2_lanes);
    if (r >= rows) return;
    const uint32_t* from = reinterpret_cast<const uint32_t*>(codes + r * pitch);
    const uint8_t* scale = scales + (r / kTileRows) * ktiles * kTileBytes + scale_in_tile(r % kTileRows, 0);
    T* to = out + r * ld;
    const int o0 = part * (lanes * kDequantU) + (threadIdx.x & (lanes - 1));
    uint32_t c[kDequantU], b[kDequantU];
#pragma unroll
    for (int u = 0; u < kDequantU; ++u) {
        const int o = o0 + u * lanes;
        c[u] = o < octs ? from[o] : 0u;
        b[u] = o < octs ? scale[scale_of_oct(o)] : 0u;
    }
#pragma unroll
    for (int u = 0; u < kDequantU; ++u) {
        const int o = o0 + u * lanes;
        if (o >= octs) break;
        const float s = scale_of(b[u]);
        float v[8];
        decode8(c[u], v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= s;
        store8<T, W>(to + o * 8, min(8, cols - o * 8), v);
    }
}

// ------------------------------------------------------------------------------------------------ flat vectors

template <typename T, int W, int WR, int U>
__global__ void __launch_bounds__(256) compress_kernel(const T* grad, float* __restrict__ residual,
                                                       int64_t d, uint8_t* __restrict__ codes,
                                                       uint8_t* __restrict__ scales) {
    begin();
    const int64_t first = (int64_t)blockIdx.x * (256 * U) + threadIdx.x;
    const int64_t octs = blocks_of(d) * 4;                            // whole blocks
    float g[U][8], r[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t at = (first + u * 256) * 8;
        const int n = (int)max((int64_t)0, min((int64_t)8, d - at));
        load8<T, W>(n ? grad + at : grad, n, g[u]);
        load8<float, WR>(n ? residual + at : residual, n, r[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t o = first + u * 256, at = o * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) g[u][k] += r[u][k];               // one fp32 addition
        const uint32_t byte = scale_byte(block_max(max8(g[u])));
        const uint32_t c = encode(g[u], byte);
        if (o >= octs) continue;
        *reinterpret_cast<uint32_t*>(codes + o * 4) = c;
        if ((threadIdx.x & 3) == 0) scales[o >> 2] = (uint8_t)byte;
        float v[8];
        decode8(c, v);
        const float s = scale_of(byte);
#pragma unroll
        for (int k = 0; k < 8; ++k) g[u][k] = fmaf(-v[k], s, g[u][k]);   // v s is exact: one rounding
        const int n = (int)max((int64_t)0, min((int64_t)8, d - at));
        if (n) store8<float, WR>(residual + at, n, g[u]);
    }
}

// The workers are added in their order, in fp32 (a decoded value has two significant bits), then scaled by 1/N.  A thread
// takes half a block (one 8-byte load of codes and one scale for sixteen values: the kernel is bound by its instructions,
// eight values per scale took 49 us where sixteen take 38) and loads those of A workers before it uses any.
template <int W, int A>
__global__ void __launch_bounds__(256) mean_kernel(const uint8_t* codes, const uint8_t* scales,
                                                   int n_workers, int64_t d, float* __restrict__ out) {
    begin();
    const int64_t nb = blocks_of(d), h = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (h >= nb * 2) return;
    const uint2* cp = reinterpret_cast<const uint2*>(codes) + h;
    const uint8_t* sp = scales + (h >> 1);
    float sum[2][8] = {};
    for (int w0 = 0; w0 < n_workers; w0 += A) {
        uint2 c[A];
        uint32_t b[A];
#pragma unroll
        for (int i = 0; i < A; ++i) {
            const bool on = w0 + i < n_workers;
            c[i] = on ? cp[(w0 + i) * nb * 2] : make_uint2(0, 0);
            b[i] = on ? sp[(w0 + i) * nb] : 0u;
        }
#pragma unroll
        for (int i = 0; i < A; ++i) {
            const float s = scale_of(b[i]);
            float v[8];
            decode8(c[i].x, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[0][k] = fmaf(v[k], s, sum[0][k]);           // (+ 0 behind the last worker)
            decode8(c[i].y, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[1][k] = fmaf(v[k], s, sum[1][k]);
        }
    }
    const float inv = 1.0f / (float)n_workers;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int64_t at = h * 16 + u * 8;
        if (at >= d) break;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[u][k] *= inv;
        store8<float, W>(out + at, (int)min((int64_t)8, d - at), sum[u]);
    }
}

// ------------------------------------------------------------------------------------------------ host side

static bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

template <typename... P, typename... Q>
static int launch(void (*kernel)(P...), int64_t grid, int threads, size_t smem, cudaStream_t stream, Q... args) {
    if (grid > 0x7fffffff) return SIDCO_E_SIZE;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
    if (e != cudaSuccess) return (int)e;
    sidco_internal::note_launch();
    return 0;
}

// Widest access (at most `most` bytes) with which every row of 8-element groups can be moved.
static int width_of(const void* p, int64_t row_bytes, int most, int element) {
    int w = most;
    while (w > element && (!aligned(p, w) || row_bytes % w)) w /= 2;
    return w;
}

template <typename T, int W>
static int launch_quantize(const QuantArgs& a, int64_t grid, cudaStream_t s) {
    return launch(quantize_kernel<T, W>, grid, kQuantThreads, a.codes_t ? kQuantSmem : 0, s, a);
}

template <typename T>
static int quantize_typed(const QuantArgs& a, int64_t grid, cudaStream_t s) {
    switch (width_of(a.x, a.ld * sizeof(T), 16, sizeof(T))) {
        case 16: return launch_quantize<T, 16>(a, grid, s);
        case 8: return launch_quantize<T, 8>(a, grid, s);
        default: return launch_quantize<T, sizeof(T)>(a, grid, s);
    }
}

template <typename T>
static int dequantize_typed(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out, int64_t ld,
                            cudaStream_t s) {
    const int64_t octs = (cols + 7) / 8, pitch = blocks_of(cols) * 16, ktiles = (blocks_of(cols) + 3) / 4;
    int log2_lanes = 0;                                               // lanes of a row: a warp, fewer for short rows
    while (log2_lanes < 5 && (1 << log2_lanes) < octs) ++log2_lanes;
    const int64_t per_cta = 256 >> log2_lanes, along = kDequantU << log2_lanes, parts = (octs + along - 1) / along;
    const auto go = [&](auto kernel) {
        return launch(kernel, (rows + per_cta - 1) / per_cta * parts, 256, 0, s, codes, scales, rows, cols, pitch, ktiles,
                      (T*)out, ld, octs, log2_lanes, parts);
    };
    switch (width_of(out, ld * sizeof(T), 16, sizeof(T))) {
        case 16: return go(dequantize_kernel<T, 16>);
        case 8: return go(dequantize_kernel<T, 8>);
        default: return go(dequantize_kernel<T, sizeof(T)>);
    }
}

template <typename T>
static int compress_typed(const void* grad, float* residual, int64_t d, uint8_t* codes, uint8_t* scales, cudaStream_t s) {
    constexpr int U = 2, kMost = sizeof(T) * 8, kLeast = sizeof(T);
    const int64_t grid = (blocks_of(d) * 4 + 256 * U - 1) / (256 * U);
    if (aligned(grad, kMost) && aligned(residual, 32))
        return launch(compress_kernel<T, kMost, 32, U>, grid, 256, 0, s, (const T*)grad, residual, d, codes, scales);
    return launch(compress_kernel<T, kLeast, 4, U>, grid, 256, 0, s, (const T*)grad, residual, d, codes, scales);
}

constexpr int64_t kMaxDim = ((int64_t)1 << 31) - ((int64_t)1 << 16);

}  // namespace sidco_mx4

extern "C" {

int64_t sidco_mx4_code_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || rows > sidco_mx4::kMaxDim || cols > sidco_mx4::kMaxDim) return SIDCO_E_SIZE;
    return rows * sidco_mx4::blocks_of(cols) * 16;
}

int64_t sidco_mx4_scale_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || rows > sidco_mx4::kMaxDim || cols > sidco_mx4::kMaxDim) return SIDCO_E_SIZE;
    return (rows + 127) / 128 * ((sidco_mx4::blocks_of(cols) + 3) / 4) * sidco_mx4::kTileBytes;
}

int sidco_mx4_quantize(const void* x, int x_type, int64_t rows, int64_t cols, int64_t ld, uint8_t* codes, uint8_t* scales,
                       uint8_t* codes_t, uint8_t* scales_t, void* stream) {
    using namespace sidco_mx4;
    if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return SIDCO_E_SIZE;
    if (x_type < SIDCO_T_F32 || x_type > SIDCO_T_F16) return SIDCO_E_TYPE;
    if (ld < cols) return SIDCO_E_PARAMS;
    if (rows == 0 || cols == 0) return 0;
    if (!x || (!codes && !codes_t) || !codes != !scales || !codes_t != !scales_t) return SIDCO_E_NULL;
    const size_t size = x_type == SIDCO_T_F32 ? 4 : 2;
    if (!aligned(x, size) || !aligned(codes, 16) || !aligned(scales, 16) || !aligned(codes_t, 16) || !aligned(scales_t, 16))
        return SIDCO_E_ALIGN;
    QuantArgs a{x, rows, cols, ld, codes, scales, codes_t, scales_t, blocks_of(cols) * 16, blocks_of(rows) * 16,
                (blocks_of(cols) + 3) / 4, (blocks_of(rows) + 3) / 4, (cols + kQuantCols - 1) / kQuantCols};
    const int64_t grid = (rows + kTileRows - 1) / kTileRows * (kTileRows / kQuantRows) * a.tiles_c;
    if (grid > 0x7fffffff) return SIDCO_E_SIZE;
    cudaStream_t s = (cudaStream_t)stream;
    if (x_type == SIDCO_T_F32) return quantize_typed<float>(a, grid, s);
    if (x_type == SIDCO_T_BF16) return quantize_typed<__nv_bfloat16>(a, grid, s);
    return quantize_typed<__half>(a, grid, s);
}

int sidco_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out, int out_type,
                         int64_t ld, void* stream) {
    using namespace sidco_mx4;
    if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return SIDCO_E_SIZE;
    if (out_type < SIDCO_T_F32 || out_type > SIDCO_T_F16) return SIDCO_E_TYPE;
    if (ld < cols) return SIDCO_E_PARAMS;
    if (rows == 0 || cols == 0) return 0;
    if (!codes || !scales || !out) return SIDCO_E_NULL;
    if (!aligned(codes, 16) || !aligned(scales, 16) || !aligned(out, out_type == SIDCO_T_F32 ? 4 : 2)) return SIDCO_E_ALIGN;
    cudaStream_t s = (cudaStream_t)stream;
    if (out_type == SIDCO_T_F32) return dequantize_typed<float>(codes, scales, rows, cols, out, ld, s);
    if (out_type == SIDCO_T_BF16) return dequantize_typed<__nv_bfloat16>(codes, scales, rows, cols, out, ld, s);
    return dequantize_typed<__half>(codes, scales, rows, cols, out, ld, s);
}

int sidco_mx4_compress(const void* grad, int grad_type, float* residual, int64_t d, uint8_t* codes, uint8_t* scales,
                       void* stream) {
    using namespace sidco_mx4;
    if (d < 0 || d > kMaxDim) return SIDCO_E_SIZE;
    if (grad_type < SIDCO_T_F32 || grad_type > SIDCO_T_F16) return SIDCO_E_TYPE;
    if (d == 0) return 0;
    if (!grad || !residual || !codes || !scales) return SIDCO_E_NULL;
    const uintptr_t size = grad_type == SIDCO_T_F32 ? 4 : 2;
    if (!aligned(grad, size) || !aligned(residual, 4) || !aligned(codes, 16)) return SIDCO_E_ALIGN;
    const uintptr_t g = (uintptr_t)grad, r = (uintptr_t)residual;
    if (g < r + (uintptr_t)d * 4 && r < g + (uintptr_t)d * size) return SIDCO_E_ALIAS;
    cudaStream_t s = (cudaStream_t)stream;
    if (grad_type == SIDCO_T_F32) return compress_typed<float>(grad, residual, d, codes, scales, s);
    if (grad_type == SIDCO_T_BF16) return compress_typed<__nv_bfloat16>(grad, residual, d, codes, scales, s);
    return compress_typed<__half>(grad, residual, d, codes, scales, s);
}

int sidco_mx4_mean(const uint8_t* codes_all, const uint8_t* scales_all, int n_workers, int64_t d, float* out_dense,
                   void* stream) {
    using namespace sidco_mx4;
    if (n_workers < 1 || n_workers > SIDCO_AGG_MAX_WORKERS) return SIDCO_E_PARAMS;
    if (d < 0 || d > kMaxDim) return SIDCO_E_SIZE;
    if (d == 0) return 0;
    if (!codes_all || !scales_all || !out_dense) return SIDCO_E_NULL;
    if (!aligned(codes_all, 16) || !aligned(out_dense, 4)) return SIDCO_E_ALIGN;
    cudaStream_t s = (cudaStream_t)stream;
    const auto go = [&](auto kernel) {
        return launch(kernel, (blocks_of(d) * 2 + 255) / 256, 256, 0, s, codes_all, scales_all, n_workers, d, out_dense);
    };
    if (!aligned(out_dense, 32)) return go(mean_kernel<4, 4>);
    return n_workers == 1 ? go(mean_kernel<32, 1>) : n_workers == 2 ? go(mean_kernel<32, 2>) : go(mean_kernel<32, 4>);
}

}  // extern "C"
