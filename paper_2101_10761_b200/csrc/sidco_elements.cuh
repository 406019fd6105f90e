// What the operators on rows of elements share: conversions of the element types, accesses of several neighbours, the
// counter-based generator of the dropout, and launches.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sidco.h"

namespace sidco_elements {

// ---------------------------------------------------------------------------------------------- elements

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half narrow<__half>(float x) { return __float2half_rn(x); }

// N neighbours (4 or 8) from an address aligned to 16 bytes or to their size, whichever is less.
template <int N, typename T> __device__ __forceinline__ void load(const T* p, float (&v)[N]) {
    alignas(16) T t[N];
    constexpr int kBytes = N * (int)sizeof(T);
    if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(t) = *reinterpret_cast<const uint2*>(p);
    else
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4*>(t)[i] = reinterpret_cast<const uint4*>(p)[i];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = widen(t[i]);
}

template <int N, typename T> __device__ __forceinline__ void store(T* p, const float (&v)[N]) {
    alignas(16) T t[N];
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = narrow<T>(v[i]);
    constexpr int kBytes = N * (int)sizeof(T);
    if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(t);
    else
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(t)[i];
}

// N words that start `shift` bytes (even, below 16) into w.
template <int N> __device__ __forceinline__ void shift_words(uint32_t (&w)[N + 4], int shift) {
    if (shift & 4) {
#pragma unroll
        for (int i = 0; i < N + 3; ++i) w[i] = w[i + 1];
    }
    if (shift & 8) {
#pragma unroll
        for (int i = 0; i < N + 2; ++i) w[i] = w[i + 2];
    }
    const int bits = (shift & 2) * 8;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], bits);
}

constexpr int size_of(int type) { return type == SIDCO_T_F32 ? 4 : 2; }

// Whether `n` neighbours of a row that starts at p, with rows `ld` elements apart, can be accessed by load / store.
inline bool aligned(const void* p, int64_t ld, int type, int n) {
    const int64_t bytes = size_of(type) * n < 16 ? size_of(type) * n : 16;
    return (uintptr_t)p % (uintptr_t)bytes == 0 && ld * size_of(type) % bytes == 0;
}

inline bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
    return a && b && (uintptr_t)a < (uintptr_t)b + (uintptr_t)b_bytes && (uintptr_t)b < (uintptr_t)a + (uintptr_t)a_bytes;
}

// Bytes between the first element of the first row and the last of the last.
inline int64_t extent(int64_t rows, int64_t cols, int64_t ld, int type) {
    return rows && cols ? ((rows - 1) * ld + cols) * size_of(type) : 0;
}

// f(T*) for the element type.
template <typename F> int with_type(int type, F f) {
    switch (type) {
        case SIDCO_T_F32: return f((float*)nullptr);
        case SIDCO_T_BF16: return f((__nv_bfloat16*)nullptr);
        default: return f((__half*)nullptr);
    }
}

// A token or label: 32 or 64 bits.
__device__ __forceinline__ int64_t token_at(const void* tokens, bool wide, int64_t i) {
    return wide ? static_cast<const int64_t*>(tokens)[i] : static_cast<const int32_t*>(tokens)[i];
}

// ---------------------------------------------------------------------------------------------- dropout
//
// Words 4b .. 4b+3 belong to elements 4b .. 4b+3: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", 2011) of the counter (b, call) under the key `seed`: ten rounds of two 32 x 32 -> 64-bit products and two
// three-input xors per four elements.  The rounds' keys come from the host: added up in the kernel they took a fifth of its
// instructions.

struct Dropout {
    uint32_t key[10][2];              // of every round: the seed plus multiples of the generator's constants
    uint32_t last;                    // words up to this one drop (p = (last + 1) 2^-32)
    float factor;                     // 1 / (1 - p)
    uint64_t call;
    const uint64_t* step;             // device; added to call
};

__device__ __forceinline__ uint64_t call_of(const Dropout& d) { return d.step ? d.call + *d.step : d.call; }

// The words of N blocks; c[q][0] and c[q][1] hold their numbers.
template <int N> __device__ __forceinline__ void random_rounds(const Dropout& d, uint64_t call, uint32_t (&c)[N][4]) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
        c[q][2] = (uint32_t)call;
        c[q][3] = (uint32_t)(call >> 32);
    }
#pragma unroll
    for (int r = 0; r < 10; ++r)
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const uint64_t a = (uint64_t)c[q][0] * 0xD2511F53u, b = (uint64_t)c[q][2] * 0xCD9E8D57u;
            c[q][0] = (uint32_t)(b >> 32) ^ c[q][1] ^ d.key[r][0];
            c[q][2] = (uint32_t)(a >> 32) ^ c[q][3] ^ d.key[r][1];
            c[q][1] = (uint32_t)b;
            c[q][3] = (uint32_t)a;
        }
}

// Blocks (low, high), (low + 1, high) ..: they do not pass 2^32 in their low word.
template <int N>
__device__ __forceinline__ void random_blocks(const Dropout& d, uint64_t call, uint32_t low, uint32_t high, uint32_t (&c)[N][4]) {
#pragma unroll
    for (int q = 0; q < N; ++q) c[q][0] = low + q, c[q][1] = high;
    random_rounds(d, call, c);
}

// Any N blocks from `block` on.
template <int N> __device__ __forceinline__ void random_blocks(const Dropout& d, uint64_t call, uint64_t block, uint32_t (&c)[N][4]) {
#pragma unroll
    for (int q = 0; q < N; ++q) c[q][0] = (uint32_t)(block + q), c[q][1] = (uint32_t)((block + q) >> 32);
    random_rounds(d, call, c);
}

__device__ __forceinline__ bool dropped(const Dropout& d, uint32_t word) { return word <= d.last; }

// v of the N elements (a multiple of four) from element 4 * block on.  What is dropped becomes zero whatever it was.
template <int N> __device__ __forceinline__ void drop(const Dropout& d, uint64_t call, uint64_t block, float (&v)[N]) {
    uint32_t c[N / 4][4];
    random_blocks(d, call, block, c);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = dropped(d, c[i / 4][i % 4]) ? 0.0f : v[i] * d.factor;
}

// Checks p and fills d; *on: whether anything is dropped.
inline int make_dropout(float p, uint64_t seed, uint64_t call, const uint64_t* step, Dropout* d, bool* on) {
    if (!(p >= 0.0f && p <= 1.0f)) return SIDCO_E_PARAMS;
    if ((uintptr_t)step % 8) return SIDCO_E_ALIGN;
    const uint64_t words = (uint64_t)((double)p * 4294967296.0 + 0.5);
    *on = words > 0;
    for (uint32_t r = 0; r < 10; ++r) {
        d->key[r][0] = (uint32_t)seed + r * 0x9E3779B9u;
        d->key[r][1] = (uint32_t)(seed >> 32) + r * 0xBB67AE85u;
    }
    d->last = (uint32_t)(words - 1);
    d->factor = p < 1.0f ? (float)(1.0 / (1.0 - (double)p)) : 0.0f;
    d->call = call;
    d->step = step;
    return 0;
}

// ---------------------------------------------------------------------------------------------- launches

// A launch whose set-up may overlap the kernel before it in the stream (which it waits for itself).
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, int cluster, A&&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace sidco_elements
