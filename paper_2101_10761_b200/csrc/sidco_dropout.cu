// Dropout from a counter-based generator: y = keep ? x / (1 - p) : 0, plus a residual.  The mask is a function of the
// element's index, the seed and the number of the call, so that the backward pass is the same kernel on dy and nothing is
// stored.  Bound by memory: reads x (and the residual), writes y.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/sidco.h"
#include "sidco_elements.cuh"
#include "sidco_internal.h"
#include "sidco_tc.cuh"

namespace sidco_dropout_impl {

using namespace sidco_elements;

constexpr int kThreads = 256;

// kEach elements as they lie: 16 bytes, or four single ones.
template <typename T, bool kVector> struct Few {
    static constexpr int kEach = kVector ? 16 / (int)sizeof(T) : 4;
    alignas(16) T t[kEach];
    __device__ __forceinline__ void read(const T* p, int64_t left) {
        if (kVector && left >= kEach) {
            *reinterpret_cast<uint4*>(t) = *reinterpret_cast<const uint4*>(p);
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j) t[j] = j < left ? p[j] : narrow<T>(0.0f);
        }
    }
    __device__ __forceinline__ void write(T* p, int64_t left) const {
        if (kVector && left >= kEach) {
            *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(t);
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                if (j < left) p[j] = t[j];
        }
    }
};

// Two times kEach elements per thread, kept as they lie while the words are drawn.  With dropout the generator's products
// bound this, not memory: 67 M bf16 elements take 68 us without a residual and 71 us with one (41 and 59 us with nothing to draw).
template <typename T, bool kDrop, bool kVector, bool kResidual>
__global__ void __launch_bounds__(kThreads)
    dropout_kernel(const T* x, const T* residual, T* out, int64_t n, const Dropout d) {
    constexpr int kEach = Few<T, kVector>::kEach, kSpan = kThreads * kEach, kTimes = 2;
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const uint64_t call = kDrop ? call_of(d) : 0;
    Few<T, kVector> a[kTimes], r[kTimes];
    const int64_t first = (int64_t)blockIdx.x * kTimes * kSpan + threadIdx.x * kEach;
#pragma unroll
    for (int k = 0; k < kTimes; ++k) {
        const int64_t i = first + k * kSpan;
        if (i < n) a[k].read(x + i, n - i);
        if (kResidual && i < n) r[k].read(residual + i, n - i);
    }
#pragma unroll
    for (int k = 0; k < kTimes; ++k) {
        const int64_t i = first + k * kSpan;
        // (a span's elements lie in one aligned power of two: the high word of their blocks is the span's)
        const uint64_t base = ((uint64_t)blockIdx.x * kTimes + k) * (kSpan / 4);
        uint32_t w[kEach / 4][4];
        if (kDrop) random_blocks(d, call, (uint32_t)base + threadIdx.x * (kEach / 4), (uint32_t)(base >> 32), w);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const float v = widen(a[k].t[j]), add = kResidual ? widen(r[k].t[j]) : 0.0f;
            float y = v;
            if (kDrop && kResidual) y = dropped(d, w[j / 4][j % 4]) ? add : fmaf(v, d.factor, add);
            else if (kDrop) y = dropped(d, w[j / 4][j % 4]) ? 0.0f : v * d.factor;
            else if (kResidual) y = v + add;
            a[k].t[j] = narrow<T>(y);
        }
        if (i < n) a[k].write(out + i, n - i);
    }
}

template <typename T, bool kVector>
__global__ void __launch_bounds__(kThreads) scale_gradient_kernel(T* x, int64_t n, const float* factor) {
    constexpr int kEach = Few<T, kVector>::kEach;
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const float f = *factor;
    if (f == 1.0f) return;
    for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kEach; i < n; i += (int64_t)gridDim.x * kThreads * kEach) {
        Few<T, kVector> a;
        a.read(x + i, n - i);
#pragma unroll
        for (int j = 0; j < kEach; ++j) a.t[j] = narrow<T>(widen(a.t[j]) * f);
        a.write(x + i, n - i);
    }
}

// Four at a time from fp32 to another type; reads and writes everything once, whatever the factor.
template <typename T, bool kVector>
__global__ void __launch_bounds__(kThreads) round_gradient_kernel(const float* x, int64_t n, const float* factor, T* out) {
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const float f = *factor;
    for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * kThreads * 4) {
        float v[4];
        if (kVector && i + 4 <= n) {
            load(x + i, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] *= f;
            store(out + i, v);
        } else {
            for (int j = 0; j < 4 && i + j < n; ++j) out[i + j] = narrow<T>(x[i + j] * f);
        }
    }
}

}  // namespace sidco_dropout_impl

extern "C" {

int sidco_scale_gradient(void* x, int type, int64_t n, const float* factor, void* stream) {
    using namespace sidco_dropout_impl;
    if (n < 0 || n > ((int64_t)1 << 40)) return SIDCO_E_SIZE;
    if (type < SIDCO_T_F32 || type > SIDCO_T_F16) return SIDCO_E_TYPE;
    if (n == 0) return 0;
    if (!x || !factor) return SIDCO_E_NULL;
    if ((uintptr_t)x % size_of(type) || (uintptr_t)factor % 4) return SIDCO_E_ALIGN;
    if (overlap(x, n * size_of(type), factor, 4)) return SIDCO_E_ALIAS;
    // (few CTAs: the usual factor is one, and then they only have to end)
    const int64_t blocks = std::min<int64_t>((n + 8 * kThreads - 1) / (8 * kThreads), 148 * 8);
    const int rc = with_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return (int)launch((uintptr_t)x % 16 ? scale_gradient_kernel<T, false> : scale_gradient_kernel<T, true>, dim3((unsigned)blocks),
                           kThreads, 0, (cudaStream_t)stream, 1, (T*)x, n, factor);
    });
    if (rc == 0) sidco_internal::note_launch();
    return rc;
}

int sidco_round_gradient(const float* x, int64_t n, const float* factor, void* out, int type, void* stream) {
    using namespace sidco_dropout_impl;
    if (n < 0 || n > ((int64_t)1 << 40)) return SIDCO_E_SIZE;
    if (type < SIDCO_T_F32 || type > SIDCO_T_F16) return SIDCO_E_TYPE;
    if (n == 0) return 0;
    if (!x || !factor || !out) return SIDCO_E_NULL;
    if ((uintptr_t)x % 4 || (uintptr_t)factor % 4 || (uintptr_t)out % size_of(type)) return SIDCO_E_ALIGN;
    if (overlap(out, n * size_of(type), x, n * 4) || overlap(out, n * size_of(type), factor, 4)) return SIDCO_E_ALIAS;
    const int64_t blocks = std::min<int64_t>((n + 8 * kThreads - 1) / (8 * kThreads), 148 * 8);
    const int rc = with_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const bool vector = (uintptr_t)x % 16 == 0 && (uintptr_t)out % (4 * sizeof(T)) == 0;
        return (int)launch(vector ? round_gradient_kernel<T, true> : round_gradient_kernel<T, false>, dim3((unsigned)blocks), kThreads,
                           0, (cudaStream_t)stream, 1, x, n, factor, (T*)out);
    });
    if (rc == 0) sidco_internal::note_launch();
    return rc;
}

int sidco_dropout(const void* x, int type, int64_t n, float p, uint64_t seed, uint64_t call,
                             const uint64_t* step, const void* residual, void* out, void* stream) {
    using namespace sidco_dropout_impl;
    if (n < 0 || n > ((int64_t)1 << 40)) return SIDCO_E_SIZE;
    if (type < SIDCO_T_F32 || type > SIDCO_T_F16) return SIDCO_E_TYPE;
    Dropout d;
    bool on;
    if (const int rc = make_dropout(p, seed, call, step, &d, &on)) return rc;
    if (n == 0) return 0;
    if (!x || !out) return SIDCO_E_NULL;
    const int64_t bytes = n * size_of(type);
    if (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)out) % (uintptr_t)size_of(type)) return SIDCO_E_ALIGN;
    if ((x != out && overlap(x, bytes, out, bytes)) || (residual != out && overlap(residual, bytes, out, bytes)))
        return SIDCO_E_ALIAS;
    const bool vector = ((uintptr_t)x | (uintptr_t)residual | (uintptr_t)out) % 16 == 0;
    const int rc = with_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const auto go = [&](auto kernel, int each) {
            const int64_t per = 2 * kThreads * each;
            return (int)launch(kernel, dim3((unsigned)((n + per - 1) / per)), kThreads, 0, (cudaStream_t)stream, 1, (const T*)x,
                               (const T*)residual, (T*)out, n, d);
        };
        constexpr int kWide = Few<T, true>::kEach, kNarrow = Few<T, false>::kEach;
        if (residual)
            return on ? vector ? go(dropout_kernel<T, true, true, true>, kWide) : go(dropout_kernel<T, true, false, true>, kNarrow)
                      : vector ? go(dropout_kernel<T, false, true, true>, kWide) : go(dropout_kernel<T, false, false, true>, kNarrow);
        return on ? vector ? go(dropout_kernel<T, true, true, false>, kWide) : go(dropout_kernel<T, true, false, false>, kNarrow)
                  : vector ? go(dropout_kernel<T, false, true, false>, kWide) : go(dropout_kernel<T, false, false, false>, kNarrow);
    });
    if (rc == 0) sidco_internal::note_launch();
    return rc;
}

}  // extern "C"
