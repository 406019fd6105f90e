// Dropout from a counter-based generator: y = keep ? x / (1 - p) : 0, plus a residual.  The mask is a function of the
// element's index, the seed and the number of the call, so that the backward pass is the same kernel on dy and nothing is
// stored.  Bound by memory: reads x (and the residual), writes y.
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sidco.h"
#include "sidco_elements.cuh"
#include "sidco_internal.h"
#include "sidco_tc.cuh"

namespace sidco_dropout_impl {

using namespace sidco_elements;

constexpr int kThreads = 256;

// kEach neighbours per thread: 32 bytes, or 16 where they cannot be accessed at once.
template <typename T, bool kVector> constexpr int kEachOf = (kVector ? 32 : 16) / (int)sizeof(T);

template <typename T, bool kDrop, bool kVector>
__global__ void __launch_bounds__(kThreads)
    dropout_kernel(const T* x, const T* residual, T* out, int64_t n, const Dropout d) {
    constexpr int kEach = kEachOf<T, kVector>;
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kEach;
    if (i >= n) return;
    float v[kEach], r[kEach] = {};
    const bool whole = kVector && i + kEach <= n;
    if (whole) {
        load(x + i, v);
        if (residual) load(residual + i, r);
    } else {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            v[j] = i + j < n ? widen(x[i + j]) : 0.0f;
            if (residual && i + j < n) r[j] = widen(residual[i + j]);
        }
    }
    if (kDrop) {
        // (a CTA's elements lie in one aligned span: the high word of their blocks is the CTA's)
        const uint64_t base = (uint64_t)blockIdx.x * (kThreads * kEach / 4);
        uint32_t w[kEach / 4][4];
        random_blocks(d, call_of(d), (uint32_t)base + threadIdx.x * (kEach / 4), (uint32_t)(base >> 32), w);
        if (residual) {
#pragma unroll
            for (int j = 0; j < kEach; ++j) v[j] = dropped(d, w[j / 4][j % 4]) ? r[j] : fmaf(v[j], d.factor, r[j]);
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j) v[j] = dropped(d, w[j / 4][j % 4]) ? 0.0f : v[j] * d.factor;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kEach; ++j) v[j] = residual ? v[j] + r[j] : v[j];
    }
    if (whole) {
        store(out + i, v);
    } else {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (i + j < n) out[i + j] = narrow<T>(v[j]);
    }
}

}  // namespace sidco_dropout_impl

extern "C" int sidco_dropout(const void* x, int type, int64_t n, float p, uint64_t seed, uint64_t call,
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
    const int64_t per = (int64_t)kThreads * (vector ? 32 : 16) / size_of(type), blocks = (n + per - 1) / per;
    const int rc = with_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const auto kernel = on ? vector ? dropout_kernel<T, true, true> : dropout_kernel<T, true, false>
                               : vector ? dropout_kernel<T, false, true> : dropout_kernel<T, false, false>;
        return (int)launch(kernel, dim3((unsigned)blocks), kThreads, 0, (cudaStream_t)stream, 1, (const T*)x,
                           (const T*)residual, (T*)out, n, d);
    });
    if (rc == 0) sidco_internal::note_launch();
    return rc;
}
