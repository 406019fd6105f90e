// Lookup of the rows of a table by token, with scaling and dropout, and the gradient of the table.
//
//   y[i] = scale * dropout(table[t_i]);      dT[v] (+)= scale * sum over i with t_i = v, in order of i, of dropout(dy[i])
//
// Both are bound by memory.  The gradient is deterministic: the tokens are sorted (stable, radix) and every row is a sum of
// fp32 terms in an order that depends on the tokens alone; no atomics.
//   sort_kernel  the first cluster sorts (token, position); the other CTAs meanwhile fill the table's gradient with zeros
//   sum_kernel   a warp takes a chunk of sorted positions and a slab of columns; runs of one token that lie inside the chunk
//                are finished, what reaches beyond its ends becomes a partial sum
//   join_kernel  adds the partial sums of runs that cross chunks, in order
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/sidco.h"
#include "sidco_elements.cuh"
#include "sidco_internal.h"
#include "sidco_tc.cuh"

namespace sidco_embedding_impl {

using namespace sidco_elements;

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------------------------- lookup

// A group is N neighbours of the flat output whose first index is a multiple of N, so that it starts a block of the generator.
// kVector: rows hold whole groups and are aligned for them.  Otherwise a row's first and last group may be shared with its
// neighbours, and each takes its own part.
template <typename TI, typename TO, int N, bool kVector, bool kDrop>
__global__ void __launch_bounds__(kThreads)
    lookup_kernel(const TI* __restrict__ table, int64_t vocab, int cols, int64_t ld, const void* __restrict__ tokens, int wide,
                  int64_t n, float scale, TO* __restrict__ out, int64_t ldo, const Dropout d, int lanes, int32_t* status) {
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const int lane = threadIdx.x & (lanes - 1), rows = kThreads / lanes;
    const uint64_t call = kDrop ? call_of(d) : 0;
    for (int64_t i = (int64_t)blockIdx.x * rows + threadIdx.x / lanes; i < n; i += (int64_t)gridDim.x * rows) {
        const int64_t t = token_at(tokens, wide, i);
        const bool known = t >= 0 && t < vocab;
        if (status && t >= vocab && lane == 0 && blockIdx.y == 0) atomicOr(status, SIDCO_EMBEDDING_ST_TOKEN);
        const int64_t base = i * cols;                                // of the flat output
        const int shift = kVector ? 0 : (int)(base % N);
        const TI* row = table + (known ? t * ld : 0);
        TO* to = out + i * ldo;
        const int groups = (shift + cols + N - 1) / N;
        for (int g = blockIdx.y * lanes + lane; g < groups; g += gridDim.y * lanes) {
            const int c = g * N - shift;
            float v[N] = {};
            if (known) {
                if (kVector) {
                    load(row + c, v);
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (c + j >= 0 && c + j < cols) v[j] = widen(row[c + j]);
                }
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] *= scale;
                if (kDrop) drop(d, call, (uint64_t)(base + c) / 4, v);
            }
            if (kVector) {
                store(to + c, v);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (c + j >= 0 && c + j < cols) to[c + j] = narrow<TO>(v[j]);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- sorting
//
// Least significant digit first, eight bits at most per pass.  Items lie in contiguous parts per CTA, and within a CTA per
// warp, so that (CTA, warp, step, lane) is the order of the items and ranking by it is stable.  A pass: every warp counts its
// digits (lanes of one digit find each other by a match), counts become offsets (over warps in shared memory, over the CTAs
// of the cluster in theirs), every warp places its items.  CTAs meet at cluster barriers; nothing spins.
// Padding and tokens outside the table get the largest key and end up behind the others.

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortMost = 8;                                          // CTAs of the sorting cluster
constexpr int kDigits = 256;

struct Sort {
    const void* tokens;
    int wide;
    uint32_t n;
    int64_t vocab;
    uint32_t* keys[2];
    uint32_t* at[2];
    int passes, bits;                 // bits per pass
    void* fill;                       // gradient to be set to zero, or NULL
    int64_t rows, row_bytes, pitch_bytes;
};

__device__ __forceinline__ uint32_t remote_load4(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}

// 0xff for 16-byte units of a row from its first aligned byte on, single bytes at its ends (rows may have any alignment)
__device__ void fill_rows(const Sort& s, int64_t worker, int64_t workers) {
    if (s.pitch_bytes == s.row_bytes) {                               // one row
        uint8_t* p = static_cast<uint8_t*>(s.fill);
        const int64_t bytes = s.rows * s.row_bytes;
        const int64_t head = min(bytes, (int64_t)((16 - (uintptr_t)p % 16) % 16)), units = (bytes - head) / 16;
        uint4* q = reinterpret_cast<uint4*>(p + head);
        for (int64_t i = worker * kSortThreads + threadIdx.x; i < units; i += workers * kSortThreads) q[i] = uint4{};
        if (worker == 0) {
            for (int64_t i = threadIdx.x; i < head; i += kSortThreads) p[i] = 0;
            for (int64_t i = head + units * 16 + threadIdx.x; i < bytes; i += kSortThreads) p[i] = 0;
        }
        return;
    }
    for (int64_t r = worker * kSortWarps + threadIdx.x / 32; r < s.rows; r += workers * kSortWarps) {
        uint8_t* p = static_cast<uint8_t*>(s.fill) + r * s.pitch_bytes;
        const int64_t head = min(s.row_bytes, (int64_t)((16 - (uintptr_t)p % 16) % 16)), units = (s.row_bytes - head) / 16;
        uint4* q = reinterpret_cast<uint4*>(p + head);
        for (int64_t i = threadIdx.x & 31; i < units; i += 32) q[i] = uint4{};
        for (int64_t i = threadIdx.x & 31; i < head; i += 32) p[i] = 0;
        for (int64_t i = head + units * 16 + (threadIdx.x & 31); i < s.row_bytes; i += 32) p[i] = 0;
    }
}

__global__ void __launch_bounds__(kSortThreads) sort_kernel(const Sort s, int ctas) {
    __shared__ uint32_t s_count[kSortWarps][kDigits];                 // of every warp, then its next place
    __shared__ uint32_t s_total[kDigits];                             // of the CTA
    __shared__ uint32_t s_warp[8];
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    if ((int)blockIdx.x >= ctas) {
        fill_rows(s, (int64_t)blockIdx.x - ctas, (int64_t)gridDim.x - ctas);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x;
    // whole steps of 32 items per warp
    const uint32_t per_warp = (uint32_t)(((uint64_t)s.n + (uint64_t)ctas * kSortWarps * 32 - 1) / ((uint64_t)ctas * kSortWarps * 32)) * 32;
    const uint64_t from = (uint64_t)(rank * kSortWarps + warp) * per_warp;
    const uint32_t first = (uint32_t)min(from, (uint64_t)s.n), end = (uint32_t)min(from + per_warp, (uint64_t)s.n);
    for (int pass = 0; pass < s.passes; ++pass) {
        const int shift = pass * s.bits;
        const uint32_t mask = (1u << s.bits) - 1;
        const uint32_t *keys = s.keys[pass & 1], *at = s.at[pass & 1];
        uint32_t *to_keys = s.keys[(pass & 1) ^ 1], *to_at = s.at[(pass & 1) ^ 1];
        const auto key_of = [&](uint32_t i) -> uint32_t {
            if (pass) return __ldcg(keys + i);
            const int64_t t = token_at(s.tokens, s.wide, i);
            return t >= 0 && t < s.vocab ? (uint32_t)t : (uint32_t)s.vocab;
        };
        for (int i = lane; i < kDigits; i += 32) s_count[warp][i] = 0;
        __syncwarp();
        for (uint32_t i = first; i < end; i += 32) {
            const bool mine = i + lane < end;
            const uint32_t digit = mine ? key_of(i + lane) >> shift & mask : kDigits;
            const uint32_t same = __match_any_sync(0xffffffffu, digit);
            if (mine && (same & ((1u << lane) - 1)) == 0) s_count[warp][digit] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        if (threadIdx.x < kDigits) {
            uint32_t sum = 0;
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = s_count[w][threadIdx.x];
                s_count[w][threadIdx.x] = sum;
                sum += c;
            }
            s_total[threadIdx.x] = sum;
        }
        __syncthreads();
        if (ctas > 1) sidco_tc::cluster_sync();
        uint32_t before = 0, all = 0;                                 // this digit in the CTAs before / in all
        if (threadIdx.x < kDigits) {
            for (int c = 0; c < ctas; ++c) {
                const uint32_t v = ctas > 1 ? remote_load4(sidco_tc::in_cta(sidco_tc::smem_addr(s_total + threadIdx.x), c))
                                            : s_total[threadIdx.x];
                if (c < (int)rank) before += v;
                all += v;
            }
            uint32_t up = all;                                        // digits up to this one: within the warp, then over warps
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, up, o);
                if (lane >= o) up += v;
            }
            if (lane == 31) s_warp[warp] = up;
            before += up - all;
        }
        __syncthreads();
        if (threadIdx.x < kDigits) {
            for (int w = 0; w < warp; ++w) before += s_warp[w];
            for (int w = 0; w < kSortWarps; ++w) s_count[w][threadIdx.x] += before;
        }
        __syncthreads();
        for (uint32_t i = first; i < end; i += 32) {
            const bool mine = i + lane < end;
            const uint32_t key = mine ? key_of(i + lane) : 0, digit = mine ? key >> shift & mask : kDigits;
            const uint32_t same = __match_any_sync(0xffffffffu, digit), lower = same & ((1u << lane) - 1);
            const uint32_t place = mine ? s_count[warp][digit] + __popc(lower) : 0;
            __syncwarp();
            if (mine) {
                if (lower == 0) s_count[warp][digit] = place + __popc(same);
                to_keys[place] = key;
                to_at[place] = pass ? __ldcg(at + i + lane) : i + lane;
            }
            __syncwarp();
        }
        // (what the other CTAs have placed is read in the next pass; their totals have been read)
        __threadfence();
        __syncthreads();
        if (ctas > 1) sidco_tc::cluster_sync();
    }
}

// ---------------------------------------------------------------------------------------------- sums

struct Sums {
    const uint32_t *keys, *at;        // sorted
    uint32_t n, vocab;
    int cols, chunk;                  // sorted positions per warp, at most 32
    int64_t ld_dy, ldd;
    float scale;
    int add;
    float* partial;                   // [chunks][2][cols]: of the run that enters a chunk and of the one that leaves it
};

constexpr int kEach = 4;              // columns per lane
constexpr int kSlab = 32 * kEach;
constexpr int kAhead = 8;             // rows in flight

template <typename T, bool kVector>
__device__ __forceinline__ void load_slab(const T* p, int left, float (&v)[kEach]) {
    if (kVector) {
        if (left >= kEach) load(p, v);
    } else {
#pragma unroll
        for (int j = 0; j < kEach; ++j) v[j] = j < left ? widen(p[j]) : 0.0f;
    }
}

template <typename TO, bool kVector>
__device__ __forceinline__ void write_slab(const Sums& s, TO* row, int left, const float (&sum)[kEach]) {
    if (left <= 0) return;
    float v[kEach] = {};
    if (s.add) load_slab<TO, kVector>(row, left, v);
#pragma unroll
    for (int j = 0; j < kEach; ++j) v[j] += sum[j] * s.scale;
    if (kVector) {
        store(row, v);
    } else {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (j < left) row[j] = narrow<TO>(v[j]);
    }
}

template <bool kVector> __device__ __forceinline__ void write_partial(float* p, int left, const float (&sum)[kEach]) {
    if (left <= 0) return;
    if (kVector) {
        store(p, sum);
    } else {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (j < left) p[j] = sum[j];
    }
}

// Dropout of kEach columns from c on of row i.
template <bool kVector>
__device__ __forceinline__ void drop_slab(const Dropout& d, uint64_t call, int64_t first, float (&v)[kEach]) {
    if (kVector || first % 4 == 0) {
        drop(d, call, (uint64_t)first / 4, v);
        return;
    }
    uint32_t a[4], b[4];
    random4(d, call, (uint64_t)first / 4, a);
    random4(d, call, (uint64_t)first / 4 + 1, b);
    const int shift = (int)(first % 4);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        uint32_t w = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k == j + shift) w = k < 4 ? a[k & 3] : b[k & 3];
        v[j] = w <= d.last ? 0.0f : v[j] * d.factor;
    }
}

template <typename TI, typename TO, bool kVector, bool kDrop>
__global__ void __launch_bounds__(kThreads)
    sum_kernel(const TI* __restrict__ dy, TO* __restrict__ out, const Sums s, const Dropout d, uint32_t chunks, int slabs) {
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const int lane = threadIdx.x & 31;
    const uint64_t unit = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (unit >= (uint64_t)chunks * slabs) return;
    const uint32_t chunk = (uint32_t)(unit / slabs);
    const int c = (int)(unit % slabs) * kSlab + lane * kEach, left = s.cols - c;
    const uint32_t first = chunk * s.chunk, count = min((uint32_t)s.chunk, s.n - first);
    // (lane l holds the l-th key and position; behind them the key of the next chunk)
    const uint32_t my_key = first + lane < s.n ? s.keys[first + lane] : s.vocab;
    const uint32_t my_at = lane < (int)count ? s.at[first + lane] : 0;
    const uint32_t before = first ? s.keys[first - 1] : s.vocab;
    const uint32_t behind = first + count < s.n ? s.keys[first + count] : s.vocab;
    const uint64_t call = kDrop ? call_of(d) : 0;
    float* partial = s.partial + (uint64_t)chunk * 2 * s.cols + c;
    float sum[kEach] = {};
    bool entered = true;                                              // the run began before this chunk
    {
        const uint32_t key0 = __shfl_sync(0xffffffffu, my_key, 0);
        if (key0 >= s.vocab) return;
        entered = key0 == before;
    }
    for (uint32_t k = 0; k < count; k += kAhead) {
        float v[kAhead][kEach];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const uint32_t key = __shfl_sync(0xffffffffu, my_key, (int)(k + j) & 31), at = __shfl_sync(0xffffffffu, my_at, (int)(k + j) & 31);
#pragma unroll
            for (int e = 0; e < kEach; ++e) v[j][e] = 0.0f;
            if (k + j < count && key < s.vocab && left > 0) load_slab<TI, kVector>(dy + at * s.ld_dy + c, left, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (k + j >= count) break;
            const uint32_t key = __shfl_sync(0xffffffffu, my_key, (int)(k + j)), at = __shfl_sync(0xffffffffu, my_at, (int)(k + j));
            const uint32_t in_next = __shfl_sync(0xffffffffu, my_key, (int)(k + j + 1) & 31);
            if (key >= s.vocab) return;                               // (nothing but padding from here on)
            if (kDrop) drop_slab<kVector>(d, call, (int64_t)at * s.cols + c, v[j]);
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum[e] += v[j][e];
            const bool last = k + j + 1 == count;
            const uint32_t next = last ? behind : in_next;
            if (next == key && !last) continue;
            if (next != key && !entered) write_slab<TO, kVector>(s, out + (int64_t)key * s.ldd + c, left, sum);
            else write_partial<kVector>(partial + (entered ? 0 : s.cols), left, sum);
            entered = false;
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum[e] = 0.0f;
        }
    }
}

// A run that leaves the chunk in which it began: its partial sums, one per chunk, in order.
template <typename TO, bool kVector>
__global__ void __launch_bounds__(kThreads) join_kernel(TO* __restrict__ out, const Sums s, uint32_t chunks, int slabs) {
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const uint64_t unit = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (unit >= (uint64_t)chunks * slabs) return;
    const uint32_t chunk = (uint32_t)(unit / slabs);
    const int lane = threadIdx.x & 31, c = (int)(unit % slabs) * kSlab + lane * kEach, left = s.cols - c;
    const uint32_t first = chunk * s.chunk, next = first + s.chunk;
    if (next >= s.n) return;
    const uint32_t key = s.keys[next - 1];
    if (key >= s.vocab || s.keys[next] != key) return;                // it ends here
    if (s.keys[first] == key && first && s.keys[first - 1] == key) return;      // it began earlier
    // how many of the following chunks it reaches: looked up by 32 lanes at a time
    uint32_t more = 0;
    for (;;) {
        const uint64_t p = (uint64_t)next + (uint64_t)(more + lane) * s.chunk;
        const uint32_t in = __ballot_sync(0xffffffffu, p < s.n && s.keys[p] == key);
        more += in == 0xffffffffu ? 32 : __ffs(~in) - 1;
        if (in != 0xffffffffu) break;
    }
    if (left <= 0) return;
    const float* p = s.partial + (uint64_t)chunk * 2 * s.cols + c;
    float sum[kEach];
    load_slab<float, kVector>(p + s.cols, left, sum);
    for (uint32_t k = 1; k <= more; k += kAhead) {
        float v[kAhead][kEach];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) v[j][e] = 0.0f;
            if (k + j <= more) load_slab<float, kVector>(p + (uint64_t)(k + j) * 2 * s.cols, left, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum[e] += v[j][e];
    }
    write_slab<TO, kVector>(s, out + (int64_t)key * s.ldd + c, left, sum);
}

// ---------------------------------------------------------------------------------------------- host side

constexpr int64_t kMostRows = ((int64_t)1 << 31) - ((int64_t)1 << 16);
constexpr int64_t kMostCols = (int64_t)1 << 24;

// Sorted positions per warp: 32 where there are many.
static int chunk_of(int64_t n, int64_t cols) {
    const int64_t slabs = (cols + kSlab - 1) / kSlab;
    int chunk = 32;
    while (chunk > 8 && n * slabs / chunk < 4096) chunk /= 2;
    return chunk;
}

struct Layout {
    int64_t keys[2], at[2], partial, bytes;
};

static Layout layout_of(int64_t n, int64_t cols) {
    Layout l{};
    const int64_t list = (n * 4 + 255) / 256 * 256, chunk = chunk_of(n, cols);
    l.keys[0] = 0;
    l.keys[1] = list;
    l.at[0] = 2 * list;
    l.at[1] = 3 * list;
    l.partial = 4 * list;
    l.bytes = l.partial + (n + chunk - 1) / chunk * 2 * cols * 4;
    return l;
}

static int check(int64_t n, int64_t vocab, int64_t cols) {
    return n < 0 || vocab < 0 || cols < 0 || n > kMostRows || vocab > kMostRows || cols > kMostCols ? SIDCO_E_SIZE : 0;
}

static cudaError_t sm_count(int* sms) {
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    return e != cudaSuccess ? e : cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
}

}  // namespace sidco_embedding_impl

extern "C" {

int sidco_embedding(const void* table, int table_type, int64_t vocab, int64_t cols, int64_t ld, const void* tokens,
                    int token_type, int64_t n, float scale, float p, uint64_t seed, uint64_t call, const uint64_t* step,
                    void* out, int out_type, int64_t ldo, int32_t* status, void* stream) {
    using namespace sidco_embedding_impl;
    if (const int rc = check(n, vocab, cols)) return rc;
    if (table_type < SIDCO_T_F32 || table_type > SIDCO_T_F16 || out_type < SIDCO_T_F32 || out_type > SIDCO_T_F16 ||
        (token_type != SIDCO_T_I32 && token_type != SIDCO_T_I64))
        return SIDCO_E_TYPE;
    if (ld < cols || ldo < cols) return SIDCO_E_PARAMS;
    Dropout d;
    bool on;
    if (const int rc = make_dropout(p, seed, call, step, &d, &on)) return rc;
    if (n > 0 && cols > 0 && ((!table && vocab > 0) || !tokens || !out)) return SIDCO_E_NULL;
    if ((uintptr_t)table % size_of(table_type) || (uintptr_t)out % size_of(out_type) ||
        (uintptr_t)tokens % (token_type == SIDCO_T_I64 ? 8 : 4) || (uintptr_t)status % 4)
        return SIDCO_E_ALIGN;
    const int64_t out_bytes = extent(n, cols, ldo, out_type);
    if (overlap(out, out_bytes, table, extent(vocab, cols, ld, table_type)) ||
        overlap(out, out_bytes, tokens, n * (token_type == SIDCO_T_I64 ? 8 : 4)))
        return SIDCO_E_ALIAS;
    cudaStream_t s = (cudaStream_t)stream;
    if (status) {
        const cudaError_t e = cudaMemsetAsync(status, 0, sizeof(int32_t), s);
        if (e != cudaSuccess) return (int)e;
    }
    if (n == 0 || cols == 0) return 0;
    const auto fits = [&](int k) {
        return cols % k == 0 && aligned(table, ld, table_type, k) && aligned(out, ldo, out_type, k);
    };
    const int vector = fits(8) ? 8 : fits(4) ? 4 : 0;
    const int64_t groups = vector ? cols / vector : (cols + 3) / 4 + 1;
    int lanes = 8;
    while (lanes < kThreads && lanes < groups) lanes *= 2;
    const int64_t rows = kThreads / lanes;
    const unsigned wide_grid = (unsigned)std::min<int64_t>((groups + lanes - 1) / lanes, 65535);
    const dim3 grid((unsigned)std::min<int64_t>((n + rows - 1) / rows, 0x7fffffff), wide_grid);
    const int rc = with_type(table_type, [&](auto* a) {
        return with_type(out_type, [&](auto* b) {
            using TI = std::remove_pointer_t<decltype(a)>;
            using TO = std::remove_pointer_t<decltype(b)>;
            const auto kernel = vector == 8   ? on ? lookup_kernel<TI, TO, 8, true, true> : lookup_kernel<TI, TO, 8, true, false>
                                : vector == 4 ? on ? lookup_kernel<TI, TO, 4, true, true> : lookup_kernel<TI, TO, 4, true, false>
                                : on          ? lookup_kernel<TI, TO, 4, false, true>
                                              : lookup_kernel<TI, TO, 4, false, false>;
            return (int)launch(kernel, grid, kThreads, 0, s, 1, (const TI*)table, vocab, (int)cols, ld, tokens,
                               (int)(token_type == SIDCO_T_I64), n, scale, (TO*)out, ldo, d, lanes, status);
        });
    });
    if (rc == 0) sidco_internal::note_launch();
    return rc;
}

int64_t sidco_embedding_grad_workspace_bytes(int64_t n, int64_t vocab, int64_t cols) {
    using namespace sidco_embedding_impl;
    if (check(n, vocab, cols)) return SIDCO_E_SIZE;
    return layout_of(n, cols).bytes;
}

int sidco_embedding_grad(const void* dy, int dy_type, int64_t ld_dy, const void* tokens, int token_type, int64_t n,
                         int64_t vocab, int64_t cols, float scale, float p, uint64_t seed, uint64_t call,
                         const uint64_t* step, void* dtable, int dtable_type, int64_t ldd, int add, void* workspace,
                         size_t workspace_bytes, void* stream) {
    using namespace sidco_embedding_impl;
    if (const int rc = check(n, vocab, cols)) return rc;
    if (dy_type < SIDCO_T_F32 || dy_type > SIDCO_T_F16 || dtable_type < SIDCO_T_F32 || dtable_type > SIDCO_T_F16 ||
        (token_type != SIDCO_T_I32 && token_type != SIDCO_T_I64))
        return SIDCO_E_TYPE;
    if (ld_dy < cols || ldd < cols) return SIDCO_E_PARAMS;
    Dropout d;
    bool on;
    if (const int rc = make_dropout(p, seed, call, step, &d, &on)) return rc;
    if (vocab == 0 || cols == 0 || (n == 0 && add)) return 0;
    if (!dtable || (n > 0 && (!dy || !tokens))) return SIDCO_E_NULL;
    if ((uintptr_t)dy % size_of(dy_type) || (uintptr_t)dtable % size_of(dtable_type) ||
        (uintptr_t)tokens % (token_type == SIDCO_T_I64 ? 8 : 4))
        return SIDCO_E_ALIGN;
    const Layout l = layout_of(n, cols);
    if (n > 0 && (!workspace || workspace_bytes < (size_t)l.bytes || (uintptr_t)workspace % 256)) return SIDCO_E_WORKSPACE;
    const int64_t token_bytes = n * (token_type == SIDCO_T_I64 ? 8 : 4), dy_bytes = extent(n, cols, ld_dy, dy_type);
    const int64_t out_bytes = extent(vocab, cols, ldd, dtable_type), used = n > 0 ? l.bytes : 0;
    if (overlap(dtable, out_bytes, dy, dy_bytes) || overlap(dtable, out_bytes, tokens, token_bytes) ||
        overlap(workspace, used, dy, dy_bytes) || overlap(workspace, used, tokens, token_bytes) ||
        overlap(workspace, used, dtable, out_bytes))
        return SIDCO_E_ALIAS;
    int sms = 0;
    cudaError_t e = sm_count(&sms);
    if (e != cudaSuccess) return (int)e;
    cudaStream_t st = (cudaStream_t)stream;
    uint8_t* ws = static_cast<uint8_t*>(workspace);

    Sort so{};
    so.tokens = tokens;
    so.wide = token_type == SIDCO_T_I64;
    so.n = (uint32_t)n;
    so.vocab = vocab;
    for (int i = 0; i < 2; ++i) {
        so.keys[i] = reinterpret_cast<uint32_t*>(ws + l.keys[i]);
        so.at[i] = reinterpret_cast<uint32_t*>(ws + l.at[i]);
    }
    int bits = 1;
    while ((vocab >> bits) > 0) ++bits;                               // keys 0 .. vocab
    so.passes = n > 0 ? (bits + 7) / 8 : 0;
    so.bits = n > 0 ? (bits + so.passes - 1) / so.passes : 0;
    so.fill = add ? nullptr : dtable;
    so.rows = vocab;
    so.row_bytes = cols * size_of(dtable_type);
    so.pitch_bytes = vocab > 1 ? ldd * size_of(dtable_type) : so.row_bytes;
    // one CTA up to 32 items per lane, then the whole cluster
    const int ctas = n <= 4 * kSortThreads ? 1 : kSortMost;
    int grid = ctas;
    if (!add) grid += std::max(ctas, (2 * sms - ctas) / ctas * ctas);
    e = launch(sort_kernel, dim3((unsigned)grid), kSortThreads, 0, st, ctas, so, ctas);
    if (e != cudaSuccess) return (int)e;
    sidco_internal::note_launch();
    if (n == 0) return 0;

    Sums su{};
    su.keys = so.keys[so.passes & 1];
    su.at = so.at[so.passes & 1];
    su.n = (uint32_t)n;
    su.vocab = (uint32_t)vocab;
    su.cols = (int)cols;
    su.chunk = chunk_of(n, cols);
    su.ld_dy = ld_dy;
    su.ldd = ldd;
    su.scale = scale;
    su.add = add != 0;
    su.partial = reinterpret_cast<float*>(ws + l.partial);
    const uint32_t chunks = (uint32_t)((n + su.chunk - 1) / su.chunk);
    const int slabs = (int)((cols + kSlab - 1) / kSlab);
    const int64_t blocks = ((int64_t)chunks * slabs + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffff) return SIDCO_E_SIZE;
    const bool vector = cols % kEach == 0 && aligned(dy, ld_dy, dy_type, kEach) && aligned(dtable, ldd, dtable_type, kEach);
    const int rc = with_type(dtable_type, [&](auto* b) {
        using TO = std::remove_pointer_t<decltype(b)>;
        const int first = with_type(dy_type, [&](auto* a) {
            using TI = std::remove_pointer_t<decltype(a)>;
            const auto kernel = vector ? on ? sum_kernel<TI, TO, true, true> : sum_kernel<TI, TO, true, false>
                                       : on ? sum_kernel<TI, TO, false, true> : sum_kernel<TI, TO, false, false>;
            return (int)launch(kernel, dim3((unsigned)blocks), kThreads, 0, st, 1, (const TI*)dy, (TO*)dtable, su, d, chunks,
                               slabs);
        });
        if (first) return first;
        sidco_internal::note_launch();
        const auto join = vector ? join_kernel<TO, true> : join_kernel<TO, false>;
        return (int)launch(join, dim3((unsigned)blocks), kThreads, 0, st, 1, (TO*)dtable, su, chunks, slabs);
    });
    if (rc == 0) sidco_internal::note_launch();
    return rc;
}

}  // extern "C"
