// Lookup of the rows of a table by token, with scaling and dropout, and the gradient of the table.
//
//   y[i] = scale * dropout(table[t_i]);      dT[v] (+)= scale * sum over i with t_i = v, in order of i, of dropout(dy[i])
//
// Both are bound by memory.  The gradient is deterministic: the tokens are sorted (stable, radix) and every row is a sum of
// fp32 terms in an order that depends on the tokens alone; no atomics.  Few tokens take one launch (few_kernel), more take three:
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

// N neighbours of a row at a time: `lanes` lanes have a row, each kAhead groups of it in flight; a warp has 32 / lanes rows.
// kVector: rows are aligned for groups and hold whole ones.  Otherwise groups start where the flat output's index is a multiple
// of four, so that they are blocks of the generator, and a row's first and last group may be shared with its neighbours.
constexpr int kAhead = 4;

template <typename TI, typename TO, int N, bool kVector, bool kDrop>
__global__ void __launch_bounds__(kThreads)
    lookup_kernel(const TI* __restrict__ table, int64_t vocab, int cols, int64_t ld, const void* __restrict__ tokens, int wide,
                  int64_t n, float scale, TO* __restrict__ out, int64_t ldo, const Dropout d, int lanes, int spans, int32_t* status) {
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const int lane = threadIdx.x & (lanes - 1), rows = 32 / lanes;
    const uint64_t call = kDrop ? call_of(d) : 0;
    const int64_t workers = (int64_t)gridDim.x * (kThreads / 32), units = (n + rows - 1) / rows * spans;
    // (a unit: the rows of a warp, one span of `lanes` x kAhead groups of them)
    for (int64_t u = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32; u < units; u += workers) {
        const int64_t i = u / spans * rows + (threadIdx.x & 31) / lanes;
        if (i >= n) continue;
        const int span = (int)(u % spans);
        const int64_t t = token_at(tokens, wide, i);
        const bool known = t >= 0 && t < vocab;
        if (status && t >= vocab && lane == 0 && span == 0) atomicOr(status, SIDCO_EMBEDDING_ST_TOKEN);
        const int64_t base = i * cols;                                // of the flat output
        const int shift = kVector ? 0 : (int)(base % 4);
        const TI* row = table + (known ? t * ld : 0);
        TO* to = out + i * ldo;
        const int first = (span * kAhead * lanes + lane) * N - shift;
        float v[kAhead][N];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int c = first + k * lanes * N;
            if (kVector) {
                if (known && c < cols) load(row + c, v[k]);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) v[k][j] = known && c + j >= 0 && c + j < cols ? widen(row[c + j]) : 0.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int c = first + k * lanes * N;
            if (c >= cols) break;
#pragma unroll
            for (int j = 0; j < N; ++j) v[k][j] = known ? v[k][j] * scale : 0.0f;
            if (kDrop) drop(d, call, (uint64_t)(base + c), v[k]);
            if (kVector) {
                store(to + c, v[k]);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (c + j >= 0 && c + j < cols) to[c + j] = narrow<TO>(v[k][j]);
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
constexpr int kBatch = 8;                                             // steps whose reads are in flight together

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

__global__ void __launch_bounds__(kSortThreads) sort_kernel(const Sort s) {
    __shared__ uint32_t s_count[kSortWarps][kDigits];                 // of every warp, then its next place
    __shared__ uint32_t s_total[kDigits];                             // of the CTA
    __shared__ uint32_t s_base[4][kDigits];                           // where a quarter of the warps begins
    __shared__ uint32_t s_warp[8];
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    constexpr int ctas = kSortMost;
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
        for (uint32_t i0 = first; i0 < end; i0 += 32 * kBatch) {
            uint32_t key[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) key[k] = key_of(min(i0 + k * 32 + lane, end - 1));
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (i0 + k * 32 >= end) break;
                const bool mine = i0 + k * 32 + lane < end;
                const uint32_t digit = mine ? key[k] >> shift & mask : kDigits;
                const uint32_t same = __match_any_sync(0xffffffffu, digit);
                if (mine && (same & ((1u << lane) - 1)) == 0) s_count[warp][digit] += __popc(same);
                __syncwarp();
            }
        }
        __syncthreads();
        // offsets of the warps, by a quarter of them per thread; totals
        const int digit = threadIdx.x % kDigits, quarter = threadIdx.x / kDigits;
        {
            uint32_t c[kSortWarps / 4], sum = 0;
#pragma unroll
            for (int w = 0; w < kSortWarps / 4; ++w) c[w] = s_count[quarter * (kSortWarps / 4) + w][digit];
#pragma unroll
            for (int w = 0; w < kSortWarps / 4; ++w) {
                s_count[quarter * (kSortWarps / 4) + w][digit] = sum;
                sum += c[w];
            }
            s_base[quarter][digit] = sum;
        }
        __syncthreads();
        if (threadIdx.x < kDigits) s_total[digit] = s_base[0][digit] + s_base[1][digit] + s_base[2][digit] + s_base[3][digit];
        sidco_tc::cluster_sync();
        uint32_t before = 0;
        if (threadIdx.x < kDigits) {
            uint32_t all = 0;                                         // this digit in the CTAs before / in all
            for (int c = 0; c < kSortMost; ++c) {
                const uint32_t v = remote_load4(sidco_tc::in_cta(sidco_tc::smem_addr(s_total + digit), c));
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
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t v = s_base[q][digit];
                s_base[q][digit] = before;
                before += v;
            }
        }
        __syncthreads();
        for (uint32_t i0 = first; i0 < end; i0 += 32 * kBatch) {
            uint32_t key[kBatch], from[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const uint32_t i = min(i0 + k * 32 + lane, end - 1);
                key[k] = key_of(i);
                from[k] = pass ? __ldcg(at + i) : i;
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (i0 + k * 32 >= end) break;
                const bool mine = i0 + k * 32 + lane < end;
                const uint32_t digit = mine ? key[k] >> shift & mask : kDigits;
                const uint32_t same = __match_any_sync(0xffffffffu, digit), lower = same & ((1u << lane) - 1);
                const uint32_t next = mine ? s_count[warp][digit] + __popc(lower) : 0;
                __syncwarp();
                if (mine) {
                    if (lower == 0) s_count[warp][digit] = next + __popc(same);
                    const uint32_t place = s_base[warp / (kSortWarps / 4)][digit] + next;
                    to_keys[place] = key[k];
                    to_at[place] = from[k];
                }
                __syncwarp();
            }
        }
        // what the other CTAs have placed is read in the next pass (the barrier orders it); their totals have been read
        sidco_tc::cluster_sync();
    }
}

// ---------------------------------------------------------------------------------------------- sums

struct Sums {
    const uint32_t *keys, *at;        // sorted
    uint32_t n, vocab;
    int cols, chunk;                  // sorted positions per warp, at most 32
    int64_t ld_dy, ldd;
    uintptr_t lo, hi;                 // dy
    float scale;
    int add;
    float* partial;                   // [chunks][2][pitch]: of the run that enters a chunk and of the one that leaves it
    int64_t pitch;
};

constexpr int kEach = 8;              // columns per lane
constexpr int kSlab = 32 * kEach;

// kEach elements of a row of dy as they lie.  kVector: aligned and whole.  Otherwise of any alignment: two (three) aligned
// 16-byte reads are put together; where these would leave dy, at its ends, single elements are read.
template <typename T, bool kVector> struct Raw {
    static constexpr int kWords = kEach * (int)sizeof(T) / 4, kRead = kWords + (kVector ? 0 : 4);
    uint32_t w[kRead];
    __device__ __forceinline__ void read(const T* p, int left, const Sums& s) {
        const uintptr_t start = (uintptr_t)p & ~(uintptr_t)15;
        if (kVector || (start >= s.lo && start + kRead * 4 <= s.hi)) {
#pragma unroll
            for (int i = 0; i < kRead / 4; ++i) {
                const uint4 v = reinterpret_cast<const uint4*>(start)[i];
                w[i * 4] = v.x, w[i * 4 + 1] = v.y, w[i * 4 + 2] = v.z, w[i * 4 + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kRead; ++i) w[i] = 0;
            // (laid down as if it had been read: `shift` bytes in)
            const int shift = (int)((uintptr_t)p & 15);
            if constexpr (sizeof(T) == 4) {
                uint32_t e[kEach];
#pragma unroll
                for (int j = 0; j < kEach; ++j) e[j] = j < left ? reinterpret_cast<const uint32_t*>(p)[j] : 0;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (shift == 4 * k)
#pragma unroll
                        for (int j = 0; j < kEach; ++j) w[(j + k) % kRead] = e[j];
            } else {
                uint16_t e[kEach];
#pragma unroll
                for (int j = 0; j < kEach; ++j) e[j] = j < left ? reinterpret_cast<const uint16_t*>(p)[j] : 0;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (shift == 2 * k)
#pragma unroll
                        for (int j = 0; j < kEach; ++j) w[(j + k) / 2 % kRead] |= (uint32_t)e[j] << ((j + k) % 2 * 16);
            }
        }
    }
    __device__ __forceinline__ void widened(const T* p, float (&v)[kEach]) {
        if constexpr (!kVector) shift_words<kWords>(w, (int)((uintptr_t)p & 15));
        const T* t = reinterpret_cast<const T*>(w);
#pragma unroll
        for (int j = 0; j < kEach; ++j) v[j] = widen(t[j]);
    }
};

// vector: 8 or 4 columns can be written at once (and there are whole ones), or 1.
template <typename TO>
__device__ __forceinline__ void write_row(const Sums& s, TO* row, int left, int vector, const float (&sum)[kEach]) {
    if (left <= 0) return;
    float v[kEach] = {};
    if (vector == 8) {
        if (s.add) load(row, v);
#pragma unroll
        for (int j = 0; j < kEach; ++j) v[j] += sum[j] * s.scale;
        store(row, v);
    } else if (vector == 4) {
        float h[2][4] = {};
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (s.add) load(row + (left >= 8 ? i * 4 : 0), h[i]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) h[i][j] += sum[i * 4 + j] * s.scale;
        store(row, h[0]);
        if (left >= 8) store(row + 4, h[1]);
    } else {
        if (s.add) {
#pragma unroll
            for (int j = 0; j < kEach; ++j) v[j] = widen(row[min(j, left - 1)]);
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (j < left) row[j] = narrow<TO>(v[j] + sum[j] * s.scale);
    }
}

// Sorted positions 0 .. count-1 of a chunk, for one slab of columns: row_at(k) is the position's row of dy, ends(k) whether a
// run ends behind it, done(k) takes a run's sum (in `sum`) there.  The next row comes while one is added: with more rows in
// flight per warp fewer warps fit, and the generator's code is there once per row.
template <typename TI, bool kVector, bool kDrop, typename RowAt, typename Ends, typename Done>
__device__ __forceinline__ void add_up(const TI* dy, const Sums& s, const Dropout& d, uint64_t call, int c, int left, int count,
                                       RowAt row_at, Ends ends, Done done, float (&sum)[kEach]) {
    Raw<TI, kVector> raw, coming;
    uint32_t at = 0, at_next = 0;
    if (count > 0) {
        at_next = row_at(0);
        if (left > 0) coming.read(dy + at_next * s.ld_dy + c, left, s);
    }
#pragma unroll 1
    for (int k = 0; k < count; ++k) {
        raw = coming;
        at = at_next;
        at_next = row_at(min(k + 1, count - 1));
        if (left > 0 && k + 1 < count) coming.read(dy + at_next * s.ld_dy + c, left, s);
        float v[kEach];
        raw.widened(dy + at * s.ld_dy + c, v);
        if (kDrop) {
            const uint64_t first = (uint64_t)at * s.cols + c;
            if (first % 4 == 0) drop(d, call, first, v);              // (the same for the whole warp)
            else drop<kEach, false>(d, call, first, v);
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) sum[e] += v[e];
        if (ends(k)) {
            done(k);
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum[e] = 0.0f;
        }
    }
}

template <typename TI, typename TO, bool kVector, bool kDrop>
__global__ void __launch_bounds__(kThreads, 4)
    sum_kernel(const TI* __restrict__ dy, TO* __restrict__ out, const Sums s, const Dropout d, uint32_t chunks, int slabs, int out_vector) {
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const int lane = threadIdx.x & 31;
    const uint64_t unit = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (unit >= (uint64_t)chunks * slabs) return;
    const uint32_t chunk = (uint32_t)(unit / slabs);
    const int c = (int)(unit % slabs) * kSlab + lane * kEach, left = s.cols - c;
    const uint32_t first = chunk * s.chunk;
    const int count = (int)min((uint32_t)s.chunk, s.n - first);
    // (lane l holds the l-th key and position)
    const uint32_t my_key = lane < count ? s.keys[first + lane] : s.vocab;
    const uint32_t my_at = lane < count ? s.at[first + lane] : 0;
    const uint32_t before = first ? s.keys[first - 1] : s.vocab;
    const uint32_t behind = first + count < s.n ? s.keys[first + count] : s.vocab;
    const uint64_t call = kDrop ? call_of(d) : 0;
    const int valid = __popc(__ballot_sync(0xffffffffu, my_key < s.vocab));        // (padding is behind all others)
    if (valid == 0) return;
    uint32_t next = __shfl_down_sync(0xffffffffu, my_key, 1);
    if (lane == count - 1) next = behind;
    const uint32_t ends = __ballot_sync(0xffffffffu, my_key != next);              // a run ends behind position l
    bool entered = __shfl_sync(0xffffffffu, my_key, 0) == before;                  // the run began before this chunk
    float* partial = s.partial + (uint64_t)chunk * 2 * s.pitch + c;
    float sum[kEach] = {};
    add_up<TI, kVector, kDrop>(
        dy, s, d, call, c, left, valid, [&](int k) { return __shfl_sync(0xffffffffu, my_at, k); },
        [&](int k) { return (ends >> k & 1) != 0; },
        [&](int k) {
            const uint32_t key = __shfl_sync(0xffffffffu, my_key, k);
            if (!entered) write_row(s, out + (int64_t)key * s.ldd + c, left, out_vector, sum);
            else if (left > 0) store(partial, sum);
            entered = false;
        },
        sum);
    if (valid == count && !(ends >> (count - 1) & 1) && left > 0) store(partial + (entered ? 0 : s.pitch), sum);
}

// A run that leaves the chunk in which it began: its partial sums, one per chunk, in order.
template <typename TO>
__global__ void __launch_bounds__(kThreads, 2) join_kernel(TO* __restrict__ out, const Sums s, uint32_t chunks, int slabs, int out_vector) {
    constexpr int kRows = 8;
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
    const float* p = s.partial + (uint64_t)chunk * 2 * s.pitch + c;
    float sum[kEach];
    load(p + s.pitch, sum);
    for (uint32_t k = 1; k <= more; k += kRows) {
        float v[kRows][kEach];
#pragma unroll
        for (int j = 0; j < kRows; ++j) load(p + (uint64_t)min(k + j, more) * 2 * s.pitch, v[j]);
#pragma unroll
        for (int j = 0; j < kRows; ++j)
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum[e] += k + j <= more ? v[j][e] : 0.0f;
    }
    write_row(s, out + (int64_t)key * s.ldd + c, left, out_vector, sum);
}

// ---------------------------------------------------------------------------------------------- few tokens
//
// Up to kFewMost tokens take one launch: a CTA has a range of the table's rows and a slab of its columns.  It picks its tokens
// out of all, sends zeros to the rows that have none (they leave while it goes on), and ranks its tokens by counting; its warps take equal parts of
// the sorted list, whose runs they join in shared memory where they cross from one part to the next.  Nobody waits for another
// CTA.  (Three launches took 25 us for 700 tokens of 10000 x 1500, this takes FEWUS.)

constexpr int kFewMost = 2048, kFewThreads = 512, kFewWarps = kFewThreads / 32, kFewEach = kFewMost / kFewThreads;
constexpr int kFewRange = 8192;       // rows of a range, at most

struct Few {
    const void* tokens;
    int wide, n;
    int64_t vocab, rows;              // of the table, per CTA
    int fill;                         // rows without tokens become zero: 1 by stores, 2 by bulk copies
};

template <typename TI, typename TO, bool kVector, bool kDrop>
__global__ void __launch_bounds__(kFewThreads, 2)
    few_kernel(const TI* __restrict__ dy, TO* out, const Few f, const Sums s, const Dropout d, int slabs, int out_vector) {
    __shared__ uint32_t s_key[kFewMost], s_sorted[kFewMost];          // row within the range
    __shared__ uint16_t s_from[kFewMost], s_at[kFewMost];
    __shared__ uint32_t s_mark[kFewRange / 32];                       // rows that have tokens
    __shared__ int s_part[kFewEach][kFewWarps];
    __shared__ __align__(16) float s_sum[kFewWarps][kSlab];           // of the run that enters a part
    __shared__ __align__(16) uint8_t s_zero[kSlab * 4];
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row0 = blockIdx.x / slabs * f.rows;
    const int rows = (int)min(f.rows, f.vocab - row0);
    const int c0 = (int)(blockIdx.x % slabs) * kSlab, c = c0 + lane * kEach, left = s.cols - c;
    if (rows <= 0) return;
    int64_t t[kFewEach];
#pragma unroll
    for (int k = 0; k < kFewEach; ++k) {
        const int i = k * kFewThreads + threadIdx.x;
        t[k] = i < f.n ? token_at(f.tokens, f.wide, i) - row0 : -1;
    }
    for (int i = threadIdx.x; i < kFewRange / 32; i += kFewThreads) s_mark[i] = 0;
    if (threadIdx.x < kSlab / 4) reinterpret_cast<uint4*>(s_zero)[threadIdx.x] = uint4{};
    sidco_tc::fence_async_shared();
    // the range's tokens, in order
    uint32_t in[kFewEach];
#pragma unroll
    for (int k = 0; k < kFewEach; ++k) {
        in[k] = __ballot_sync(0xffffffffu, t[k] >= 0 && t[k] < rows);
        if (lane == 0) s_part[k][warp] = __popc(in[k]);
    }
    __syncthreads();
    int found = 0;
#pragma unroll
    for (int k = 0; k < kFewEach; ++k) {
        if (k * kFewThreads >= f.n) break;
        int up = lane < kFewWarps ? s_part[k][lane] : 0;
        const int mine = up;
#pragma unroll
        for (int o = 1; o < kFewWarps; o *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, up, o);
            if (lane >= o) up += v;
        }
        const int to = found + __shfl_sync(0xffffffffu, up - mine, warp) + __popc(in[k] & ((1u << lane) - 1));
        found += __shfl_sync(0xffffffffu, up, kFewWarps - 1);
        if (t[k] >= 0 && t[k] < rows) {
            s_key[to] = (uint32_t)t[k], s_from[to] = (uint16_t)(k * kFewThreads + threadIdx.x);
            atomicOr(&s_mark[t[k] / 32], 1u << (t[k] % 32));
        }
    }
    __syncthreads();
    // the other rows become zero: by bulk copies, which leave the load path free, where rows are aligned for them
    if (f.fill) {
        const int width = min(kSlab, s.cols - c0);
        if (f.fill == 2) {
            for (int r = threadIdx.x; r < rows; r += kFewThreads)
                if (!(s_mark[r / 32] >> (r % 32) & 1))
                    sidco_tc::bulk_store(out + (row0 + r) * s.ldd + c0, sidco_tc::smem_addr(s_zero), width * (int)sizeof(TO));
            sidco_tc::bulk_store_commit();
        } else {
            for (int r = warp; r < rows; r += kFewWarps)
                if (!(s_mark[r / 32] >> (r % 32) & 1))
                    for (int i = lane; i < width; i += 32) out[(row0 + r) * s.ldd + c0 + i] = narrow<TO>(0.0f);
        }
    }
    // stable order by key: how many come before each
    for (int i = threadIdx.x; i < found; i += kFewThreads) {
        const uint32_t key = s_key[i];
        int before = 0;
#pragma unroll 8
        for (int j = 0; j < found; ++j) before += s_key[j] < key || (s_key[j] == key && j < i);
        s_sorted[before] = key;
        s_at[before] = s_from[i];
    }
    __syncthreads();
    const uint64_t call = kDrop ? call_of(d) : 0;
    const int part = (found + kFewWarps - 1) / kFewWarps, first = min(found, warp * part), count = min(part, found - first);
    bool entered = count > 0 && first > 0 && s_sorted[first - 1] == s_sorted[first];
    float sum[kEach] = {};
    add_up<TI, kVector, kDrop>(
        dy, s, d, call, c, left, count, [&](int k) { return (uint32_t)s_at[first + k]; },
        [&](int k) { return first + k + 1 == found || s_sorted[first + k + 1] != s_sorted[first + k]; },
        [&](int k) {
            if (!entered) write_row(s, out + (row0 + s_sorted[first + k]) * s.ldd + c, left, out_vector, sum);
            else store(&s_sum[warp][lane * kEach], sum);
            entered = false;
        },
        sum);
    const bool leaves = count > 0 && first + count < found && s_sorted[first + count] == s_sorted[first + count - 1];
    if (leaves && entered) store(&s_sum[warp][lane * kEach], sum);
    __syncthreads();
    if (leaves && !entered) {                                         // a run that began here goes on
        const uint32_t key = s_sorted[first + count - 1];
        for (int w = warp + 1; w * part < found && s_sorted[w * part] == key; ++w) {
            float v[kEach];
            load(&s_sum[w][lane * kEach], v);
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum[e] += v[e];
        }
        write_row(s, out + (row0 + key) * s.ldd + c, left, out_vector, sum);
    }
    if (f.fill == 2) sidco_tc::bulk_store_wait_read();                // (shared memory stays until the zeros have left it)
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
    int64_t keys[2], at[2], partial, pitch, bytes;
};

static Layout layout_of(int64_t n, int64_t cols) {
    Layout l{};
    if (n <= kFewMost) return l;                                      // (one launch, no lists)
    const int64_t list = (n * 4 + 255) / 256 * 256, chunk = chunk_of(n, cols);
    l.keys[0] = 0;
    l.keys[1] = list;
    l.at[0] = 2 * list;
    l.at[1] = 3 * list;
    l.partial = 4 * list;
    l.pitch = (cols + kEach - 1) / kEach * kEach;
    l.bytes = l.partial + (n + chunk - 1) / chunk * 2 * l.pitch * 4;
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
    int lanes = 1;
    while (lanes < 32 && lanes < groups) lanes *= 2;
    const int64_t spans = (groups + lanes * kAhead - 1) / (lanes * kAhead), rows = 32 / lanes;
    int sms = 0;
    if (const cudaError_t e = sm_count(&sms); e != cudaSuccess) return (int)e;
    // (eight CTAs are resident per SM; four rounds of them even out)
    const dim3 grid((unsigned)std::min<int64_t>(((n + rows - 1) / rows * spans + kThreads / 32 - 1) / (kThreads / 32), 32 * sms));
    const int rc = with_type(table_type, [&](auto* a) {
        return with_type(out_type, [&](auto* b) {
            using TI = std::remove_pointer_t<decltype(a)>;
            using TO = std::remove_pointer_t<decltype(b)>;
            const auto kernel = vector == 8   ? on ? lookup_kernel<TI, TO, 8, true, true> : lookup_kernel<TI, TO, 8, true, false>
                                : vector == 4 ? on ? lookup_kernel<TI, TO, 4, true, true> : lookup_kernel<TI, TO, 4, true, false>
                                : on          ? lookup_kernel<TI, TO, 4, false, true>
                                              : lookup_kernel<TI, TO, 4, false, false>;
            return (int)launch(kernel, grid, kThreads, 0, s, 1, (const TI*)table, vocab, (int)cols, ld, tokens,
                               (int)(token_type == SIDCO_T_I64), n, scale, (TO*)out, ldo, d, lanes, (int)spans, status);
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
    if (l.bytes > 0 && (!workspace || workspace_bytes < (size_t)l.bytes || (uintptr_t)workspace % 256)) return SIDCO_E_WORKSPACE;
    const int64_t token_bytes = n * (token_type == SIDCO_T_I64 ? 8 : 4), dy_bytes = extent(n, cols, ld_dy, dy_type);
    const int64_t out_bytes = extent(vocab, cols, ldd, dtable_type), used = l.bytes;
    if (overlap(dtable, out_bytes, dy, dy_bytes) || overlap(dtable, out_bytes, tokens, token_bytes) ||
        overlap(workspace, used, dy, dy_bytes) || overlap(workspace, used, tokens, token_bytes) ||
        overlap(workspace, used, dtable, out_bytes))
        return SIDCO_E_ALIAS;
    int sms = 0;
    cudaError_t e = sm_count(&sms);
    if (e != cudaSuccess) return (int)e;
    cudaStream_t st = (cudaStream_t)stream;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const bool vector = cols % kEach == 0 && (uintptr_t)dy % 16 == 0 && ld_dy * size_of(dy_type) % 16 == 0;
    const int out_vector = cols % 8 == 0 && aligned(dtable, ldd, dtable_type, 8)   ? 8
                           : cols % 4 == 0 && aligned(dtable, ldd, dtable_type, 4) ? 4
                                                                                   : 1;
    const int slabs = (int)((cols + kSlab - 1) / kSlab);
    Sums su{};
    su.n = (uint32_t)n;
    su.vocab = (uint32_t)vocab;
    su.cols = (int)cols;
    su.ld_dy = ld_dy;
    su.ldd = ldd;
    su.lo = (uintptr_t)dy;
    su.hi = (uintptr_t)dy + (uintptr_t)dy_bytes;
    su.scale = scale;
    su.add = add != 0;

    if (n <= kFewMost) {
        // as many ranges of rows as give every SM two CTAs, at least eight rows each where rows are to be filled
        const int64_t size = size_of(dtable_type);
        const bool bulk = (uintptr_t)dtable % 16 == 0 && ldd * size % 16 == 0 && cols * size % 16 == 0;
        Few f{tokens, token_type == SIDCO_T_I64, (int)n, vocab, 0, add ? 0 : bulk ? 2 : 1};
        const int64_t ranges = std::max<int64_t>(std::min<int64_t>(2 * sms / slabs, (vocab + 7) / 8), (vocab + kFewRange - 1) / kFewRange);
        f.rows = (vocab + ranges - 1) / ranges;
        if (ranges * slabs > 0x7fffffff) return SIDCO_E_SIZE;
        const int rc = with_type(dtable_type, [&](auto* b) {
            using TO = std::remove_pointer_t<decltype(b)>;
            return with_type(dy_type, [&](auto* a) {
                using TI = std::remove_pointer_t<decltype(a)>;
                const auto kernel = vector ? on ? few_kernel<TI, TO, true, true> : few_kernel<TI, TO, true, false>
                                           : on ? few_kernel<TI, TO, false, true> : few_kernel<TI, TO, false, false>;
                return (int)launch(kernel, dim3((unsigned)(ranges * slabs)), kFewThreads, 0, st, 1, (const TI*)dy,
                                   (TO*)dtable, f, su, d, slabs, out_vector);
            });
        });
        if (rc == 0) sidco_internal::note_launch();
        return rc;
    }

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
    so.passes = (bits + 7) / 8;
    so.bits = (bits + so.passes - 1) / so.passes;
    so.fill = add ? nullptr : dtable;
    so.rows = vocab;
    so.row_bytes = cols * size_of(dtable_type);
    so.pitch_bytes = vocab > 1 ? ldd * size_of(dtable_type) : so.row_bytes;
    const int ctas = kSortMost;
    int grid = ctas;
    if (!add) grid += std::max(ctas, (2 * sms - ctas) / ctas * ctas);
    e = launch(sort_kernel, dim3((unsigned)grid), kSortThreads, 0, st, ctas, so);
    if (e != cudaSuccess) return (int)e;
    sidco_internal::note_launch();

    su.keys = so.keys[so.passes & 1];
    su.at = so.at[so.passes & 1];
    su.chunk = chunk_of(n, cols);
    su.partial = reinterpret_cast<float*>(ws + l.partial);
    su.pitch = l.pitch;
    const uint32_t chunks = (uint32_t)((n + su.chunk - 1) / su.chunk);
    const int64_t blocks = ((int64_t)chunks * slabs + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffff) return SIDCO_E_SIZE;
    const int rc = with_type(dtable_type, [&](auto* b) {
        using TO = std::remove_pointer_t<decltype(b)>;
        const int first = with_type(dy_type, [&](auto* a) {
            using TI = std::remove_pointer_t<decltype(a)>;
            const auto kernel = vector ? on ? sum_kernel<TI, TO, true, true> : sum_kernel<TI, TO, true, false>
                                       : on ? sum_kernel<TI, TO, false, true> : sum_kernel<TI, TO, false, false>;
            return (int)launch(kernel, dim3((unsigned)blocks), kThreads, 0, st, 1, (const TI*)dy, (TO*)dtable, su, d, chunks,
                               slabs, out_vector);
        });
        if (first) return first;
        sidco_internal::note_launch();
        return (int)launch(join_kernel<TO>, dim3((unsigned)blocks), kThreads, 0, st, 1, (TO*)dtable, su, chunks, slabs,
                           out_vector);
    });
    if (rc == 0) sidco_internal::note_launch();
    return rc;
}

}  // extern "C"
