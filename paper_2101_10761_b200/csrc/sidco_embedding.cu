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
constexpr int kEach = 8;              // neighbours of a row per lane

// kEach elements of a row as they lie.  kVector: aligned and whole.  Otherwise of any alignment: two (three) aligned 16-byte
// reads are put together; where these would leave the matrix, [lo, hi), single elements are read.
template <typename T, bool kVector> struct Raw {
    static constexpr int kWords = kEach * (int)sizeof(T) / 4, kRead = kWords + (kVector ? 0 : 4);
    uint32_t w[kRead];
    __device__ __forceinline__ void read(const T* p, int left, uintptr_t lo, uintptr_t hi) {
        const uintptr_t start = (uintptr_t)p & ~(uintptr_t)15;
        if (kVector || (start >= lo && start + kRead * 4 <= hi)) {
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


// ---------------------------------------------------------------------------------------------- lookup

// N neighbours of a row at a time: `lanes` lanes have a row, each kAhead groups of it in flight; a warp has 32 / lanes rows.
// kVector: rows are aligned for groups and hold whole ones.  Otherwise groups start where the flat output's index is a multiple
// of four, so that they are blocks of the generator, and a row's first and last group may be shared with its neighbours.
constexpr int kAhead = 4;

template <typename TI, typename TO, int N, bool kVector, bool kDrop>
__global__ void __launch_bounds__(kThreads, 4)
    lookup_kernel(const TI* table, int64_t vocab, int cols, int64_t ld, const void* tokens, int wide,
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
        alignas(16) TI raw[kAhead][N];                                // (as they lie: registers make warps)
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int c = first + k * lanes * N;
            if (kVector) {
                constexpr int kBytes = N * (int)sizeof(TI);
                if (known && c < cols) {
                    if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(raw[k]) = *reinterpret_cast<const uint2*>(row + c);
                    else
#pragma unroll
                        for (int i16 = 0; i16 < kBytes / 16; ++i16)
                            reinterpret_cast<uint4*>(raw[k])[i16] = reinterpret_cast<const uint4*>(row + c)[i16];
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) raw[k][j] = known && c + j >= 0 && c + j < cols ? row[c + j] : narrow<TI>(0.0f);
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int c = first + k * lanes * N;
            if (c >= cols) break;
            float v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = known ? widen(raw[k][j]) * scale : 0.0f;
            if (kDrop) drop(d, call, (uint64_t)(base + c) / 4, v);
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

// Rows without alignment, behind one another in `out`, which is aligned itself: groups of eight neighbours of the flat output,
// written at once; a group belongs to the row in which it begins, and fetches the elements of the next one by one.
template <typename TI, typename TO, bool kDrop>
__global__ void __launch_bounds__(kThreads, 4)
    flat_lookup_kernel(const TI* table, int64_t vocab, int cols, int64_t ld, const void* tokens, int wide,
                       int64_t n, float scale, TO* __restrict__ out, const Dropout d, int lanes, int each, int spans, int32_t* status) {
    constexpr int kGroups = 2;                                        // in flight
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const int lane = threadIdx.x & (lanes - 1), rows = 32 / lanes;
    const uint64_t call = kDrop ? call_of(d) : 0;
    const uintptr_t lo = (uintptr_t)table, hi = vocab ? (uintptr_t)(table + (vocab - 1) * ld + cols) : lo;
    const int64_t workers = (int64_t)gridDim.x * (kThreads / 32), units = (n + rows - 1) / rows * spans, all = n * cols;
    for (int64_t u = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32; u < units; u += workers) {
        const int64_t i = u / spans * rows + (threadIdx.x & 31) / lanes;
        if (i >= n) continue;
        const int span = (int)(u % spans);
        const int64_t t = token_at(tokens, wide, i);
        const bool known = t >= 0 && t < vocab;
        if (status && t >= vocab && lane == 0 && span == 0) atomicOr(status, SIDCO_EMBEDDING_ST_TOKEN);
        const int64_t base = i * cols;
        const TI* row = table + (known ? t * ld : 0);
        const int first = (int)(-base & 7) + (span * each * lanes + lane) * kEach;
#pragma unroll 1
        for (int k0 = 0; k0 < each; k0 += kGroups) {
            Raw<TI, false> raw[kGroups];
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
                const int c = first + (k0 + k) * lanes * kEach;
                if (known && c < cols && k0 + k < each) raw[k].read(row + c, cols - c, lo, hi);
            }
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
                const int c = first + (k0 + k) * lanes * kEach;
                if (c >= cols || k0 + k >= each) break;
                float v[kEach] = {};
                if (known) raw[k].widened(row + c, v);
                if (c + kEach > cols) {
                    int64_t r = i;
                    int at = c;
                    const TI* from = known ? row : nullptr;
#pragma unroll
                    for (int j = 0; j < kEach; ++j) {
                        while (at >= cols && r < n) {                 // (rows may be shorter than a group)
                            at -= cols;
                            if (++r < n) {
                                const int64_t other = token_at(tokens, wide, r);
                                from = other >= 0 && other < vocab ? table + other * ld : nullptr;
                            }
                        }
                        if (r > i) v[j] = r < n && from ? widen(from[at]) : 0.0f;
                        ++at;
                    }
                }
#pragma unroll
                for (int j = 0; j < kEach; ++j) v[j] *= scale;
                if (kDrop) drop(d, call, (uint64_t)(base + c) / 4, v);
                TO* to = out + base + c;
                if (base + c + kEach <= all) {
                    store(to, v);
                } else {
#pragma unroll
                    for (int j = 0; j < kEach; ++j)
                        if (base + c + j < all) to[j] = narrow<TO>(v[j]);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- sorting
//
// Least significant digit first, nine bits at most per pass.  Items lie in contiguous parts per CTA, and within a CTA per
// warp, so that (CTA, warp, step, lane) is the order of the items and ranking by it is stable.  A pass: every warp counts its
// digits (lanes of one digit find each other by votes), counts become offsets (over warps in shared memory, over the CTAs
// of the cluster in theirs), every warp places its items.  CTAs meet at cluster barriers; nothing spins.
// Padding and tokens outside the table get the largest key and end up behind the others.
// Bound by the writes: 32 items of a warp go to 32 places (key and position apart took twice as long), and by five barriers a
// pass.  65536 tokens of 5003 words 26 us.

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortMost = 16;                                         // CTAs of the sorting cluster
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kParts = kSortThreads / kDigits;
constexpr int kBatch = 8;                                             // steps whose reads are in flight together
constexpr int kSortSmem = kSortWarps * kDigits * 4;

struct Sort {
    const void* tokens;
    int wide;
    uint32_t n;
    int64_t vocab;
    uint2* items[2];                  // (key, position)
    int passes, bits;                 // bits per pass
    int ctas;                         // that sort
    void* fill;                       // gradient to be set to zero, or NULL
    int64_t rows, row_bytes, pitch_bytes;
};

__device__ __forceinline__ uint32_t remote_load4(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}

// Zeros: 16-byte units of a row from its first aligned byte on, single bytes at its ends (rows may have any alignment).
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

// The lanes whose digit is this lane's, by a vote per bit.
__device__ __forceinline__ uint32_t lanes_alike(uint32_t digit, int bits, bool mine) {
    uint32_t same = __ballot_sync(0xffffffffu, mine);
    for (int b = 0; b < bits; ++b) {
        const uint32_t set = __ballot_sync(0xffffffffu, digit >> b & 1);
        same &= digit >> b & 1 ? set : ~set;
    }
    return same;
}

__global__ void __launch_bounds__(kSortThreads) sort_kernel(const Sort s) {
    extern __shared__ uint32_t s_counts[];                            // [warp][digit]: how many, then where its next goes
    __shared__ uint32_t s_total[kDigits];                             // of the CTA
    __shared__ uint32_t s_base[kParts][kDigits];                      // where a part of the warps begins
    __shared__ uint32_t s_warp[kDigits / 32];
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    if ((int)blockIdx.x >= s.ctas) {
        fill_rows(s, (int64_t)blockIdx.x - s.ctas, (int64_t)gridDim.x - s.ctas);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x;
    uint32_t* count = s_counts + warp * kDigits;
    // whole steps of 32 items per warp
    const uint64_t warps = s.ctas * kSortWarps;
    const uint32_t per_warp = (uint32_t)((s.n + warps * 32 - 1) / (warps * 32)) * 32;
    const uint64_t from = (rank * kSortWarps + warp) * (uint64_t)per_warp;
    const uint32_t first = (uint32_t)min(from, (uint64_t)s.n), end = (uint32_t)min(from + per_warp, (uint64_t)s.n);
    const uint32_t mask = (1u << s.bits) - 1;
    for (int pass = 0; pass < s.passes; ++pass) {
        const int shift = pass * s.bits;
        const uint2* items = s.items[pass & 1];
        uint2* to = s.items[(pass & 1) ^ 1];
        uint2 item[kBatch];
        const auto read = [&](uint32_t i0) {
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const uint32_t i = min(i0 + k * 32 + lane, end - 1);
                if (pass) {
                    item[k] = __ldcg(items + i);
                } else {
                    const int64_t t = token_at(s.tokens, s.wide, i);
                    item[k] = make_uint2(t >= 0 && t < s.vocab ? (uint32_t)t : (uint32_t)s.vocab, i);
                }
            }
        };
        for (int i = lane; i < kDigits; i += 32) count[i] = 0;
        __syncwarp();
        for (uint32_t i0 = first; i0 < end; i0 += 32 * kBatch) {
            read(i0);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (i0 + k * 32 >= end) break;
                const bool mine = i0 + k * 32 + lane < end;
                const uint32_t digit = item[k].x >> shift & mask, same = lanes_alike(digit, s.bits, mine);
                if (mine && (same & ((1u << lane) - 1)) == 0) count[digit] += __popc(same);
                __syncwarp();
            }
        }
        __syncthreads();
        // offsets of the warps, by a part of them per thread; totals
        const int digit = threadIdx.x % kDigits, part = threadIdx.x / kDigits;
        {
            uint32_t c[kSortWarps / kParts], sum = 0;
            uint32_t* at = s_counts + part * (kSortWarps / kParts) * kDigits + digit;
#pragma unroll
            for (int w = 0; w < kSortWarps / kParts; ++w) c[w] = at[w * kDigits];
#pragma unroll
            for (int w = 0; w < kSortWarps / kParts; ++w) {
                at[w * kDigits] = sum;
                sum += c[w];
            }
            s_base[part][digit] = sum;
        }
        __syncthreads();
        if (threadIdx.x < kDigits) {
            uint32_t sum = 0;
#pragma unroll
            for (int q = 0; q < kParts; ++q) sum += s_base[q][digit];
            s_total[digit] = sum;
        }
        sidco_tc::cluster_sync();
        uint32_t before = 0;
        if (threadIdx.x < kDigits) {
            uint32_t v[kSortMost], all = 0;                           // this digit in the CTAs before / in all
#pragma unroll
            for (int c = 0; c < kSortMost; ++c) v[c] = c >= s.ctas ? 0 : remote_load4(sidco_tc::in_cta(sidco_tc::smem_addr(s_total + digit), c));
#pragma unroll
            for (int c = 0; c < kSortMost; ++c) {
                if (c < (int)rank) before += v[c];
                all += v[c];
            }
            uint32_t up = all;                                        // digits up to this one: within the warp, then over warps
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t w = __shfl_up_sync(0xffffffffu, up, o);
                if (lane >= o) up += w;
            }
            if (lane == 31) s_warp[warp] = up;
            before += up - all;
        }
        __syncthreads();
        if (threadIdx.x < kDigits) {
            for (int w = 0; w < warp; ++w) before += s_warp[w];
#pragma unroll
            for (int q = 0; q < kParts; ++q) {
                const uint32_t w = s_base[q][digit];
                s_base[q][digit] = before;
                before += w;
            }
        }
        __syncthreads();
        const uint32_t* base = s_base[warp / (kSortWarps / kParts)];
        for (uint32_t i0 = first; i0 < end; i0 += 32 * kBatch) {
            if (per_warp > 32 * kBatch) read(i0);                     // (a single batch is still there)
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (i0 + k * 32 >= end) break;
                const bool mine = i0 + k * 32 + lane < end;
                const uint32_t digit = item[k].x >> shift & mask, same = lanes_alike(digit, s.bits, mine), lower = same & ((1u << lane) - 1);
                const uint32_t next = mine ? count[digit] + __popc(lower) : 0;
                __syncwarp();
                if (mine) {
                    if (lower == 0) count[digit] = next + __popc(same);
                    to[base[digit] + next] = item[k];
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
    const uint2* items;               // sorted (key, position)
    uint32_t n, vocab;
    int cols, chunk;                  // sorted positions per warp, at most 32
    int64_t ld_dy, ldd;
    uintptr_t lo, hi;                 // dy
    float scale;                      // times the dropout's factor
    int add;
    float* partial;                   // [chunks][2][pitch]: of the run that enters a chunk and of the one that leaves it
    int64_t pitch;
};

constexpr int kSlab = 32 * kEach;

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
// run ends behind it, done(k) takes a run's sum (in `sum`) there.  kRows rows come while kRows are added: one where words are
// drawn (that is bound by the generator's products, and its code is there once), four otherwise.
template <int kRows, typename TI, bool kVector, bool kDrop, typename RowAt, typename Ends, typename Done>
__device__ __forceinline__ void add_up(const TI* dy, const Sums& s, const Dropout& d, uint64_t call, int c, int left, int count,
                                       RowAt row_at, Ends ends, Done done, float (&sum)[kEach]) {
    Raw<TI, kVector> now[kRows], next[kRows];
    uint32_t at[kRows], at_next[kRows];
    const auto read = [&](int k) {
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            at_next[j] = row_at(min(k + j, count - 1));
            if (left > 0 && k + j < count) next[j].read(dy + at_next[j] * s.ld_dy + c, left, s.lo, s.hi);
        }
    };
    const int lane = threadIdx.x & 31;
    const bool whole = s.cols % 4 == 0;                               // every row starts a block of the generator
    uint32_t extra[1][4] = {};
    if (count > 0) read(0);
#pragma unroll 1
    for (int k = 0; k < count; k += kRows) {
#pragma unroll
        for (int j = 0; j < kRows; ++j) now[j] = next[j], at[j] = at_next[j];
        read(k + kRows);
        // Where rows start inside a block, a lane's last elements lie in its neighbour's first block, and the last lane's in one
        // that nobody has: lane l draws that one for the l-th of the next 32 rows.
        if (kDrop && !whole && k % 32 == 0)
            random_blocks(d, call, ((uint64_t)row_at(min(k + lane, count - 1)) * s.cols + (c - lane * kEach)) / 4 + 2 * 32, extra);
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            if (k + j >= count) break;
            float v[kEach];
            now[j].widened(dy + at[j] * s.ld_dy + c, v);
            if (kDrop) {                                              // (the factor is part of the scale)
                const uint64_t first = (uint64_t)at[j] * s.cols + c;
                const int shift = (int)(first % 4);                   // (the same for the whole warp)
                uint32_t w[2][4];
                random_blocks(d, call, first / 4, w);
                if (shift) {
                    uint32_t q[kEach + 3];
#pragma unroll
                    for (int e = 0; e < kEach; ++e) q[e] = w[e / 4][e % 4];
#pragma unroll
                    for (int e = 0; e < 3; ++e) {
                        const uint32_t mine = __shfl_sync(0xffffffffu, extra[0][e], (k + j) % 32);
                        q[kEach + e] = __shfl_down_sync(0xffffffffu, w[0][e], 1);
                        if (lane == 31) q[kEach + e] = mine;
                    }
                    if (shift & 1) {
#pragma unroll
                        for (int e = 0; e < kEach + 2; ++e) q[e] = q[e + 1];
                    }
                    if (shift & 2) {
#pragma unroll
                        for (int e = 0; e < kEach; ++e) q[e] = q[e + 2];
                    }
#pragma unroll
                    for (int e = 0; e < kEach; ++e) w[e / 4][e % 4] = q[e];
                }
#pragma unroll
                for (int e = 0; e < kEach; ++e)
                    if (!dropped(d, w[e / 4][e % 4])) sum[e] += v[e];
            } else {
#pragma unroll
                for (int e = 0; e < kEach; ++e) sum[e] += v[e];
            }
            if (ends(k + j)) {
                done(k + j);
#pragma unroll
                for (int e = 0; e < kEach; ++e) sum[e] = 0.0f;
            }
        }
    }
}

template <typename TI, typename TO, bool kVector, bool kDrop>
__global__ void __launch_bounds__(kThreads, kDrop ? 4 : 2)
    sum_kernel(const TI* dy, TO* __restrict__ out, const Sums s, const Dropout d, uint32_t chunks, int slabs, int out_vector) {
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const int lane = threadIdx.x & 31;
    const uint64_t unit = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (unit >= (uint64_t)chunks * slabs) return;
    const uint64_t call = kDrop ? call_of(d) : 0;
    float sum[kEach] = {};
    const uint32_t chunk = (uint32_t)(unit / slabs);
    const int c = (int)(unit % slabs) * kSlab + lane * kEach, left = s.cols - c;
    const uint32_t first = chunk * s.chunk;
    const int count = (int)min((uint32_t)s.chunk, s.n - first);
    // (lane l holds the l-th key and position)
    const uint2 mine = lane < count ? s.items[first + lane] : make_uint2(s.vocab, 0);
    const uint32_t my_key = mine.x, my_at = mine.y;
    const uint32_t before = first ? s.items[first - 1].x : s.vocab;
    const uint32_t behind = first + count < s.n ? s.items[first + count].x : s.vocab;
    const int valid = __popc(__ballot_sync(0xffffffffu, my_key < s.vocab));        // (padding is behind all others)
    if (valid == 0) return;
    uint32_t next = __shfl_down_sync(0xffffffffu, my_key, 1);
    if (lane == count - 1) next = behind;
    const uint32_t ends = __ballot_sync(0xffffffffu, my_key != next);              // a run ends behind position l
    bool entered = __shfl_sync(0xffffffffu, my_key, 0) == before;                  // the run began before this chunk
    float* partial = s.partial + (uint64_t)chunk * 2 * s.pitch + c;
    add_up<kDrop ? 1 : 4, TI, kVector, kDrop>(
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

constexpr int kJoinEach = 4, kJoinSlab = 32 * kJoinEach;              // columns per lane: a long run needs many rows in flight

// A run that leaves the chunk in which it began: its partial sums, one per chunk, in order.
template <typename TO>
__global__ void __launch_bounds__(kThreads, 2) join_kernel(TO* __restrict__ out, const Sums s, uint32_t chunks, int slabs, int out_vector) {
    constexpr int kRows = 16;
    sidco_tc::wait_prerequisites();
    sidco_tc::launch_dependents();
    const uint64_t unit = (uint64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (unit >= (uint64_t)chunks * slabs) return;
    const uint32_t chunk = (uint32_t)(unit / slabs);
    const int lane = threadIdx.x & 31, c = (int)(unit % slabs) * kJoinSlab + lane * kJoinEach, left = s.cols - c;
    const uint32_t first = chunk * s.chunk, next = first + s.chunk;
    if (next >= s.n) return;
    // (all four at once: most warps have nothing to do, and should know it after one trip to memory)
    const uint32_t key = s.items[next - 1].x, behind = s.items[next].x, begin = s.items[first].x,
                   before = first ? s.items[first - 1].x : 0xffffffffu;
    if (key >= s.vocab || behind != key) return;                      // it ends here
    if (begin == key && before == key) return;                        // it began earlier
    // how many of the following chunks it reaches: looked up by 32 lanes at a time
    uint32_t more = 0;
    for (;;) {
        const uint64_t p = (uint64_t)next + (uint64_t)(more + lane) * s.chunk;
        const uint32_t in = __ballot_sync(0xffffffffu, p < s.n && s.items[p].x == key);
        more += in == 0xffffffffu ? 32 : __ffs(~in) - 1;
        if (in != 0xffffffffu) break;
    }
    if (left <= 0) return;
    const float* p = s.partial + (uint64_t)chunk * 2 * s.pitch + c;
    float sum[kJoinEach];
    load(p + s.pitch, sum);
    for (uint32_t k = 1; k <= more; k += kRows) {
        float v[kRows][kJoinEach];
#pragma unroll
        for (int j = 0; j < kRows; ++j) load(p + (uint64_t)min(k + j, more) * 2 * s.pitch, v[j]);
#pragma unroll
        for (int j = 0; j < kRows; ++j)
#pragma unroll
            for (int e = 0; e < kJoinEach; ++e) sum[e] += k + j <= more ? v[j][e] : 0.0f;
    }
    const float whole[kEach] = {sum[0], sum[1], sum[2], sum[3]};
    write_row(s, out + (int64_t)key * s.ldd + c, min(left, kJoinEach), min(out_vector, kJoinEach), whole);
}

// ---------------------------------------------------------------------------------------------- few tokens
//
// Up to kFewMost tokens take one launch: a CTA has a range of the table's rows and a slab of its columns.  It picks its tokens
// out of all, sends zeros to the rows that have none (they leave while it goes on), and ranks its tokens by counting; its warps take equal parts of
// the sorted list, whose runs they join in shared memory where they cross from one part to the next.  Nobody waits for another
// CTA.  (Three launches took 25 us for 700 tokens of 10000 x 1500, this takes 16.)

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
    few_kernel(const TI* dy, TO* out, const Few f, const Sums s, const Dropout d, int slabs, int out_vector) {
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
    add_up<1, TI, kVector, kDrop>(
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
    int64_t items[2], partial, pitch, bytes;
};

static Layout layout_of(int64_t n, int64_t cols) {
    Layout l{};
    if (n <= kFewMost) return l;                                      // (one launch, no lists)
    const int64_t list = (n * 8 + 255) / 256 * 256, chunk = chunk_of(n, cols);
    l.items[0] = 0;
    l.items[1] = list;
    l.partial = 2 * list;
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
    const bool flat = !vector && ldo == cols && (uintptr_t)out % 16 == 0;
    const int64_t groups = vector ? cols / vector : flat ? (cols + 7) / 8 : (cols + 3) / 4 + 1;
    int lanes = 1;
    while (lanes < 32 && lanes < groups) lanes *= 2;
    // (rows without alignment: up to eight groups per lane, as many in every span)
    const int64_t most = flat ? 8 : kAhead, spans = (groups + lanes * most - 1) / (lanes * most), rows = 32 / lanes;
    const int each = (int)((groups + lanes * spans - 1) / (lanes * spans));
    int sms = 0;
    if (const cudaError_t e = sm_count(&sms); e != cudaSuccess) return (int)e;
    // (eight CTAs are resident per SM; four rounds of them even out)
    const dim3 grid((unsigned)std::min<int64_t>(((n + rows - 1) / rows * spans + kThreads / 32 - 1) / (kThreads / 32), 32 * sms));
    const int rc = with_type(table_type, [&](auto* a) {
        return with_type(out_type, [&](auto* b) {
            using TI = std::remove_pointer_t<decltype(a)>;
            using TO = std::remove_pointer_t<decltype(b)>;
            if (flat)
                return (int)launch(on ? flat_lookup_kernel<TI, TO, true> : flat_lookup_kernel<TI, TO, false>, grid, kThreads, 0, s, 1,
                                   (const TI*)table, vocab, (int)cols, ld, tokens, (int)(token_type == SIDCO_T_I64), n, scale,
                                   (TO*)out, d, lanes, each, (int)spans, status);
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
    su.scale = on ? scale * d.factor : scale;
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
        so.items[i] = reinterpret_cast<uint2*>(ws + l.items[i]);
    }
    int bits = 1;
    while ((vocab >> bits) > 0) ++bits;                               // keys 0 .. vocab
    so.passes = (bits + kDigitBits - 1) / kDigitBits;
    so.bits = (bits + so.passes - 1) / so.passes;
    so.fill = add ? nullptr : dtable;
    so.rows = vocab;
    so.row_bytes = cols * size_of(dtable_type);
    so.pitch_bytes = vocab > 1 ? ldd * size_of(dtable_type) : so.row_bytes;
    // Sixteen CTAs sort faster than eight (65536 tokens 25 us instead of 34), but clusters of sixteen leave SMs out, and the
    // zeros, which take longer than the sorting, want all of them (32768 x 2048 of 128000 154 us instead of 161).
    so.ctas = add ? kSortMost : kSortMost / 2;
    const int grid = add ? so.ctas : 2 * sms / so.ctas * so.ctas;
    e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) e = launch(sort_kernel, dim3((unsigned)grid), kSortThreads, kSortSmem, st, so.ctas, so);
    if (e != cudaSuccess) return (int)e;
    sidco_internal::note_launch();

    su.items = so.items[so.passes & 1];
    su.chunk = chunk_of(n, cols);
    su.partial = reinterpret_cast<float*>(ws + l.partial);
    su.pitch = l.pitch;
    const uint32_t chunks = (uint32_t)((n + su.chunk - 1) / su.chunk);
    const int64_t blocks = ((int64_t)chunks * slabs + kThreads / 32 - 1) / (kThreads / 32);
    const int join_slabs = (int)((cols + kJoinSlab - 1) / kJoinSlab);
    const int64_t join_blocks = ((int64_t)chunks * join_slabs + kThreads / 32 - 1) / (kThreads / 32);
    if (join_blocks > 0x7fffffff) return SIDCO_E_SIZE;
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
        return (int)launch(join_kernel<TO>, dim3((unsigned)join_blocks), kThreads, 0, st, 1, (TO*)dtable, su, chunks, join_slabs,
                           out_vector);
    });
    if (rc == 0) sidco_internal::note_launch();
    return rc;
}

}  // extern "C"
