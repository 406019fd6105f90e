// Softmax cross entropy of an output projection, s = scale * X W^T over a large vocabulary, with its gradients.  The products
// run on the tensor cores (bf16 or fp16 operands, fp32 sums in tensor memory).  The logits are never stored; with gradients
// wanted their exponentials are, in 16 bits, for a piece of the rows at a time.
//
//   lse_i = log sum_v exp s_iv;   loss_i = lse_i - s_i,y_i;   total = sum_i c_i loss_i
//   D_iv = c_i scale (exp(s_iv - lse_i) - [v = y_i]);   dX = D W;   dW (+)= D^T X
//
//   prepare_kernel  rows with a label are gathered (the others cost nothing from here on and their contents, NaN included,
//                   reach nothing); W is copied if its rows do not suit tensor copies or its type is another
//   logits_kernel   tiles of X W^T; of each half of a tile's columns the largest logit and the sum of exponentials, and
//                   with gradients e = exp(s - largest) in 16 bits
//   scale_kernel    lse and loss of a row; e becomes D in place; the entry of the label is computed from its fp32 logit
//                   (without gradients loss_kernel: losses only, the last row adds up the total)
//   grads_kernel    dX and dW as one list of tiles, and the total
//   join_kernel     adds the parts of dX where its sums over the vocabulary were split
//
// Why not the logits, or a second product in place of e: e is a relative quantity, so 16 bits cost it half a step of 2^-11
// whatever the size of the logit, and reading and writing it once costs a seventh of computing the
// logits again (0.38 ms against 2.8 ms at 4096 x 128000 x 4096).  What it takes is bounded: rows go in pieces, so that e never takes more than
// 512 MB or what the gradient of W takes in 32 bits, whichever is more; over several pieces dW is summed in fp32.
// D is rounded twice (as e, in fp16, and as D, in the operands' type); dX and dW are sums of such terms in fp32, rounded once
// to their type.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "../../include/sidco.h"
#include "sidco_elements.cuh"
#include "sidco_internal.h"
#include "sidco_tc.cuh"

namespace sidco_ce {

using namespace sidco_tc;
using namespace sidco_elements;

constexpr int kTile = 256;            // rows and columns of a pair's tile
constexpr int kStageK = 64;           // 128 bytes of 16-bit elements
constexpr int kUnit = 64 * 128;       // a box: 64 rows of 128 bytes
constexpr int kStages = 6;
constexpr int kStageBytes = 4 * kUnit;
constexpr int kBox = 32 * 128;        // of an epilogue warp
constexpr int kThreads = 320;
constexpr int kSmem = kStages * kStageBytes + 8 * kBox + 1024;
constexpr int kBand = 16;             // tile rows
constexpr int kMostParts = 16;
constexpr int kPairs = 74;            // of a whole B200: what the split of dX is planned for

struct Head {                         // written by prepare_kernel
    int counted;                      // rows with a label
    float lift, unlift;               // factor that D is stored times, and its inverse
    int done;                         // rows whose loss is known
    int parts;                        // of dX's sums, for the piece at work (scale_kernel)
};

struct Sizes {
    int rows, vocab, hidden;
    int piece, first;                 // rows per piece, first gathered row of this one
};

__device__ int g_timeouts;

template <typename T> constexpr bool kIsHalf = std::is_same<T, __half>::value;
// e is held in fp16 whatever the type of the operands, times 2^14: eleven bits down to 2^-28 of the largest of its half tile,
// nothing below 2^-39.  (In bf16 its rounding would be as large as that of D, and add to it in every entry.)
constexpr float kUp = 14.0f;
// Sums in tensor memory are cut to fp32, not rounded, so that logits come out short by a part that grows with `hidden`: measured
// 0.25 to 0.3 times 2^-24 for every 16 products, from 256 to 16384 products, whether they cancel or not.  The mean of it is put
// back with the scale, at no cost: 4096 products 2.1e-5 off in the mean square -> 4.9e-6 (logits around 4), losses of 4096 x 32000 x 4096
// 1.4e-6 -> 5.3e-7.  That is the share of sums whose terms cancel; of such that only grow more is cut (1.6 times 2^-24 for every
// 16 products), and of a single product nothing: what is put back is then the error, 4.1e-6 of the logit at hidden 4096.  It
// goes no further than 16384 products, 1.65e-5 (at 2^20 it would be 1e-3 of a row whose products are mostly zero).
constexpr double kCut = 0.27 * 0x1p-24 / 16;
constexpr int64_t kCutMost = 16384;

__device__ __forceinline__ int rows_of_piece(const Sizes& z, const Head* head) {
    return max(0, min(z.piece, head->counted - z.first));
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 t = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}

// ---------------------------------------------------------------------------------------------- gathering

constexpr int kPrepareThreads = 256;

struct Prepare {
    const void* x;
    int64_t ldx;
    const void* w;
    int64_t ldw;
    const void* labels;
    int wide;
    const float* weights;
    float scale;
    int rows, vocab, hidden;
    int64_t pitch;                    // elements between rows of the copies
    void* x_to;
    void* w_to;                       // NULL: W is used where it is
    void* dx;                         // NULL: not wanted
    int dx_wide;                      // in fp32
    int64_t lddx;
    float *each, *total;              // NULL: not wanted
    Head* head;
    int *map, *target;
    float* weight;
    int32_t* status;
    int x_blocks, x_rows;             // CTAs for the rows of X, rows of each
    int w_vector, dx_vector;          // rows can be accessed 16 bytes at once
};

// An aligned 16 bytes in elements of kSize, of which some may lie outside [lo, hi): those are not read.
template <int kSize> __device__ __noinline__ uint4 load_edge(uintptr_t at, uintptr_t lo, uintptr_t hi) {
    uint64_t h[2] = {};
#pragma unroll 1
    for (int b = 0; b < 16; b += kSize) {
        const uintptr_t p = at + b;
        uint64_t v = 0;
        if (p >= lo && p < hi) v = kSize == 2 ? *reinterpret_cast<const uint16_t*>(p) : *reinterpret_cast<const uint32_t*>(p);
        if (b < 8) h[0] |= v << (8 * b);
        else h[1] |= v << (8 * (b - 8));
    }
    return make_uint4((uint32_t)h[0], (uint32_t)(h[0] >> 32), (uint32_t)h[1], (uint32_t)(h[1] >> 32));
}

constexpr int kCopyAhead = 4;

// One warp copies a row of 16-bit elements of any alignment to an aligned one whose padding may be written too: aligned
// 16-byte reads, put together from two neighbours.  [lo, hi): the matrix.
__device__ __forceinline__ void copy_bits(const void* from, void* to, int cols, uintptr_t lo, uintptr_t hi, int lane) {
    const uintptr_t start = (uintptr_t)from & ~(uintptr_t)15;
    const int shift = (int)((uintptr_t)from & 15), units = (cols + 7) / 8;
    if (start < lo || start + 16 * (units + 1) > hi) {                // the first and the last row: single elements
        for (int i0 = lane; i0 < cols; i0 += 32 * 16) {
            uint16_t v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = static_cast<const uint16_t*>(from)[min(i0 + k * 32, cols - 1)];
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (i0 + k * 32 < cols) static_cast<uint16_t*>(to)[i0 + k * 32] = v[k];
        }
    } else if (shift) {
        for (int i0 = lane; i0 < units; i0 += 32 * kCopyAhead) {
            uint4 a[kCopyAhead], b[kCopyAhead];                       // (all reads before the first write)
#pragma unroll
            for (int k = 0; k < kCopyAhead; ++k) {
                const int i = min(i0 + k * 32, units - 1);
                a[k] = reinterpret_cast<const uint4*>(start)[i];
                b[k] = reinterpret_cast<const uint4*>(start)[i + 1];
            }
#pragma unroll
            for (int k = 0; k < kCopyAhead; ++k) {
                uint32_t w[8] = {a[k].x, a[k].y, a[k].z, a[k].w, b[k].x, b[k].y, b[k].z, b[k].w};
                shift_words<4>(w, shift);
                if (i0 + k * 32 < units) static_cast<uint4*>(to)[i0 + k * 32] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    } else {
        for (int i0 = lane; i0 < units; i0 += 32 * kCopyAhead) {
            uint4 a[kCopyAhead];
#pragma unroll
            for (int k = 0; k < kCopyAhead; ++k) a[k] = reinterpret_cast<const uint4*>(start)[min(i0 + k * 32, units - 1)];
#pragma unroll
            for (int k = 0; k < kCopyAhead; ++k)
                if (i0 + k * 32 < units) static_cast<uint4*>(to)[i0 + k * 32] = a[k];
        }
    }
}

template <typename T, typename TI>
__device__ __forceinline__ void copy_row(const TI* from, T* to, int cols, bool vector, uintptr_t lo, uintptr_t hi, int lane) {
    if constexpr (std::is_same<T, TI>::value) {
        copy_bits(from, to, cols, lo, hi, lane);
    } else {
        if (vector) {                                                 // four fp32 at a time
            const int whole = cols / 4;
            for (int i0 = lane; i0 < whole; i0 += 32 * kCopyAhead) {
                float4 v[kCopyAhead];
#pragma unroll
                for (int k = 0; k < kCopyAhead; ++k) v[k] = reinterpret_cast<const float4*>(from)[min(i0 + k * 32, whole - 1)];
#pragma unroll
                for (int k = 0; k < kCopyAhead; ++k)
                    if (i0 + k * 32 < whole)
                        reinterpret_cast<uint2*>(to)[i0 + k * 32] = make_uint2(pack2<T>(v[k].x, v[k].y), pack2<T>(v[k].z, v[k].w));
            }
            for (int i = whole * 4 + lane; i < cols; i += 32) to[i] = narrow<T>(from[i]);
        } else {
            for (int i0 = lane; i0 < cols; i0 += 32 * kCopyAhead) {
                float v[kCopyAhead];
#pragma unroll
                for (int k = 0; k < kCopyAhead; ++k) v[k] = from[min(i0 + k * 32, cols - 1)];
#pragma unroll
                for (int k = 0; k < kCopyAhead; ++k)
                    if (i0 + k * 32 < cols) to[i0 + k * 32] = narrow<T>(v[k]);
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ void zero_row(T* to, int cols, bool vector, int lane) {
    const T zero = narrow<T>(0.0f);
    constexpr int kPer = 16 / (int)sizeof(T);
    if (vector) {
        for (int i = lane; i < cols / kPer; i += 32) reinterpret_cast<uint4*>(to)[i] = uint4{};
        for (int i = cols / kPer * kPer + lane; i < cols; i += 32) to[i] = zero;
    } else {
        for (int i = lane; i < cols; i += 32) to[i] = zero;
    }
}

__device__ __forceinline__ bool has_label(int64_t y, int vocab) { return y >= 0 && y < vocab; }

// Sum over the CTA, in all threads.
__device__ __forceinline__ int block_sum(int v, int* s_part) {
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
    __syncthreads();
    int all = 0;
    for (int i = 0; i < kPrepareThreads / 32; ++i) all += s_part[i];
    return all;
}

template <typename T, typename TW>
__global__ void __launch_bounds__(kPrepareThreads) prepare_kernel(const Prepare a) {
    __shared__ int s_part[kPrepareThreads / 32];
    __shared__ uint32_t s_most[kPrepareThreads / 32];
    __shared__ int s_to[kPrepareThreads];                             // where a row goes, or -1
    wait_prerequisites();
    launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((int)blockIdx.x >= a.x_blocks) {
        const int64_t workers = (int64_t)(gridDim.x - a.x_blocks) * (kPrepareThreads / 32);
        for (int64_t r = (int64_t)(blockIdx.x - a.x_blocks) * (kPrepareThreads / 32) + warp; r < a.vocab; r += workers)
            copy_row(static_cast<const TW*>(a.w) + r * a.ldw, static_cast<T*>(a.w_to) + r * a.pitch, a.hidden, a.w_vector,
                     (uintptr_t)a.w, (uintptr_t)(static_cast<const TW*>(a.w) + (a.vocab - 1) * a.ldw + a.hidden), lane);
        return;
    }
    // labelled rows before this CTA's and in all; the largest weight (every CTA counts for itself: nobody waits)
    const int first = min(a.rows, (int)blockIdx.x * a.x_rows), end = min(a.rows, first + a.x_rows);
    int before = 0, all = 0;
    uint32_t most = 0;
    for (int i = threadIdx.x; i < a.rows; i += kPrepareThreads) {
        const bool has = has_label(token_at(a.labels, a.wide, i), a.vocab);
        all += has;
        before += has && i < first;
        if (has && a.weights) most = max(most, __float_as_uint(a.weights[i]) & 0x7fffffffu);
    }
    before = block_sum(before, s_part);
    all = block_sum(all, s_part);
    if (blockIdx.x == 0) {
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) s_most[warp] = most;
        __syncthreads();
        if (threadIdx.x == 0) {
            Head h;
            h.counted = all;
            h.done = 0;
            h.parts = 1;
            if (!all && a.total) *a.total = 0.0f;                     // (otherwise the last row's CTA writes it)
            for (int i = 0; i < kPrepareThreads / 32; ++i) most = max(most, s_most[i]);
            // The largest |c scale| becomes a power of two: rows of that weight, all of them where the weights are equal, have
            // D near -2^k (1 - p) at their labels, which is rounded by less than a half step where p is small (and not by the
            // same amount in every row).  In fp16 2^14, so that D keeps eleven bits down to 2^-28 of it.
            h.lift = h.unlift = 1.0f;
            const float top = fabsf((a.weights ? __uint_as_float(most) : all ? 1.0f / (float)all : 0.0f) * a.scale);
            if (top > 0x1p-100f && top < 0x1p100f) {
                h.lift = (kIsHalf<T> ? 0x1p14f : 1.0f) / top;
                h.unlift = top * (kIsHalf<T> ? 0x1p-14f : 1.0f);
            } else if (kIsHalf<T> && top > 0.0f && top < INFINITY) {
                h.lift = top < 1.0f ? 0x1p100f : 0x1p-100f;
                h.unlift = 1.0f / h.lift;
            }
            *a.head = h;
        }
        // the rows behind the last, up to a whole step of the products over rows
        const int up = (all + kStageK - 1) / kStageK * kStageK;
        for (int r = all + warp; r < up; r += kPrepareThreads / 32)
            zero_row(static_cast<T*>(a.x_to) + r * a.pitch, a.hidden, true, lane);
    }
    for (int r0 = first; r0 < end; r0 += kPrepareThreads) {
        const int r = r0 + threadIdx.x;
        const int64_t y = r < end ? token_at(a.labels, a.wide, r) : -1;
        const bool has = has_label(y, a.vocab);
        if (a.status && y >= a.vocab) atomicOr(a.status, SIDCO_CROSS_ENTROPY_ST_LABEL);
        const uint32_t in = __ballot_sync(0xffffffffu, has);
        __syncthreads();
        if (lane == 0) s_part[warp] = __popc(in);
        __syncthreads();
        int to = before + __popc(in & ((1u << lane) - 1));
        for (int i = 0; i < kPrepareThreads / 32; ++i) {
            if (i < warp) to += s_part[i];
            before += s_part[i];
        }
        s_to[threadIdx.x] = has ? to : -1;
        if (has) {
            a.map[to] = r;
            a.target[to] = (int)y;
            a.weight[to] = a.weights ? a.weights[r] : 1.0f / (float)all;
        } else if (r < end && a.each) {
            a.each[r] = 0.0f;
        }
        __syncthreads();
        for (int i = warp; i < min(kPrepareThreads, end - r0); i += kPrepareThreads / 32) {
            if (s_to[i] >= 0)
                copy_bits(static_cast<const T*>(a.x) + (r0 + i) * a.ldx, static_cast<T*>(a.x_to) + s_to[i] * a.pitch, a.hidden,
                          (uintptr_t)a.x, (uintptr_t)(static_cast<const T*>(a.x) + (a.rows - 1) * a.ldx + a.hidden), lane);
            else if (a.dx && a.dx_wide)
                zero_row(static_cast<float*>(a.dx) + (r0 + i) * a.lddx, a.hidden, a.dx_vector, lane);
            else if (a.dx)
                zero_row(static_cast<T*>(a.dx) + (r0 + i) * a.lddx, a.hidden, a.dx_vector, lane);
        }
    }
}

// ---------------------------------------------------------------------------------------------- products
//
// Tiles of 256 x 256 by pairs of CTAs, each with 128 rows of A and half of B's 256 rows; K in stages of 64; two sets of sums
// in tensor memory, so that the sums of one tile are taken out under the products of the next.
//   warp 0     feeds the stages        warp 1     issues the products (first CTA)
//   warps 2-9  take the sums out: a quarter of the CTA's 128 rows, half of the columns each
// An operand whose rows run along K is K-major; one whose rows run along M or N is read as it lies, MN-major, so that
// no transpose of D, X or W is ever made.
//
// Measured: 4096 x 128000 x 4096 in bf16 10.3 ms in a loop (1.25 PFLOP/s; 1000 W hold the clock at 1.1 GHz; one call alone
// 9.1 ms: logits 2.8, e to D 0.38, gradients 5.8), of which the tensor pipe is busy all the time.  Small ones are bound by whole
// rounds of tiles and by the ways in and out: of 700 x 10000 x 1500 the logits take 25 us, 120 tiles on 74 pairs, two rounds of
// 8 us behind 2 us until the first stage and 4 us for the last sums to leave; the gradients 40 us, of which a tile of dW, eleven
// stages (3.8 us) long, takes 4.5 us to leave.

struct Operand {
    const CUtensorMap* map;
    bool mn;                          // rows of the matrix run along K: a unit is 64 of them, 64 elements of M or N wide
    int row0;                         // added to the matrix's row
};

// One or two units: 64 or 128 M or N indices from `at` on, stage k.
__device__ __forceinline__ void load_operand(uint32_t dst, const Operand& o, int at, int k, int units, uint32_t bar) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (u == units) break;
        if (o.mn) tensor_load_2d_pair(dst + u * kUnit, o.map, (at + u * 64) * 2, o.row0 + k * kStageK, bar);
        else tensor_load_2d_pair(dst + u * kUnit, o.map, k * 128, o.row0 + at + u * 64, bar);
    }
}

template <typename T> __device__ __forceinline__ uint32_t shape_of(bool a_mn, bool b_mn, int width) {
    const uint32_t type = kIsHalf<T> ? 0 : 1;
    return (1u << 4) | (type << 7) | (type << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(width >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
}

struct Job {                          // a tile, or a part of K of one
    Operand a, b;
    int ti, tj, width;                // columns: fewer in the last tile of a row, a multiple of 32
    int from, to;                     // stages
    int kind, part;
    bool dry;                         // the way out is only walked through
};

struct Shared {
    uint64_t full[kStages], free[kStages], sums[2], taken[2];
    uint32_t tmem;
    int failed;
};

__device__ __forceinline__ int width_of(int tj, int columns) { return min(kTile, (columns - tj * kTile + 31) / 32 * 32); }

// The three roles over the jobs that next(it, job) gives; finish(job, sums, row, column, box, take) takes a tile's sums out and
// calls take() when it has read them; ahead(job, row, column) comes before the sums are there.
template <typename T, typename Next, typename Finish, typename Ahead>
__device__ __forceinline__ void run_jobs(Shared& s, uint8_t* smem, Next next, Finish finish, Ahead ahead) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank(), stage0 = smem_addr(smem), tmem = s.tmem;
    Job j;
    if (warp == 0) {
        if (elect_one()) {
            int st = 0;
            uint32_t round = 0;
            bool ok = true;
            for (int it = 0; ok && next(it, j); ++it) {
                // (of B each CTA holds half of the tile's columns)
                const int row_a = j.ti * kTile + (int)rank * 128, row_b = j.tj * kTile + (int)rank * (j.width / 2);
                const int units_b = j.width > 128 ? 2 : 1;
                for (int k = j.from; k < j.to; ++k) {
                    const uint32_t a = stage0 + st * kStageBytes, bar = smem_addr(&s.full[st]);
                    ok = mbar_wait(smem_addr(&s.free[st]), (round & 1) ^ 1, &s.failed);
                    if (!ok) break;
                    if (rank == 0) mbar_expect_tx(bar, 2 * (2 + units_b) * kUnit);
                    load_operand(a, j.a, row_a, k, 2, bar);
                    load_operand(a + 2 * kUnit, j.b, row_b, k, units_b, bar);
                    if (++st == kStages) { st = 0; ++round; }
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {                                              // (the whole warp waits, one thread issues)
            int st = 0;
            uint32_t round = 0;
            bool ok = true;
            for (int it = 0; ok && next(it, j); ++it) {
                const int buf = it & 1;
                const uint32_t sums = tmem + buf * kTile;
                const uint32_t a_step = j.a.mn ? 2048 : 32, a_lead = j.a.mn ? kUnit : 16;
                const uint32_t b_step = j.b.mn ? 2048 : 32, b_lead = j.b.mn ? kUnit : 16;
                const uint32_t shape = shape_of<T>(j.a.mn, j.b.mn, j.width);
                ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&s.taken[buf]), ((it >> 1) & 1) ^ 1, &s.failed));
                for (int k = j.from; k < j.to && ok; ++k) {
                    ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&s.full[st]), round & 1, &s.failed));
                    if (!ok) break;
                    fence_after_sync();
                    const uint32_t a = stage0 + st * kStageBytes, b = a + 2 * kUnit;
                    if (elect_one()) {
#pragma unroll
                        for (int q = 0; q < kStageK / 16; ++q)
                            mma_f16_pair(sums, swizzled_operand(a + q * a_step, a_lead, 1024),
                                         swizzled_operand(b + q * b_step, b_lead, 1024), shape, k > j.from || q > 0);
                        tc_commit_pair(smem_addr(&s.free[st]));
                        if (k + 1 == j.to) tc_commit_pair(smem_addr(&s.sums[buf]));
                    }
                    __syncwarp();
                    if (++st == kStages) { st = 0; ++round; }
                }
            }
        }
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t taken[2] = {in_cta(smem_addr(&s.taken[0]), 0), in_cta(smem_addr(&s.taken[1]), 0)};
        // Before the first sums are there, the way out is walked through once without writing anything: its instructions then
        // lie in the SM's caches when the first tile is done (the first tile took 7 us instead of 4).
        Job coming;
        bool more = next(0, coming);
        for (int it = -1; more; ++it) {
            const int buf = it & 1;
            j = coming;
            j.dry = it < 0;
            if (it >= 0) more = next(it + 1, coming);
            if (it >= 0) ahead(j, (int)rank * 128 + quarter * 32, half * 128);
            if (it >= 0) {
                const bool ok = mbar_wait(smem_addr(&s.sums[buf]), (it >> 1) & 1, &s.failed);
                if (!__all_sync(0xffffffffu, ok)) break;
                fence_after_sync();
            }
            finish(j, tmem + buf * kTile + half * 128 + ((uint32_t)(quarter * 32) << 16), (int)rank * 128 + quarter * 32,
                   half * 128, smem + kStages * kStageBytes + (warp - 2) * kBox, [&] {
                       fence_before_sync();
                       __syncwarp();
                       if (lane == 0 && it >= 0) mbar_arrive_cluster_relaxed(taken[buf]);
                   });
        }
    }
}

__device__ __forceinline__ uint8_t* set_up(Shared& s, uint8_t* raw) {
    const int warp = threadIdx.x >> 5;
    if (warp == 1) tmem_alloc_pair(&s.tmem, 512);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(smem_addr(&s.full[i]), 1);
            mbar_init(smem_addr(&s.free[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&s.sums[i]), 1);
            mbar_init(smem_addr(&s.taken[i]), 16);                    // eight warps of both CTAs
        }
        s.failed = 0;
        mbar_init_fence();
    }
    fence_before_sync();
    __syncthreads();
    cluster_sync();
    fence_after_sync();
    return (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
}

__device__ __forceinline__ void tear_down(Shared& s, int* timeouts) {
    __syncwarp();
    fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s.failed) {
        atomicAdd(timeouts, 1);
        let_work_end();
    }
    __syncthreads();
    cluster_sync();
    if ((threadIdx.x >> 5) == 1) tmem_free_pair(s.tmem, 512);
}

// ---------------------------------------------------------------------------------------------- logits

struct Logits {
    Sizes z;
    const Head* head;
    const int* target;
    float scale2;                     // scale log2(e): logits in powers of two
    float2* stats;                    // [rows of a piece][2 tiles]: largest, sum of 2^(s - largest)
    int tiles_n;
    float* label;                     // logit of the label
    int store;                        // e is wanted
    int* timeouts;
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 1) __cluster_dims__(2)
    logits_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                  const __grid_constant__ CUtensorMap map_e, const Logits g) {
    extern __shared__ uint8_t s_raw[];
    __shared__ Shared s;
    uint8_t* smem = set_up(s, s_raw);
    wait_prerequisites();
    fence_async_all();                                                // (ordinary stores of the kernels before, read by copies)
    launch_dependents();
    const int lane = threadIdx.x & 31;
    const int rows = rows_of_piece(g.z, g.head), tiles_m = (rows + kTile - 1) / kTile, total = tiles_m * g.tiles_n;
    const int n_pairs = gridDim.x / 2, stages = (g.z.hidden + kStageK - 1) / kStageK;
    // tiles in bands of tile rows, column by column, so that pairs at work at the same time share operands in L2: W is read once
    // for each band, whose rows of X stay there
    const auto next = [&](int it, Job& j) {
        const int64_t i = blockIdx.x / 2 + (int64_t)it * n_pairs;
        if (i >= total) return false;
        const int per = kBand * g.tiles_n, band = (int)(i / per), in = (int)(i - (int64_t)band * per), high = min(kBand, tiles_m - band * kBand);
        j = Job{{&map_x, false, g.z.first}, {&map_w, false, 0}, band * kBand + in % high, in / high, width_of(in / high, g.z.vocab), 0, stages,
                0, 0, false};
        return true;
    };
    const auto finish = [&](const Job& j, uint32_t sums, int row_in, int col_in, uint8_t* box, auto take) {
        const int r0 = j.ti * kTile + row_in, r = r0 + lane, c0 = j.tj * kTile + col_in;
        uint32_t acc[128];
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_load32_async(sums + q * 32, *reinterpret_cast<uint32_t(*)[32]>(acc + q * 32));
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_load_wait(*reinterpret_cast<uint32_t(*)[32]>(acc + q * 32));
        take();
        const bool mine = r < rows && !j.dry;
        const int target = mine ? g.target[g.z.first + r] - c0 : -1;
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < 128; ++i) {
            float v = __uint_as_float(acc[i]) * g.scale2;
            if (c0 + 128 > g.z.vocab && c0 + i >= g.z.vocab) v = -INFINITY;
            acc[i] = __float_as_uint(v);
            most = fmaxf(most, v);
        }
        if (__any_sync(0xffffffffu, (unsigned)target < 128u)) {       // a few tiles only
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < 128; ++i)
                if (target == i) v = __uint_as_float(acc[i]);
            if ((unsigned)target < 128u) g.label[r] = v;
        }
        const float base = (most == -INFINITY ? 0.0f : most) - kUp;         // (nothing but -inf: zeros)
        float sum[4] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (g.store) {
                if (lane == 0) bulk_store_wait_read();
                __syncwarp();
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                uint32_t t[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = exp2_fast(__uint_as_float(acc[h * 64 + q * 8 + 2 * i]) - base);
                    const float b = exp2_fast(__uint_as_float(acc[h * 64 + q * 8 + 2 * i + 1]) - base);
                    sum[i] += a + b;
                    t[i] = pack2<__half>(a, b);
                }
                if (g.store)
                    *reinterpret_cast<uint4*>(box + lane * 128 + ((q ^ (lane & 7)) << 4)) = make_uint4(t[0], t[1], t[2], t[3]);
            }
            if (g.store) {
                fence_async_shared();
                __syncwarp();
                if (lane == 0) {
                    if (r0 < rows && c0 + h * 64 < g.z.vocab && !j.dry) tensor_store_2d(&map_e, c0 + h * 64, r0, smem_addr(box));
                    bulk_store_commit();
                }
            }
        }
        if (mine)
            g.stats[(int64_t)r * 2 * g.tiles_n + c0 / 128] =
                make_float2(most, ((sum[0] + sum[1]) + (sum[2] + sum[3])) * 0x1p-14f);
    };
    run_jobs<T>(s, smem, next, finish, [](const Job&, int, int) {});
    if ((threadIdx.x >> 5) >= 2 && lane == 0) bulk_store_wait();
    tear_down(s, g.timeouts);
}

// ---------------------------------------------------------------------------------------------- from e to D

constexpr int kScaleThreads = 256;

struct Scale {
    Sizes z;
    Head* head;
    const int *map, *target;
    const float* weight;
    float scale;
    const float2* stats;
    int tiles_n;
    const float* label;
    void* e;                          // NULL: no gradients
    int64_t pitch;
    float *each, *total;              // NULL: not wanted
    float* share;                     // weight times loss, of the gathered rows
    int64_t part_rows;                // room for parts of dX
    int dw;                           // dW is wanted
};

// Stages that a tile of dW takes: its own, but not fewer than pass while its sums leave (4.5 us; a stage takes 0.35).
__host__ __device__ inline int stages_of_dw(int rows) {
    const int steps = (rows + kStageK - 1) / kStageK;
    return steps > 13 ? steps : 13;
}

// What p parts of dX's sums over the vocabulary cost, in stages of a pair: its longest list of units, or its share of all work,
// and writing and reading the parts (a stage lasts 512 cycles, in which an SM pair moves about 24 KB).
__host__ __device__ inline float cost_of_parts(int p, int rows, int vocab, int hidden, bool dw) {
    const int tiles_m = (rows + kTile - 1) / kTile, tiles_h = (hidden + kTile - 1) / kTile;
    const int steps_v = (vocab + kStageK - 1) / kStageK, steps_r = stages_of_dw(rows);
    const float units = (float)tiles_m * tiles_h * p, unit = (float)((steps_v + p - 1) / p);
    const float work_w = dw ? (float)((vocab + kTile - 1) / kTile) * tiles_h * steps_r : 0.0f;
    const float even = ((float)tiles_m * tiles_h * steps_v + work_w) / kPairs + (dw ? 0.5f * steps_r : 0.0f);
    const float joined = p > 1 ? (float)p * rows * hidden * 8 / kPairs / 24576 + 12 : 0.0f;
    return fmaxf(ceilf(units / kPairs) * unit, even) + joined;
}

__host__ __device__ inline bool parts_fit(int p, int rows, int vocab, int64_t room) {
    return p == 1 || (p <= kMostParts && p <= (vocab + kStageK - 1) / kStageK && (int64_t)p * rows <= room);
}

__device__ __forceinline__ double lanes_sum(double v) {
#pragma unroll
    for (int o = 16; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// log2 of the sum of a row's exponentials, by a whole warp: no barrier, every warp of a row's CTA finds it for itself.
__device__ __forceinline__ float lse2_of(const float2* stats, int parts, int lane) {
    float most = -INFINITY, sum = 0.0f;
    for (int i0 = lane; i0 < parts; i0 += 32 * 4) {
        float2 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = i0 + k * 32 < parts ? stats[i0 + k * 32] : make_float2(-INFINITY, 0.0f);
        float top = most;
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, v[k].x);
        sum *= most == top ? 1.0f : exp2f(most - top);                // (both may be -inf)
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += v[k].x == -INFINITY ? v[k].y : v[k].y * exp2f(v[k].x - top);       // (y is 0 or NaN there)
        most = top;
    }
    float top = most;
#pragma unroll
    for (int o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    sum *= most == top ? 1.0f : exp2f(most - top);
#pragma unroll
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return top + log2f(sum);
}

constexpr float kLn2 = 0.693147180559945f;

// The loss of gathered row r of the piece; one thread.
__device__ __forceinline__ void finish_row(const Scale& a, int r, float weight, float loss) {
    if (a.each) a.each[a.map[a.z.first + r]] = loss;
    a.share[a.z.first + r] = weight * loss;
}

// Without gradients: a warp per row, and the last row to arrive adds up the total.
__global__ void __launch_bounds__(kScaleThreads) loss_kernel(const Scale a) {
    __shared__ double s_sum[kScaleThreads / 32];
    __shared__ int s_last;
    wait_prerequisites();
    launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rows = rows_of_piece(a.z, a.head);
    const int first = blockIdx.x * (kScaleThreads / 32), r = first + warp;
    if (first >= rows) return;
    if (r < rows) {
        const float own = a.label[r], weight = a.weight[a.z.first + r];
        const float lse = lse2_of(a.stats + (int64_t)r * 2 * a.tiles_n, (a.z.vocab + 127) / 128, lane);
        if (lane == 0) finish_row(a, r, weight, (lse - own) * kLn2);
    }
    if (!a.total) return;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        const int mine = min(kScaleThreads / 32, rows - first);       // (all rows of all pieces are counted)
        s_last = atomicAdd(&a.head->done, mine) + mine == a.head->counted;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    double total = 0.0;
    for (int i = threadIdx.x; i < a.head->counted; i += kScaleThreads) total += __ldcg(a.share + i);
    total = lanes_sum(total);
    if (lane == 0) s_sum[warp] = total;
    __syncthreads();
    if (threadIdx.x == 0) {
        total = 0.0;
#pragma unroll
        for (int i = 0; i < kScaleThreads / 32; ++i) total += s_sum[i];
        *a.total = (float)total;
    }
}

template <typename T> __global__ void __launch_bounds__(kScaleThreads) scale_kernel(const Scale a) {
    wait_prerequisites();
    launch_dependents();
    const int rows = rows_of_piece(a.z, a.head), r = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    T* e = static_cast<T*>(a.e) + r * a.pitch;
    // (where there are few rows, several CTAs share one)
    const int all = (a.z.vocab + 7) / 8, share = (all + (int)gridDim.y - 1) / (int)gridDim.y;
    const int from = (int)blockIdx.y * share, vectors = min(all, from + share);
    if (r == 0 && blockIdx.y == 0 && warp == kScaleThreads / 32 - 1) {                   // a lane per number of parts
        const int p = lane + 1;
        const uint32_t cost = parts_fit(p, rows, a.z.vocab, a.part_rows)
                                  ? __float_as_uint(cost_of_parts(p, rows, a.z.vocab, a.z.hidden, a.dw)) : 0xffffffffu;
        const uint32_t least = __reduce_min_sync(0xffffffffu, cost);
        const int best = __ffs(__ballot_sync(0xffffffffu, cost == least));
        if (lane == 0) a.head->parts = best;
    }
    if (r >= rows) {
        if (r < (rows + kStageK - 1) / kStageK * kStageK)
            for (int i = from + threadIdx.x; i < vectors; i += kScaleThreads) reinterpret_cast<uint4*>(e)[i] = uint4{};
        return;
    }
    const float2* stats = a.stats + (int64_t)r * 2 * a.tiles_n;
    // (vectors of the row are read a batch ahead; the first batch comes while its statistics are added up)
    constexpr int kAhead = 4;
    uint4 bits[kAhead];
    const auto read = [&](int i0) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k * kScaleThreads;
            if (i < vectors) bits[k] = reinterpret_cast<const uint4*>(e)[i];
        }
    };
    read(from + threadIdx.x);
    const float own = a.label[r];                                     // in powers of two
    const float weight = a.weight[a.z.first + r], c = weight * a.scale * a.head->lift;
    const int target = a.target[a.z.first + r];
    const float lse = lse2_of(stats, (a.z.vocab + 127) / 128, lane);
    if (threadIdx.x == 0 && blockIdx.y == 0) finish_row(a, r, weight, (lse - own) * kLn2);
    for (int i0 = from + threadIdx.x; i0 < vectors; i0 += kAhead * kScaleThreads) {
        uint4 now[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) now[k] = bits[k];
        read(i0 + kAhead * kScaleThreads);
        float top[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) top[k] = stats[min(i0 + k * kScaleThreads, vectors - 1) / 16].x;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k * kScaleThreads;
            const float f = top[k] == -INFINITY ? c : c * exp2f(top[k] - lse - kUp);
            alignas(16) __half t[8];
            *reinterpret_cast<uint4*>(t) = now[k];
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = widen(t[j]) * f;
            if (target / 8 == i) {
                const float d = c * expm1f((own - lse) * kLn2);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (target % 8 == j) v[j] = d;
            }
            if (i < vectors) store(e + i * 8, v);
        }
    }
}

// ---------------------------------------------------------------------------------------------- gradients

struct Grads {
    Sizes z;
    const Head* head;
    const int* map;
    void* dx;                         // NULL: not wanted
    int64_t lddx;
    float* dx_parts;                  // [parts][labelled rows of the piece][pitch], where the sums over the vocabulary are split
    void* dw;                         // NULL: not wanted
    int64_t lddw;
    int add;
    float* dw_sums;                   // [vocab][pitch], over pieces
    int more, last;                   // not the first piece, the last piece
    const float* share;
    float* total;                     // NULL: not wanted
    int64_t pitch;
    int dx_unit, dw_unit;             // bytes that rows are aligned to, at most 16
    int* timeouts;
};

// The way out of a warp's 32 rows x 128 columns of sums: a lane has a row; rounded to their type, 128 bytes of each row go
// through shared memory (a box, its 16-byte units swizzled by row), so that neighbouring lanes write neighbouring bytes.
// They are rounded before because the bandwidth of shared memory, which the operands of the products share, bounds this; and
// what they are added to is read by the lane that has the row, all of it before the first use (behind a branch per element,
// or between the writes, every read would wait for the one before).

__device__ __forceinline__ const uint8_t* in_box(const uint8_t* box, int r, int byte) {
    return box + r * 128 + (((byte >> 4) ^ (r & 7)) << 4) + (byte & 15);
}

// A box to rows of `out` (at the first of its columns) of which `left` columns exist.  row: of this lane, or -1.
// unit: 16 or 8 bytes that rows are aligned to, or less.
template <typename TO>
__device__ __forceinline__ void put_box(const uint8_t* box, int row, TO* out, int64_t ld, int left, int unit) {
    constexpr int kSize = (int)sizeof(TO), kCols = 128 / kSize, kEdge = 16 / kSize;
    const int lane = threadIdx.x & 31;
    if (left < kCols) {                                               // the last columns: single elements
#pragma unroll 4
        for (int i = lane; i < 32 * kCols; i += 32) {
            const int r = i / kCols, c = i % kCols, at = __shfl_sync(0xffffffffu, row, r);
            if (at >= 0 && c < left) out[at * ld + c] = *reinterpret_cast<const TO*>(in_box(box, r, c * kSize));
        }
    } else if (unit == 16) {
        uint4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const uint4*>(in_box(box, i * 4 + lane / 8, lane % 8 * 16));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = __shfl_sync(0xffffffffu, row, i * 4 + lane / 8);
            if (at >= 0) reinterpret_cast<uint4*>(out + at * ld)[lane % 8] = v[i];
        }
    } else if (unit == 8) {
        uint2 v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = *reinterpret_cast<const uint2*>(in_box(box, i * 2 + lane / 16, lane % 16 * 8));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = __shfl_sync(0xffffffffu, row, i * 2 + lane / 16);
            if (at >= 0) reinterpret_cast<uint2*>(out + at * ld)[lane % 16] = v[i];
        }
    } else {
        // the aligned 16-byte units inside the row's 128 bytes, then the elements before and behind them (none, or 16 bytes)
#pragma unroll 1
        for (int i0 = 0; i0 < 8; i0 += 4) {
            uint32_t w[4][8];
            uint8_t* to[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = (i0 + i) * 4 + lane / 8, at = __shfl_sync(0xffffffffu, row, r);
                to[i] = reinterpret_cast<uint8_t*>(out + at * ld);
                const int b = (int)(-(uintptr_t)to[i] & 15) + lane % 8 * 16;
                to[i] = at >= 0 && b + 16 <= 128 ? to[i] + b : nullptr;
                const uint4 lo = *reinterpret_cast<const uint4*>(in_box(box, r, b & 0x70));
                const uint4 hi = *reinterpret_cast<const uint4*>(in_box(box, r, (b + 16) & 0x70));
                w[i][0] = lo.x, w[i][1] = lo.y, w[i][2] = lo.z, w[i][3] = lo.w;
                w[i][4] = hi.x, w[i][5] = hi.y, w[i][6] = hi.z, w[i][7] = hi.w;
                shift_words<4>(w[i], b & 15);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (to[i]) *reinterpret_cast<uint4*>(to[i]) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
        }
        TO edge[kEdge];
#pragma unroll
        for (int i = 0; i < kEdge; ++i) {
            const int r = (i * 32 + lane) / kEdge, at = __shfl_sync(0xffffffffu, row, r);
            const int front = (int)(-(uintptr_t)(out + at * ld) & 15), e = lane % kEdge * kSize;
            edge[i] = *reinterpret_cast<const TO*>(in_box(box, r, e < front ? e : 112 + e));
        }
#pragma unroll
        for (int i = 0; i < kEdge; ++i) {
            const int at = __shfl_sync(0xffffffffu, row, (i * 32 + lane) / kEdge);
            uint8_t* to = reinterpret_cast<uint8_t*>(out + at * ld);
            const int front = (int)(-(uintptr_t)to & 15), e = lane % kEdge * kSize;
            if (at >= 0 && front) *reinterpret_cast<TO*>(to + (e < front ? e : 112 + e)) = edge[i];
        }
    }
}

struct Added {
    bool out;                         // what `out` holds is added after the factor; it lies in [lo, hi)
    uintptr_t lo, hi;
    const float* sums;                // added before the factor, aligned; or NULL
    int64_t pitch;
};

template <typename TO, typename Take>
__device__ __forceinline__ void put_tile(uint32_t tmem, uint8_t* box, int row, TO* out, int64_t ld, int left, float factor, int unit,
                                         const Added& more, Take take) {
    constexpr int kSize = (int)sizeof(TO), kCols = 128 / kSize, kSteps = 128 / kCols;
    const int lane = threadIdx.x & 31;
    uint32_t old[36];
    const auto read_old = [&](int q) {
        const uintptr_t first = (uintptr_t)(out + max(row, 0) * ld + q * kCols), start = first & ~(uintptr_t)15;
        if (__all_sync(0xffffffffu, start >= more.lo && start + 144 <= more.hi)) {
#pragma unroll
            for (int i = 0; i < 9; ++i) {
                const uint4 v = reinterpret_cast<const uint4*>(start)[i];
                old[i * 4] = v.x, old[i * 4 + 1] = v.y, old[i * 4 + 2] = v.z, old[i * 4 + 3] = v.w;
            }
        } else {                                                      // at the ends of the matrix
#pragma unroll
            for (int i = 0; i < 9; ++i) {
                const uint4 v = load_edge<kSize>(start + 16 * i, more.lo, more.hi);
                old[i * 4] = v.x, old[i * 4 + 1] = v.y, old[i * 4 + 2] = v.z, old[i * 4 + 3] = v.w;
            }
        }
    };
#pragma unroll 1
    for (int q = 0; q < kSteps; ++q) {
        const int here = left - q * kCols;
        if (more.out && here > 0) read_old(q);
        uint32_t acc[kCols];
#pragma unroll
        for (int i = 0; i < kCols / 32; ++i)
            tmem_load32(tmem + q * kCols + i * 32, *reinterpret_cast<uint32_t(*)[32]>(acc + i * 32));
        if (q + 1 == kSteps) take();
        if (here <= 0) continue;
        if (more.sums) {
            const float4* from = reinterpret_cast<const float4*>(more.sums + max(row, 0) * more.pitch + q * kCols);
#pragma unroll
            for (int i = 0; i < kCols / 4; ++i) {
                const float4 v = from[i];
                acc[i * 4] = __float_as_uint(__uint_as_float(acc[i * 4]) + v.x);
                acc[i * 4 + 1] = __float_as_uint(__uint_as_float(acc[i * 4 + 1]) + v.y);
                acc[i * 4 + 2] = __float_as_uint(__uint_as_float(acc[i * 4 + 2]) + v.z);
                acc[i * 4 + 3] = __float_as_uint(__uint_as_float(acc[i * 4 + 3]) + v.w);
            }
        }
#pragma unroll
        for (int i = 0; i < kCols; ++i) acc[i] = __float_as_uint(__uint_as_float(acc[i]) * factor);
        if (more.out) {
            if (unit < 16) shift_words<32>(old, (int)((uintptr_t)(out + max(row, 0) * ld + q * kCols) & 15));
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                if constexpr (kSize == 4) {
                    acc[i] = __float_as_uint(__uint_as_float(acc[i]) + __uint_as_float(old[i]));
                } else {
                    const TO* t = reinterpret_cast<const TO*>(&old[i]);
                    acc[2 * i] = __float_as_uint(__uint_as_float(acc[2 * i]) + widen(t[0]));
                    acc[2 * i + 1] = __float_as_uint(__uint_as_float(acc[2 * i + 1]) + widen(t[1]));
                }
            }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (kSize == 4) t[j] = acc[i * 4 + j];
                else t[j] = pack2<TO>(__uint_as_float(acc[i * 8 + 2 * j]), __uint_as_float(acc[i * 8 + 2 * j + 1]));
            }
            *reinterpret_cast<uint4*>(box + lane * 128 + ((i ^ (lane & 7)) << 4)) = make_uint4(t[0], t[1], t[2], t[3]);
        }
        __syncwarp();
        put_box(box, row, out + q * kCols, ld, here, unit);
    }
}

template <typename T, typename TW, typename TX>
__global__ void __launch_bounds__(kThreads, 1) __cluster_dims__(2)
    grads_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                 const __grid_constant__ CUtensorMap map_d, const Grads g) {
    extern __shared__ uint8_t s_raw[];
    __shared__ Shared s;
    uint8_t* smem = set_up(s, s_raw);
    wait_prerequisites();
    fence_async_all();                                                // (ordinary stores of the kernels before, read by copies)
    launch_dependents();
    const int lane = threadIdx.x & 31;
    const int rows = rows_of_piece(g.z, g.head), tiles_m = (rows + kTile - 1) / kTile;
    const int tiles_h = (g.z.hidden + kTile - 1) / kTile, tiles_v = (g.z.vocab + kTile - 1) / kTile;
    const int n_pairs = gridDim.x / 2, pair = blockIdx.x / 2;
    const int steps_v = (g.z.vocab + kStageK - 1) / kStageK, steps_r = (rows + kStageK - 1) / kStageK;
    const float unlift = g.head->unlift;
    const int parts = g.head->parts;
    // dX first, its long sums split into parts, then dW.  Where the units of dX do not come out even, the pairs with one
    // less take as many tiles of dW ahead of the others as last as long.
    const int per_part = tiles_m * tiles_h, n_dx = g.dx ? per_part * parts : 0, n_dw = g.dw && steps_r ? tiles_v * tiles_h : 0;
    const int heavy = n_dx % n_pairs, light = n_pairs - heavy, units = n_dx / n_pairs + (pair < heavy);
    const int ahead = heavy ? steps_v / parts / stages_of_dw(rows) : 0;
    const int early = (int)min((int64_t)n_dw, (int64_t)ahead * light);
    const int my_early = pair < heavy ? 0 : max(0, (early - (pair - heavy) + light - 1) / light);
    const auto next = [&](int it, Job& j) {
        if (it < units) {
            const int u = it * n_pairs + pair, part = u / per_part, t = u - part * per_part;
            j = Job{{&map_d, false, 0}, {&map_w, true, 0}, t % tiles_m, t / tiles_m, width_of(t / tiles_m, g.z.hidden),
                    (int)((int64_t)steps_v * part / parts), (int)((int64_t)steps_v * (part + 1) / parts), 0, part, false};
            return true;
        }
        it -= units;
        const int t = it < my_early ? pair - heavy + it * light : early + (it - my_early) * n_pairs + pair;
        if (t >= n_dw) return false;
        j = Job{{&map_d, true, 0}, {&map_x, true, g.z.first}, t / tiles_h, t % tiles_h, width_of(t % tiles_h, g.z.hidden), 0, steps_r,
                1, 0, false};
        return true;
    };
    const auto finish = [&](const Job& j, uint32_t sums, int row_in, int col_in, uint8_t* box, auto take) {
        const int r = j.ti * kTile + row_in + lane, col = j.tj * kTile + col_in, left = g.z.hidden - col;
        const bool is_dx = j.kind == 0, split = is_dx && parts > 1;
        if (left <= 0) {
            take();
            return;
        }
        const int row = j.dry || r >= (is_dx ? rows : g.z.vocab) ? -1 : is_dx && !split ? g.map[g.z.first + r] : r;
        // (rows of the workspace are whole: their columns do not end inside a step)
        if (split || (!is_dx && !g.last)) {
            float* out = split ? g.dx_parts + (int64_t)j.part * rows * g.pitch : g.dw_sums;
            const Added more{false, 0, 0, !is_dx && g.more ? out + col : nullptr, g.pitch};
            put_tile(sums, box, row, out + col, g.pitch, (int)g.pitch - col, 1.0f, 16, more, take);
        } else if (is_dx) {
            put_tile(sums, box, row, static_cast<TX*>(g.dx) + col, g.lddx, left, unlift, g.dx_unit, Added{}, take);
        } else {
            TW* out = static_cast<TW*>(g.dw);
            const Added more{g.add != 0, (uintptr_t)out, (uintptr_t)(out + (g.z.vocab - 1) * g.lddw + g.z.hidden),
                             g.more ? g.dw_sums + col : nullptr, g.pitch};
            put_tile(sums, box, row, out + col, g.lddw, left, unlift, g.dw_unit, more, take);
        }
    };
    // what a tile of dW is added to is brought into L2 while its products run (a tile earlier it was slower)
    const auto ahead_of = [&](const Job& j, int row_in, int col_in) {
        const int r = j.ti * kTile + row_in + lane, col = j.tj * kTile + col_in, left = min(128, g.z.hidden - col);
        if (j.kind == 0 || !g.add || !g.last || r >= g.z.vocab || left <= 0) return;
        const TW* at = static_cast<const TW*>(g.dw) + r * g.lddw + col;
        for (int c = 0; c < left; c += 128 / (int)sizeof(TW)) prefetch_l2(at + c);
        prefetch_l2(at + left - 1);
    };
    // the total, by a warp that has nothing to issue: the 256 sums that loss_kernel's last CTA would take, eight to a lane
    if (blockIdx.x == 1 && threadIdx.x / 32 == 1 && g.last && g.total && g.head->counted) {
        double sum[8] = {}, total = 0.0;
        for (int i = lane; i < g.head->counted; i += 256)
#pragma unroll
            for (int w = 0; w < 8; ++w)
                if (i + w * 32 < g.head->counted) sum[w] += g.share[i + w * 32];
#pragma unroll
        for (int w = 0; w < 8; ++w) total += lanes_sum(sum[w]);
        if (lane == 0) *g.total = (float)total;
        __syncwarp();
    }
    run_jobs<T>(s, smem, next, finish, ahead_of);
    // a piece without rows has no products: what the pieces before have left, or nothing, is still the gradient
    if (g.dw && steps_r == 0 && (g.last || !g.more)) {
        TW* out = static_cast<TW*>(g.dw);
        for (int64_t r = blockIdx.x; r < g.z.vocab; r += gridDim.x)
            for (int c = threadIdx.x; c < g.z.hidden; c += kThreads) {
                const float v = g.more ? g.dw_sums[r * g.pitch + c] : 0.0f;
                TW* to = out + r * g.lddw + c;
                if (!g.last) g.dw_sums[r * g.pitch + c] = v;
                else if (g.add) { if (g.more) *to = narrow<TW>(widen(*to) + v * unlift); }
                else *to = narrow<TW>(v * unlift);
            }
    }
    tear_down(s, g.timeouts);
}

// ---------------------------------------------------------------------------------------------- joining

constexpr int kJoinThreads = 256;

// dX = the parts of its sums, in order (where they are one part after all, it has nothing to do: few CTAs).
template <typename TX>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const Grads g) {
    wait_prerequisites();
    launch_dependents();
    const int rows = rows_of_piece(g.z, g.head), parts = g.head->parts;
    if (parts == 1) return;
    const float unlift = g.head->unlift;
    const int fours = (g.z.hidden + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x; i < (int64_t)rows * fours; i += (int64_t)gridDim.x * kJoinThreads) {
        const int r = (int)(i / fours), c = (int)(i % fours) * 4;
        const float* p = g.dx_parts + (int64_t)r * g.pitch + c;
        float v[4] = {};
        for (int k0 = 0; k0 < parts; k0 += 4) {
            float o[4][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) load(p + (int64_t)min(k0 + k, parts - 1) * rows * g.pitch, o[k]);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += k0 + k < parts ? o[k][j] : 0.0f;
        }
        TX* out = static_cast<TX*>(g.dx) + g.map[g.z.first + r] * g.lddx + c;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= unlift;
        if (g.dx_unit >= 4 * (int)sizeof(TX) && c + 4 <= g.z.hidden) {
            store(out, v);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < g.z.hidden) out[j] = narrow<TX>(v[j]);
        }
    }
}

// ---------------------------------------------------------------------------------------------- host side

constexpr int64_t kMostRows = (int64_t)1 << 28, kMostVocab = (int64_t)1 << 28, kMostHidden = (int64_t)1 << 20;

static int64_t up_to(int64_t n, int64_t step) { return (n + step - 1) / step * step; }

struct Plan {
    int64_t pitch, e_pitch;           // of the copies of X and W, of e
    int64_t piece, pieces, tiles_n;
    int64_t part_rows;                // room for the parts of dX: rows of any part
    int64_t head, map, target, weight, share, label, stats, x, w, e, dx_parts, dw_sums, bytes;
    bool countable;                   // its tiles can be counted in 31 bits
};

static Plan plan_of(int64_t rows, int64_t vocab, int64_t hidden, int grads, bool copy_w, int64_t piece_rows) {
    Plan p{};
    p.pitch = up_to(hidden, 64);
    p.e_pitch = up_to(vocab, 64);
    p.tiles_n = (vocab + kTile - 1) / kTile;
    if (piece_rows > 0) p.piece = up_to(piece_rows, kTile);
    else p.piece = std::max<int64_t>(kTile, std::max<int64_t>((int64_t)1 << 29, grads & 2 ? vocab * p.pitch * 4 : 0) / (p.e_pitch * 2) / kTile * kTile);
    if (!grads && piece_rows <= 0)                                     // (only the statistics: 16 bytes per tile and row)
        p.piece = std::max<int64_t>(kTile, ((int64_t)1 << 29) / (p.tiles_n * 16) / kTile * kTile);
    p.piece = std::min(p.piece, up_to(rows, kTile));
    p.pieces = (rows + p.piece - 1) / p.piece;
    // how many rows have a label is known on the device only, and with it the number of parts: room for what any number of
    // rows takes (sixteen are looked at)
    for (int i = 1; grads & 1 && i <= 16; ++i) {
        const int64_t some = std::min(rows, std::max<int64_t>(1, std::min(rows, p.piece) * i / 16));
        int parts = 1;
        for (int n = 2; parts_fit(n, (int)some, (int)vocab, (int64_t)1 << 60); ++n)
            if (cost_of_parts(n, (int)some, (int)vocab, (int)hidden, grads & 2) <
                cost_of_parts(parts, (int)some, (int)vocab, (int)hidden, grads & 2))
                parts = n;
        if (parts > 1) p.part_rows = std::max(p.part_rows, parts * some);
    }
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up_to(bytes, 256);
        return here;
    };
    p.head = take(sizeof(Head));
    p.map = take(rows * 4);
    p.target = take(rows * 4);
    p.weight = take(rows * 4);
    p.share = take(rows * 4);
    p.label = take(p.piece * 4);
    p.stats = take(p.piece * p.tiles_n * 16);
    p.x = take(up_to(rows, kStageK) * p.pitch * 2);
    p.w = take(copy_w ? vocab * p.pitch * 2 : 0);
    p.e = take(grads ? p.piece * p.e_pitch * 2 : 0);
    p.dx_parts = take(p.part_rows * p.pitch * 4);
    p.dw_sums = take(grads & 2 && p.pieces > 1 ? vocab * p.pitch * 4 : 0);
    p.bytes = at;
    const int64_t most = (int64_t)1 << 30, tiles_h = (hidden + kTile - 1) / kTile, tiles_m = p.piece / kTile;
    p.countable = tiles_m <= most / p.tiles_n && tiles_h <= most / p.tiles_n && tiles_m <= most / (tiles_h * kMostParts);
    return p;
}

static int check(int64_t rows, int64_t vocab, int64_t hidden, int64_t piece_rows) {
    return rows < 0 || vocab < 0 || hidden < 0 || rows > kMostRows || vocab > kMostVocab || hidden > kMostHidden ||
                   piece_rows < 0 || piece_rows > kMostRows
               ? SIDCO_E_SIZE
               : 0;
}

// W cannot be read in place by tensor copies.
static bool needs_copy(const void* w, int w_type, int64_t ldw, int type) {
    return w_type != type || (uintptr_t)w % 16 || ldw * 2 % 16;
}

// Bytes, 16 at most, that all rows are aligned to.
static int unit_of(const void* p, int64_t ld, int type) {
    int n = 16;
    while (n > 1 && ((uintptr_t)p % (uintptr_t)n || ld * size_of(type) % n)) n /= 2;
    return n;
}

template <typename T, typename TW, typename TX> static cudaError_t prepare_device(int* pairs) {
    const auto most = cudaFuncAttributeMaxDynamicSharedMemorySize;
    cudaError_t e;
    if ((e = cudaFuncSetAttribute(logits_kernel<T>, most, kSmem)) != cudaSuccess ||
        (e = cudaFuncSetAttribute(grads_kernel<T, TW, TX>, most, kSmem)) != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(pairs, grads_kernel<T, TW, TX>, &cfg);
    return e == cudaSuccess && *pairs < 1 ? cudaErrorInvalidConfiguration : e;
}

struct Call {
    const void* x;
    int type;
    int64_t ldx;
    const void* w;
    int w_type;
    int64_t ldw;
    const void* labels;
    int label_type;
    const float* weights;
    float scale;
    int64_t rows, vocab, hidden;
    float *each, *total;
    void* dx;
    int dx_type;
    int64_t lddx;
    void* dw;
    int dw_type;
    int64_t lddw;
    int add;
    int32_t* status;
    uint8_t* ws;
    cudaStream_t s;
};

#define SIDCO_CE_LAUNCH(...)                                     \
    do {                                                         \
        const cudaError_t e_ = launch(__VA_ARGS__);              \
        if (e_ != cudaSuccess) return (int)e_;                   \
        sidco_internal::note_launch();                           \
    } while (0)

template <typename T, typename TW, typename TX> static int run(const Call& c, const Plan& p, bool copy_w) {
    static std::atomic<int> pairs_of[64];
    int dev = 0, sms = 0, *timeouts = nullptr;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return (int)e;
    if (dev < 0 || dev >= 64) return SIDCO_E_SIZE;
    if (!pairs_of[dev].load()) {             // (setting it twice from two threads is harmless)
        int n = 0;
        if ((e = prepare_device<T, TW, TX>(&n)) != cudaSuccess) return (int)e;
        pairs_of[dev].store(n);
    }
    const int pairs = pairs_of[dev].load();
    if ((e = cudaGetSymbolAddress((void**)&timeouts, g_timeouts)) != cudaSuccess ||
        (e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess)
        return (int)e;
    Head* head = reinterpret_cast<Head*>(c.ws + p.head);
    int *map = reinterpret_cast<int*>(c.ws + p.map), *target = reinterpret_cast<int*>(c.ws + p.target);
    float* weight = reinterpret_cast<float*>(c.ws + p.weight);
    const void* w = copy_w ? c.ws + p.w : c.w;
    const int64_t w_pitch = copy_w || c.vocab == 1 ? p.pitch : c.ldw;  // (a single row may have any distance)
    const bool grads = c.dx || c.dw;
    // (before the first launch: what they refuse leaves the outputs as they were)
    CUtensorMap map_x, map_w, map_e{}, map_d{};
    if (!sidco_internal::byte_map(&map_x, c.ws + p.x, c.hidden * 2, up_to(c.rows, kStageK), p.pitch * 2, 128, 64, true) ||
        !sidco_internal::byte_map(&map_w, w, c.hidden * 2, c.vocab, w_pitch * 2, 128, 64, true) ||
        (grads && (!sidco_internal::out_map(&map_e, c.ws + p.e, c.type, p.e_pitch, p.piece, p.e_pitch, 64, 32) ||
                   !sidco_internal::byte_map(&map_d, c.ws + p.e, c.vocab * 2, p.piece, p.e_pitch * 2, 128, 64, true))))
        return SIDCO_E_UNSUPPORTED;

    Prepare a{};
    a.x = c.x, a.ldx = c.ldx, a.w = c.w, a.ldw = c.ldw, a.labels = c.labels, a.wide = c.label_type == SIDCO_T_I64;
    a.weights = c.weights, a.scale = c.scale;
    a.rows = (int)c.rows, a.vocab = (int)c.vocab, a.hidden = (int)c.hidden, a.pitch = p.pitch;
    a.x_to = c.ws + p.x, a.w_to = copy_w ? c.ws + p.w : nullptr;
    a.dx = c.dx, a.dx_wide = c.dx_type == SIDCO_T_F32, a.lddx = c.lddx, a.each = c.each, a.total = c.total;
    a.head = head, a.map = map, a.target = target, a.weight = weight;
    a.status = c.status;
    a.x_blocks = (int)std::min<int64_t>(c.rows, sms), a.x_rows = (int)((c.rows + a.x_blocks - 1) / a.x_blocks);
    a.w_vector = unit_of(c.w, c.ldw, c.w_type) == 16, a.dx_vector = unit_of(c.dx, c.lddx, c.dx_type) == 16;
    const unsigned blocks = (unsigned)(a.x_blocks + (copy_w ? std::min<int64_t>((c.vocab + 7) / 8, 16 * sms) : 0));
    if (c.w_type == SIDCO_T_F32) SIDCO_CE_LAUNCH(prepare_kernel<T, float>, dim3(blocks), kPrepareThreads, 0, c.s, 1, a);
    else SIDCO_CE_LAUNCH(prepare_kernel<T, T>, dim3(blocks), kPrepareThreads, 0, c.s, 1, a);

    float* share = reinterpret_cast<float*>(c.ws + p.share);
    const float scale2 = (float)(c.scale * 1.4426950408889634 * (1 + kCut * std::min(c.hidden, kCutMost)));
    for (int64_t i = 0; i < p.pieces; ++i) {
        const Sizes z{(int)c.rows, (int)c.vocab, (int)c.hidden, (int)p.piece, (int)(i * p.piece)};
        const int64_t most = std::min(p.piece, c.rows - z.first);      // rows if all have labels
        Logits l{z, head, target, scale2, reinterpret_cast<float2*>(c.ws + p.stats), (int)p.tiles_n,
                 reinterpret_cast<float*>(c.ws + p.label), grads, timeouts};
        const int64_t tiles = (most + kTile - 1) / kTile * p.tiles_n;
        SIDCO_CE_LAUNCH(logits_kernel<T>, dim3((unsigned)(2 * std::min<int64_t>(pairs, tiles))), kThreads, kSmem, c.s, 1, map_x,
                        map_w, map_e, l);
        Scale k{z, head, map, target, weight, c.scale, l.stats, l.tiles_n, l.label, grads ? c.ws + p.e : nullptr, p.e_pitch,
                c.each, c.total, share, p.part_rows, c.dw != nullptr};
        if (!grads) {
            SIDCO_CE_LAUNCH(loss_kernel, dim3((unsigned)((most + 7) / 8)), kScaleThreads, 0, c.s, 1, k);
            continue;
        }
        const int64_t shares = std::max<int64_t>(1, std::min(4 * sms / up_to(most, kStageK), c.vocab / (8 * 4 * kScaleThreads)));
        SIDCO_CE_LAUNCH(scale_kernel<T>, dim3((unsigned)up_to(most, kStageK), (unsigned)shares), kScaleThreads, 0, c.s, 1, k);
        Grads g{z, head, map, c.dx, c.lddx, reinterpret_cast<float*>(c.ws + p.dx_parts), c.dw, c.lddw, c.add,
                reinterpret_cast<float*>(c.ws + p.dw_sums), i > 0, i + 1 == p.pieces, share, c.total, p.pitch,
                unit_of(c.dx, c.lddx, c.dx_type), unit_of(c.dw, c.lddw, c.dw_type), timeouts};
        SIDCO_CE_LAUNCH((grads_kernel<T, TW, TX>), dim3(2 * (unsigned)pairs), kThreads, kSmem, c.s, 1, map_x, map_w, map_d, g);
        if (c.dx && p.part_rows)
            SIDCO_CE_LAUNCH(join_kernel<TX>, dim3((unsigned)std::min<int64_t>((most * ((c.hidden + 3) / 4) + kJoinThreads - 1) / kJoinThreads, 8 * sms)),
                            kJoinThreads, 0, c.s, 1, g);
    }
    return 0;
}

template <typename T> static int run(const Call& c, const Plan& p, bool copy_w) {
    const bool wide_x = c.dx && c.dx_type == SIDCO_T_F32;
    if (c.dw && c.dw_type == SIDCO_T_F32) return wide_x ? run<T, float, float>(c, p, copy_w) : run<T, float, T>(c, p, copy_w);
    return wide_x ? run<T, T, float>(c, p, copy_w) : run<T, T, T>(c, p, copy_w);
}

}  // namespace sidco_ce

int sidco_internal::cross_entropy_timeouts(int* count) {
    return (int)cudaMemcpyFromSymbol(count, sidco_ce::g_timeouts, sizeof(int));
}

extern "C" {

int64_t sidco_linear_cross_entropy_workspace_bytes(const void* w, int type, int w_type, int64_t ldw, int64_t rows, int64_t vocab,
                                                   int64_t hidden, int grads, int64_t piece_rows) {
    using namespace sidco_ce;
    if (check(rows, vocab, hidden, piece_rows)) return SIDCO_E_SIZE;
    if ((type != SIDCO_T_BF16 && type != SIDCO_T_F16) || (w_type != SIDCO_T_F32 && w_type != type)) return SIDCO_E_TYPE;
    if (grads < 0 || grads > 3 || ldw < hidden) return SIDCO_E_PARAMS;
    if (rows == 0 || vocab == 0 || hidden == 0) return 0;
    const Plan p = plan_of(rows, vocab, hidden, grads, needs_copy(w, w_type, ldw, type), piece_rows);
    return p.countable ? p.bytes : SIDCO_E_SIZE;
}

int sidco_linear_cross_entropy_typed(const void* x, int type, int64_t ldx, const void* w, int w_type, int64_t ldw,
                                     const void* labels, int label_type, const float* row_weights, float scale, int64_t rows,
                                     int64_t vocab, int64_t hidden, float* row_losses, float* loss, void* dx, int dx_type,
                                     int64_t lddx, void* dw, int dw_type, int64_t lddw, int add_dw, int64_t piece_rows,
                                     int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace sidco_ce;
    if (const int rc = check(rows, vocab, hidden, piece_rows)) return rc;
    if ((type != SIDCO_T_BF16 && type != SIDCO_T_F16) || (w_type != SIDCO_T_F32 && w_type != type) ||
        (dx && dx_type != SIDCO_T_F32 && dx_type != type) || (dw && dw_type != SIDCO_T_F32 && dw_type != type) ||
        (label_type != SIDCO_T_I32 && label_type != SIDCO_T_I64))
        return SIDCO_E_TYPE;
    if (ldx < hidden || ldw < hidden || (dx && lddx < hidden) || (dw && lddw < hidden) || !(scale - scale == 0.0f))
        return SIDCO_E_PARAMS;
    if (hidden == 0 || vocab == 0) return SIDCO_E_SIZE;
    const int64_t label_size = label_type == SIDCO_T_I64 ? 8 : 4;
    if (rows > 0 && (!x || !w || !labels)) return SIDCO_E_NULL;
    if ((uintptr_t)x % 2 || (dx && (uintptr_t)dx % size_of(dx_type)) || (uintptr_t)w % size_of(w_type) ||
        (dw && (uintptr_t)dw % size_of(dw_type)) || (uintptr_t)labels % (uintptr_t)label_size || (uintptr_t)row_weights % 4 || (uintptr_t)row_losses % 4 ||
        (uintptr_t)loss % 4 || (uintptr_t)status % 4)
        return SIDCO_E_ALIGN;
    cudaStream_t s = (cudaStream_t)stream;
    const int grads = (dx ? 1 : 0) | (dw ? 2 : 0);
    const bool copy_w = needs_copy(w, w_type, ldw, type);
    if (rows > 0) {
        const Plan p = plan_of(rows, vocab, hidden, grads, copy_w, piece_rows);
        if (!p.countable) return SIDCO_E_SIZE;
        if (!workspace || workspace_bytes < (size_t)p.bytes || (uintptr_t)workspace % 256) return SIDCO_E_WORKSPACE;
        // every buffer that is written against every other
        const struct { const void* p; int64_t bytes; bool out; } all[] = {
            {dx, extent(rows, hidden, lddx, dx_type), true}, {dw, extent(vocab, hidden, lddw, dw_type), true},
            {row_losses, rows * 4, true},                 {loss, 4, true},
            {workspace, p.bytes, true},                   {status, 4, true},
            {x, extent(rows, hidden, ldx, type), false},  {w, extent(vocab, hidden, ldw, w_type), false},
            {labels, rows * label_size, false},           {row_weights, rows * 4, false}};
        const int n = (int)(sizeof(all) / sizeof(all[0]));
        for (int i = 0; i < n; ++i)
            for (int k = i + 1; k < n; ++k)
                if (all[i].out && overlap(all[i].p, all[i].bytes, all[k].p, all[k].bytes)) return SIDCO_E_ALIAS;
        if (status) {
            const cudaError_t e = cudaMemsetAsync(status, 0, sizeof(int32_t), s);
            if (e != cudaSuccess) return (int)e;
        }
        const Call c{x, type, ldx, w, w_type, ldw, labels, label_type, row_weights, scale, rows, vocab, hidden, row_losses, loss,
                     dx, dx_type, lddx, dw, dw_type, lddw, add_dw != 0, status, static_cast<uint8_t*>(workspace), s};
        return type == SIDCO_T_BF16 ? run<__nv_bfloat16>(c, p, copy_w) : run<__half>(c, p, copy_w);
    }
    // no rows: no loss, no gradient
    cudaError_t e = cudaSuccess;
    if (status) e = cudaMemsetAsync(status, 0, sizeof(int32_t), s);
    if (e == cudaSuccess && loss) e = cudaMemsetAsync(loss, 0, sizeof(float), s);
    if (e == cudaSuccess && dw && !add_dw)
        e = cudaMemset2DAsync(dw, lddw * size_of(dw_type), 0, hidden * size_of(dw_type), vocab, s);
    return (int)e;
}

int sidco_linear_cross_entropy(const void* x, int type, int64_t ldx, const void* w, int w_type, int64_t ldw, const void* labels,
                               int label_type, const float* row_weights, float scale, int64_t rows, int64_t vocab,
                               int64_t hidden, float* row_losses, float* loss, void* dx, int64_t lddx, void* dw, int dw_type,
                               int64_t lddw, int add_dw, int64_t piece_rows, int32_t* status, void* workspace,
                               size_t workspace_bytes, void* stream) {
    return sidco_linear_cross_entropy_typed(x, type, ldx, w, w_type, ldw, labels, label_type, row_weights, scale, rows, vocab, hidden,
                                            row_losses, loss, dx, type, lddx, dw, dw_type, lddw, add_dw, piece_rows, status,
                                            workspace, workspace_bytes, stream);
}

}  // extern "C"
