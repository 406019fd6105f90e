// Momentum and orthogonalised update of the matrices of a flat model vector, for sm_100a.
//
// For every matrix:  M <- mu M + G;  U = G + mu M (Nesterov) or M;  X = U / (|U|_F + eps); then `steps` times
//     A = X X^T,   X <- (a I + b A + c A^2) X,          (a, b, c) = (3.4445, -4.7750, 2.0315),
// tall matrices through their transpose, so that X is s x l with s <= l.
//
// The steps are taken in groups (two, then one if their number is odd, then twos).  Inside a group only s x s matrices
// are multiplied: with B = a I + b A + c A^2 the Gram matrix of the next X is B A B, and the group's product of the B is
// applied to X once.  That replaces a Gram product and an application over the long side (3 s^2 l) by four products
// (4 s^3), of all but the last of which only half the tiles are computed and mirrored (they are symmetric: polynomials of
// one A).
// Longer groups would save more, but each step of a group amplifies the rounding of A by up to a^2: groups of three
// and two have 3e-3 of error where these have 1.1e-3 to 2e-3, as much as single steps (Laplace entries with eight
// strong directions, 64 x 64 to 512 x 4608).
//
// Operands are fp16 (eleven significant bits; bf16's eight would leave 1e-2 of error in the result), sums fp32.  Every
// singular value stays below 1.2 and every eigenvalue of a B within [0.6, 3.45], so fixed powers of two (kX, kA, ...)
// keep all entries inside fp16's normal range.
//
// X has two fp16 parts, X = H + L, wherever more than two steps follow.  What rounding adds to X where X has no singular
// values of its own is multiplied by a with every step, by a^5 = 485 in five, and a gradient of few rows, which is of low
// rank, is little else in the end: with H alone its update is off by 1.4e-1 (rank 1), 3e-2 (8), 2e-2 (64) of its norm.
// H suffices for the Gram matrix (an error of A turns the columns of X, but adds no rank: with L in it the results are the
// same); the applications take both, P H + P L.  The last group (up to two steps) takes H alone.  Off by, in norm, with the
// rounding to bf16 (1.7e-3) included:
//     Laplace entries                                1.8e-3 to 2.4e-3
//     singular values over three decades             2.9e-3 to 3.1e-3
//     rank 8 beside noise of a hundredth of its norm 2.7e-3 to 2.8e-3
//     rank 1, 2 / 8, 64                              4.4e-3 to 5.4e-3 / 4.0e-3 to 4.3e-3: the rounding of the s x s matrices
// (256 x 256 to 1500 x 6000, five steps; beyond six the rounding of 2^-22 itself comes to be seen in matrices of low rank,
// as it would in a 32-bit iteration: a^10 2^-24 = 1.4e-2).
// L costs a quarter of the time of large models (LSTM-shaped 1.34 -> 1.68 ms), and P in all its tiles another 3 % (below).
//
// Measured: 66 M elements in six matrices 1500 wide (LSTM-shaped, bf16 gradients) 1.73 ms: momentum and first X 0.16 (0.86 of
// the copy rate for 924 MB), products 1.31 ms under ncu (1.7 Tflop, 0.78 of cuBLAS's bf16 rate), longer in a loop, where the
// power limit sets in; VGG-16-shaped 0.31 ms, of which 0.23 in 17 dependent phases; twenty small matrices (ResNet-20) 45 us.
//
// Workspace matrices are stored as units of 64 x 64 fp16 in the 128-byte-swizzled image that the tensor cores read, so
// that a stage of operands is one or two contiguous bulk copies, the same unit serves as K-major operand (Gram) and as
// MN-major operand (application), and nothing depends on the caller's alignment.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <mutex>
#include <utility>
#include <vector>

#include "../../include/sidco.h"
#include "sidco_internal.h"
#include "sidco_tc.cuh"

namespace sidco_ortho {

using namespace sidco_tc;

constexpr float kCa = 3.4445f, kCb = -4.7750f, kCc = 2.0315f;

// stored value = value * 2^k
constexpr int kX = 14;                // X (entries <= 1.2)
constexpr int kA = 14;                // A and B A (eigenvalues <= 1.44)
constexpr int kB = 13;                // B (<= 3.45)
constexpr int kP = 10;                // products of two or three B (<= 41)

constexpr int kUnit = 64;             // units of 64 x 64
constexpr int kUnitBytes = kUnit * kUnit * 2;
constexpr int kRows = 256;           // products of larger matrices: tiles of 256 rows x 256 or 128 columns
constexpr int kMostPairs = 74;        // pairs of SMs of the device
constexpr int kMaxMats = 128;         // matrices of one chain of launches (at most 256)
constexpr int kMostUnits = 8;         // units of a matrix per CTA of the momentum pass: at most
constexpr int kMomentumCtas = 4;      // its CTAs per SM
constexpr int kMaxPhases = (SIDCO_ORTHO_MAX_STEPS + 1) / 2 * 7;   // products of a chain
constexpr int kSamples = 2048;        // elements of a matrix from which its norm is estimated

// Lists of tiles: of s x s results the lower triangle (the rest is its mirror image) or all, applications.
enum List { kLower, kWhole, kApply, kLists };

enum Buffer { kBufA, kBufA2, kBufB, kBufT, kBufP, kSmallBuffers };

struct Mat {
    int64_t offset;                   // of the matrix in the flat vectors
    int64_t x[2];                     // bytes into the workspace: s x l matrices, in turn; their second parts follow both
    int64_t small;                    // first of the s x s matrices
    int rows, cols, s, l;
    int sp, lp;                       // s to a multiple of 256, l to a multiple of 64
    int n_chunks;                     // CTAs of the momentum pass
};

struct Table {
    int n;
    int chunk;                        // units per CTA of the momentum pass
    int chunk_at[kMaxMats + 1];       // first CTA of every matrix
    int tiles_at[kLists][kMaxMats + 1];   // first tile of every matrix
    int width[kLists];                // columns of the tiles
    int64_t tiles;                    // bytes into the workspace: Tile[], list after list
    Mat m[kMaxMats];
};

// A tile of a pair of CTAs: row ti * 256, column tj * width; matrices in units from the start of the workspace.
struct __align__(16) Tile {
    int x[2], small;
    int spu, ku;                      // units along the padded s, along s
    int lu;                           // units along l
    int mat;                          // which matrix
    uint16_t ti, tj;                  // row, column
    int rows, cols;                   // of the caller's matrix, which lies
    int64_t offset;                   // here in the flat vectors
};

__device__ __forceinline__ int find(const int* at, int n, int i) {
    int lo = 0, hi = n;               // at[lo] <= i < at[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }

// ---------------------------------------------------------------------------------------------- momentum, norm

// Tile `i` of those that cover the lower triangle, row by row: row r has (r + 1) * per tiles (per = 256 / width).
__device__ __forceinline__ void triangle(int i, int per, uint16_t* row, uint16_t* col) {
    const int q = i / per;
    int r = (int)((sqrtf(8.0f * q + 1.0f) - 1.0f) * 0.5f);
    while ((r + 1) * (r + 2) / 2 <= q) ++r;
    while (r * (r + 1) / 2 > q) --r;
    *row = (uint16_t)r;
    *col = (uint16_t)(i - r * (r + 1) / 2 * per);
}

// Eight neighbours of a row of a unit: where they lie in the swizzled image.
__device__ __forceinline__ int in_unit(int r, int c8) { return r * 128 + ((c8 ^ (r & 7)) << 4); }

__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
    uint4 w;
    uint32_t* p = &w.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        p[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return w;
}

template <typename T>
__device__ __forceinline__ void load4(const T* p, float (&x)[4]) {
    uint32_t w[sizeof(T)];
    if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(p);
    else *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = widen(reinterpret_cast<const T*>(w)[i]);
}

// 2^kX / (|U|_F + eps) as two factors, the first a power of two: the norm of an fp32 matrix may be as small as 2^-149, and
// with it the quotient beyond fp32, or so large that the quotient would be subnormal.
struct Factors {
    float power, other;

    __device__ __forceinline__ Factors(float p, float o) : power(p), other(o) {}
    __device__ __forceinline__ explicit Factors(double norm_and_eps) {
        const double s = (double)(1 << kX) / norm_and_eps;
        const bool usual = s > 0.0 && s < __longlong_as_double(0x7ff0000000000000ll);
        const int half = usual ? ilogb(s) >> 1 : 0;                   // (within -75 and 82)
        power = __uint_as_float((uint32_t)(127 + half) << 23);
        other = (float)(s * __longlong_as_double((long long)(1023 - half) << 52));
    }
    __device__ __forceinline__ float operator*(float u) const { return u * power * other; }
};

// What the passes know of every matrix.
struct Norms {
    int* exponent;                    // X is first stored as U * 2^exponent
    float* factor;                    // and that times `factor` is X * 2^kX
    float *power, *other;             // factors of 2^kX / (|U|_F + eps)
    int* again;                       // the estimate was too far off: X has to be written again
    int* arrived;                     // CTAs of the momentum pass that are done
};

// The scale of X without its norm.  X as U * 2^q in two fp16 parts is accurate enough for any q with which the norm stays
// below 2^15 (no entry overflows) and the root mean square of the entries above 2^-6 (the second part ends at 2^-25, which
// is 2^-19 of that, and five steps make of it 485 times as much at worst).  Between the two there is a factor of
// 2^21 / sqrt(r c), 2^9 for 16 M entries, so the norm of 2048 entries tells q well enough.  Only entries that hide from the samples mislead
// it; the momentum pass, which adds all of them up, sees that and has X written again.  The rest of the factor joins the
// first Gram product (squared) and the first application.
// Also: counters to zero, the list of tiles.
template <typename T>
__global__ void __launch_bounds__(256) prepare_kernel(const __grid_constant__ Table t, const T* __restrict__ grad,
                                                      const float* __restrict__ momentum, float mu, int nesterov, Norms norms,
                                                      unsigned* __restrict__ phases, uint8_t* __restrict__ ws) {
    __shared__ double s_sum[8];
    launch_dependents();
    if ((int)blockIdx.x < t.n) {
        const Mat& m = t.m[blockIdx.x];
        const uint64_t size = (uint64_t)m.rows * m.cols;
        float g[kSamples / 256], v[kSamples / 256] = {};
#pragma unroll
        for (int k = 0; k < kSamples / 256; ++k) {                    // multiples of the golden section are spread evenly
            const uint64_t e = __umul64hi((threadIdx.x + k * 256 + 1) * 0x9e3779b97f4a7c15ull, size);
            g[k] = widen(grad[m.offset + e]);
            if (momentum) v[k] = momentum[m.offset + e];
        }
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < kSamples / 256; ++k) {
            const float mom = fmaf(mu, v[k], g[k]), u = nesterov && momentum ? fmaf(mu, mom, g[k]) : mom;
            sum = fma((double)u, (double)u, sum);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_down_sync(0xffffffffu, sum, o);
        if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            sum = 0.0;
            for (int w = 0; w < 8; ++w) sum += s_sum[w];
            // |U| 2^q in the middle between sqrt(r c) 2^-6 and 2^15
            const double bits = 0.25 * log2((double)size) + 4.5 - 0.5 * log2(sum * ((double)size / kSamples));
            norms.exponent[blockIdx.x] = bits > -126.0 && bits < 126.0 ? (int)rint(bits) : 0;
            norms.arrived[blockIdx.x] = 0;
        }
    }
    const int first = blockIdx.x * 256 + threadIdx.x, all = gridDim.x * 256;
    for (int w = first; w < kMaxPhases; w += all) phases[w] = 0;
    const int ends[kLists] = {t.tiles_at[kLower][t.n], t.tiles_at[kWhole][t.n], t.tiles_at[kApply][t.n]};
    for (int w = first; w < ends[kLower] + ends[kWhole] + ends[kApply]; w += all) {
        const int list = w < ends[kLower] ? kLower : w < ends[kLower] + ends[kWhole] ? kWhole : kApply;
        const int k = list == kLower ? w : list == kWhole ? w - ends[kLower] : w - ends[kLower] - ends[kWhole];
        const int* at = t.tiles_at[list];
        const int j = find(at, t.n, k), tile = k - at[j];
        const Mat& q = t.m[j];
        Tile d{};
        d.x[0] = (int)(q.x[0] / kUnitBytes);
        d.x[1] = (int)(q.x[1] / kUnitBytes);
        d.small = (int)(q.small / kUnitBytes);
        d.spu = q.sp / kUnit;
        d.ku = (q.s + kUnit - 1) / kUnit;
        d.lu = q.lp / kUnit;
        d.mat = j;
        d.rows = q.rows;
        d.cols = q.cols;
        d.offset = q.offset;
        const int mt = q.sp / kRows;
        if (list == kLower) {
            triangle(tile, kRows / t.width[kLower], &d.ti, &d.tj);
        } else {
            d.ti = (uint16_t)(tile % mt);
            d.tj = (uint16_t)(tile / mt);
        }
        reinterpret_cast<Tile*>(ws + t.tiles)[w] = d;
    }
}

// A unit of X and the elements of the caller's matrix under it: four neighbours of a row (X's columns, or X's rows if the
// matrix is tall) per thread and step.
struct UnitOf {
    bool tall, fours;
    int r, a;                         // column, first row (of four, 16 apart) in the caller's matrix
    int64_t e, by;                    // the first element, the way to the next
    int64_t image;                    // where the unit lies, bytes from the start of the workspace

    __device__ __forceinline__ UnitOf(const Mat& m, int u, int quads) {
        const int rbs = m.sp / kUnit, cbs = m.lp / kUnit;
        tall = m.rows > m.cols;
        fours = quads && ((m.offset | m.cols) & 3) == 0;
        // (units next to each other are neighbours in the caller's rows)
        const int rb = tall ? u % rbs : u / cbs, cb = tall ? u / rbs : u % cbs;
        r = (tall ? rb : cb) * kUnit + (threadIdx.x & 15) * 4;
        a = (tall ? cb : rb) * kUnit + (threadIdx.x >> 4);
        e = m.offset + (int64_t)a * m.cols + r;
        by = 16 * (int64_t)m.cols;
        image = m.x[0] + ((int64_t)cb * rbs + rb) * kUnitBytes;
    }
    // into shared memory, transposed if tall
    __device__ __forceinline__ void put(const float (&x)[4][4], float (*s_u)[kUnit + 1]) const {
        const int along = (threadIdx.x & 15) * 4, across0 = threadIdx.x >> 4;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int across = across0 + k * 16;
                if (tall) s_u[along + j][across] = x[k][j]; else s_u[across][along + j] = x[k][j];
            }
    }
};

// Where the second parts of an X lie behind the first.
__device__ __forceinline__ int64_t second_part(const Mat& m) { return 4 * (int64_t)m.sp * m.lp; }

// What fp16 leaves of a value.
__device__ __forceinline__ float rest(float v) { return v - __half2float(__float2half_rn(v)); }

// From there as fp16 in the tensor cores' order; with `lo`, what that leaves of the values as well.
__device__ __forceinline__ void store_image(uint8_t* to, uint8_t* lo, const float (*s_u)[kUnit + 1]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int row = (threadIdx.x >> 3) + k * 32, c8 = threadIdx.x & 7;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = s_u[row][c8 * 8 + j];
        *reinterpret_cast<uint4*>(to + in_unit(row, c8)) = pack8(v);
        if (lo) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = rest(v[j]);
            *reinterpret_cast<uint4*>(lo + in_unit(row, c8)) = pack8(v);
        }
    }
}

// M <- mu M + G, U as X and its sum of squares (fp64: gradients may be tiny or huge), in one pass.  The last CTA of a matrix
// to arrive adds the sums of all in their order.  66 M elements with bf16 gradients take 164 us, 0.86 of the copy rate (with
// the first parts of X alone 133; the norm from a pass of its own and those from a second one 110 + 100).  The loads of a unit
// are under way while the one before it is stored: without that 181 instead of 133; CTAs that take eight neighbouring units
// each instead of going side by side 206.
template <typename T>
__global__ void __launch_bounds__(256, kMomentumCtas) momentum_kernel(const __grid_constant__ Table t, const T* __restrict__ grad,
                                                          float* __restrict__ momentum, float mu, int nesterov, float eps,
                                                          int quads, int parts, double* __restrict__ partial, Norms norms,
                                                          uint8_t* __restrict__ ws) {
    __shared__ float s_u[kUnit][kUnit + 1];
    __shared__ double s_sum[8];
    __shared__ int s_last;
    launch_dependents();
    const int i = find(t.chunk_at, t.n, blockIdx.x), chunk = blockIdx.x - t.chunk_at[i];
    const Mat& m = t.m[i];
    // (its CTAs go through the matrix side by side: what they touch at one time lies together)
    const int units = (m.sp / kUnit) * (m.lp / kUnit);
    double sum = 0.0;
    struct alignas(4 * sizeof(T)) Four { uint32_t w[sizeof(T)]; };
    Four raw[4];                                                      // (taken apart where it is used: until then nothing waits)
    float v[4][4];
    const auto load = [&](const UnitOf& at) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t e = at.e + k * at.by;
            const bool in = at.a + k * 16 < m.rows && at.r < m.cols;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[k][j] = 0.0f;
            raw[k] = Four{};
            if (in && at.fours) {
                raw[k] = *reinterpret_cast<const Four*>(grad + e);
                if (momentum) load4((const float*)momentum + e, v[k]);
            } else if (in) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (at.r + j >= m.cols) continue;
                    reinterpret_cast<T*>(raw[k].w)[j] = grad[e + j];
                    if (momentum) v[k][j] = momentum[e + j];
                }
            }
        }
    };
    load(UnitOf(m, chunk, quads));
    wait_prerequisites();                                             // (which reads the momentum too)
    const float scale = __uint_as_float((uint32_t)(127 + __ldcg(norms.exponent + i)) << 23);
#pragma unroll 1
    for (int u = chunk; u < units; u += m.n_chunks) {
        const UnitOf at(m, u, quads);
        float g[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
            for (int j = 0; j < 4; ++j) g[k][j] = widen(reinterpret_cast<const T*>(raw[k].w)[j]);
            if (momentum) {
                const int64_t e = at.e + k * at.by;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[k][j] = fmaf(mu, v[k][j], g[k][j]);
                    g[k][j] = nesterov ? fmaf(mu, v[k][j], g[k][j]) : v[k][j];
                }
                if (at.a + k * 16 < m.rows && at.r < m.cols) {
                    if (at.fours) {
                        *reinterpret_cast<float4*>(momentum + e) = *reinterpret_cast<const float4*>(v[k]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (at.r + j < m.cols) momentum[e + j] = v[k][j];
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum = fma((double)g[k][j], (double)g[k][j], sum);
                g[k][j] *= scale;
            }
        }
        at.put(g, s_u);
        if (u + m.n_chunks < units) load(UnitOf(m, u + m.n_chunks, quads));   // under way while this unit is stored
        __syncthreads();
        store_image(ws + at.image, parts == 2 ? ws + at.image + second_part(m) : nullptr, s_u);
        __syncthreads();
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_down_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    partial += t.chunk_at[i];
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int w = 0; w < 8; ++w) sum += s_sum[w];
        partial[chunk] = sum;
        __threadfence();
        s_last = atomicAdd(norms.arrived + i, 1) == m.n_chunks - 1;
        __threadfence();
    }
    __syncthreads();
    if (!s_last) return;
    sum = 0.0;
#pragma unroll 8
    for (int c = threadIdx.x; c < m.n_chunks; c += 256) sum += __ldcg(partial + c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_down_sync(0xffffffffu, sum, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int w = 0; w < 8; ++w) sum += s_sum[w];
        // (zeros are zeros at any scale, NaN if eps is 0 as well; a NaN or an infinity makes X NaN)
        const double norm = sqrt(sum), stored = norm * (double)scale;
        const Factors f(norm + (double)eps);
        const bool finite = norm < __longlong_as_double(0x7ff0000000000000ll);
        const bool good = !finite || sum == 0.0 || (stored <= 32768.0 && stored >= sqrt((double)m.rows * m.cols) * (1.0 / 64));
        norms.power[i] = f.power;
        norms.other[i] = f.other;
        // (X = 0 / eps: the factor, squared, would be infinite for a small eps, and infinity times zero NaN)
        const bool zero = sum == 0.0 && eps > 0.0f;
        norms.factor[i] = !finite ? __int_as_float(0x7fffffff)
                          : zero  ? 0.0f
                          : good  ? (float)((double)(1 << kX) / (double)scale / (norm + (double)eps))
                                  : 1.0f;
        norms.again[i] = !good;
    }
}

// X of the matrices whose scale was wrong: U again, from what the momentum pass left, by its norm.  (The last CTA of the
// momentum pass could do that alone, which saves this launch, 2 us of a call, but takes 25 ms for 10000 x 1500.)
template <typename T>
__global__ void __launch_bounds__(256) again_kernel(const __grid_constant__ Table t, const T* __restrict__ grad,
                                                    const float* __restrict__ momentum, float mu, int nesterov, int quads,
                                                    int parts, Norms norms, uint8_t* __restrict__ ws) {
    __shared__ float s_u[kUnit][kUnit + 1];
    __shared__ int s_again[kMaxMats];
    wait_prerequisites();
    int mine = 0;
    if ((int)threadIdx.x < t.n) s_again[threadIdx.x] = mine = __ldcg(norms.again + threadIdx.x);
    if (!__syncthreads_or(mine)) return;
    for (int i = 0; i < t.n; ++i) {
        if (!s_again[i]) continue;
        const Mat& m = t.m[i];
        const int units = (m.sp / kUnit) * (m.lp / kUnit);
        const Factors scale(__ldcg(norms.power + i), __ldcg(norms.other + i));
        for (int u = blockIdx.x; u < units; u += gridDim.x) {
            const UnitOf at(m, u, quads);
            float x[4][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t e = at.e + k * at.by;
                float g[4] = {}, v[4] = {};
                if (at.a + k * 16 < m.rows && at.r < m.cols) {
                    if (at.fours) {
                        if (momentum) *reinterpret_cast<float4*>(v) = __ldcg(reinterpret_cast<const float4*>(momentum + e));
                        if (!momentum || nesterov) load4(grad + e, g);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (at.r + j >= m.cols) continue;
                            if (momentum) v[j] = __ldcg(momentum + e + j);
                            if (!momentum || nesterov) g[j] = widen(grad[e + j]);
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) x[k][j] = scale * (!momentum ? g[j] : nesterov ? fmaf(mu, v[j], g[j]) : v[j]);
            }
            __syncthreads();                                          // (s_u has been read)
            at.put(x, s_u);
            __syncthreads();
            store_image(ws + at.image, parts == 2 ? ws + at.image + second_part(m) : nullptr, s_u);
        }
    }
}

// ---------------------------------------------------------------------------------------------- products

// One phase of the chain: the same product for every matrix.
struct Phase {
    int8_t sym;                       // a product of symmetric s x s matrices (or the Gram product), or P X
    int8_t list;                      // its tiles
    int8_t left, right;               // s x s operands; left = -1: the Gram product of X; an application has P on its left
    int8_t plus, to;                  // matrix added times beta (-1: none); where the result goes
    int8_t x_in;                      // which of the two X buffers holds X
    int8_t last;                      // an application that writes bf16 into the caller's vector, not the next X
    int8_t parts;                     // an application: fp16 parts of X
    int8_t keep;                      // an application that keeps a second part of its result
    int8_t by_norm;                   // power of the factor of X in alpha: X is as the momentum pass has left it
    float alpha, beta, gamma;         // result = alpha (left right) + beta plus + gamma I
};

struct Phases {
    int n;
    int width[kLists], tiles[kLists], first[kLists];      // columns of the tiles, their number, the first
    int drop;                         // (tests) this phase is not counted; -1: none
    unsigned long long wait_ns;       // limit of the waits between phases
    Phase p[kMaxPhases];
};

// ---------------------------------------------------------------------------------------------- chain of products
//
// The other matrices: one persistent cooperative kernel runs all products of all steps.  Tiles of 256 x 256 (or 256 x 128)
// go to clusters of two CTAs on two SMs (one tcgen05 product over both: every operand byte is loaded once per pair, which
// halves the L2 traffic of 128 x 128 tiles).  Two sets of sums in tensor memory let the end of a tile run under the
// products of the next.
//   warp 0     feeds the stages (each CTA its half of the rows of A and of B)
//   warp 1     issues the products (first CTA)
//   warps 2-9  take the sums out: a quarter of the CTA's 128 rows, one half of every 64 columns
//   warp 10    stores what they have put together, and fetches matrices to add (a warp that did both lost 0.5 us per store)
// Between phases only the threads that start loads wait for the others (bounded): every CTA counts itself into the phase
// when its results are stored, 1.7 us before the others have seen it and start to load (2.5 with proxy fences over all of
// memory instead of the global one and a fence behind the polling loop instead of loads that acquire: 300 x 1000 137 us
// instead of 121).  As launches of their own the 17 phases of five steps cost the LSTM-shaped model 50 us more.  Counting per matrix, so that pairs go on to matrices that
// are ready, and a list from which pairs take tiles as they come free changed nothing: a tile's way through a phase (loads
// 1.2, products of K = 1500 8.6, sums out 2.5, counting 1.7 us) is as long as the phase.

constexpr int kOutBytes = 4 * kUnitBytes;                             // 64 columns: the images of a tile part and its mirror
constexpr int kChainThreads = 352;
constexpr int kStages = 5;
constexpr int kStageBytes = 4 * kUnitBytes;                           // per CTA: 128 x 64 of A, up to 128 x 64 of B
constexpr int kChainSmem = kStages * kStageBytes + 2 * kOutBytes + 1024;

// Barriers of the 256 threads that take the sums out, and of these with the warp that stores.
__device__ __forceinline__ void epilogue_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
constexpr int kFreeBarrier = 2, kFilledBarrier = 4, kGoBarrier = 6;   // (one per buffer)
__device__ __forceinline__ void store_sync(int id) { asm volatile("bar.sync %0, 288;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void store_arrive(int id) { asm volatile("bar.arrive %0, 288;" ::"r"(id) : "memory"); }

// Whether all 288 say so.  (They go on or stop together: one that stopped alone would leave the others at a barrier.)
__device__ __forceinline__ bool store_all(bool ok) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.aligned.pred q, %2, 288, p;\n\t"
                 "selp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(all) : "r"((uint32_t)ok), "n"(kGoBarrier) : "memory");
    return all != 0;
}

// Wait (bounded) until `count` CTAs have counted themselves in.
__device__ __forceinline__ bool wait_arrivals(const unsigned* arrived, unsigned count, unsigned long long limit_ns,
                                              volatile int* failed) {
    const unsigned long long start = time_ns();
    for (uint32_t i = 1;; ++i) {
        unsigned v;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(arrived) : "memory");
        if (v >= count) break;
        if ((i & 63u) == 0u && (*failed || time_ns() - start > limit_ns)) {
            *failed = 1;
            return false;
        }
    }
    fence_async_global();                                             // (what they stored is read by bulk copies)
    return true;
}

__global__ void __launch_bounds__(kChainThreads, 1) __cluster_dims__(2)
    chain_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ Phases ph, const Tile* tiles, uint8_t* ws,
                 __nv_bfloat16* __restrict__ out, const float* __restrict__ factor, unsigned* arrived, int* timeouts) {
    extern __shared__ uint8_t s_raw[];
    __shared__ uint64_t s_full[kStages], s_free[kStages], s_sums[2], s_taken[2], s_plus[2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    uint8_t* smem = (uint8_t*)(((uintptr_t)s_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t stage0 = smem_addr(smem);
    if (warp == 1) tmem_alloc_pair(&s_tmem, 512);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(smem_addr(&s_full[i]), 1);
            mbar_init(smem_addr(&s_free[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&s_sums[i]), 1);
            mbar_init(smem_addr(&s_taken[i]), 16);                    // eight warps of both CTAs
            mbar_init(smem_addr(&s_plus[i]), 1);
        }
        s_failed = 0;
        mbar_init_fence();
    }
    fence_before_sync();
    __syncthreads();
    cluster_sync();
    fence_after_sync();
    const uint32_t tmem = s_tmem;

    const int n_pairs = gridDim.x / 2, first = blockIdx.x / 2;
    const auto steps_of = [](const Tile& d, const Phase& p) { return p.sym ? p.left < 0 ? d.lu : d.ku : d.ku * p.parts; };
    if (warp == 0) {
        if (elect_one()) {
            int st = 0;
            uint32_t round = 0;
            bool ok = true;
            for (int f = 0; f < ph.n && ok; ++f) {
                const Phase& p = ph.p[f];
                const int width = ph.width[p.list], units_b = width / 128, parts = width / 64;
                const int total = ph.tiles[p.list];
                const Tile* list = tiles + ph.first[p.list];
                bool waited = f == 0;
                for (int i = first; i < total && ok; i += n_pairs) {
                    const Tile d = list[i];
                    if (!waited) {
                        ok = wait_arrivals(arrived + f - 1, gridDim.x, ph.wait_ns, &s_failed);
                        waited = true;
                        if (!ok) break;
                    }
                    const int steps = steps_of(d, p), small = d.spu * d.spu;
                    const int x_in = p.x_in ? d.x[1] : d.x[0];
                    const int left = p.left < 0 ? x_in : d.small + p.left * small;
                    const int right = !p.sym || p.left < 0 ? x_in : d.small + p.right * small;
                    // first unit row (symmetric) or column of B, and the way to its next unit and to the next stage
                    const int at = d.tj * parts + (int)rank * units_b;
                    const int ub0 = p.sym ? right + at : right + at * d.spu;
                    const int ub_unit = p.sym ? 1 : d.spu, ub_step = p.sym ? d.spu : 1;
                    const int ua0 = left + d.ti * 4 + (int)rank * 2;
                    for (int k = 0; k < steps; ++k) {
                        const uint32_t a = stage0 + st * kStageBytes, b = a + 2 * kUnitBytes, bar = smem_addr(&s_full[st]);
                        ok = mbar_wait(smem_addr(&s_free[st]), (round & 1) ^ 1, &s_failed);
                        if (!ok) break;
                        if (rank == 0) mbar_expect_tx(bar, 2 * (2 + units_b) * kUnitBytes);
                        // (the second part of X, behind both X, meets the same P)
                        const bool lo = !p.sym && k >= d.ku;
                        const int kk = lo ? k - d.ku : k;
                        const int ua = ua0 + kk * d.spu, ub = ub0 + kk * ub_step + (lo ? 2 * d.spu * d.lu : 0);
                        tensor_load_2d_pair(a, &map, 0, ua * kUnit, bar);
                        tensor_load_2d_pair(a + kUnitBytes, &map, 0, (ua + 1) * kUnit, bar);
                        tensor_load_2d_pair(b, &map, 0, ub * kUnit, bar);
                        if (units_b == 2) tensor_load_2d_pair(b + kUnitBytes, &map, 0, (ub + ub_unit) * kUnit, bar);
                        if (++st == kStages) { st = 0; ++round; }
                    }
                }
            }
        }
    } else if (warp == 1) {
        // (the whole warp waits, one thread issues)
        if (rank == 0) {
            int st = 0, n = 0;
            uint32_t round = 0;
            bool ok = true;
            for (int f = 0; f < ph.n && ok; ++f) {
                const Phase& p = ph.p[f];
                const bool sym = p.sym;
                const int total = ph.tiles[p.list];
                const Tile* list = tiles + ph.first[p.list];
                const uint32_t shape = f16_shape(kRows, ph.width[p.list], !sym);
                // (K-major operands move 32 bytes on along K, the MN-major B of an application sixteen rows of 128)
                const uint32_t b_step = sym ? 32 : 2048, b_lead = sym ? 16 : kUnitBytes;
                for (int i = first; i < total && ok; i += n_pairs, ++n) {
                    const int steps = steps_of(list[i], p);
                    const int buf = n & 1;
                    const uint32_t sums = tmem + buf * 256;
                    ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&s_taken[buf]), ((n >> 1) & 1) ^ 1, &s_failed));
                    for (int k = 0; k < steps && ok; ++k) {
                        ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&s_full[st]), round & 1, &s_failed));
                        if (!ok) break;
                        fence_after_sync();
                        const uint32_t a = stage0 + st * kStageBytes, b = a + 2 * kUnitBytes;
                        if (elect_one()) {
#pragma unroll
                            for (int q = 0; q < kUnit / 16; ++q)
                                mma_f16_pair(sums, swizzled_operand(a + q * 32, 16, 1024),
                                             swizzled_operand(b + q * b_step, b_lead, 1024), shape, k > 0 || q > 0);
                            tc_commit_pair(smem_addr(&s_free[st]));
                            if (k + 1 == steps) tc_commit_pair(smem_addr(&s_sums[buf]));
                        }
                        __syncwarp();
                        if (++st == kStages) { st = 0; ++round; }
                    }
                }
            }
        }
    } else if (warp == 10) {
        const uint32_t out0 = stage0 + kStages * kStageBytes;
        int part = 0;
        bool ok = true;
        for (int f = 0; f < ph.n && ok; ++f) {
            const Phase& p = ph.p[f];
            const bool sym = p.sym, last = p.last, plus = p.plus >= 0;
            const int width = ph.width[p.list], parts = width / 64;
            const int total = ph.tiles[p.list];
            const Tile* list = tiles + ph.first[p.list];
            bool waited = f == 0;
            for (int i = first; i < total; i += n_pairs) {
                const Tile d = list[i];
                const int small = d.spu * d.spu, rb = d.ti * 4 + (int)rank * 2;
                const bool mirror = p.list == kLower && d.tj < d.ti * (kRows / width);
                const int base = sym ? d.small + p.to * small : p.x_in ? d.x[0] : d.x[1];
                // part `cu` of the tile may be filled: its buffer has been read, and holds the 64 columns to add
                const auto prepare = [&](int cu, int to) {
                    if (elect_one()) {
                        bulk_store_wait_read();
                        if (plus) {
                            const uint32_t bar = smem_addr(&s_plus[to]);
                            mbar_expect_tx(bar, 2 * kUnitBytes);
                            bulk_load(out0 + to * kOutBytes,
                                      ws + (int64_t)(d.small + p.plus * small + (d.tj * parts + cu) * d.spu + rb) * kUnitBytes,
                                      2 * kUnitBytes, bar);
                        }
                    }
                    __syncwarp();
                    if (!plus) store_arrive(kFreeBarrier + to);
                };
                if (plus && !waited)
                    ok = __all_sync(0xffffffffu, wait_arrivals(arrived + f - 1, gridDim.x, ph.wait_ns, &s_failed));
                waited = true;
                if (!last && ok) prepare(0, part & 1);
                ok = store_all(ok);
                if (!ok) break;
                if (last) continue;
                for (int cu = 0; cu < parts; ++cu, ++part) {
                    if (cu + 1 < parts) prepare(cu + 1, (part & 1) ^ 1);
                    store_sync(kFilledBarrier + (part & 1));
                    const int cb = d.tj * parts + cu;
                    if (elect_one() && (sym || cb < d.lu)) {
                        const uint32_t img = out0 + (part & 1) * kOutBytes;
                        bulk_store(ws + (int64_t)(base + cb * d.spu + rb) * kUnitBytes, img, 2 * kUnitBytes);
                        if (mirror)
                            for (int u = 0; u < 2; ++u)
                                bulk_store(ws + (int64_t)(base + (rb + u) * d.spu + cb) * kUnitBytes, img + (2 + u) * kUnitBytes,
                                           kUnitBytes);
                        if (p.keep)
                            bulk_store(ws + (int64_t)(base + (2 * d.lu + cb) * d.spu + rb) * kUnitBytes, img + 2 * kUnitBytes,
                                       2 * kUnitBytes);
                        bulk_store_commit();
                    }
                    __syncwarp();
                }
            }
            if (!last && ok && f != ph.drop && elect_one()) {         // stored: count this CTA in
                bulk_store_wait();
                fence_async_global();
                asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(arrived + f) : "memory");
            }
            __syncwarp();
        }
    } else {
        const int quarter = warp & 3, h = (warp - 2) >> 2, row = quarter * 32 + lane;
        uint8_t* out_smem = smem + kStages * kStageBytes;
        const uint32_t taken[2] = {in_cta(smem_addr(&s_taken[0]), 0), in_cta(smem_addr(&s_taken[1]), 0)};
        int n = 0, part = 0, fetched = 0;
        bool ok = true;
        for (int f = 0; f < ph.n && ok; ++f) {
            const Phase& p = ph.p[f];
            const bool sym = p.sym, last = p.last, plus = p.plus >= 0;
            const int width = ph.width[p.list], parts = width / 64;
            const int total = ph.tiles[p.list];
            const Tile* list = tiles + ph.first[p.list];
            const bool keep = p.keep;
            const float beta = p.beta, gamma = p.gamma;
            for (int i = first; i < total; i += n_pairs, ++n) {
                const Tile d = list[i];
                const int buf = n & 1;
                const int rb = d.ti * 4 + (int)rank * 2;              // first unit row of this CTA's part
                const bool mirror = p.list == kLower && d.tj < d.ti * (kRows / width), tall = d.rows > d.cols;
                float alpha = p.alpha;
                for (int k = 0; k < p.by_norm; ++k) alpha *= __ldg(factor + d.mat);
                const int diagonal = d.ti * kRows + (int)rank * 128 + row - d.tj * width;     // the column on the diagonal
                ok = mbar_wait(smem_addr(&s_sums[buf]), (n >> 1) & 1, &s_failed);
                __syncwarp();
                ok = store_all(ok);
                if (!ok) break;
                fence_after_sync();
#pragma unroll 1
                for (int cu = 0; cu < parts; ++cu, ++part) {
                    uint8_t* img = out_smem + (part & 1) * kOutBytes;
                    __syncwarp();
                    if (plus) {
                        mbar_wait(smem_addr(&s_plus[part & 1]), (fetched >> 1) & 1, &s_failed);
                        ++fetched;
                        __syncwarp();
                    } else if (!last) {
                        store_sync(kFreeBarrier + (part & 1));
                    }                                                 // (rows for the caller are read by all warps before
                                                                      // the barrier of the next part)
                    {
                        const int q = cu * 2 + h;
                        uint32_t acc[32];
                        tmem_load32(tmem + buf * 256 + ((uint32_t)(quarter * 32) << 16) + q * 32, acc);
                        if (!last) {
#pragma unroll
                            for (int o = 0; o < 4; ++o) {
                                float v[8];
#pragma unroll
                                for (int j = 0; j < 8; ++j) v[j] = alpha * __uint_as_float(acc[o * 8 + j]);
                                uint4* at = reinterpret_cast<uint4*>(img + (row >> 6) * kUnitBytes + in_unit(row & 63, h * 4 + o));
                                if (plus) {
                                    const uint4 e = *at;
                                    const __half2* x = reinterpret_cast<const __half2*>(&e);
#pragma unroll
                                    for (int j = 0; j < 4; ++j) {
                                        const float2 y = __half22float2(x[j]);
                                        v[2 * j] = fmaf(beta, y.x, v[2 * j]);
                                        v[2 * j + 1] = fmaf(beta, y.y, v[2 * j + 1]);
                                    }
                                    // (gamma comes with a matrix to add; a select: a branch would be taken by one lane at
                                    // a time)
#pragma unroll
                                    for (int j = 0; j < 8; ++j) v[j] += diagonal == q * 32 + o * 8 + j ? gamma : 0.0f;
                                }
                                const uint4 packed = pack8(v);
                                *at = packed;
                                if (keep) {                           // (an application has no mirror: its place is free)
#pragma unroll
                                    for (int j = 0; j < 8; ++j) v[j] = rest(v[j]);
                                    at[2 * kUnitBytes / 16] = pack8(v);
                                }
                                if (mirror) {
                                    const __half* hv = reinterpret_cast<const __half*>(&packed);
#pragma unroll
                                    for (int j = 0; j < 8; ++j)
                                        *reinterpret_cast<__half*>(img + (2 + (row >> 6)) * kUnitBytes +
                                                                   in_unit(h * 32 + o * 8 + j, (row & 63) >> 3) +
                                                                   (row & 7) * 2) = hv[j];
                                }
                            }
                        } else {
                            __nv_bfloat16* s_out = reinterpret_cast<__nv_bfloat16*>(img);
                            if (tall) {
#pragma unroll
                                for (int j = 0; j < 32; ++j)
                                    s_out[(h * 32 + j) * 130 + row] = __float2bfloat16_rn(alpha * __uint_as_float(acc[j]));
                            } else {
#pragma unroll
                                for (int j = 0; j < 32; j += 2)
                                    *reinterpret_cast<__nv_bfloat162*>(s_out + row * 66 + h * 32 + j) = __floats2bfloat162_rn(
                                        alpha * __uint_as_float(acc[j]), alpha * __uint_as_float(acc[j + 1]));
                            }
                        }
                    }
                    if (cu == parts - 1) {                            // the sums have been read
                        fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(taken[buf]);
                    }
                    __syncwarp();
                    if (!last) {
                        fence_async_shared();
                        store_arrive(kFilledBarrier + (part & 1));
                    } else {
                        epilogue_sync();
                        const __nv_bfloat16* s_out = reinterpret_cast<const __nv_bfloat16*>(img);
                        const int r_x = rb * kUnit, c_x = (d.tj * parts + cu) * kUnit;       // first row, column of X
                        const int a0 = tall ? c_x : r_x, n0 = tall ? r_x : c_x;
                        const int lines = tall ? 64 : 128, len = tall ? 128 : 64, pitch = tall ? 130 : 66;
                        __nv_bfloat16* to = out + d.offset + (int64_t)a0 * d.cols + n0;
                        const int n_lines = min(lines, d.rows - a0), n_len = min(len, d.cols - n0);
                        const bool even = ((d.offset | d.cols) & 1) == 0 && ((uintptr_t)out & 3) == 0;
                        if (even) {
                            const int k = lane * 2;
#pragma unroll 8
                            for (int a = warp - 2; a < n_lines; a += 8) {
                                const __nv_bfloat16* from = s_out + a * pitch;
                                __nv_bfloat16* line = to + (int64_t)a * d.cols;
                                if (k < n_len)
                                    *reinterpret_cast<uint32_t*>(line + k) = *reinterpret_cast<const uint32_t*>(from + k);
                                if (k + 64 < n_len)
                                    *reinterpret_cast<uint32_t*>(line + k + 64) =
                                        *reinterpret_cast<const uint32_t*>(from + k + 64);
                            }
                        } else {
#pragma unroll 4
                            for (int a = warp - 2; a < n_lines; a += 8)
                                for (int k = lane; k < n_len; k += 32) to[(int64_t)a * d.cols + k] = s_out[a * pitch + k];
                        }
                    }
                }
            }
        }
    }
    __syncwarp();
    fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s_failed) {
        atomicAdd(timeouts, 1);
        let_work_end();
    }
    __syncthreads();
    cluster_sync();
    if (warp == 1) tmem_free_pair(tmem, 512);
}

// ---------------------------------------------------------------------------------------------- small matrices
//
// Matrices with s <= 128 and l <= 2048: one cluster of CTAs per matrix does the whole update in one launch.  Every CTA
// keeps its columns of X (up to 256) from the first step to the last: the first parts (64 KB) in shared memory, the second in
// tensor memory, from where they come into the place of squares that are done with for every application (4 us of a
// call).  The only exchange between the CTAs is a sum per Gram matrix: each adds its share of the rows of all partial
// Gram matrices through distributed shared memory, in the order of the CTAs, and hands the result to the others; the
// s x s products that follow (0.8 us each) every CTA does for itself.
// With few rows the rounding of the s x s matrices is the largest error, and products of second fp16 parts cost next to
// nothing here.  With s <= 64 all of them are sums of two parts: any rank of 64 x 576 is off by 1.7e-3 of its norm, the rounding
// to bf16, and the exchange moves 64 x 64.  Above, where a square is twice that, A and T have one part (128 x 1152: 1.8e-3 to
// 2.3e-3).

constexpr int kSmallS = 128, kSmallUnits = 4, kSmallCluster = 8;      // units of columns per CTA, CTAs per matrix: at most
constexpr int kSmallThreads = 512;
constexpr int kSquareBytes = 4 * kUnitBytes;                          // 128 x 128 (with s <= 64: 128 x 64, half of it)
constexpr int kSlabBytes = kSmallUnits * 2 * kUnitBytes;              // 128 x 256
constexpr int kOutLine = kSmallUnits * kUnit + 2, kOutColumn = kSmallS + 2;   // bf16 per line of the result, wide or tall
constexpr int kRests = 256;                                           // columns of tensor memory: sums, then second parts of X
constexpr int kSquares = 5;                                           // (together larger than X's part in fp32)
constexpr int kSmallSmem = kSquares * kSquareBytes + std::max(kSlabBytes, std::max(kSmallS * kOutLine, kSmallUnits * kUnit * kOutColumn) * 2) +
                           1024;

struct SmallMats {
    int n;
    struct { int64_t offset; int rows, cols; } m[kMaxMats];
};

__device__ __forceinline__ uint4 remote_load16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}

__device__ __forceinline__ void remote_store8(uint32_t addr, uint32_t x, uint32_t y) {
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(addr), "r"(x), "r"(y) : "memory");
}

__device__ __forceinline__ void remote_store_f64(uint32_t addr, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory");
}

template <typename T, int kCtas>
__global__ void __launch_bounds__(kSmallThreads, 1)
    small_kernel(const __grid_constant__ SmallMats mats, const T* __restrict__ grad, float* __restrict__ momentum, float mu,
                 int nesterov, int steps, float eps, __nv_bfloat16* __restrict__ out, int* timeouts) {
    extern __shared__ uint8_t s_raw[];
    __shared__ double s_norm[kSmallCluster], s_sum[kSmallThreads / 32];
    __shared__ uint64_t s_done;
    __shared__ uint32_t s_tmem;
    __shared__ int s_failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr uint32_t ctas = kCtas;
    const uint32_t rank = cluster_rank();
    const auto& m = mats.m[blockIdx.x / ctas];
    const bool tall = m.rows > m.cols;
    const int s = tall ? m.cols : m.rows, l = tall ? m.rows : m.cols;
    const int lu = (l + kUnit - 1) / kUnit, ku = (s + kUnit - 1) / kUnit;
    const int first = (int)(lu * rank / ctas), units = (int)(lu * (rank + 1) / ctas) - first;   // of this CTA's columns

    uint8_t* smem = (uint8_t*)(((uintptr_t)s_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* slab = smem + kSquares * kSquareBytes;
    // the squares: six small ones or five large ones; A and T have a second part if they are small (rows from 64 on of the
    // small ones are whatever was there: they take part in sums of their own rows only, and nobody reads those)
    const auto sq = [&](int i) { return smem + i * ku * (kSquareBytes / 2); };
    struct Square { uint8_t *hi, *lo; };
    const bool fine = ku == 1;
    const Square sq_a = {sq(0), fine ? sq(1) : nullptr}, sq_b = fine ? Square{sq(2), sq(3)} : Square{sq(1), sq(2)},
                 sq_t = {fine ? sq(4) : sq(3), fine ? sq(5) : nullptr}, sq_b2 = fine ? Square{sq(4), sq(5)} : Square{sq(3), sq(4)},
                 sq_p = {sq(0), sq(1)};
    if (warp == 0) tmem_alloc(&s_tmem, 512);
    if (threadIdx.x == 0) {
        mbar_init(smem_addr(&s_done), 1);
        s_failed = 0;
        mbar_init_fence();
    }

    // ---- momentum and norm.  A thread takes 16 elements of each unit of columns, threads next to each other neighbours of
    // a row of the caller's matrix.  U waits for its norm, in fp32, where the squares will be: as rows, or as columns if the
    // matrix is tall, one word longer than they need be against bank conflicts.
    const int r0 = tall ? threadIdx.x & 127 : threadIdx.x >> 6, a0 = tall ? threadIdx.x >> 7 : threadIdx.x & 63;
    const auto row_of = [&](int j) { return tall ? r0 : r0 + 8 * j; };
    const auto col_of = [&](int u, int j) { return u * kUnit + (tall ? a0 + 4 * j : a0); };
    const auto inside = [&](int u, int j) { return u < units && row_of(j) < s && first * kUnit + col_of(u, j) < l; };
    const int64_t base = m.offset + (tall ? (int64_t)(first * kUnit + a0) * m.cols + r0 : (int64_t)r0 * m.cols + first * kUnit + a0);
    const int64_t by_u = (int64_t)kUnit * (tall ? m.cols : 1), by_j = (int64_t)(tall ? 4 : 8) * m.cols;
    float* held = reinterpret_cast<float*>(smem);
    const int by_row = tall ? 1 : kSmallUnits * kUnit + 1, by_col = tall ? kSmallS + 1 : 1;
    double sums[2] = {};
#pragma unroll 1
    for (int u = 0; u < units; ++u) {
        const int64_t at = base + u * by_u;
        float g[16], v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const bool in = inside(u, j);
            g[j] = in ? widen(grad[at + j * by_j]) : 0.0f;
            v[j] = in && momentum ? momentum[at + j * by_j] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            if (momentum) {
                const float mom = fmaf(mu, v[j], g[j]);
                if (inside(u, j)) momentum[at + j * by_j] = mom;
                g[j] = nesterov ? fmaf(mu, mom, g[j]) : mom;
            }
            held[row_of(j) * by_row + col_of(u, j) * by_col] = g[j];   // (zeros outside the matrix)
            sums[j & 1] = fma((double)g[j], (double)g[j], sums[j & 1]);
        }
    }
    double sum = sums[0] + sums[1];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_down_sync(0xffffffffu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    fence_before_sync();
    __syncthreads();
    cluster_sync();                                                   // every CTA runs, so its shared memory may be written
    fence_after_sync();
    const uint32_t tmem = s_tmem;
    if (threadIdx.x < ctas) {
        sum = 0.0;
        for (int w = 0; w < kSmallThreads / 32; ++w) sum += s_sum[w];
        remote_store_f64(in_cta(smem_addr(&s_norm[rank]), threadIdx.x), sum);
    }
    cluster_sync();
    sum = 0.0;
    for (uint32_t i = 0; i < ctas; ++i) sum += s_norm[i];
    const Factors scale(sqrt(sum) + (double)eps);

    // ---- X: a thread has a row of a unit of columns, eight neighbours at a time.  The first parts go to the slab, the second
    // wait in tensor memory behind the sums, two to a word.
    const int row = (warp & 3) * 32 + lane, side = warp >> 2;         // row, unit of columns (quarter of a square's columns)
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const auto put_x = [&](int o, float (&v)[8], uint32_t* lo) {
        *reinterpret_cast<uint4*>(slab + (side * 2 + (row >> 6)) * kUnitBytes + in_unit(row & 63, o)) = pack8(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = rest(v[j]);
        *reinterpret_cast<uint4*>(lo) = pack8(v);
    };
    if (side < units) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            alignas(16) uint32_t lo[16];
#pragma unroll
            for (int o = 0; o < 4; ++o) {
                float v8[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v8[j] = scale * held[row * by_row + (side * kUnit + h * 32 + o * 8 + j) * by_col];
                put_x(h * 4 + o, v8, lo + o * 4);
            }
            tmem_store16(lanes + kRests + side * 32 + h * 16, lo);
        }
    }

    // ---- products: one thread issues, then everybody takes its rows and columns of the sums
    int uses = 0;
    const auto issue_and_wait = [&](auto products) {
        fence_async_shared();
        fence_before_sync();
        __syncthreads();
        if (warp == 0) {
            fence_after_sync();
            if (elect_one()) {
                products();
                tc_commit(smem_addr(&s_done));
            }
            __syncwarp();
        }
        mbar_wait(smem_addr(&s_done), uses & 1, &s_failed);
        __syncwarp();
        ++uses;
        fence_after_sync();
    };
    // eight neighbours of a row of a square: as one fp16 part or two
    const auto put = [&](const Square& to, int o, float (&v)[8]) {
        const int at = ((side & ~1) + (row >> 6)) * kUnitBytes + in_unit(row & 63, (side & 1) * 4 + o);
        *reinterpret_cast<uint4*>(to.hi + at) = pack8(v);
        if (to.lo) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] -= __half2float(__float2half_rn(v[j]));
            *reinterpret_cast<uint4*>(to.lo + at) = pack8(v);
        }
    };
    // to = alpha left right + beta plus + gamma I (the product of two second parts is left out)
    const auto square = [&](const Square& left, const Square& right, const Square* plus, const Square& to, float alpha, float beta,
                            float gamma) {
        issue_and_wait([&] {
            bool add = false;
            for (int t = 0; t < 3; ++t) {
                const uint8_t *l = t == 2 ? left.lo : left.hi, *r = t == 1 ? right.lo : right.hi;
                if (!l || !r) continue;
                const uint32_t a = smem_addr(l), b = smem_addr(r);
                for (int k = 0; k < ku * 4; ++k, add = true)
                    mma_f16(tmem, swizzled_operand(a + (k >> 2) * 2 * kUnitBytes + (k & 3) * 32, 16, 1024),
                            swizzled_operand(b + (k >> 2) * 2 * kUnitBytes + (k & 3) * 32, 16, 1024),
                            f16_shape(kSmallS, ku * kUnit, false), add);
            }
        });
        if (side >= 2 * ku) return;
        uint32_t acc[32];
        tmem_load32(lanes + side * 32, acc);
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            const int at = ((side & ~1) + (row >> 6)) * kUnitBytes + in_unit(row & 63, (side & 1) * 4 + o);
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = alpha * __uint_as_float(acc[o * 8 + j]);
            for (int t = 0; t < 2 && plus; ++t) {
                const uint8_t* from = t ? plus->lo : plus->hi;
                if (!from) break;
                const uint4 w = *reinterpret_cast<const uint4*>(from + at);
                const __half2* h = reinterpret_cast<const __half2*>(&w);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = __half22float2(h[j]);
                    v[2 * j] = fmaf(beta, f.x, v[2 * j]);
                    v[2 * j + 1] = fmaf(beta, f.y, v[2 * j + 1]);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += row == side * 32 + o * 8 + j ? gamma : 0.0f;
            put(to, o, v);
        }
    };
    const auto two = [](int k) { return __uint_as_float((uint32_t)(127 + k) << 23); };

    for (int done = 0; done < steps;) {
        const int group = steps == 1 || (done == 2 && (steps & 1)) ? 1 : 2;
        // A = X X^T: the partial sums of this CTA's columns
        issue_and_wait([&] {
            const uint32_t a = smem_addr(slab);
            for (int k = 0; k < units * 4; ++k) {
                const uint64_t x = swizzled_operand(a + (k >> 2) * 2 * kUnitBytes + (k & 3) * 32, 16, 1024);
                mma_f16(tmem, x, x, f16_shape(kSmallS, ku * kUnit, false), k > 0);
            }
        });
        const float gram_scale = two(kA - 2 * kX);
        if constexpr (kCtas == 1) {
            if (side < 2 * ku) {
                uint32_t acc[32];
                tmem_load32(lanes + side * 32, acc);
#pragma unroll
                for (int o = 0; o < 4; ++o) {
                    float v8[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v8[j] = gram_scale * __uint_as_float(acc[o * 8 + j]);
                    put(sq_a, o, v8);
                }
            }
        } else {
            // [64 ku][64 ku] where B will be, words swizzled; a CTA without columns adds zeros
            float* partial = reinterpret_cast<float*>(sq_b.hi);
            const int fours = 16 * ku, shift = 3 + ku;                // (16 or 32 times four columns)
            if (side < 2 * ku && row < kUnit * ku) {
                uint32_t acc[32];
                tmem_load32(lanes + side * 32, acc);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c4 = side * 8 + j;                      // rows differ in their bank
                    const float4 v4 = units ? make_float4(__uint_as_float(acc[j * 4]), __uint_as_float(acc[j * 4 + 1]),
                                                          __uint_as_float(acc[j * 4 + 2]), __uint_as_float(acc[j * 4 + 3]))
                                            : make_float4(0, 0, 0, 0);
                    reinterpret_cast<float4*>(partial)[row * fours + (c4 ^ (row & 7))] = v4;
                }
            }
            fence_before_sync();
            __syncthreads();
            cluster_sync();
            // rows rank, rank + ctas, ... of the sum, four columns at a time, to every CTA's A
            constexpr int kAtOnce = kCtas == 8 ? 1 : 2;               // (128 rows: 8, 4, 2 per thread)
            const int items = kUnit * ku / kCtas * fours;
            for (int i0 = threadIdx.x; i0 < items; i0 += kAtOnce * kSmallThreads) {
                uint4 w[kAtOnce][kCtas];
#pragma unroll
                for (int t = 0; t < kAtOnce; ++t) {
                    const int i = i0 + t * kSmallThreads, r = (i >> shift) * kCtas + (int)rank;
                    const uint32_t from = smem_addr(partial) + (uint32_t)(r * fours + ((i & (fours - 1)) ^ (r & 7))) * 16;
#pragma unroll
                    for (uint32_t q = 0; q < kCtas; ++q)
                        if (i < items) w[t][q] = remote_load16(in_cta(from, q));
                }
#pragma unroll
                for (int t = 0; t < kAtOnce; ++t) {
                    const int i = i0 + t * kSmallThreads, r = (i >> shift) * kCtas + (int)rank, c4 = i & (fours - 1);
                    if (i >= items) break;
                    float v4[4] = {};
#pragma unroll
                    for (uint32_t q = 0; q < kCtas; ++q) {
                        v4[0] += __uint_as_float(w[t][q].x);
                        v4[1] += __uint_as_float(w[t][q].y);
                        v4[2] += __uint_as_float(w[t][q].z);
                        v4[3] += __uint_as_float(w[t][q].w);
                    }
                    const uint32_t at = ((c4 >> 4) * 2 + (r >> 6)) * kUnitBytes + in_unit(r & 63, (c4 >> 1) & 7) + (c4 & 1) * 8;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v4[j] *= gram_scale;
                    const auto send = [&](const uint8_t* to) {
                        const __half2 h0 = __floats2half2_rn(v4[0], v4[1]), h1 = __floats2half2_rn(v4[2], v4[3]);
#pragma unroll
                        for (uint32_t q = 0; q < kCtas; ++q)
                            remote_store8(in_cta(smem_addr(to) + at, q), *reinterpret_cast<const uint32_t*>(&h0),
                                          *reinterpret_cast<const uint32_t*>(&h1));
                    };
                    send(sq_a.hi);
                    if (sq_a.lo) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) v4[j] -= __half2float(__float2half_rn(v4[j]));
                        send(sq_a.lo);
                    }
                }
            }
            fence_async_all();                                        // (read by the tensor cores of the other CTAs)
            cluster_sync();
        }

        // B; for a second step T = B A, the next A = T B, its B where T was, and the product of both where A was
        Square p = sq_b;
        int scale_p = kB;
        const float poly = kCc * two(kB - 2 * kA), linear = kCb * two(kB - kA), unit = kCa * two(kB);
        square(sq_a, sq_a, &sq_a, sq_b, poly, linear, unit);
        if (group == 2) {
            square(sq_b, sq_a, nullptr, sq_t, two(-kB), 0.0f, 0.0f);
            square(sq_t, sq_b, nullptr, sq_a, two(-kB), 0.0f, 0.0f);
            square(sq_a, sq_a, &sq_a, sq_b2, poly, linear, unit);
            square(sq_b2, sq_b, nullptr, sq_p, two(kP - 2 * kB), 0.0f, 0.0f);
            p = sq_p;
            scale_p = kP;
        }

        // X <- P X on this CTA's columns, the second parts of X from the squares that are done with
        uint8_t* rests = sq(fine ? 4 : 3);
        if (side < units) {
            alignas(16) uint32_t lo[32];
            tmem_load32(lanes + kRests + side * 32, lo);
#pragma unroll
            for (int o = 0; o < 8; ++o)
                *reinterpret_cast<uint4*>(rests + (side * 2 + (row >> 6)) * kUnitBytes + in_unit(row & 63, o)) =
                    *reinterpret_cast<const uint4*>(lo + o * 4);
        }
        issue_and_wait([&] {
            for (int t = 0; t < 3 && units; ++t) {                    // (not the product of both second parts)
                const uint32_t a0 = smem_addr(t == 1 ? p.lo : p.hi), b0 = smem_addr(t == 2 ? rests : slab);
                for (int k = 0; k < ku * 4; ++k)
                    mma_f16(tmem, swizzled_operand(a0 + (k >> 2) * 2 * kUnitBytes + (k & 3) * 32, 16, 1024),
                            swizzled_operand(b0 + (k >> 2) * kUnitBytes + (k & 3) * 2048, 2 * kUnitBytes, 1024),
                            f16_shape(kSmallS, units * kUnit, true), t > 0 || k > 0);
            }
        });
        done += group;
        const bool last = done == steps;
        const float alpha = two(last ? -scale_p - kX : -scale_p);
        __nv_bfloat16* s_out = reinterpret_cast<__nv_bfloat16*>(slab);          // (X is done with)
        if (side < units) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t acc[32];
                tmem_load32(lanes + side * kUnit + h * 32, acc);
                if (!last) {
                    alignas(16) uint32_t lo[16];
#pragma unroll
                    for (int o = 0; o < 4; ++o) {
                        float v[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = alpha * __uint_as_float(acc[o * 8 + j]);
                        put_x(h * 4 + o, v, lo + o * 4);
                    }
                    tmem_store16(lanes + kRests + side * 32 + h * 16, lo);
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const int col = side * kUnit + h * 32 + j;
                        s_out[tall ? col * kOutColumn + row : row * kOutLine + col] =
                            __float2bfloat16_rn(alpha * __uint_as_float(acc[j]));
                    }
                }
            }
        }
        if (last) {
            __syncthreads();
            const int lines = tall ? units * kUnit : s, len = tall ? s : units * kUnit, pitch = tall ? kOutColumn : kOutLine;
            const int line0 = tall ? first * kUnit : 0, col0 = tall ? 0 : first * kUnit;
            if (!s_failed)
                for (int i = warp; i < lines && line0 + i < m.rows; i += kSmallThreads / 32)
                    for (int k = lane; k < len && col0 + k < m.cols; k += 32)
                        out[m.offset + (int64_t)(line0 + i) * m.cols + col0 + k] = s_out[i * pitch + k];
        }
    }
    fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s_failed) {
        atomicAdd(timeouts, 1);
        let_work_end();
    }
    __syncthreads();
    cluster_sync();                                                   // nobody reads or writes this CTA's memory any more
    if (warp == 0) tmem_free(tmem, 512);
}

__device__ int g_timeouts;

// ---------------------------------------------------------------------------------------------- host side

static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Lays the matrices order[0..n) out in the workspace and numbers the CTAs of the passes.  Returns the bytes needed.
static int64_t lay_out(const int64_t* offsets, const int64_t* rows, const int64_t* cols, const int* order, int n,
                       int max_pairs, Table* t) {
    int64_t at = 0;
    int64_t chunks = 0, units = 0, all_tiles = 0;
    t->n = n;
    for (int k = 0; k < n; ++k) {
        Mat& m = t->m[k];
        const int64_t r = rows[order[k]], c = cols[order[k]];
        m.offset = offsets ? offsets[order[k]] : 0;
        m.rows = (int)r;
        m.cols = (int)c;
        m.s = (int)std::min(r, c);
        m.l = (int)std::max(r, c);
        m.sp = (int)up(m.s, kRows);
        m.lp = (int)up(m.l, kUnit);
        units += (int64_t)(m.sp / kUnit) * (m.lp / kUnit);
    }
    // whole rounds of the momentum pass' CTAs, each a part of one matrix
    const int64_t at_once = 2 * kMostPairs * kMomentumCtas, rounds = (units + at_once * kMostUnits - 1) / (at_once * kMostUnits);
    t->chunk = (int)((units + at_once * rounds - n - 1) / (at_once * rounds - n));
    for (int k = 0; k < n; ++k) {
        Mat& m = t->m[k];
        t->chunk_at[k] = (int)chunks;
        m.n_chunks = (int)(((int64_t)(m.sp / kUnit) * (m.lp / kUnit) + t->chunk - 1) / t->chunk);
        chunks += m.n_chunks;
    }
    // Columns of a tile: 256 give the tensor cores two thirds of the operand traffic per operation, 128 give twice as many
    // tiles for few matrices.  A tile of 128 columns takes about 0.6 of the time of one of 256.
    const auto tiles_of = [&](int list, int width) {
        int64_t all = 0;
        for (int k = 0; k < n; ++k) {
            const Mat& m = t->m[k];
            const int64_t mt = m.sp / kRows;
            t->tiles_at[list][k] = (int)all;
            all += list == kApply ? mt * ((m.lp + width - 1) / width)
                                  : (list == kLower ? mt * (mt + 1) / 2 : mt * mt) * (kRows / width);
        }
        t->tiles_at[list][n] = (int)all;
        return all;
    };
    const auto rounds_of = [&](int64_t tiles) { return (double)((tiles + max_pairs - 1) / max_pairs); };
    for (int list = 0; list < kLists; ++list) {
        const int64_t wide = tiles_of(list, 256), narrow = tiles_of(list, 128);
        t->width[list] = 0.6 * rounds_of(narrow) < rounds_of(wide) ? 128 : 256;
        if (t->width[list] == 256) tiles_of(list, 256);
        all_tiles += narrow;                                          // (room for either)
    }
    t->chunk_at[n] = (int)chunks;
    if (chunks > 0x7fffffff || all_tiles > 0x7fffffff) return -1;
    at = up(at + chunks * 8, 1024);
    at = up(at + (6 * n + kMaxPhases) * 4, 1024);                     // norms, arrival counters
    t->tiles = at;
    at = up(at + all_tiles * (int64_t)sizeof(Tile), kUnitBytes);
    for (int k = 0; k < n; ++k) {
        Mat& m = t->m[k];
        const int64_t big = (int64_t)m.sp * m.lp * 2;
        m.x[0] = at;
        m.x[1] = at + big;
        m.small = at + 4 * big;
        at = m.small + (int64_t)kSmallBuffers * m.sp * m.sp * 2;
    }
    return at;
}

static bool is_small(int64_t rows, int64_t cols) {
    return std::min(rows, cols) <= kSmallS && std::max(rows, cols) <= kSmallCluster * kSmallUnits * kUnit;
}

// CTAs of a cluster that holds a small matrix.
static int small_ctas(int64_t l) {
    int ctas = 1;
    while ((int64_t)ctas * kSmallUnits * kUnit < l) ctas *= 2;
    return ctas;
}

// The small matrices or the others; longer ones first, so that the last tiles of a launch are short ones.
static std::vector<int> order_of(const int64_t* rows, const int64_t* cols, int n, bool small) {
    std::vector<int> o;
    for (int i = 0; i < n; ++i)
        if (rows[i] > 0 && cols[i] > 0 && is_small(rows[i], cols[i]) == small) o.push_back(i);
    std::stable_sort(o.begin(), o.end(), [&](int x, int y) {
        return std::max(rows[x], cols[x]) > std::max(rows[y], cols[y]);
    });
    return o;
}

static int check_shapes(const int64_t* rows, const int64_t* cols, int n) {
    if (n < 0) return SIDCO_E_PARAMS;
    if (n > 0 && (!rows || !cols)) return SIDCO_E_NULL;
    for (int i = 0; i < n; ++i) {
        if (rows[i] < 0 || cols[i] < 0 || rows[i] > SIDCO_ORTHO_MAX_DIM || cols[i] > SIDCO_ORTHO_MAX_DIM) return SIDCO_E_SIZE;
        if (std::min(rows[i], cols[i]) > SIDCO_ORTHO_MAX_SHORT) return SIDCO_E_SIZE;
    }
    return 0;
}

// The matrices lie apart from each other, and so do the parts of the vectors that they take up.
static int check_places(const int64_t* offsets, const int64_t* rows, const int64_t* cols, int n, uintptr_t grad, uintptr_t size,
                        uintptr_t momentum, uintptr_t out) {
    std::vector<std::pair<int64_t, int64_t>> at;
    for (int i = 0; i < n; ++i) {
        if (offsets[i] < 0 || offsets[i] > (int64_t)1 << 46) return SIDCO_E_SEGMENTS;
        if (rows[i] && cols[i]) at.emplace_back(offsets[i], offsets[i] + rows[i] * cols[i]);
    }
    std::sort(at.begin(), at.end());
    for (size_t i = 1; i < at.size(); ++i)
        if (at[i].first < at[i - 1].second) return SIDCO_E_SEGMENTS;
    const uintptr_t lo = (uintptr_t)at.front().first, hi = (uintptr_t)at.back().second;
    const auto meet = [&](uintptr_t p, uintptr_t p_size, uintptr_t q, uintptr_t q_size) {
        return p + lo * p_size < q + hi * q_size && q + lo * q_size < p + hi * p_size;
    };
    if (meet(grad, size, out, 2) || (momentum && (meet(grad, size, momentum, 4) || meet(out, 2, momentum, 4)))) return SIDCO_E_ALIAS;
    return 0;
}

static int64_t workspace_bytes(const int64_t* rows, const int64_t* cols, int n) {
    const std::vector<int> order = order_of(rows, cols, n, false);
    std::vector<Table> t(1);
    int64_t most = 0;
    for (size_t from = 0; from < order.size(); from += kMaxMats) {
        const int64_t b = lay_out(nullptr, rows, cols, order.data() + from, (int)std::min<size_t>(kMaxMats, order.size() - from),
                                  kMostPairs, t.data());
        if (b < 0) return SIDCO_E_SIZE;
        most = std::max(most, b);
    }
    return most;
}

// A launch whose set-up may overlap the end of the kernel before it (which it waits for itself).
template <typename... Args>
static cudaError_t launch(void (*kernel)(Args...), dim3 grid, int threads, size_t smem, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    if (e == cudaSuccess) sidco_internal::note_launch();
    return e;
}

static std::atomic<unsigned long long> g_wait_ns{kWaitLimitNs};
static std::atomic<int> g_drop_phase{-1};

static cudaError_t resident_pairs(int* n) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(kChainThreads);
    cfg.dynamicSmemBytes = kChainSmem;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(n, chain_kernel, &cfg);
    *n = std::min(*n, kMostPairs);
    return e == cudaSuccess && *n < 1 ? cudaErrorInvalidConfiguration : e;
}

// A stream on which the small matrices run beside the momentum pass of the others (not beside their products: a
// cooperative launch waits for the SMs, 169 us become 214 with four matrices of 128 x 1152).  It takes over from the caller's
// stream and hands back to it within one call, under the lock.  Its CTAs need whole SMs, which they get only if they come
// first: the stream has priority, and the caller's goes on when this one has been reached (300 x 1000 beside five of
// 64 x 576: 128 us, 174 one after the other; 126 alone).
// Every stream of a caller has one of its own: with one for all, a call would wait for whatever another caller's stream is
// held up by.  They are kept (a stream's id is never given to another); callers' streams after the first kMostBesides
// of a device take their small matrices themselves.
constexpr int kMostBesides = 16;

struct Beside {
    unsigned long long of = 0;        // id of the caller's stream
    cudaStream_t stream = nullptr;
    cudaEvent_t fork = nullptr, ready = nullptr, join = nullptr;
    std::mutex lock;

    cudaError_t create() {
        cudaError_t e;
        if (!stream) {
            int least, greatest;
            if ((e = cudaDeviceGetStreamPriorityRange(&least, &greatest)) != cudaSuccess) return e;
            if ((e = cudaStreamCreateWithPriority(&stream, cudaStreamNonBlocking, greatest)) != cudaSuccess) return e;
        }
        for (cudaEvent_t* event : {&fork, &ready, &join})
            if (!*event && (e = cudaEventCreateWithFlags(event, cudaEventDisableTiming)) != cudaSuccess) return e;
        return cudaSuccess;
    }
    cudaError_t begin(cudaStream_t from) {
        cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;     // (another thread may be capturing)
        cudaError_t e = cudaThreadExchangeStreamCaptureMode(&mode);
        if (e != cudaSuccess) return e;
        e = create();
        const cudaError_t back = cudaThreadExchangeStreamCaptureMode(&mode);
        if (e != cudaSuccess || (e = back) != cudaSuccess) return e;
        if ((e = cudaEventRecord(fork, from)) != cudaSuccess) return e;
        if ((e = cudaStreamWaitEvent(stream, fork, 0)) != cudaSuccess) return e;
        if ((e = cudaEventRecord(ready, stream)) != cudaSuccess) return e;
        return cudaStreamWaitEvent(from, ready, 0);
    }
    cudaError_t end(cudaStream_t to) {
        const cudaError_t e = cudaEventRecord(join, stream);
        return e != cudaSuccess ? e : cudaStreamWaitEvent(to, join, 0);
    }
};

// The one of a caller's stream, null if there are no more.
static cudaError_t beside_of(int dev, cudaStream_t s, Beside** found) {
    static Beside all[64][kMostBesides];
    static int used[64];
    static std::mutex lock;
    unsigned long long id;
    const cudaError_t e = cudaStreamGetId(s, &id);
    if (e != cudaSuccess) return e;
    const std::lock_guard<std::mutex> hold(lock);
    Beside *b = all[dev], *end = b + used[dev];
    while (b < end && b->of != id) ++b;
    if (b == end && used[dev] < kMostBesides) {
        b->of = id;
        end = b + 1;
        ++used[dev];
    }
    *found = b < end ? b : nullptr;
    return cudaSuccess;
}

template <typename T>
static cudaError_t chain(const Table& t, const void* grad, float* momentum, float mu, int nesterov, int steps, float eps,
                         uint16_t* out, uint8_t* ws, int64_t ws_bytes, int max_pairs, int* timeouts, cudaStream_t s) {
    cudaError_t e;
    double* partial = reinterpret_cast<double*>(ws);
    const int64_t at = up((int64_t)t.chunk_at[t.n] * 8, 1024);
    int* words = reinterpret_cast<int*>(ws + at);
    const Norms norms = {words,           (float*)(words + t.n), (float*)(words + 2 * t.n), (float*)(words + 3 * t.n),
                         words + 4 * t.n, words + 5 * t.n};
    unsigned* phases = (unsigned*)(words + 6 * t.n);
    // 16-byte accesses (where the matrix allows them)
    const int quads = (uintptr_t)grad % (4 * sizeof(T)) == 0 && (uintptr_t)momentum % 16 == 0;
    // (a plain launch: the first kernel waits for everything before it)
    int n_tiles = 0, most_tiles = 0;
    for (int list = 0; list < kLists; ++list) {
        n_tiles += t.tiles_at[list][t.n];
        most_tiles = std::max(most_tiles, t.tiles_at[list][t.n]);
    }
    prepare_kernel<T><<<std::max(t.n, std::min(2 * kMostPairs, (n_tiles + 255) / 256)), 256, 0, s>>>(
        t, (const T*)grad, (const float*)momentum, mu, nesterov, norms, phases, ws);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    sidco_internal::note_launch();
    if ((e = launch(momentum_kernel<T>, dim3(t.chunk_at[t.n]), 256, 0, s, t, (const T*)grad, momentum, mu, nesterov, eps, quads,
                    steps > 2 ? 2 : 1, partial, norms, ws)) != cudaSuccess)
        return e;
    if ((e = launch(again_kernel<T>, dim3(4 * kMostPairs), 256, 0, s, t, (const T*)grad, (const float*)momentum, mu, nesterov,
                    quads, steps > 2 ? 2 : 1, norms, ws)) != cudaSuccess)
        return e;
    // the workspace as rows of 128 bytes; a box is one unit (its bytes are in the tensor cores' order already)
    CUtensorMap map{};
    if (!sidco_internal::byte_map(&map, ws, 128, ws_bytes / 128, 128, 128, kUnit, false)) return cudaErrorNotSupported;
    Phases ph{};
    ph.wait_ns = g_wait_ns.load();
    ph.drop = g_drop_phase.load();
    for (int list = 0, first = 0; list < kLists; ++list) {
        ph.width[list] = t.width[list];
        ph.tiles[list] = t.tiles_at[list][t.n];
        ph.first[list] = first;
        first += ph.tiles[list];
    }
    const auto two = [](int k) { return ldexpf(1.0f, k); };
    int in = 0;
    const auto sym = [&](int left, int right, int plus, int to, float alpha, float beta, float gamma, int list = kLower) {
        const int by_norm = ph.n == 0 ? 2 : 0;                        // (the first Gram product)
        ph.p[ph.n++] = Phase{1, (int8_t)list, (int8_t)left, (int8_t)right, (int8_t)plus, (int8_t)to, (int8_t)in, 0, 1, 0, (int8_t)by_norm,
                             alpha, beta, gamma};
    };
    const auto polynomial = [&](int a, int to) {
        sym(a, a, a, to, kCc * two(kB - 2 * kA), kCb * two(kB - kA), kCa * two(kB));
    };
    const auto group_at = [&](int done) { return steps == 1 || (done == 2 && steps % 2) ? 1 : 2; };
    for (int done = 0; done < steps;) {
        const int group = group_at(done);
        sym(-1, -1, -1, kBufA, two(kA - 2 * kX), 0.0f, 0.0f);
        polynomial(kBufA, kBufB);
        if (group == 2) {
            sym(kBufB, kBufA, -1, kBufT, two(-kB), 0.0f, 0.0f);                       // B A
            sym(kBufT, kBufB, -1, kBufA2, two(-kB), 0.0f, 0.0f);                      // the next A = B A B
            polynomial(kBufA2, kBufT);
            // (both factors are rounded, so their product is only nearly symmetric, and a mirror image of one half, taken
            // for P, would turn the columns of an X of low rank: 512 x 2304 of rank 8 off by 6.0e-3 instead of 4.2e-3)
            sym(kBufT, kBufB, -1, kBufP, two(kP - 2 * kB), 0.0f, 0.0f, kWhole);
        }
        done += group;
        const int scale_p = group == 2 ? kP : kB, last = done == steps, by_norm = done == group;
        const int keep = !last && done + group_at(done) < steps;      // (what the last group takes has one part)
        ph.p[ph.n++] = Phase{0, kApply, (int8_t)(group == 2 ? kBufP : kBufB), 0, -1, 0, (int8_t)in, (int8_t)last,
                             (int8_t)(last ? 1 : 2), (int8_t)keep, (int8_t)by_norm, last ? two(-scale_p - kX) : two(-scale_p), 0.0f, 0.0f};
        in ^= 1;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2 * std::min(max_pairs, most_tiles));
    cfg.blockDim = dim3(kChainThreads);
    cfg.dynamicSmemBytes = kChainSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeCooperative;                         // all CTAs are resident: they wait for one another
    attr.val.cooperative = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, chain_kernel, map, ph, (const Tile*)(ws + t.tiles), ws, (__nv_bfloat16*)out,
                           (const float*)norms.factor, phases, timeouts);
    if (e == cudaSuccess) sidco_internal::note_launch();
    return e;
}

template <typename T>
static cudaError_t allow_small() {
    for (const auto kernel : {small_kernel<T, 1>, small_kernel<T, 2>, small_kernel<T, 4>, small_kernel<T, 8>}) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallSmem);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// Small matrices with equally many CTAs each: a cluster as large as the longest needs.
template <typename T>
static cudaError_t small_launch(const SmallMats& mats, int ctas, const void* grad, float* momentum, float mu, int nesterov,
                                int steps, float eps, uint16_t* out, int* timeouts, cudaStream_t s) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(mats.n * ctas);
    cfg.blockDim = dim3(kSmallThreads);
    cfg.dynamicSmemBytes = kSmallSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = ctas;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const auto kernel = ctas == 1 ? small_kernel<T, 1> : ctas == 2 ? small_kernel<T, 2> : ctas == 4 ? small_kernel<T, 4> : small_kernel<T, 8>;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, mats, (const T*)grad, momentum, mu, nesterov, steps, eps,
                                             (__nv_bfloat16*)out, timeouts);
    if (e == cudaSuccess) sidco_internal::note_launch();
    return e;
}

}  // namespace sidco_ortho

int sidco_internal::orthogonalize_timeouts(int* count) {
    return (int)cudaMemcpyFromSymbol(count, sidco_ortho::g_timeouts, sizeof(int));
}

int sidco_set_product_test_hooks(long long wait_us, int drop_phase) {
    if (wait_us < 0 || wait_us > 2000000 || drop_phase < -1) return SIDCO_E_PARAMS;
    sidco_ortho::g_wait_ns.store(wait_us ? (unsigned long long)wait_us * 1000ull : sidco_tc::kWaitLimitNs);
    sidco_ortho::g_drop_phase.store(drop_phase);
    const int zero = 0;
    return (int)cudaMemcpyToSymbol(sidco_ortho::g_timeouts, &zero, sizeof(int));
}

static int orthogonalize(const void* grad, int grad_type, float* momentum, float mu, int nesterov, const int64_t* offsets,
                        const int64_t* rows, const int64_t* cols, int n_mats, int steps, float eps, uint16_t* out_bf16,
                        void* workspace, size_t workspace_bytes, void* stream) {
    using namespace sidco_ortho;
    int rc = check_shapes(rows, cols, n_mats);
    if (rc) return rc;
    if (grad_type < SIDCO_T_F32 || grad_type > SIDCO_T_F16) return SIDCO_E_TYPE;
    if (steps < 1 || steps > SIDCO_ORTHO_MAX_STEPS || !(eps >= 0.0f) || !(mu >= 0.0f && mu < 1.0f)) return SIDCO_E_PARAMS;
    const std::vector<int> order = order_of(rows, cols, n_mats, false), small = order_of(rows, cols, n_mats, true);
    if (order.empty() && small.empty()) return 0;
    if (!grad || !out_bf16 || !offsets || (!workspace && !order.empty())) return SIDCO_E_NULL;
    const uintptr_t size = grad_type == SIDCO_T_F32 ? 4 : 2;
    if ((uintptr_t)grad % size || (uintptr_t)momentum % 4 || (uintptr_t)out_bf16 % 2) return SIDCO_E_ALIGN;
    if ((rc = check_places(offsets, rows, cols, n_mats, (uintptr_t)grad, size, (uintptr_t)momentum, (uintptr_t)out_bf16)))
        return rc;
    const int64_t need = sidco_ortho::workspace_bytes(rows, cols, n_mats);
    if (need < 0) return (int)need;
    if (need > 0 && ((uintptr_t)workspace % 256 || workspace_bytes < (size_t)need)) return SIDCO_E_WORKSPACE;
    static std::atomic<int> pair_count[64];   // pairs of CTAs that are resident at once
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return (int)e;
    if (dev < 0 || dev >= 64) return SIDCO_E_SIZE;
    if (!pair_count[dev].load()) {           // (setting it twice from two threads is harmless)
        const auto most = cudaFuncAttributeMaxDynamicSharedMemorySize;
        int pairs = 0;
        if ((e = allow_small<float>()) != cudaSuccess || (e = allow_small<__nv_bfloat16>()) != cudaSuccess ||
            (e = allow_small<__half>()) != cudaSuccess ||
            (e = cudaFuncSetAttribute(chain_kernel, most, kChainSmem)) != cudaSuccess ||
            (e = resident_pairs(&pairs)) != cudaSuccess)
            return (int)e;
        pair_count[dev] = pairs;
    }
    const int max_pairs = pair_count[dev].load();
    int* timeouts = nullptr;
    if ((e = cudaGetSymbolAddress((void**)&timeouts, g_timeouts)) != cudaSuccess) return (int)e;
    cudaStream_t s = (cudaStream_t)stream;
    const auto run_small = [&](cudaStream_t on) {
        cudaError_t r = cudaSuccess;
        for (size_t from = 0; from < small.size() && r == cudaSuccess;) {
            SmallMats mats;
            const int64_t longest = std::max(rows[small[from]], cols[small[from]]);
            const int ctas = small_ctas(longest);
            for (mats.n = 0; from < small.size() && mats.n < kMaxMats; ++from, ++mats.n)
                mats.m[mats.n] = {offsets[small[from]], (int)rows[small[from]], (int)cols[small[from]]};
            if (grad_type == SIDCO_T_F32)
                r = small_launch<float>(mats, ctas, grad, momentum, mu, nesterov, steps, eps, out_bf16, timeouts, on);
            else if (grad_type == SIDCO_T_BF16)
                r = small_launch<__nv_bfloat16>(mats, ctas, grad, momentum, mu, nesterov, steps, eps, out_bf16, timeouts, on);
            else
                r = small_launch<__half>(mats, ctas, grad, momentum, mu, nesterov, steps, eps, out_bf16, timeouts, on);
        }
        return r;
    };
    // (a stream that is being captured keeps to itself: a graph being built and a running call must not meet on a stream)
    cudaStreamCaptureStatus capture;
    if ((e = cudaStreamIsCapturing(s, &capture)) != cudaSuccess) return (int)e;
    Beside* beside = nullptr;
    if (!small.empty() && !order.empty() && capture == cudaStreamCaptureStatusNone &&
        (e = beside_of(dev, s, &beside)) != cudaSuccess)
        return (int)e;
    std::unique_lock<std::mutex> hold;
    if (beside) {
        hold = std::unique_lock<std::mutex>(beside->lock);
        if ((e = beside->begin(s)) != cudaSuccess) return (int)e;
        e = run_small(beside->stream);
    } else if (!small.empty()) {
        e = run_small(s);
    }
    if (e != cudaSuccess && !beside) return (int)e;
    std::vector<Table> t(1);
    for (size_t from = 0; from < order.size() && e == cudaSuccess; from += kMaxMats) {
        lay_out(offsets, rows, cols, order.data() + from, (int)std::min<size_t>(kMaxMats, order.size() - from),
                max_pairs, t.data());
        uint8_t* ws = (uint8_t*)workspace;
        if (grad_type == SIDCO_T_F32)
            e = chain<float>(t[0], grad, momentum, mu, nesterov, steps, eps, out_bf16, ws, need, max_pairs, timeouts, s);
        else if (grad_type == SIDCO_T_BF16)
            e = chain<__nv_bfloat16>(t[0], grad, momentum, mu, nesterov, steps, eps, out_bf16, ws, need, max_pairs, timeouts, s);
        else
            e = chain<__half>(t[0], grad, momentum, mu, nesterov, steps, eps, out_bf16, ws, need, max_pairs, timeouts, s);
    }
    if (beside) {                            // (also after an error: what was forked is joined)
        const cudaError_t r = beside->end(s);
        if (e == cudaSuccess) e = r;
    }
    return (int)e;
}

extern "C" {

int64_t sidco_orthogonalize_workspace_bytes(const int64_t* rows, const int64_t* cols, int n_mats) {
    try {
        const int rc = sidco_ortho::check_shapes(rows, cols, n_mats);
        return rc ? rc : sidco_ortho::workspace_bytes(rows, cols, n_mats);
    } catch (...) {                          // (the host tables did not fit)
        return SIDCO_E_SIZE;
    }
}

int sidco_orthogonalize(const void* grad, int grad_type, float* momentum, float mu, int nesterov, const int64_t* offsets,
                        const int64_t* rows, const int64_t* cols, int n_mats, int steps, float eps, uint16_t* out_bf16,
                        void* workspace, size_t workspace_bytes, void* stream) {
    try {
        return orthogonalize(grad, grad_type, momentum, mu, nesterov, offsets, rows, cols, n_mats, steps, eps, out_bf16, workspace,
                             workspace_bytes, stream);
    } catch (...) {                          // (the host tables did not fit)
        return (int)cudaErrorMemoryAllocation;
    }
}

}  // extern "C"
