// Orthogonalised updates for gfx950 (MI355X): matrices of a plan brought near to the orthogonal factor of their polar
// decomposition by Newton-Schulz products, and the optimiser step that takes such updates.
//
// A matrix M, turned so that its n rows are no more than its m columns, is scaled to X = M / (|M| + eps) and iterated:
//     A = X X^T,   B = b A + c A^2,   X <- a X + B X,
// which maps every singular value s of X to a s + b s^3 + c s^5.  All three products have the form C[i][j] = sum_k P[i][k] Q[j][k]
// with both operands' rows contiguous, for which X is kept in two layouts, as it lies in memory (R) and transposed (T), and A and B
// need none but their own.  A and A^2 are symmetric: tiles on and above the diagonal are formed, and stored twice.  Where matrices are
// wide, several steps are taken in squares alone (steps_of).
//
// Operands are fp16 numbers times a power of two that the host knows beforehand: |X| <= 1 in the spectral norm, and the polynomial
// says what that bound becomes, so that no element leaves [-2^14, 2^14] and those 2^-28 of the bound keep 11 bits.
//   FP16    one product a term.  A, B and X are rounded to 11 bits as operands; X itself is held in 22 (hi + lo) where a X is
//           added.  Result: 2e-4 to 3e-3 off (relative, depending on how the singular values are spread; 400 each of normal numbers:
//           64 x 200 2.3e-3 at most, 16 x 56 3.0e-3, 2 x 14 1.2e-2), as little as a result in bf16 is rounded by; bf16 operands are
//           1e-2 to 4e-2 off.
//   FP16X3  operands are hi + lo, 22 bits, and a product is hi hi + hi lo + lo hi: what fp32 products give, 2e-6 to 4e-6 off, or, where
//           several steps are taken at once, 2e-6 to 7e-6.
//
// What bounds it (MI355X; fp16 products of 8192 x 8192 by the vendor's library: 1240 TFLOP/s, for which the chip lowers its clock to
// 2 GHz and below): the matrix cores.  FP16X3, 32 of 2048 x 2048, three products counted: X <- a X + B X 1490 us or 1107 TFLOP/s, of which
// the tiles' ends, 12 bytes read and written an element, take a third, and symmetric products 830 us, 1120 of the tiles that are formed;
// FP16, whose ends are 10 bytes beside a third of the products, 710 us or 775 TFLOP/s, and 340 us or 910.  Ends and products most likely
// share the chip's power: workgroups that start apart, loads before stores and fewer instructions in the ends bring 1 % or nothing,
// while the same launch over other numbers takes 12 % less.  Whole calls: 0.9B model, one step, FP16X3, 71.5 ms (74 on another card); 8
// of 2048 x 5632, FP16, 4.5 ms; one of 512 x 512, FP16X3, 107 us, most of it 18 launches of 6 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "plan.h"
#include "sparseloco.h"

namespace {

using namespace splc;

constexpr int kThreads = 256;
constexpr int kPad = 64;                                     // row lengths of the operands are multiples of it, zeros behind the end
constexpr int kMostMatrices = 128;                           // of a batch: their descriptions are kernel arguments
constexpr int64_t kBatchElements = (int64_t)1 << 33;         // fp16 numbers of a batch's operands (16 GiB), but one matrix at the least
constexpr int kMostSide = 1 << 22;                           // rows and columns: offsets inside a tile's rows stay in 32 bits
constexpr int kMostSteps = SPLC_MAX_ORTHO_STEPS;

typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef float vfloat2 __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

__host__ __device__ inline int padded(int n) { return (n + kPad - 1) / kPad * kPad; }
// From a row to the next: an odd number of 128 bytes (256 where elements are hi + lo), so that the same piece of many rows lies in
// many channels of the cache (32 of 2048 x 2048, X <- a X + B X, when this was taken: FP16X3 1575 -> 1501 us, FP16 855 -> 753).
__host__ __device__ inline int stride(int n) { return (n + kPad - 1) / kPad % 2 ? padded(n) : padded(n) + kPad; }

struct Matrix {
    int64_t at;                                              // of its planes in the workspace, in elements
    int rows, cols, tensor, first;                           // first: of its workgroups in a launch
    __host__ __device__ int n() const { return rows < cols ? rows : cols; }
    __host__ __device__ bool tall() const { return rows > cols; }
    __host__ __device__ int64_t r_plane() const { return (int64_t)rows * stride(cols); }
    __host__ __device__ int64_t t_plane() const { return (int64_t)cols * stride(rows); }
    __host__ __device__ int64_t a_plane() const { return (int64_t)n() * stride(n()); }
};
struct Batch {
    int count, groups;                                       // groups: that have work in a launch
    Matrix of[kMostMatrices];
};
// Operands of a matrix: R and T of this step and of the next (one place for both where the third product does not read it: R of a
// wide matrix, T of a tall one), and squares: A, B and more.  Their elements are hi + lo where they are split, 32 of hi and the same 32
// of lo side by side, so that a row of 32 for the products is 128 bytes (4 % of a call with FP16X3); otherwise hi alone, and lo of R,
// which is no operand then, behind it.
template <bool SPLIT>
struct Planes {
    static constexpr int kParts = SPLIT ? 2 : 1;
    _Float16 *r_first, *t_first, *s_first;
    int64_t r_next, t_next, s_next;
    __host__ __device__ static int64_t elements(const Matrix& m, int squares) {
        return 2 * m.r_plane() * (m.tall() ? 2 : 1) + kParts * m.t_plane() * (m.tall() ? 1 : 2) + squares * kParts * m.a_plane();
    }
    __device__ __forceinline__ Planes(_Float16* ws, const Matrix& m) {
        r_first = ws + m.at;
        r_next = m.tall() ? 2 * m.r_plane() : 0;
        t_first = r_first + 2 * m.r_plane() + r_next;
        t_next = m.tall() ? 0 : kParts * m.t_plane();
        s_first = t_first + kParts * m.t_plane() + t_next;
        s_next = kParts * m.a_plane();
    }
    // Of hi of element (row, col) from an operand's first, rows of `ld`; and of lo from there in R.
    static __device__ __forceinline__ int64_t place(int row, int col, int ld) {
        return (int64_t)row * ld * kParts + (SPLIT ? (col & ~31) * 2 + (col & 31) : col);
    }
    static __device__ __forceinline__ int64_t r_lo(const Matrix& m) { return SPLIT ? 32 : m.r_plane(); }
    __device__ __forceinline__ _Float16* square(int i) const { return s_first + i * s_next; }
    __device__ __forceinline__ _Float16* r(int odd) const { return r_first + odd * r_next; }
    __device__ __forceinline__ _Float16* t(int odd) const { return t_first + odd * t_next; }
};

// The batch of a kernel whose first argument it is, where the arguments lie: it is indexed, and would be copied for that.
typedef __attribute__((address_space(4))) const Batch ArgumentBatch;
__device__ __forceinline__ ArgumentBatch* batch_argument() { return (ArgumentBatch*)__builtin_amdgcn_kernarg_segment_ptr(); }

// The matrix of a workgroup, and the workgroup's place in it.
__device__ __forceinline__ Matrix matrix_of(ArgumentBatch* batch, int group, int& place) {
    auto at = [&](int i) { return Matrix{batch->of[i].at, batch->of[i].rows, batch->of[i].cols, batch->of[i].tensor, batch->of[i].first}; };
    Matrix m = at(0);                                        // (a load that waits for no other: the usual one of a small launch)
    if (batch->count > 1) {
        int low = 0, high = batch->count;                    // the last one that begins at `group` or before is in [low, high)
        while (high - low > 1) {
            const int middle = (low + high) / 2;
            if (batch->of[middle].first <= group) low = middle;
            else high = middle;
        }
        m = at(low);
    }
    place = group - m.first;
    return m;
}

// Which of `groups` pieces of work a workgroup takes: neighbouring ones go to the same of the eight dies, which has 32 compute units
// and a cache of its own, 32 after another; those that do not fill all dies that way are shared out evenly.  -1: none.
__device__ __forceinline__ int group_of(int groups) {
    constexpr int kDies = 8, kRun = 32;
    const int die = blockIdx.x % kDies, i = blockIdx.x / kDies, full = groups / (kDies * kRun);
    if (i < full * kRun) return (i / kRun * kDies + die) * kRun + i % kRun;
    const int left = groups - full * kDies * kRun, each = (left + kDies - 1) / kDies, j = i - full * kRun;
    return j < each && die * each + j < left ? full * kDies * kRun + die * each + j : -1;
}

// Pairs: a 32-bit word of two fp16 numbers.  What hi leaves is exact, formed by an fma that takes hi as it is (`minus` is -1).
__device__ __forceinline__ void split2(float x, float y, float minus, half2& hi, half2& lo) {
    hi = __builtin_convertvector((vfloat2{x, y}), half2);
    lo = __builtin_convertvector((vfloat2{fmaf((float)hi.x, minus, x), fmaf((float)hi.y, minus, y)}), half2);
}
// The lower (upper) halves of two words.
__device__ __forceinline__ uint32_t lower(uint32_t first, uint32_t second) { return __builtin_amdgcn_perm(second, first, 0x05040100); }
__device__ __forceinline__ uint32_t upper(uint32_t first, uint32_t second) { return __builtin_amdgcn_perm(second, first, 0x07060302); }

__device__ __forceinline__ void split(float x, _Float16& hi, _Float16& lo) {
    hi = (_Float16)x;
    lo = (_Float16)(x - (float)hi);
}

// ---------------------------------------------------------------- what is orthogonalised

// Four consecutive elements from `at` on of a run that has n of them, +0 behind its end.
template <class T>
__device__ __forceinline__ float4 four(const T* p, uint32_t at, uint32_t n) {
    if (at + 4 <= n) return widened(cached_load4(p + at));
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (at < n) v.x = widened(p[at]);
    if (at + 1 < n) v.y = widened(p[at + 1]);
    if (at + 2 < n) v.z = widened(p[at + 2]);
    return v;
}
struct Momentum {
    float beta, rest;
    int nesterov;
};
// The matrix's elements as the orthogonalisation takes them: those of a tensor, or the step's update from momentum and gradient.
template <class T>
struct Plain {
    const T* const* x;
    __device__ __forceinline__ float4 operator()(int tensor, int64_t at, uint32_t n, float) const { return four(x[tensor] + at, 0, n); }
};
template <class G>
struct Update {
    const G* const* grad;
    float* const* m;                                         // the new momentum
    Momentum how;
    __device__ __forceinline__ float one(float moment, float g) const { return how.nesterov ? fmaf(how.beta, moment, how.rest * g) : moment; }
    __device__ __forceinline__ float4 operator()(int tensor, int64_t at, uint32_t n, float factor) const {
        const float4 moment = four(m[tensor] + at, 0, n), g = four(grad[tensor] + at, 0, n);
        return make_float4(one(moment.x, factor * g.x), one(moment.y, factor * g.y), one(moment.z, factor * g.z), one(moment.w, factor * g.w));
    }
};

__device__ __forceinline__ bool gradient_factor(const float* grad_scale, float& factor) {
    factor = grad_scale ? *grad_scale : 1.f;
    return factor - factor == 0.f;
}

__device__ __forceinline__ double group_sum(double x, double* shared) {
    for (int step = 32; step > 0; step >>= 1) x += __shfl_down(x, step);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < kThreads / 64; ++w) x += shared[w];
    return x;
}

__device__ __forceinline__ double squares(float4 v, double sum) {
    sum = fma((double)v.x, (double)v.x, sum);
    sum = fma((double)v.y, (double)v.y, sum);
    sum = fma((double)v.z, (double)v.z, sum);
    return fma((double)v.w, (double)v.w, sum);
}

// m = beta m + (1 - beta) g, and the sum of squares of a chunk of the update.
template <class G>
__global__ __launch_bounds__(kThreads) void momentum_kernel(const ChunkDesc* __restrict__ chunks, Update<G> update,
                                                            const float* __restrict__ grad_scale, double* __restrict__ partial) {
    __shared__ double shared[kThreads / 64];
    const ChunkDesc d = chunks[blockIdx.x];
    float factor;
    if (!gradient_factor(grad_scale, factor)) return;
    float* m = update.m[d.tensor] + d.offset;
    const G* grad = update.grad[d.tensor] + d.offset;
    const Momentum how = update.how;
    float4 g[4], x[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uint32_t at = s * 1024 + threadIdx.x * 4;
        g[s] = four(grad, at, d.n_c);
        x[s] = four(m, at, d.n_c);
    }
    double sum = 0.0;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uint32_t at = s * 1024 + threadIdx.x * 4;
        auto one = [&](float& moment, float gradient) {
            gradient *= factor;
            moment = fmaf(how.rest, gradient, how.beta * moment);
            return update.one(moment, gradient);
        };
        float4 u;
        u.x = one(x[s].x, g[s].x);
        u.y = one(x[s].y, g[s].y);
        u.z = one(x[s].z, g[s].z);
        u.w = one(x[s].w, g[s].w);
        if (at + 4 <= d.n_c) {
            stream_store4(m + at, x[s]);
        } else {
            if (at < d.n_c) m[at] = x[s].x;
            if (at + 1 < d.n_c) m[at + 1] = x[s].y;
            if (at + 2 < d.n_c) m[at + 2] = x[s].z;
        }
        sum = squares(u, sum);
    }
    sum = group_sum(sum, shared);
    if (threadIdx.x == 0) partial[d.id] = sum;
}

template <class T>
__global__ __launch_bounds__(kThreads) void squares_kernel(const ChunkDesc* __restrict__ chunks, const T* const* __restrict__ x,
                                                           double* __restrict__ partial) {
    __shared__ double shared[kThreads / 64];
    const ChunkDesc d = chunks[blockIdx.x];
    const T* p = x[d.tensor] + d.offset;
    float4 v[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) v[s] = four(p, s * 1024 + threadIdx.x * 4, d.n_c);
    double sum = 0.0;
#pragma unroll
    for (int s = 0; s < 4; ++s) sum = squares(v[s], sum);
    sum = group_sum(sum, shared);
    if (threadIdx.x == 0) partial[d.id] = sum;
}

// 1 / (|M| + eps) of every tensor, from its chunks' sums.
__global__ __launch_bounds__(kThreads) void inverse_norm_kernel(const int64_t* __restrict__ numel, const double* __restrict__ partial,
                                                                double eps, double* __restrict__ inverse) {
    __shared__ double shared[kThreads / 64];
    __shared__ int64_t first_of[kThreads / 64];
    int64_t first = 0;
    for (int i = threadIdx.x; i < (int)blockIdx.x; i += kThreads) first += (numel[i] + kChunk - 1) / kChunk;
    for (int step = 32; step > 0; step >>= 1) first += __shfl_xor(first, step);
    if ((threadIdx.x & 63) == 0) first_of[threadIdx.x >> 6] = first;
    __syncthreads();
    first = 0;
    for (int w = 0; w < kThreads / 64; ++w) first += first_of[w];
    const int64_t chunks = (numel[blockIdx.x] + kChunk - 1) / kChunk;
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < chunks; i += kThreads) sum += partial[first + i];
    sum = group_sum(sum, shared);
    if (threadIdx.x == 0) inverse[blockIdx.x] = 1.0 / (sqrt(sum) + eps);
}

// X of the first step in both layouts, 64 x 64 elements a workgroup.
template <class From, bool SPLIT>
__global__ __launch_bounds__(kThreads) void scale_kernel(Batch, From from, const float* __restrict__ grad_scale,
                                                         const double* __restrict__ inverse, float range, _Float16* __restrict__ ws) {
    __shared__ float tile[64][65];
    float factor;
    if (!gradient_factor(grad_scale, factor)) return;
    int place;
    const Matrix m = matrix_of(batch_argument(), (int)blockIdx.x, place);
    const Planes<SPLIT> planes(ws, m);
    const int across = padded(m.cols) / 64, r0 = place / across * 64, c0 = place % across * 64;
    const int ldc = stride(m.cols), ldr = stride(m.rows), line = threadIdx.x / 16, four_of = threadIdx.x % 16 * 4;
    const double scale = inverse[m.tensor] * (double)range;
    constexpr int kEach = 4, kLines = kThreads / 16;         // rows of a lane, four columns of each; then columns, four rows of each
    float4 x[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int r = r0 + line + i * kLines, c = c0 + four_of;
        x[i] = r < m.rows && c < m.cols ? from(m.tensor, (int64_t)r * m.cols + c, (uint32_t)(m.cols - c < 4 ? m.cols - c : 4), factor)
                                        : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    auto split4 = [](const float* v, half4& hi, half4& lo) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            _Float16 h, l;
            split(v[e], h, l);
            hi[e] = h;
            lo[e] = l;
        }
    };
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int r = r0 + line + i * kLines, c = c0 + four_of;
        const float v[4] = {(float)((double)x[i].x * scale), (float)((double)x[i].y * scale), (float)((double)x[i].z * scale),
                            (float)((double)x[i].w * scale)};
#pragma unroll
        for (int e = 0; e < 4; ++e) tile[line + i * kLines][four_of + e] = v[e];
        if (r >= m.rows) continue;
        half4 hi, lo;
        split4(v, hi, lo);
        _Float16* p = planes.r(0) + planes.place(r, c, ldc);
        *(half4*)p = hi;
        *(half4*)(p + planes.r_lo(m)) = lo;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int c = c0 + line + i * kLines, r = r0 + four_of;
        if (c >= m.cols) break;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = tile[four_of + e][line + i * kLines];
        half4 hi, lo;
        split4(v, hi, lo);
        _Float16* p = planes.t(0) + planes.place(c, r, ldr);
        *(half4*)p = hi;
        if (SPLIT) *(half4*)(p + 32) = lo;
    }
}

// ---------------------------------------------------------------- products

// GRAM: X X^T into a square.  SQUARE: a square times a square, which commute.  APPLY: a square times X; LAST: the result's step.
enum { GRAM = 0, SQUARE = 1, APPLY = 2, LAST = 3 };

// One product: sum * product + old * own + other * more, in the result's range.  The squares p and q that it multiplies (APPLY: p alone),
// those that it adds (other: -1, none) and the one that it writes; APPLY adds to X itself.
struct Product {
    int step;
    float product, own, more;
    int8_t p, q, old, other, out;
};
struct Result {                                              // of the last step
    int to;                                                  // SPLC_F32, SPLC_BF16: the matrix itself; -1: the parameters' step
    void* const* out;                                        // tensors, or theta
    uint16_t* const* copy;
    const float* decay;
    float size, shrink;
    int adjust;
};

typedef __attribute__((address_space(1))) const void global_void;
typedef __attribute__((address_space(3))) void shared_void;

// How a tile of C = P Q^T is shared out: WR x WC waves with IR x 1 blocks of SIDE x SIDE elements each in their registers, or (WK) WK
// waves with the same block, which take turns along k.  DEEP: buffers for BK of k.
template <int WR_, int WC_, int WK_, int IR_, int SIDE_, int BK_, int DEEP_, bool SPLIT_>
struct Shape {
    static constexpr int WR = WR_, WC = WC_, WK = WK_, IR = IR_, kSide = SIDE_, BK = BK_, kDeep = DEEP_;
    static constexpr int kWaves = WR_ * WC_ * WK_, kLanes = kWaves * 64, kTile = WC_ * SIDE_;
    static constexpr bool SPLIT = SPLIT_;
    static constexpr int kBytes = DEEP_ * 2 * kTile * BK_ * (SPLIT_ ? 4 : 2), kWavesASimd = (kWaves + 3) / 4 * (2 * kBytes <= 160 * 1024 ? 2 : 1);
    static_assert(kPad % BK_ == 0, "whole rows of operands");
    static_assert(WR_ * IR_ == WC_, "square tiles");
    static_assert(WK_ == 1 || (WC_ == 1 && IR_ == 1), "one block where waves share k");
    // Workgroups of a launch for a matrix: all of its tiles, or those on and above its diagonal, column by column.  Tiles cover the
    // padding of rows of operands, too, which they clear.
    static __host__ __device__ int down(int rows) { return (padded(rows) + kTile - 1) / kTile; }
    static int64_t tiles(const Matrix& m) { return (int64_t)down(m.rows) * down(m.cols); }
    static int64_t triangle(const Matrix& m) { return (int64_t)down(m.n()) * (down(m.n()) + 1) / 2; }
    static __device__ __forceinline__ void triangle_place(int place, int& ti, int& tj) {
        tj = (int)((sqrtf(8.f * (float)place + 1.f) - 1.f) * 0.5f);
        while (tj * (tj + 1) / 2 > place) --tj;
        while ((tj + 1) * (tj + 2) / 2 <= place) ++tj;
        ti = place - tj * (tj + 1) / 2;
    }
};

// Element (row, col) of a wave's block of sums in LDS: groups of four columns are exchanged by the row, so that writing four columns
// of many rows, reading eight columns of eight rows and reading eight rows of eight columns each find all banks (where SIDE is 64).
template <int SIDE>
__device__ __forceinline__ int in_block(int row, int group) { return row * SIDE + ((group ^ row ^ (row >> 3)) & (SIDE / 4 - 1)) * 4; }

// A row of fp16 numbers in LDS is ROW / 8 pieces of 16 bytes, and the pieces of a row are exchanged by its number: of 16 consecutive
// rows, the same piece lies in 16 different places of the 256 bytes that the banks are wide, as reading it in 16 lanes at once needs.
template <int ROW>
__device__ __forceinline__ int exchange(int row) {
    constexpr int kPieces = ROW / 8, kBeside = 16 / kPieces > 1 ? 16 / kPieces : 1;   // rows that lie side by side in the banks
    return row / kBeside & (kPieces < 16 ? kPieces - 1 : 15);
}

// BK elements (hi, lo) of every row of P and Q at a time go to LDS, without passing registers, while those before them are multiplied.
// Then the sums pass LDS, block by block, to be finished and stored along rows of C, 16 bytes a lane, and once more along its columns
// for the transposed (or mirrored) copy.  (0.9B model, one step: sums stored from where the products leave them, tiles of 128, 141 ms;
// through LDS 126; tiles of 256 120; operands of the next 16 of k read beside the products 114.5; hi and lo side by side 106; large
// batches 92; steps in squares 76; loads issued between products 72; sums ended in pairs of numbers 71.4.)
template <class S, int STEP>
__global__ __launch_bounds__(S::kLanes, S::kWavesASimd) void product_kernel(Batch, Product f, Result result, int odd,
                                                                            const float* __restrict__ grad_scale, _Float16* __restrict__ ws) {
    constexpr bool SPLIT = S::SPLIT;
    constexpr int SIDE = S::kSide;
    constexpr int kParts = SPLIT ? 2 : 1, BK = S::BK, kRow = BK * kParts, kPieces = kRow / 8, kRowsALoad = 64 / kPieces;
    constexpr int kLoads = S::kTile * kRow / 512 / S::kWaves;    // of a wave for P, and as many for Q
    static_assert(kLoads * S::kWaves * 512 == S::kTile * kRow, "whole loads");
    __shared__ __align__(1024) union {
        struct {
            _Float16 p[S::kTile * kRow], q[S::kTile * kRow];
        } operands[S::kDeep];
        float blocks[S::kWaves][SIDE * SIDE];
    } lds;
    static_assert(sizeof(lds) <= 160 * 1024, "LDS");

    int place;
    const int group = group_of(batch_argument()->groups);
    if (group < 0) return;
    const Matrix m = matrix_of(batch_argument(), group, place);
    const Planes<SPLIT> planes(ws, m);
    const int n = m.n(), ldn = stride(n), ldc = stride(m.cols), ldr = stride(m.rows);
    int ti, tj;
    if (STEP == GRAM || STEP == SQUARE) {
        S::triangle_place(place, ti, tj);
    } else {
        ti = place % S::down(m.rows);
        tj = place / S::down(m.rows);
    }
    const _Float16 *p, *q;
    int p_rows, q_rows, depth, ld_p, ld_q;
    if (STEP == GRAM) {
        p = q = m.tall() ? planes.t(odd) : planes.r(odd);
        p_rows = q_rows = n;
        depth = padded(m.tall() ? m.rows : m.cols);
        ld_p = ld_q = m.tall() ? ldr : ldc;
    } else if (STEP == SQUARE) {
        p = planes.square(f.p);
        q = planes.square(f.q);
        p_rows = q_rows = n;
        depth = padded(n);
        ld_p = ld_q = ldn;
    } else {
        p = m.tall() ? planes.r(odd) : planes.square(f.p);
        q = m.tall() ? planes.square(f.p) : planes.t(odd);
        p_rows = m.rows;
        q_rows = m.cols;
        depth = padded(n);
        ld_p = ld_q = ldn;
    }
    depth *= kParts;                                         // fp16 numbers of a row
    ld_p *= kParts;
    ld_q *= kParts;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = ti * S::kTile, col0 = tj * S::kTile;
    // (rows that are not there, up to all of a tile's, are read as the last one that is)
    const int first[2] = {row0 < p_rows ? row0 : p_rows - 1, col0 < q_rows ? col0 : q_rows - 1};
    const _Float16* from[2] = {p + (int64_t)first[0] * ld_p, q + (int64_t)first[1] * ld_q};
    uint32_t offset[2][kLoads];                              // of this lane's 16 bytes from the tile's first element, in elements
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const int last = (side ? q_rows : p_rows) - 1 - first[side];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = (wave + i * S::kWaves) * kRowsALoad + lane / kPieces, piece = (lane % kPieces) ^ exchange<kRow>(row);
            offset[side][i] = (uint32_t)(row < last ? row : last) * (uint32_t)(side ? ld_q : ld_p) + (uint32_t)piece * 8u;
        }
    }
    auto fetch = [&](int k, int buffer) {
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            _Float16* to = side ? lds.operands[buffer].q : lds.operands[buffer].p;
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                __builtin_amdgcn_global_load_lds((global_void*)(from[side] + k + offset[side][i]),
                                                 (shared_void*)(to + (wave + i * S::kWaves) * 512), 16, 0, 0);
        }
    };
    constexpr int kI = SIDE / 32 * S::IR, kJ = SIDE / 32, kSteps = BK / 16 / S::WK;
    v16f sum[kI][kJ];
#pragma unroll
    for (int i = 0; i < kI; ++i) {
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[i][j][e] = 0.f;
        }
    }
    const int wave_k = wave % S::WK, wave_at = wave / S::WK;
    const int wave_row = wave_at / S::WC * (SIDE * S::IR), wave_col = wave_at % S::WC * SIDE;
    struct Operands {
        half8 x[kI][kParts], y[kJ][kParts];
    };
    constexpr bool kTriangle = STEP == GRAM || STEP == SQUARE;
    const int rows = kTriangle ? n : m.rows, cols = kTriangle ? n : m.cols, ld = kTriangle ? ldn : ldc, ld_t = kTriangle ? ldn : ldr;
    // a X is added here, to X as hi + lo, and not as part of B: its sums would be four times as large, and so would their roundings
    // (1.4 times the error of fp32 products where it is 0.7 times so).
    constexpr bool kOld = STEP != GRAM, kOldLo = STEP != SQUARE || SPLIT;
    const int64_t r_lo = planes.r_lo(m);
    const _Float16* old = STEP == SQUARE ? planes.square(f.old) : planes.r(odd);
    _Float16* to = kTriangle ? planes.square(f.out) : planes.r(odd ^ 1);
    _Float16* to_t = kTriangle ? to : planes.t(odd ^ 1);
    // Passes over a block, by one wave or by all that share it: 8 columns a lane along its rows, then 8 rows a lane along its columns.
    constexpr int kAcross = SIDE / 8, kDown = 64 / kAcross, kPasses = SIDE / kDown / S::WK > 0 ? SIDE / kDown / S::WK : 1;
    const bool passes = wave_k * kPasses * kDown < SIDE;
    half8 old_hi[kOld ? kPasses : 1], old_lo[kOld && kOldLo ? kPasses : 1];
    auto load_old = [&](int block_row, int block_col) {
        if (!kOld || !passes) return;
#pragma unroll
        for (int pass = 0; pass < kPasses; ++pass) {
            const int row = block_row + (wave_k * kPasses + pass) * kDown + lane / kAcross, col = block_col + lane % kAcross * 8;
            if (row >= rows || col >= ld) continue;
            const _Float16* from_old = old + planes.place(row, col, ld);
            old_hi[pass] = *(const half8*)from_old;
            if (kOldLo) old_lo[pass] = *(const half8*)(from_old + (STEP == SQUARE ? 32 : r_lo));
        }
    };
    if (S::WK > 1) load_old(row0, col0);                     // (few registers: their latency passes beside the products')
    const int swap = exchange<kRow>(lane & 31);
    auto load = [&](Operands& o, int buffer, int kk) {
        const int at = (wave_k * kSteps + kk) * 2 + (lane >> 5), hi = SPLIT ? (at & ~3) * 2 + (at & 3) : at;
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            const int piece = ((hi + part * 4) ^ swap) * 8;
#pragma unroll
            for (int i = 0; i < kI; ++i)
                o.x[i][part] = *(const half8*)&lds.operands[buffer].p[(wave_row + i * 32 + (lane & 31)) * kRow + piece];
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                o.y[j][part] = *(const half8*)&lds.operands[buffer].q[(wave_col + j * 32 + (lane & 31)) * kRow + piece];
        }
    };
    // Waits for what was fetched first of so many fetches, and for the operands from LDS; then for all waves.
    constexpr int kAhead = S::kDeep - 1, kWaiting = (kAhead - 1) * 2 * kLoads;
    static_assert(kWaiting < 64, "loads that a wave counts");
    auto arrived = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((kWaiting & 15) | kWaiting >> 4 << 14 | 7 << 4);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto multiply = [&](const Operands& o) {
#pragma unroll
        for (int term = SPLIT ? 2 : 0; term >= 0; --term) {
#pragma unroll
            for (int i = 0; i < kI; ++i) {
#pragma unroll
                for (int j = 0; j < kJ; ++j)                 // columns of C in a lane's registers, rows over the lanes
                    sum[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.y[j][term == 1], o.x[i][term == 2], sum[i][j], 0, 0, 0);
            }
        }
    };
    // Loads from LDS (and fetches) issue between products, which take the matrix cores longer than that.
    constexpr int kProducts = kI * kJ * (SPLIT ? 3 : 1), kReads = (kI + kJ) * kParts, kFetches = 2 * kLoads;
    auto interleave = [&](bool fetches) {
        constexpr int kFirst = 1;
#pragma unroll
        for (int i = 0; i < kProducts; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (fetches && i >= kFirst && i - kFirst < kFetches) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            if (i < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
    };
    Operands now, next;
    const int last = depth - kRow;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(i * kRow < last ? i * kRow : last, i);
    arrived();
    fetch(kAhead * kRow < last ? kAhead * kRow : last, kAhead);
    load(now, 0, 0);
    // The operands of the next 16 of k come from LDS while those at hand are multiplied, across the barrier too: it says that all waves
    // have read a buffer to its end, and that the next one has arrived.  (Behind the end of k the last part is fetched again, so that
    // what a wave waits for is always as many loads; nothing reads it.)
    int buffer = 0;
    for (int k = 0; k < last; k += kRow) {
        const int after = buffer + 1 < S::kDeep ? buffer + 1 : 0, ahead = k + S::kDeep * kRow;
#pragma unroll
        for (int kk = 0; kk + 1 < kSteps; ++kk) {
            load(next, buffer, kk + 1);
            multiply(now);
            interleave(false);
            now = next;
        }
        arrived();
        fetch(ahead < last ? ahead : last, buffer);
        load(next, after, 0);
        multiply(now);
        interleave(true);
        now = next;
        buffer = after;
    }
#pragma unroll
    for (int kk = 0; kk < kSteps; ++kk) {
        if (kk + 1 < kSteps) load(next, buffer, kk + 1);
        multiply(now);
        now = next;
    }
    // The last fetches are still under way, and have to have landed, of all waves, before sums take the operands' place in LDS: a barrier
    // by itself waits for no load.
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(15 << 8 | 7 << 4);            // vmcnt(0)
    asm volatile("" ::: "memory");
    if (STEP == LAST && result.to < 0) {
        float factor;
        if (!gradient_factor(grad_scale, factor)) return;
    }
    float keep = 0.f, size = 0.f;
    if (STEP == LAST && result.to < 0) {
        const float rows = (float)m.rows, cols = (float)m.cols;
        keep = 1.f - (result.decay ? result.shrink * result.decay[m.tensor] : result.shrink);
        size = result.size * (result.adjust == SPLC_MUON_ASPECT ? sqrtf(fmaxf(1.f, rows / cols))
                              : result.adjust == SPLC_MUON_RMS  ? 0.2f * sqrtf(fmaxf(rows, cols))
                                                                : 1.f);
    }
    float minus = -1.f;
    asm("" : "+s"(minus));                                   // (an fma with a known -1 would become a conversion and a subtraction)
    __syncthreads();
#pragma unroll
    for (int half = 0; half < S::IR; ++half) {
        const int block_row = row0 + wave_row + half * SIDE, block_col = col0 + wave_col;
        if (kTriangle && block_row > block_col) continue;    // below the diagonal: another block's mirror image
        const bool whole = block_row + SIDE <= rows && block_col + SIDE <= cols;
        float* mine = lds.blocks[wave];
        if (S::WK == 1) load_old(block_row, block_col);
#pragma unroll
        for (int i = 0; i < SIDE / 32; ++i) {
#pragma unroll
            for (int j = 0; j < SIDE / 32; ++j) {
                // register e of lane l: row l % 32, column 8 (e / 4) + 4 (l / 32) + e % 4
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    vfloat4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = f.product * sum[half * (SIDE / 32) + i][j][g * 4 + e];
                    *(float4*)&mine[in_block<SIDE>(i * 32 + (lane & 31), j * 8 + g * 2 + (lane >> 5))] = make_float4(v.x, v.y, v.z, v.w);
                }
            }
        }
        if (S::WK > 1) {
            __syncthreads();
            mine = lds.blocks[0];
        }
#pragma unroll
        for (int pass = 0; pass < kPasses; ++pass) {
            if (!passes) break;
            const int in_row = (wave_k * kPasses + pass) * kDown + lane / kAcross, row = block_row + in_row;
            const int in_col = lane % kAcross * 8, col = block_col + in_col;
            float* at[2] = {mine + in_block<SIDE>(in_row, in_col / 4), mine + in_block<SIDE>(in_row, in_col / 4 + 1)};
            float v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float4 x = *(const float4*)at[h];
#pragma unroll
                for (int w = 1; w < S::WK; ++w) {
                    const float4 y = *(const float4*)(at[h] + w * SIDE * SIDE);
                    x.x += y.x;
                    x.y += y.y;
                    x.z += y.z;
                    x.w += y.w;
                }
                v[4 * h] = x.x;
                v[4 * h + 1] = x.y;
                v[4 * h + 2] = x.z;
                v[4 * h + 3] = x.w;
            }
            const bool there = row < rows && col < ld;
            if (kOld && there) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (kOldLo) v[e] = fmaf((float)old_lo[pass][e], f.own, v[e]);
                    v[e] = fmaf((float)old_hi[pass][e], f.own, v[e]);
                }
            }
            if (STEP == SQUARE && SPLIT && f.other >= 0 && there) {
                const _Float16* from_other = planes.square(f.other) + planes.place(row, col, ld);
                const half8 hi = *(const half8*)from_other, lo = *(const half8*)(from_other + 32);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf((float)hi[e], f.more, fmaf((float)lo[e], f.more, v[e]));
            }
            if (STEP != LAST) {
                if (!whole) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!there || col + e >= cols) v[e] = 0.f;
                }
                union {
                    half8 all;
                    half2 of[4];
                    uint32_t word[4];
                } hi, lo;
                uint32_t word[8];
                constexpr bool kLo = SPLIT || STEP == APPLY;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (kLo) split2(v[2 * e], v[2 * e + 1], minus, hi.of[e], lo.of[e]);
                    else hi.of[e] = __builtin_convertvector((vfloat2{v[2 * e], v[2 * e + 1]}), half2);
                }
                if (there) {
                    _Float16* dst = to + planes.place(row, col, ld);
                    *(half8*)dst = hi.all;
                    if (kLo) *(half8*)(dst + (STEP == APPLY ? r_lo : 32)) = lo.all;
                }
                // back as a word an element: hi, and lo above it where the transposed copy has it
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t first = hi.word[e / 2], second = SPLIT ? lo.word[e / 2] : 0;
                    word[e] = SPLIT ? (e % 2 ? upper(first, second) : lower(first, second)) : e % 2 ? first >> 16 : first;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) *(uint4*)at[h] = make_uint4(word[4 * h], word[4 * h + 1], word[4 * h + 2], word[4 * h + 3]);
            } else if (there) {
                const int64_t place_of = (int64_t)row * m.cols + col;
                const int count = m.cols - col < 8 ? m.cols - col : 8;
                if (result.to < 0) {
                    float* theta = static_cast<float*>(result.out[m.tensor]) + place_of;
                    uint16_t* copy = result.copy ? result.copy[m.tensor] + place_of : nullptr;
                    if (count == 8) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float4 x = cached_load4(theta + 4 * h);
                            x.x = fmaf(-size, v[4 * h], x.x * keep);
                            x.y = fmaf(-size, v[4 * h + 1], x.y * keep);
                            x.z = fmaf(-size, v[4 * h + 2], x.z * keep);
                            x.w = fmaf(-size, v[4 * h + 3], x.w * keep);
                            stream_store4(theta + 4 * h, x);
                            if (copy) stream_store4(copy + 4 * h, x);
                        }
                    } else {
                        for (int e = 0; e < count; ++e) {
                            const float now = fmaf(-size, v[e], theta[e] * keep);
                            theta[e] = now;
                            if (copy) copy[e] = (uint16_t)bf16_pair(now, 0.f);
                        }
                    }
                } else if (result.to == SPLC_BF16) {
                    uint16_t* out = static_cast<uint16_t*>(result.out[m.tensor]) + place_of;
                    if (count == 8) {
                        stream_store4(out, make_float4(v[0], v[1], v[2], v[3]));
                        stream_store4(out + 4, make_float4(v[4], v[5], v[6], v[7]));
                    } else {
                        for (int e = 0; e < count; ++e) out[e] = (uint16_t)bf16_pair(v[e], 0.f);
                    }
                } else {
                    float* out = static_cast<float*>(result.out[m.tensor]) + place_of;
                    if (count == 8) {
                        stream_store4(out, make_float4(v[0], v[1], v[2], v[3]));
                        stream_store4(out + 4, make_float4(v[4], v[5], v[6], v[7]));
                    } else {
                        for (int e = 0; e < count; ++e) out[e] = v[e];
                    }
                }
            }
        }
        if (STEP == LAST || (kTriangle && block_row == block_col)) {
            if (S::IR > 1) __builtin_amdgcn_wave_barrier();
            continue;
        }
        if (S::WK > 1) __syncthreads();
        else __builtin_amdgcn_wave_barrier();                // (LDS takes a wave's accesses in their order)
#pragma unroll 2
        for (int pass = 0; pass < kPasses; ++pass) {
            if (!passes) break;
            const int in_col = (wave_k * kPasses + pass) * kDown + lane % kDown, in_row = lane / kDown * 8;
            const int col = block_col + in_col, row = block_row + in_row;
            uint32_t word[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) word[e] = __float_as_uint(mine[in_block<SIDE>(in_row + e, in_col >> 2) + (in_col & 3)]);
            if (col < cols && row < ld_t) {
                _Float16* dst = to_t + planes.place(col, row, ld_t);
                *(uint4*)dst = make_uint4(lower(word[0], word[1]), lower(word[2], word[3]), lower(word[4], word[5]), lower(word[6], word[7]));
                if (SPLIT)
                    *(uint4*)(dst + 32) = make_uint4(upper(word[0], word[1]), upper(word[2], word[3]), upper(word[4], word[5]), upper(word[6], word[7]));
            }
        }
        if (S::IR > 1) __builtin_amdgcn_wave_barrier();
    }
}

// ---------------------------------------------------------------- host

bool finite64(double v) { return std::isfinite(v); }

// The largest value in [0, most], at its end or where the derivative vanishes.
double largest(double a, double b, double c, double most) {  // of |a x + b x^3 + c x^5|
    auto p = [&](double x) { return std::fabs(x * (a + x * x * (b + x * x * c))); };
    double found = p(most);
    // a + 3 b y + 5 c y^2 = 0, y = x^2
    if (c == 0.0) {
        if (b != 0.0 && -a / (3 * b) > 0.0 && -a / (3 * b) < most * most) found = std::max(found, p(std::sqrt(-a / (3 * b))));
        return found;
    }
    const double in_root = 9 * b * b - 20 * a * c;
    if (in_root >= 0.0)
        for (double sign : {-1.0, 1.0}) {
            const double y = (-3 * b + sign * std::sqrt(in_root)) / (10 * c);
            if (y > 0.0 && y < most * most) found = std::max(found, p(std::sqrt(y)));
        }
    return found;
}
double largest_even(double b, double c, double most) {       // of |b y + c y^2|, y in [0, most]
    auto p = [&](double y) { return std::fabs(y * (b + c * y)); };
    double found = p(most);
    if (c != 0.0 && -b / (2 * c) > 0.0 && -b / (2 * c) < most) found = std::max(found, p(-b / (2 * c)));
    return found;
}

// The products of all steps in their order, with the powers of two that their results are held times.
struct Steps {
    std::vector<Product> of;
    float first = 0.f;                                       // of X before the first step
};
// Several steps at once in squares alone, which are the smaller matrices where X is wide: one step, X <- p(A) X with p(A) = a + B,
// makes A into p A p, and for several of them
//     A = X X^T;   for each:  B = b A + c A^2,  Q <- p Q,  A <- p (p A);   X <- Q X,
// where only the first A and the last product have X's long side.  Q is held without its multiple of 1, alpha, as B is: both are zero
// where X is small.  alpha is what roundings of Q and of A grow by before they come to X: at most 64, of at most three steps
// (40 for the usual polynomial; five steps without a new A from X: 60 times the error).  900 x 1801, beside fp32 products: usual, normal
// numbers 2.4e-6 and 2.4e-6 off, with four strong directions 6.6e-6 and 3.5e-6; three polynomials of alpha 63 5.6e-6 and 1.2e-6.
constexpr double kMostAlpha = 64.0;
constexpr int kMostAtOnce = 3, kSquares = 2, kSquaresAtOnce = 5;

bool steps_of(const double* coefficients, int steps, bool at_once, Steps& s) {
    static const double usual[] = {3.4445, -4.7750, 2.0315};
    if (steps < 1 || steps > kMostSteps) return false;
    // (a bound may be as small as polynomials that shrink X make it)
    auto range = [](double bound) { return bound > 0.0 ? 14 - (int)std::ceil(std::log2(bound)) : 14; };
    // B, or Q without its multiple of 1, beside that multiple: what is 2^-40 of it is nothing to 22 bits, and its range stays near.
    auto beside = [&](double bound, double one) { return range(std::max(bound, std::ldexp(std::fabs(one), -40))); };
    auto power = [](double v, int exponent) { return (float)std::ldexp(v, exponent); };
    auto at = [&](int k) { return coefficients ? coefficients + 3 * k : usual; };
    double most = 1.0;                                       // bound on the singular values of X
    int x = range(most);
    s.of.clear();
    s.first = power(1.0, x);
    for (int k = 0; k < steps; ++k)
        for (int i = 0; i < 3; ++i)
            if (!finite64(at(k)[i]) || std::fabs(at(k)[i]) > 1e4) return false;
    for (int k = 0; k < steps;) {
        int count = 1;
        double alpha = at(k)[0];
        while (at_once && count < kMostAtOnce && k + count < steps && std::fabs(alpha * at(k + count)[0]) <= kMostAlpha)
            alpha *= at(k + count++)[0];
        // |Q - alpha| for singular values up to the bound, at many of them; half as much again for those between.
        std::vector<double> largest_q((size_t)count, 0.0);
        for (int i = 0; count > 1 && i <= 512; ++i) {
            double v = most * i / 512, q = 1.0, of_one = 1.0;
            for (int j = 0; j < count; ++j) {
                const double* p = at(k + j);
                const double f = p[0] + v * v * (p[1] + v * v * p[2]);
                q *= f;
                v *= f;
                of_one *= p[0];
                largest_q[(size_t)j] = std::max(largest_q[(size_t)j], 1.5 * std::fabs(q - of_one));
            }
        }
        int a = range(most * most), q = 0, in_q = 0, in_b = 1, free = 3;
        s.of.push_back({GRAM, power(1.0, a - 2 * x), 0.f, 0.f, 0, 0, 0, -1, 0});
        alpha = 1.0;
        for (int j = 0; j < count; ++j) {
            const double* p = at(k + j);
            const int b = beside(largest_even(p[1], p[2], most * most), p[0]);
            s.of.push_back({SQUARE, power(p[2], b - 2 * a), power(p[1], b - a), 0.f, 0, 0, 0, -1, (int8_t)in_b});
            if (j == 0) {
                q = b;
                in_q = in_b;
                in_b = 3;
                free = 4;
            } else {
                const int next_q = beside(largest_q[(size_t)j], alpha * p[0]);
                s.of.push_back({SQUARE, power(1.0, next_q - b - q), power(p[0], next_q - q), power(alpha, next_q - b), (int8_t)in_b,
                                (int8_t)in_q, (int8_t)in_q, (int8_t)in_b, (int8_t)free});
                q = next_q;
                std::swap(in_q, free);                       // (what was Q is free, and B is below)
                std::swap(in_b, free);
            }
            alpha *= p[0];
            const double grown = largest(p[0], p[1], p[2], most);
            if (!finite64(grown) || grown > 1024.0) return false;
            if (j + 1 < count) {
                const int holds_b = j == 0 ? in_q : free;    // B of this step
                const int t = range(most * grown), next_a = range(grown * grown);
                s.of.push_back({SQUARE, power(1.0, t - b - a), power(p[0], t - a), 0.f, (int8_t)holds_b, 0, 0, -1, 2});
                s.of.push_back({SQUARE, power(1.0, next_a - b - t), power(p[0], next_a - t), 0.f, (int8_t)holds_b, 2, 2, -1, 0});
                a = next_a;
            }
            most = grown;
        }
        k += count;
        const int next = k < steps ? range(most) : 0;
        s.of.push_back({k < steps ? APPLY : LAST, power(1.0, next - q - x), power(alpha, next - x), 0.f, (int8_t)in_q, 0, 0, -1, 0});
        x = next;
    }
    return true;
}

// Tiles of a launch by their side, 32 << size, and what they take (us) where the longest product has `depth` terms: as many rounds as
// tiles fit on 256 compute units, one, or two of those that LDS holds twice (of which the last half, alone on its units, takes 0.55 of
// a round), and for a round what was measured.  MI355X, us: 32 of 2048 x 2048, FP16X3, products of 2048 terms, 8 rounds of 256 tiles 1500;
// 3 of 5630 x 2050, symmetric ones of 2050 and of 5630 terms, a round of 128 tiles 125 and 301; 9 of 768 x 2048, of 768 and 2048 terms, 3
// rounds of 64 tiles 38 and 72.  Where tiles of 32 x 32 all run at once latency counts, and those are shortest: one of 512 x 512, the
// whole call, 110 us, with tiles of 64 155; of 768 x 768, which has more of them, 214 and 184.
enum { TINY, SMALL, MIDDLE, LARGE };
struct Tile {
    int size;
    double us;
};
Tile tile_of(const int64_t (&tiles)[4], double depth, bool split) {
    if (tiles[TINY] <= (split ? 256 : 512)) return {TINY, 3.0 + depth * 0.006};
    auto rounds = [](int64_t n, bool twice) {
        if (!twice) return (double)((n + 255) / 256);
        return (double)(n / 512) + (n % 512 == 0 ? 0.0 : n % 512 <= 256 ? 0.55 : 1.0);
    };
    const double us[3] = {rounds(tiles[SMALL], !split) * (split ? 4.5 + 0.0103 * depth : 2.0 + 0.0116 * depth),
                          rounds(tiles[MIDDLE], true) * (split ? 6.0 + 0.055 * depth : 7.0 + 0.0226 * depth),
                          rounds(tiles[LARGE], false) * (split ? 37.0 + 0.07 * depth : 40.0 + 0.0245 * depth)};
    const int best = (int)(std::min_element(us, us + 3) - us);
    return {SMALL + best, us[best]};
}
// Of a product of some matrices: symmetric or not, along their longer sides or their shorter ones.
template <class Matrices>
Tile tile_of(const Matrices& all, int count, bool triangle, bool along, bool split) {
    int64_t tiles[4] = {0, 0, 0, 0}, depth = 0;
    for (int m = 0; m < count; ++m) {
        for (int i = 0; i < 4; ++i) {
            const int64_t side = 32 << i, down = (padded(all[m].rows) + side - 1) / side, across = (padded(all[m].cols) + side - 1) / side;
            const int64_t n = std::min(down, across);
            tiles[i] += triangle ? n * (n + 1) / 2 : down * across;
        }
        depth = std::max<int64_t>(depth, along ? std::max(all[m].rows, all[m].cols) : all[m].n());
    }
    return tile_of(tiles, (double)depth, split);
}

// Whether matrices that are wide enough take several steps at once (with operands as exact as fp32 only).  In flops of five steps, units
// of n^3 and m = r n, that is 6 r + 14 instead of 15 r + 5, but 18 launches instead of 15, and apart from the others.  So by what the
// launches take, where that is 15 % less.  MI355X, ms, with steps at once and without: 9 of 768 x 2048 beside 12 of 768 x 768 1.36 and
// 1.46, 3 of 5630 x 2050 2.88 and 4.13, the 0.9B model 71.8 and 87.8 (before sums ended in pairs).
bool wide(const Matrix& m) { return 2 * std::max(m.rows, m.cols) >= 3 * m.n(); }
double estimated(const std::vector<Matrix>& all, int grams, int squares, int applies) {
    auto launch = [&](bool triangle, bool along) { return 2.0 + tile_of(all, (int)all.size(), triangle, along, true).us; };
    return all.empty() ? 0.0 : grams * launch(true, true) + squares * launch(true, false) + applies * launch(false, false);
}

struct Shapes {
    std::vector<Batch> batches;                              // first those whose matrices take several steps at once
    size_t at_once = 0;                                      // so many
    int64_t planes = 0, chunks = 0;                          // elements of the largest batch's planes; chunks of all tensors
};
int64_t ws_bytes(const Shapes& s, int tensors) { return 2 * s.planes + 8 * (s.chunks + tensors) + 128; }

// Batches of like size; the longest products first, so that those that are left at the end of a launch are short ones.
void add_batches(std::vector<Matrix>& all, bool split, int squares, Shapes& s) {
    std::stable_sort(all.begin(), all.end(), [](const Matrix& x, const Matrix& y) { return std::max(x.rows, x.cols) > std::max(y.rows, y.cols); });
    auto size = [&](const Matrix& m) { return split ? Planes<true>::elements(m, squares) : Planes<false>::elements(m, squares); };
    int64_t total = 0, at = 0;
    for (const Matrix& m : all) total += size(m);
    const int64_t each = total / std::max<int64_t>(1, (total + kBatchElements - 1) / kBatchElements);
    for (const Matrix& m : all) {
        if (&m == all.data() || s.batches.back().count == kMostMatrices || at >= each || at + size(m) > kBatchElements) {
            s.batches.push_back(Batch{0, 0, {}});
            at = 0;
        }
        Batch& b = s.batches.back();
        b.of[b.count] = m;
        b.of[b.count++].at = at;
        at += size(m);
        s.planes = std::max(s.planes, at);
    }
}

int shapes(const std::vector<int64_t>& numel, const int64_t* rows, int matmul, Shapes& s) {
    if (!rows || (matmul != SPLC_MATMUL_FP16 && matmul != SPLC_MATMUL_FP16X3)) return SPLC_EINVAL;
    const bool split = matmul == SPLC_MATMUL_FP16X3;
    std::vector<Matrix> all, apart, others;
    for (size_t i = 0; i < numel.size(); ++i) {
        const int64_t n = numel[i];
        if (rows[i] < 0 || (n > 0 && (rows[i] < 1 || n % rows[i] != 0))) return SPLC_EINVAL;
        if (n == 0) continue;
        if (rows[i] > kMostSide || n / rows[i] > kMostSide) return SPLC_EINVAL;
        s.chunks += (n + kChunk - 1) / kChunk;
        const Matrix m{0, (int)rows[i], (int)(n / rows[i]), (int)i, 0};
        all.push_back(m);
        (split && wide(m) ? apart : others).push_back(m);
    }
    if (apart.empty() || 0.85 * estimated(all, 5, 5, 5) <= estimated(apart, 2, 14, 2) + estimated(others, 5, 5, 5)) {
        apart.clear();
        others = std::move(all);
    }
    add_batches(apart, split, kSquaresAtOnce, s);
    s.at_once = s.batches.size();
    add_batches(others, split, kSquares, s);
    return SPLC_OK;
}

// The number of workgroups of a launch, and where each matrix's begin.
template <class Count>
int place(Batch& b, Count count) {
    int64_t total = 0;
    for (int i = 0; i < b.count; ++i) {
        b.of[i].first = (int)total;
        total += count(b.of[i]);
    }
    b.groups = (int)total;
    return b.groups;
}

// One product of every matrix of the batch.
template <bool SPLIT, int STEP>
void product(Batch& b, const Product& f, const Result& result, int odd, const float* grad_scale, _Float16* ws, hipStream_t st) {
    using Large = Shape<2, 4, 1, 2, 64, SPLIT ? 32 : 64, 2, SPLIT>;
    using Middle = Shape<2, 2, 1, 1, 64, SPLIT ? 32 : 64, 2, SPLIT>;
    using Small = Shape<1, 1, 4, 1, 64, 64, 4, SPLIT>;
    using Tiny = Shape<1, 1, 4, 1, 32, 64, 8, SPLIT>;
    auto launch = [&](auto shape) {
        using S = decltype(shape);
        const int groups = place(b, STEP == GRAM || STEP == SQUARE ? S::triangle : S::tiles);
        hipLaunchKernelGGL((product_kernel<S, STEP>), dim3((unsigned)(groups + 7) / 8 * 8), dim3(S::kLanes), 0, st, b, f, result, odd,
                           grad_scale, ws);
    };
    switch (tile_of(b.of, b.count, STEP == GRAM || STEP == SQUARE, STEP == GRAM, SPLIT).size) {
        case LARGE: return launch(Large());
        case MIDDLE: return launch(Middle());
        case SMALL: return launch(Small());
        default: return launch(Tiny());
    }
}

template <bool SPLIT>
void products(Batch& b, const Steps& s, const Result& result, const float* grad_scale, _Float16* ws, hipStream_t st) {
    int odd = 0;
    for (const Product& f : s.of) switch (f.step) {
        case GRAM: product<SPLIT, GRAM>(b, f, result, odd, grad_scale, ws, st); break;
        case SQUARE: product<SPLIT, SQUARE>(b, f, result, odd, grad_scale, ws, st); break;
        case APPLY: product<SPLIT, APPLY>(b, f, result, odd, grad_scale, ws, st); odd ^= 1; break;
        default: product<SPLIT, LAST>(b, f, result, odd, grad_scale, ws, st);
    }
}

template <class From>
int orthogonalised(Shapes& shape, int matmul, const Steps (&steps)[2], const From& from, const float* grad_scale, const double* inverse,
                   const Result& result, _Float16* ws, hipStream_t st) {
    for (size_t i = 0; i < shape.batches.size(); ++i) {
        Batch& b = shape.batches[i];
        const Steps& s = steps[i < shape.at_once];
        const int tiles = place(b, [](const Matrix& m) { return (int64_t)(padded(m.rows) / 64) * (padded(m.cols) / 64); });
        auto launch = [&](auto split) {
            constexpr bool SPLIT = decltype(split)::value;
            hipLaunchKernelGGL((scale_kernel<From, SPLIT>), dim3((unsigned)tiles), dim3(kThreads), 0, st, b, from, grad_scale, inverse, s.first,
                               ws);
            products<SPLIT>(b, s, result, grad_scale, ws, st);
        };
        if (matmul == SPLC_MATMUL_FP16X3) launch(std::true_type());
        else launch(std::false_type());
    }
    return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
}

// The parts of a workspace: planes, sums of the chunks, inverse norms.
struct Space {
    _Float16* planes;
    double *partial, *inverse;
};
Space space(void* ws, const Shapes& s) {
    char* at = static_cast<char*>(ws);
    Space p;
    p.planes = reinterpret_cast<_Float16*>(at);
    p.partial = reinterpret_cast<double*>(at + (2 * s.planes + 127) / 128 * 128);
    p.inverse = p.partial + s.chunks;
    return p;
}

int check_ws(const sparseloco_plan* plan, const int64_t* rows, const double* coefficients, int steps, double eps, int matmul, void* ws,
             int64_t bytes, Shapes& shape, Steps (&s)[2]) {
    const int rc = shapes(plan->numel, rows, matmul, shape);
    if (rc != SPLC_OK) return rc;
    if (!steps_of(coefficients, steps, false, s[0]) || (shape.at_once > 0 && !steps_of(coefficients, steps, true, s[1]))) return SPLC_EINVAL;
    if (!finite64(eps) || eps < 0.0 || !ws || bytes < ws_bytes(shape, plan->n_tensors)) return SPLC_EINVAL;
    return aligned(ws, 128) ? SPLC_OK : SPLC_EALIGN;
}

}  // namespace

extern "C" {

int64_t sparseloco_orthogonalize_ws_bytes(const sparseloco_plan* plan, const int64_t* rows, int matmul) {
    try {
        Shapes s;
        if (!plan) return SPLC_EINVAL;
        const int rc = shapes(plan->numel, rows, matmul, s);
        return rc == SPLC_OK ? ws_bytes(s, plan->n_tensors) : rc;
    } catch (...) {
        return SPLC_ENOMEM;
    }
}

int64_t sparseloco_orthogonalize_choice(int n_matrices, const int64_t* rows, const int64_t* columns, int matmul, int* choice) {
    try {
        if (n_matrices < 0 || (n_matrices > 0 && (!rows || !columns))) return SPLC_EINVAL;
        std::vector<int64_t> numel;
        for (int i = 0; i < n_matrices; ++i) {
            if (rows[i] < 1 || rows[i] > kMostSide || columns[i] < 1 || columns[i] > kMostSide) return SPLC_EINVAL;
            numel.push_back(rows[i] * columns[i]);
        }
        Shapes s;
        const int rc = n_matrices > 0 ? shapes(numel, rows, matmul, s) : SPLC_OK;
        if (rc != SPLC_OK) return rc;
        for (size_t i = 0; choice && i < s.batches.size(); ++i) {
            const Batch& b = s.batches[i];
            const bool split = matmul == SPLC_MATMUL_FP16X3;
            const auto side = [&](bool triangle, bool along) { return 32 << tile_of(b.of, b.count, triangle, along, split).size; };
            for (int m = 0; m < b.count; ++m) {
                int* of = choice + 5 * (int64_t)b.of[m].tensor;
                of[0] = i < s.at_once;
                of[1] = (int)i;
                of[2] = side(true, true);
                of[3] = side(true, false);
                of[4] = side(false, false);
            }
        }
        return ws_bytes(s, n_matrices);
    } catch (...) {
        return SPLC_ENOMEM;
    }
}

int sparseloco_orthogonalize(const sparseloco_plan* plan, const int64_t* rows, const sparseloco_tensors* x, const sparseloco_tensors* out,
                             int replica, const double* coefficients, int steps, double eps, int matmul, void* ws, int64_t bytes,
                             void* stream) {
    try {
        if (!plan || !x || !out || replica < 0) return SPLC_EINVAL;
        Shapes shape;
        Steps s[2];
        int rc = check_ws(plan, rows, coefficients, steps, eps, matmul, ws, bytes, shape, s);
        if (rc != SPLC_OK) return rc;
        for (const sparseloco_tensors* t : {x, out}) {
            if ((rc = check_tensors(plan, t, t->dtype, 1)) != SPLC_OK) return rc;
            if (t->n_sets > 1 && replica >= t->n_sets) return SPLC_EINVAL;
        }
        if ((rc = current_device_is(plan->device)) != SPLC_OK) return rc;
        if (shape.chunks == 0) return SPLC_OK;
        const Space p = space(ws, shape);
        hipStream_t st = static_cast<hipStream_t>(stream);
        const Result result{out->dtype, set_table<void*>(out, replica), nullptr, nullptr, 0.f, 0.f, 0};
        auto run = [&](auto type) {
            using T = decltype(type);
            const T* const* from = set_table<const T*>(x, replica);
            hipLaunchKernelGGL(squares_kernel<T>, dim3((unsigned)plan->n_update), dim3(kThreads), 0, st, plan->d_update, from, p.partial);
            hipLaunchKernelGGL(inverse_norm_kernel, dim3((unsigned)plan->n_tensors), dim3(kThreads), 0, st, plan->d_numel, p.partial, eps,
                               p.inverse);
            return orthogonalised(shape, matmul, s, Plain<T>{from}, nullptr, p.inverse, result, p.planes, st);
        };
        return x->dtype == SPLC_BF16 ? run(uint16_t()) : run(float());
    } catch (...) {
        return SPLC_ENOMEM;
    }
}

int sparseloco_muon_step(const sparseloco_plan* plan, const int64_t* rows, const sparseloco_tensors* theta, const sparseloco_tensors* grads,
                         const sparseloco_tensors* m, int replica, const sparseloco_muon* how, const float* grad_scale,
                         const float* decay, const sparseloco_tensors* theta_bf16, void* ws, int64_t bytes, void* stream) {
    try {
        if (!plan || !theta || !grads || !m || !how || replica < 0) return SPLC_EINVAL;
        for (double v : {how->lr, how->weight_decay})
            if (!finite64(v) || v < 0.0 || !finite((float)v)) return SPLC_EINVAL;
        if (!(how->momentum >= 0.0 && how->momentum < 1.0) || !finite((float)(how->lr * how->weight_decay))) return SPLC_EINVAL;
        if (how->adjust != SPLC_MUON_NONE && how->adjust != SPLC_MUON_ASPECT && how->adjust != SPLC_MUON_RMS) return SPLC_EINVAL;
        Shapes shape;
        Steps s[2];
        int rc = check_ws(plan, rows, how->coefficients, how->steps, how->eps, how->matmul, ws, bytes, shape, s);
        if (rc != SPLC_OK) return rc;
        for (const sparseloco_tensors* t : {theta, m, grads, theta_bf16}) {
            if (!t) continue;
            const int dtype = t == grads ? grads->dtype : t == theta_bf16 ? (int)SPLC_BF16 : (int)SPLC_F32;
            if ((rc = check_tensors(plan, t, dtype, 1)) != SPLC_OK) return rc;
            if (t->n_sets > 1 && replica >= t->n_sets) return SPLC_EINVAL;
        }
        if (!aligned(grad_scale, 4) || !aligned(decay, 4)) return SPLC_EALIGN;
        if ((rc = current_device_is(plan->device)) != SPLC_OK) return rc;
        if (shape.chunks == 0) return SPLC_OK;
        const Space p = space(ws, shape);
        hipStream_t st = static_cast<hipStream_t>(stream);
        const Result result{-1, set_table<void*>(theta, replica), theta_bf16 ? set_table<uint16_t*>(theta_bf16, replica) : nullptr, decay,
                            (float)how->lr, (float)(how->lr * how->weight_decay), how->adjust};
        auto run = [&](auto type) {
            using G = decltype(type);
            const Update<G> update{set_table<const G*>(grads, replica), set_table<float*>(m, replica),
                                   {(float)how->momentum, (float)(1.0 - how->momentum), how->nesterov != 0}};
            hipLaunchKernelGGL(momentum_kernel<G>, dim3((unsigned)plan->n_update), dim3(kThreads), 0, st, plan->d_update, update, grad_scale,
                               p.partial);
            hipLaunchKernelGGL(inverse_norm_kernel, dim3((unsigned)plan->n_tensors), dim3(kThreads), 0, st, plan->d_numel, p.partial,
                               how->eps, p.inverse);
            return orthogonalised(shape, how->matmul, s, update, grad_scale, p.inverse, result, p.planes, st);
        };
        return grads->dtype == SPLC_BF16 ? run(uint16_t()) : run(float());
    } catch (...) {
        return SPLC_ENOMEM;
    }
}

}  // extern "C"
