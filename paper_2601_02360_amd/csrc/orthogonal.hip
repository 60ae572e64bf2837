// Orthogonalised updates for gfx950 (MI355X): matrices of a plan brought near to the orthogonal factor of their polar
// decomposition by Newton-Schulz products, and the optimiser step that takes such updates.
//
// A matrix M, turned so that its n rows are no more than its m columns, is scaled to X = M / (|M| + eps) and iterated:
//     A = X X^T,   B = b A + c A^2,   X <- a X + B X,
// which maps every singular value s of X to a s + b s^3 + c s^5.  All three products have the form C[i][j] = sum_k P[i][k] Q[j][k]
// with both operands' rows contiguous, for which X is kept in two layouts, as it lies in memory (R) and transposed (T), and A and B
// need none but their own.  A and A^2 are symmetric: tiles on and above the diagonal are formed, and stored twice.
//
// Operands are fp16 numbers times a power of two that the host knows beforehand: |X| <= 1 in the spectral norm, and the polynomial
// says what that bound becomes, so that no element leaves [-2^14, 2^14] and those 2^-28 of the bound keep 11 bits.
//   FP16    one product a term.  A, B and X are rounded to 11 bits as operands; X itself is held in 22 (hi + lo) where a X is
//           added.  Result: 2e-4 to 2e-3 off (relative, depending on how the singular values are spread), as little as a result in
//           bf16 is rounded by; bf16 operands are 1e-2 to 4e-2 off.
//   FP16X3  operands are hi + lo, 22 bits, and a product is hi hi + hi lo + lo hi: what fp32 products give.
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
constexpr int kMostMatrices = 48;                            // of a batch: their descriptions are kernel arguments
constexpr int64_t kBatchElements = (int64_t)1 << 27;         // a batch takes matrices until it has so many
constexpr int kMostSide = 1 << 22;                           // rows and columns: offsets inside a tile's rows stay in 32 bits
constexpr int kMostSteps = SPLC_MAX_ORTHO_STEPS;

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

__host__ __device__ inline int padded(int n) { return (n + kPad - 1) / kPad * kPad; }

struct Matrix {
    int64_t at;                                              // of its planes in the workspace, in elements
    int rows, cols, tensor, first;                           // first: of its workgroups in a launch
    __host__ __device__ int n() const { return rows < cols ? rows : cols; }
    __host__ __device__ bool tall() const { return rows > cols; }
    __host__ __device__ int64_t r_plane() const { return (int64_t)rows * padded(cols); }
    __host__ __device__ int64_t t_plane() const { return (int64_t)cols * padded(rows); }
    __host__ __device__ int64_t a_plane() const { return (int64_t)n() * padded(n()); }
};
struct Batch {
    int count;
    Matrix of[kMostMatrices];
};
// Planes of a matrix: R of this step and of the next (hi, lo), T likewise (hi, and lo if SPLIT), A and B.
template <bool SPLIT>
struct Planes {
    static constexpr int kParts = SPLIT ? 2 : 1;
    _Float16 *r_first, *t_first, *a, *b;                     // lo follows hi
    int64_t r_next, t_next;
    __host__ __device__ static int64_t elements(const Matrix& m) {
        return 4 * m.r_plane() + 2 * kParts * m.t_plane() + 2 * kParts * m.a_plane();
    }
    __device__ __forceinline__ Planes(_Float16* ws, const Matrix& m) {
        _Float16* p = ws + m.at;
        r_first = p;
        r_next = 2 * m.r_plane();
        t_first = p += 2 * r_next;
        t_next = kParts * m.t_plane();
        a = p += 2 * t_next;
        b = p + kParts * m.a_plane();
    }
    __device__ __forceinline__ _Float16* r(int odd) const { return r_first + odd * r_next; }
    __device__ __forceinline__ _Float16* t(int odd) const { return t_first + odd * t_next; }
};

// The matrix of a workgroup, and the workgroup's place in it.
__device__ __forceinline__ const Matrix& matrix_of(const Batch& batch, uint32_t group, int& place) {
    int i = 0;
    while (i + 1 < batch.count && (uint32_t)batch.of[i + 1].first <= group) ++i;
    place = (int)group - batch.of[i].first;
    return batch.of[i];
}

__device__ __forceinline__ void split(float x, _Float16& hi, _Float16& lo) {
    hi = (_Float16)x;
    lo = (_Float16)(x - (float)hi);
}

// ---------------------------------------------------------------- what is orthogonalised

struct Momentum {
    float beta, rest;
    int nesterov;
};
// The matrix's elements as the orthogonalisation takes them: those of a tensor, or the step's update from momentum and gradient.
template <class T>
struct Plain {
    const T* const* x;
    __device__ __forceinline__ float operator()(int tensor, int64_t at, float) const { return widened(x[tensor][at]); }
};
template <class G>
struct Update {
    const G* const* grad;
    float* const* m;                                         // the new momentum
    Momentum how;
    __device__ __forceinline__ float operator()(int tensor, int64_t at, float factor) const {
        const float moment = m[tensor][at];
        return how.nesterov ? fmaf(how.beta, moment, how.rest * (factor * widened(grad[tensor][at]))) : moment;
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

// m = beta m + (1 - beta) g, and the sum of squares of a chunk of the update.
template <class G>
__global__ __launch_bounds__(kThreads) void momentum_kernel(const ChunkDesc* __restrict__ chunks, Update<G> update,
                                                            const float* __restrict__ grad_scale, double* __restrict__ partial) {
    __shared__ double shared[kThreads / 64];
    const ChunkDesc d = chunks[blockIdx.x];
    float factor;
    if (!gradient_factor(grad_scale, factor)) return;
    float* m = update.m[d.tensor];
    const G* grad = update.grad[d.tensor];
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < d.n_c; i += kThreads) {
        const int64_t at = (int64_t)d.offset + i;
        const float g = factor * widened(grad[at]);
        const float moment = fmaf(update.how.rest, g, update.how.beta * m[at]);
        m[at] = moment;
        const double u = update.how.nesterov ? fmaf(update.how.beta, moment, update.how.rest * g) : moment;
        sum = fma(u, u, sum);
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
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < d.n_c; i += kThreads) sum = fma((double)widened(p[i]), (double)widened(p[i]), sum);
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
__global__ __launch_bounds__(kThreads) void scale_kernel(Batch batch, From from, const float* __restrict__ grad_scale,
                                                         const double* __restrict__ inverse, float range, _Float16* __restrict__ ws) {
    __shared__ float tile[64][65];
    float factor;
    if (!gradient_factor(grad_scale, factor)) return;
    int place;
    const Matrix& m = matrix_of(batch, blockIdx.x, place);
    const Planes<SPLIT> planes(ws, m);
    const int across = padded(m.cols) / 64, r0 = place / across * 64, c0 = place % across * 64;
    const int ldc = padded(m.cols), ldr = padded(m.rows), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const double scale = inverse[m.tensor] * (double)range;
    for (int i = wave; i < 64; i += kThreads / 64) {
        const int r = r0 + i, c = c0 + lane;
        const float x = r < m.rows && c < m.cols ? (float)((double)from(m.tensor, (int64_t)r * m.cols + c, factor) * scale) : 0.f;
        tile[i][lane] = x;
        if (r < m.rows) {
            _Float16* p = planes.r(0) + (int64_t)r * ldc + c;
            split(x, p[0], p[m.r_plane()]);
        }
    }
    __syncthreads();
    for (int i = wave; i < 64; i += kThreads / 64) {
        const int c = c0 + i, r = r0 + lane;
        if (c >= m.cols) break;
        _Float16 hi, lo;
        split(tile[lane][i], hi, lo);
        _Float16* p = planes.t(0) + (int64_t)c * ldr + r;
        p[0] = hi;
        if (SPLIT) p[m.t_plane()] = lo;
    }
}

// ---------------------------------------------------------------- products

enum { GRAM = 0, POLYNOMIAL = 1, APPLY = 2, LAST = 3 };

// The factors of one product: its result is old * own + sum * product, in the result's range.
struct Factors {
    float own, product;
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

// A tile of T x T elements of C = P Q^T, kept in the registers of W x W waves; BK elements of every row of P and Q at a time go
// to LDS, without passing registers, while the BK before them are multiplied.  A row of BK fp16 numbers is BK / 8 pieces of 16
// bytes; the pieces of a row are exchanged by its number, so that 8 lanes that read a piece of 8 rows find them in 8 different
// places of the 128 bytes that LDS gives a cycle.
template <int T, int W, int BK, bool SPLIT, int STEP>
__global__ __launch_bounds__(W* W * 64) void product_kernel(Batch batch, Factors f, Result result, int odd,
                                                           const float* __restrict__ grad_scale, _Float16* __restrict__ ws) {
    constexpr int kParts = SPLIT ? 2 : 1, kWaves = W * W, kSide = T / W / 32, kPieces = BK / 8, kRowsALoad = 64 / kPieces;
    constexpr int kLoads = T * BK * 2 / 1024 / kWaves;       // of a wave for one plane of one operand
    constexpr int kPlane = T * BK;
    static_assert(kLoads * kWaves * 1024 == T * BK * 2, "whole loads");
    __shared__ __align__(1024) _Float16 lds[2][2 * kParts][kPlane];

    float factor;
    if (!gradient_factor(grad_scale, factor)) return;
    int place;
    const Matrix m = matrix_of(batch, blockIdx.x, place);
    const Planes<SPLIT> planes(ws, m);
    const int n = m.n(), ldn = padded(n), ldc = padded(m.cols), ldr = padded(m.rows);
    int ti, tj;
    if (STEP == GRAM || STEP == POLYNOMIAL) {                // column by column of the upper triangle
        tj = (int)((sqrtf(8.f * (float)place + 1.f) - 1.f) * 0.5f);
        while (tj * (tj + 1) / 2 > place) --tj;
        while ((tj + 1) * (tj + 2) / 2 <= place) ++tj;
        ti = place - tj * (tj + 1) / 2;
    } else {
        const int down = (m.rows + T - 1) / T;
        ti = place % down;
        tj = place / down;
    }
    const _Float16 *p, *q;
    int64_t p_lo = 0, q_lo = 0;                              // from hi to lo
    int p_rows, q_rows, depth;
    if (STEP == GRAM) {
        p = q = m.tall() ? planes.t(odd) : planes.r(odd);
        p_lo = q_lo = m.tall() ? m.t_plane() : m.r_plane();
        p_rows = q_rows = n;
        depth = m.tall() ? ldr : ldc;
    } else if (STEP == POLYNOMIAL) {
        p = q = planes.a;
        p_lo = q_lo = m.a_plane();
        p_rows = q_rows = n;
        depth = ldn;
    } else {
        p = m.tall() ? planes.r(odd) : planes.b;
        q = m.tall() ? planes.b : planes.t(odd);
        p_lo = m.tall() ? m.r_plane() : m.a_plane();
        q_lo = m.tall() ? m.a_plane() : m.t_plane();
        p_rows = m.rows;
        q_rows = m.cols;
        depth = ldn;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = ti * T, col0 = tj * T;
    const _Float16* from[2] = {p + (int64_t)row0 * depth, q + (int64_t)col0 * depth};
    const int64_t to_lo[2] = {p_lo, q_lo};
    uint32_t offset[2][kLoads];                              // of this lane's 16 bytes from the tile's first element, in elements
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int row = (wave + i * kWaves) * kRowsALoad + lane / kPieces;
        const int piece = (lane % kPieces) ^ (BK == 64 ? row & 7 : (row >> 1) & 3);
        const int in_p = row0 + row < p_rows ? row : p_rows - 1 - row0, in_q = col0 + row < q_rows ? row : q_rows - 1 - col0;
        offset[0][i] = (uint32_t)in_p * (uint32_t)depth + (uint32_t)piece * 8u;
        offset[1][i] = (uint32_t)in_q * (uint32_t)depth + (uint32_t)piece * 8u;
    }
    auto fetch = [&](int k, int buffer) {
#pragma unroll
        for (int side = 0; side < 2; ++side) {
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
                const _Float16* base = from[side] + (part ? to_lo[side] : 0) + k;
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
                    __builtin_amdgcn_global_load_lds((global_void*)(base + offset[side][i]),
                                                     (shared_void*)&lds[buffer][side * kParts + part][(wave + i * kWaves) * 512], 16, 0, 0);
            }
        }
    };
    v16f sum[kSide][kSide];
#pragma unroll
    for (int i = 0; i < kSide; ++i) {
#pragma unroll
        for (int j = 0; j < kSide; ++j) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[i][j][e] = 0.f;
        }
    }
    const int wave_row = wave / W * (T / W), wave_col = wave % W * (T / W);
    const int swap = BK == 64 ? lane & 7 : (lane >> 1) & 3;
    fetch(0, 0);
    for (int k = 0, buffer = 0; k < depth; k += BK, buffer ^= 1) {
        __syncthreads();                                     // what was fetched is there, and the other buffer has been read
        if (k + BK < depth) fetch(k + BK, buffer ^ 1);
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk) {
            const int piece = ((kk * 2 + (lane >> 5)) ^ swap) * 8;
            half8 x[kSide][kParts], y[kSide][kParts];
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
#pragma unroll
                for (int i = 0; i < kSide; ++i) {
                    x[i][part] = *(const half8*)&lds[buffer][part][(wave_row + i * 32 + (lane & 31)) * BK + piece];
                    y[i][part] = *(const half8*)&lds[buffer][kParts + part][(wave_col + i * 32 + (lane & 31)) * BK + piece];
                }
            }
#pragma unroll
            for (int term = SPLIT ? 2 : 0; term >= 0; --term) {
#pragma unroll
                for (int i = 0; i < kSide; ++i) {
#pragma unroll
                    for (int j = 0; j < kSide; ++j)          // columns of C in a lane's registers, rows over the lanes
                        sum[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(y[j][term == 1], x[i][term == 2], sum[i][j], 0, 0, 0);
                }
            }
        }
    }
    // Register e of lane l: row l % 32, column 8 (e / 4) + 4 (l / 32) + e % 4.
    const float keep = STEP == LAST && result.to < 0 ? 1.f - (result.decay ? result.shrink * result.decay[m.tensor] : result.shrink) : 0.f;
    float size = 0.f;
    if (STEP == LAST && result.to < 0) {
        const float rows = (float)m.rows, cols = (float)m.cols;
        size = result.size * (result.adjust == SPLC_MUON_ASPECT ? sqrtf(fmaxf(1.f, rows / cols))
                              : result.adjust == SPLC_MUON_RMS  ? 0.2f * sqrtf(fmaxf(rows, cols))
                                                                : 1.f);
    }
#pragma unroll
    for (int i = 0; i < kSide; ++i) {
        const int row = row0 + wave_row + i * 32 + (lane & 31);
#pragma unroll
        for (int j = 0; j < kSide; ++j) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = col0 + wave_col + j * 32 + g * 8 + (lane >> 5) * 4;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = f.product * sum[i][j][g * 4 + e];
                if (STEP == GRAM || STEP == POLYNOMIAL) {
                    _Float16* to = STEP == GRAM ? planes.a : planes.b;
                    if (row < n && col < ldn) {
                        const int64_t at = (int64_t)row * ldn + col;
                        if (STEP == POLYNOMIAL) {
                            const half4 hi = *(const half4*)(planes.a + at);
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = fmaf(f.own, (float)hi[e], v[e]);
                            if (SPLIT) {
                                const half4 lo = *(const half4*)(planes.a + m.a_plane() + at);
#pragma unroll
                                for (int e = 0; e < 4; ++e) v[e] = fmaf(f.own, (float)lo[e], v[e]);
                            }
                        }
                        half4 hi, lo;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            _Float16 h, l;
                            split(col + e < n ? v[e] : 0.f, h, l);
                            hi[e] = h;
                            lo[e] = l;
                        }
                        *(half4*)(to + at) = hi;
                        if (SPLIT) *(half4*)(to + m.a_plane() + at) = lo;
                        if (ti != tj) {                      // (row < n: this tile lies above the diagonal, all of its rows exist)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if (col + e >= n) break;
                                _Float16* mirrored = to + (int64_t)(col + e) * ldn + row;
                                mirrored[0] = hi[e];
                                if (SPLIT) mirrored[m.a_plane()] = lo[e];
                            }
                        }
                    }
                } else {
                    const bool there = row < m.rows && col < ldc;
                    if (there) {
                        const int64_t at = (int64_t)row * ldc + col;
                        const half4 hi = *(const half4*)(planes.r(odd) + at), lo = *(const half4*)(planes.r(odd) + m.r_plane() + at);
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = fmaf(f.own, (float)hi[e] + (float)lo[e], v[e]);
                    }
                    if (STEP == APPLY) {
                        half4 hi, lo;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            _Float16 h, l;
                            split(there && col + e < m.cols ? v[e] : 0.f, h, l);
                            hi[e] = h;
                            lo[e] = l;
                        }
                        if (there) {
                            _Float16* to = planes.r(odd ^ 1) + (int64_t)row * ldc + col;
                            *(half4*)to = hi;
                            *(half4*)(to + m.r_plane()) = lo;
                        }
                        if (row < ldr) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if (col + e >= m.cols) break;
                                _Float16* to = planes.t(odd ^ 1) + (int64_t)(col + e) * ldr + row;
                                to[0] = hi[e];
                                if (SPLIT) to[m.t_plane()] = lo[e];
                            }
                        }
                    } else if (there) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (col + e >= m.cols) break;
                            const int64_t at = (int64_t)row * m.cols + col + e;
                            if (result.to < 0) {
                                float* theta = static_cast<float*>(result.out[m.tensor]) + at;
                                const float now = fmaf(-size, v[e], *theta * keep);
                                *theta = now;
                                if (result.copy) result.copy[m.tensor][at] = (uint16_t)bf16_pair(now, 0.f);
                            } else if (result.to == SPLC_BF16) {
                                static_cast<uint16_t*>(result.out[m.tensor])[at] = (uint16_t)bf16_pair(v[e], 0.f);
                            } else {
                                static_cast<float*>(result.out[m.tensor])[at] = v[e];
                            }
                        }
                    }
                }
            }
        }
    }
}

// ---------------------------------------------------------------- host

bool finite64(double v) { return std::isfinite(v); }

// Largest |p| for x in [0, most], p odd or plain of the form x^k (a + b x^2 + c x^4) sampled where its derivative vanishes.
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

// The powers of two that A, B and X are held times, and the factors of the three products of every step.
struct Steps {
    int count = 0;
    float first = 0.f;                                       // of X before the first step
    Factors gram[kMostSteps], polynomial[kMostSteps], apply[kMostSteps];
};
bool ranges(const double* coefficients, int steps, Steps& s) {
    static const double usual[] = {3.4445, -4.7750, 2.0315};
    if (steps < 1 || steps > kMostSteps) return false;
    auto range = [](double bound) { return 14 - (int)std::ceil(std::log2(std::max(bound, 1e-3))); };
    double most = 1.0;                                       // bound on the singular values of X
    int x = range(most);
    s.count = steps;
    s.first = (float)std::ldexp(1.0, x);
    for (int k = 0; k < steps; ++k) {
        const double* p = coefficients ? coefficients + 3 * k : usual;
        for (int i = 0; i < 3; ++i)
            if (!finite64(p[i]) || std::fabs(p[i]) > 1e4) return false;
        const int a = range(most * most), b = range(largest_even(p[1], p[2], most * most));
        const bool last = k + 1 == steps;
        most = largest(p[0], p[1], p[2], most);
        if (!finite64(most) || most > 1024.0) return false;
        const int next = last ? 0 : range(most);
        s.gram[k] = {0.f, (float)std::ldexp(1.0, a - 2 * x)};
        s.polynomial[k] = {(float)std::ldexp(p[1], b - a), (float)std::ldexp(p[2], b - 2 * a)};
        s.apply[k] = {(float)std::ldexp(p[0], next - x), (float)std::ldexp(1.0, next - b - x)};
        x = next;
    }
    return true;
}

struct Shapes {
    std::vector<Batch> batches;
    int64_t planes = 0, chunks = 0;                          // elements of the largest batch's planes; chunks of all tensors
};
int64_t ws_bytes(const Shapes& s, int tensors) { return 2 * s.planes + 8 * (s.chunks + tensors) + 128; }

int shapes(const sparseloco_plan* plan, const int64_t* rows, int matmul, Shapes& s) {
    if (!plan || !rows || (matmul != SPLC_MATMUL_FP16 && matmul != SPLC_MATMUL_FP16X3)) return SPLC_EINVAL;
    const bool three = matmul == SPLC_MATMUL_FP16X3;
    s.chunks = plan->n_update;
    int64_t elements = 0, at = 0;
    for (int i = 0; i < plan->n_tensors; ++i) {
        const int64_t n = plan->numel[(size_t)i];
        if (rows[i] < 0 || (n > 0 && (rows[i] < 1 || n % rows[i] != 0))) return SPLC_EINVAL;
        if (n == 0) continue;
        if (rows[i] > kMostSide || n / rows[i] > kMostSide) return SPLC_EINVAL;
        const Matrix m{0, (int)rows[i], (int)(n / rows[i]), i, 0};
        if (s.batches.empty() || s.batches.back().count == kMostMatrices || elements >= kBatchElements) {
            s.batches.push_back(Batch{0, {}});
            elements = at = 0;
        }
        Batch& b = s.batches.back();
        b.of[b.count] = m;
        b.of[b.count++].at = at;
        at += three ? Planes<true>::elements(m) : Planes<false>::elements(m);
        elements += n;
        s.planes = std::max(s.planes, at);
    }
    return SPLC_OK;
}

// The number of workgroups of a launch, and where each matrix's begin.
template <class Count>
uint32_t place(Batch& b, Count count) {
    int64_t total = 0;
    for (int i = 0; i < b.count; ++i) {
        b.of[i].first = (int)total;
        total += count(b.of[i]);
    }
    return (uint32_t)total;
}

template <int T, int W, int BK, bool SPLIT>
void products(Batch& b, const Steps& s, const Result& result, const float* grad_scale, _Float16* ws, hipStream_t st) {
    constexpr int kLanes = W * W * 64;
    auto half = [](const Matrix& m) { const int64_t t = (m.n() + T - 1) / T; return t * (t + 1) / 2; };
    auto all = [](const Matrix& m) { return (int64_t)((m.rows + T - 1) / T) * ((m.cols + T - 1) / T); };
    for (int k = 0; k < s.count; ++k) {
        const int odd = k & 1;
        const uint32_t sides = place(b, half);
        hipLaunchKernelGGL((product_kernel<T, W, BK, SPLIT, GRAM>), dim3(sides), dim3(kLanes), 0, st, b, s.gram[k], result, odd, grad_scale,
                           ws);
        hipLaunchKernelGGL((product_kernel<T, W, BK, SPLIT, POLYNOMIAL>), dim3(sides), dim3(kLanes), 0, st, b, s.polynomial[k], result, odd,
                           grad_scale, ws);
        const uint32_t tiles = place(b, all);
        if (k + 1 < s.count)
            hipLaunchKernelGGL((product_kernel<T, W, BK, SPLIT, APPLY>), dim3(tiles), dim3(kLanes), 0, st, b, s.apply[k], result, odd,
                               grad_scale, ws);
        else
            hipLaunchKernelGGL((product_kernel<T, W, BK, SPLIT, LAST>), dim3(tiles), dim3(kLanes), 0, st, b, s.apply[k], result, odd,
                               grad_scale, ws);
    }
}

template <class From>
int orthogonalised(Shapes& shape, int matmul, const Steps& steps, const From& from, const float* grad_scale, const double* inverse,
                   const Result& result, _Float16* ws, hipStream_t st) {
    for (Batch& b : shape.batches) {
        const uint32_t tiles = place(b, [](const Matrix& m) { return (int64_t)(padded(m.rows) / 64) * (padded(m.cols) / 64); });
        if (matmul == SPLC_MATMUL_FP16X3) {
            hipLaunchKernelGGL((scale_kernel<From, true>), dim3(tiles), dim3(kThreads), 0, st, b, from, grad_scale, inverse, steps.first, ws);
            products<128, 2, 32, true>(b, steps, result, grad_scale, ws, st);
        } else {
            hipLaunchKernelGGL((scale_kernel<From, false>), dim3(tiles), dim3(kThreads), 0, st, b, from, grad_scale, inverse, steps.first, ws);
            products<128, 2, 64, false>(b, steps, result, grad_scale, ws, st);
        }
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
             int64_t bytes, Shapes& shape, Steps& s) {
    const int rc = shapes(plan, rows, matmul, shape);
    if (rc != SPLC_OK) return rc;
    if (!ranges(coefficients, steps, s) || !finite64(eps) || eps < 0.0 || !ws || bytes < ws_bytes(shape, plan->n_tensors)) return SPLC_EINVAL;
    return aligned(ws, 128) ? SPLC_OK : SPLC_EALIGN;
}

}  // namespace

extern "C" {

int64_t sparseloco_orthogonalize_ws_bytes(const sparseloco_plan* plan, const int64_t* rows, int matmul) {
    try {
        Shapes s;
        const int rc = shapes(plan, rows, matmul, s);
        return rc == SPLC_OK ? ws_bytes(s, plan->n_tensors) : rc;
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
        Steps s;
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
        Steps s;
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
