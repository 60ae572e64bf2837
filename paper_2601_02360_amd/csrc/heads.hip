// Queries and keys of a replica's attention for gfx950 (MI355X): rotated by their positions, and normed for each head in the
// same pass, with the gradient of that.
//
// A head of `d` channels is d / 2 pairs: pair i turns by position * frequencies[i] for i < r, and not at all behind.  A lane
// holds V pairs of a head, L = 2^n lanes a head, 64 / L heads a wave at once; a wave takes a token (or, where there are few,
// a share of its heads) and keeps the cosines and sines of its pairs for all of the token's heads.  Angles are formed as turns,
// position * (frequency / 2 pi), of which only the fraction is kept: fp32 would be off by 2^-24 of the whole angle, 1e-2 at position
// 131072, and fp64 by 2^-52 of it, 2^-22 at 2^30 radians; so the quotient and the product are two doubles each, and positions of 64
// bits too.  Everything else is fp32, rounded once to the tensors' type.
//
// What bounds it (MI355X): memory, or the launch.  bf16, heads of 128 channels: 32768 x 40 heads rotated 125 us or 5.4 TB/s, 16384 x 32
// normed and rotated 55 us or 4.9, their gradient 85 us or 4.7, 5 of them the join; one token of 40 heads 4 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>

#include "plan.h"
#include "sparseloco.h"

namespace {

using namespace splc;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMostDim = SPLC_MAX_HEAD_DIM;
constexpr uint32_t kFillingWaves = 4096;                     // four a SIMD: where a token's heads are no longer shared out
constexpr uint32_t kMostGroups = 1u << 20;                   // workgroups of a launch: those lanes are counted in 32 bits
constexpr uint32_t kGradGroups = 1024;
constexpr int kJoinThreads = 1024, kJoinRows = 16;         // lanes of a row of workgroups' sums: 16 channels

template <class T>
struct View {
    T* at;
    int64_t token, head;                                     // strides in elements
    int heads;
};
struct Rotation {
    const void* positions;
    const double* frequencies;
    int wide;                                                // positions in 64 bits
    int r;                                                   // pairs that turn
    float magnitude, sign;
};

template <class T, int V>
struct Vector {
    typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <class T>
struct Vector<T, 1> {
    typedef T type;
};

__device__ __forceinline__ float wide_of(float v) { return v; }
__device__ __forceinline__ float wide_of(uint16_t v) { return widened(v); }

template <class T, int V>
__device__ __forceinline__ void widen(typename Vector<T, V>::type v, float* x) {
    if constexpr (V == 1) {
        x[0] = wide_of(v);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = wide_of(v[j]);
    }
}
template <int V>
__device__ __forceinline__ void store_narrow(float* p, const float* x) {
    typename Vector<float, V>::type v;
    if constexpr (V == 1) {
        v = x[0];
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = x[j];
    }
    __builtin_nontemporal_store(v, (SPLC_GLOBAL typename Vector<float, V>::type*)p);
}
template <int V>
__device__ __forceinline__ void store_narrow(uint16_t* p, const float* x) {
    if constexpr (V == 1) {
        *(SPLC_GLOBAL uint16_t*)p = (uint16_t)bf16_pair(x[0], 0.f);
    } else {
        typedef uint32_t words __attribute__((ext_vector_type(V / 2)));
        words w;
        if constexpr (V == 2) {
            w = bf16_pair(x[0], x[1]);
        } else {
#pragma unroll
            for (int j = 0; j < V / 2; ++j) w[j] = bf16_pair(x[2 * j], x[2 * j + 1]);
        }
        __builtin_nontemporal_store(__builtin_bit_cast(typename Vector<uint16_t, V>::type, w), (SPLC_GLOBAL typename Vector<uint16_t, V>::type*)p);
    }
}

// Pairs of a head as a lane holds them: C runs of V, in two vectors of V channels each that neighbouring lanes continue.  Where the
// halves lie apart, the vectors hold the first and the second coordinates; where pairs lie side by side, one vector lies in each half
// of the head (or is one of two coordinates, V = 1).
template <class T, int V, bool SIDE>
struct Lanes {
    static constexpr int C = V == 1 ? 4 : V == 2 ? 2 : 1;    // 64 lanes x C x V pairs: 512 channels at the least
    int first[C], second[C];                                 // where the run's first and second V channels begin
    bool there[C];

    __device__ __forceinline__ Lanes(int lane, int per_head, int d, int r) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int p = (lane + c * per_head) * V;
            there[c] = p < d / 2;
            if (SIDE) {
                first[c] = V == 1 ? 2 * p : p;
                second[c] = V == 1 ? 2 * p + 1 : p + d / 2;
            } else if (p < r) {
                first[c] = p;
                second[c] = p + r;
            } else {                                         // behind the rotated channels, halved likewise
                first[c] = p + r;
                second[c] = p + d / 2;
            }
        }
    }
    // A head's channels as they are in memory.
    struct Raw {
        typename Vector<T, V>::type a[C], b[C];
    };
    __device__ __forceinline__ void load(const T* head, Raw& raw) const {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (!there[c]) continue;
            raw.a[c] = *(const SPLC_GLOBAL typename Vector<T, V>::type*)(head + first[c]);
            raw.b[c] = *(const SPLC_GLOBAL typename Vector<T, V>::type*)(head + second[c]);
        }
    }
    __device__ __forceinline__ void take(const Raw& raw, float (&x)[C][2 * V]) const {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (there[c]) {
                widen<T, V>(raw.a[c], x[c]);
                widen<T, V>(raw.b[c], x[c] + V);
            } else {
#pragma unroll
                for (int j = 0; j < 2 * V; ++j) x[c][j] = 0.f;
            }
        }
    }
    __device__ __forceinline__ void store(T* head, const float (&x)[C][2 * V]) const {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (there[c]) {
                store_narrow<V>(head + first[c], x[c]);
                store_narrow<V>(head + second[c], x[c] + V);
            }
        }
    }
};

// x s, or x (-s).  COPIES: +0 where s is a zero, whatever x is; subtracted, that changes nothing, so that channels behind the pairs that
// turn, whose sine is 0 and cosine 1, are copied also beside infinities and NaN, and zeros keep their sign.  (Where heads are normed,
// nothing is copied, and one element that is not finite makes its head NaN; there the compiler's own product costs fewer registers:
// 16384 x 32 heads of 128 bf16 channels 55 us for 63.)
template <bool COPIES, bool NEGATIVE>
__device__ __forceinline__ float by_sine(float x, float s) {
    float product;
    if (!COPIES) return NEGATIVE ? x * -s : x * s;
    if (NEGATIVE) asm("v_mul_legacy_f32 %0, %1, -%2" : "=v"(product) : "v"(x), "v"(s));
    else asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(product) : "v"(x), "v"(s));
    return product;
}

constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591243e-18;    // 1 / (2 pi)

template <int V, int C>
struct Turn {
    float cos[C][V], sin[C][V];

    // A wave's lanes form the angles of a token, one pair each, and take what their own pairs need from LDS, which keeps a wave's
    // accesses in their order.
    template <bool SIDE>
    __device__ __forceinline__ void at(const Rotation& how, int64_t token, int wave_lane, int lane, int per_head, int d, float2* shared) {
        double whole, rest = 0.0;                                // together the position
        if (how.wide) {
            const int64_t at = static_cast<const int64_t*>(how.positions)[token];
            const double upper = ldexp((double)(int32_t)(at >> 32), 32), lower = (double)(uint32_t)at;
            whole = upper + lower;
            rest = lower - (whole - upper);
        } else {
            whole = (double)static_cast<const int32_t*>(how.positions)[token];
        }
        __builtin_amdgcn_wave_barrier();
        for (int p = wave_lane; p < how.r; p += 64) {
            const double f = how.frequencies[p], g = f * kTurn, g_rest = fma(f, kTurn, -g) + f * kTurnRest;
            const double product = whole * g, small = fma(whole, g, -product) + fma(whole, g_rest, rest * g);
            double turns = product - rint(product) + small;
            turns -= rint(turns);
            float2 v;
            sincospif(2.f * (float)turns, &v.y, &v.x);
            v.x *= how.magnitude;
            v.y *= how.magnitude * how.sign;
            shared[p] = v;
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int run = (lane + c * per_head) * V;
                const int p = !SIDE || V == 1 ? run + j : j < V / 2 ? run / 2 + j : (run + d / 2) / 2 + j - V / 2;
                const float2 v = shared[p < kMostDim / 2 ? p : 0];
                cos[c][j] = p < how.r ? v.x : 1.f;
                sin[c][j] = p < how.r ? v.y : 0.f;
            }
        }
    }
    // (x, y) by the angle; BACK: by its opposite.
    template <bool SIDE, bool BACK, bool COPIES>
    __device__ __forceinline__ void turn(float (&x)[C][2 * V]) const {
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float &a = x[c][SIDE ? 2 * j : j], &b = x[c][SIDE ? 2 * j + 1 : V + j];
                const float s = sin[c][j], u = a, v = b;
                a = fmaf(u, cos[c][j], -by_sine<COPIES, BACK>(v, s));
                b = fmaf(v, cos[c][j], -by_sine<COPIES, !BACK>(u, s));
            }
        }
    }
};

// Sum over the lanes of a head, in all of them.
__device__ __forceinline__ float head_sum(float x, int per_head) {
    for (int step = per_head >> 1; step > 0; step >>= 1) x += __shfl_xor(x, step);
    return x;
}
template <int N, int C>
__device__ __forceinline__ float dot(const float (&x)[C][N], const float (&y)[C][N]) {
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int j = 0; j < N; ++j) sum = fmaf(x[c][j], y[c][j], sum);
    }
    return sum;
}
// Gains as fp32 in LDS for all waves of a workgroup, and a lane's from there: in registers they would cost waves.
__device__ __forceinline__ void keep_gain(float* kept, const void* gain, int bf16, int d) {
    if (!gain) return;
    for (int i = threadIdx.x; i < d; i += kThreads)
        kept[i] = bf16 ? widened(static_cast<const uint16_t*>(gain)[i]) : static_cast<const float*>(gain)[i];
}
template <class T, int V, bool SIDE, int C>
__device__ __forceinline__ void take_gain(const Lanes<T, V, SIDE>& lanes, const float* kept, float (&w)[C][2 * V]) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int a = lanes.there[c] ? lanes.first[c] : 0, b = lanes.there[c] ? lanes.second[c] : 0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            w[c][j] = kept[a + j];
            w[c][V + j] = kept[b + j];
        }
    }
}

// How a launch's waves share the tokens: wave i takes heads `part`, part + parts, ... (in runs of 64 / L) of token i / parts.
struct Shares {
    int64_t tokens;
    int d, per_head, lane_bits, parts;
};

template <class T>
struct Forward {
    View<const T> in[2];
    View<T> out[2];
    const void* gain[2];
    int gain_bf16;
    float eps, inverse_d;
};

// Loads of so many runs of heads are under way at once, the first of them while the angles are formed.  More cost registers, and with
// them waves.  16384 x 32 heads of 128 bf16 channels: norm 55 us (4: 72, of one wave less a SIMD), gradient, when both
// sides were one workgroup's, 96 (2: 109), now 85.  (Of the variants that keep to these bounds, two put registers aside in memory, both for
// eight pairs a lane, half a head apart: the norm one, the gradient three.)
constexpr int kRunsAhead = 3, kWavesASimd = 5;
constexpr int grad_runs_ahead(int v) { return v == 8 ? 1 : 2; }
constexpr int grad_waves_a_simd(int v) { return v == 8 ? 4 : 3; }

template <class T, int V, bool SIDE, bool NORM>
__global__ __launch_bounds__(kThreads, kWavesASimd) void heads_kernel(Forward<T> args, Rotation how, Shares share) {
    using Mine = Lanes<T, V, SIDE>;
    constexpr int C = Mine::C;
    __shared__ float2 angles[kWaves][kMostDim / 2];
    const int lane = threadIdx.x & 63, in_head = lane & (share.per_head - 1), slot = lane >> share.lane_bits;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at_once = 64 >> share.lane_bits;
    const Mine mine(in_head, share.per_head, share.d, how.r);
    const int64_t items = share.tokens * share.parts;
    const int first_runs = (args.in[0].heads + at_once - 1) / at_once, runs = first_runs + (args.in[1].heads + at_once - 1) / at_once;
    __shared__ __align__(16) float gains[NORM ? 2 : 1][NORM ? kMostDim : 1];
    if (NORM) {
        keep_gain(gains[0], args.gain[0], args.gain_bf16, share.d);
        keep_gain(gains[NORM], args.gain[1], args.gain_bf16, share.d);
        __syncthreads();
    }
    for (int64_t item = (int64_t)blockIdx.x * kWaves + wave; item < items; item += (int64_t)gridDim.x * kWaves) {
        const int64_t token = item / share.parts;
        const int part = (int)(item - token * share.parts);
        Turn<V, C> turn;
        for (int run = part; run < runs; run += kRunsAhead * share.parts) {
            typename Mine::Raw raw[kRunsAhead];
#pragma unroll
            for (int u = 0; u < kRunsAhead; ++u) {
                const int r = run + u * share.parts, side = r >= first_runs;
                const int head = (side ? r - first_runs : r) * at_once + slot;
                const View<const T>& in = side ? args.in[1] : args.in[0];
                if (r < runs && head < in.heads) mine.load(in.at + token * in.token + head * in.head, raw[u]);
            }
            if (run == part) turn.template at<SIDE>(how, token, lane, in_head, share.per_head, share.d, angles[wave]);
#pragma unroll
            for (int u = 0; u < kRunsAhead; ++u) {
                const int r = run + u * share.parts, side = r >= first_runs;
                const int head = (side ? r - first_runs : r) * at_once + slot;
                const View<T>& out = side ? args.out[1] : args.out[0];
                if (r >= runs || head >= out.heads) continue;    // (sums below are among the lanes of one head)
                float x[C][2 * V];
                mine.take(raw[u], x);
                if (NORM) {
                    const float inverse = rsqrtf(fmaf(head_sum(dot(x, x), share.per_head), args.inverse_d, args.eps));
                    float w[C][2 * V];
                    take_gain(mine, gains[side ? NORM : 0], w);
#pragma unroll
                    for (int c = 0; c < C; ++c) {
#pragma unroll
                        for (int j = 0; j < 2 * V; ++j) x[c][j] = x[c][j] * inverse * w[c][j];
                    }
                }
                turn.template turn<SIDE, false, !NORM>(x);
                mine.store(out.at + token * out.token + head * out.head, x);
            }
        }
    }
}

// ---------------------------------------------------------------- gradient
//
// With n = 1 / sqrt(mean x^2 + eps), y = R (w x n), and g = R^T dy:  dw = sum of g x n over tokens and heads,
// h = g w,  dx = n (h - x n mean(h x n)).  x is read again: n is one number for two passes over a head's registers.
// Sums of dw stay in a lane's registers over all of its tokens; a workgroup's are joined in LDS, and the workgroups' by
// join_kernel, each in an order that the sizes alone decide.
template <class T>
struct Backward {
    View<const T> dy[2], x[2];
    View<T> dx[2];
    const void* gain[2];
    int gain_bf16;
    float eps, inverse_d;
    float* partial;                                          // [workgroup][d]
    int groups[2], parts[2];                                 // workgroups of the queries, then of the keys; shares of a token's heads
};

template <class T, int V, bool SIDE>
__global__ __launch_bounds__(kThreads, grad_waves_a_simd(V)) void heads_grad_kernel(Backward<T> args, Rotation how, Shares share) {
    using Mine = Lanes<T, V, SIDE>;
    constexpr int C = Mine::C;
    constexpr int kAhead = grad_runs_ahead(V);
    __shared__ float sums[kWaves][kMostDim];
    __shared__ float2 angles[kWaves][kMostDim / 2];
    const int lane = threadIdx.x & 63, in_head = lane & (share.per_head - 1), slot = lane >> share.lane_bits;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at_once = 64 >> share.lane_bits;
    const Mine mine(in_head, share.per_head, share.d, how.r);
    __shared__ __align__(16) float gain[kMostDim];
    const int side = (int)blockIdx.x >= args.groups[0];      // queries or keys: the sums of one gain take registers
    const int group = side ? blockIdx.x - args.groups[0] : blockIdx.x, groups = args.groups[side], parts = args.parts[side];
    const int64_t items = share.tokens * parts;
    const View<const T> in = args.x[side], grad = args.dy[side];
    const View<T> out = args.dx[side];
    const int runs = (in.heads + at_once - 1) / at_once;
    keep_gain(gain, args.gain[side], args.gain_bf16, share.d);
    __syncthreads();
    float dw[C][2 * V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) dw[c][j] = 0.f;
    }
    for (int64_t item = (int64_t)group * kWaves + wave; item < items; item += (int64_t)groups * kWaves) {
        const int64_t token = item / parts;
        const int part = (int)(item - token * parts);
        Turn<V, C> turn;
        for (int run = part; run < runs; run += kAhead * parts) {
            typename Mine::Raw raw_x[kAhead], raw_g[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int head = (run + u * parts) * at_once + slot;
                if (head >= in.heads) continue;
                mine.load(in.at + token * in.token + head * in.head, raw_x[u]);
                mine.load(grad.at + token * grad.token + head * grad.head, raw_g[u]);
            }
            if (run == part) turn.template at<SIDE>(how, token, lane, in_head, share.per_head, share.d, angles[wave]);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int head = (run + u * parts) * at_once + slot;
                if (head >= in.heads) continue;          // (sums below are among the lanes of one head)
                float x[C][2 * V], g[C][2 * V], w[C][2 * V];
                mine.take(raw_x[u], x);
                mine.take(raw_g[u], g);
                const float inverse = rsqrtf(fmaf(head_sum(dot(x, x), share.per_head), args.inverse_d, args.eps));
                turn.template turn<SIDE, true, false>(g);
                take_gain(mine, gain, w);
#pragma unroll
                for (int c = 0; c < C; ++c) {
#pragma unroll
                    for (int j = 0; j < 2 * V; ++j) {
                        x[c][j] *= inverse;
                        dw[c][j] = fmaf(g[c][j], x[c][j], dw[c][j]);
                        g[c][j] *= w[c][j];
                    }
                }
                const float mean = head_sum(dot(g, x), share.per_head) * args.inverse_d;
#pragma unroll
                for (int c = 0; c < C; ++c) {
#pragma unroll
                    for (int j = 0; j < 2 * V; ++j) x[c][j] = inverse * fmaf(-mean, x[c][j], g[c][j]);
                }
                mine.store(out.at + token * out.token + head * out.head, x);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) {
            float sum = dw[c][j];
            for (int step = share.per_head; step < 64; step <<= 1) sum += __shfl_xor(sum, step);
            if (slot == 0 && mine.there[c]) sums[wave][j < V ? mine.first[c] + j : mine.second[c] + j - V] = sum;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < share.d; i += kThreads) {
        float sum = sums[0][i];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) sum += sums[v][i];
        args.partial[(int64_t)blockIdx.x * share.d + i] = sum;
    }
}

// Sums of the workgroups' partial sums, 16 channels of one gain a workgroup, all of its loads at once.
__global__ __launch_bounds__(kJoinThreads) void heads_join_kernel(const float* __restrict__ partial, int q_groups, int k_groups, int d,
                                                                  float* dq_gain, float* dk_gain, int accumulate) {
    constexpr int kParts = kJoinThreads / kJoinRows, kEach = kGradGroups / kParts;
    __shared__ float sums[kJoinThreads];
    const int i = blockIdx.x * kJoinRows + threadIdx.x % kJoinRows, part = threadIdx.x / kJoinRows;
    const int groups = blockIdx.y ? k_groups : q_groups;
    if (blockIdx.y) partial += (int64_t)q_groups * d;
    float v[kEach], sum = 0.f;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int g = part + e * kParts;
        v[e] = i < d && g < groups ? partial[(int64_t)g * d + i] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) sum += v[e];
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int half = kParts / 2; half > 0; half /= 2) {
        if (part < half) sums[threadIdx.x] = sum += sums[threadIdx.x + half * kJoinRows];
        __syncthreads();
    }
    if (part > 0 || i >= d) return;
    float* out = (blockIdx.y ? dk_gain : dq_gain) + i;
    *out = accumulate ? *out + sum : sum;
}

// ---------------------------------------------------------------- host

bool fine_rotation(const sparseloco_rotation* how, int d) {
    return how && how->positions && how->frequencies && (how->position_bytes == 4 || how->position_bytes == 8) && how->pairs >= 1 &&
           how->pairs <= d / 2 && std::isfinite((float)how->magnitude);
}

// A list of heads can be walked: strides that keep every offset in 62 bits, and for one that is written to no element twice.
bool fine_heads(const sparseloco_heads* h, int64_t tokens, int d, bool written) {
    constexpr int64_t kFar = (int64_t)1 << 40;
    if (h->heads < 0 || h->heads > SPLC_MAX_HEADS) return false;
    if (h->heads == 0 || tokens == 0) return true;
    if (!h->data || h->token_stride < 0 || h->head_stride < 0 || h->token_stride > kFar || h->head_stride > kFar) return false;
    if (tokens > 1 && h->token_stride > ((int64_t)1 << 61) / tokens) return false;
    if (!written) return true;
    const int64_t s = h->token_stride, t = h->head_stride;
    const bool by_token = (tokens == 1 || s >= (h->heads - 1) * t + d) && (h->heads == 1 || t >= d);
    const bool by_head = (h->heads == 1 || t >= (tokens - 1) * s + d) && (tokens == 1 || s >= d);
    return by_token || by_head;
}

// Arguments that all three operators share; `lists`: queries and keys of the inputs and the outputs, keys NULL in all or none.
struct List {
    const sparseloco_heads *q, *k;
    bool written;
};
int check(const List* lists, int n, int dtype, int64_t tokens, int d, const sparseloco_rotation* how) {
    if ((dtype != SPLC_F32 && dtype != SPLC_BF16) || tokens < 0 || tokens > INT32_MAX || d < 2 || d > kMostDim || d % 2 != 0)
        return SPLC_EINVAL;
    for (int i = 0; i < n; ++i) {
        if (!lists[i].q || (lists[i].k == nullptr) != (lists[0].k == nullptr)) return SPLC_EINVAL;
        if (lists[i].q->heads != lists[0].q->heads || (lists[i].k && lists[i].k->heads != lists[0].k->heads)) return SPLC_EINVAL;
        if (!fine_heads(lists[i].q, tokens, d, lists[i].written) || (lists[i].k && !fine_heads(lists[i].k, tokens, d, lists[i].written)))
            return SPLC_EINVAL;
    }
    if (tokens > 0 && !fine_rotation(how, d)) return SPLC_EINVAL;
    // What is written of the queries (the last list) is not to be read of the keys, and the other way round: one may come before the other.
    const List& out = lists[n - 1];
    if (out.k && tokens > 0 && out.q->heads > 0 && out.k->heads > 0)
        for (int i = 0; i < n; ++i)
            if (out.q->data == lists[i].k->data || out.k->data == lists[i].q->data) return SPLC_EINVAL;
    // In place is element for element.
    auto elsewhere = [&](const sparseloco_heads* in, const sparseloco_heads* written) {
        return in && tokens > 0 && in->heads > 0 && in->data == written->data &&
               ((tokens > 1 && in->token_stride != written->token_stride) || (in->heads > 1 && in->head_stride != written->head_stride));
    };
    for (int i = 0; i < n - 1; ++i)
        if (elsewhere(lists[i].q, out.q) || elsewhere(lists[i].k, out.k)) return SPLC_EINVAL;
    const size_t size = dtype == SPLC_F32 ? 4 : 2;
    for (int i = 0; i < n; ++i)
        if (!aligned(lists[i].q->data, size) || (lists[i].k && !aligned(lists[i].k->data, size))) return SPLC_EALIGN;
    if (tokens > 0 && (!aligned(how->positions, (size_t)how->position_bytes) || !aligned(how->frequencies, 8))) return SPLC_EALIGN;
    return SPLC_OK;
}
int check_gains(const void* q_gain, const void* k_gain, int gain_dtype, double eps, bool keys) {
    if ((gain_dtype != SPLC_F32 && gain_dtype != SPLC_BF16) || !q_gain || (keys && !k_gain)) return SPLC_EINVAL;
    if (!std::isfinite((float)eps) || eps < 0.0) return SPLC_EINVAL;
    const size_t size = gain_dtype == SPLC_F32 ? 4 : 2;
    return aligned(q_gain, size) && aligned(k_gain, size) ? SPLC_OK : SPLC_EALIGN;
}

template <class T>
View<T> view(const sparseloco_heads* h) {
    if (!h) return {nullptr, 0, 0, 0};
    return {static_cast<T*>(h->data), h->token_stride, h->head_stride, h->heads};
}
Rotation rotation(const sparseloco_rotation* how, bool inverse) {
    return {how->positions, how->frequencies, how->position_bytes == 8, how->pairs, (float)how->magnitude, inverse ? -1.f : 1.f};
}

// Pairs that a lane holds side by side: 16 bytes' worth, or as many as all runs can have.
int run_of_pairs(int dtype, int d, int r, bool side) {
    for (int v = dtype == SPLC_BF16 ? 8 : 4; v > 1; v /= 2)
        if (side ? d / 2 % v == 0 : r % v == 0 && (d / 2 - r) % v == 0) return v;
    return 1;
}

Shares shares(int64_t tokens, int d, int v, int q_heads, int k_heads) {
    Shares s{tokens, d, 1, 0, 1};
    while (s.per_head * v < d / 2 && s.per_head < 64) {
        s.per_head *= 2;
        ++s.lane_bits;
    }
    const int at_once = 64 / s.per_head;
    const int runs = (q_heads + at_once - 1) / at_once + (k_heads + at_once - 1) / at_once;
    s.parts = (int)std::min<int64_t>(runs, std::max<int64_t>(1, kFillingWaves / std::max<int64_t>(tokens, 1)));
    return s;
}

template <class Run>
int with_variant(int dtype, int v, bool side, Run run) {
    auto of = [&](auto type, auto width) {
        if (side) run(type, width, std::true_type());
        else run(type, width, std::false_type());
    };
    auto narrow = [&](auto type) {
        if (v == 4) of(type, std::integral_constant<int, 4>());
        else if (v == 2) of(type, std::integral_constant<int, 2>());
        else of(type, std::integral_constant<int, 1>());
    };
    if (dtype == SPLC_F32) narrow(float());
    else if (v == 8) of(uint16_t(), std::integral_constant<int, 8>());
    else narrow(uint16_t());
    return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
}

template <bool NORM>
int forward(const List& in, const List& out, int dtype, int64_t tokens, int d, const void* q_gain, const void* k_gain, int gain_dtype,
            double eps, const sparseloco_rotation* how, bool inverse, void* stream) {
    const int q_heads = in.q->heads, k_heads = in.k ? in.k->heads : 0;
    if (tokens == 0 || q_heads + k_heads == 0) return SPLC_OK;
    const bool side = how->interleaved != 0;
    const int v = run_of_pairs(dtype, d, how->pairs, side);
    const Shares s = shares(tokens, d, v, q_heads, k_heads);
    const uint32_t groups = (uint32_t)std::min<int64_t>((tokens * s.parts + kWaves - 1) / kWaves, kMostGroups);
    return with_variant(dtype, v, side, [&](auto type, auto width, auto pairs_side) {
        using T = decltype(type);
        const Forward<T> args{{view<const T>(in.q), view<const T>(in.k)}, {view<T>(out.q), view<T>(out.k)}, {q_gain, k_gain},
                              gain_dtype == SPLC_BF16, (float)eps, 1.f / (float)d};
        hipLaunchKernelGGL((heads_kernel<T, decltype(width)::value, decltype(pairs_side)::value, NORM>), dim3(groups), dim3(kThreads), 0,
                           static_cast<hipStream_t>(stream), args, rotation(how, inverse), s);
    });
}

uint32_t grad_groups(int64_t tokens) { return (uint32_t)std::min<int64_t>(std::max<int64_t>(tokens, 1), kGradGroups); }

}  // namespace

extern "C" {

int sparseloco_rotary(const sparseloco_heads* q, const sparseloco_heads* k, int dtype, int64_t tokens, int head_dim,
                      const sparseloco_rotation* how, int inverse, const sparseloco_heads* q_out, const sparseloco_heads* k_out,
                      void* stream) {
    const List lists[] = {{q, k, false}, {q_out, k_out, true}};
    const int rc = check(lists, 2, dtype, tokens, head_dim, how);
    if (rc != SPLC_OK) return rc;
    return forward<false>(lists[0], lists[1], dtype, tokens, head_dim, nullptr, nullptr, SPLC_F32, 0.0, how, inverse != 0, stream);
}

int sparseloco_qk_norm_rotary(const sparseloco_heads* q, const sparseloco_heads* k, int dtype, int64_t tokens, int head_dim,
                              const void* q_gain, const void* k_gain, int gain_dtype, double eps, const sparseloco_rotation* how,
                              const sparseloco_heads* q_out, const sparseloco_heads* k_out, void* stream) {
    const List lists[] = {{q, k, false}, {q_out, k_out, true}};
    int rc = check(lists, 2, dtype, tokens, head_dim, how);
    if (rc != SPLC_OK) return rc;
    if ((rc = check_gains(q_gain, k_gain, gain_dtype, eps, k != nullptr)) != SPLC_OK) return rc;
    return forward<true>(lists[0], lists[1], dtype, tokens, head_dim, q_gain, k_gain, gain_dtype, eps, how, false, stream);
}

int64_t sparseloco_qk_norm_rotary_grad_ws_bytes(int64_t tokens, int q_heads, int k_heads, int head_dim) {
    if (tokens < 0 || tokens > INT32_MAX || q_heads < 0 || q_heads > SPLC_MAX_HEADS || k_heads < 0 || k_heads > SPLC_MAX_HEADS ||
        head_dim < 2 || head_dim > kMostDim || head_dim % 2 != 0)
        return SPLC_EINVAL;
    return (int64_t)grad_groups(tokens) * 2 * head_dim * 4;
}

int sparseloco_qk_norm_rotary_grad(const sparseloco_heads* grad_q_out, const sparseloco_heads* grad_k_out, const sparseloco_heads* q,
                                   const sparseloco_heads* k, int dtype, int64_t tokens, int head_dim, const void* q_gain,
                                   const void* k_gain, int gain_dtype, double eps, const sparseloco_rotation* how,
                                   const sparseloco_heads* grad_q, const sparseloco_heads* grad_k, float* grad_q_gain,
                                   float* grad_k_gain, int accumulate, void* ws, int64_t ws_bytes, void* stream) {
    const List lists[] = {{grad_q_out, grad_k_out, false}, {q, k, false}, {grad_q, grad_k, true}};
    int rc = check(lists, 3, dtype, tokens, head_dim, how);
    if (rc != SPLC_OK) return rc;
    if ((rc = check_gains(q_gain, k_gain, gain_dtype, eps, k != nullptr)) != SPLC_OK) return rc;
    const int q_heads = q->heads, k_heads = k ? k->heads : 0;
    if (!grad_q_gain || (k != nullptr) != (grad_k_gain != nullptr) || !ws) return SPLC_EINVAL;
    if (ws_bytes < sparseloco_qk_norm_rotary_grad_ws_bytes(tokens, q_heads, k_heads, head_dim)) return SPLC_EINVAL;
    if (!aligned(grad_q_gain, 4) || !aligned(grad_k_gain, 4) || !aligned(ws, 4)) return SPLC_EALIGN;
    // (two workgroups at once add to them)
    if (k && std::abs(reinterpret_cast<intptr_t>(grad_q_gain) - reinterpret_cast<intptr_t>(grad_k_gain)) < 4 * (intptr_t)head_dim) return SPLC_EINVAL;
    int groups[2] = {0, 0};
    if (tokens > 0 && q_heads + k_heads > 0) {
        const bool side = how->interleaved != 0;
        const int v = run_of_pairs(dtype, head_dim, how->pairs, side);
        const Shares s = shares(tokens, head_dim, v, q_heads, k_heads);
        // With eight pairs a lane as many workgroups as run at once, 1024, shared out by the heads of either side: 16384 tokens x 32
        // heads of 128 bf16 channels 85 us, with 1024 for either side 91.  Lanes of fewer pairs, all of fp32 among them, gain from
        // more: 16384 x 24 heads of 80 fp32 channels 61 us so, 53 with 1024 for either side.
        const int at_once = 64 / s.per_head;
        int parts[2] = {1, 1};
        for (int keys = 0; keys < 2; ++keys) {
            const int heads = keys ? k_heads : q_heads, runs = (heads + at_once - 1) / at_once;
            if (heads == 0) continue;
            parts[keys] = (int)std::min<int64_t>(runs, std::max<int64_t>(1, kFillingWaves / tokens));
            const int64_t share = v == 8 ? std::max<int64_t>(1, (int64_t)kGradGroups * heads / (q_heads + k_heads)) : kGradGroups;
            const int64_t most = std::min<int64_t>(grad_groups(tokens), share);
            groups[keys] = (int)std::min<int64_t>((tokens * parts[keys] + kWaves - 1) / kWaves, most);
        }
        rc = with_variant(dtype, v, side, [&](auto type, auto width, auto pairs_side) {
            using T = decltype(type);
            const Backward<T> args{{view<const T>(grad_q_out), view<const T>(grad_k_out)}, {view<const T>(q), view<const T>(k)},
                                   {view<T>(grad_q), view<T>(grad_k)}, {q_gain, k_gain}, gain_dtype == SPLC_BF16, (float)eps,
                                   1.f / (float)head_dim, static_cast<float*>(ws), {groups[0], groups[1]}, {parts[0], parts[1]}};
            hipLaunchKernelGGL((heads_grad_kernel<T, decltype(width)::value, decltype(pairs_side)::value>), dim3((unsigned)(groups[0] + groups[1])), dim3(kThreads),
                               0, static_cast<hipStream_t>(stream), args, rotation(how, false), s);
        });
        if (rc != SPLC_OK) return rc;
    }
    hipLaunchKernelGGL(heads_join_kernel, dim3((head_dim + kJoinRows - 1) / kJoinRows, k ? 2 : 1), dim3(kJoinThreads), 0,
                       static_cast<hipStream_t>(stream), static_cast<const float*>(ws), groups[0], groups[1], head_dim, grad_q_gain, grad_k_gain,
                       accumulate);
    return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
}

}  // extern "C"
