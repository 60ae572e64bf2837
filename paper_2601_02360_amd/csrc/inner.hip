// The inner step for gfx950 (MI355X): the norm of all gradients with the factor that clips it, and AdamW over all tensors of
// a plan with both moments in fp32 or in 8 bits.
//
// All three are element-wise over the tensors, whatever the plan's layout: they walk its flat chunks (4096 consecutive
// elements, one workgroup at a time), lane `tid` holding, for slot s = 0..3 and j = 0..3, element s*1024 + tid*4 + j, as in
// the outer update.  They are bound by memory traffic, and move little that does not have to be moved (rocprofv3, fetched and
// written: both AdamW steps within 0.5 % of it, the bf16 norm 3.7 % more).  MI355X, the 0.9B model (888 M parameters):
//   norm           2 bytes a parameter (bf16, packed tensors)     0.257 ms   6.9 TB/s
//   AdamW          28 (bf16 gradients, fp32 moments, bf16 copy)   4.43 ms    5.6 TB/s
//   AdamW, 8 bits  16.1 (the same; aligned tensors)               2.43 ms    5.9 TB/s
//                  16.1 (the same; packed tensors)                2.70 ms    5.3 TB/s
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "launch_rules.h"
#include "plan.h"
#include "sparseloco.h"

namespace {

using namespace splc;

constexpr int kThreads = 256;            // one workgroup per chunk
constexpr int kNormGroups = SPLC_NORM_WS_BYTES / 8, kJoinThreads = 1024;

// Which of a vector's four elements are present: those from `from` to `to`.  WHOLE: all.
struct Present {
    uint32_t from, to;
    __device__ __forceinline__ bool all() const { return from == 0 && to == 4; }
    __device__ __forceinline__ bool has(uint32_t j) const { return from <= j && j < to; }
};
// Of the vector at place `at`, where the places lo .. hi - 1 hold elements.
__device__ __forceinline__ Present present(uint32_t at, uint32_t lo, uint32_t hi) {
    return {lo > at ? (lo - at < 4u ? lo - at : 4u) : 0u, hi > at ? (hi - at < 4u ? hi - at : 4u) : 0u};
}
// Four elements at p, +0 for those that are not present.
template <bool WHOLE, class T>
__device__ __forceinline__ float4 load_present(const T* p, Present n) {
    if (WHOLE) return widened(stream_load4(p));
    if (n.all()) return widened(cached_load4(p));
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (n.has(0)) v.x = widened(p[0]);
    if (n.has(1)) v.y = widened(p[1]);
    if (n.has(2)) v.z = widened(p[2]);
    if (n.has(3)) v.w = widened(p[3]);
    return v;
}
template <bool WHOLE>
__device__ __forceinline__ void store_present(float* p, Present n, float4 v) {
    if (WHOLE || n.all()) {
        stream_store4(p, v);
        return;
    }
    if (n.has(0)) p[0] = v.x;
    if (n.has(1)) p[1] = v.y;
    if (n.has(2)) p[2] = v.z;
    if (n.has(3)) p[3] = v.w;
}
template <bool WHOLE>
__device__ __forceinline__ void store_present(uint16_t* p, Present n, float4 v) {
    if (WHOLE || n.all()) {
        stream_store4(p, v);
        return;
    }
    const uint32_t lo = bf16_pair(v.x, v.y), hi = bf16_pair(v.z, v.w);
    if (n.has(0)) p[0] = (uint16_t)lo;
    if (n.has(1)) p[1] = (uint16_t)(lo >> 16);
    if (n.has(2)) p[2] = (uint16_t)hi;
    if (n.has(3)) p[3] = (uint16_t)(hi >> 16);
}

// ---------------------------------------------------------------- norm

// Sum over the workgroup, valid in lane 0 of wave 0; the order of the additions is fixed.
template <int THREADS>
__device__ __forceinline__ double group_sum(double x, double* shared) {
    for (int step = 32; step > 0; step >>= 1) x += __shfl_down(x, step);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < THREADS / 64; ++w) x += shared[w];
    return x;
}

// Sum of squares, formed and added in 64 bits: no fp32 value's square overflows or vanishes there, and no order of adding
// 10^9 of them loses anything that fp32 shows; at a multiply-add per element the vector ALU has time for it.  A workgroup takes
// every so manieth chunk, and one more workgroup adds the partial sums: 2048 x 2048, which caches hold, 3.4 to 5.4 us and 1.9 us.
template <class T>
__global__ __launch_bounds__(kThreads) void norm_partial_kernel(const ChunkDesc* __restrict__ chunks, uint32_t n_chunks,
                                                                const T* const* __restrict__ grad_tab,
                                                                double* __restrict__ partial) {
    __shared__ double shared[kThreads / 64];
    const uint32_t tid = threadIdx.x;
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < n_chunks; c += gridDim.x) {
        const ChunkDesc d = chunks[c];
        const T* g = grad_tab[d.tensor] + d.offset;
        float4 x[4];
        if (d.n_c == kChunk) {
#pragma unroll
            for (int s = 0; s < 4; ++s) x[s] = load_present<true>(g + s * 1024 + tid * 4, {0, 4});
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s)
                x[s] = load_present<false>(g + s * 1024 + tid * 4, present((uint32_t)s * 1024 + tid * 4, 0, d.n_c));
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            sum = fma((double)x[s].x, (double)x[s].x, sum);
            sum = fma((double)x[s].y, (double)x[s].y, sum);
            sum = fma((double)x[s].z, (double)x[s].z, sum);
            sum = fma((double)x[s].w, (double)x[s].w, sum);
        }
    }
    sum = group_sum<kThreads>(sum, shared);
    if (tid == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(const double* __restrict__ partial, uint32_t n, float max_norm,
                                                                 float* __restrict__ out) {
    __shared__ double shared[kJoinThreads / 64];
    static_assert(kNormGroups == 2 * kJoinThreads, "two partial sums a lane");
    const uint32_t i = threadIdx.x, j = i + kJoinThreads;
    const double sum = group_sum<kJoinThreads>((i < n ? partial[i] : 0.0) + (j < n ? partial[j] : 0.0), shared);
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum);
        out[0] = (float)norm;
        const bool fine = out[0] - out[0] == 0.f;
        out[1] = !fine ? __uint_as_float(0x7FC00000u) : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
    }
}

// ---------------------------------------------------------------- AdamW

// One step's numbers, rounded once from 64 bits.
struct StepNumbers {
    float beta1, rest1, beta2, rest2;    // rest = 1 - beta
    float size;                          // lr / (1 - beta1^step)
    float root_factor;                   // 1 / sqrt(1 - beta2^step)
    float eps;
    float shrink;                        // lr * weight_decay
};

// m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2, the second product and the sum rounded together.
__device__ __forceinline__ void moments(const StepNumbers& n, float g, float& m, float& v) {
    m = fmaf(n.rest1, g, n.beta1 * m);
    v = fmaf(n.rest2, g * g, n.beta2 * v);
}
// theta (1 - lr wd) - lr m^ / (sqrt(v^) + eps), with the bias corrections m^ = m / (1 - beta1^t), v^ = v / (1 - beta2^t).
__device__ __forceinline__ float stepped(const StepNumbers& n, float keep, float theta, float m, float root) {
    return theta * keep - n.size * (m / (root * n.root_factor + n.eps));
}

// The factor on the gradients; false if it is not finite: then nothing is to be changed.
__device__ __forceinline__ bool gradient_factor(const float* grad_scale, float& factor) {
    factor = grad_scale ? *grad_scale : 1.f;
    return factor - factor == 0.f;
}

// Four elements.
__device__ __forceinline__ void adamw4(const StepNumbers& n, float keep, float factor, float4 g, float4& t, float4& m, float4& v) {
    auto one = [&](float& th, float gradient, float& mm, float& vv) {
        moments(n, factor * gradient, mm, vv);
        th = stepped(n, keep, th, mm, sqrtf(vv));
    };
    one(t.x, g.x, m.x, v.x);
    one(t.y, g.y, m.y, v.y);
    one(t.z, g.z, m.z, v.z);
    one(t.w, g.w, m.w, v.w);
}

// A workgroup's elements begin where theta has a multiple of 256 bytes, up to 63 elements before its chunk, and end as many
// before the next one's; the first of a tensor begins with it, and the last ends with it, up to 63 elements beyond 4096.  With
// tensors packed into flat buffers, the usual case of others than aligned ones, that holds for all arrays.  (0.9B parameters
// packed at multiples of eight bytes, bf16 gradients and copy: 5.16 ms with chunks as they lie, 4.57 so; without the streaming hint
// instead 5.14.)  Division and square root are rounded to nearest: memory leaves the time for them.
template <class G>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const ChunkDesc* __restrict__ chunks, const int64_t* __restrict__ numel,
                                                         float* const* __restrict__ theta_tab,
                                                         const G* const* __restrict__ grad_tab,
                                                         float* const* __restrict__ m_tab, float* const* __restrict__ v_tab,
                                                         uint16_t* const* __restrict__ copy_tab, StepNumbers numbers,
                                                         const float* __restrict__ grad_scale,
                                                         const float* __restrict__ decay) {
    const ChunkDesc d = chunks[blockIdx.x];
    float factor;
    if (!gradient_factor(grad_scale, factor)) return;
    const float keep = 1.f - (decay ? numbers.shrink * decay[d.tensor] : numbers.shrink);
    const uint32_t tid = threadIdx.x;
    float* theta = theta_tab[d.tensor];
    const uint32_t lead = (uint32_t)(reinterpret_cast<uintptr_t>(theta) / 4) & 63u;
    const bool first = d.offset == 0, last = (int64_t)d.offset + d.n_c == numel[d.tensor];
    const int64_t from = (int64_t)d.offset - lead;           // element at place 0
    theta += from;
    float *m = m_tab[d.tensor] + from, *v = v_tab[d.tensor] + from;
    const G* grad = grad_tab[d.tensor] + from;
    uint16_t* copy = copy_tab ? copy_tab[d.tensor] + from : nullptr;
    if (d.n_c == kChunk && (lead == 0 || !(first || last))) {
        float4 t4[4], g4[4], m4[4], v4[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const uint32_t at = (uint32_t)s * 1024 + tid * 4;
            g4[s] = widened(stream_load4(grad + at));
            m4[s] = stream_load4(m + at);
            v4[s] = stream_load4(v + at);
            t4[s] = stream_load4(theta + at);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const uint32_t at = (uint32_t)s * 1024 + tid * 4;
            adamw4(numbers, keep, factor, g4[s], t4[s], m4[s], v4[s]);
            stream_store4(m + at, m4[s]);
            stream_store4(v + at, v4[s]);
            stream_store4(theta + at, t4[s]);
            if (copy) stream_store4(copy + at, t4[s]);
        }
        return;
    }
    const uint32_t lo = first ? lead : 0, hi = last ? d.n_c + lead : (uint32_t)kChunk;
    for (uint32_t at = tid * 4; at < hi; at += 1024) {
        const Present n = present(at, lo, hi);
        if (n.from >= n.to) continue;
        float4 g4 = load_present<false>(grad + at, n), m4 = load_present<false>(m + at, n), v4 = load_present<false>(v + at, n),
               t4 = load_present<false>(theta + at, n);
        adamw4(numbers, keep, factor, g4, t4, m4, v4);
        store_present<false>(m + at, n, m4);
        store_present<false>(v + at, n, v4);
        store_present<false>(theta + at, n, t4);
        if (copy) store_present<false>(copy + at, n, t4);
    }
}

// ---------------------------------------------------------------- AdamW, moments in 8 bits
//
// A block is 256 consecutive elements of a chunk: one slot of one wave, four elements a lane, so that its largest magnitude
// is found inside a wave and everything of a chunk stays in its lanes' registers from the first load to the last store.  Held are
// m / scale and sqrt(v) / scale as e4m3 numbers (largest 448), scale = largest of the block / 448: a number of exponent as well as
// mantissa bits, because the step divides one moment by the other and so needs a block's small elements as exactly as its
// large ones, and the root, which has half of v's range of exponents.

constexpr float kMost8 = 448.f;

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    for (int step = 32; step > 0; step >>= 1) {
        const uint32_t y = __shfl_xor(x, step);
        x = x > y ? x : y;
    }
    return x;
}
__device__ __forceinline__ float magnitude(float x) { return __uint_as_float(__float_as_uint(x) & 0x7FFFFFFFu); }
// The largest magnitude of a block (lane: four of its elements).  As integers non-negative floats keep their order, and
// infinities and NaN come out on top: a block that holds one gets a scale that shows it.
__device__ __forceinline__ float block_max(float4 x) {
    auto bits = [](float v) { return __float_as_uint(v) & 0x7FFFFFFFu; };
    const uint32_t a = bits(x.x) > bits(x.y) ? bits(x.x) : bits(x.y), b = bits(x.z) > bits(x.w) ? bits(x.z) : bits(x.w);
    return __uint_as_float(wave_max(a > b ? a : b));
}
// Below this a block's values are held as zeros (448 over it stays finite; no square root of an fp32 number is so small).
constexpr float kLeastHeld = 0x1p-118f;

// y (0 <= y <= 448, or a rounding more) as an e4m3 number: to the upper neighbour where the fraction of the gap that y
// covers, plus threshold / 2^20, reaches 1.  Times 2^-120 an e4m3 number's exponent and mantissa are bits 20 to 26 of the
// fp32 pattern, those of its subnormals too, and the bits below them are the fraction.
__device__ __forceinline__ uint32_t e4m3_between(float y, uint32_t threshold) {
    const uint32_t code = (__float_as_uint(y * 0x1p-120f) + threshold) >> 20;
    return code < 126u ? code : 126u;
}
// Thresholds walk through the unit interval from element to element and from step to step: multiples, modulo 1, of the two
// numbers of the plane's golden-ratio sequence, 1 / p and 1 / p^2 with p^3 = p + 1.
constexpr uint32_t kPlaceStep = 0xC13FA9A9u, kTimeStep = 0x91E10DA5u;

__device__ __forceinline__ float4 unheld(uint32_t codes, float scale) {
    typedef float vfloat2 __attribute__((ext_vector_type(2)));
    const vfloat2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
    return make_float4(lo.x * scale, lo.y * scale, hi.x * scale, hi.y * scale);
}

template <bool WHOLE, class G>
__device__ __forceinline__ void adamw_8bit_body(const ChunkDesc& d, float* theta, const G* grad, uint32_t* m_codes,
                                                float* m_scale, uint32_t* v_codes, float* v_scale, uint16_t* copy,
                                                const StepNumbers& numbers, uint32_t now, float factor, float keep) {
    const uint32_t tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    float4 t4[4], g4[4];
    uint32_t mc[4], vc[4];
    float ms[4], vs[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uint32_t at = (uint32_t)s * 1024 + tid * 4;
        const Present n = present(at, 0, d.n_c);
        g4[s] = load_present<WHOLE>(grad + at, n);
        mc[s] = __builtin_nontemporal_load((SPLC_GLOBAL uint32_t*)(m_codes + s * 256 + tid));
        vc[s] = __builtin_nontemporal_load((SPLC_GLOBAL uint32_t*)(v_codes + s * 256 + tid));
        ms[s] = m_scale[s * 4 + wave];
        vs[s] = v_scale[s * 4 + wave];
        t4[s] = load_present<WHOLE>(theta + at, n);
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uint32_t at = (uint32_t)s * 1024 + tid * 4;
        const Present n = present(at, 0, d.n_c);
        if (!WHOLE) {                                         // what lies behind a tensor's end counts as zero
            const uint32_t mask = n.to == 4 ? 0xFFFFFFFFu : (1u << (8 * n.to)) - 1u;
            mc[s] &= mask;
            vc[s] &= mask;
        }
        float4 m = unheld(mc[s], ms[s]), r = unheld(vc[s], vs[s]);
        auto one = [&](float& th, float g, float& mm, float& root) {
            float v = root * root;
            moments(numbers, factor * g, mm, v);
            root = sqrtf(v);
            th = stepped(numbers, keep, th, mm, root);
        };
        one(t4[s].x, g4[s].x, m.x, r.x);
        one(t4[s].y, g4[s].y, m.y, r.y);
        one(t4[s].z, g4[s].z, m.z, r.z);
        one(t4[s].w, g4[s].w, m.w, r.w);
        store_present<WHOLE>(theta + at, n, t4[s]);
        if (copy) store_present<WHOLE>(copy + at, n, t4[s]);

        const float m_most = block_max(m), r_most = block_max(r);
        const float m_inverse = m_most < kLeastHeld ? 0.f : kMost8 * (1.f / m_most), r_inverse = r_most < kLeastHeld ? 0.f : kMost8 * (1.f / r_most);
        const uint32_t place = (d.id * (uint32_t)kChunk + at) * kPlaceStep + now;
        uint32_t m_new = 0, v_new = 0;
        auto hold = [&](float mm, float root, uint32_t j) {
            const uint32_t at_m = place + j * kPlaceStep, at_v = at_m + 0x80000000u;
            const uint32_t code = e4m3_between(magnitude(mm) * m_inverse, at_m >> 12) | (mm * m_inverse < 0.f ? 0x80u : 0u);
            const float y = root * r_inverse;
            uint32_t root_code = e4m3_between(y, at_v >> 12);
            if (y > 0.f && root_code == 0) root_code = 1;     // a root of zero under a moment would make a step of m / eps
            m_new |= code << (8 * j);
            v_new |= root_code << (8 * j);
        };
        hold(m.x, r.x, 0);
        hold(m.y, r.y, 1);
        hold(m.z, r.z, 2);
        hold(m.w, r.w, 3);
        __builtin_nontemporal_store(m_new, (SPLC_GLOBAL uint32_t*)(m_codes + s * 256 + tid));
        __builtin_nontemporal_store(v_new, (SPLC_GLOBAL uint32_t*)(v_codes + s * 256 + tid));
        if ((tid & 63) == 0) {
            m_scale[s * 4 + wave] = m_most < kLeastHeld ? 0.f : m_most * (1.f / kMost8);
            v_scale[s * 4 + wave] = r_most < kLeastHeld ? 0.f : r_most * (1.f / kMost8);
        }
    }
}

template <class G>
__global__ __launch_bounds__(kThreads) void adamw_8bit_kernel(const ChunkDesc* __restrict__ chunks,
                                                              float* const* __restrict__ theta_tab,
                                                              const G* const* __restrict__ grad_tab,
                                                              uint8_t* __restrict__ m_codes, float* __restrict__ m_scale,
                                                              uint8_t* __restrict__ v_codes, float* __restrict__ v_scale,
                                                              uint16_t* const* __restrict__ copy_tab, StepNumbers numbers,
                                                              uint32_t now, const float* __restrict__ grad_scale,
                                                              const float* __restrict__ decay) {
    const ChunkDesc d = chunks[blockIdx.x];
    float factor;
    if (!gradient_factor(grad_scale, factor)) return;
    const float keep = 1.f - (decay ? numbers.shrink * decay[d.tensor] : numbers.shrink);
    float* theta = theta_tab[d.tensor] + d.offset;
    const G* grad = grad_tab[d.tensor] + d.offset;
    uint16_t* copy = copy_tab ? copy_tab[d.tensor] + d.offset : nullptr;
    const uint64_t chunk = d.id;
    uint32_t *mc = reinterpret_cast<uint32_t*>(m_codes + chunk * kChunk), *vc = reinterpret_cast<uint32_t*>(v_codes + chunk * kChunk);
    float *ms = m_scale + chunk * 16, *vs = v_scale + chunk * 16;
    if (d.n_c == kChunk) adamw_8bit_body<true>(d, theta, grad, mc, ms, vc, vs, copy, numbers, now, factor, keep);
    else adamw_8bit_body<false>(d, theta, grad, mc, ms, vc, vs, copy, numbers, now, factor, keep);
}

// ---------------------------------------------------------------- host side

bool finite64(double v) { return v - v == 0.0; }

// The step's numbers; false where an argument is out of its range or a number leaves fp32's.
bool step_numbers(const sparseloco_adamw* how, StepNumbers& n) {
    if (!how || how->step < 1) return false;
    for (double beta : {how->beta1, how->beta2})
        if (!(beta >= 0.0 && beta < 1.0)) return false;
    for (double v : {how->lr, how->eps, how->weight_decay})
        if (!finite64(v) || v < 0.0) return false;
    n.beta1 = (float)how->beta1;
    n.rest1 = (float)(1.0 - how->beta1);
    n.beta2 = (float)how->beta2;
    n.rest2 = (float)(1.0 - how->beta2);
    n.size = (float)(how->lr / (1.0 - std::pow(how->beta1, (double)how->step)));
    n.root_factor = (float)(1.0 / std::sqrt(1.0 - std::pow(how->beta2, (double)how->step)));
    n.eps = (float)how->eps;
    n.shrink = (float)(how->lr * how->weight_decay);
    return finite(n.size) && finite(n.root_factor) && finite(n.eps) && finite(n.shrink);
}

// What both forms of the step take: parameters fp32, gradients fp32 or bf16, perhaps a bf16 copy, the step's numbers.
int check_step(const sparseloco_plan* plan, const sparseloco_tensors* theta, const sparseloco_tensors* grads, int replica,
               const sparseloco_adamw* how, const float* grad_scale, const float* decay, const sparseloco_tensors* theta_bf16,
               StepNumbers& numbers) {
    if (!plan || !theta || !grads || replica < 0 || !step_numbers(how, numbers)) return SPLC_EINVAL;
    int rc;
    if ((rc = check_tensors(plan, theta, SPLC_F32, 1)) != SPLC_OK) return rc;
    if ((rc = check_tensors(plan, grads, grads->dtype, 1)) != SPLC_OK) return rc;
    if (theta_bf16 && (rc = check_tensors(plan, theta_bf16, SPLC_BF16, 1)) != SPLC_OK) return rc;
    for (const sparseloco_tensors* t : {theta, grads, theta_bf16})
        if (t && t->n_sets > 1 && replica >= t->n_sets) return SPLC_EINVAL;
    if (!aligned(grad_scale, 4) || !aligned(decay, 4)) return SPLC_EALIGN;
    return current_device_is(plan->device);
}

}  // namespace

extern "C" {

int64_t sparseloco_plan_num_flat_chunks(const sparseloco_plan* plan) { return plan ? plan->n_update : SPLC_EINVAL; }

int sparseloco_grad_norm(const sparseloco_plan* plan, const sparseloco_tensors* grads, int replica, float max_norm,
                         float* norm_out, void* ws, void* stream) {
    if (!plan || !grads || !norm_out || !ws || replica < 0 || !(max_norm > 0.f)) return SPLC_EINVAL;
    int rc = check_tensors(plan, grads, grads->dtype, 1);
    if (rc != SPLC_OK) return rc;
    if (grads->n_sets > 1 && replica >= grads->n_sets) return SPLC_EINVAL;
    if (!aligned(norm_out, 4) || !aligned(ws, 8)) return SPLC_EALIGN;
    if ((rc = current_device_is(plan->device)) != SPLC_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    double* partial = static_cast<double*>(ws);
    const uint32_t n = (uint32_t)plan->n_update, groups = n < (uint32_t)kNormGroups ? n : (uint32_t)kNormGroups;
    if (groups > 0) {
        if (grads->dtype == SPLC_BF16)
            hipLaunchKernelGGL(norm_partial_kernel<uint16_t>, dim3(groups), dim3(kThreads), 0, st, plan->d_update, n,
                               set_table<const uint16_t*>(grads, replica), partial);
        else
            hipLaunchKernelGGL(norm_partial_kernel<float>, dim3(groups), dim3(kThreads), 0, st, plan->d_update, n,
                               set_table<const float*>(grads, replica), partial);
    }
    hipLaunchKernelGGL(norm_join_kernel, dim3(1), dim3(kJoinThreads), 0, st, partial, groups, max_norm, norm_out);
    return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
}

int sparseloco_adamw_step(const sparseloco_plan* plan, const sparseloco_tensors* theta, const sparseloco_tensors* grads,
                          const sparseloco_tensors* m, const sparseloco_tensors* v, int replica, const sparseloco_adamw* how,
                          const float* grad_scale, const float* decay, const sparseloco_tensors* theta_bf16, void* stream) {
    StepNumbers numbers;
    int rc = check_step(plan, theta, grads, replica, how, grad_scale, decay, theta_bf16, numbers);
    if (rc != SPLC_OK) return rc;
    for (const sparseloco_tensors* t : {m, v}) {
        if ((rc = check_tensors(plan, t, SPLC_F32, 1)) != SPLC_OK) return rc;
        if (t->n_sets > 1 && replica >= t->n_sets) return SPLC_EINVAL;
    }
    if (plan->n_update == 0) return SPLC_OK;
    auto launch = [&](auto kernel, auto grad_tab) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)plan->n_update), dim3(kThreads),
                           plan->n_update >= splc::kFewStreamsAdamw ? reserve_lds(1, 0) : 0u, static_cast<hipStream_t>(stream),
                           plan->d_update, plan->d_numel, set_table<float*>(theta, replica), grad_tab,
                           set_table<float*>(m, replica), set_table<float*>(v, replica),
                           theta_bf16 ? set_table<uint16_t*>(theta_bf16, replica) : nullptr, numbers, grad_scale, decay);
    };
    if (grads->dtype == SPLC_BF16) launch(adamw_kernel<uint16_t>, set_table<const uint16_t*>(grads, replica));
    else launch(adamw_kernel<float>, set_table<const float*>(grads, replica));
    return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
}

int sparseloco_adamw_step_8bit(const sparseloco_plan* plan, const sparseloco_tensors* theta, const sparseloco_tensors* grads,
                               int replica, uint8_t* m, float* m_scale, uint8_t* v, float* v_scale,
                               const sparseloco_adamw* how, const float* grad_scale, const float* decay,
                               const sparseloco_tensors* theta_bf16, void* stream) {
    StepNumbers numbers;
    int rc = check_step(plan, theta, grads, replica, how, grad_scale, decay, theta_bf16, numbers);
    if (rc != SPLC_OK) return rc;
    if (plan->n_update == 0) return SPLC_OK;
    if (!m || !m_scale || !v || !v_scale) return SPLC_EINVAL;
    if (!aligned(m, 4) || !aligned(m_scale, 4) || !aligned(v, 4) || !aligned(v_scale, 4)) return SPLC_EALIGN;
    const uint32_t now = (uint32_t)how->step * kTimeStep;
    auto launch = [&](auto kernel, auto grad_tab) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)plan->n_update), dim3(kThreads),
                           reserve_lds(splc::kAdamw8GroupsPerUnit, 0), static_cast<hipStream_t>(stream),
                           plan->d_update, set_table<float*>(theta, replica), grad_tab, m, m_scale,
                           v, v_scale, theta_bf16 ? set_table<uint16_t*>(theta_bf16, replica) : nullptr, numbers, now,
                           grad_scale, decay);
    };
    if (grads->dtype == SPLC_BF16) launch(adamw_8bit_kernel<uint16_t>, set_table<const uint16_t*>(grads, replica));
    else launch(adamw_8bit_kernel<float>, set_table<const float*>(grads, replica));
    return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
}

}  // extern "C"
