// Token embeddings for gfx950 (MI355X): the lookup in the split table of section 2.4, out = scale (T_S[x] + T_perp[x]) +
// PosEmbed, and the gradient of T_S, whose row v is scale times the sum of grad_out over the tokens x_t = v.
//
// The gradient is deterministic: tokens are sorted by the row they belong to, equal ones by position, and a row's sum is
// formed by one wave (or, of a token that is frequent, by several in fixed parts, joined in order).  The sort and the sums
// are described below.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "plan.h"
#include "sparseloco.h"

namespace {

using namespace splc;

typedef __bf16 vbf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float widened(float v) { return v; }
__device__ __forceinline__ float widened(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float4 widened(float4 v) { return v; }
__device__ __forceinline__ float4 widened(uint2 v) {
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                       __uint_as_float(v.y & 0xFFFF0000u));
}
// Rounded to nearest, ties to even.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    const vbf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = (uint16_t)bf16_pair(v, v); }
__device__ __forceinline__ void put4(float* p, float4 v) { stream_store4(p, v); }
__device__ __forceinline__ void put4(uint16_t* p, float4 v) {
    const vuint2 t = {bf16_pair(v.x, v.y), bf16_pair(v.z, v.w)};
    __builtin_nontemporal_store(t, (SPLC_GLOBAL vuint2*)p);
}
// n (1..4) elements at p.
template <class T>
__device__ __forceinline__ float4 load_some(const T* p, int n) {
    if (n == 4) return widened(cached_load4(p));
    float4 v = make_float4(widened(p[0]), 0.f, 0.f, 0.f);
    if (n > 1) v.y = widened(p[1]);
    if (n > 2) v.z = widened(p[2]);
    return v;
}
template <class T>
__device__ __forceinline__ void store_some(T* p, int n, float4 v) {
    if (n == 4) {
        put4(p, v);
        return;
    }
    store1(p, v.x);
    if (n > 1) store1(p + 1, v.y);
    if (n > 2) store1(p + 2, v.z);
}
__device__ __forceinline__ int row_of(int32_t id, int vocab) { return id < 0 ? 0 : (id < vocab ? id : vocab - 1); }

// ---------------------------------------------------------------- lookup

constexpr int kLookupSpan = 1024;        // columns a wave takes: four vectors of four a lane

template <class T, class O>
__global__ __launch_bounds__(256) void lookup_kernel(const T* __restrict__ table, const T* __restrict__ t_perp,
                                                     const int32_t* __restrict__ ids, int vocab, const T* __restrict__ pos,
                                                     int seq, float scale, O* __restrict__ out, int64_t rows, int d) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t row = (int64_t)blockIdx.x * 4 + wave;
    if (row >= rows) return;
    const int64_t from = (int64_t)row_of(ids[row], vocab) * d;
    const int col = (int)blockIdx.y * kLookupSpan + lane * 4;
    const T* a = table + from;
    const T* b = t_perp ? t_perp + from : nullptr;
    const T* p = pos ? pos + (row % seq) * d : nullptr;
    float4 x[4], y[4], z[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = col + 256 * k, n = d - c < 4 ? d - c : 4;
        if (n <= 0) continue;
        x[k] = load_some(a + c, n);
        if (b) y[k] = load_some(b + c, n);
        if (p) z[k] = load_some(p + c, n);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = col + 256 * k, n = d - c < 4 ? d - c : 4;
        if (n <= 0) continue;
        float4 v = x[k];
        if (b) v = make_float4(v.x + y[k].x, v.y + y[k].y, v.z + y[k].z, v.w + y[k].w);
        v = make_float4(v.x * scale, v.y * scale, v.z * scale, v.w * scale);
        if (p) v = make_float4(v.x + z[k].x, v.y + z[k].y, v.z + z[k].z, v.w + z[k].w);
        store_some(out + row * d + c, n, v);
    }
}

// ---------------------------------------------------------------- gradient: order of the tokens
//
// Row v of the table belongs to bucket v % buckets and is row v / buckets in it, so that the frequent tokens, which mostly
// have low numbers, lie in different buckets.  One workgroup sorts a segment of 16384 tokens in LDS by (bucket, row in it),
// stably: two counting passes, first by the row, then by the bucket.  In each a wave owns consecutive items and counts
// them by itself, so that an item's place is the number of smaller ones, of equal ones in earlier waves, and of equal ones
// before it in its own.

constexpr int kSegment = 16384, kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kItems = kSegment / kSortThreads;              // items of a lane
constexpr int kMaxBuckets = 2560, kMaxBucketRows = 128;
constexpr int kWindow = 128;                                 // entries of the sorted order that one partial sum covers
constexpr uint32_t kNone = 0xFFFFFFFFu;

struct Entry {
    uint32_t token;                      // position in token_ids
    uint32_t key;                        // bucket * rows of a bucket + row in it
};

struct SortShared {
    uint16_t count[kSortWaves * kMaxBuckets];
    uint16_t order[kSegment];            // after the first pass: the segment's tokens by row in their bucket
    uint32_t wave_total[kSortWaves];
};

// From digit[j] of a lane's items (kNone: no item), item j of lane l of wave w being number (w * batches + j) * 64 + l: the
// places place[j] in their stable order.  begins(digit, place) is told where each digit begins.  Returns the number of items.
template <class Begins>
__device__ __forceinline__ uint32_t stable_places(SortShared& sh, const uint32_t (&digit)[kItems], uint32_t (&place)[kItems],
                                                  uint32_t batches, uint32_t digits, int bits, Begins begins) {
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pitch = (digits + 1) & ~1u;
    uint32_t* words = reinterpret_cast<uint32_t*>(sh.count);
    for (uint32_t i = tid; i < kSortWaves * pitch / 2; i += kSortThreads) words[i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kItems; ++j)
        if (digit[j] != kNone) atomicAdd(words + (wave * pitch + digit[j]) / 2, (digit[j] & 1) ? 1u << 16 : 1u);
    __syncthreads();
    const uint32_t each = (digits + kSortThreads - 1) / kSortThreads, first = tid * each;
    uint32_t sum = 0;
    for (uint32_t i = first; i < first + each && i < digits; ++i)
        for (uint32_t w = 0; w < kSortWaves; ++w) sum += sh.count[w * pitch + i];
    uint32_t upto = sum;                                     // inclusive over the wave
    for (int step = 1; step < 64; step <<= 1) {
        const uint32_t y = __shfl_up(upto, step);
        if ((int)lane >= step) upto += y;
    }
    if (lane == 63) sh.wave_total[wave] = upto;
    __syncthreads();
    uint32_t run = upto - sum, total = 0;
    for (uint32_t w = 0; w < kSortWaves; ++w) {
        if (w < wave) run += sh.wave_total[w];
        total += sh.wave_total[w];
    }
    for (uint32_t i = first; i < first + each && i < digits; ++i) {
        begins(i, run);
        for (uint32_t w = 0; w < kSortWaves; ++w) {
            const uint32_t n = sh.count[w * pitch + i];
            sh.count[w * pitch + i] = (uint16_t)run;         // (below 16384, the last ones at most 16384)
            run += n;
        }
    }
    __syncthreads();
    volatile uint16_t* next = sh.count + wave * pitch;       // (this wave's alone: its LDS accesses keep their order)
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        if ((uint32_t)j >= batches) break;
        const bool there = digit[j] != kNone;
        uint64_t same = __ballot(there);
        for (int b = 0; b < bits; ++b) {
            const uint64_t ones = __ballot((digit[j] >> b) & 1);
            same &= ((digit[j] >> b) & 1) ? ones : ~ones;
        }
        const uint32_t before = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0u));
        place[j] = kNone;
        if (there) {
            place[j] = next[digit[j]] + before;
            if (before == 0) next[digit[j]] = (uint16_t)(place[j] + __popcll(same));
        }
        __builtin_amdgcn_wave_barrier();
    }
    return total;
}

__global__ __launch_bounds__(kSortThreads) void sort_tokens_kernel(const int32_t* __restrict__ ids, uint32_t rows, int vocab,
                                                                   int32_t ignore_id, uint32_t buckets, uint32_t bucket_rows,
                                                                   int bucket_bits, int row_bits, uint32_t* __restrict__ begin,
                                                                   Entry* __restrict__ entries) {
    __shared__ SortShared sh;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t base = blockIdx.x * (uint32_t)kSegment, n = rows - base < kSegment ? rows - base : kSegment;
    ids += base;
    begin += (uint64_t)blockIdx.x * (buckets + 1);
    entries += base;
    uint32_t digit[kItems], place[kItems];
    uint32_t batches = (n + kSortThreads - 1) / kSortThreads;
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        const uint32_t t = (wave * batches + j) * 64 + lane;
        digit[j] = kNone;
        if ((uint32_t)j < batches && t < n) {
            const int32_t id = ids[t];
            if (ignore_id < 0 || id != ignore_id) digit[j] = (uint32_t)row_of(id, vocab) / buckets;
        }
    }
    const uint32_t m = stable_places(sh, digit, place, batches, bucket_rows, row_bits, [](uint32_t, uint32_t) {});
#pragma unroll
    for (int j = 0; j < kItems; ++j)
        if ((uint32_t)j < batches && place[j] != kNone) sh.order[place[j]] = (uint16_t)((wave * batches + j) * 64 + lane);
    __syncthreads();
    batches = (m + kSortThreads - 1) / kSortThreads;
    uint32_t token[kItems], key[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        const uint32_t i = (wave * batches + j) * 64 + lane;
        digit[j] = kNone;
        if ((uint32_t)j < batches && i < m) {
            token[j] = sh.order[i];
            const uint32_t v = (uint32_t)row_of(ids[token[j]], vocab);
            digit[j] = v % buckets;
            key[j] = digit[j] * bucket_rows + v / buckets;
        }
    }
    const uint32_t all = stable_places(sh, digit, place, batches, buckets, bucket_bits,
                                       [&](uint32_t bucket, uint32_t at) { begin[bucket] = at; });
    if (tid == 0) begin[buckets] = all;
#pragma unroll
    for (int j = 0; j < kItems; ++j)
        if ((uint32_t)j < batches && place[j] != kNone) entries[place[j]] = Entry{base + token[j], key[j]};
}

// ---------------------------------------------------------------- gradient: sums
//
// A wave takes one bucket's rows in one span of columns.  A lane has VEC consecutive columns: four, or one where the table
// is narrow.

// The lane's columns of a slice.  The last vector of a row whose length is no multiple of four holds fewer: it is read as the
// four elements that end with the row (`back` elements earlier), and its elements are brought to the front.
template <int VEC>
struct Columns {
    int col, n, back;
    __device__ __forceinline__ Columns(int d, int slice, int slices, int lane) {
        const int vecs = (d + VEC - 1) / VEC, each = (vecs + slices - 1) / slices, at = slice * each + lane;
        const bool mine = lane < each && at < vecs;
        col = at * VEC;
        n = mine ? (d - col < VEC ? d - col : VEC) : 0;
        back = mine ? VEC - n : 0;
    }
};
template <int VEC>
struct Sums {
    float v[VEC];
};
template <int VEC, class G>
__device__ __forceinline__ Sums<VEC> load_grad(const G* grad, uint64_t token, int d, const Columns<VEC>& at) {
    Sums<VEC> s;
    if constexpr (VEC == 4) {
        const float4 x = widened(stream_load4(grad + token * (uint64_t)d + at.col - at.back));
        s.v[0] = x.x; s.v[1] = x.y; s.v[2] = x.z; s.v[3] = x.w;
    } else {
        s.v[0] = widened(grad[token * (uint64_t)d + at.col]);
    }
    return s;
}
template <int VEC>
__device__ __forceinline__ void add(Sums<VEC>& a, const Sums<VEC>& b) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) a.v[j] += b.v[j];
}

constexpr int kBatch = 16;               // rows of grad_out in flight

// Windows of the sorted order that lie inside one row's run: their sums, so that a frequent token's run is not left to one wave.
template <int VEC, class G>
__global__ __launch_bounds__(64) void window_sums_kernel(const G* __restrict__ grad, const uint32_t* __restrict__ begin,
                                                         const Entry* __restrict__ entries, uint32_t buckets, int d, int slices,
                                                         float* __restrict__ partial) {
    const uint32_t window = blockIdx.x, segment = window / (kSegment / kWindow);
    const uint32_t first = window * kWindow, last = first + kWindow - 1;
    if (last - segment * kSegment >= begin[(uint64_t)segment * (buckets + 1) + buckets]) return;
    if (entries[first].key != entries[last].key) return;
    const Columns<VEC> at(d, blockIdx.y, slices, threadIdx.x);
    if (at.n == 0) return;
    Sums<VEC> sum = {};
    for (int e = 0; e < kWindow; e += kBatch) {
        Sums<VEC> x[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) x[k] = load_grad<VEC>(grad, entries[first + e + k].token, d, at);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) add(sum, x[k]);
    }
    float* to = partial + (uint64_t)window * slices * 64 * VEC + ((uint64_t)blockIdx.y * 64 + threadIdx.x) * VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j) to[j] = sum.v[j];
}

// Writes a row's columns: scale * sum, added to what is there if asked to.
template <int VEC, class O>
__device__ __forceinline__ void store_row(O* out, const Columns<VEC>& at, Sums<VEC> s, float scale, bool accumulate) {
    if constexpr (VEC == 4) {
        if (at.back & 1) { s.v[0] = s.v[1]; s.v[1] = s.v[2]; s.v[2] = s.v[3]; }
        if (at.back & 2) { s.v[0] = s.v[2]; s.v[1] = s.v[3]; }
        float4 x = make_float4(s.v[0] * scale, s.v[1] * scale, s.v[2] * scale, s.v[3] * scale);
        if (accumulate) {
            const float4 was = load_some(out + at.col, at.n);
            x = make_float4(was.x + x.x, was.y + x.y, was.z + x.z, was.w + x.w);
        }
        store_some(out + at.col, at.n, x);
    } else {
        store1(out + at.col, accumulate ? widened(out[at.col]) + s.v[0] * scale : s.v[0] * scale);
    }
}

template <int VEC, bool MANY, class G, class O>
__global__ __launch_bounds__(64) void row_sums_kernel(const G* __restrict__ grad, const uint32_t* __restrict__ begin,
                                                      const Entry* __restrict__ entries, const float* __restrict__ partial,
                                                      uint32_t segments, uint32_t buckets, uint32_t bucket_rows, int vocab, int d,
                                                      int slices, float scale, bool accumulate, O* __restrict__ out) {
    extern __shared__ float held[];                          // MANY: [row in the bucket][VEC][64]
    const uint32_t bucket = blockIdx.x / (uint32_t)slices, slice = blockIdx.x % (uint32_t)slices, lane = threadIdx.x;
    const Columns<VEC> at(d, (int)slice, slices, (int)lane);
    if (at.n == 0) return;
    uint64_t touched[kMaxBucketRows / 64] = {};
    uint32_t row = kNone, next = 0;                          // the run that `sum` belongs to; first row not yet written
    Sums<VEC> sum = {};
    auto out_row = [&](uint32_t r) { return out + ((uint64_t)r * buckets + bucket) * (uint64_t)d; };
    auto empty_rows = [&](uint32_t upto) {                   // rows next .. upto - 1 got nothing
        if (!accumulate)
            for (uint32_t r = next; r < upto && (uint64_t)r * buckets + bucket < (uint64_t)vocab; ++r)
                store_row<VEC>(out_row(r), at, Sums<VEC>{}, 0.f, false);
    };
    auto done = [&]() {                                      // the run ends
        if (row == kNone) return;
        if constexpr (MANY) {
            const bool more = (touched[row / 64] >> (row % 64)) & 1;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float* h = held + (row * VEC + j) * 64 + lane;
                *h = more ? *h + sum.v[j] : sum.v[j];
            }
            touched[row / 64] |= 1ull << (row % 64);
        } else {
            empty_rows(row);
            store_row<VEC>(out_row(row), at, sum, scale, accumulate);
            next = row + 1;
        }
    };
    for (uint32_t segment = 0; segment < segments; ++segment) {
        const uint32_t* b = begin + (uint64_t)segment * (buckets + 1) + bucket;
        const uint32_t origin = segment * kSegment, end = origin + b[1];
        uint32_t e = origin + b[0];
        row = kNone;
        while (e < end) {
            const uint32_t r = entries[e].key - bucket * bucket_rows;
            if (partial && e % kWindow == 0 && e + kWindow <= end && entries[e + kWindow - 1].key == entries[e].key) {
                const float* from = partial + (uint64_t)(e / kWindow) * slices * 64 * VEC + ((uint64_t)slice * 64 + lane) * VEC;
                Sums<VEC> x;
#pragma unroll
                for (int j = 0; j < VEC; ++j) x.v[j] = from[j];
                if (r == row) {
                    add(sum, x);
                } else {
                    done();
                    row = r;
                    sum = x;
                }
                e += kWindow;
                continue;
            }
            const uint32_t n = kBatch - e % kBatch < end - e ? kBatch - e % kBatch : end - e;
            Sums<VEC> x[kBatch];
            uint32_t rows[kBatch];
#pragma unroll
            for (uint32_t k = 0; k < kBatch; ++k) {
                const Entry entry = entries[e + (k < n ? k : n - 1)];
                rows[k] = entry.key - bucket * bucket_rows;
                x[k] = load_grad<VEC>(grad, entry.token, d, at);
            }
#pragma unroll
            for (uint32_t k = 0; k < kBatch; ++k) {
                if (k >= n) break;
                if (rows[k] == row) {
                    add(sum, x[k]);
                } else {
                    done();
                    row = rows[k];
                    sum = x[k];
                }
            }
            e += n;
        }
        done();
    }
    if constexpr (MANY) {
        for (uint32_t r = 0; r < bucket_rows && (uint64_t)r * buckets + bucket < (uint64_t)vocab; ++r) {
            Sums<VEC> s = {};
            const bool some = (touched[r / 64] >> (r % 64)) & 1;
            if (!some && accumulate) continue;
            if (some)
#pragma unroll
                for (int j = 0; j < VEC; ++j) s.v[j] = held[(r * VEC + j) * 64 + lane];
            store_row<VEC>(out_row(r), at, s, scale, accumulate);
        }
    } else {
        empty_rows(bucket_rows);
    }
}

// ---------------------------------------------------------------- host side

int bits_of(uint32_t values) {           // bits that tell 0 .. values - 1 apart
    int bits = 0;
    while (bits < 31 && (1u << bits) < values) ++bits;
    return bits;
}

// How a table's rows are dealt to buckets.
struct Buckets {
    uint32_t rows_each, count;
    explicit Buckets(int vocab) {
        rows_each = ((uint32_t)vocab + kMaxBuckets - 1) / kMaxBuckets;
        count = ((uint32_t)vocab + rows_each - 1) / rows_each;
    }
};
constexpr int64_t kMaxVocab = (int64_t)kMaxBuckets * kMaxBucketRows;

int vec_of(int d) { return d < 256 ? 1 : 4; }
int slices_of(int d) { return ((d + vec_of(d) - 1) / vec_of(d) + 63) / 64; }

// The workspace: where every segment's buckets begin, the entries, the windows' sums.
struct GradSpace {
    int64_t segments, begin, entries, partial, bytes;
    GradSpace(int64_t rows, int vocab, int d) {
        const Buckets b(vocab);
        segments = (rows + kSegment - 1) / kSegment;
        begin = 0;
        entries = (segments * (b.count + 1) * 4 + 255) / 256 * 256;
        partial = entries + (rows * (int64_t)sizeof(Entry) + 255) / 256 * 256;
        bytes = partial + segments * (kSegment / kWindow) * slices_of(d) * 64 * vec_of(d) * 4;
    }
};

bool grad_sizes_fit(int64_t rows, int vocab, int d) {
    return rows >= 0 && rows < (int64_t)1 << 31 && vocab >= 1 && vocab <= kMaxVocab && d >= 1 && d < 1 << 24;
}

}  // namespace

extern "C" {

int sparseloco_embedding_lookup(const void* table, const void* t_perp, int table_dtype, const int32_t* token_ids, int vocab,
                                const void* pos_embed, int seq_len, float scale, void* out, int out_dtype, int64_t rows, int d,
                                void* stream) {
    if (!table || (rows > 0 && (!token_ids || !out)) || vocab < 1 || rows < 0 || rows >= (int64_t)1 << 31 || d < 1 || d >= 1 << 24 ||
        !finite(scale) || (pos_embed && seq_len < 1))
        return SPLC_EINVAL;
    for (int dtype : {table_dtype, out_dtype})
        if (dtype != SPLC_F32 && dtype != SPLC_BF16) return SPLC_EINVAL;
    const size_t in = table_dtype == SPLC_BF16 ? 2 : 4;
    if (!aligned(table, in) || !aligned(t_perp, in) || !aligned(pos_embed, in) || !aligned(token_ids, 4) ||
        !aligned(out, out_dtype == SPLC_BF16 ? 2 : 4))
        return SPLC_EALIGN;
    if (rows == 0) return SPLC_OK;
    const dim3 grid((unsigned)((rows + 3) / 4), (unsigned)((d + kLookupSpan - 1) / kLookupSpan));
    auto launch = [&](auto element, auto result) {
        using T = decltype(element);
        using O = decltype(result);
        hipLaunchKernelGGL((lookup_kernel<T, O>), grid, dim3(256), 0, static_cast<hipStream_t>(stream),
                           static_cast<const T*>(table), static_cast<const T*>(t_perp), token_ids, vocab,
                           static_cast<const T*>(pos_embed), seq_len, scale, static_cast<O*>(out), rows, d);
    };
    if (table_dtype == SPLC_F32 && out_dtype == SPLC_F32) launch(float{}, float{});
    else if (table_dtype == SPLC_F32) launch(float{}, uint16_t{});
    else if (out_dtype == SPLC_F32) launch(uint16_t{}, float{});
    else launch(uint16_t{}, uint16_t{});
    return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
}

int64_t sparseloco_embedding_grad_ws_bytes(int64_t rows, int vocab, int d) {
    if (!grad_sizes_fit(rows, vocab, d)) return SPLC_EINVAL;
    return GradSpace(rows, vocab, d).bytes;
}

int sparseloco_embedding_grad(const void* grad_out, int grad_dtype, const int32_t* token_ids, int64_t rows, int vocab, int d,
                              float scale, int32_t ignore_id, void* grad_table, int table_dtype, int accumulate, void* ws,
                              int64_t ws_bytes, void* stream) {
    if (!grad_sizes_fit(rows, vocab, d) || !grad_table || !finite(scale)) return SPLC_EINVAL;
    if (rows > 0 && (!grad_out || !token_ids || !ws)) return SPLC_EINVAL;
    for (int dtype : {grad_dtype, table_dtype})
        if (dtype != SPLC_F32 && dtype != SPLC_BF16) return SPLC_EINVAL;
    if (!aligned(grad_out, grad_dtype == SPLC_BF16 ? 2 : 4) || !aligned(grad_table, table_dtype == SPLC_BF16 ? 2 : 4) ||
        !aligned(token_ids, 4) || !aligned(ws, 8))
        return SPLC_EALIGN;
    const GradSpace space(rows, vocab, d);
    if (ws_bytes < space.bytes) return SPLC_EINVAL;
    const Buckets b(vocab);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    char* at = static_cast<char*>(ws);
    uint32_t* begin = reinterpret_cast<uint32_t*>(at + space.begin);
    Entry* entries = reinterpret_cast<Entry*>(at + space.entries);
    float* partial = reinterpret_cast<float*>(at + space.partial);
    const int slices = slices_of(d);
    const uint32_t segments = (uint32_t)space.segments;
    if (segments > 0)
        hipLaunchKernelGGL(sort_tokens_kernel, dim3(segments), dim3(kSortThreads), 0, st, token_ids, (uint32_t)rows, vocab, ignore_id,
                           b.count, b.rows_each, bits_of(b.count), bits_of(b.rows_each), begin, entries);
    const bool windows = rows >= 2048;
    auto launch = [&](auto vec, auto gradient, auto result) {
        constexpr int VEC = decltype(vec)::value;
        using G = decltype(gradient);
        using O = decltype(result);
        if (windows)
            hipLaunchKernelGGL((window_sums_kernel<VEC, G>), dim3((unsigned)(rows / kWindow), (unsigned)slices), dim3(64), 0, st,
                               static_cast<const G*>(grad_out), begin, entries, b.count, d, slices, partial);
        const dim3 grid((unsigned)(b.count * (uint32_t)slices));
        if (segments > 1)
            hipLaunchKernelGGL((row_sums_kernel<VEC, true, G, O>), grid, dim3(64), b.rows_each * VEC * 64 * sizeof(float), st,
                               static_cast<const G*>(grad_out), begin, entries, windows ? partial : nullptr, segments, b.count,
                               b.rows_each, vocab, d, slices, scale, accumulate != 0, static_cast<O*>(grad_table));
        else
            hipLaunchKernelGGL((row_sums_kernel<VEC, false, G, O>), grid, dim3(64), 0, st, static_cast<const G*>(grad_out), begin,
                               entries, windows ? partial : nullptr, segments, b.count, b.rows_each, vocab, d, slices, scale,
                               accumulate != 0, static_cast<O*>(grad_table));
    };
    auto by_type = [&](auto vec) {
        if (grad_dtype == SPLC_F32 && table_dtype == SPLC_F32) launch(vec, float{}, float{});
        else if (grad_dtype == SPLC_F32) launch(vec, float{}, uint16_t{});
        else if (table_dtype == SPLC_F32) launch(vec, uint16_t{}, float{});
        else launch(vec, uint16_t{}, uint16_t{});
    };
    if (vec_of(d) == 4) by_type(std::integral_constant<int, 4>{});
    else by_type(std::integral_constant<int, 1>{});
    return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
}

}  // extern "C"
