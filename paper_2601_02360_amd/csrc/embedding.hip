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

__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = (uint16_t)bf16_pair(v, v); }
// The last n of v's elements at p.
template <class T>
__device__ __forceinline__ void store_last(T* p, int n, float4 v) {
    if (n == 4) {
        stream_store4(p, v);
        return;
    }
    if (n == 3) store1(p + n - 3, v.y);
    if (n > 1) store1(p + n - 2, v.z);
    store1(p + n - 1, v.w);
}
__device__ __forceinline__ float4 plus(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ int row_of(int32_t id, int vocab) { return max(0, min(id, vocab - 1)); }

// ---------------------------------------------------------------- lookup

constexpr int64_t kMostTurns = 1 << 20;  // (a launch has fewer than 2^32 lanes)

// Bound by memory: rows of the table in the order of the tokens, and out.  A wave takes ROWS tokens in one span of columns, and two
// to four vectors of every array are in flight: two of one row, or, of spans of at most 256 columns, one of four (65536 tokens of
// 50304, d 256, bf16: 15.4 -> 11.7 us; d 150, fp32, two tables: 18.0 -> 14.3).
// Workgroups go to the eight XCDs round-robin by number, and spans go with them: with four spans an XCD's L2 is asked for one fourth of
// every table row and of PosEmbed, and holds four times as many of them.  But a span is 1.25 to 2.5 KB of a row where there are several
// (more in rows above 20 KB: there are eight at most), since waves that read less of it at once wait longer than they read.  MI355X, 16384 tokens of 32000, tables that no cache holds, both
// fp32 tables and positions to bf16: d 2048 in 1 / 2 / 4 / 8 spans 44.2 / 41.6 / 40.1 / 41.4 us (165 MB that cannot be done without, 4.1
// TB/s; a copy reaches 4.8), d 4096 in 4 / 8 96 / 91; 60000 of d 672, bf16, in 1 / 4 22.9 / 38.4; spans of 1 to 2 KB: d 2050, bf16, 23.9
// for 20.3.  out without the streaming hint: 45.0 instead of 40.1.
// NARROW: rows of at most 128 columns, of which a wave takes as many at once as it has `lanes` lanes for (22817 tokens, d 106: 8.0 -> 5.5
// us; 65536, d 64: 18.9 -> 6.4, and 4.7 with four times as many).
template <bool NARROW, int ROWS, class T, class O>
__global__ __launch_bounds__(256) void lookup_kernel(const T* __restrict__ table, const T* __restrict__ t_perp,
                                                     const int32_t* __restrict__ ids, int vocab, const T* __restrict__ pos,
                                                     int seq, float scale, O* __restrict__ out, int64_t rows, int d, int spans,
                                                     int width, int lanes) {
    constexpr int COLS = ROWS == 1 ? 2 : 1;                  // vectors of a row at once
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = NARROW ? threadIdx.x % lanes : threadIdx.x & 63;
    const int at_once = (NARROW ? 256 / lanes : 4) * ROWS;   // rows a workgroup takes at once
    const int span = (int)(blockIdx.x % (unsigned)spans);
    const int end = (span + 1) * width < d ? (span + 1) * width : d;
    for (int64_t row = (int64_t)(blockIdx.x / (unsigned)spans) * at_once + (NARROW ? (int)threadIdx.x / lanes : wave) * ROWS; row < rows;
         row += (int64_t)(gridDim.x / (unsigned)spans) * at_once) {
        int64_t from[ROWS];
        const T* p[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int64_t at = row + r < rows ? row + r : rows - 1;      // (the last row once more, and not written)
            from[r] = (int64_t)row_of(ids[at], vocab) * d;
            p[r] = pos ? pos + (int64_t)((uint32_t)at % (uint32_t)seq) * d : nullptr;
        }
        for (int c = span * width + lane * 4; c < end; c += 256 * COLS) {
            decltype(cached_load4(table)) x[ROWS * COLS], y[ROWS * COLS], z[ROWS * COLS];        // as they lie in memory
#pragma unroll
            for (int k = 0; k < ROWS * COLS; ++k) {
                const int at = c + 256 * (k % COLS), r = k / COLS, four = at + 4 <= d ? at : d - 4;     // (the row's last four)
                if (at >= end) continue;
                x[k] = cached_load4(table + from[r] + four);
                if (t_perp) y[k] = cached_load4(t_perp + from[r] + four);
                if (pos) z[k] = cached_load4(p[r] + four);
            }
#pragma unroll
            for (int k = 0; k < ROWS * COLS; ++k) {
                const int at = c + 256 * (k % COLS), n = d - at < 4 ? d - at : 4, r = k / COLS;
                if (at >= end || row + r >= rows) continue;
                float4 v = widened(x[k]);
                if (t_perp) v = plus(v, widened(y[k]));
                v = make_float4(v.x * scale, v.y * scale, v.z * scale, v.w * scale);
                if (pos) v = plus(v, widened(z[k]));
                store_last(out + (row + r) * d + at, n, v);
            }
        }
    }
}

// Rows of fewer than four columns: an element a lane.
template <class T, class O>
__global__ __launch_bounds__(256) void lookup_short_kernel(const T* __restrict__ table, const T* __restrict__ t_perp,
                                                           const int32_t* __restrict__ ids, int vocab, const T* __restrict__ pos,
                                                           int seq, float scale, O* __restrict__ out, int64_t rows, int d) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * d; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / d, c = i % d, at = (int64_t)row_of(ids[row], vocab) * d + c;
        float v = widened(table[at]);
        if (t_perp) v += widened(t_perp[at]);
        v *= scale;
        if (pos) v += widened(pos[(int64_t)((uint32_t)row % (uint32_t)seq) * d + c]);
        store1(out + i, v);
    }
}

// ---------------------------------------------------------------- gradient: order of the tokens
//
// Entries (table row, token) are sorted by row, equal rows by token.  A workgroup has 64 or 128 entries of a run and finds their
// places in it by looking at all others of the run; runs are kDirect long where that is all, else kRun, and up to eight at a
// time become one, every entry finding its place by itself: the number of smaller entries in each of the other runs, by binary
// search.  Tokens that are left out, and what fills the last windows, have row kNone and token 0 and come last.
//
// Where the table is written whole, its zeros are written by further workgroups of these launches, which have little else to
// do with the memory; rows that have tokens are written again later.
//
// MI355X: 64 tokens 3.1 us, 4096 at once 4.5, 16384 8.5; 65537 in runs 8.7, merged in 5.9 and 8.7, of which 4 are the launch and a chain
// of loads.  Bound by the vector ALU and LDS, which take every token through 7 (8) steps of search for every 64 (128) others of its run.

constexpr uint32_t kNone = 0x7FFFFFFFu;
constexpr int kBlock = 512;              // the number of entries is a multiple of this
// Above 64 MB of zeros the launches that write them take longer than the order, and one more has room for it: at once / in runs,
// whole call, 16384 bf16 rows of 2048 of 50304: 88.5 / 84.1 us, of 32000: 65.2 / 61.9, of 16000: 44.9 / 42.9, of 8000: 34.2 / 34.4; added
// to what is there, 43.1 / 46.
constexpr uint64_t kFewZeros = 1 << 22;  // vectors
constexpr uint32_t kRun = 2048, kDirect = 16384, kOrderThreads = 1024, kMergeThreads = 512, kFanIn = 8;

// A launch's share of the zeros: 16-byte vectors from `at`, workgroup by workgroup.
struct Zeros {
    uint4* at;
    uint64_t vectors;
};
constexpr uint32_t kZeroSpan = 512;      // vectors a workgroup writes (50304 rows of 768: 26.6 us, 1024: 28.3, 2048: 30.4, 256: 36.7)
constexpr uint32_t kMostZeroGroups = 1 << 20;
__device__ __forceinline__ void write_zeros(const Zeros& z, uint32_t group) {
    typedef uint32_t vuint4 __attribute__((ext_vector_type(4)));
    for (uint64_t from = (uint64_t)group * kZeroSpan; from < z.vectors; from += (uint64_t)kMostZeroGroups * kZeroSpan)
        for (uint32_t i = threadIdx.x; i < kZeroSpan; i += blockDim.x)
            if (from + i < z.vectors) __builtin_nontemporal_store(vuint4{0, 0, 0, 0}, (SPLC_GLOBAL vuint4*)(z.at + from + i));
}

// The order of every run of `run` entries.  A workgroup has KEYS of a run's entries, puts these in order by comparing each with each, and
// finds for every other of the run before which of them it goes, by binary search; the numbers of those add up to places.
// 64 where that gives few workgroups, 128 in runs of kRun (65537 tokens: 10.8 and 8.6 us, 256: 13.1).
constexpr uint32_t kAtOnce = 4;                              // searches of a lane side by side
constexpr uint32_t kCopies = 8;                              // of a count, by lanes: those that add to the same one wait for each other
                                                             // (one token 16384 times: 19.4 -> 7.5 us, frequencies 1 / rank 9.2 -> 8.5)
template <uint32_t KEYS, class O>
__global__ __launch_bounds__(kOrderThreads) void order_tokens_kernel(const int32_t* __restrict__ ids, uint32_t rows, int vocab,
                                                                     int32_t ignore_id, uint32_t run, uint32_t groups,
                                                                     uint32_t* __restrict__ row, uint32_t* __restrict__ token,
                                                                     Zeros zeros, O* table,
                                                                     uint64_t table_size, uint32_t head, uint32_t tail) {
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (blockIdx.x >= groups) {
        if (blockIdx.x == groups) {
            if (tid < head) table[tid] = O(0);
            if (tid < tail) table[table_size - 1 - tid] = O(0);
        }
        write_zeros(zeros, blockIdx.x - groups);
        return;
    }
    const uint32_t base = blockIdx.x * KEYS, run_from = base / run * run, run_to = rows < run_from + run ? rows : run_from + run;
    if (base >= rows) {                                      // (these only fill the last windows)
        if (tid < KEYS) {
            row[base + tid] = kNone;
            token[base + tid] = 0;
        }
        return;
    }
    auto row_named = [&](int32_t id) { return ignore_id < 0 || id != ignore_id ? (uint32_t)row_of(id, vocab) : kNone; };
    auto key = [&](uint32_t i) { return base + i < rows ? row_named(ids[base + i]) : kNone; };
    // the KEYS by 64; a wave compares 64 of them with kEach of 64
    constexpr uint32_t kSets = KEYS / 64, kWaves = kOrderThreads / 64 / kSets, kEach = KEYS / kWaves;
    static_assert(kEach <= 64 && 64 % kEach == 0 && KEYS * kCopies <= kOrderThreads, "a set's waves share the comparisons");
    __shared__ uint32_t smaller[kWaves][KEYS], sorted[KEYS], from[KEYS], before[KEYS * kCopies];
    const uint32_t set = wave % kSets, part = wave / kSets;
    const uint32_t mine = key(set * 64 + lane), others = key(part * kEach / 64 * 64 + lane);
    uint32_t j = run_from + tid;
    int32_t id[kAtOnce];
    auto load = [&]() {
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) {
            const uint32_t at = j + k * kOrderThreads;
            id[k] = ids[at < run_to ? at : run_to - 1];
        }
    };
    load();
    uint32_t count = 0;
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) {
        const uint32_t other = __builtin_amdgcn_readlane(others, part * kEach % 64 + k);
        count += other < mine || (other == mine && part * kEach + k < set * 64 + lane) ? 1 : 0;
    }
    smaller[part][set * 64 + lane] = count;
    if (tid < KEYS * kCopies) before[tid] = 0;               // how many others come just before each key
    __syncthreads();
    if (part == 0) {
        uint32_t place = 0;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) place += smaller[w][set * 64 + lane];
        sorted[place] = mine;                                // the KEYS in order,
        from[place] = set * 64 + lane;                       // and which they were
    }
    __syncthreads();
    while (j < run_to) {
        // how many of the KEYS go before it, those of rows below `limit`: four bytes for each
        uint32_t limit[kAtOnce], below[kAtOnce] = {};
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) {
            const uint32_t at = j + k * kOrderThreads;
            limit[k] = at < run_to && at / KEYS != blockIdx.x ? row_named(id[k]) + (at < base ? 0 : 1) : ~0u;      // (~0: all)
        }
        j += kAtOnce * kOrderThreads;
        if (j - tid < run_to) load();
        auto key_at = [&](uint32_t bytes) { return *reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(sorted) + bytes); };
#pragma unroll
        for (uint32_t step = KEYS / 2; step > 0; step /= 2)
#pragma unroll
            for (uint32_t k = 0; k < kAtOnce; ++k) below[k] |= key_at(below[k] + (step - 1) * 4) < limit[k] ? step * 4 : 0;
        bool before_one[kAtOnce];
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) before_one[k] = key_at(below[k]) >= limit[k];
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k)
            if (before_one[k]) atomicAdd(&before[below[k] / 4 * kCopies + lane % kCopies], 1u);
    }
    __syncthreads();
    if (wave > 0) return;
    uint32_t sums[kSets], sum = 0;                           // a lane has kSets that follow each other
#pragma unroll
    for (uint32_t k = 0; k < kSets; ++k) {
#pragma unroll
        for (uint32_t c = 0; c < kCopies; ++c) sum += before[(lane * kSets + k) * kCopies + c];
        sums[k] = sum;
    }
    uint32_t upto = sum;
    for (uint32_t step = 1; step < 64; step *= 2) {
        const uint32_t lower = __shfl_up(upto, step);
        if (lane >= step) upto += lower;
    }
#pragma unroll
    for (uint32_t k = 0; k < kSets; ++k) {
        const uint32_t i = lane * kSets + k, r = sorted[i], at = base + from[i];
        const uint32_t place = at < rows ? run_from + i + (upto - sum) + sums[k] : at;
        row[place] = r;
        token[place] = r == kNone ? 0 : at;
    }
}

// Sorted runs of `length` entries (the last one of all may be shorter), kFanIn of them at a time, to one run.  Of every run
// kSamples entries at equal distances lie in LDS for the first steps of the search; from a distance of 32 on the others are in one
// cache line.
template <uint32_t SAMPLES>
__global__ __launch_bounds__(kMergeThreads) void merge_runs_kernel(const uint32_t* __restrict__ row, const uint32_t* __restrict__ token,
                                                                   uint32_t entries, uint32_t length, uint32_t* __restrict__ row_out,
                                                                   uint32_t* __restrict__ token_out, uint32_t groups, Zeros zeros) {
    if (blockIdx.x >= groups) {
        write_zeros(zeros, blockIdx.x - groups);
        return;
    }
    __shared__ uint32_t sample[kFanIn * SAMPLES];           // the last entry of each stretch
    static_assert(kBlock % kMergeThreads == 0 && kRun % kMergeThreads == 0, "whole workgroups");
    const uint32_t i = blockIdx.x * kMergeThreads + threadIdx.x;
    const uint32_t run = blockIdx.x * kMergeThreads / length, first = run / kFanIn * kFanIn, stretch = length / SAMPLES;
    uint32_t some[kFanIn * SAMPLES / kMergeThreads];
#pragma unroll
    for (uint32_t s = 0; s < kFanIn * SAMPLES / kMergeThreads; ++s) {
        const uint64_t at = (uint64_t)first * length + (uint64_t)(s * kMergeThreads + threadIdx.x + 1) * stretch - 1;
        some[s] = at < entries ? row[at] : kNone;
    }
    const uint32_t r = row[i], t = token[i];
#pragma unroll
    for (uint32_t s = 0; s < kFanIn * SAMPLES / kMergeThreads; ++s) sample[s * kMergeThreads + threadIdx.x] = some[s];
    __syncthreads();
    uint32_t below[kFanIn] = {};                             // entries that go before this one; the searches go side by side
    uint32_t limit[kFanIn];                                  // those of rows below it; of equal rows earlier runs' entries do
#pragma unroll
    for (uint32_t k = 0; k < kFanIn; ++k) limit[k] = first + k < run ? r + 1 : r;
#pragma unroll
    for (uint32_t step = SAMPLES / 2; step > 0; step /= 2)
#pragma unroll
        for (uint32_t k = 0; k < kFanIn; ++k) below[k] += sample[k * SAMPLES + step - 1 + below[k]] < limit[k] ? step : 0;
    // (all stretches but the last at most are counted: whether that one goes before is for what follows to find)
    if (stretch == 1) {
#pragma unroll
        for (uint32_t k = 0; k < kFanIn; ++k) below[k] += sample[k * SAMPLES + below[k]] < limit[k] ? 1 : 0;
    } else {
#pragma unroll
        for (uint32_t k = 0; k < kFanIn; ++k) below[k] *= stretch;
        for (uint32_t step = stretch; step > 0; step /= 2) {
            uint32_t seen[kFanIn];
            bool inside[kFanIn];
#pragma unroll
            for (uint32_t k = 0; k < kFanIn; ++k) {
                const uint64_t at = (uint64_t)(first + k) * length + below[k] + step - 1;
                inside[k] = below[k] + step <= length && at < entries;
                seen[k] = inside[k] ? row[at] : kNone;
            }
#pragma unroll
            for (uint32_t k = 0; k < kFanIn; ++k)
                below[k] += inside[k] && seen[k] < limit[k] ? step : 0;
        }
    }
    uint32_t place = first * length + (i - run * length);
#pragma unroll
    for (uint32_t k = 0; k < kFanIn; ++k) place += first + k == run ? 0 : below[k];
    row_out[place] = r;
    token_out[place] = t;
}

// ---------------------------------------------------------------- gradient: sums
//
// Sums are kept in registers: grad_out is read once, in rows, and every row of the table is written once, by one wave.  A lane has
// VEC consecutive columns: four, or one where the table is narrow.  Windows that lie inside one run are summed first, where there
// are many tokens, so that a frequent token's run is not left to few waves (one that makes up 7 % of 65537: 69 windows instead of 4400
// rows).  Bound by memory: MI355X, 65537 fp32 rows of 2050 into 32001 rows, frequencies 1 / rank, added to what is there: windows 34 us
// (4.9 TB/s), runs 120 us (4.7 TB/s); 16384 bf16 rows of 2048: runs 24 us (18 where caches hold part).  One token throughout: 92 and 33 us, 20 (with
// zeros) and 10 us.  Small calls wait: 4096 bf16 rows of 1792 of 388, 11 us.  grad_out is read without the streaming hint, which loses
// lines that two slices share (65537 rows of few different tokens: 180 us with it, 128).

// The lane's columns of a slice.  The last vector of a row whose length is no multiple of four holds fewer: it is read as the
// four elements that end with the row (`back` elements earlier), of which the last ones are the lane's.
template <int VEC>
struct Columns {
    int col, n, back;
    __device__ __forceinline__ Columns(int d, int slice, int slices, int lane) {
        const int vecs = (d + VEC - 1) / VEC, each = (vecs + slices - 1) / slices, at = slice * each + lane;
        const bool mine = lane < each && at < vecs;
        col = mine ? at * VEC : 0;                           // (a lane without columns reads the first and writes nothing)
        n = mine ? (d - col < VEC ? d - col : VEC) : 0;
        back = mine ? VEC - n : 0;
    }
};
// Which window (their number is a multiple of eight) and which slice of its columns a workgroup takes: those of the same rows
// follow each other on one XCD, so that lines which two slices share meet in one L2.
struct Unit {
    uint32_t window, slice;
    __device__ __forceinline__ Unit(uint32_t group, uint32_t slices) {
        const uint32_t place = group / 8;
        window = place / slices * 8 + group % 8;
        slice = place % slices;
    }
};
// Up to so many entries a long run is left to the waves of a workgroup, without windows' sums.  Without / with them, whole call: 2415
// bf16 rows of 1792 of 388: 12.6 / 13.7 us, 4096 of 2048 of 32000: 47.4 / 49.1, 4096 fp32 rows of 2048 of 700: 16.8 / 19.3 (one token
// throughout: 59.5 / 19.6); 5135 fp32 rows of 448 of 258: 18.5 / 15.4, 8192 of 512 of 1000: 21.6 / 16.2, 8192 bf16 rows of 2048 of 32000:
// 55.1 / 52.9.
constexpr uint32_t kFewEntries = 4096;
template <int VEC>
struct Sums {
    float v[VEC];
};
template <int VEC, class G>
__device__ __forceinline__ Sums<VEC> load_grad(const G* grad, uint64_t token, int d, const Columns<VEC>& at) {
    Sums<VEC> s;
    if constexpr (VEC == 4) {
        const float4 x = widened(cached_load4(grad + token * (uint64_t)d + at.col - at.back));
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

constexpr int kWindow = 64;              // entries of a workgroup, one a lane; and those that one partial sum covers
constexpr int kPiece = 8;                // of which a wave has so many: rows in flight (16: 2415 bf16 rows of 1792, 21.2 for 19.5 us)
constexpr int kSumWaves = kWindow / kPiece;
constexpr int kFlight = 16;              // rows in flight where a wave has little else to hold
static_assert(kWindow == 64 && kBlock % (8 * kWindow) == 0, "windows in eights");

// Windows of entries that lie inside one run: their sums, so that a frequent token's run is not left to one wave.
template <int VEC, class G>
__global__ __launch_bounds__(kWindow / kFlight * 64) void window_sums_kernel(const G* __restrict__ grad, const uint32_t* __restrict__ row,
                                                         const uint32_t* __restrict__ token, int d, int slices,
                                                         float* __restrict__ partial, uint32_t groups, Zeros zeros) {
    if (blockIdx.x >= groups) {
        write_zeros(zeros, blockIdx.x - groups);
        return;
    }
    constexpr uint32_t kWaves = kWindow / kFlight;
    __shared__ float parts[kWaves - 1][VEC][64];
    const Unit unit(blockIdx.x, (uint32_t)slices);
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = unit.window * kWindow;
    if (row[first] != row[first + kWindow - 1] || row[first] == kNone) return;
    const Columns<VEC> at(d, (int)unit.slice, slices, (int)lane);
    Sums<VEC> x[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) x[k] = load_grad<VEC>(grad, token[first + wave * kFlight + k], d, at);
#pragma unroll
    for (int k = 1; k < kFlight; ++k) add(x[0], x[k]);
#pragma unroll
    for (int j = 0; j < VEC; ++j)
        if (wave > 0) parts[wave - 1][j][lane] = x[0].v[j];
    __syncthreads();
    if (wave > 0) return;
    float* to = partial + (((uint64_t)unit.window * slices + unit.slice) * 64 + lane) * VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        for (uint32_t w = 0; w < kWaves - 1; ++w) x[0].v[j] += parts[w][j][lane];
        to[j] = x[0].v[j];
    }
}

// Writes a row's columns: scale * sum, added to what is there if asked to.
template <int VEC, class O>
__device__ __forceinline__ void store_row(O* out, const Columns<VEC>& at, Sums<VEC> s, float scale, const Sums<VEC>* was) {
    if constexpr (VEC == 4) {
        float4 x = make_float4(s.v[0] * scale, s.v[1] * scale, s.v[2] * scale, s.v[3] * scale);
        if (was) x = plus(make_float4(was->v[0], was->v[1], was->v[2], was->v[3]), x);
        store_last(out + at.col, at.n, x);
    } else {
        store1(out + at.col, was ? was->v[0] + s.v[0] * scale : s.v[0] * scale);
    }
}
template <int VEC, class O>
__device__ __forceinline__ Sums<VEC> load_row(const O* out, const Columns<VEC>& at) {
    Sums<VEC> s;
    if constexpr (VEC == 4) {
        const float4 x = widened(stream_load4(out + at.col - at.back));
        s.v[0] = x.x; s.v[1] = x.y; s.v[2] = x.z; s.v[3] = x.w;
    } else {
        s.v[0] = widened(out[at.col]);
    }
    return s;
}

// A workgroup takes one window in one span of columns, each of its waves a piece, of which every entry's row of grad_out is read once.
// Runs that begin and end inside a piece are written at once.  A piece's wave has, besides, the sum of its last run so far and that of
// the entries at its front which belong to a run from an earlier piece: the latter go through LDS to the wave in whose piece
// that run begins.  The one run that may leave the window is followed by all waves in turn: MANY: by whole windows' sums, else, and
// in its last window, in pieces; their parts go the same way.
template <int VEC, bool ADDED, bool MANY, class G, class O>
__global__ __launch_bounds__(kSumWaves * 64) void row_sums_kernel(const G* __restrict__ grad, const uint32_t* __restrict__ row,
                                                     const uint32_t* __restrict__ token, const float* __restrict__ partial,
                                                     uint32_t entries, int d, int slices, float scale, O* __restrict__ out) {
    __shared__ float parts[2][kSumWaves][VEC][64];
    const Unit unit(blockIdx.x, (uint32_t)slices);
    const uint32_t slice = unit.slice;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t e = unit.window * kWindow, q = wave * kPiece;  // the window's first entry, and the piece's in it
    const uint32_t rows = row[e + lane], tokens = token[e + lane];               // an entry a lane
    const uint32_t previous = e > 0 ? row[e - 1] : kNone, next = e + kWindow < entries ? row[e + kWindow] : kNone;
    const uint32_t leaving = __builtin_amdgcn_readlane(rows, kWindow - 1);
    if (__builtin_amdgcn_readlane(rows, 0) == kNone || (e > 0 && leaving == previous)) return;     // nothing begins here
    const Columns<VEC> at(d, (int)slice, slices, (int)lane);
    auto out_row = [&](uint32_t r) { return out + (uint64_t)r * (uint64_t)d; };

    uint32_t r[kPiece];
#pragma unroll
    for (uint32_t i = 0; i < kPiece; ++i) r[i] = __builtin_amdgcn_readlane(rows, q + i);
    const uint32_t before = q > 0 ? __builtin_amdgcn_readlane(rows, q - 1) : previous, last = r[kPiece - 1];
    const bool from_before = q + e > 0;
    const bool mine = last != kNone && !(from_before && last == before);         // the last run begins in this piece
    Sums<VEC> sum = {}, head = {};
    if (r[0] != kNone && !(e > 0 && last == previous)) {
        Sums<VEC> x[kPiece];
#pragma unroll
        for (uint32_t i = 0; i < kPiece; ++i) x[i] = load_grad<VEC>(grad, __builtin_amdgcn_readlane(tokens, q + i), d, at);
        // x becomes the sums of the runs up to here
#pragma unroll
        for (uint32_t i = 1; i < kPiece; ++i)
            if (r[i] == r[i - 1]) {
                Sums<VEC> upto = x[i - 1];
                add(upto, x[i]);
                x[i] = upto;
            }
#pragma unroll
        for (uint32_t i = 0; i < kPiece; ++i)
            if (r[i] == before) head = x[i];
        auto written = [&](uint32_t i) { return r[i] != r[i + 1] && r[i] != kNone && !(from_before && r[i] == before); };
        if (at.n > 0)
#pragma unroll
            for (uint32_t half = 0; half < kPiece; half += kPiece / 2) {
                Sums<VEC> was[kPiece / 2];
#pragma unroll
                for (uint32_t i = 0; i < kPiece / 2; ++i)
                    if (ADDED && half + i + 1 < kPiece && written(half + i)) was[i] = load_row<VEC>(out_row(r[half + i]), at);
#pragma unroll
                for (uint32_t i = 0; i < kPiece / 2; ++i)
                    if (half + i + 1 < kPiece && written(half + i))
                        store_row<VEC>(out_row(r[half + i]), at, x[half + i], scale, ADDED ? &was[i] : nullptr);
            }
        sum = x[kPiece - 1];
    }
    const bool shared = leaving != kNone && next == leaving; // (its run begins in this window)
    Sums<VEC> part = {};
    if (shared) {
        uint32_t from = e + kWindow, stop = from, n;
        do {                                                 // windows that begin with it
            const uint32_t w = stop + lane * kWindow;
            const uint64_t others = __ballot(w >= entries || row[w] != leaving);
            n = others == 0 ? 64 : (uint32_t)__builtin_ctzll(others);
            stop += n * kWindow;
        } while (n == 64);
        const uint64_t others = __ballot(row[stop - kWindow + lane] != leaving);
        if (others != 0) stop -= kWindow - (uint32_t)__builtin_ctzll(others);
        if constexpr (MANY) {
            const uint32_t whole = (stop - from) / kWindow;
            for (uint32_t b = wave; b < whole; b += kPiece * kSumWaves) {
                Sums<VEC> x[kPiece];
#pragma unroll
                for (uint32_t i = 0; i < kPiece; ++i) {
                    const uint32_t w = b + i * kSumWaves < whole ? b + i * kSumWaves : whole - 1;
                    const float* of = partial + (((uint64_t)(from / kWindow + w) * slices + slice) * 64 + lane) * VEC;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) x[i].v[j] = of[j];
                }
#pragma unroll
                for (uint32_t i = 0; i < kPiece; ++i)
                    if (b + i * kSumWaves < whole) add(part, x[i]);
            }
            from += whole * kWindow;
        }
        // a wave takes every so manieth piece of kRows entries, and has the tokens of some at a time in its lanes
        constexpr uint32_t kRows = MANY ? kPiece : kFlight, kRound = kRows * kSumWaves;
        for (uint32_t b = from + wave * kRows; b < stop; b += 64 / kRows * kRound) {
            const uint32_t entry = b + lane / kRows * kRound + lane % kRows;
            const uint32_t its = token[entry < stop ? entry : stop - 1];
#pragma unroll 1
            for (uint32_t k = 0; k < 64 / kRows && b + k * kRound < stop; ++k) {
                Sums<VEC> x[kRows];
#pragma unroll
                for (uint32_t i = 0; i < kRows; ++i) x[i] = load_grad<VEC>(grad, __builtin_amdgcn_readlane(its, k * kRows + i), d, at);
#pragma unroll
                for (uint32_t i = 0; i < kRows; ++i)
                    if (b + k * kRound + i < stop) add(part, x[i]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        parts[0][wave][j][lane] = head.v[j];
        if (shared) parts[1][wave][j][lane] = part.v[j];
    }
    __syncthreads();
    if (!mine || at.n == 0) return;
    auto add_part = [&](uint32_t which, uint32_t w) {
        Sums<VEC> x;
#pragma unroll
        for (int j = 0; j < VEC; ++j) x.v[j] = parts[which][w][j][lane];
        add(sum, x);
    };
    Sums<VEC> was;
    if (ADDED) was = load_row<VEC>(out_row(last), at);
    for (uint32_t w = wave + 1; w < kSumWaves && __builtin_amdgcn_readlane(rows, w * kPiece) == last; ++w) add_part(0, w);
    if (shared && last == leaving)
        for (uint32_t w = 0; w < kSumWaves; ++w) add_part(1, w);
    store_row<VEC>(out_row(last), at, sum, scale, ADDED ? &was : nullptr);
}

// ---------------------------------------------------------------- host side

int vec_of(int d) { return d < 256 ? 1 : 4; }
int slices_of(int d) { return ((d + vec_of(d) - 1) / vec_of(d) + 63) / 64; }
// The workspace: entries (rows and tokens) of two stages of the sort in turn, the windows' sums.
struct GradSpace {
    int64_t entries, row[2], token[2], partial, bytes;
    GradSpace(int64_t rows, int d) {
        entries = (rows + kBlock - 1) / kBlock * kBlock;
        row[0] = 0;
        token[0] = row[0] + 4 * entries;
        row[1] = token[0] + 4 * entries;
        token[1] = row[1] + 4 * entries;
        partial = token[1] + 4 * entries;
        bytes = partial + entries / kWindow * slices_of(d) * 64 * vec_of(d) * 4;
    }
};

bool grad_sizes_fit(int64_t rows, int vocab, int d) {
    if (rows < 0 || rows >= (int64_t)1 << 30 || vocab < 1 || d < 1 || d >= 1 << 24) return false;
    return rows * (d < 64 ? 64 : d) < (int64_t)1 << 34;       // (a launch has fewer than 2^32 lanes)
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
    int spans = 1;                                            // 1, 2, 4 or 8, of whole vectors
    while (spans < 8 && spans * (2560 / (int)in) <= d) spans *= 2;
    const int width = ((d + spans - 1) / spans + 3) / 4 * 4;
    int lanes = 64;                                           // for a row; 16, 32 or 64
    while (lanes > 16 && d <= lanes * 2) lanes /= 2;
    const int each = width <= 256 ? 4 : 1;                    // rows of a wave at once
    const int64_t turns = ((rows + each - 1) / each * lanes + 255) / 256, groups = (turns < kMostTurns ? turns : kMostTurns) * spans;
    auto launch = [&](auto element, auto result) {
        using T = decltype(element);
        using O = decltype(result);
        auto with = [&](auto kernel, auto... layout) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, static_cast<hipStream_t>(stream),
                               static_cast<const T*>(table), static_cast<const T*>(t_perp), token_ids, vocab,
                               static_cast<const T*>(pos_embed), seq_len, scale, static_cast<O*>(out), rows, d, layout...);
        };
        if (d < 4) with(lookup_short_kernel<T, O>);
        else if (lanes < 64) with(lookup_kernel<true, 4, T, O>, spans, width, lanes);
        else if (each == 4) with(lookup_kernel<false, 4, T, O>, spans, width, lanes);
        else with(lookup_kernel<false, 1, T, O>, spans, width, lanes);
    };
    if (table_dtype == SPLC_F32 && out_dtype == SPLC_F32) launch(float{}, float{});
    else if (table_dtype == SPLC_F32) launch(float{}, uint16_t{});
    else if (out_dtype == SPLC_F32) launch(uint16_t{}, float{});
    else launch(uint16_t{}, uint16_t{});
    return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
}

int64_t sparseloco_embedding_grad_ws_bytes(int64_t rows, int vocab, int d) {
    if (!grad_sizes_fit(rows, vocab, d)) return SPLC_EINVAL;
    return GradSpace(rows, d).bytes;
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
    const GradSpace space(rows, d);
    if (ws_bytes < space.bytes) return SPLC_EINVAL;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const uint32_t slices = (uint32_t)slices_of(d);
    const uint32_t entries = (uint32_t)space.entries, windows = entries / kWindow;
    uint32_t *row[2], *token[2];
    for (int k = 0; k < 2; ++k) {
        row[k] = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + space.row[k]);
        token[k] = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + space.token[k]);
    }
    float* partial = reinterpret_cast<float*>(static_cast<char*>(ws) + space.partial);

    // the table in elements before its 16-byte vectors, vectors, and elements behind them; and the launches' shares of these
    const uint64_t size = (uint64_t)vocab * (uint64_t)d, element = table_dtype == SPLC_BF16 ? 2 : 4;
    uint64_t head = (16 - (reinterpret_cast<uintptr_t>(grad_table) & 15)) % 16 / element;
    if (head > size) head = size;
    const uint64_t vectors = accumulate ? 0 : (size - head) * element / 16;
    const uint64_t tail = size - head - vectors * 16 / element;
    uint4* vector = reinterpret_cast<uint4*>(static_cast<char*>(grad_table) + head * element);
    const bool many = entries > kFewEntries, merged = many && (entries > kDirect || vectors > kFewZeros);
    const uint32_t run = merged ? kRun : kDirect;
    const uint64_t sort_share = many ? vectors / 2 : vectors, merge_share = merged ? vectors / 4 : 0;
    const Zeros shares[3] = {{vector, sort_share}, {vector + sort_share, merge_share},
                             {vector + sort_share + merge_share, vectors - sort_share - merge_share}};
    auto groups_of = [](const Zeros& z) {
        const uint64_t spans = (z.vectors + kZeroSpan - 1) / kZeroSpan;
        return (uint32_t)(spans < kMostZeroGroups ? spans : kMostZeroGroups);
    };

    auto sort = [&](auto result) {
        using O = decltype(result);
        const uint32_t more = accumulate ? 0 : groups_of(shares[0]) + (shares[0].vectors == 0 ? 1 : 0);
        auto order = [&](auto kernel, uint32_t keys) {
            if (entries / keys + more > 0)
                hipLaunchKernelGGL(kernel, dim3(entries / keys + more), dim3(kOrderThreads), 0, st, token_ids, (uint32_t)rows, vocab,
                                   ignore_id, run, entries / keys, row[0], token[0], shares[0], static_cast<O*>(grad_table), size,
                                   (uint32_t)head, (uint32_t)tail);
        };
        if (merged) order(order_tokens_kernel<128, O>, 128);
        else order(order_tokens_kernel<64, O>, 64);
    };
    if (table_dtype == SPLC_F32) sort(float{});
    else sort(uint16_t{});
    if (rows == 0) return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
    int in = 0;
    for (uint64_t length = run; length < entries; length *= kFanIn, in ^= 1) {
        const Zeros share = length == run ? shares[1] : Zeros{nullptr, 0};
        const uint32_t groups = entries / kMergeThreads;
        auto merge = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(groups + groups_of(share)), dim3(kMergeThreads), 0, st, row[in], token[in], entries,
                               (uint32_t)length, row[in ^ 1], token[in ^ 1], groups, share);
        };
        if (length == kRun) merge(merge_runs_kernel<2048>);
        else merge(merge_runs_kernel<1024>);
    }
    auto sums = [&](auto vec, auto gradient, auto result) {
        constexpr int VEC = decltype(vec)::value;
        using G = decltype(gradient);
        using O = decltype(result);
        const uint32_t groups = windows * slices;
        if (many)
            hipLaunchKernelGGL((window_sums_kernel<VEC, G>), dim3(groups + groups_of(shares[2])), dim3(kWindow / kFlight * 64), 0, st,
                               static_cast<const G*>(grad_out), row[in], token[in], d, (int)slices, partial, groups,
                               shares[2]);
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(groups), dim3(kSumWaves * 64), 0, st,
                               static_cast<const G*>(grad_out), row[in], token[in], partial, entries, d, (int)slices, scale,
                               static_cast<O*>(grad_table));
        };
        if (many && accumulate) launch(row_sums_kernel<VEC, true, true, G, O>);
        else if (many) launch(row_sums_kernel<VEC, false, true, G, O>);
        else if (accumulate) launch(row_sums_kernel<VEC, true, false, G, O>);
        else launch(row_sums_kernel<VEC, false, false, G, O>);
    };
    auto by_type = [&](auto vec) {
        if (grad_dtype == SPLC_F32 && table_dtype == SPLC_F32) sums(vec, float{}, float{});
        else if (grad_dtype == SPLC_F32) sums(vec, float{}, uint16_t{});
        else if (table_dtype == SPLC_F32) sums(vec, uint16_t{}, float{});
        else sums(vec, uint16_t{}, uint16_t{});
    };
    if (vec_of(d) == 4) by_type(std::integral_constant<int, 4>{});
    else by_type(std::integral_constant<int, 1>{});
    return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
}

}  // extern "C"
