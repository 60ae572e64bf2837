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
        stream_store4(p, v);
        return;
    }
    store1(p, v.x);
    if (n > 1) store1(p + 1, v.y);
    if (n > 2) store1(p + 2, v.z);
}
__device__ __forceinline__ int row_of(int32_t id, int vocab) { return id < 0 ? 0 : (id < vocab ? id : vocab - 1); }

// ---------------------------------------------------------------- lookup

constexpr int64_t kMostTurns = 1 << 21;  // (a launch has fewer than 2^32 lanes)

// Bound by memory: rows of the table in the order of the tokens, and out.  A wave takes ROWS tokens in one span of columns, and two
// to four vectors of every array are in flight: two of one row, or, of spans of at most 256 columns, one of four (65536 tokens of
// 50304, d 256, bf16: 15.4 -> 11.7 us; d 150, fp32, two tables: 18.0 -> 14.3).
// Workgroups go to the eight XCDs round-robin by number, and spans go with them: with four spans an XCD's L2 is asked for one fourth of
// every table row and of PosEmbed, and holds four times as many of them.  But a span is 1 to 2 KB of a row where there are several,
// since waves that read less of it at once wait longer than they read.  MI355X, 16384 tokens of 32000, d 2048, both fp32 tables and
// positions to bf16, 1 / 2 / 4 / 8 spans: 44.2 / 41.6 / 40.1 / 41.4 us (165 MB that cannot be done without, 4.1 TB/s; a copy reaches
// 4.8); 65536 of 50304, d 768, bf16, 1 / 2 / 4 spans: 31.0 / 43.0 / 64.8.  out without the streaming hint: 45.0 instead of 40.1.
// NARROW: rows of at most 128 columns, of which a wave takes as many at once as it has `lanes` lanes for (22817 tokens, d 106: 8.0 -> 5.5
// us; 65536, d 64: 18.9 -> 6.4, and 5.0 with four times as many).
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
            float4 x[ROWS * COLS], y[ROWS * COLS], z[ROWS * COLS];
#pragma unroll
            for (int k = 0; k < ROWS * COLS; ++k) {
                const int at = c + 256 * (k % COLS), n = d - at < 4 ? d - at : 4, r = k / COLS;
                if (at >= end) continue;
                x[k] = load_some(table + from[r] + at, n);
                if (t_perp) y[k] = load_some(t_perp + from[r] + at, n);
                if (pos) z[k] = load_some(p[r] + at, n);
            }
#pragma unroll
            for (int k = 0; k < ROWS * COLS; ++k) {
                const int at = c + 256 * (k % COLS), n = d - at < 4 ? d - at : 4, r = k / COLS;
                if (at >= end || row + r >= rows) continue;
                float4 v = x[k];
                if (t_perp) v = make_float4(v.x + y[k].x, v.y + y[k].y, v.z + y[k].z, v.w + y[k].w);
                v = make_float4(v.x * scale, v.y * scale, v.z * scale, v.w * scale);
                if (pos) v = make_float4(v.x + z[k].x, v.y + z[k].y, v.z + z[k].z, v.w + z[k].w);
                store_some(out + (row + r) * d + at, n, v);
            }
        }
    }
}

// ---------------------------------------------------------------- gradient: order of the tokens
//
// Entries (table row, token) are sorted by row, equal rows by token.  A workgroup sorts a block of 2048 in registers and LDS
// (bitonically, by row * 2048 + place in the block); then up to eight sorted runs at a time become one, every entry finding its place
// by itself: the number of smaller entries in each of the other runs, by binary search.  Tokens that are left out, and what fills the last
// block, have row kNone and token 0 and come last.
//
// Where the table is written whole, its zeros are written by further workgroups of these launches, which have little else to
// do with the memory; rows that have tokens are written again later.
//
// MI355X: sorting a block takes 7 us (64 tokens 2.7), bound by the vector ALU of its compute unit; merging 5 to 9 us, of which 4 are
// the launch and a chain of loads.

constexpr int kBlock = 2048, kBlockBits = 11, kSortThreads = 1024, kFanIn = 8;
constexpr int kItems = kBlock / kSortThreads;                // elements of a lane while it sorts
constexpr uint32_t kNone = 0x7FFFFFFFu, kMaxVocab = (1u << (32 - kBlockBits)) - 1;

// A launch's share of the zeros: 16-byte vectors from `at`, workgroup by workgroup.
struct Zeros {
    uint4* at;
    uint64_t vectors;
};
constexpr int kZeroSpan = 512;           // vectors a workgroup writes (50304 rows of 768: 26.6 us, 1024: 28.3, 2048: 30.4, 256: 36.7)
constexpr uint32_t kMostZeroGroups = 1 << 20;
__device__ __forceinline__ void write_zeros(const Zeros& z, uint32_t group) {
    typedef uint32_t vuint4 __attribute__((ext_vector_type(4)));
    for (uint64_t from = (uint64_t)group * kZeroSpan; from < z.vectors; from += (uint64_t)kMostZeroGroups * kZeroSpan)
        for (uint32_t i = threadIdx.x; i < kZeroSpan; i += blockDim.x)
            if (from + i < z.vectors) __builtin_nontemporal_store(vuint4{0, 0, 0, 0}, (SPLC_GLOBAL vuint4*)(z.at + from + i));
}

// The value that lane (this one ^ MASK) has.  Inside rows of 16 lanes by the vector ALU's own lane moves.
template <int MASK>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
    auto move = [](uint32_t v, auto control) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(control)::value, 0xF, 0xF, true);
    };
    using std::integral_constant;
    if constexpr (MASK == 1) return move(x, integral_constant<int, 0xB1>{});             // quads: 1 0 3 2
    else if constexpr (MASK == 2) return move(x, integral_constant<int, 0x4E>{});        // quads: 2 3 0 1
    else if constexpr (MASK == 3) return move(x, integral_constant<int, 0x1B>{});        // quads: 3 2 1 0
    else if constexpr (MASK == 4) return lane_xor<3>(lane_xor<7>(x));
    else if constexpr (MASK == 7) return move(x, integral_constant<int, 0x141>{});       // eights turned round
    else if constexpr (MASK == 8) return move(x, integral_constant<int, 0x128>{});       // rows turned by eight
    else if constexpr (MASK == 15) return move(x, integral_constant<int, 0x140>{});      // rows turned round
    else return __shfl_xor(x, MASK);
}

// The sort of a block: sorted runs of SIZE / 2 become runs of SIZE.  Every element meets the one whose number differs in the bits of
// MASK, first all below SIZE (so that one of the two runs is taken backwards), then one bit at a time, and of the two the one with
// the lower number keeps the smaller.  A lane's elements have the numbers first + 64 k.
using Items = uint32_t[kItems];
struct SortShared {
    uint32_t x[2][kBlock];
};
template <uint32_t MASK>
__device__ __forceinline__ void meet(Items& x, uint32_t first, uint32_t bit, SortShared& shared, uint32_t& side) {
    Items y;
    if constexpr (MASK >= 64 * kItems) {
#pragma unroll
        for (int k = 0; k < kItems; ++k) shared.x[side][first + 64 * k] = x[k];
        __syncthreads();                                     // (the other side is written next: nobody reads it any more)
#pragma unroll
        for (int k = 0; k < kItems; ++k) y[k] = shared.x[side][(first + 64 * k) ^ MASK];
        side ^= 1;
    } else {
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const uint32_t other = x[k ^ (int)(MASK / 64)];
            if constexpr (MASK % 64 == 0) y[k] = other;
            else y[k] = lane_xor<MASK % 64>(other);
        }
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const uint32_t smaller = x[k] < y[k] ? x[k] : y[k], larger = x[k] < y[k] ? y[k] : x[k];
        x[k] = ((first + 64 * k) & bit) == 0 ? smaller : larger;
    }
}
template <uint32_t BIT>
__device__ __forceinline__ void meet_by_bits(Items& x, uint32_t first, SortShared& shared, uint32_t& side) {
    if constexpr (BIT > 0) {
        meet<BIT>(x, first, BIT, shared, side);
        meet_by_bits<BIT / 2>(x, first, shared, side);
    }
}
// Up to the first `count` elements; those behind them are in order already.
template <uint32_t SIZE>
__device__ __forceinline__ void merge_up(Items& x, uint32_t first, uint32_t count, SortShared& shared, uint32_t& side) {
    if (SIZE >= 2 * count) return;
    meet<SIZE - 1>(x, first, SIZE / 2, shared, side);
    meet_by_bits<SIZE / 4>(x, first, shared, side);
    if constexpr (SIZE < kBlock) merge_up<SIZE * 2>(x, first, count, shared, side);
}

// head, tail: how many elements of the table lie before and behind its 16-byte vectors; the first further workgroup writes them.
template <class O>
__global__ __launch_bounds__(kSortThreads) void sort_tokens_kernel(const int32_t* __restrict__ ids, uint32_t rows, int vocab,
                                                                   int32_t ignore_id, uint32_t blocks, uint32_t* __restrict__ row,
                                                                   uint32_t* __restrict__ token, Zeros zeros, O* table,
                                                                   uint64_t table_size, uint32_t head, uint32_t tail) {
    const uint32_t tid = threadIdx.x;
    if (blockIdx.x >= blocks) {
        if (blockIdx.x == blocks) {
            if (tid < head) table[tid] = O(0);
            if (tid < tail) table[table_size - 1 - tid] = O(0);
        }
        write_zeros(zeros, blockIdx.x - blocks);
        return;
    }
    __shared__ SortShared shared;
    const uint32_t first = (tid >> 6) * (64 * kItems) + (tid & 63);      // the lane's elements: first + 64 k
    const uint32_t base = blockIdx.x * (uint32_t)kBlock;
    Items x;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const uint32_t at = first + 64 * k;
        uint32_t r = kMaxVocab;
        if (base + at < rows) {
            const int32_t id = ids[base + at];
            if (ignore_id < 0 || id != ignore_id) r = (uint32_t)row_of(id, vocab);
        }
        x[k] = r << kBlockBits | at;
    }
    uint32_t side = 0;
    merge_up<2>(x, first, rows - base < kBlock ? rows - base : kBlock, shared, side);
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const uint32_t r = x[k] >> kBlockBits;
        row[base + first + 64 * k] = r == kMaxVocab ? kNone : r;
        token[base + first + 64 * k] = r == kMaxVocab ? 0 : base + (x[k] & (kBlock - 1));   // (read, and not used)
    }
}

// Sorted runs of `length` entries (the last one of all may be shorter), kFanIn of them at a time, to one run.  Of every run
// SAMPLES entries at equal distances lie in LDS for the first steps of the search: all of them while runs are blocks, of longer
// ones 1024, and from a distance of 32 on the others are in one cache line.
template <bool BLOCKS, uint32_t SAMPLES, uint32_t THREADS>
__global__ __launch_bounds__(THREADS) void merge_runs_kernel(const uint32_t* __restrict__ row, const uint32_t* __restrict__ token,
                                                             uint32_t entries, uint32_t length, uint32_t* __restrict__ row_out,
                                                             uint32_t* __restrict__ token_out, uint32_t groups, Zeros zeros) {
    if (blockIdx.x >= groups) {
        write_zeros(zeros, blockIdx.x - groups);
        return;
    }
    __shared__ uint32_t sample[kFanIn * SAMPLES];            // the last entry of each stretch
    static_assert(!BLOCKS || SAMPLES == kBlock, "all entries of a block");
    const uint32_t i = blockIdx.x * THREADS + threadIdx.x;   // (the number of entries is a multiple of 2048, as is a run's)
    const uint32_t run = blockIdx.x * THREADS / length, first = run / kFanIn * kFanIn, stretch = BLOCKS ? 1 : length / SAMPLES;
    uint32_t some[kFanIn * SAMPLES / THREADS];
#pragma unroll
    for (uint32_t s = 0; s < kFanIn * SAMPLES / THREADS; ++s) {
        const uint64_t at = (uint64_t)first * length + (uint64_t)(s * THREADS + threadIdx.x + 1) * stretch - 1;
        some[s] = at < entries ? row[at] : kNone;
    }
    const uint32_t r = row[i], t = token[i];
#pragma unroll
    for (uint32_t s = 0; s < kFanIn * SAMPLES / THREADS; ++s) sample[s * THREADS + threadIdx.x] = some[s];
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
    if constexpr (BLOCKS) {
#pragma unroll
        for (uint32_t k = 0; k < kFanIn; ++k)
            below[k] += sample[k * SAMPLES + below[k]] < limit[k] ? 1 : 0;
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
// A wave takes the runs of equal rows that begin in one piece of 16 entries, in one span of columns, and keeps their sums in
// registers: grad_out is read once, in rows, and every row of the table is written once, by one wave.  A lane has VEC consecutive
// columns: four, or one where the table is narrow.  A run that goes on behind its piece is followed by its wave, through the sums of
// whole windows, which other waves have formed before (a token that makes up 7 % of 65537: 69 windows in 5 batches instead of 4400
// rows).  Bound by memory: MI355X, 65537 fp32 rows of 2050 into 32001 rows, frequencies 1 / rank, added to what is there: windows 42 us
// (4.5 TB/s), runs 126 us (4.5 TB/s); 16384 bf16 rows of 2048: runs 21 us.  One token throughout: 98 and 145 us, 18 and 41 us.  grad_out
// is read without the streaming hint, which loses lines that two slices share (65537 rows of few different tokens: 180 us with it, 128).

// The lane's columns of a slice.  The last vector of a row whose length is no multiple of four holds fewer: it is read as the
// four elements that end with the row (`back` elements earlier), and its elements are brought to the front.
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
// Which piece or window (their number is a multiple of eight) and which slice of its columns a wave takes.  A workgroup's waves,
// up to four, are independent; they and the other workgroups of the same rows follow each other on one XCD, so that lines which two
// slices share meet in one L2.
struct Unit {
    uint32_t item, slice;
    __device__ __forceinline__ Unit(uint32_t group, uint32_t slices) {
        const uint32_t waves = blockDim.x / 64, groups = (slices + waves - 1) / waves, place = group / 8;
        item = place / groups * 8 + group % 8;
        slice = place % groups * waves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    }
};
constexpr uint32_t kMostWaves = 4;
// Up to so many entries a workgroup's waves take a piece together (below), instead of windows' sums and a wave by itself.  Together /
// with windows, whole call: 2415 bf16 rows of 1792 of 388: 23.3 / 29.7 us, 4096 of 2048 of 32000: 53.5 / 55.7, 4096 fp32 rows of 256 of
// 3000: 22.5 / 24.5; 8192 of 2048 of 32000: 60.4 / 59.0, 8192 of 512 of 1000: 34.6 / 28.5, 16000 of 1024 of 500: 57.6 / 33.1.
constexpr uint32_t kTogetherMost = 4096;
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

constexpr int kPiece = 16;               // entries of a piece: rows of grad_out in flight
constexpr int kWindow = 64;              // entries that one partial sum covers: those a wave looks at together
static_assert(kWindow <= 64 && kBlock % kWindow == 0 && kWindow % kPiece == 0, "a wave walks whole windows");

// Windows of entries that lie inside one run: their sums, so that a frequent token's run is not left to one wave.
template <int VEC, class G>
__global__ __launch_bounds__(kMostWaves * 64) void window_sums_kernel(const G* __restrict__ grad, const uint32_t* __restrict__ row,
                                                         const uint32_t* __restrict__ token, int d, int slices,
                                                         float* __restrict__ partial, uint32_t groups, Zeros zeros) {
    if (blockIdx.x >= groups) {
        write_zeros(zeros, blockIdx.x - groups);
        return;
    }
    const Unit unit(blockIdx.x, (uint32_t)slices);
    const uint32_t slice = unit.slice, lane = threadIdx.x & 63, first = unit.item * kWindow;
    if (slice >= (uint32_t)slices || row[first] != row[first + kWindow - 1] || row[first] == kNone) return;
    const Columns<VEC> at(d, (int)slice, slices, (int)lane);
    Sums<VEC> sum = {};
    for (int e = 0; e < kWindow; e += kPiece) {
        Sums<VEC> x[kPiece];
#pragma unroll
        for (int k = 0; k < kPiece; ++k) x[k] = load_grad<VEC>(grad, token[first + e + k], d, at);
#pragma unroll
        for (int k = 0; k < kPiece; ++k) add(sum, x[k]);
    }
    float* to = partial + (((uint64_t)unit.item * slices + slice) * 64 + lane) * VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j) to[j] = sum.v[j];
}

// Writes a row's columns: scale * sum, added to what is there if asked to.
template <int VEC, class O>
__device__ __forceinline__ void store_row(O* out, const Columns<VEC>& at, Sums<VEC> s, float scale, const Sums<VEC>* was) {
    if constexpr (VEC == 4) {
        if (at.back & 1) { s.v[0] = s.v[1]; s.v[1] = s.v[2]; s.v[2] = s.v[3]; }
        if (at.back & 2) { s.v[0] = s.v[2]; s.v[1] = s.v[3]; }
        float4 x = make_float4(s.v[0] * scale, s.v[1] * scale, s.v[2] * scale, s.v[3] * scale);
        if (was) x = make_float4(was->v[0] + x.x, was->v[1] + x.y, was->v[2] + x.z, was->v[3] + x.w);
        store_some(out + at.col, at.n, x);
    } else {
        store1(out + at.col, was ? was->v[0] + s.v[0] * scale : s.v[0] * scale);
    }
}
template <int VEC, class O>
__device__ __forceinline__ Sums<VEC> load_row(const O* out, const Columns<VEC>& at) {
    Sums<VEC> s;
    if constexpr (VEC == 4) {
        const float4 x = at.n == 4 ? widened(stream_load4(out + at.col)) : load_some(out + at.col, at.n);
        s.v[0] = x.x; s.v[1] = x.y; s.v[2] = x.z; s.v[3] = x.w;
    } else {
        s.v[0] = widened(out[at.col]);
    }
    return s;
}

// TOGETHER: for few tokens, which leave most of the chip idle and make a launch for windows' sums too dear.  A workgroup's four waves
// take one piece and slice; the first does what a wave does otherwise, and what goes on behind the piece's window is divided among
// them, window by window, and joined in their order (runs of 2000 tokens of 300, fp32, d 2048: 22 -> 13 us).
template <int VEC, bool ADDED, bool TOGETHER, class G, class O>
__global__ __launch_bounds__(kMostWaves * 64) void row_sums_kernel(const G* __restrict__ grad, const uint32_t* __restrict__ row,
                                                      const uint32_t* __restrict__ token, const float* __restrict__ partial,
                                                      uint32_t entries, int d, int slices, float scale,
                                                      O* __restrict__ out) {
    uint32_t piece, slice, wave = 0;
    if constexpr (TOGETHER) {
        piece = blockIdx.x / (uint32_t)slices;
        slice = blockIdx.x % (uint32_t)slices;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    } else {
        const Unit unit(blockIdx.x, (uint32_t)slices);
        piece = unit.item;
        slice = unit.slice;
        if (slice >= (uint32_t)slices) return;
    }
    const uint32_t lane = threadIdx.x & 63;
    // the piece's window, an entry a lane (their number is a multiple of 2048); the piece begins at entry q of it
    uint32_t e = piece * kPiece / kWindow * kWindow;
    const uint32_t q = piece * kPiece % kWindow;
    uint32_t rows = row[e + lane % kWindow], tokens = token[e + lane % kWindow];
    auto row_at = [&](uint32_t k) { return __builtin_amdgcn_readlane(rows, k); };
    uint32_t now = q > 0 ? row_at(q - 1) : (e > 0 ? row[e - 1] : kNone);         // the run that `sum` belongs to
    const uint32_t last = row_at(q + kPiece - 1);
    if (row_at(q) == kNone || (piece > 0 && last == now)) return;                // nothing begins here
    const Columns<VEC> at(d, (int)slice, slices, (int)lane);
    Sums<VEC> sum = {};
    auto out_row = [&](uint32_t r) { return out + (uint64_t)r * (uint64_t)d; };
    // Rows of grad_out of entries k .. k + 15 of the window at hand; those from `end` on are read as the last one before it.
    auto load = [&](Sums<VEC> (&x)[kPiece], uint32_t k, uint32_t end) {
#pragma unroll
        for (uint32_t i = 0; i < kPiece; ++i)
            x[i] = load_grad<VEC>(grad, __builtin_amdgcn_readlane(tokens, k + i < end ? k + i : end - 1), d, at);
    };
    // How far the entries from k on belong to `now`.
    auto run_end = [&](uint32_t k) {
        const uint64_t others = k < kWindow ? __ballot(rows != now && lane < kWindow) >> k << k : 0;
        return others == 0 ? kWindow : (uint32_t)__builtin_ctzll(others);
    };
    auto add_run = [&](uint32_t k, uint32_t end) {
        for (; k < end; k += kPiece) {
            Sums<VEC> x[kPiece];
            load(x, k, end);
#pragma unroll
            for (uint32_t i = 0; i < kPiece; ++i)
                if (k + i < end) add(sum, x[i]);
        }
    };
    if (!TOGETHER || wave == 0) {
        Sums<VEC> x[kPiece];
        uint32_t r[kPiece];
        load(x, q, q + kPiece);
#pragma unroll
        for (uint32_t i = 0; i < kPiece; ++i) r[i] = row_at(q + i);
        // x becomes the sums of the runs up to here: those that end inside the piece are written, unless they began before it
#pragma unroll
        for (uint32_t i = 1; i < kPiece; ++i)
            if (r[i] == r[i - 1]) {
                Sums<VEC> upto = x[i - 1];
                add(upto, x[i]);
                x[i] = upto;
            }
        auto written = [&](uint32_t i) { return r[i] != now && r[i] != kNone && r[i] != last; };
#pragma unroll
        for (uint32_t half = 0; half < kPiece; half += kPiece / 2) {
            Sums<VEC> was[kPiece / 2];
            if (ADDED && at.n > 0)
#pragma unroll
                for (uint32_t i = 0; i < kPiece / 2; ++i)
                    if (i + half + 1 < kPiece && r[half + i] != r[half + i + 1] && written(half + i))
                        was[i] = load_row<VEC>(out_row(r[half + i]), at);
            if (at.n > 0)
#pragma unroll
                for (uint32_t i = 0; i < kPiece / 2; ++i)
                    if (i + half + 1 < kPiece && r[half + i] != r[half + i + 1] && written(half + i))
                        store_row<VEC>(out_row(r[half + i]), at, x[half + i], scale, ADDED ? &was[i] : nullptr);
        }
        sum = x[kPiece - 1];
    }
    if (last == kNone) return;
    now = last;
    uint32_t end = run_end(q + kPiece);
    if (!TOGETHER || wave == 0) add_run(q + kPiece, end);
    if constexpr (TOGETHER) {
        for (uint32_t w = e + (wave + 1) * kWindow; end == kWindow && w < entries; w += kMostWaves * kWindow) {
            rows = row[w + lane % kWindow];
            tokens = token[w + lane % kWindow];
            const uint32_t stop = run_end(0);
            add_run(0, stop);
            if (stop < kWindow) break;
        }
        if (end == kWindow) {                                // (the same for all four)
            __shared__ float parts[kMostWaves - 1][VEC][64];
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (wave > 0) parts[wave - 1][j][lane] = sum.v[j];
            __syncthreads();
            for (uint32_t w = 0; w < kMostWaves - 1; ++w) {
                Sums<VEC> x;
#pragma unroll
                for (int j = 0; j < VEC; ++j) x.v[j] = parts[w][j][lane];
                add(sum, x);
            }
        }
        if (wave > 0) return;
    } else {
        while (end == kWindow && (e += kWindow) < entries) { // the run goes on in the next window, and in whole ones, up to 16 at a time
            const uint32_t w = e + lane * kWindow;
            const bool whole = lane < kPiece && w < entries && row[w] == now && row[w + kWindow - 1] == now;
            const uint32_t n = (uint32_t)__builtin_ctzll(~__ballot(whole));
            if (n > 0) {
                Sums<VEC> x[kPiece];
#pragma unroll
                for (uint32_t i = 0; i < kPiece; ++i) {
                    const float* from = partial + ((((uint64_t)(e / kWindow) + (i < n ? i : n - 1)) * slices + slice) * 64 + lane) * VEC;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) x[i].v[j] = from[j];
                }
#pragma unroll
                for (uint32_t i = 0; i < kPiece; ++i)
                    if (i < n) add(sum, x[i]);
                e += (n - 1) * kWindow;
                continue;
            }
            rows = row[e + lane % kWindow];
            tokens = token[e + lane % kWindow];
            end = run_end(0);
            add_run(0, end);
        }
    }
    if (at.n > 0) {
        Sums<VEC> was;
        if (ADDED) was = load_row<VEC>(out_row(now), at);
        store_row<VEC>(out_row(now), at, sum, scale, ADDED ? &was : nullptr);
    }
}

// ---------------------------------------------------------------- host side

int vec_of(int d) { return d < 256 ? 1 : 4; }
int slices_of(int d) { return ((d + vec_of(d) - 1) / vec_of(d) + 63) / 64; }
// How the workgroups of the sums take a row's slices: `groups` of them, of `waves` waves.
struct Slices {
    uint32_t count, groups, waves, lanes;
    explicit Slices(int d) {
        count = (uint32_t)slices_of(d);
        groups = (count + kMostWaves - 1) / kMostWaves;
        waves = (count + groups - 1) / groups;
        lanes = groups * waves * 64;
    }
};

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
    if (rows < 0 || rows >= (int64_t)1 << 30 || vocab < 1 || vocab >= (int)kMaxVocab || d < 1 || d >= 1 << 24) return false;
    const int64_t entries = (rows + kBlock - 1) / kBlock * kBlock;
    const int64_t lanes = entries > kTogetherMost ? Slices(d).lanes : Slices(d).count * kMostWaves * 64;       // for a piece
    return entries / kPiece * lanes < (int64_t)1 << 32;       // (of one launch)
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
    int spans = 1;                                            // 1, 2 or 4, of whole vectors
    while (spans < 4 && spans * (2048 / (int)in) < d) spans *= 2;
    const int width = ((d + spans - 1) / spans + 3) / 4 * 4;
    int lanes = 64;                                           // for a row; 16, 32 or 64
    while (lanes > 16 && d <= lanes * 2) lanes /= 2;
    const int each = width <= 256 ? 4 : 1;                    // rows of a wave at once
    const int64_t turns = ((rows + each - 1) / each * lanes + 255) / 256, groups = (turns < kMostTurns ? turns : kMostTurns) * spans;
    auto launch = [&](auto element, auto result) {
        using T = decltype(element);
        using O = decltype(result);
        auto with = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, static_cast<hipStream_t>(stream),
                               static_cast<const T*>(table), static_cast<const T*>(t_perp), token_ids, vocab,
                               static_cast<const T*>(pos_embed), seq_len, scale, static_cast<O*>(out), rows, d, spans, width, lanes);
        };
        if (lanes < 64) with(lookup_kernel<true, 4, T, O>);
        else if (each == 4) with(lookup_kernel<false, 4, T, O>);
        else with(lookup_kernel<false, 1, T, O>);
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
    const Slices slices(d);
    const uint32_t entries = (uint32_t)space.entries, blocks = entries / kBlock;
    const bool merged = blocks > 1, many = entries > kTogetherMost;
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
    const uint64_t sort_share = merged ? vectors / 2 : vectors, merge_share = many ? vectors / 4 : vectors - sort_share;
    const Zeros shares[3] = {{vector, sort_share}, {vector + sort_share, merge_share},
                             {vector + sort_share + merge_share, vectors - sort_share - merge_share}};
    auto groups_of = [](const Zeros& z) {
        const uint64_t spans = (z.vectors + kZeroSpan - 1) / kZeroSpan;
        return (uint32_t)(spans < kMostZeroGroups ? spans : kMostZeroGroups);
    };

    auto sort = [&](auto result) {
        using O = decltype(result);
        const uint32_t more = accumulate ? 0 : groups_of(shares[0]) + (shares[0].vectors == 0 ? 1 : 0);
        if (blocks + more > 0)
            hipLaunchKernelGGL(sort_tokens_kernel<O>, dim3(blocks + more), dim3(kSortThreads), 0, st, token_ids, (uint32_t)rows, vocab,
                               ignore_id, blocks, row[0], token[0], shares[0], static_cast<O*>(grad_table), size, (uint32_t)head,
                               (uint32_t)tail);
    };
    if (table_dtype == SPLC_F32) sort(float{});
    else sort(uint16_t{});
    if (rows == 0) return hipGetLastError() == hipSuccess ? SPLC_OK : SPLC_EHIP;
    int in = 0;
    for (uint64_t length = kBlock; length < entries; length *= kFanIn, in ^= 1) {
        const bool blocks_yet = length == kBlock;
        const Zeros share = blocks_yet ? shares[1] : Zeros{nullptr, 0};
        auto merge = [&](auto kernel, uint32_t threads) {
            hipLaunchKernelGGL(kernel, dim3(entries / threads + groups_of(share)), dim3(threads), 0, st, row[in], token[in], entries,
                               (uint32_t)length, row[in ^ 1], token[in ^ 1], entries / threads, share);
        };
        if (blocks_yet) merge(merge_runs_kernel<true, kBlock, 512>, 512);
        else merge(merge_runs_kernel<false, 1024, 512>, 512);
    }
    auto sums = [&](auto vec, auto gradient, auto result) {
        constexpr int VEC = decltype(vec)::value;
        using G = decltype(gradient);
        using O = decltype(result);
        const uint32_t window_groups = entries / kWindow * slices.groups;
        if (many)
            hipLaunchKernelGGL((window_sums_kernel<VEC, G>), dim3(window_groups + groups_of(shares[2])), dim3(slices.waves * 64), 0, st,
                               static_cast<const G*>(grad_out), row[in], token[in], d, (int)slices.count, partial, window_groups,
                               shares[2]);
        auto launch = [&](auto kernel, uint32_t groups, uint32_t waves) {
            hipLaunchKernelGGL(kernel, dim3(groups), dim3(waves * 64), 0, st, static_cast<const G*>(grad_out), row[in], token[in], partial,
                               entries, d, (int)slices.count, scale, static_cast<O*>(grad_table));
        };
        const uint32_t pieces = entries / kPiece;
        if (many && accumulate) launch(row_sums_kernel<VEC, true, false, G, O>, pieces * slices.groups, slices.waves);
        else if (many) launch(row_sums_kernel<VEC, false, false, G, O>, pieces * slices.groups, slices.waves);
        else if (accumulate) launch(row_sums_kernel<VEC, true, true, G, O>, pieces * slices.count, kMostWaves);
        else launch(row_sums_kernel<VEC, false, true, G, O>, pieces * slices.count, kMostWaves);
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
