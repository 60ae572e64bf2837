// A plan and a bound tensor list as the library's sources see them, the argument checks that the entry points share, and
// 16-byte accesses to the tensors.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <vector>

#include "sparseloco.h"

namespace splc {

constexpr int kChunk = SPLC_CHUNK;

struct ChunkDesc {
    uint32_t tensor;                     // index into the pointer tables
    uint32_t n_c;                        // elements in this chunk (kChunk unless it is an edge chunk)
    uint64_t offset;                     // element offset of local index 0 inside its tensor
    uint32_t stride;                     // elements between local rows: 64 (flat) or the matrix's columns (tile)
    uint8_t h;                           // local rows present (1..64)
    uint8_t w;                           // width of every row but the last
    uint8_t last_w;                      // width of the last row (flat tail), = w for a tile
    uint8_t vec;                         // bit 0: complete (all 4096 elements present), every 4-element vector whole;
                                         // bit 1: and every row of a bf16 array starts at a dword
    uint32_t id;                         // chunk number (position of its message in pairs / scales / values)
    uint32_t reserved;
};
static_assert(sizeof(ChunkDesc) == 32, "chunk table entries are 32 bytes");

// Streaming accesses: every dense array is touched exactly once per launch, so loads and stores
// carry the non-temporal hint (measured on MI355X: 3 reads + 1 write streams at ~6.0 TB/s with
// the hint against ~5.6 TB/s without).
// The vector types promise only 4-byte alignment: rows of a tile start at any multiple of 4 bytes,
// and global memory accepts dword-aligned multi-dword accesses.
typedef float vfloat4 __attribute__((ext_vector_type(4), aligned(4)));

// Every tensor lives in global memory; saying so lets the compiler emit global_ instead of flat_
// instructions.
#define SPLC_GLOBAL __attribute__((address_space(1)))
typedef uint32_t vuint2 __attribute__((ext_vector_type(2), aligned(2)));        // rows of bf16 may start at any element
__device__ __forceinline__ float4 stream_load4(const float* p) {
    vfloat4 v = __builtin_nontemporal_load((const SPLC_GLOBAL vfloat4*)p);
    return make_float4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ uint2 stream_load4(const uint16_t* p) {       // four bf16
    vuint2 v = __builtin_nontemporal_load((const SPLC_GLOBAL vuint2*)p);
    return make_uint2(v.x, v.y);
}
__device__ __forceinline__ float4 cached_load4(const float* p) {
    vfloat4 v = *(const SPLC_GLOBAL vfloat4*)p;
    return make_float4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ uint2 cached_load4(const uint16_t* p) {
    vuint2 v = *(const SPLC_GLOBAL vuint2*)p;
    return make_uint2(v.x, v.y);
}
template <bool STREAM, class T>
__device__ __forceinline__ auto load4(const T* p) {
    if constexpr (STREAM) return stream_load4(p);
    else return cached_load4(p);
}
__device__ __forceinline__ void stream_store4(float* p, float4 v) {
    vfloat4 t = {v.x, v.y, v.z, v.w};
    __builtin_nontemporal_store(t, (SPLC_GLOBAL vfloat4*)p);
}

// fp32 and bf16 elements as fp32 (bf16 is the upper half of the word), one and four at a time.
__device__ __forceinline__ float widened(float v) { return v; }
__device__ __forceinline__ float widened(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float4 widened(float4 v) { return v; }
__device__ __forceinline__ float4 widened(uint2 v) {
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                       __uint_as_float(v.y & 0xFFFF0000u));
}
// Two as bf16, rounded to nearest, ties to even.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    typedef __bf16 vbf16x2 __attribute__((ext_vector_type(2)));
    const vbf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ void stream_store4(uint16_t* p, float4 v) {
    const vuint2 t = {bf16_pair(v.x, v.y), bf16_pair(v.z, v.w)};
    __builtin_nontemporal_store(t, (SPLC_GLOBAL vuint2*)p);
}

}  // namespace splc

struct sparseloco_plan {
    int device = 0;
    int n_tensors = 0;
    int kappa = 0;
    int quant = SPLC_QUANT_2BIT;
    int select = SPLC_SELECT_AUTO;
    uint32_t* radix_counter = nullptr;   // diagnostic (sparseloco_plan_set_radix_counter), normally null
    int64_t n_chunks = 0;
    int64_t n_params = 0;
    std::vector<int64_t> numel;
    int layout = SPLC_LAYOUT_FLAT;
    // Chunk table, ordered [edge chunks | complete, odd row length | other complete ones]; every entry carries its chunk
    // number.  The edge chunks, which take a little longer, come first so that they do not form the tail of the launch.
    // The compression of a large tiled plan takes complete tiles four at a time where four lie side by side ("strips", one
    // entry each: origin, stride and chunk number of the first tile); only the other chunks are in the table above.  Its
    // outer update, which is element-wise, walks the tensors as flat chunks (a table of its own).
    // One device allocation holds [chunks | strips | flat chunks of the update | every chunk one by one | numel].
    splc::ChunkDesc* d_chunks = nullptr;
    splc::ChunkDesc* h_chunks = nullptr; // pinned source of the asynchronous upload, kept until destroy
    int64_t n_entries = 0;               // entries of the chunk table (= n_chunks unless there are strips)
    int64_t n_gen = 0;                   // edge chunks among them
    int64_t n_strips = 0;
    splc::ChunkDesc* d_strips = nullptr; // inside d_chunks' allocation
    splc::ChunkDesc* d_update = nullptr; // = d_chunks for a flat plan; numbered tensor by tensor
    int64_t n_update = 0, n_update_gen = 0;
    splc::ChunkDesc* d_all = nullptr;    // every chunk one by one, for all other kernels (= d_chunks without strips)
    int64_t n_all_gen = 0;
    int64_t* d_numel = nullptr;          // elements of each tensor
};

// n_sets lists of n_tensors device pointers, set-major, resident on the device.
struct sparseloco_tensors {
    int device = 0;
    int n_tensors = 0;
    int n_sets = 0;
    int dtype = SPLC_F32;
    bool disjoint = false;               // no tensor shares memory with another (looked at where it matters: small plans)
    size_t room = 0;                     // pointers that the tables hold
    void** d_table = nullptr;
    void** h_table = nullptr;            // pinned source of the upload
};

namespace splc {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool finite(float v) { return v == v && v - v == 0.f; }

inline int current_device_is(int device) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return SPLC_EHIP;
    return dev == device ? SPLC_OK : SPLC_EPLAN;
}

// A binding fits the plan: same device, same tensor count, the wanted element type, enough sets.
inline int check_tensors(const sparseloco_plan* plan, const sparseloco_tensors* t, int dtype, int min_sets) {
    if (!t) return SPLC_EINVAL;
    if (t->device != plan->device || t->n_tensors != plan->n_tensors || t->dtype != dtype) return SPLC_EPLAN;
    return t->n_sets >= min_sets ? SPLC_OK : SPLC_EINVAL;
}
// Device table of set `set` of a binding (a single-set binding serves every set index).
template <class T>
T const* set_table(const sparseloco_tensors* t, int set) {
    return reinterpret_cast<T const*>(t->d_table + (size_t)(t->n_sets == 1 ? 0 : set) * (size_t)t->n_tensors);
}

// LDS that a launch reserves so that only `groups_per_unit` of its workgroups, which use `used` bytes
// each, fit on a compute unit.  LDS is handed out in 1280-byte units.
inline unsigned reserve_lds(int groups_per_unit, size_t used) {
    const size_t share = 160 * 1024 / (size_t)groups_per_unit / 1280 * 1280;
    return used < share ? (unsigned)(share - used) : 0u;
}

}  // namespace splc
