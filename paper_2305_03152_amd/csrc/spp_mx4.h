// Rows in MXFP4 and the element types of the operators on gathered rows: what their kernels share.
//
// A row of D columns is nb = ceil(D/32) blocks of 32 columns (the last one filled up with zeros): sixteen bytes of E2M1 codes
// per block (column 2j of a block in the low half of its byte j), then one E8M0 byte per block, then zeros up to a multiple
// of sixteen bytes.  Codes before scales, so that a lane takes a block in one aligned 16-byte load.
#pragma once

#include "spp_common.h"
#include "spp_device.h"

#include <atomic>

namespace spp {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

template <class T> struct Elem;                      // four and eight elements of a type as vectors
template <> struct Elem<float> { typedef f32x4 v4; };
template <> struct Elem<_Float16> { typedef f16x4 v4; typedef f16x8 v8; };
template <> struct Elem<__bf16> { typedef bf16x4 v4; typedef bf16x8 v8; };

static inline size_t type_bytes(int32_t type) { return type == SPP_F32 ? 4 : 2; }
static inline bool is_type(int32_t type) { return type == SPP_F32 || type == SPP_F16 || type == SPP_BF16; }
static inline int mx4_blocks(int32_t D) { return (D + 31) / 32; }
static inline int mx4_bytes(int32_t D) { return (17 * mx4_blocks(D) + 15) / 16 * 16; }

// 2^(byte - 127) as a float; byte 255 is the format's NaN.
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte == 0u ? 0x00400000u : byte << 23);
}

// Which rows a call has: as given, or counted on the device, never more than the caller's buffers hold.
__device__ __forceinline__ int64_t rows_of(int64_t n, const int64_t* d_n) {
    if (!d_n) return n;
    const int64_t c = *d_n;
    return c < 0 ? 0 : c < n ? c : n;
}

// Which of `items` equal pieces of a stream of memory a workgroup takes, from `at` by `step` up to `end`.  Consecutive workgroups go
// to the eight XCDs in turn: each XCD gets a contiguous eighth of the stream.  Plain writes of 1.3 GB, tiles of 16 KB: 6.1 to 6.4 TB/s so,
// 4.8 to 5.5 with the tiles dealt out in order.
struct Share {
    int64_t at, end, step;
    __device__ __forceinline__ explicit Share(int64_t items) : Share(items, 1, 0) {}
    // The same for the wavefronts of a workgroup, side by side.
    __device__ __forceinline__ Share(int64_t items, int waves) : Share(items, waves, (int)threadIdx.x >> 6) {}
    __device__ __forceinline__ Share(int64_t items, int waves, int wave) {
        const bool all = gridDim.x >= 8;
        const unsigned x = all ? blockIdx.x & 7 : 0;
        at = (all ? items * x >> 3 : 0) + (int64_t)(all ? blockIdx.x >> 3 : blockIdx.x) * waves + wave;
        end = all ? items * (x + 1) >> 3 : items;
        step = (int64_t)(all ? (gridDim.x - x + 7) >> 3 : gridDim.x) * waves;
    }
};
// The same with as many pieces as there are workgroups: a workgroup's one.
__device__ __forceinline__ unsigned own_piece() {
    const unsigned x = blockIdx.x & 7, more = gridDim.x & 7;
    return x * (gridDim.x >> 3) + (x < more ? x : more) + (blockIdx.x >> 3);
}

// A vector at an address that is aligned to its elements only: one access all the same.
template <class V> struct Loose { V v; } __attribute__((packed, aligned(2)));

// Lists of packed rows, each with a matrix Y of its own: the operands of the product and of its gradient.
constexpr int kRowLists = SPP_MAX_ROW_LISTS;
static_assert(kRowLists == kWave, "a wavefront's lanes hold a list each");
struct RowTable {
    const uint8_t* rows[kRowLists];
    void*          y[kRowLists];
    const int64_t* d_n[kRowLists];
    int64_t        ld[kRowLists];
    int32_t        n[kRowLists];
    uint8_t        group[kRowLists];
    int32_t        n_lists;
};
// Lane j has list j: its rows, and the tiles of all lists up to it.  The count of a list may have to be fetched: one round trip.
struct Lists {
    int rows, upto, tiles;
    __device__ __forceinline__ Lists(const RowTable& t, int tile_rows) {
        const int j = lane_id();
        rows = j < t.n_lists ? (int)rows_of(t.n[j], t.d_n[j]) : 0;
        tiles = (int)(((int64_t)rows + tile_rows - 1) / tile_rows);
        upto = wave_inclusive_scan(tiles);
    }
    __device__ __forceinline__ int total() const { return __builtin_amdgcn_readlane(upto, kWave - 1); }
    __device__ __forceinline__ int list_of(int tile) const { return __builtin_amdgcn_readfirstlane(__popcll(__ballot(upto <= tile))); }
    __device__ __forceinline__ int rows_in(int list) const { return __builtin_amdgcn_readlane(rows, list); }
    __device__ __forceinline__ int first_tile(int list) const { return __builtin_amdgcn_readlane(upto - tiles, list); }
};

// Host: the checks that the product and the gradient share; fills the table, and *most with the rows the lists can hold.
int row_table(const char* who, const spp_row_list* lists, int32_t n_lists, int32_t n_groups, int32_t D, int32_t H, int32_t type,
              RowTable& t, int64_t* most);


// More dynamic LDS than 64 KB has to be allowed to a kernel, once per device.
struct LdsLimit {
    std::atomic<int> most[kPoolDevices] = {};
    int allow(const spp_ctx* ctx, const void* kernel, int lds) {
        if (lds <= 65536 || (ctx->device < kPoolDevices && most[ctx->device].load(std::memory_order_relaxed) >= lds)) return SPP_OK;
        SPP_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 163840));
        if (ctx->device < kPoolDevices) most[ctx->device].store(163840, std::memory_order_relaxed);
        return SPP_OK;
    }
};

}  // namespace spp
