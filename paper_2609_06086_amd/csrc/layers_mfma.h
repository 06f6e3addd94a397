#pragma once
// Matrix instructions of the layer operators: a wave multiplies 32 x 16 by 16 x 32
// values of a 16-bit type.  Lane l holds eight neighbouring values along the sum, from 8 (l / 32) on, of row (first
// operand) or column (second) l % 32, and of the result column l % 32, rows (r & 3) + 8 (r >> 2) + 4 (l / 32), r in [0, 16).
#include "layers_device.h"

#include <type_traits>

namespace pl {

using Acc = float __attribute__((ext_vector_type(16)));
using HalfVec = _Float16 __attribute__((ext_vector_type(8)));
using BrainVec = __bf16 __attribute__((ext_vector_type(8)));
using Words4 = uint32_t __attribute__((ext_vector_type(4)));

template <class T>
__device__ __forceinline__ Acc mfma(Words4 a, Words4 b, Acc c);
template <>
__device__ __forceinline__ Acc mfma<BF16>(Words4 a, Words4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(BrainVec, a), __builtin_bit_cast(BrainVec, b), c,
                                                   0, 0, 0);
}
template <>
__device__ __forceinline__ Acc mfma<F16>(Words4 a, Words4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(HalfVec, a), __builtin_bit_cast(HalfVec, b), c, 0,
                                                  0, 0);
}

// 16 x 32 by 32 x 16: lane l holds eight neighbouring values from 8 (l / 16) on of row or column l % 16, and of the result
// column l % 16, rows 4 (l / 16) + r.
using Acc4 = float __attribute__((ext_vector_type(4)));
template <class T>
__device__ __forceinline__ Acc4 mfma16(Words4 a, Words4 b, Acc4 c) {
    if constexpr (std::is_same_v<T, BF16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(BrainVec, a), __builtin_bit_cast(BrainVec, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(HalfVec, a), __builtin_bit_cast(HalfVec, b), c, 0, 0, 0);
}

using Rsrc = __amdgpu_buffer_rsrc_t;

__device__ __forceinline__ Rsrc buffer(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00027000);
}

// Four rows of a column of 16-bit values that lie row by row in LDS.
// The sixteen lanes of a quarter of the wave bring the addresses of 4 rows x 16 values, four neighbouring values a lane,
// row by row, and lane l of them gets the rows of value l % 16.
__device__ __forceinline__ uint2 read_turned(__attribute__((address_space(3))) const void *lds) {
    using Four = short __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Four *)lds));
}

// 16 bytes a lane from a buffer to LDS, at `to` + 16 lane; an offset past the buffer's end brings zeros.  Before a turned read
// the compiler waits for every such load that it knows of, though it may be meant for another stage.  OWN loads are instructions that it
// does not know: nothing but the caller's own wait for vmcnt says that they are done.  Their s_nop stands for the waits that
// the compiler puts between what writes m0 or the descriptor's registers and such a load.
template <bool OWN>
__device__ __forceinline__ void copy_to_lds(Rsrc from, uint32_t offset, uint16_t *to) {
    using Place = __attribute__((address_space(3))) void *;
    if constexpr (OWN)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :: "s"(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(Place)to)), "v"(offset), "s"(from) : "memory", "m0");
    else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (Place)to, 16, offset, 0, 0, 0);
}
constexpr uint32_t kNowhere = 0x80000000u;

// Two values rounded to nearest even, in one instruction.
template <class T>
__device__ __forceinline__ uint32_t pair(float lo, float hi) {
    using Two = typename T::raw __attribute__((ext_vector_type(2)));
    using Floats = float __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((Floats){lo, hi}, Two));
}

// How the compiler is to mix what a block of code does: first N of a kind, and so on, in the order of the calls.
constexpr int kMatrix = 0x8, kReadLds = 0x100;
template <int KIND, int N>
__device__ __forceinline__ void then() {
    __builtin_amdgcn_sched_group_barrier(KIND, N, 0);
}

// Which of the ranges [offsets[r], offsets[r + 1]) of rows a tile belongs to.  Range r has the tiles from
// offsets[r] / size + r on: that leaves each range one more than its rows fill at least, so no list of tiles is needed, and
// at most one tile a range stays empty.  A wave looks 64 offsets over at a time, a level of 64 for each factor of 64.
struct Place {
    uint32_t range, begin, end;    // begin: the tile's first row, end: the range's
    bool there;
};

__device__ __forceinline__ uint32_t bound_of(const int32_t *offsets, uint32_t r, uint32_t rows) {
    return (uint32_t)min(max(offsets[r], 0), (int32_t)rows);
}

__device__ __forceinline__ Place place_of(const int32_t *offsets, uint32_t ranges, uint32_t rows, uint32_t tile, uint32_t size) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t first = 0, n = ranges;    // the range is one of [first, first + n)
    while (n > 1) {
        const uint32_t step = (n + 63) / 64, r = first + min(lane * step, n - 1);
        const bool before = lane * step < n && bound_of(offsets, r, rows) / size + r <= tile;
        const uint32_t k = (uint32_t)__popcll(__ballot(before));    // offsets ascend: the first k
        const uint32_t at = k ? (k - 1) * step : 0;
        first += at;
        n = min(step, n - at);
    }
    first = __builtin_amdgcn_readfirstlane(first);
    const uint32_t begin = bound_of(offsets, first, rows), end = max(begin, bound_of(offsets, first + 1, rows));
    const uint32_t t = tile - min(tile, begin / size + first);
    Place p;
    p.range = first;
    p.there = tile >= begin / size + first && t < (end - begin + size - 1) / size;
    p.begin = p.there ? begin + t * size : begin;
    p.end = end;
    return p;
}
inline uint64_t tiles_for(uint64_t rows, uint64_t ranges, uint32_t size) { return rows / size + ranges; }

// Blocks from a.first on, in as many launches as it takes: a grid holds less than 2^32 threads.  Each begins at a multiple of 8, so
// that blocks go round the XCDs as in one.
template <class K, class A>
inline int launch_blocks(K kernel, A a, uint64_t blocks, uint32_t threads, void *hip_stream) {
    const uint64_t most = 0xffffffffull / threads / 8 * 8;
    for (uint64_t at = 0; at < blocks; at += most) {
        a.first = (uint32_t)at;
        kernel<<<(uint32_t)(blocks - at < most ? blocks - at : most), threads, 0, (hipStream_t)hip_stream>>>(a);
        PL_TRY(launched());
    }
    return POSEIDON_OK;
}
constexpr uint64_t kBlocksMost = 0x7fffff00u;    // of a call

}  // namespace pl
