// What the kernels of the language-model operators share: element types, packed sequences,
// windows of memory, sums over lanes.
#pragma once

#include <hip/hip_runtime.h>

#include "csb_internal.hpp"
#include "csbrnn_lm.h"

namespace csb {

constexpr int64_t kMaxWorkgroups = (1 << 24) - 1;    // of 256 threads: a grid has fewer than 2^32 threads

inline bool known_type(int32_t type) { return type == CSB_VAL_F32 || type == CSB_VAL_F16 || type == CSB_VAL_BF16; }
inline int32_t type_size(int32_t type) { return type == CSB_VAL_F32 ? 4 : 2; }

template <int VF> struct Elem;
template <> struct Elem<CSB_VAL_F32> { using T = float; };
template <> struct Elem<CSB_VAL_F16> { using T = _Float16; };
template <> struct Elem<CSB_VAL_BF16> { using T = __bf16; };

// Tiles of `1 << shift` packed places that a sequence's places fall into, numbered so that the number is known from
// the offsets alone: sequence i has the numbers from (start_i >> shift) + i on.  Its tiles are at most
// (end_i >> shift) - (start_i >> shift) + 1, so the ranges do not overlap and (total >> shift) + n_seq numbers are enough; those
// of a range that no tile has do nothing.
inline int64_t tile_numbers(int64_t total, int64_t n_seq, int shift) { return (total >> shift) + n_seq; }

#ifdef __HIPCC__
constexpr float kMostBf16 = 0x1.fep127f;       // the largest bfloat16 number

// Where a sequence starts and ends: d_start's offsets, or equal lengths; never outside [0, total].
__device__ __forceinline__ int64_t clamp64(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ void sequence_range(const int32_t *start, int64_t i, int64_t each, int64_t total, int64_t *first, int64_t *end) {
    if (start) {
        *first = clamp64(start[i], 0, total);
        *end = clamp64(start[i + 1], *first, total);
    } else {
        *first = i * each;
        *end = *first + each;
    }
}

// The sequence that tile number `tile` belongs to: one less than the count of sequences whose numbers
// start at or below it (no offsets: sequences of `each` places).  All threads of the workgroup call it (one barrier for 256 sequences).
__device__ __forceinline__ int tile_sequence(const int32_t *start, int n_seq, int64_t total, int shift, int64_t tile, int64_t each = 0) {
    int n = 0;
    for (int base = 0; base < n_seq; base += (int)blockDim.x) {
        const int i = base + (int)threadIdx.x;
        const int below = __syncthreads_count(i < n_seq && ((start ? clamp64(start[i], 0, total) : i * each) >> shift) + i <= tile);
        n += below;
        if (below < (int)blockDim.x) break;
    }
    return n - 1;
}

// Memory from `base` on, `bytes` of it: reads past them give zero, writes past them do nothing, so that every lane may take part in every
// access and the wavefront knows how many are in flight.
using window_t = __amdgpu_buffer_rsrc_t;
constexpr uint32_t kOutside = 0x80000000u;     // an offset past any window
__device__ __forceinline__ window_t window(const void *base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00020000);
}
template <int N> struct RawBits { using type = uint32_t; };
template <> struct RawBits<2> { using type = uint16_t; };
template <typename T> using raw_t = typename RawBits<sizeof(T)>::type;        // a number as it is stored
template <typename T> __device__ __forceinline__ raw_t<T> window_load(window_t w, uint32_t at) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_raw_buffer_load_b16(w, (int)at, 0, 0);
    else return __builtin_amdgcn_raw_buffer_load_b32(w, (int)at, 0, 0);
}
template <typename T> __device__ __forceinline__ void window_store(window_t w, uint32_t at, T v) {
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), w, (int)at, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), w, (int)at, 0, 0);
}

// Requests to memory stay in the order written, so that a wait in a loop is for as many of them in its first turn as in the others.
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }

// The value of lane (lane + 16 - N) % 16 of the lane's row of 16.
template <int N> __device__ __forceinline__ float row_rotated(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, false));
}
#endif

}  // namespace csb
