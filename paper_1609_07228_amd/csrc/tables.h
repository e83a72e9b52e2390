// What the kernels on tables of small floating-point codes (mx.hip, f8.hip) share: element types, scales, neighbouring lanes'
// values, loads into LDS, limits of a launch.
#pragma once
#include "common.h"

#include <stdint.h>

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Outputs larger than the L2 caches are stored past them (10^6 x 128 float32 read back: 102 -> 81 us); smaller ones are left there
// for whoever reads them next.
constexpr int64_t kStreamBytes = (int64_t)32 << 20;
// A launch takes fewer than 2^32 threads.  Rows that a kernel takes one by one go in slices of so many workgroups of 256.
constexpr int64_t kSliceBlocks = (int64_t)1 << 23;
inline bool launch_fits(int64_t blocks, int64_t threads) { return blocks <= 4294967295LL / threads; }

constexpr int64_t kMaxRows = 2147483647LL - 65536;

// (64 KiB and less need no leave, and asking for it takes a microsecond)
inline hipError_t allow_lds(const void *kernel, int bytes)
{
    return bytes > 65536 ? hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) : hipSuccess;
}
inline size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool dtype_ok(int32_t dtype) { return dtype == EFANNA_F32 || dtype == EFANNA_F16 || dtype == EFANNA_BF16; }
inline bool aligned_for(const void *p, int32_t dtype) { return ((uintptr_t)p & (dtype == EFANNA_F32 ? 3 : 1)) == 0; }

// 2^(b - 127); 255 stands for NaN
__device__ inline float scale_value(u32 b)
{
    return __uint_as_float(b == 0 ? 0x00400000u : b == 255 ? 0x7FC00000u : b << 23);
}

// ---- element types -------------------------------------------------------------------------------------
template <class T> __device__ inline float to_float(T x) { return (float)x; }
template <class T> __device__ inline T from_float(float x) { return (T)x; }      // to nearest, ties to even

// Eight values from or to any address that suits the element (the last ones of a row: fewer).
template <class T>
__device__ inline void load_eight(const T *p, int left, float (&v)[8])
{
    typedef T Piece __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
    constexpr int kPer = 16 / sizeof(T);
    if (left >= 8) {
#pragma unroll
        for (int i = 0; i < 8; i += kPer) {
            const Piece x = *(const Piece *)(p + i);
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[i + j] = to_float(x[j]);
        }
    } else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < left ? to_float(p[j]) : 0.0f;
}

// ---- lanes and LDS -------------------------------------------------------------------------------------
// A neighbour's value by row operations (no trip through LDS): the other lane of a pair, of a pair of pairs; the lane 4 or
// 8 further within a row of 16, around its end; the eight lanes of half a row in reverse.
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kDown4 = 0x120 + 12, kDown8 = 0x120 + 8, kMirror8 = 0x141;
template <int CTRL> __device__ inline u32 lane_from(u32 x) { return (u32)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true); }
template <int CTRL> __device__ inline float lane_from(float x) { return __uint_as_float(lane_from<CTRL>(__float_as_uint(x))); }

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;
__device__ inline void stage_lds(const void *from, void *to, int lane_bytes_16)
{
    if (lane_bytes_16) __builtin_amdgcn_global_load_lds((global_void *)from, (lds_void *)to, 16, 0, 0);
    else __builtin_amdgcn_global_load_lds((global_void *)from, (lds_void *)to, 4, 0, 0);
}
template <int N> __device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

}  // namespace

#define EF_DTYPE(dtype, T, ...)                                      \
    do {                                                             \
        if ((dtype) == EFANNA_F32) { typedef float T; __VA_ARGS__; } \
        else if ((dtype) == EFANNA_F16) { typedef _Float16 T; __VA_ARGS__; } \
        else { typedef __bf16 T; __VA_ARGS__; }                      \
    } while (0)
