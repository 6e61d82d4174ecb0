// Elements of bf16 and fp32 arrays at any place of a flat array: chunks of 16 bytes and groups of eight, aligned to the element only
// (the memory path takes such accesses whole; the compiler is told by the packed types).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace am {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

template <int ALIGN> struct __attribute__((packed, aligned(ALIGN))) Chunk16 { u32x4 v; };

template <int ALIGN> struct __attribute__((packed, aligned(ALIGN))) Chunk8 { u32x2 v; };

template <typename T> __device__ __forceinline__ u32x4 load16(const T *p) { return reinterpret_cast<const Chunk16<sizeof(T)> *>(p)->v; }
template <typename T> __device__ __forceinline__ void store16(T *p, u32x4 v) { reinterpret_cast<Chunk16<sizeof(T)> *>(p)->v = v; }

// the same past the caches, for what is written once and is larger than they are
typedef u32x4 __attribute__((aligned(2))) u32x4_anywhere;
template <typename T> __device__ __forceinline__ void stream16(T *p, u32x4 v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4_anywhere *>(p)); }
template <typename T> __device__ __forceinline__ void store8bytes(T *p, u32x2 v) { reinterpret_cast<Chunk8<sizeof(T)> *>(p)->v = v; }

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return (float)x; }
template <typename T> __device__ __forceinline__ T from_f32(float x) { return (T)x; }       // nearest even

// Eight consecutive elements as fp32; elements past the first `valid` read as 0 and are not touched in memory.
struct F8 { float v[8]; };

template <typename T> __device__ __forceinline__ F8 load8(const T *p, int valid)
{
    F8 r;
    if (valid >= 8) {
        if constexpr (sizeof(T) == 4) {
            const f32x4 a = __builtin_bit_cast(f32x4, load16(p)), b = __builtin_bit_cast(f32x4, load16(p + 4));
#pragma unroll
            for (int j = 0; j < 4; ++j) { r.v[j] = a[j]; r.v[4 + j] = b[j]; }
        } else {
            const u32x4 t = load16(p);
#pragma unroll
            for (int j = 0; j < 4; ++j) { r.v[2 * j] = __uint_as_float(t[j] << 16); r.v[2 * j + 1] = __uint_as_float(t[j] & 0xFFFF0000u); }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) r.v[j] = j < valid ? to_f32(p[j]) : 0.f;
    }
    return r;
}

template <typename T, bool STREAM = false> __device__ __forceinline__ void store8(T *p, int valid, const F8 &x)
{
    if (valid >= 8) {
        if constexpr (sizeof(T) == 4) {
            const u32x4 a = __builtin_bit_cast(u32x4, f32x4{x.v[0], x.v[1], x.v[2], x.v[3]}), b = __builtin_bit_cast(u32x4, f32x4{x.v[4], x.v[5], x.v[6], x.v[7]});
            if constexpr (STREAM) { stream16(p, a); stream16(p + 4, b); }
            else { store16(p, a); store16(p + 4, b); }
        } else {
            const bf16x8 h = {(__bf16)x.v[0], (__bf16)x.v[1], (__bf16)x.v[2], (__bf16)x.v[3], (__bf16)x.v[4], (__bf16)x.v[5], (__bf16)x.v[6], (__bf16)x.v[7]};
            if constexpr (STREAM) stream16(p, __builtin_bit_cast(u32x4, h));
            else store16(p, __builtin_bit_cast(u32x4, h));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < valid) p[j] = from_f32<T>(x.v[j]);
    }
}

}  // namespace am
