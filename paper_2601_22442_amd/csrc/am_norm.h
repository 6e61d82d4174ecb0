// The global gradient norm over many tensors, for clipping:  norm = sqrt(sum g^2),  factor = norm <= max ? 1 : max / norm,  g <- factor g.
//
// Bound by memory: a gradient is read once for the norm (and written once when it is packed into the flat array), and once more
// for the product with the factor, which no store can precede.  The tensors of a launch travel as kernel arguments, so a call copies nothing
// to the device; each is cut into parts of a fixed length, one workgroup a part.  Squares are summed in fp64, in an order that
// depends on the sizes alone: a float's square neither overflows nor vanishes there.  Packing 8 x 117M bf16 gradients of 30 tensors takes 683 us for
// 3.76 GB (5.5 TB/s); clipping 2 x 3.2M fp32 in 24 tensors at odd places 6.8 + 9.7 us.
#pragma once
#include "am_elem.h"

namespace am {

constexpr uint32_t kNormMaxReplicas = 32;
constexpr uint32_t kNormPointers = 304;      // replicas x tensors of a launch: the arguments stay below 4 KB
constexpr uint32_t kNormTensors = 64;        // tensors of a launch

struct NormTable {
    void *g[kNormPointers];                  // [replica][tensor of this launch]
    void *out[kNormMaxReplicas];             // flat arrays, all NULL: none
    uint64_t at[kNormTensors];               // where a tensor starts in a flat array
    uint64_t numel[kNormTensors];
    uint32_t first_part[kNormTensors + 1];   // of a tensor, among this launch's parts
    uint64_t bf16;                           // bit of a tensor: bf16, else fp32
    uint32_t tensors, part_elements;
    uint32_t parts_before, parts_all;        // parts of a replica in the launches before this one, and in all of them
    uint32_t out_bf16;
};
static_assert(sizeof(NormTable) < 4096, "kernel arguments");

constexpr int kNormThreads = 256;

// A part of one tensor: every thread takes 16 bytes at a time.  use(element index, number of valid elements, values)
template <typename T, typename F>
__device__ __forceinline__ void each_vector(const T *g, uint64_t first, uint64_t last, F use)
{
    constexpr int V = 16 / (int)sizeof(T);
    constexpr int U = 4;                     // loads of a thread on their way
    for (uint64_t i = first + threadIdx.x * V; i < last; i += (uint64_t)kNormThreads * V * U) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t e = i + (uint64_t)u * kNormThreads * V;
            if (e + V <= last) raw[u] = load16(g + e);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t e = i + (uint64_t)u * kNormThreads * V;
            if (e >= last) continue;
            const int valid = last - e < (uint64_t)V ? (int)(last - e) : V;
            float x[V];
            if (valid == V) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if constexpr (sizeof(T) == 4) x[j] = __uint_as_float(raw[u][j]);
                    else x[j] = __uint_as_float(j & 1 ? raw[u][j / 2] & 0xFFFF0000u : raw[u][j / 2] << 16);
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] = j < valid ? to_f32(g[e + j]) : 0.f;
            }
            use(e, valid, x);
        }
    }
}

template <typename O, int V>
__device__ __forceinline__ void store_vector(O *p, int valid, const float (&x)[V])
{
    if (valid == V) {
        if constexpr (sizeof(O) == 4) {
#pragma unroll
            for (int h = 0; h < V / 4; ++h) store16(p + 4 * h, __builtin_bit_cast(u32x4, f32x4{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]}));
        } else if constexpr (V == 8) {
            const bf16x8 h = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3], (__bf16)x[4], (__bf16)x[5], (__bf16)x[6], (__bf16)x[7]};
            store16(p, __builtin_bit_cast(u32x4, h));
        } else {
            const bf16x4 h = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
            store8bytes(p, __builtin_bit_cast(u32x2, h));
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < valid) p[j] = from_f32<O>(x[j]);
    }
}

// which tensor of the launch part `part` belongs to
__device__ __forceinline__ uint32_t tensor_of(const NormTable &a, uint32_t part)
{
    uint32_t lo = 0, hi = a.tensors;         // first_part[lo] <= part < first_part[hi]
    while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) / 2u;
        if (a.first_part[mid] <= part) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double sum_of_workgroup(double x)
{
    __shared__ double red[kNormThreads];
    red[threadIdx.x] = x;
    __syncthreads();
    for (uint32_t off = kNormThreads / 2; off > 0; off >>= 1) {
        if (threadIdx.x < off) red[threadIdx.x] += red[threadIdx.x + off];
        __syncthreads();
    }
    return red[0];
}

// grid = (parts, replicas).  PACK: 0 = no flat arrays, 1 = fp32, 2 = bf16
template <typename T, int PACK>
__device__ __forceinline__ double norm_part(const T *g, void *out, uint64_t first, uint64_t last)
{
    double acc = 0.;
    each_vector(g, first, last, [&](uint64_t e, int valid, const auto &x) {
        constexpr int V = 16 / (int)sizeof(T);
#pragma unroll
        for (int j = 0; j < V; ++j) acc += (double)x[j] * (double)x[j];
        if constexpr (PACK == 1) store_vector<float>(static_cast<float *>(out) + e, valid, x);
        if constexpr (PACK == 2) store_vector<__bf16>(static_cast<__bf16 *>(out) + e, valid, x);
    });
    return acc;
}

template <int PACK>
__global__ void __launch_bounds__(kNormThreads)
k_norm_parts(const NormTable a, double *__restrict__ partial)
{
    const uint32_t part = blockIdx.x, rep = blockIdx.y, t = tensor_of(a, part);
    const uint64_t first = (uint64_t)(part - a.first_part[t]) * a.part_elements;
    const uint64_t last = a.numel[t] - first < a.part_elements ? a.numel[t] : first + a.part_elements;
    const void *g = a.g[rep * a.tensors + t];
    char *out = static_cast<char *>(a.out[rep]) + a.at[t] * (PACK == 2 ? 2u : 4u);
    const double acc = (a.bf16 >> t) & 1u ? norm_part<__bf16, PACK>(static_cast<const __bf16 *>(g), out, first, last)
                                          : norm_part<float, PACK>(static_cast<const float *>(g), out, first, last);
    const double sum = sum_of_workgroup(acc);
    if (threadIdx.x == 0) partial[(uint64_t)rep * a.parts_all + a.parts_before + part] = sum;
}

// What follows from a replica's parts: the same sum, in the same order, wherever it is formed.  By a whole workgroup.
struct NormAndFactor { float norm, factor; };
__device__ __forceinline__ NormAndFactor norm_of_parts(const double *__restrict__ partial, uint32_t parts, double max_norm)
{
    double acc = 0.;
#pragma unroll 8
    for (uint32_t i = threadIdx.x; i < parts; i += kNormThreads) acc += partial[i];
    const double n = sqrt(sum_of_workgroup(acc));
    return {(float)n, n <= max_norm ? 1.f : (float)(max_norm / n)};
}

// one workgroup a replica
__global__ void __launch_bounds__(kNormThreads)
k_norm_finish(const double *__restrict__ partial, uint32_t parts, double max_norm, float *__restrict__ norm, float *__restrict__ factor)
{
    const NormAndFactor r = norm_of_parts(partial + (uint64_t)blockIdx.x * parts, parts, max_norm);
    if (threadIdx.x == 0) { norm[blockIdx.x] = r.norm; factor[blockIdx.x] = r.factor; }
}

template <typename T, typename O>
__device__ __forceinline__ void scale_part(const T *g, O *out, uint64_t first, uint64_t last, float factor)
{
    each_vector(g, first, last, [&](uint64_t e, int valid, const auto &x) {
        constexpr int V = 16 / (int)sizeof(T);
        float y[V];
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = x[j] * factor;
        store_vector(out + e, valid, y);
    });
}

// grid = (parts, replicas); without flat arrays in place, where a factor of one leaves nothing to do.  FINISH: every workgroup forms its
// replica's factor itself, and the first ones of the call's first launch write it down.
template <bool FINISH>
__global__ void __launch_bounds__(kNormThreads)
k_norm_scale(const NormTable a, const double *__restrict__ partial, double max_norm, float *__restrict__ norm, float *__restrict__ factors)
{
    const uint32_t part = blockIdx.x, rep = blockIdx.y, t = tensor_of(a, part);
    float factor;
    if constexpr (FINISH) {
        const NormAndFactor r = norm_of_parts(partial + (uint64_t)rep * a.parts_all, a.parts_all, max_norm);
        factor = r.factor;
        if (part == 0u && a.parts_before == 0u && threadIdx.x == 0) { norm[rep] = r.norm; factors[rep] = r.factor; }
    } else {
        factor = factors[rep];
    }
    const uint64_t first = (uint64_t)(part - a.first_part[t]) * a.part_elements;
    const uint64_t last = a.numel[t] - first < a.part_elements ? a.numel[t] : first + a.part_elements;
    void *g = a.g[rep * a.tensors + t];
    const bool bf16 = (a.bf16 >> t) & 1u;
    if (!a.out[rep]) {
        if (factor == 1.f) return;
        if (bf16) scale_part(static_cast<const __bf16 *>(g), static_cast<__bf16 *>(g), first, last, factor);
        else scale_part(static_cast<const float *>(g), static_cast<float *>(g), first, last, factor);
    } else if (a.out_bf16) {
        __bf16 *out = static_cast<__bf16 *>(a.out[rep]) + a.at[t];
        if (bf16) scale_part(static_cast<const __bf16 *>(g), out, first, last, factor);
        else scale_part(static_cast<const float *>(g), out, first, last, factor);
    } else {
        float *out = static_cast<float *>(a.out[rep]) + a.at[t];
        if (bf16) scale_part(static_cast<const __bf16 *>(g), out, first, last, factor);
        else scale_part(static_cast<const float *>(g), out, first, last, factor);
    }
}

}  // namespace am
