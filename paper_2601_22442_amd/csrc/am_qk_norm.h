// Norms and rotation of queries and keys, forward and backward.
//
//   r = 1 / sqrt(mean x^2 + eps),  n = r x,  u = n g,  pairs (a, b) of u -> (a c - b s, b c + a s)
//   backward:  du = the pairs of d turned back (a c + b s, b c - a s),  dg = sum du n,  dn = du g,  dx = r (dn - n mean(dn n))
//
// Bound by memory: a head is read once and written once.  A head belongs to a few neighbouring lanes, each of which holds both
// elements of V pairs, so that the rotation needs no exchange and the mean is a butterfly among those lanes.  Pairs that are not
// rotated take c = 1, s = 0.  V = 8 (pairs lie in whole chunks of eight elements) or 1 (anything).
#pragma once
#include "am_elem.h"

namespace am {

constexpr uint32_t kQkMaxReplicas = 32;
constexpr int kQkThreads = 256;

struct QkArgs {
    const void *x[2][kQkMaxReplicas];            // q, k
    const void *gain[2][kQkMaxReplicas];
    void *out[2][kQkMaxReplicas];                // forward: the result; backward: dx
    const void *d[2][kQkMaxReplicas];            // backward: the result's gradient
    const int32_t *positions[kQkMaxReplicas];    // all NULL: token mod rows
    const float *cos, *sin;
    uint64_t stride[2];                          // of x from token to token
    uint32_t tokens, heads[2], dim, rotated, interleaved, rows;
    uint32_t want_gain[2];                       // backward: the gain's gradient is wanted
    uint32_t parts;                              // backward: workgroups of a replica
    float eps;
    float *partial;                              // backward: [replica][part][q, k][dim]
};

// Where the elements of pair j of a head are: the first at place_a, the second at place_a + place_step; and the column of the table (rotated pairs only)
__device__ __forceinline__ uint32_t place_a(const QkArgs &p, uint32_t j)
{
    const uint32_t half = p.rotated / 2u;
    if (j < half) return p.interleaved ? 2u * j : j;
    return p.rotated + (p.interleaved ? 2u * (j - half) : j - half);
}
__device__ __forceinline__ uint32_t place_step(const QkArgs &p, uint32_t j)
{
    if (p.interleaved) return 1u;
    return j < p.rotated / 2u ? p.rotated / 2u : (p.dim - p.rotated) / 2u;
}

// V pairs from pair j on, of which `valid` (V = 1) or all (V = 8) exist
template <typename T, int V>
__device__ __forceinline__ void load_pairs(const QkArgs &p, const T *head, uint32_t j, float (&a)[V], float (&b)[V])
{
    const T *at = head + place_a(p, j);
    if constexpr (V == 8) {
        if (p.interleaved) {
            const F8 l = load8(at, 8), h = load8(at + 8, 8);
#pragma unroll
            for (int i = 0; i < 4; ++i) { a[i] = l.v[2 * i]; b[i] = l.v[2 * i + 1]; a[4 + i] = h.v[2 * i]; b[4 + i] = h.v[2 * i + 1]; }
        } else {
            const F8 l = load8(at, 8), h = load8(at + place_step(p, j), 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) { a[i] = l.v[i]; b[i] = h.v[i]; }
        }
    } else {
        a[0] = to_f32(at[0]);
        b[0] = to_f32(at[place_step(p, j)]);
    }
}

template <typename T, int V>
__device__ __forceinline__ void store_pairs(const QkArgs &p, T *head, uint32_t j, const float (&a)[V], const float (&b)[V])
{
    T *at = head + place_a(p, j);
    if constexpr (V == 8) {
        F8 l, h;
        if (p.interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { l.v[2 * i] = a[i]; l.v[2 * i + 1] = b[i]; h.v[2 * i] = a[4 + i]; h.v[2 * i + 1] = b[4 + i]; }
            store8(at, 8, l);
            store8(at + 8, 8, h);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) { l.v[i] = a[i]; h.v[i] = b[i]; }
            store8(at, 8, l);
            store8(at + place_step(p, j), 8, h);
        }
    } else {
        at[0] = from_f32<T>(a[0]);
        at[place_step(p, j)] = from_f32<T>(b[0]);
    }
}

template <int V>
__device__ __forceinline__ void load_angles(const QkArgs &p, uint32_t row, uint32_t j, float (&c)[V], float (&s)[V])
{
    const uint32_t half = p.rotated / 2u;
    if (j >= half) {
#pragma unroll
        for (int i = 0; i < V; ++i) { c[i] = 1.f; s[i] = 0.f; }
    } else if (row >= p.rows) {
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = s[i] = __builtin_nanf("");
    } else {
        const float *pc = p.cos + (uint64_t)row * half + j, *ps = p.sin + (uint64_t)row * half + j;
        if constexpr (V == 8) {
            const F8 x = load8(pc, 8), y = load8(ps, 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) { c[i] = x.v[i]; s[i] = y.v[i]; }
        } else {
            c[0] = pc[0];
            s[0] = ps[0];
        }
    }
}

// sum over the `lanes` (a power of two) neighbouring lanes of a head
__device__ __forceinline__ float sum_lanes(float x, int lanes)
{
    for (int off = 1; off < lanes; off <<= 1) x += __shfl_xor(x, off, 64);
    return x;
}

struct QkHead { uint32_t token, which, head; };      // which: 0 = q, 1 = k
__device__ __forceinline__ QkHead head_of(const QkArgs &p, uint64_t at)
{
    const uint32_t all = p.heads[0] + p.heads[1];
    QkHead h;
    h.token = (uint32_t)(at / all);
    h.head = (uint32_t)(at % all);
    h.which = h.head >= p.heads[0];
    h.head -= h.which ? p.heads[0] : 0u;
    return h;
}

// V pairs a lane, N times; L lanes a head.  grid = (parts, replicas); heads are dealt out in turn.
template <typename T, int V, int N, bool BACKWARD>
__global__ void __launch_bounds__(kQkThreads)
k_qk_norm(const QkArgs p, const int lanes)
{
    extern __shared__ float sums[];               // backward: [q, k][groups of the workgroup][dim]
    const uint32_t rep = blockIdx.y, lane = threadIdx.x & (uint32_t)(lanes - 1), group = threadIdx.x / (uint32_t)lanes;
    const uint32_t groups = kQkThreads / (uint32_t)lanes, pairs = p.dim / 2u;
    const uint64_t all = (uint64_t)p.tokens * (p.heads[0] + p.heads[1]), stride = (uint64_t)gridDim.x * groups;
    const float inv = 1.f / (float)p.dim;
    float ga[2][N][V], gb[2][N][V], da[2][N][V], db[2][N][V];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t j = (lane + (uint32_t)(k * lanes)) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) ga[w][k][i] = gb[w][k][i] = da[w][k][i] = db[w][k][i] = 0.f;
            if (p.heads[w] && j < pairs) load_pairs<T, V>(p, static_cast<const T *>(p.gain[w][rep]), j, ga[w][k], gb[w][k]);
        }
    // every lane of a head's group takes part in each turn, so that the butterflies stay whole
    for (uint64_t at = (uint64_t)blockIdx.x * groups + group; at < all; at += stride) {
        const QkHead h = head_of(p, at);
        const uint32_t w = h.which;
        const uint64_t dense = ((uint64_t)h.token * p.heads[w] + h.head) * p.dim;
        const T *x = static_cast<const T *>(p.x[w][rep]) + (uint64_t)h.token * p.stride[w] + (uint64_t)h.head * p.dim;
        const uint32_t row = p.positions[rep] ? (uint32_t)p.positions[rep][h.token] : p.rows ? h.token % p.rows : 0u;
        float a[N][V], b[N][V], ea[N][V], eb[N][V], c[N][V], s[N][V], square = 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t j = (lane + (uint32_t)(k * lanes)) * V;
            if (j < pairs) {
                load_pairs<T, V>(p, x, j, a[k], b[k]);
                if constexpr (BACKWARD) load_pairs<T, V>(p, static_cast<const T *>(p.d[w][rep]) + dense, j, ea[k], eb[k]);
                load_angles<V>(p, row, j, c[k], s[k]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) a[k][i] = b[k][i] = ea[k][i] = eb[k][i] = c[k][i] = s[k][i] = 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) square += a[k][i] * a[k][i] + b[k][i] * b[k][i];
        const float r = rsqrtf(sum_lanes(square, lanes) * inv + p.eps);
        T *out = static_cast<T *>(p.out[w][rep]) + dense;
        if constexpr (!BACKWARD) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const uint32_t j = (lane + (uint32_t)(k * lanes)) * V;
                float oa[V], ob[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float ua = a[k][i] * r * (w ? ga[1][k][i] : ga[0][k][i]), ub = b[k][i] * r * (w ? gb[1][k][i] : gb[0][k][i]);
                    oa[i] = ua * c[k][i] - ub * s[k][i];
                    ob[i] = ub * c[k][i] + ua * s[k][i];
                }
                if (j < pairs) store_pairs<T, V>(p, out, j, oa, ob);
            }
        } else {
            float dot = 0.f;
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float ua = ea[k][i] * c[k][i] + eb[k][i] * s[k][i], ub = eb[k][i] * c[k][i] - ea[k][i] * s[k][i];
                    a[k][i] *= r;
                    b[k][i] *= r;
                    const float sa = ua * a[k][i], sb = ub * b[k][i];
                    if (w) { da[1][k][i] += sa; db[1][k][i] += sb; }
                    else { da[0][k][i] += sa; db[0][k][i] += sb; }
                    ea[k][i] = ua * (w ? ga[1][k][i] : ga[0][k][i]);
                    eb[k][i] = ub * (w ? gb[1][k][i] : gb[0][k][i]);
                    dot += ea[k][i] * a[k][i] + eb[k][i] * b[k][i];
                }
            const float mean = sum_lanes(dot, lanes) * inv;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const uint32_t j = (lane + (uint32_t)(k * lanes)) * V;
                float oa[V], ob[V];
#pragma unroll
                for (int i = 0; i < V; ++i) { oa[i] = r * (ea[k][i] - a[k][i] * mean); ob[i] = r * (eb[k][i] - b[k][i] * mean); }
                if (j < pairs) store_pairs<T, V>(p, out, j, oa, ob);
            }
        }
    }
    if constexpr (BACKWARD) {
        // the groups' sums, joined in their order; one of q and k after the other, so that LDS holds one
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            if (!p.want_gain[w]) continue;            // (the same for the whole launch)
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const uint32_t j = (lane + (uint32_t)(k * lanes)) * V;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (j + i < pairs) {
                        const uint32_t pa = place_a(p, j + i);
                        sums[group * p.dim + pa] = da[w][k][i];
                        sums[group * p.dim + pa + place_step(p, j + i)] = db[w][k][i];
                    }
            }
            __syncthreads();
            for (uint32_t e = threadIdx.x; e < p.dim; e += kQkThreads) {
                float t = 0.f;
                for (uint32_t g = 0; g < groups; ++g) t += sums[g * p.dim + e];
                p.partial[(((uint64_t)rep * p.parts + blockIdx.x) * 2u + w) * p.dim + e] = t;
            }
        }
    }
}

struct QkGainArgs {
    void *dgain[2][kQkMaxReplicas];
    const float *partial;
    uint32_t parts, dim, accumulate;
};

// grid = (elements / 16, q or k, replicas): sixteen elements by sixteen shares of the parts, joined in fp64 in a fixed order
template <typename O>
__global__ void __launch_bounds__(256)
k_qk_gain(const QkGainArgs p)
{
    __shared__ double red[16][17];
    O *out = static_cast<O *>(p.dgain[blockIdx.y][blockIdx.z]);
    if (!out) return;
    const uint32_t i = threadIdx.x & 15u, r = threadIdx.x >> 4, e = blockIdx.x * 16u + i;
    double t = 0.;
    if (e < p.dim)
        for (uint32_t k = r; k < p.parts; k += 16u) t += (double)p.partial[(((uint64_t)blockIdx.z * p.parts + k) * 2u + blockIdx.y) * p.dim + e];
    red[r][i] = t;
    __syncthreads();
    if (r == 0u && e < p.dim) {
        for (int k = 1; k < 16; ++k) t += red[k][i];
        if (p.accumulate) t += (double)to_f32(out[e]);
        out[e] = from_f32<O>((float)t);
    }
}

}  // namespace am
