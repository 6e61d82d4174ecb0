// Matrix products of the layers, with their epilogue, for gfx950:  C[m][n] = epilogue(sum_k A(m, k) B(n, k)).
//
//   y  = act(x w^T + b) + r      A = x            B = w            (both hold the summed index k side by side)
//   dx = dz w                    A = dz           B = w            (w's rows are k: "across")
//   dw = dz^T x                  A = dz, across   B = x, across
//
// A workgroup owns a tile of C and walks k in steps of 128 bytes.  LDS holds the step's part of both operands, 16 bytes a chunk;
// an operand that holds k side by side is kept [row][8 chunks] and read as one chunk a lane, one that holds it across is kept
// [k][row] and turned by the transposing LDS read (bf16) or read element by element (fp32).  Which k of a step a lane gets is
// the same for both operands, and a sum does not ask for their order.  Chunks change places so that a wave's reads spread over
// the banks: chunk c of row r lies at c ^ (r & 7); across, pairs of chunks move with k.
// The matrix instruction takes B as its first operand, so that a lane ends with four neighbouring n of one m.  The epilogue passes
// them through LDS, wave by wave, so that eight lanes read and write 128 bytes side by side.
#pragma once
#include "am_elem.h"

namespace am {

constexpr uint32_t kLinearMaxReplicas = 32;
constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4;

// ---------------------------------------------------------------------------------------------
// activations, in fp32
// ---------------------------------------------------------------------------------------------
// exp(-|x|)-based forms: no overflow for any finite z, and NaN stays NaN
__device__ __forceinline__ float sigmoid_f32(float z) { return 1.0f / (1.0f + __expf(-z)); }
__device__ __forceinline__ float gelu_tanh_inner(float z) { return 0.7978845608028654f * (z + 0.044715f * z * z * z); }

template <int ACT> __device__ __forceinline__ float act_f32(float z)
{
    if constexpr (ACT == kActRelu) return z < 0.f ? 0.f : z;
    if constexpr (ACT == kActGelu) return 0.5f * z * (1.0f + erff(z * 0.7071067811865476f));
    if constexpr (ACT == kActGeluTanh) return z * sigmoid_f32(2.0f * gelu_tanh_inner(z));        // (1 + tanh u) / 2 = sigmoid(2 u)
    if constexpr (ACT == kActSilu) return z * sigmoid_f32(z);
    return z;
}

template <int ACT> __device__ __forceinline__ float act_grad_f32(float z)
{
    if constexpr (ACT == kActRelu) return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
    if constexpr (ACT == kActGelu) {
        const float e = __expf(-0.5f * z * z);
        return 0.5f * (1.0f + erff(z * 0.7071067811865476f)) + (e > 0.f ? 0.3989422804014327f * z * e : 0.f);      // (no infinity times zero)
    }
    if constexpr (ACT == kActGeluTanh) {
        const float s = sigmoid_f32(2.0f * gelu_tanh_inner(z));
        const float t = s * (1.0f - s);
        return s + (t > 0.f ? z * t * 1.5957691216057308f * (1.0f + 0.134145f * z * z) : 0.f);
    }
    if constexpr (ACT == kActSilu) {
        const float s = sigmoid_f32(z), t = s * (1.0f - s);
        return s + (t > 0.f ? z * t : 0.f);
    }
    return 1.f;
}

// ---------------------------------------------------------------------------------------------
// arguments
// ---------------------------------------------------------------------------------------------
struct ProductArgs {
    const void *a[kLinearMaxReplicas], *b[kLinearMaxReplicas];
    void *c[kLinearMaxReplicas];
    const void *bias[kLinearMaxReplicas];      // by n; all NULL: none
    const void *add[kLinearMaxReplicas];       // added after the activation, in C's type; all NULL: none (may be C itself)
    void *pre[kLinearMaxReplicas];             // z in the operands' type; all NULL: not kept
    uint32_t m, n, k;
    uint32_t lda, ldb, ldc, ldadd, ldpre;      // elements from row to row as the operands lie in memory
    uint32_t tiles_m, tiles_n, replicas;
    uint32_t act, out_f32;                     // activation; C and what is added are fp32 whatever the operands
    uint32_t splits, split_k;                  // workgroup s of a tile takes k in [s split_k, (s + 1) split_k); split_k is a multiple of the step
    float *partial;                            // [split][replica][m][n] when splits > 1
};

__device__ __forceinline__ void apply_act(uint32_t act, F8 &x)
{
    switch (act) {               // the same for the whole launch
    case kActRelu:
#pragma unroll
        for (int j = 0; j < 8; ++j) x.v[j] = act_f32<kActRelu>(x.v[j]);
        break;
    case kActGelu:
#pragma unroll
        for (int j = 0; j < 8; ++j) x.v[j] = act_f32<kActGelu>(x.v[j]);
        break;
    case kActGeluTanh:
#pragma unroll
        for (int j = 0; j < 8; ++j) x.v[j] = act_f32<kActGeluTanh>(x.v[j]);
        break;
    case kActSilu:
#pragma unroll
        for (int j = 0; j < 8; ++j) x.v[j] = act_f32<kActSilu>(x.v[j]);
        break;
    default: break;
    }
}

__device__ __forceinline__ void add8(F8 &x, const F8 &y)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) x.v[j] += y.v[j];
}

// bias, activation, addition and rounding of eight neighbouring n of row m; `valid` of them are inside
template <typename T>
__device__ __forceinline__ void finish8(const ProductArgs &p, uint32_t rep, uint32_t m, uint32_t n, int valid, const F8 &bias, F8 x)
{
    add8(x, bias);
    if (p.pre[rep]) store8(static_cast<T *>(p.pre[rep]) + (uint64_t)m * p.ldpre + n, valid, x);
    apply_act(p.act, x);
    const uint64_t at = (uint64_t)m * p.ldc + n, from = (uint64_t)m * p.ldadd + n;
    if (sizeof(T) == 2 && p.out_f32) {
        if (p.add[rep]) add8(x, load8(static_cast<const float *>(p.add[rep]) + from, valid));
        store8(static_cast<float *>(p.c[rep]) + at, valid, x);
    } else {
        if (p.add[rep]) add8(x, load8(static_cast<const T *>(p.add[rep]) + from, valid));
        store8(static_cast<T *>(p.c[rep]) + at, valid, x);
    }
}

template <typename T>
__device__ __forceinline__ F8 bias8(const ProductArgs &p, uint32_t rep, uint32_t n, int valid)
{
    return p.bias[rep] ? load8(static_cast<const T *>(p.bias[rep]) + n, valid) : F8{};
}

// ---------------------------------------------------------------------------------------------
// operands
// ---------------------------------------------------------------------------------------------
template <typename T> constexpr int kChunk = 16 / (int)sizeof(T);       // elements of a chunk
template <typename T> constexpr int kStep = 128 / (int)sizeof(T);       // k of a step: eight chunks

// A chunk of which the first `valid` elements exist; the others read as 0.
template <typename T> __device__ __forceinline__ u32x4 load_chunk(const T *p, int valid)
{
    if (valid >= kChunk<T>) return load16(p);
    u32x4 r = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < kChunk<T> - 1; ++j) {
        if (j < valid) {
            if constexpr (sizeof(T) == 4) r[j] = __float_as_uint(p[j]);
            else r[j / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, p[j]) << (16 * (j & 1));
        }
    }
    return r;
}

// One operand's part of a tile: R rows (m or n) by a step of k, brought in by NT threads.
template <typename T, int R, int NT, bool ACROSS>
struct Operand {
    static constexpr int kPerThread = R * 8 / NT;
    static constexpr int kRowChunks = R / kChunk<T>;
    static constexpr int kBytes = R * 128;
    static_assert(R * 8 % NT == 0, "chunks divide over the threads");

    const T *base;
    uint64_t ld;
    int rows_left;           // rows of the operand from this tile's first on

    __device__ __forceinline__ void init(const void *p, uint32_t ld_, uint32_t row0, uint32_t rows)
    {
        ld = ld_;
        base = static_cast<const T *>(p) + (ACROSS ? (uint64_t)row0 : (uint64_t)row0 * ld_);
        rows_left = (int)(rows - row0);
    }
    static __device__ __forceinline__ uint32_t place(int q)       // byte offset in LDS of chunk number q
    {
        if constexpr (ACROSS) {
            const int k = q / kRowChunks, c = q % kRowChunks;
            return (uint32_t)((k * kRowChunks + swizzle(k, c)) * 16);
        } else {
            const int r = q / 8, c = q % 8;
            return (uint32_t)((r * 8 + (c ^ (r & 7))) * 16);
        }
    }
    static __device__ __forceinline__ int swizzle(int k, int c)
    {
        if constexpr (sizeof(T) == 2) return c ^ ((k & 3) << 1);                 // a turned read takes two chunks of four neighbouring k
        else return c ^ (((k >> 2) & (kRowChunks >= 16 ? 3 : 1)) << 2);          // an element read takes four chunks of k, k + 4, k + 8, k + 12
    }
    // this thread's chunks of the step at k0; k_left elements of k exist from there on
    __device__ __forceinline__ void load(u32x4 (&reg)[kPerThread], uint32_t k0, int k_left, int tid) const
    {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const int q = i * NT + tid;
            if constexpr (ACROSS) {
                const int k = q / kRowChunks, r = q % kRowChunks * kChunk<T>;
                reg[i] = load_chunk(base + ((uint64_t)k0 + k) * ld + r, k < k_left ? rows_left - r : 0);
            } else {
                const int r = q / 8, k = q % 8 * kChunk<T>;
                reg[i] = load_chunk(base + (uint64_t)r * ld + k0 + k, r < rows_left ? k_left - k : 0);
            }
        }
    }
    static __device__ __forceinline__ void keep(const u32x4 (&reg)[kPerThread], char *lds, int tid)
    {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) *reinterpret_cast<u32x4 *>(lds + place(i * NT + tid)) = reg[i];
    }
    // What lane `lane` gives the matrix instruction for rows row .. row + 15 in half h of the step: for row + lane % 16 the
    // chunk of k number 4 h + lane / 16.
    static __device__ __forceinline__ u32x4 fragment(const char *lds, int row, int h, int lane)
    {
        const int i = lane & 15, g = lane >> 4;
        if constexpr (!ACROSS) {
            return *reinterpret_cast<const u32x4 *>(lds + place((row + i) * 8 + h * 4 + g));
        } else if constexpr (sizeof(T) == 2) {
            // lane i of sixteen reads four rows of k + i / 4 and gets four k of row i
            typedef __attribute__((address_space(3))) bf16x4 *lds_ptr;
            const int c = row / 8 + ((i >> 1) & 1), k = h * 32 + g * 8 + (i >> 2);
            const char *at = lds + (i & 1) * 8;
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_ptr)(at + (k * kRowChunks + swizzle(k, c)) * 16));
            const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_ptr)(at + ((k + 4) * kRowChunks + swizzle(k + 4, c)) * 16));
            const u32x2 l = __builtin_bit_cast(u32x2, lo), u = __builtin_bit_cast(u32x2, hi);
            return u32x4{l[0], l[1], u[0], u[1]};
        } else {
            const int k = h * 16 + g * 4, r = row + i;
            u32x4 f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = *reinterpret_cast<const uint32_t *>(lds + ((k + j) * kRowChunks + swizzle(k + j, r / 4)) * 16 + (r & 3) * 4);
            return f;
        }
    }
};

template <typename T> __device__ __forceinline__ f32x4 multiply(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
        return c;
    }
}

// Which tile, replica and part of k a workgroup takes.  Workgroup b runs on XCD b mod 8: each XCD gets a contiguous stretch of the
// order, which walks eight rows of tiles at a time, so that what its L2 holds of both operands serves many of its tiles.
struct Where { uint32_t tile_m, tile_n, replica, split; };
__device__ __forceinline__ Where where(const ProductArgs &p, uint32_t block, uint32_t blocks)
{
    const uint32_t xcd = block & 7u, per = blocks >> 3, rest = blocks & 7u;
    uint32_t id = xcd * per + (xcd < rest ? xcd : rest) + (block >> 3);
    const uint32_t tiles = p.tiles_m * p.tiles_n;
    Where w;
    const uint32_t outer = id / tiles;
    id -= outer * tiles;
    w.replica = outer % p.replicas;
    w.split = outer / p.replicas;
    const uint32_t band = id / (8u * p.tiles_n), first = band * 8u, in_band = id - band * 8u * p.tiles_n;
    const uint32_t high = p.tiles_m - first < 8u ? p.tiles_m - first : 8u;
    w.tile_m = first + in_band % high;
    w.tile_n = in_band / high;
    return w;
}

// BM x BN tile, WM x WN waves, each BM / WM by BN / WN.  LDS: two steps of both operands, one read while the next is on its way
// through registers; one barrier a step.
template <typename T, int BM, int BN, int WM, int WN, bool A_ACROSS, bool B_ACROSS>
__global__ void __launch_bounds__(64 * WM * WN, 2)
k_product(const ProductArgs p)
{
    constexpr int NT = 64 * WM * WN, MF = BM / WM / 16, NF = BN / WN / 16;
    using A = Operand<T, BM, NT, A_ACROSS>;
    using B = Operand<T, BN, NT, B_ACROSS>;
    constexpr int kStage = A::kBytes + B::kBytes;
    extern __shared__ __align__(16) char lds[];

    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Where w = where(p, blockIdx.x, gridDim.x);
    const uint32_t m0 = w.tile_m * BM, n0 = w.tile_n * BN;
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    const uint32_t k_first = w.split * p.split_k;
    const uint32_t k_end = p.k - k_first < p.split_k ? p.k : k_first + p.split_k;
    const int steps = (int)((k_end - k_first + kStep<T> - 1) / kStep<T>);

    A a;
    B b;
    a.init(p.a[w.replica], p.lda, m0, p.m);
    b.init(p.b[w.replica], p.ldb, n0, p.n);
    f32x4 acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    u32x4 ra[A::kPerThread], rb[B::kPerThread];
    a.load(ra, k_first, (int)(k_end - k_first), tid);
    b.load(rb, k_first, (int)(k_end - k_first), tid);
    A::keep(ra, lds, tid);
    B::keep(rb, lds + A::kBytes, tid);
    for (int t = 0; t < steps; ++t) {
        __syncthreads();              // step t is in LDS, and nobody reads the other half any more
        const char *cur = lds + (t & 1) * kStage;
        if (t + 1 < steps) {
            const uint32_t k0 = k_first + (uint32_t)(t + 1) * kStep<T>;
            a.load(ra, k0, (int)(k_end - k0), tid);
            b.load(rb, k0, (int)(k_end - k0), tid);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 fa[MF], fb[NF];
#pragma unroll
            for (int j = 0; j < NF; ++j) fb[j] = B::fragment(cur + A::kBytes, wn + j * 16, h, lane);
#pragma unroll
            for (int i = 0; i < MF; ++i) fa[i] = A::fragment(cur, wm + i * 16, h, lane);
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int j = 0; j < NF; ++j) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j]);
        }
        if (t + 1 < steps) {
            char *next = lds + ((t + 1) & 1) * kStage;
            A::keep(ra, next, tid);
            B::keep(rb, next + A::kBytes, tid);
        }
    }

    // The wave's sums through its own part of LDS, at most 64 rows at a time: [row][n], chunks of four n moved by the row.
    constexpr int kRows = BM / WM < 64 ? BM / WM : 64, kCols = BN / WN, kLanesARow = kCols / 8;
    static_assert(kRows * kCols * 4 * WM * WN <= 2 * kStage, "the sums fit");
    char *mine = lds + wave * (kRows * kCols * 4);
    const int col = lane % kLanesARow * 8;
    const uint32_t n = n0 + (uint32_t)(wn + col);
    const int valid = n >= p.n ? 0 : p.n - n < 8u ? (int)(p.n - n) : 8;
    const bool whole = p.splits <= 1u;
    const F8 bias = whole ? bias8<T>(p, w.replica, n, valid) : F8{};
    __syncthreads();
#pragma unroll
    for (int part = 0; part < BM / WM / kRows; ++part) {
#pragma unroll
        for (int i = 0; i < kRows / 16; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                const int row = i * 16 + (lane & 15), c = j * 4 + (lane >> 4);
                *reinterpret_cast<f32x4 *>(mine + (row * (kCols / 4) + (c ^ (row & (kCols / 4 - 1)))) * 16) = acc[part * (kRows / 16) + i][j];
            }
        // (one wave's LDS accesses are done in order)
#pragma unroll 1
        for (int row = lane / kLanesARow; row < kRows; row += 64 / kLanesARow) {
            const uint32_t m = m0 + (uint32_t)(wm + part * kRows + row);
            if (m >= p.m || valid == 0) continue;
            F8 x;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 t = *reinterpret_cast<const f32x4 *>(mine + (row * (kCols / 4) + ((col / 4 + h) ^ (row & (kCols / 4 - 1)))) * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) x.v[h * 4 + j] = t[j];
            }
            if (whole) finish8<T>(p, w.replica, m, n, valid, bias, x);
            else store8(p.partial + (((uint64_t)w.split * p.replicas + w.replica) * p.m + m) * p.n + n, valid, x);
        }
    }
}

// The parts of k that workgroups summed apart, joined in their order, and the epilogue.
template <typename T>
__global__ void __launch_bounds__(256)
k_product_join(const ProductArgs p)
{
    const uint32_t groups = (p.n + 7u) / 8u, rep = blockIdx.z;
    const uint64_t all = (uint64_t)groups * p.m;
    for (uint64_t at = (uint64_t)blockIdx.x * 256u + threadIdx.x; at < all; at += (uint64_t)gridDim.x * 256u) {
        const uint32_t m = (uint32_t)(at / groups), n = (uint32_t)(at % groups) * 8u;
        const int valid = p.n - n < 8u ? (int)(p.n - n) : 8;
        F8 x = {};
        for (uint32_t s = 0; s < p.splits; ++s) add8(x, load8(p.partial + (((uint64_t)s * p.replicas + rep) * p.m + m) * p.n + n, valid));
        finish8<T>(p, rep, m, n, valid, bias8<T>(p, rep, n, valid), x);
    }
}

// ---------------------------------------------------------------------------------------------
// dz = dy act'(z) and its column sums
// ---------------------------------------------------------------------------------------------
struct ColumnArgs {
    const void *dy[kLinearMaxReplicas], *pre[kLinearMaxReplicas];
    void *dz[kLinearMaxReplicas];                // all NULL: not written
    void *db[kLinearMaxReplicas];
    uint32_t m, n, lddy, ldpre, lddz;
    uint32_t rows_per_part, parts, accumulate;
    float *partial;                              // [replica][part][n]; NULL: no sums wanted
};

// A workgroup takes 256 columns of rows_per_part rows: eight rows at a time, eight columns a thread.
template <typename T, int ACT>
__global__ void __launch_bounds__(256)
k_columns(const ColumnArgs p)
{
    __shared__ float sums[8][256];
    const uint32_t rep = blockIdx.z, tid = threadIdx.x, c = tid & 31u, r = tid >> 5;
    const uint32_t n = blockIdx.x * 256u + c * 8u;
    const int valid = p.n <= n ? 0 : (p.n - n < 8u ? (int)(p.n - n) : 8);
    const uint32_t first = blockIdx.y * p.rows_per_part, last = p.m - first < p.rows_per_part ? p.m : first + p.rows_per_part;
    F8 acc = {};
    if (valid > 0) {
        for (uint32_t m = first + r; m < last; m += 8u) {
            F8 d = load8(static_cast<const T *>(p.dy[rep]) + (uint64_t)m * p.lddy + n, valid);
            if constexpr (ACT != kActNone) {
                const F8 z = load8(static_cast<const T *>(p.pre[rep]) + (uint64_t)m * p.ldpre + n, valid);
#pragma unroll
                for (int j = 0; j < 8; ++j) d.v[j] *= act_grad_f32<ACT>(z.v[j]);
            }
            if (p.dz[rep]) store8(static_cast<T *>(p.dz[rep]) + (uint64_t)m * p.lddz + n, valid, d);
            add8(acc, d);
        }
    }
    if (!p.partial) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[r][c * 8u + j] = acc.v[j];
    __syncthreads();
    const uint32_t col = blockIdx.x * 256u + tid;
    if (col >= p.n) return;
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += sums[j][tid];
    p.partial[((uint64_t)rep * p.parts + blockIdx.y) * p.n + col] = s;
}

// the parts of a column's sum in their order; no parts: zero
template <typename O>
__global__ void __launch_bounds__(256)
k_columns_join(const ColumnArgs p)
{
    const uint32_t rep = blockIdx.y, n = blockIdx.x * 256u + threadIdx.x;
    if (n >= p.n) return;
    double s = 0.;
    for (uint32_t i = 0; i < p.parts; ++i) s += (double)p.partial[((uint64_t)rep * p.parts + i) * p.n + n];
    O *out = static_cast<O *>(p.db[rep]) + n;
    *out = from_f32<O>((float)(p.accumulate ? s + (double)to_f32(*out) : s));
}

// clears rows of one length (a gradient of no rows)
template <typename O>
__global__ void __launch_bounds__(256)
k_clear(const ProductArgs p, uint64_t elements)
{
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < elements; i += (uint64_t)gridDim.x * 256u) static_cast<O *>(p.c[blockIdx.y])[i] = from_f32<O>(0.f);
}

}  // namespace am
