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
    uint32_t k_whole;                          // k rounded up to whole chunks where the operand that holds it side by side has zeros there, else k
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

static __device__ const u32x4 zero_chunk = {0u, 0u, 0u, 0u};

// One operand's part of a tile: R rows (m or n) by a step of S chunks of k (eight or four), brought in by NT threads.
template <typename T, int R, int NT, bool ACROSS, int S>
struct Operand {
    static constexpr int kStep = S * kChunk<T>;              // k of a step
    static constexpr int kPerThread = R * S / NT;
    static constexpr int kRowChunks = R / kChunk<T>;
    static constexpr int kBytes = R * S * 16;
    static_assert(R * S % NT == 0 && (S == 8 || S == 4), "chunks divide over the threads");

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
            const int r = q / S;
            return (uint32_t)((r * S + turned(r, q % S)) * 16);
        }
    }
    static __device__ __forceinline__ int turned(int r, int c) { return S == 8 ? c ^ (r & 7) : c ^ (r >> 1 & 3); }      // eight rows, 128 bytes of banks
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
                const int r = q / S, k = q % S * kChunk<T>;
                reg[i] = load_chunk(base + (uint64_t)r * ld + k0 + k, r < rows_left ? k_left - k : 0);
            }
        }
    }
    // The same straight from memory into LDS, for operands in whole chunks (see direct_ok on the host): one wave's share of the
    // chunks, in the order they have in LDS, so a lane asks for the chunk whose place is its own.  offset[]: bytes from
    // base at k = 0, found once.  Rows past the end repeat the last ones (their products are not stored); chunks past the end of k are zeros.
    __device__ __forceinline__ void offsets(uint32_t (&offset)[kPerThread], int wave, int lane) const
    {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const int q = (wave * kPerThread + i) * 64 + lane;
            if constexpr (ACROSS) {
                const int k = q / kRowChunks, r = swizzle(k, q % kRowChunks) * kChunk<T>, last = (rows_left - 1) / kChunk<T> * kChunk<T>;
                offset[i] = (uint32_t)(k * (uint32_t)ld + (r < last ? r : last)) * (uint32_t)sizeof(T);
            } else {
                const int r = q / S, c = turned(r, q % S);
                offset[i] = (uint32_t)((r < rows_left ? r : rows_left - 1) * (uint32_t)ld + c * kChunk<T>) * (uint32_t)sizeof(T);
            }
        }
    }
    __device__ __forceinline__ void direct(char *lds, const uint32_t (&offset)[kPerThread], uint32_t k0, int k_left, int wave, int lane) const
    {
        const char *from = reinterpret_cast<const char *>(base + (ACROSS ? (uint64_t)k0 * ld : (uint64_t)k0));
        char *to = lds + wave * kPerThread * 1024;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const char *at = from + offset[i];
            if (k_left < kStep) {                 // (the last step alone)
                const int q = (wave * kPerThread + i) * 64 + lane;
                const int k = ACROSS ? q / kRowChunks : turned(q / S, q % S) * kChunk<T>;
                at = k < k_left ? at : reinterpret_cast<const char *>(&zero_chunk);
            }
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)at, (__attribute__((address_space(3))) void *)(to + i * 1024), 16, 0, 0);
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
            return *reinterpret_cast<const u32x4 *>(lds + place((row + i) * S + h * 4 + g));
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

// The wave's sums (rows wm of the tile at m0, columns wn of that at n0) through its own part of LDS, at most 64 rows at a time, kept
// [row][n] with chunks of four n moved by the row, then the epilogue.
template <typename T, int ROWS, int COLS>
__device__ __forceinline__ void finish_wave(const ProductArgs &p, const Where &w, f32x4 (&acc)[ROWS / 16][COLS / 16], char *lds, uint32_t m_first, uint32_t n_first, int wave, int lane)
{
    constexpr int kRows = ROWS < 64 ? ROWS : 64, kCols = COLS, kLanesARow = kCols / 8;
    char *mine = lds + wave * (kRows * kCols * 4);
    const int col = lane % kLanesARow * 8;
    const uint32_t n = n_first + (uint32_t)col;
    const int valid = n >= p.n ? 0 : p.n - n < 8u ? (int)(p.n - n) : 8;
    const bool whole = p.splits <= 1u;
    const F8 bias = whole ? bias8<T>(p, w.replica, n, valid) : F8{};
#pragma unroll
    for (int part = 0; part < ROWS / kRows; ++part) {
#pragma unroll
        for (int i = 0; i < kRows / 16; ++i)
#pragma unroll
            for (int j = 0; j < COLS / 16; ++j) {
                const int row = i * 16 + (lane & 15), c = j * 4 + (lane >> 4);
                *reinterpret_cast<f32x4 *>(mine + (row * (kCols / 4) + (c ^ (row & (kCols / 4 - 1)))) * 16) = acc[part * (kRows / 16) + i][j];
            }
        // (one wave's LDS accesses are done in order)
#pragma unroll 1
        for (int row = lane / kLanesARow; row < kRows; row += 64 / kLanesARow) {
            const uint32_t m = m_first + (uint32_t)(part * kRows + row);
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

// A step's products of one wave: cur holds the step, and what `ahead` writes meanwhile lies elsewhere in LDS.
template <typename T, typename A, typename B, int MF, int NF>
__device__ __forceinline__ void products(const char *__restrict__ cur, f32x4 (&acc)[MF][NF], int wm, int wn, int lane)
{
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
}

// The next step's chunks set out for `next`, then the products of the step in `cur`.
template <typename T, typename A, typename B, int MF, int NF>
__device__ __forceinline__ void direct_step(const char *__restrict__ cur, char *__restrict__ next, const A &a, const B &b,
                                            const uint32_t (&oa)[A::kPerThread], const uint32_t (&ob)[B::kPerThread], uint32_t k0, int ka, int kb,
                                            bool more, f32x4 (&acc)[MF][NF], int wm, int wn, int wave, int lane)
{
    if (more) {
        a.direct(next, oa, k0, ka, wave, lane);
        b.direct(next + A::kBytes, ob, k0, kb, wave, lane);
    }
    products<T, A, B, MF, NF>(cur, acc, wm, wn, lane);
}

// BM x BN tile, WM x WN waves, each BM / WM by BN / WN.  LDS: two steps of both operands, one read while the next is on its way
// (DIRECT: straight from memory, else through registers); one barrier a step.
template <typename T, int BM, int BN, int WM, int WN, bool A_ACROSS, bool B_ACROSS, bool DIRECT>
__global__ void __launch_bounds__(64 * WM * WN, 2)
k_product(const ProductArgs p)
{
    constexpr int NT = 64 * WM * WN, MF = BM / WM / 16, NF = BN / WN / 16;
    using A = Operand<T, BM, NT, A_ACROSS, 8>;
    using B = Operand<T, BN, NT, B_ACROSS, 8>;
    constexpr int kStep = A::kStep;
    constexpr int kStage = A::kBytes + B::kBytes;
    extern __shared__ __align__(16) char lds[];

    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Where w = where(p, blockIdx.x, gridDim.x);
    const uint32_t m0 = w.tile_m * BM, n0 = w.tile_n * BN;
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    const uint32_t k_first = w.split * p.split_k;
    const uint32_t k_end = p.k - k_first < p.split_k ? p.k : k_first + p.split_k;
    const int steps = (int)((k_end - k_first + kStep - 1) / kStep);

    A a;
    B b;
    a.init(p.a[w.replica], p.lda, m0, p.m);
    b.init(p.b[w.replica], p.ldb, n0, p.n);
    f32x4 acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    if constexpr (DIRECT) {
        uint32_t oa[A::kPerThread], ob[B::kPerThread];
        a.offsets(oa, wave, lane);
        b.offsets(ob, wave, lane);
        // k_end is that of k as it is summed; an operand that holds k side by side has zeros up to a whole chunk
        const int extra = (int)(p.k_whole - p.k);
        int left = (int)(k_end - k_first);
        const auto ends = [&](int l, bool across) { return across ? l : l + extra; };
        a.direct(lds, oa, k_first, ends(left, A_ACROSS), wave, lane);
        b.direct(lds + A::kBytes, ob, k_first, ends(left, B_ACROSS), wave, lane);
        for (int t = 0; t < steps; ++t) {
            __syncthreads();              // step t has come, and nobody reads the other half any more
            left -= kStep;
            direct_step<T, A, B, MF, NF>(lds + (t & 1) * kStage, lds + ((t + 1) & 1) * kStage, a, b, oa, ob, k_first + (uint32_t)(t + 1) * kStep,
                                         ends(left, A_ACROSS), ends(left, B_ACROSS), t + 1 < steps, acc, wm, wn, wave, lane);
        }
    } else {
        u32x4 ra[A::kPerThread], rb[B::kPerThread];
        a.load(ra, k_first, (int)(k_end - k_first), tid);
        b.load(rb, k_first, (int)(k_end - k_first), tid);
        A::keep(ra, lds, tid);
        B::keep(rb, lds + A::kBytes, tid);
        for (int t = 0; t < steps; ++t) {
            __syncthreads();              // step t is in LDS, and nobody reads the other half any more
            if (t + 1 < steps) {
                const uint32_t k0 = k_first + (uint32_t)(t + 1) * kStep;
                a.load(ra, k0, (int)(k_end - k0), tid);
                b.load(rb, k0, (int)(k_end - k0), tid);
            }
            products<T, A, B, MF, NF>(lds + (t & 1) * kStage, acc, wm, wn, lane);
            if (t + 1 < steps) {
                char *next = lds + ((t + 1) & 1) * kStage;
                A::keep(ra, next, tid);
                B::keep(rb, next + A::kBytes, tid);
            }
        }
    }

    __syncthreads();
    static_assert(BM / WM * (BN / WN) * 4 * NT / 64 / (BM / WM > 64 ? BM / WM / 64 : 1) <= 2 * kStage, "the sums fit");
    finish_wave<T, BM / WM, BN / WN>(p, w, acc, lds, m0 + (uint32_t)wm, n0 + (uint32_t)wn, wave, lane);
}

// The 256 x 256 tile of bf16, eight waves of 128 x 64 each, two to a SIMD: while one of the two multiplies, the other reads its
// next fragments from LDS and sets out loads.  Steps of 64 bytes of k in four stages of LDS.  The waves of the second group of
// four run half a step behind: between two barriers group 0 does memory for step q (interval 2q), then products (2q + 1); group 1
// memory in 2q + 1, products in 2q + 2.  What the barriers then promise:
//   step q is read in intervals 2q and 2q + 1, and the reads are over by the end of 2q + 2 (a wave's products wait for them);
//   group 0 sets out step q + 2 in interval 2q, over step q - 2, read until 2q - 2; group 1 sets out its share of step q + 3 in
//   2q + 1, over step q - 1, read until 2q;
//   step q + 1 must be there before interval 2q + 2: group 0 waits for its share at the end of 2q + 1, when steps q + 1 and q + 2
//   are on their way, group 1 at the end of 2q + 1 too, with q + 1, q + 2 and q + 3 on their way.
// Steps past the end set out zeros, so that the counts stay.
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
template <int COUNT> __device__ __forceinline__ void wait_loads()      // until at most COUNT vector memory accesses of the wave are on their way
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COUNT) : "memory");
}

template <typename A, typename B, int MF, int NF>
__device__ __forceinline__ void large_fetch(const char *__restrict__ cur, char *__restrict__ ahead, const A &a, const B &b, const uint32_t (&oa)[A::kPerThread],
                                            const uint32_t (&ob)[B::kPerThread], uint32_t k0, int ka, int kb, u32x4 (&fa)[MF], u32x4 (&fb)[NF], int wm, int wn, int wave, int lane)
{
#pragma unroll
    for (int j = 0; j < NF; ++j) fb[j] = B::fragment(cur + A::kBytes, wn + j * 16, 0, lane);
#pragma unroll
    for (int i = 0; i < MF; ++i) fa[i] = A::fragment(cur, wm + i * 16, 0, lane);
    a.direct(ahead, oa, k0, ka, wave, lane);
    b.direct(ahead + A::kBytes, ob, k0, kb, wave, lane);
}

template <bool A_ACROSS, bool B_ACROSS>
__global__ void __launch_bounds__(512, 2)
k_product_large(const ProductArgs p)
{
    typedef __bf16 T;
    constexpr int BM = 256, BN = 256, NT = 512, MF = 8, NF = 4;
    using A = Operand<T, BM, NT, A_ACROSS, 4>;
    using B = Operand<T, BN, NT, B_ACROSS, 4>;
    constexpr int kStep = A::kStep, kStage = A::kBytes + B::kBytes, kLoads = A::kPerThread + B::kPerThread;
    extern __shared__ __align__(16) char lds[];

    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), group = wave >> 2;
    const Where w = where(p, blockIdx.x, gridDim.x);
    const uint32_t m0 = w.tile_m * BM, n0 = w.tile_n * BN;
    const int wm = wave / 4 * 128, wn = wave % 4 * 64;
    const uint32_t k_first = w.split * p.split_k;
    const uint32_t k_end = p.k - k_first < p.split_k ? p.k : k_first + p.split_k;
    const int steps = (int)((k_end - k_first + kStep - 1) / kStep);

    A a;
    B b;
    a.init(p.a[w.replica], p.lda, m0, p.m);
    b.init(p.b[w.replica], p.ldb, n0, p.n);
    uint32_t oa[A::kPerThread], ob[B::kPerThread];
    a.offsets(oa, wave, lane);
    b.offsets(ob, wave, lane);
    f32x4 acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int extra = (int)(p.k_whole - p.k), all = (int)(k_end - k_first);
    const auto set_out = [&](int step) {
        char *to = lds + (step & 3) * kStage;
        const uint32_t k0 = step < steps ? k_first + (uint32_t)step * kStep : k_first;      // (past the end: no address of it is used)
        const int left = all - step * kStep;
        a.direct(to, oa, k0, A_ACROSS ? left : left + extra, wave, lane);
        b.direct(to + A::kBytes, ob, k0, B_ACROSS ? left : left + extra, wave, lane);
    };
    set_out(0);
    set_out(1);
    if (group) { set_out(2); wait_loads<2 * kLoads>(); }
    else wait_loads<kLoads>();
    meet();
    if (group) meet();
    for (int q = 0; q < steps; ++q) {
        u32x4 fa[MF], fb[NF];
        const int s = q + 2 + group, left = all - s * kStep;
        const uint32_t k0 = s < steps ? k_first + (uint32_t)s * kStep : k_first;
        large_fetch<A, B, MF, NF>(lds + (q & 3) * kStage, lds + (s & 3) * kStage, a, b, oa, ob, k0, A_ACROSS ? left : left + extra, B_ACROSS ? left : left + extra,
                                  fa, fb, wm, wn, wave, lane);
        if (group) wait_loads<2 * kLoads>();
        meet();
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j]);
        __builtin_amdgcn_s_setprio(0);
        if (!group) wait_loads<kLoads>();
        meet();
    }
    if (!group) meet();
    wait_loads<0>();
    __syncthreads();
    finish_wave<T, 128, 64>(p, w, acc, lds, m0 + (uint32_t)wm, n0 + (uint32_t)wn, wave, lane);
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
            if (p.dz[rep]) store8(static_cast<T *>(p.dz[rep]) + (uint64_t)m * p.lddz + n, 8, d);       // (rows are padded to eight with zeros)
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
