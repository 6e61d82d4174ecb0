// Host side of am_linear and am_linear_backward: argument checks, the choice of tiles, workspace and launches.
#include <cstring>

#include "am_error.h"
#include "am_linear.h"
#include "am_product_plan.h"

namespace {

using am::ProductArgs;
using am_host::ProductPlan;
using am_host::aligned;
using am_host::fail;

constexpr uint64_t kMaxExtent = 1ull << 31;
enum Form { kRows, kInputGradient, kWeightGradient };      // x w^T; dz w; dz^T x

uint64_t or_dense(uint64_t stride, uint64_t dense) { return stride ? stride : dense; }

am_status check_config(const am_linear_config *c)
{
    if (!c) return fail(AM_EINVAL, "config is NULL");
    if (c->replicas == 0 || c->replicas > AM_MAX_REPLICAS) return fail(AM_EINVAL, "replicas=%u out of range [1, %u]", c->replicas, AM_MAX_REPLICAS);
    if (c->dtype > AM_BF16 || c->grad_dtype > AM_BF16) return fail(AM_EINVAL, "unknown dtype");
    if (c->dtype == AM_F32 && c->grad_dtype == AM_BF16) return fail(AM_EINVAL, "grad_dtype = bf16 needs dtype = bf16");
    if (c->act > AM_ACT_SILU) return fail(AM_EINVAL, "unknown act %u", c->act);
    if (c->rows >= kMaxExtent || c->in == 0 || c->in >= kMaxExtent || c->out == 0 || c->out >= kMaxExtent)
        return fail(AM_EINVAL, "rows=%llu in=%llu out=%llu out of range (in, out >= 1; all below 2^31)", (unsigned long long)c->rows,
                    (unsigned long long)c->in, (unsigned long long)c->out);
    const struct { const char *name; uint64_t stride, least; } strides[] = {
        {"x_stride", c->x_stride, c->in}, {"y_stride", c->y_stride, c->out}, {"pre_stride", c->pre_stride, c->out},
        {"residual_stride", c->residual_stride, c->out}, {"dx_stride", c->dx_stride, c->in}};
    for (const auto &s : strides)
        if (s.stride && (s.stride < s.least || s.stride >= kMaxExtent))
            return fail(AM_EINVAL, "%s=%llu is shorter than a row of %llu or not below 2^31", s.name, (unsigned long long)s.stride, (unsigned long long)s.least);
    return AM_OK;
}

am_status check_table(const char *name, const void *const *p, const am_linear_config &c, uint32_t dtype)
{
    if (!p) return fail(AM_EINVAL, "%s is NULL", name);
    for (uint32_t i = 0; i < c.replicas; ++i) {
        if (!p[i]) return fail(AM_EINVAL, "%s[%u] is NULL", name, i);
        if (!aligned(p[i], dtype == AM_BF16 ? 2 : 4)) return fail(AM_EALIGN, "%s[%u] is not aligned to its elements", name, i);
    }
    return AM_OK;
}

#define AM_TABLE(name, dtype)                                                                                       \
    do {                                                                                                            \
        const am_status s_ = check_table(#name, const_cast<const void *const *>(buf->name), *cfg, dtype);           \
        if (s_ != AM_OK) return s_;                                                                                 \
    } while (0)

am_status check_forward(const am_linear_config *cfg, const am_linear_buffers *buf)
{
    const am_status s = check_config(cfg);
    if (s != AM_OK) return s;
    if (!buf) return fail(AM_EINVAL, "buffers is NULL");
    if (cfg->rows == 0) return AM_OK;
    AM_TABLE(x, cfg->dtype);
    AM_TABLE(w, cfg->dtype);
    AM_TABLE(y, cfg->dtype);
    if (buf->bias) AM_TABLE(bias, cfg->dtype);
    if (buf->residual) AM_TABLE(residual, cfg->dtype);
    if (buf->pre) AM_TABLE(pre, cfg->dtype);
    return AM_OK;
}

am_status check_backward(const am_linear_config *cfg, const am_linear_buffers *buf)
{
    const am_status s = check_config(cfg);
    if (s != AM_OK) return s;
    if (!buf) return fail(AM_EINVAL, "buffers is NULL");
    if (!buf->dx && !buf->dw && !buf->db) return fail(AM_EINVAL, "no gradient is wanted: dx, dw and db are NULL");
    if (buf->dw) AM_TABLE(dw, cfg->grad_dtype);
    if (buf->db) AM_TABLE(db, cfg->grad_dtype);
    if (cfg->rows == 0) return AM_OK;
    AM_TABLE(dy, cfg->dtype);
    if (cfg->act != AM_ACT_NONE) AM_TABLE(pre, cfg->dtype);
    if (buf->dx) { AM_TABLE(dx, cfg->dtype); AM_TABLE(w, cfg->dtype); }
    if (buf->dw) AM_TABLE(x, cfg->dtype);
    return AM_OK;
}

// ---- workspace ------------------------------------------------------------------------------
uint64_t up256(uint64_t x) { return (x + 255u) & ~255ull; }

ProductPlan plan_product(const am_linear_config &c, Form form)
{
    const bool bf16 = c.dtype == AM_BF16;
    if (form == kRows) return am_host::product_plan(bf16, c.replicas, c.rows, c.out, c.in);
    if (form == kInputGradient) return am_host::product_plan(bf16, c.replicas, c.rows, c.in, c.out);
    return am_host::product_plan(bf16, c.replicas, c.out, c.in, c.rows);
}

uint64_t partial_bytes(const am_linear_config &c, Form form)
{
    const ProductPlan p = plan_product(c, form);
    if (p.splits <= 1) return 0;
    const uint64_t elements = form == kRows ? c.rows * c.out : form == kInputGradient ? c.rows * c.in : c.out * c.in;
    return up256(4u * p.splits * c.replicas * elements);
}

// backward: dz | column sums' parts | parts of a product (dx's and dw's take turns)
struct BackwardSpace {
    uint64_t dz_pitch, dz_bytes, sums_bytes, partial, total;
    uint32_t rows_per_part, parts;
};
BackwardSpace backward_space(const am_linear_config &c, const am_linear_buffers &b)
{
    BackwardSpace s = {};
    const uint64_t size = c.dtype == AM_BF16 ? 2u : 4u;
    s.dz_pitch = (c.out + 7u) & ~7ull;
    if (c.act != AM_ACT_NONE && (b.dx || b.dw)) s.dz_bytes = up256(size * c.replicas * c.rows * s.dz_pitch);
    if (b.db || s.dz_bytes) am_host::column_parts(c.replicas, c.rows, c.out, &s.rows_per_part, &s.parts);
    if (b.db) s.sums_bytes = up256(4u * c.replicas * (uint64_t)s.parts * c.out);
    const uint64_t dx = b.dx ? partial_bytes(c, kInputGradient) : 0, dw = b.dw ? partial_bytes(c, kWeightGradient) : 0;
    s.partial = dx > dw ? dx : dw;
    s.total = s.dz_bytes + s.sums_bytes + s.partial;
    return s;
}

am_status check_space(const am_linear_buffers *buf, uint64_t need)
{
    if (need == 0) return AM_OK;
    if (!buf->workspace) return fail(AM_EINVAL, "workspace is NULL, %llu bytes needed", (unsigned long long)need);
    if (!aligned(buf->workspace, 256)) return fail(AM_EALIGN, "workspace is not 256-byte aligned");
    if (buf->workspace_bytes < need)
        return fail(AM_ENOMEM, "workspace has %llu bytes, %llu needed", (unsigned long long)buf->workspace_bytes, (unsigned long long)need);
    return AM_OK;
}

// ---- launches -------------------------------------------------------------------------------
am_status launch_kernel(void (*kernel)(ProductArgs), ProductArgs &a, uint32_t tile, uint32_t threads, uint32_t lds, hipStream_t stream)
{
    a.tiles_m = (a.m + tile - 1) / tile;
    a.tiles_n = (a.n + tile - 1) / tile;
    const uint64_t blocks = (uint64_t)a.tiles_m * a.tiles_n * a.replicas * a.splits;
    if (blocks >= kMaxExtent) return fail(AM_EINVAL, "a product of %llu tiles is too large for one launch", (unsigned long long)blocks);
    if (lds > 65536u) AM_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    kernel<<<(uint32_t)blocks, threads, lds, stream>>>(a);
    AM_HIP(hipGetLastError());
    return AM_OK;
}

template <typename T, int BM, int BN, int WM, int WN, bool AA, bool BA, bool DIRECT>
am_status launch_tiles(ProductArgs &a, hipStream_t stream)
{
    static_assert(BM == BN, "square tiles");
    return launch_kernel(am::k_product<T, BM, BN, WM, WN, AA, BA, DIRECT>, a, BM, 64 * WM * WN, 2u * (BM + BN) * 128u, stream);
}

template <typename T, bool AA, bool BA, bool DIRECT>
am_status launch_shape(ProductArgs &a, const ProductPlan &p, hipStream_t stream)
{
    if constexpr (sizeof(T) == 2) {
        if (p.tile == 256) {
            if constexpr (DIRECT) return launch_kernel(am::k_product_large<AA, BA>, a, 256, 512, 131072, stream);
            else return launch_tiles<T, 256, 256, 2, 4, AA, BA, DIRECT>(a, stream);
        }
    }
    if (p.tile == 64) return launch_tiles<T, 64, 64, 2, 2, AA, BA, DIRECT>(a, stream);
    return launch_tiles<T, 128, 128, 2, 2, AA, BA, DIRECT>(a, stream);
}

// Whether an operand can be read straight into LDS: whole chunks of 16 bytes, aligned, and an offset within a tile that fits 32 bits.
// side: the length of its rows in memory (k, or across the tile's rows).
template <typename T>
bool in_chunks(const void *const *p, uint32_t replicas, uint64_t ld, uint64_t side)
{
    constexpr uint64_t chunk = 16 / sizeof(T);
    bool ok = ld % chunk == 0 && side % chunk == 0 && ld < (1ull << 22);
    for (uint32_t i = 0; i < replicas; ++i) ok = ok && aligned(p[i], 16);
    return ok;
}

template <typename T, bool AA, bool BA>
am_status launch_product(ProductArgs &a, const ProductPlan &p, bool direct, float *partial, hipStream_t stream)
{
    a.splits = p.splits;
    a.split_k = p.split_k;
    a.partial = partial;
    const am_status s = direct ? launch_shape<T, AA, BA, true>(a, p, stream) : launch_shape<T, AA, BA, false>(a, p, stream);
    if (s != AM_OK || p.splits <= 1) return s;
    const uint64_t blocks = ((uint64_t)((a.n + 7u) / 8u) * a.m + 255u) / 256u;
    am::k_product_join<T><<<dim3((uint32_t)(blocks < 4096u ? blocks : 4096u), 1, a.replicas), 256, 0, stream>>>(a);
    AM_HIP(hipGetLastError());
    return AM_OK;
}

template <typename T>
am_status forward(const am_linear_config &c, const am_linear_buffers &b, hipStream_t stream)
{
    ProductArgs a;
    std::memset(&a, 0, sizeof a);
    for (uint32_t i = 0; i < c.replicas; ++i) {
        a.a[i] = b.x[i];
        a.b[i] = b.w[i];
        a.c[i] = b.y[i];
        if (b.bias) a.bias[i] = b.bias[i];
        if (b.residual) a.add[i] = b.residual[i];
        if (b.pre) a.pre[i] = b.pre[i];
    }
    a.m = (uint32_t)c.rows; a.n = (uint32_t)c.out; a.k = (uint32_t)c.in; a.replicas = c.replicas;
    a.act = c.act;
    a.lda = (uint32_t)or_dense(c.x_stride, c.in); a.ldb = (uint32_t)c.in; a.ldc = (uint32_t)or_dense(c.y_stride, c.out);
    a.ldadd = (uint32_t)or_dense(c.residual_stride, c.out); a.ldpre = (uint32_t)or_dense(c.pre_stride, c.out);
    a.k_whole = a.k;
    const bool direct = in_chunks<T>(a.a, c.replicas, a.lda, a.k) && in_chunks<T>(a.b, c.replicas, a.ldb, a.k);
    return launch_product<T, false, false>(a, plan_product(c, kRows), direct, static_cast<float *>(b.workspace), stream);
}

template <typename T, int ACT>
void launch_columns(const am::ColumnArgs &a, uint32_t replicas, hipStream_t stream)
{
    am::k_columns<T, ACT><<<dim3((a.n + 255u) / 256u, a.parts, replicas), 256, 0, stream>>>(a);
}

template <typename T>
am_status columns(const am::ColumnArgs &a, const am_linear_config &c, hipStream_t stream)
{
    switch (c.act) {
    case AM_ACT_RELU: launch_columns<T, am::kActRelu>(a, c.replicas, stream); break;
    case AM_ACT_GELU: launch_columns<T, am::kActGelu>(a, c.replicas, stream); break;
    case AM_ACT_GELU_TANH: launch_columns<T, am::kActGeluTanh>(a, c.replicas, stream); break;
    case AM_ACT_SILU: launch_columns<T, am::kActSilu>(a, c.replicas, stream); break;
    default: launch_columns<T, am::kActNone>(a, c.replicas, stream); break;
    }
    AM_HIP(hipGetLastError());
    return AM_OK;
}

template <typename O>
am_status clear(const am_linear_config &c, void *const *p, uint64_t elements, hipStream_t stream)
{
    ProductArgs a;
    std::memset(&a, 0, sizeof a);
    for (uint32_t i = 0; i < c.replicas; ++i) a.c[i] = p[i];
    const uint64_t blocks = (elements + 255u) / 256u;
    am::k_clear<O><<<dim3((uint32_t)(blocks < 4096u ? blocks : 4096u), c.replicas), 256, 0, stream>>>(a, elements);
    AM_HIP(hipGetLastError());
    return AM_OK;
}

template <typename T, typename O>
am_status backward(const am_linear_config &c, const am_linear_buffers &b, const BackwardSpace &sp, bool accumulate, hipStream_t stream)
{
    if (c.rows == 0) {
        if (accumulate) return AM_OK;
        if (b.dw) { const am_status s = clear<O>(c, b.dw, c.out * c.in, stream); if (s != AM_OK) return s; }
        return b.db ? clear<O>(c, b.db, c.out, stream) : AM_OK;
    }
    char *ws = static_cast<char *>(b.workspace);
    char *dz = ws;
    float *sums = reinterpret_cast<float *>(ws + sp.dz_bytes), *partial = reinterpret_cast<float *>(ws + sp.dz_bytes + sp.sums_bytes);
    const bool own_dz = sp.dz_bytes != 0;
    const uint64_t dz_one = sizeof(T) * c.rows * sp.dz_pitch;
    if (b.db || own_dz) {
        am::ColumnArgs a;
        std::memset(&a, 0, sizeof a);
        for (uint32_t i = 0; i < c.replicas; ++i) {
            a.dy[i] = b.dy[i];
            if (c.act != AM_ACT_NONE) a.pre[i] = b.pre[i];
            if (own_dz) a.dz[i] = dz + dz_one * i;
            if (b.db) a.db[i] = b.db[i];
        }
        a.m = (uint32_t)c.rows; a.n = (uint32_t)c.out; a.lddz = (uint32_t)sp.dz_pitch;
        a.lddy = (uint32_t)or_dense(c.y_stride, c.out); a.ldpre = (uint32_t)or_dense(c.pre_stride, c.out);
        a.rows_per_part = sp.rows_per_part; a.parts = sp.parts; a.accumulate = accumulate;
        a.partial = b.db ? sums : nullptr;
        const am_status s = columns<T>(a, c, stream);
        if (s != AM_OK) return s;
        if (b.db) {
            am::k_columns_join<O><<<dim3((a.n + 255u) / 256u, c.replicas), 256, 0, stream>>>(a);
            AM_HIP(hipGetLastError());
        }
    }
    const uint32_t lddz = own_dz ? (uint32_t)sp.dz_pitch : (uint32_t)or_dense(c.y_stride, c.out);
    ProductArgs a;
    std::memset(&a, 0, sizeof a);
    a.replicas = c.replicas;
    for (uint32_t i = 0; i < c.replicas; ++i) a.a[i] = own_dz ? dz + dz_one * i : static_cast<const char *>(b.dy[i]);
    if (b.dx) {
        for (uint32_t i = 0; i < c.replicas; ++i) { a.b[i] = b.w[i]; a.c[i] = b.dx[i]; }
        a.m = (uint32_t)c.rows; a.n = (uint32_t)c.in; a.k = (uint32_t)c.out;
        a.lda = lddz; a.ldb = (uint32_t)c.in; a.ldc = (uint32_t)or_dense(c.dx_stride, c.in);
        a.k_whole = own_dz ? (uint32_t)sp.dz_pitch : a.k;
        const bool direct = in_chunks<T>(a.a, c.replicas, a.lda, a.k_whole) && in_chunks<T>(a.b, c.replicas, a.ldb, a.n);
        const am_status s = launch_product<T, false, true>(a, plan_product(c, kInputGradient), direct, partial, stream);
        if (s != AM_OK) return s;
    }
    if (b.dw) {
        for (uint32_t i = 0; i < c.replicas; ++i) { a.b[i] = b.x[i]; a.c[i] = b.dw[i]; if (accumulate) a.add[i] = b.dw[i]; }
        a.m = (uint32_t)c.out; a.n = (uint32_t)c.in; a.k = (uint32_t)c.rows;
        a.out_f32 = sizeof(O) == 4;
        a.lda = lddz; a.ldb = (uint32_t)or_dense(c.x_stride, c.in); a.ldc = a.ldadd = (uint32_t)c.in;
        a.k_whole = a.k;
        const bool direct = in_chunks<T>(a.a, c.replicas, a.lda, own_dz ? sp.dz_pitch : a.m) && in_chunks<T>(a.b, c.replicas, a.ldb, a.n);
        const am_status s = launch_product<T, true, true>(a, plan_product(c, kWeightGradient), direct, partial, stream);
        if (s != AM_OK) return s;
    }
    return AM_OK;
}

}  // namespace

extern "C" {

am_status am_linear_workspace(const am_linear_config *cfg, const am_linear_buffers *buf, int backward_call, uint64_t *out_bytes)
{
    if (!out_bytes) return fail(AM_EINVAL, "out_bytes is NULL");
    const am_status s = backward_call ? check_backward(cfg, buf) : check_forward(cfg, buf);
    if (s != AM_OK) return s;
    *out_bytes = cfg->rows == 0 ? 0 : backward_call ? backward_space(*cfg, *buf).total : partial_bytes(*cfg, kRows);
    return AM_OK;
}

am_status am_linear(const am_linear_config *cfg, const am_linear_buffers *buf, void *hip_stream)
{
    am_status s = check_forward(cfg, buf);
    if (s != AM_OK) return s;
    if (cfg->rows == 0) return AM_OK;
    s = check_space(buf, partial_bytes(*cfg, kRows));
    if (s != AM_OK) return s;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return cfg->dtype == AM_BF16 ? forward<__bf16>(*cfg, *buf, stream) : forward<float>(*cfg, *buf, stream);
}

am_status am_linear_backward(const am_linear_config *cfg, const am_linear_buffers *buf, int accumulate, void *hip_stream)
{
    am_status s = check_backward(cfg, buf);
    if (s != AM_OK) return s;
    BackwardSpace sp = {};
    if (cfg->rows) sp = backward_space(*cfg, *buf);
    s = check_space(buf, sp.total);
    if (s != AM_OK) return s;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (cfg->dtype == AM_F32) return backward<float, float>(*cfg, *buf, sp, accumulate != 0, stream);
    return cfg->grad_dtype == AM_F32 ? backward<__bf16, float>(*cfg, *buf, sp, accumulate != 0, stream)
                                     : backward<__bf16, __bf16>(*cfg, *buf, sp, accumulate != 0, stream);
}

}  // extern "C"
