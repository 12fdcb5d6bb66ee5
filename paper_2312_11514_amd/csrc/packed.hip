// C ABI of the weights in 4 bits and of the norm with the residual's addition (see include/lif.h for the contract of every call).
// Host side only: argument checks, launch geometry.
#include "../../include/lif.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <new>

#include "lif_host.h"
#include "lif_norm.h"
#include "lif_packed_few.h"
#include "lif_packed_make.h"

using namespace lif;

struct lif_packed {
    lif_packed_config cfg;
    PackedView view;
    int tiles;
};

namespace {

constexpr int kMaxWidth = 65536, kMaxOut = 1 << 20, kMaxRows = 1 << 19;
constexpr int kMakeBlocks = 2048;                // 8 workgroups per compute unit
constexpr int64_t kMaxStride = (int64_t)1 << 40, kMaxXStride = 1 << 22;

int bytes_of(int dtype) { return dtype == LIF_F32 ? 4 : 2; }
bool dtype_ok(int dtype) { return dtype == LIF_F32 || dtype == LIF_F16 || dtype == LIF_BF16; }

bool config_ok(const lif_packed_config* c, const char** why) {
    *why = "";
    if (!c) return (*why = "null config", false);
    if (!dtype_ok(c->dtype)) return (*why = "dtype", false);
    if (c->n_out < 1 || c->n_out > kMaxOut) return (*why = "n_out must be in 1..2^20", false);
    if (c->n_in < 8 || c->n_in > kMaxWidth || c->n_in % 8) return (*why = "n_in must be a multiple of 8 in 8..65536", false);
    if (c->group != 32 && c->group != 64 && c->group != 128) return (*why = "group must be 32, 64 or 128", false);
    if (c->zeros != 0 && c->zeros != 1) return (*why = "zeros", false);
    return true;
}
int in_tiles(const lif_packed_config& c) { return (c.n_in + kTileIn - 1) / kTileIn; }
int out_tiles(const lif_packed_config& c) { return (c.n_out + kTileOut - 1) / kTileOut; }
int row_groups(const lif_packed_config& c) { return (c.n_in + c.group - 1) / c.group; }

int launched() {
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? LIF_OK : fail(LIF_HIP_ERROR, "launch: %s", hipGetErrorString(e));
}

// Rows in memory: `width` bytes at every multiple of `stride` bytes.
struct Span {
    const void* at;
    int64_t stride, width;
    int64_t rows;
    uintptr_t first() const { return reinterpret_cast<uintptr_t>(at); }
    uintptr_t end() const { return first() + (uintptr_t)((rows - 1) * stride + width); }
};
bool same(const Span& a, const Span& b) { return a.at == b.at && (a.stride == b.stride || a.rows == 1) && a.width == b.width; }
// Whether they may share memory.  Exact where the strides are equal, so that both may be parts of one projection's rows; other strides may share no range.
bool overlap(const Span& a, const Span& b) {
    if (a.end() <= b.first() || b.end() <= a.first()) return false;
    if (a.stride != b.stride || a.rows == 1) return true;
    const int64_t ahead = (int64_t)(b.first() - a.first());
    const int64_t r = (ahead % a.stride + a.stride) % a.stride;
    return r < a.width || r + b.width > a.stride;
}

bool aligned(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }
// a stride of at least one row; `bytes` of an element, whole `unit` bytes
bool stride_ok(int64_t stride, int64_t width, int bytes, int unit) { return stride >= width && stride <= kMaxStride && stride * bytes % unit == 0; }

// Whether rows share memory with the codes or the words of the groups.
bool overlaps_matrix(const lif_packed* p, const Span& rows) {
    const int64_t codes = (int64_t)lif_packed_code_bytes(&p->cfg), groups = (int64_t)lif_packed_group_bytes(&p->cfg);
    return overlap(rows, Span{p->view.codes, codes, codes, 1}) || overlap(rows, Span{p->view.groups, groups, groups, 1});
}
// full weights, of a call that reads or writes all of them
int weights_ok(const lif_packed* p, const void* weights, int64_t stride) {
    if (!p || !weights) return fail(LIF_INVALID_ARG, "null pointer");
    const int e = bytes_of(p->cfg.dtype);
    if (!aligned(weights, 16) || !stride_ok(stride, p->cfg.n_in, e, 16))
        return fail(LIF_INVALID_ARG, "rows of weights must be 16-byte aligned, at a stride that holds them");
    if (overlaps_matrix(p, Span{weights, stride * e, (int64_t)p->cfg.n_in * e, p->cfg.n_out}))
        return fail(LIF_INVALID_ARG, "weights must not overlap the codes or the words of the groups");
    return LIF_OK;
}

}  // namespace

extern "C" {

int lif_add_norm(const lif_norm_rows* n, void* stream) {
    if (!n) return fail(LIF_INVALID_ARG, "null pointer");
    if (!dtype_ok(n->dtype)) return fail(LIF_INVALID_ARG, "dtype");
    if (n->norm != LIF_NORM_NONE && n->norm != LIF_NORM_RMS && n->norm != LIF_NORM_LAYER) return fail(LIF_INVALID_ARG, "norm");
    if (n->n_rows < 1 || n->n_rows > kMaxRows) return fail(LIF_INVALID_ARG, "n_rows must be in 1..2^19");
    if (n->width < 8 || n->width > kMaxWidth || n->width % 8) return fail(LIF_INVALID_ARG, "width must be a multiple of 8 in 8..65536");
    if (!n->x || !n->out) return fail(LIF_INVALID_ARG, "null rows");
    if (n->total && !n->residual) return fail(LIF_INVALID_ARG, "a total without a residual");
    if (!(n->eps >= 0.f) || !std::isfinite(n->eps)) return fail(LIF_INVALID_ARG, "eps must be finite and not negative");
    if (n->group != 0 && n->group != 32 && n->group != 64 && n->group != 128) return fail(LIF_INVALID_ARG, "group must be 0, 32, 64 or 128");
    if (n->group && !n->scales) return fail(LIF_INVALID_ARG, "a group without scales");
    const int e = bytes_of(n->dtype), out_e = n->scales ? 1 : e;
    if (!aligned(n->x, 16) || !aligned(n->residual, 16) || !aligned(n->total, 16) || !aligned(n->out, n->scales ? 8 : 16))
        return fail(LIF_INVALID_ARG, "rows must be 16-byte aligned, those of 8 bits 8-byte aligned");
    if (!aligned(n->weight, 4) || !aligned(n->bias, 4) || !aligned(n->scales, 4)) return fail(LIF_INVALID_ARG, "fp32 arrays must be 4-byte aligned");
    if (!stride_ok(n->x_stride, n->width, e, 16) || (n->residual && !stride_ok(n->residual_stride, n->width, e, 16)) ||
        (n->total && !stride_ok(n->total_stride, n->width, e, 16)) || !stride_ok(n->out_stride, n->width, out_e, n->scales ? 8 : 16))
        return fail(LIF_INVALID_ARG, "a row stride must hold the row and be a multiple of 16 bytes, of 8 for rows of 8 bits");
    const int64_t groups = n->group ? (n->width + n->group - 1) / n->group : 1;
    const Span x{n->x, n->x_stride * e, (int64_t)n->width * e, n->n_rows}, residual{n->residual, n->residual_stride * e, (int64_t)n->width * e, n->n_rows},
        total{n->total, n->total_stride * e, (int64_t)n->width * e, n->n_rows}, out{n->out, n->out_stride * out_e, (int64_t)n->width * out_e, n->n_rows},
        scales{n->scales, groups * 4, groups * 4, n->n_rows}, weight{n->weight, n->width * 4ll, n->width * 4ll, 1}, bias{n->bias, n->width * 4ll, n->width * 4ll, 1};
    const Span* reads[] = {&x, &residual, &weight, &bias};
    const Span* writes[] = {&out, &total, &scales};
    for (const Span* w : writes)
        for (const Span* r : reads)
            if (w->at && r->at && overlap(*w, *r) && !(r != &weight && r != &bias && same(*w, *r)))
                return fail(LIF_INVALID_ARG, "out, total and scales must not overlap x, the residual, weight or bias (or be the rows of x or the residual)");
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < i; ++j)
            if (writes[i]->at && writes[j]->at && overlap(*writes[i], *writes[j])) return fail(LIF_INVALID_ARG, "out, total and scales must not overlap");
    const bool norm = n->norm != LIF_NORM_NONE;
    const NormArgs a{static_cast<const char*>(n->x), static_cast<const char*>(n->residual), static_cast<char*>(n->total), static_cast<char*>(n->out),
                     n->scales, norm ? n->weight : nullptr, n->norm == LIF_NORM_LAYER ? n->bias : nullptr, n->x_stride, n->residual_stride,
                     n->total_stride, n->out_stride, groups, n->n_rows, n->width, n->norm, n->group, n->eps};
    hipStream_t s = (hipStream_t)stream;
    if (n->dtype == LIF_F32) launch_add_norm_f32(a, s);
    else if (n->dtype == LIF_F16) launch_add_norm_f16(a, s);
    else launch_add_norm_bf16(a, s);
    return launched();
}

size_t lif_packed_code_bytes(const lif_packed_config* cfg) {
    const char* why;
    return config_ok(cfg, &why) ? (size_t)out_tiles(*cfg) * in_tiles(*cfg) * (kTileOut * kTileIn / 2) : 0;
}

size_t lif_packed_group_bytes(const lif_packed_config* cfg) {
    const char* why;
    return config_ok(cfg, &why) ? (size_t)out_tiles(*cfg) * in_tiles(*cfg) * (kTileIn / cfg->group) * kTileOut * 4 : 0;
}

int lif_packed_create(const lif_packed_config* cfg, const lif_packed_buffers* buf, lif_packed** out) {
    const char* why;
    if (!cfg || !buf || !out) return fail(LIF_INVALID_ARG, "null pointer");
    if (!config_ok(cfg, &why)) return fail(LIF_INVALID_ARG, "configuration: %s", why);
    if (!buf->codes || !buf->groups) return fail(LIF_INVALID_ARG, "null buffer");
    if (!aligned(buf->codes, 16) || !aligned(buf->groups, 16)) return fail(LIF_INVALID_ARG, "codes and groups must be 16-byte aligned");
    if (buf->code_bytes < lif_packed_code_bytes(cfg) || buf->group_bytes < lif_packed_group_bytes(cfg))
        return fail(LIF_INVALID_ARG, "codes or groups too small");
    const int64_t code_bytes = (int64_t)lif_packed_code_bytes(cfg), group_bytes = (int64_t)lif_packed_group_bytes(cfg);
    if (overlap(Span{buf->codes, code_bytes, code_bytes, 1}, Span{buf->groups, group_bytes, group_bytes, 1}))
        return fail(LIF_INVALID_ARG, "codes and groups must not overlap");
    lif_packed* p = new (std::nothrow) lif_packed;
    if (!p) return fail(LIF_INVALID_ARG, "out of host memory");
    p->cfg = *cfg;
    p->tiles = out_tiles(*cfg) * in_tiles(*cfg);
    p->view = PackedView{static_cast<unsigned*>(buf->codes), static_cast<unsigned*>(buf->groups), cfg->n_out, cfg->n_in, cfg->group, in_tiles(*cfg),
                         in_tiles(*cfg) * (kTileIn / cfg->group)};
    *out = p;
    return LIF_OK;
}

int lif_packed_destroy(lif_packed* p) {
    delete p;
    return LIF_OK;
}

int lif_packed_quantize(lif_packed* p, const void* weights, int64_t stride, void* stream) {
    if (const int rc = weights_ok(p, weights, stride)) return rc;
    const dim3 grid(std::min(p->tiles, kMakeBlocks)), block(256);
    hipStream_t s = (hipStream_t)stream;
    const bool z = p->cfg.zeros;
#define LIF_QUANTIZE(T)                                                                                                               \
    do {                                                                                                                              \
        if (z) hipLaunchKernelGGL((k_packed_quantize<T, true>), grid, block, 0, s, p->view, static_cast<const T*>(weights), (long long)stride, p->tiles); \
        else hipLaunchKernelGGL((k_packed_quantize<T, false>), grid, block, 0, s, p->view, static_cast<const T*>(weights), (long long)stride, p->tiles);  \
    } while (0)
    if (p->cfg.dtype == LIF_F32) LIF_QUANTIZE(float);
    else if (p->cfg.dtype == LIF_F16) LIF_QUANTIZE(_Float16);
    else LIF_QUANTIZE(__bf16);
#undef LIF_QUANTIZE
    return launched();
}

int lif_packed_pack(lif_packed* p, const uint8_t* codes, const float* scales, const uint8_t* zeros, void* stream) {
    if (!p || !codes || !scales) return fail(LIF_INVALID_ARG, "null pointer");
    if ((zeros != nullptr) != (p->cfg.zeros != 0)) return fail(LIF_INVALID_ARG, "zeros go with a configuration that has them");
    if (!aligned(codes, 4) || !aligned(scales, 4)) return fail(LIF_INVALID_ARG, "codes and scales must be 4-byte aligned");
    const int64_t row = p->cfg.n_in / 2, groups = row_groups(p->cfg), n = p->cfg.n_out;
    if (overlaps_matrix(p, Span{codes, row, row, n}) || overlaps_matrix(p, Span{scales, groups * 4, groups * 4, n}) ||
        (zeros && overlaps_matrix(p, Span{zeros, groups, groups, n})))
        return fail(LIF_INVALID_ARG, "codes, scales and zeros must not overlap the arrays of the matrix");
    hipLaunchKernelGGL(k_packed_pack, dim3(std::min(p->tiles, kMakeBlocks)), dim3(256), 0, (hipStream_t)stream, p->view, codes, scales, zeros, p->tiles);
    return launched();
}

int lif_packed_dequantize(lif_packed* p, void* weights, int64_t stride, void* stream) {
    if (const int rc = weights_ok(p, weights, stride)) return rc;
    const dim3 grid(std::min(p->tiles, kMakeBlocks)), block(256);
    hipStream_t s = (hipStream_t)stream;
    if (p->cfg.dtype == LIF_F32) hipLaunchKernelGGL(k_packed_dequantize<float>, grid, block, 0, s, p->view, static_cast<float*>(weights), (long long)stride, p->tiles);
    else if (p->cfg.dtype == LIF_F16) hipLaunchKernelGGL(k_packed_dequantize<_Float16>, grid, block, 0, s, p->view, static_cast<_Float16*>(weights), (long long)stride, p->tiles);
    else hipLaunchKernelGGL(k_packed_dequantize<__bf16>, grid, block, 0, s, p->view, static_cast<__bf16*>(weights), (long long)stride, p->tiles);
    return launched();
}

int lif_packed_multiply(lif_packed* p, const lif_packed_rows* rows, void* stream) {
    if (!p || !rows) return fail(LIF_INVALID_ARG, "null pointer");
    const lif_packed_config& c = p->cfg;
    if (rows->n_rows < 1 || rows->n_rows > kMaxRows) return fail(LIF_INVALID_ARG, "n_rows must be in 1..2^19");
    if (!rows->x || !rows->out) return fail(LIF_INVALID_ARG, "null rows");
    if (rows->x_group != 0 && (rows->x_group != c.group || !rows->x_scales))
        return fail(LIF_INVALID_ARG, "x_group must be 0 or the group of the weights, with scales");
    const bool eight = rows->x_scales != nullptr;
    const int e = bytes_of(c.dtype), x_e = eight ? 1 : e;
    // (with one row there is no stride; more than 2^22 elements would take offsets of 64 bits)
    const int64_t x_stride = rows->n_rows == 1 ? c.n_in : rows->x_stride;
    if (!aligned(rows->x, eight ? 8 : 16) || !stride_ok(rows->x_stride, c.n_in, x_e, eight ? 8 : 16) || x_stride > kMaxXStride)
        return fail(LIF_INVALID_ARG, "rows of x must be 16-byte aligned at a stride that holds them, is a multiple of 16 bytes (8 bits: 8 and 8), at most 2^22");
    if (!aligned(rows->out, e) || rows->out_stride < c.n_out || rows->out_stride > kMaxStride)
        return fail(LIF_INVALID_ARG, "rows of out must be aligned to their elements, at a stride that holds them");
    if (!aligned(rows->x_scales, 4) || !aligned(rows->bias, 4)) return fail(LIF_INVALID_ARG, "fp32 arrays must be 4-byte aligned");
    const int64_t groups = rows->x_group ? row_groups(c) : 1;
    const Span x{rows->x, rows->x_stride * x_e, (int64_t)c.n_in * x_e, rows->n_rows}, out{rows->out, rows->out_stride * e, (int64_t)c.n_out * e, rows->n_rows},
        scales{rows->x_scales, groups * 4, groups * 4, rows->n_rows}, bias{rows->bias, c.n_out * 4ll, c.n_out * 4ll, 1};
    if (overlap(out, x) || (scales.at && overlap(out, scales)) || (bias.at && overlap(out, bias)) || overlaps_matrix(p, out))
        return fail(LIF_INVALID_ARG, "out must not overlap x, its scales, the bias or the matrix");
    const ProductArgs a{p->view, static_cast<const char*>(rows->x), static_cast<char*>(rows->out), rows->x_scales, rows->bias, x_stride,
                        rows->out_stride, rows->n_rows, (int32_t)groups, c.dtype};
    hipStream_t s = (hipStream_t)stream;
    const auto launch = eight && groups > 1 ? launch_product_i8_groups : eight ? launch_product_i8 : c.dtype == LIF_F32 ? launch_product_f32
                        : c.dtype == LIF_F16 ? launch_product_f16 : launch_product_bf16;
    const PackedForm form = packed_form(out_tiles(c), p->view.in_tiles, rows->n_rows, !eight && c.dtype == LIF_F32, c.group);
    if (!launch(a, form, c.zeros != 0, s)) return fail(LIF_HIP_ERROR, "no kernel for this form of product");
    return launched();
}

}  // extern "C"
