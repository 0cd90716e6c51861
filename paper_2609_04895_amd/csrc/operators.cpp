// operators.cpp - host side of the operators that take an expert pool beyond a few
// tokens and beyond 8 bits (include/cmoe.h): grouped products, the MoE layer for
// prompts, dense products with 4-bit weights, and rows into either form; validation,
// the workspace and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>

#include "checks.h"
#include "places.h"

namespace {

using namespace cmoe::host;

bool known_dtype(int t) { return t == CMOE_F32 || t == CMOE_BF16; }
bool known_format(int f) { return f == CMOE_FORMAT_DTYPE || f == CMOE_FORMAT_MX8 || f == CMOE_FORMAT_MX4; }

// Bytes of n values (a multiple of two) in a format.
int64_t held_bytes(int format, int dtype, int64_t n) {
    return format == CMOE_FORMAT_MX4 ? n / 2 : format == CMOE_FORMAT_MX8 ? n : n * (int64_t)elem(dtype);
}

// Strides that no memory has room for, and that the products below have no bits for.
bool beyond(std::initializer_list<int64_t> strides) {
    return std::any_of(strides.begin(), strides.end(), [](int64_t s) { return s > (int64_t)1 << 48; });
}

cmoe_status ready(void* stream) {
    int device = 0;
    const cmoe_status st = current_device(&device);
    return st == CMOE_OK ? check_stream(static_cast<hipStream_t>(stream), device) : st;
}

cmoe_status check_product(const cmoe_product* p) {
    if (!p) return fail(CMOE_ERR_INVALID_ARG, "product: arguments are NULL");
    if (p->N < 1 || p->m < 1 || p->d < 1 || p->rows < 0 || p->x_rows < 0)
        return fail(CMOE_ERR_INVALID_ARG, "product: N, m and d must be >= 1, rows and x_rows >= 0");
    if (!known_dtype(p->dtype) || !known_dtype(p->y_dtype)) return fail(CMOE_ERR_INVALID_ARG, "product: unknown dtype");
    if (!known_format(p->x_format) || !known_format(p->w_format) || !known_format(p->y_format))
        return fail(CMOE_ERR_INVALID_ARG, "product: unknown format");
    if (p->N > cmoe::kMaxN) return fail(CMOE_ERR_UNSUPPORTED, "product: N > 256 is not supported");
    if (p->d % 64 || p->d > 1 << 16) return fail(CMOE_ERR_UNSUPPORTED, "product: d must be a multiple of 64 up to 65536");
    if (p->m > cmoe::kProductWidth) return fail(CMOE_ERR_UNSUPPORTED, "product: m > %d is not supported", cmoe::kProductWidth);
    if (p->rows > cmoe::kProductRows) return fail(CMOE_ERR_UNSUPPORTED, "product: more than %d rows are not supported", cmoe::kProductRows);
    if (p->x_format == CMOE_FORMAT_MX4 || p->y_format == CMOE_FORMAT_MX4)
        return fail(CMOE_ERR_UNSUPPORTED, "product: only weights are held in 4 bits");
    if (p->dtype != CMOE_BF16 && (p->x_format || p->w_format || p->y_format))
        return fail(CMOE_ERR_UNSUPPORTED, "product: 8 and 4 bits go with the bf16 type");
    if (p->x_format == CMOE_FORMAT_MX8 && p->w_format == CMOE_FORMAT_DTYPE)
        return fail(CMOE_ERR_UNSUPPORTED, "product: 8-bit rows go with 8-bit or 4-bit weights");
    if (p->x_format == CMOE_FORMAT_MX8 && p->y_format == CMOE_FORMAT_DTYPE && p->y_dtype != CMOE_BF16)
        return fail(CMOE_ERR_UNSUPPORTED, "product: 8-bit rows give bf16 or 8-bit outputs");
    if (p->y_format == CMOE_FORMAT_MX8 && p->m % 32) return fail(CMOE_ERR_INVALID_ARG, "product: 8-bit outputs need m to be a multiple of 32");
    if (p->rows == 0) return CMOE_OK;
    if (!p->first || !p->x || !p->w || !p->y) return fail(CMOE_ERR_INVALID_ARG, "product: first, x, w and y are required");
    if (!p->x_row && p->x_rows < p->rows) return fail(CMOE_ERR_INVALID_ARG, "product: without x_row, x needs a row for each of y");
    if (p->x_rows < 1) return fail(CMOE_ERR_INVALID_ARG, "product: x has no rows");
    if ((p->x_format == CMOE_FORMAT_MX8) != !!p->x_scale || (p->w_format != CMOE_FORMAT_DTYPE) != !!p->w_scale ||
        (p->y_format == CMOE_FORMAT_MX8) != !!p->y_scale)
        return fail(CMOE_ERR_INVALID_ARG, "product: scales go with 8-bit and 4-bit values");
    const int64_t w_rows = (int64_t)p->m * (p->swiglu ? 2 : 1), matrix = w_rows * p->d;
    if (p->x_stride < p->d || p->y_stride < p->m || (p->N > 1 && p->w_stride < matrix))
        return fail(CMOE_ERR_INVALID_ARG, "product: a stride is less than the row or the matrix");
    if ((p->x_scale && p->x_scale_stride < p->d / 32) || (p->w_scale && p->N > 1 && p->w_scale_stride < matrix / 32) ||
        (p->y_scale && p->y_scale_stride < p->m / 32))
        return fail(CMOE_ERR_INVALID_ARG, "product: a stride of scales is less than the row or the matrix");
    if (beyond({p->x_stride, p->y_stride, p->N > 1 ? p->w_stride : 0, p->x_scale ? p->x_scale_stride : 0,
                p->w_scale && p->N > 1 ? p->w_scale_stride : 0, p->y_scale ? p->y_scale_stride : 0}))
        return fail(CMOE_ERR_UNSUPPORTED, "product: a stride of more than 2^48 is not supported");
    if (!aligned_to(p->first, 4) || !aligned_to(p->x_row, 4) || !aligned_to(p->y, p->y_format ? 4 : elem(p->y_dtype)) ||
        (p->y_format && p->y_stride % 4))
        return fail(CMOE_ERR_INVALID_ARG, "product: a pointer is not aligned to its values");
    const int64_t x_pitch = held_bytes(p->x_format, p->dtype, p->x_stride);
    const int64_t w_pitch = p->N > 1 ? held_bytes(p->w_format, p->dtype, p->w_stride) : 0;
    if (p->w_format == CMOE_FORMAT_MX4 && p->N > 1 && p->w_stride % 2) return fail(CMOE_ERR_UNSUPPORTED, "product: matrices of w must be 16-byte aligned");
    if (!aligned_to(p->x, 16) || x_pitch % 16 || !aligned_to(p->w, 16) || w_pitch % 16)
        return fail(CMOE_ERR_UNSUPPORTED, "product: rows of x and matrices of w must be 16-byte aligned");
    const int64_t y_elem = p->y_format ? 1 : (int64_t)elem(p->y_dtype);
    if (!apart({{p->y, p->rows, p->y_stride * y_elem, p->m * y_elem}, {p->y_scale, p->rows, p->y_scale_stride, p->m / 32}},
               {{p->x, p->x_rows, x_pitch, held_bytes(p->x_format, p->dtype, p->d)},
                {p->x_scale, p->x_rows, p->x_scale_stride, p->d / 32},
                {p->w, p->N, w_pitch, held_bytes(p->w_format, p->dtype, matrix)},
                {p->w_scale, p->N, p->N > 1 ? p->w_scale_stride : 0, matrix / 32},
                {p->first, 1, 0, 4 * ((int64_t)p->N + 1)},
                {p->x_row, 1, 0, 4 * (int64_t)p->rows}}))
        return fail(CMOE_ERR_INVALID_ARG, "product: an output overlaps an input or the other output");
    return CMOE_OK;
}

// inner: y is a prompt layer's own, which no caller sees; halves: as halves with scales.
hipError_t run_product(const cmoe_product* p, hipStream_t st, bool halves = false, bool inner = false) {
    cmoe::ProductArgs a{};
    a.N = p->N; a.m = p->m; a.d = p->d; a.rows = p->rows; a.x_rows = p->x_rows;
    a.swiglu = p->swiglu != 0;
    a.first = p->first; a.x_row = p->x_row;
    a.x = static_cast<const char*>(p->x);
    a.x_pitch = held_bytes(p->x_format, p->dtype, p->x_stride);
    a.x_scale = p->x_scale; a.x_scale_pitch = p->x_scale_stride;
    a.w = static_cast<const char*>(p->w);
    a.w_matrix = p->N > 1 ? held_bytes(p->w_format, p->dtype, p->w_stride) : 0;
    a.w_scale = p->w_scale; a.w_scale_matrix = p->N > 1 ? p->w_scale_stride : 0;
    a.y = p->y; a.y_stride = p->y_stride;
    a.y_scale = p->y_scale; a.y_scale_stride = p->y_scale_stride;
    a.y_kind = p->y_format ? cmoe::kProductMx8 : p->y_dtype == CMOE_BF16 ? cmoe::kProductBf16 : cmoe::kProductF32;
    a.y_aligned = p->y_stride % 4 == 0 && aligned_to(p->y, p->y_dtype == CMOE_BF16 ? 8 : 16);
    a.exact = !inner && p->y_format == CMOE_FORMAT_MX8;
    if (halves) a.y_kind = cmoe::kProductHalf;
    a.y_lines = halves || (a.y_kind == cmoe::kProductBf16 && p->m % 8 == 0 && p->y_stride % 8 == 0 && aligned_to(p->y, 16));
    if (p->dtype == CMOE_F32) return cmoe::launch_product_f32(a, st);
    if (p->x_format == CMOE_FORMAT_DTYPE) {
        a.held = p->w_format == CMOE_FORMAT_DTYPE ? cmoe::kHeldSame : p->w_format == CMOE_FORMAT_MX8 ? cmoe::kHeld8 : cmoe::kHeld4;
        return cmoe::launch_product_bf16(a, st);
    }
    a.held = p->w_format == CMOE_FORMAT_MX8 ? cmoe::kHeldSame : cmoe::kHeld4;
    return cmoe::launch_product_mx8(a, st);
}

// Offsets of the workspace's parts.
struct Parts {
    size_t z, gate, expert, row, token, mask, before, total, first, act, act_scale, out, out_scale, bytes;
};

cmoe_status check_prompt(const cmoe_moe_config* c) {
    if (!c) return fail(CMOE_ERR_INVALID_ARG, "config is NULL");
    if (c->L < 1 || c->N < 1 || c->K < 1 || c->d < 1 || c->F < 1 || c->T < 1)
        return fail(CMOE_ERR_INVALID_ARG, "L, N, K, d, F and T must be >= 1");
    if (c->K > c->N) return fail(CMOE_ERR_INVALID_ARG, "K must not exceed N");
    if (!known_dtype(c->dtype)) return fail(CMOE_ERR_INVALID_ARG, "unknown dtype");
    if (!known_format(c->weights) || !known_format(c->activations)) return fail(CMOE_ERR_INVALID_ARG, "unknown format");
    if (c->T > cmoe::kPromptTokens)
        return fail(CMOE_ERR_UNSUPPORTED, "T > %d is not supported: longer prompts go in several calls", cmoe::kPromptTokens);
    if (c->N > cmoe::kMaxN) return fail(CMOE_ERR_UNSUPPORTED, "N > 256 is not supported");
    if (c->K > cmoe::kMaxK) return fail(CMOE_ERR_UNSUPPORTED, "K > 64 is not supported");
    if (c->d % 64 || c->F % 64) return fail(CMOE_ERR_UNSUPPORTED, "d and F must be multiples of 64");
    if (c->d > 1 << 16 || c->F > 1 << 16) return fail(CMOE_ERR_UNSUPPORTED, "d and F above 65536 are not supported");
    if (c->weights != CMOE_FORMAT_DTYPE && c->dtype != CMOE_BF16)
        return fail(CMOE_ERR_UNSUPPORTED, "8-bit and 4-bit weights go with the bf16 type");
    if (c->activations == CMOE_FORMAT_MX4) return fail(CMOE_ERR_UNSUPPORTED, "activations are not held in 4 bits");
    if (c->activations == CMOE_FORMAT_MX8 && c->weights == CMOE_FORMAT_DTYPE)
        return fail(CMOE_ERR_UNSUPPORTED, "8-bit activations go with 8-bit or 4-bit weights");
    return CMOE_OK;
}

Parts prompt_parts(const cmoe_moe_config* c) {
    Parts p{};
    size_t o = 0;
    auto take = [&o](size_t bytes) {
        const size_t at = o;
        o += align256(bytes);
        return at;
    };
    const size_t T = c->T, N = c->N, rows = T * c->K, chunks = (T + cmoe::kPromptChunk - 1) / cmoe::kPromptChunk, e = elem(c->dtype);
    const bool a8 = c->activations == CMOE_FORMAT_MX8;
    p.z = take(T * N * 4);
    p.gate = take(rows * 4);
    p.expert = take(rows * 4);
    p.row = take(rows * 4);
    p.token = take(rows * 4);
    p.mask = take(chunks * N * 4);
    p.before = take(chunks * N * 4);
    p.total = take(N * 4);
    p.first = take((N + 1) * 4);
    p.act = take(rows * c->F * (a8 ? 1 : e));
    p.act_scale = take(a8 ? rows * c->F / 32 : 0);
    p.out = take(rows * c->d * e);
    p.out_scale = take(c->dtype == CMOE_BF16 ? rows * c->d / 32 : 0);
    p.bytes = o;
    return p;
}

// Where the weights of all layers lie, and the workspace.
struct Held {
    Span router, bias, experts, scales, workspace;
};
Held held(const cmoe_moe_config* c, const cmoe_moe_weights* w, const void* workspace) {
    const Span::Bytes logits = static_cast<Span::Bytes>(c->L) * c->N, pool = logits * 3 * c->d * c->F;
    auto flat = [](const void* p, Span::Bytes n) { return Span{p, 1, 0, static_cast<int64_t>(std::min<Span::Bytes>(n, INT64_MAX))}; };
    return {flat(w->w_router, logits * c->d * elem(c->dtype)), flat(w->logit_bias, logits * 4),
            flat(w->experts, c->weights == CMOE_FORMAT_MX4 ? pool / 2 : c->weights == CMOE_FORMAT_MX8 ? pool : pool * elem(c->dtype)),
            flat(c->weights != CMOE_FORMAT_DTYPE ? w->expert_scales : nullptr, pool / 32), flat(workspace, prompt_parts(c).bytes)};
}

}  // namespace

struct cmoe_prompt {
    cmoe_moe_config cfg;
    cmoe_moe_weights w;
    Held at;
    Parts parts;
    char* ws;
    hipStream_t stream;
    int device;
};

extern "C" {

cmoe_status cmoe_quantize_as(int32_t format, const void* src, int32_t dtype, int64_t rows, int64_t cols, int64_t src_stride, uint8_t* q,
                             int64_t q_stride, uint8_t* scale, int64_t scale_stride, void* stream) {
    if (format != CMOE_FORMAT_MX8 && format != CMOE_FORMAT_MX4) return fail(CMOE_ERR_INVALID_ARG, "quantize: the format must be 8 or 4 bits");
    if (rows < 0 || cols < 0) return fail(CMOE_ERR_INVALID_ARG, "quantize: rows and cols must be >= 0");
    if (!known_dtype(dtype)) return fail(CMOE_ERR_INVALID_ARG, "quantize: unknown dtype");
    if (cols % 32) return fail(CMOE_ERR_INVALID_ARG, "quantize: cols must be a multiple of 32");
    if (cols && rows > ((int64_t)1 << 34) / cols) return fail(CMOE_ERR_UNSUPPORTED, "quantize: more than 2^34 values");
    if (rows && cols) {
        const int64_t e = (int64_t)elem(dtype), q_row = held_bytes(format, dtype, cols);
        if (!src || !q || !scale) return fail(CMOE_ERR_INVALID_ARG, "quantize: src, q and scale are required");
        if (src_stride < cols || q_stride < q_row || scale_stride < cols / 32)
            return fail(CMOE_ERR_INVALID_ARG, "quantize: a row stride is less than the row");
        if (beyond({src_stride, q_stride, scale_stride})) return fail(CMOE_ERR_UNSUPPORTED, "quantize: a stride of more than 2^48 is not supported");
        if (!aligned_to(src, 16) || src_stride * e % 16 || !aligned_to(q, 16) || q_stride % 16)
            return fail(CMOE_ERR_UNSUPPORTED, "quantize: rows of src and q must be 16-byte aligned");
        if (!apart({{q, rows, q_stride, q_row}, {scale, rows, scale_stride, cols / 32}}, {{src, rows, src_stride * e, cols * e}}))
            return fail(CMOE_ERR_INVALID_ARG, "quantize: an output overlaps src or the other output");
    }
    if (format == CMOE_FORMAT_MX8) return cmoe_quantize(src, dtype, rows, cols, src_stride, q, q_stride, scale, scale_stride, stream);
    const cmoe_status st = ready(stream);
    if (st != CMOE_OK || rows == 0 || cols == 0) return st;
    const cmoe::QuantizeArgs a{dtype == CMOE_BF16, src, rows, cols, src_stride, q, q_stride, scale, scale_stride};
    const hipError_t err = cmoe::launch_quantize4(a, static_cast<hipStream_t>(stream));
    return err == hipSuccess ? CMOE_OK : hip_fail(err, "quantize");
}

cmoe_status cmoe_matvec(const cmoe_vectors* v, void* stream) {
    if (!v) return fail(CMOE_ERR_INVALID_ARG, "matvec: arguments are NULL");
    if (v->rows < 0 || v->m < 1 || v->d < 1) return fail(CMOE_ERR_INVALID_ARG, "matvec: rows must be >= 0, m and d >= 1");
    if (!known_dtype(v->dtype) || !known_dtype(v->y_dtype)) return fail(CMOE_ERR_INVALID_ARG, "matvec: unknown dtype");
    if (v->rows > cmoe::kVectorRows)
        return fail(CMOE_ERR_UNSUPPORTED, "matvec: more than %d rows are not supported: they are a grouped product of one group", cmoe::kVectorRows);
    if (v->d % 32 || v->d > 1 << 18) return fail(CMOE_ERR_UNSUPPORTED, "matvec: d must be a multiple of 32 up to 2^18");
    if (v->m > 1 << 24) return fail(CMOE_ERR_UNSUPPORTED, "matvec: m > 2^24 is not supported");
    if (v->rows) {
        if (!v->x || !v->w || !v->w_scale || !v->y) return fail(CMOE_ERR_INVALID_ARG, "matvec: x, w, w_scale and y are required");
        if (v->x_stride < v->d || v->w_stride < v->d / 2 || v->w_scale_stride < v->d / 32 || v->y_stride < v->m)
            return fail(CMOE_ERR_INVALID_ARG, "matvec: a row stride is less than the row");
        if (beyond({v->x_stride, v->w_stride, v->w_scale_stride, v->y_stride}))
            return fail(CMOE_ERR_UNSUPPORTED, "matvec: a stride of more than 2^48 is not supported");
        const int64_t e = (int64_t)elem(v->dtype), ey = (int64_t)elem(v->y_dtype);
        if (!aligned_to(v->y, ey) || !aligned_to(v->n_rows, 4)) return fail(CMOE_ERR_INVALID_ARG, "matvec: a pointer is not aligned to its values");
        if (!aligned_to(v->x, 16) || v->x_stride * e % 16 || !aligned_to(v->w, 16) || v->w_stride % 16)
            return fail(CMOE_ERR_UNSUPPORTED, "matvec: rows of x and w must be 16-byte aligned");
        if (!apart({{v->y, v->rows, v->y_stride * ey, v->m * ey}},
                   {{v->x, v->rows, v->x_stride * e, v->d * e}, {v->w, v->m, v->w_stride, v->d / 2},
                    {v->w_scale, v->m, v->w_scale_stride, v->d / 32}, {v->n_rows, 1, 0, 4}}))
            return fail(CMOE_ERR_INVALID_ARG, "matvec: y overlaps an input");
    }
    const cmoe_status st = ready(stream);
    if (st != CMOE_OK || v->rows == 0) return st;
    cmoe::MatvecArgs a{};
    a.rows = v->rows; a.m = v->m; a.d = v->d;
    a.bf16 = v->dtype == CMOE_BF16; a.y_bf16 = v->y_dtype == CMOE_BF16;
    a.x = v->x; a.x_stride = v->x_stride;
    a.w = v->w; a.w_pitch = v->w_stride;
    a.w_scale = v->w_scale; a.w_scale_pitch = v->w_scale_stride;
    a.y = v->y; a.y_stride = v->y_stride;
    a.n_rows = v->n_rows;
    a.y_aligned = v->y_stride % 4 == 0 && aligned_to(v->y, a.y_bf16 ? 8 : 16);
    const hipError_t err = cmoe::launch_matvec(a, static_cast<hipStream_t>(stream));
    return err == hipSuccess ? CMOE_OK : hip_fail(err, "matvec");
}

cmoe_status cmoe_grouped_product(const cmoe_product* p, void* stream) {
    cmoe_status st = check_product(p);
    if (st == CMOE_OK) st = ready(stream);
    if (st != CMOE_OK || p->rows == 0) return st;
    const hipError_t err = run_product(p, static_cast<hipStream_t>(stream));
    return err == hipSuccess ? CMOE_OK : hip_fail(err, "grouped product");
}

cmoe_status cmoe_prompt_query(const cmoe_moe_config* cfg, size_t* workspace_bytes) {
    const cmoe_status st = check_prompt(cfg);
    if (st != CMOE_OK) return st;
    if (!workspace_bytes) return fail(CMOE_ERR_INVALID_ARG, "size output is NULL");
    *workspace_bytes = prompt_parts(cfg).bytes;
    return CMOE_OK;
}

cmoe_status cmoe_prompt_init(const cmoe_moe_config* cfg, const cmoe_moe_weights* w, void* workspace, void* stream, cmoe_prompt** out) {
    if (out) *out = nullptr;
    cmoe_status st = check_prompt(cfg);
    if (st != CMOE_OK) return st;
    if (!w || !out) return fail(CMOE_ERR_INVALID_ARG, "weights and output handle are required");
    const bool scaled = cfg->weights != CMOE_FORMAT_DTYPE;
    if (!w->w_router || !w->experts) return fail(CMOE_ERR_INVALID_ARG, "w_router and experts are required");
    if (scaled && !w->expert_scales) return fail(CMOE_ERR_INVALID_ARG, "expert_scales is required with 8-bit and 4-bit weights");
    if (!workspace || !aligned_to(workspace, 256)) return fail(CMOE_ERR_INVALID_ARG, "a workspace is required, 256-byte aligned");
    if (!aligned_to(w->w_router, 16) || !aligned_to(w->experts, 16) || !aligned_to(w->logit_bias, 4))
        return fail(CMOE_ERR_INVALID_ARG, "w_router and experts must be 16-byte aligned, logit_bias 4-byte");
    const Held at = held(cfg, w, workspace);
    if (!apart({at.workspace}, {at.router, at.bias, at.experts, at.scales}))
        return fail(CMOE_ERR_INVALID_ARG, "the workspace overlaps a weight");
    int device = 0;
    if ((st = current_device(&device)) != CMOE_OK) return st;
    if ((st = check_stream(static_cast<hipStream_t>(stream), device)) != CMOE_OK) return st;
    // refuse what the device cannot read rather than fault later
    for (const void* p : {w->w_router, w->experts, static_cast<const void*>(scaled ? w->expert_scales : nullptr),
                          static_cast<const void*>(w->logit_bias), static_cast<const void*>(workspace)}) {
        if (!p) continue;
        hipPointerAttribute_t attr;
        if (hipPointerGetAttributes(&attr, p) != hipSuccess || attr.type != hipMemoryTypeDevice || attr.device != device) {
            (void)hipGetLastError();
            return fail(CMOE_ERR_INVALID_ARG, "a weight or the workspace is not memory of the current device");
        }
    }
    cmoe_prompt* m = new (std::nothrow) cmoe_prompt{};
    if (!m) return fail(CMOE_ERR_UNSUPPORTED, "no host memory for the handle");
    m->cfg = *cfg;
    m->w = *w;
    m->at = at;
    m->parts = prompt_parts(cfg);
    m->ws = static_cast<char*>(workspace);
    m->stream = static_cast<hipStream_t>(stream);
    m->device = device;
    *out = m;
    return CMOE_OK;
}

cmoe_status cmoe_prompt_layer(cmoe_prompt* m, const cmoe_prompt_call* c) {
    if (!m) return fail(CMOE_ERR_INVALID_ARG, "handle is NULL");
    int device = -1;
    if (hipGetDevice(&device) != hipSuccess || device != m->device) {
        (void)hipGetLastError();
        return fail(CMOE_ERR_INVALID_ARG, "the current device is not the one the handle was created on");
    }
    const cmoe_moe_config& g = m->cfg;
    const bool a8 = g.activations == CMOE_FORMAT_MX8;
    const int64_t e = (int64_t)elem(g.dtype);
    if (!c) return fail(CMOE_ERR_INVALID_ARG, "arguments are NULL");
    if (c->layer < 0 || c->layer >= g.L) return fail(CMOE_ERR_INVALID_ARG, "layer must be in [0, L)");
    if (c->T < 0 || c->T > g.T) return fail(CMOE_ERR_INVALID_ARG, "T must be in [0, the configuration's T]");
    if (c->T == 0) return CMOE_OK;
    if (!c->h || !c->y) return fail(CMOE_ERR_INVALID_ARG, "h and y are required");
    if (c->h_stride < g.d || c->y_stride < g.d) return fail(CMOE_ERR_INVALID_ARG, "a row stride of h or y is less than d");
    if (beyond({c->h_stride, c->y_stride, a8 ? c->h8_stride : 0, a8 ? c->h8_scale_stride : 0}))
        return fail(CMOE_ERR_UNSUPPORTED, "a stride of more than 2^48 is not supported");
    if (!aligned_to(c->h, 16) || c->h_stride * e % 16 || !aligned_to(c->y, 16) || c->y_stride * e % 16)
        return fail(CMOE_ERR_UNSUPPORTED, "rows of h and y must be 16-byte aligned");
    if (a8 && (!c->h8 || !c->h8_scale)) return fail(CMOE_ERR_INVALID_ARG, "h8 and h8_scale are required with 8-bit activations");
    if (a8 && (c->h8_stride < g.d || c->h8_scale_stride < g.d / 32))
        return fail(CMOE_ERR_INVALID_ARG, "a row stride of h8 or h8_scale is less than the row");
    if (a8 && (!aligned_to(c->h8, 16) || c->h8_stride % 16)) return fail(CMOE_ERR_UNSUPPORTED, "rows of h8 must be 16-byte aligned");
    if (!a8 && (c->h8 || c->h8_scale)) return fail(CMOE_ERR_INVALID_ARG, "h8 is given, but the configuration's activations are not 8-bit");
    if (!aligned_to(c->n_tokens, 4) || !aligned_to(c->selected, 4) || !aligned_to(c->gates, 4))
        return fail(CMOE_ERR_INVALID_ARG, "a pointer is not aligned to its values");
    const int64_t picks = 4 * (int64_t)c->T * g.K;
    if (!apart({m->at.workspace, {c->y, c->T, c->y_stride * e, g.d * e}, {c->selected, 1, 0, picks}, {c->gates, 1, 0, picks}},
               {{c->h, c->T, c->h_stride * e, g.d * e},
                {c->h8, c->T, c->h8_stride, g.d},
                {c->h8_scale, c->T, c->h8_scale_stride, g.d / 32},
                {c->n_tokens, 1, 0, 4},
                m->at.router, m->at.bias, m->at.experts, m->at.scales}))
        return fail(CMOE_ERR_INVALID_ARG, "an output or the workspace overlaps an input, a weight or an output");

    auto part = [m](size_t at) { return static_cast<void*>(m->ws + at); };
    cmoe::PromptArgs a{};
    a.N = g.N; a.K = g.K; a.d = g.d; a.T = c->T;
    a.bf16 = g.dtype == CMOE_BF16;
    a.w_router = static_cast<const char*>(m->w.w_router) + (size_t)c->layer * g.N * g.d * e;
    a.bias = m->w.logit_bias ? m->w.logit_bias + (size_t)c->layer * g.N : nullptr;
    a.h = c->h; a.h_stride = c->h_stride;
    a.n_tokens = c->n_tokens; a.selected = c->selected; a.gates = c->gates;
    a.y = c->y; a.y_stride = c->y_stride;
    a.z = static_cast<float*>(part(m->parts.z));
    a.gate = static_cast<float*>(part(m->parts.gate));
    a.expert = static_cast<int32_t*>(part(m->parts.expert));
    a.row = static_cast<int32_t*>(part(m->parts.row));
    a.token = static_cast<int32_t*>(part(m->parts.token));
    a.mask = static_cast<uint32_t*>(part(m->parts.mask));
    a.before = static_cast<int32_t*>(part(m->parts.before));
    a.total = static_cast<int32_t*>(part(m->parts.total));
    a.first = static_cast<int32_t*>(part(m->parts.first));
    a.out = part(m->parts.out);
    a.out_scale = static_cast<uint8_t*>(part(m->parts.out_scale));
    hipError_t err = cmoe::launch_prompt_route(a, m->stream);
    if (err != hipSuccess) return hip_fail(err, "prompt layer, routing");

    const int64_t matrix = (int64_t)g.d * g.F, layer = (int64_t)c->layer * g.N * 3 * matrix;
    const char* experts = static_cast<const char*>(m->w.experts) + held_bytes(g.weights, g.dtype, layer);
    const uint8_t* scales = g.weights != CMOE_FORMAT_DTYPE ? m->w.expert_scales + layer / 32 : nullptr;
    cmoe_product p{};
    p.N = g.N; p.rows = c->T * g.K;
    p.dtype = p.y_dtype = g.dtype;
    p.w_format = g.weights;
    p.w_stride = 3 * matrix; p.w_scale_stride = 3 * matrix / 32;
    p.first = a.first;
    // gate and up, from the tokens' rows
    p.m = g.F; p.d = g.d; p.swiglu = 1;
    p.x_rows = c->T; p.x_row = a.token;
    p.x_format = p.y_format = a8 ? CMOE_FORMAT_MX8 : CMOE_FORMAT_DTYPE;
    p.x = a8 ? c->h8 : c->h; p.x_stride = a8 ? c->h8_stride : c->h_stride;
    p.x_scale = a8 ? c->h8_scale : nullptr; p.x_scale_stride = c->h8_scale_stride;
    p.w = experts; p.w_scale = scales;
    p.y = part(m->parts.act); p.y_stride = g.F;
    p.y_scale = a8 ? static_cast<uint8_t*>(part(m->parts.act_scale)) : nullptr; p.y_scale_stride = g.F / 32;
    if ((err = run_product(&p, m->stream, false, true)) != hipSuccess) return hip_fail(err, "prompt layer, gate and up");
    // down, in the rows' order
    p.m = g.d; p.d = g.F; p.swiglu = 0;
    p.x_rows = p.rows; p.x_row = nullptr;
    p.x = p.y; p.x_stride = g.F;
    p.x_scale = p.y_scale; p.x_scale_stride = g.F / 32;
    p.w = experts + held_bytes(g.weights, g.dtype, 2 * matrix); p.w_scale = scales ? scales + 2 * matrix / 32 : nullptr;
    p.y_format = CMOE_FORMAT_DTYPE;
    p.y = part(m->parts.out); p.y_stride = g.d;
    p.y_scale = static_cast<uint8_t*>(part(m->parts.out_scale)); p.y_scale_stride = g.d / 32;
    if ((err = run_product(&p, m->stream, a.bf16, true)) != hipSuccess) return hip_fail(err, "prompt layer, down");
    err = cmoe::launch_prompt_sum(a, m->stream);
    return err == hipSuccess ? CMOE_OK : hip_fail(err, "prompt layer, sum");
}

cmoe_status cmoe_prompt_destroy(cmoe_prompt* m) {
    delete m;
    return CMOE_OK;
}

}  // extern "C"
