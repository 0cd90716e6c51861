// moe.cpp - host side of the operators without an expert cache (include/cmoe.h):
// the residual addition with its norm, rows into 8 bits, and the whole MoE layer
// for a few tokens; validation, the workspace and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>
#include <new>

#include "../../include/cmoe.h"
#include "cmoe_internal.h"

namespace {

// Error text without allocation, so that no entry point can throw.
cmoe_status fail(cmoe_status st, const char* fmt, ...) {
    char msg[256];
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    return static_cast<cmoe_status>(cmoe::set_error(st, msg));
}

cmoe_status hip_fail(hipError_t e, const char* where) {
    return fail(CMOE_ERR_HIP, "HIP error in %s: %s", where, hipGetErrorString(e));
}

bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Whether no output has the place of an input or of another output (NULL: not given).
bool own_places(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
    for (auto o = outputs.begin(); o != outputs.end(); ++o)
        if (*o && (std::find(inputs.begin(), inputs.end(), *o) != inputs.end() || std::find(outputs.begin(), o, *o) != o)) return false;
    return true;
}

// A launch goes to the current device, so the stream has to be one of its own.
cmoe_status check_stream(hipStream_t st, int device) {
    if (!st) return CMOE_OK;  // the current device's null stream
    hipDevice_t dev = -1;
    const hipError_t e = hipStreamGetDevice(st, &dev);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        return fail(CMOE_ERR_INVALID_ARG, "not a stream: %s", hipGetErrorString(e));
    }
    if (dev != device) return fail(CMOE_ERR_INVALID_ARG, "the stream belongs to device %d, the current device is %d", dev, device);
    return CMOE_OK;
}

cmoe_status current_device(int* device) {
    const hipError_t e = hipGetDevice(device);
    if (e == hipSuccess) return CMOE_OK;
    (void)hipGetLastError();
    return hip_fail(e, "hipGetDevice");
}

constexpr int32_t kMaxRows = 1 << 21;   // of one norm: its grid stays under 2^32 threads
constexpr int32_t kMaxWidth = 1 << 24;  // of one norm: a row is one workgroup's

size_t elem(int dtype) { return dtype == CMOE_BF16 ? 2 : 4; }

// What a norm needs besides its stream.  outputs: one at least has to be given.
cmoe_status check_norm(const cmoe_norm* n, bool outputs) {
    if (!n) return fail(CMOE_ERR_INVALID_ARG, "norm: arguments are NULL");
    if (n->rows < 0 || n->d < 1) return fail(CMOE_ERR_INVALID_ARG, "norm: rows must be >= 0 and d >= 1");
    if (n->dtype != CMOE_F32 && n->dtype != CMOE_BF16) return fail(CMOE_ERR_INVALID_ARG, "norm: unknown dtype");
    if (n->delta && n->delta_dtype != CMOE_F32 && n->delta_dtype != CMOE_BF16)
        return fail(CMOE_ERR_INVALID_ARG, "norm: unknown delta dtype");
    if (!(std::isfinite(n->eps) && n->eps >= 0.0f)) return fail(CMOE_ERR_INVALID_ARG, "norm: eps must be finite and >= 0");
    if (n->rows > kMaxRows) return fail(CMOE_ERR_UNSUPPORTED, "norm: more than %d rows are not supported", kMaxRows);
    if (n->d > kMaxWidth) return fail(CMOE_ERR_UNSUPPORTED, "norm: d > %d is not supported", kMaxWidth);
    if (!n->residual && n->rows) return fail(CMOE_ERR_INVALID_ARG, "norm: residual is required");
    if (outputs && n->rows && !n->h && !n->h8 && !n->residual_out) return fail(CMOE_ERR_INVALID_ARG, "norm: no output is given");
    if (!n->h8 != !n->h8_scale) return fail(CMOE_ERR_INVALID_ARG, "norm: h8 and h8_scale go together");
    if (n->h8 && n->d % 32) return fail(CMOE_ERR_INVALID_ARG, "norm: the 8-bit output needs d to be a multiple of 32");
    for (const auto& [p, stride] : {std::pair<const void*, int64_t>{n->residual, n->residual_stride},
                                    {n->delta, n->delta_stride},
                                    {n->residual_out, n->residual_out_stride},
                                    {n->h, n->h_stride},
                                    {n->h8, n->h8_stride}})
        if (p && stride < n->d) return fail(CMOE_ERR_INVALID_ARG, "norm: a row stride is less than d");
    if (n->h8 && n->h8_scale_stride < n->d / 32)
        return fail(CMOE_ERR_INVALID_ARG, "norm: the scales' row stride is less than d / 32");
    const size_t a = elem(n->dtype), ad = elem(n->delta_dtype);
    if (!aligned_to(n->residual, a) || !aligned_to(n->residual_out, a) || !aligned_to(n->weight, a) || !aligned_to(n->h, a) ||
        (n->delta && !aligned_to(n->delta, ad)) || !aligned_to(n->n_rows, 4))
        return fail(CMOE_ERR_INVALID_ARG, "norm: a pointer is not aligned to its values");
    // every element is read and written by one thread: in place is fine for the sum only
    if (n->residual_out == n->residual && n->residual && n->residual_out_stride != n->residual_stride)
        return fail(CMOE_ERR_INVALID_ARG, "norm: in place, the two residual strides must be equal");
    if (!own_places({n->h, n->h8, n->h8_scale, n->residual_out}, {n->delta, n->weight, n->n_rows}) ||
        !own_places({n->h, n->h8, n->h8_scale}, {n->residual}))
        return fail(CMOE_ERR_INVALID_ARG, "norm: an output has the place of an input or another output");
    return CMOE_OK;
}

cmoe::NormArgs norm_args(const cmoe_norm* n) {
    cmoe::NormArgs a{};
    a.rows = n->rows; a.d = n->d; a.bf16 = n->dtype == CMOE_BF16; a.delta_bf16 = n->delta_dtype == CMOE_BF16;
    a.eps = n->eps;
    a.residual = n->residual; a.residual_stride = n->residual_stride;
    a.delta = n->delta; a.delta_stride = n->delta_stride;
    a.residual_out = n->residual_out; a.residual_out_stride = n->residual_out_stride;
    a.weight = n->weight;
    a.h = n->h; a.h_stride = n->h_stride;
    a.h8 = n->h8; a.h8_stride = n->h8_stride;
    a.h8_scale = n->h8_scale; a.h8_scale_stride = n->h8_scale_stride;
    a.n_rows = n->n_rows;
    return a;
}

// Whether every row of `a` takes 16-byte accesses (8-byte ones for 8-bit rows).
bool norm_aligned(const cmoe::NormArgs& a) {
    auto row = [](const void* p, int64_t stride, size_t e, size_t n) { return !p || (aligned_to(p, n) && stride * e % n == 0); };
    const size_t e = a.bf16 ? 2 : 4, ed = a.delta_bf16 ? 2 : 4;
    return a.d % 8 == 0 && row(a.residual, a.residual_stride, e, 16) && row(a.delta, a.delta_stride, ed, 16) &&
           row(a.residual_out, a.residual_out_stride, e, 16) && row(a.h, a.h_stride, e, 16) && row(a.weight, 0, e, 16) &&
           row(a.h8, a.h8_stride, 1, 8);
}

// Offsets of the workspace's parts.
struct Parts {
    size_t plan, z, gate, expert, h, h8, h8_scale, x, act, out, total;
};

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

cmoe_status check_moe(const cmoe_moe_config* c) {
    if (!c) return fail(CMOE_ERR_INVALID_ARG, "config is NULL");
    if (c->L < 1 || c->N < 1 || c->K < 1 || c->d < 1 || c->F < 1 || c->T < 1)
        return fail(CMOE_ERR_INVALID_ARG, "L, N, K, d, F and T must be >= 1");
    if (c->K > c->N) return fail(CMOE_ERR_INVALID_ARG, "K must not exceed N");
    if (c->dtype != CMOE_F32 && c->dtype != CMOE_BF16) return fail(CMOE_ERR_INVALID_ARG, "unknown dtype");
    for (int32_t f : {c->weights, c->activations})
        if (f != CMOE_FORMAT_DTYPE && f != CMOE_FORMAT_MX8) return fail(CMOE_ERR_INVALID_ARG, "unknown format");
    if (c->T > cmoe::kMoeTokens)
        return fail(CMOE_ERR_UNSUPPORTED, "T > %d is not supported: larger batches go in several calls", cmoe::kMoeTokens);
    if (c->N > cmoe::kMaxN) return fail(CMOE_ERR_UNSUPPORTED, "N > 256 is not supported");
    if (c->K > cmoe::kMaxK) return fail(CMOE_ERR_UNSUPPORTED, "K > 64 is not supported");
    if (c->d % 64 || c->F % 64) return fail(CMOE_ERR_UNSUPPORTED, "d and F must be multiples of 64");
    if (c->d > 1 << 16 || c->F > 1 << 16) return fail(CMOE_ERR_UNSUPPORTED, "d and F above 65536 are not supported");
    if (c->weights == CMOE_FORMAT_MX8 && c->dtype != CMOE_BF16)
        return fail(CMOE_ERR_UNSUPPORTED, "8-bit weights go with the bf16 type");
    if (c->activations == CMOE_FORMAT_MX8 && c->weights != CMOE_FORMAT_MX8)
        return fail(CMOE_ERR_UNSUPPORTED, "8-bit activations go with 8-bit weights");
    return CMOE_OK;
}

Parts moe_parts(const cmoe_moe_config* c) {
    Parts p{};
    size_t o = 0;
    auto take = [&o](size_t bytes) {
        const size_t at = o;
        o += align256(bytes);
        return at;
    };
    const size_t T = c->T, d = c->d, rows = T * c->K, e = elem(c->dtype);
    const bool a8 = c->activations == CMOE_FORMAT_MX8;
    p.plan = take(sizeof(cmoe::MoePlan));
    p.z = take(T * c->N * 4);
    p.gate = take(rows * 4);
    p.expert = take(rows * 4);
    p.h = take(T * d * e);
    p.h8 = take(a8 ? T * d : 0);
    p.h8_scale = take(a8 ? T * d / 32 : 0);
    p.x = take(a8 ? T * d * 2 : 0);
    p.act = take(rows * c->F * (c->dtype == CMOE_BF16 ? 6 : 4));
    p.out = take(rows * d * 4);
    p.total = o;
    return p;
}

}  // namespace

struct cmoe_moe {
    cmoe_moe_config cfg;
    cmoe_moe_weights w;
    Parts parts;
    char* ws;
    hipStream_t stream;
    int device;
};

namespace {

cmoe_status usable(cmoe_moe* m) {
    if (!m) return fail(CMOE_ERR_INVALID_ARG, "handle is NULL");
    int device = -1;
    if (hipGetDevice(&device) != hipSuccess || device != m->device) {
        (void)hipGetLastError();
        return fail(CMOE_ERR_INVALID_ARG, "the current device is not the one the handle was created on");
    }
    return CMOE_OK;
}

// What both calls of a layer share; the layer's own inputs are checked by the caller.
cmoe_status check_call(cmoe_moe* m, const cmoe_moe_call* c) {
    const cmoe_moe_config& g = m->cfg;
    if (!c) return fail(CMOE_ERR_INVALID_ARG, "arguments are NULL");
    if (c->layer < 0 || c->layer >= g.L) return fail(CMOE_ERR_INVALID_ARG, "layer must be in [0, L)");
    if (c->T < 0 || c->T > g.T) return fail(CMOE_ERR_INVALID_ARG, "T must be in [0, the configuration's T]");
    if (!c->y && c->T) return fail(CMOE_ERR_INVALID_ARG, "y is required");
    if (c->y_stride < g.d) return fail(CMOE_ERR_INVALID_ARG, "the row stride of y is less than d");
    if (!aligned_to(c->y, 16) || c->y_stride % 4) return fail(CMOE_ERR_UNSUPPORTED, "rows of y must be 16-byte aligned");
    if (!aligned_to(c->n_tokens, 4) || !aligned_to(c->selected, 4) || !aligned_to(c->gates, 4))
        return fail(CMOE_ERR_INVALID_ARG, "a pointer is not aligned to its values");
    return CMOE_OK;
}

cmoe_status run_layer(cmoe_moe* m, const cmoe_moe_call* c, const void* h, int64_t h_stride, const uint8_t* h8, int64_t h8_stride,
                      const uint8_t* h8_scale, int64_t h8_scale_stride) {
    const cmoe_moe_config& g = m->cfg;
    const size_t e = elem(g.dtype), experts = (size_t)g.N * 3 * g.d * g.F;
    cmoe::MoeArgs a{};
    a.N = g.N; a.K = g.K; a.d = g.d; a.F = g.F; a.T = c->T;
    a.bf16 = g.dtype == CMOE_BF16;
    a.format = g.weights == CMOE_FORMAT_MX8 ? cmoe::kMoeMx8 : a.bf16 ? cmoe::kMoeBf16 : cmoe::kMoeF32;
    a.w_router = static_cast<const char*>(m->w.w_router) + (size_t)c->layer * g.N * g.d * e;
    a.bias = m->w.logit_bias ? m->w.logit_bias + (size_t)c->layer * g.N : nullptr;
    a.experts = static_cast<const char*>(m->w.experts) + (size_t)c->layer * experts * (a.format == cmoe::kMoeMx8 ? 1 : e);
    a.scales = a.format == cmoe::kMoeMx8 ? m->w.expert_scales + (size_t)c->layer * (experts / 32) : nullptr;
    a.h = h; a.h_stride = h_stride;
    a.h8 = h8; a.h8_stride = h8_stride; a.h8_scale = h8_scale; a.h8_scale_stride = h8_scale_stride;
    a.y = c->y; a.y_stride = c->y_stride;
    a.n_tokens = c->n_tokens; a.selected = c->selected; a.gates = c->gates;
    a.plan = reinterpret_cast<cmoe::MoePlan*>(m->ws + m->parts.plan);
    a.z = reinterpret_cast<float*>(m->ws + m->parts.z);
    a.gate = reinterpret_cast<float*>(m->ws + m->parts.gate);
    a.expert = reinterpret_cast<int32_t*>(m->ws + m->parts.expert);
    a.x = reinterpret_cast<uint16_t*>(m->ws + m->parts.x);
    a.act = m->ws + m->parts.act;
    a.out = reinterpret_cast<float*>(m->ws + m->parts.out);
    const hipError_t err = cmoe::launch_moe(a, m->stream);
    return err == hipSuccess ? CMOE_OK : hip_fail(err, "MoE layer");
}

}  // namespace

extern "C" {

cmoe_status cmoe_add_norm(const cmoe_norm* n, void* stream) {
    cmoe_status st = check_norm(n, true);
    if (st != CMOE_OK) return st;
    int device = 0;
    if ((st = current_device(&device)) != CMOE_OK) return st;
    if ((st = check_stream(static_cast<hipStream_t>(stream), device)) != CMOE_OK) return st;
    if (n->rows == 0) return CMOE_OK;
    const cmoe::NormArgs a = norm_args(n);
    const hipError_t e = cmoe::launch_norm(a, norm_aligned(a), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? CMOE_OK : hip_fail(e, "norm");
}

cmoe_status cmoe_quantize(const void* src, int32_t dtype, int64_t rows, int64_t cols, int64_t src_stride, uint8_t* q,
                          int64_t q_stride, uint8_t* scale, int64_t scale_stride, void* stream) {
    if (rows < 0 || cols < 0) return fail(CMOE_ERR_INVALID_ARG, "quantize: rows and cols must be >= 0");
    if (dtype != CMOE_F32 && dtype != CMOE_BF16) return fail(CMOE_ERR_INVALID_ARG, "quantize: unknown dtype");
    if (cols % 32) return fail(CMOE_ERR_INVALID_ARG, "quantize: cols must be a multiple of 32");
    if (cols && rows > ((int64_t)1 << 34) / cols) return fail(CMOE_ERR_UNSUPPORTED, "quantize: more than 2^34 values");
    if (rows && cols) {
        if (!src || !q || !scale) return fail(CMOE_ERR_INVALID_ARG, "quantize: src, q and scale are required");
        if (src_stride < cols || q_stride < cols || scale_stride < cols / 32)
            return fail(CMOE_ERR_INVALID_ARG, "quantize: a row stride is less than the row");
        const int64_t e = (int64_t)elem(dtype);
        if (!aligned_to(src, 16) || src_stride * e % 16 || !aligned_to(q, 16) || q_stride % 16)
            return fail(CMOE_ERR_UNSUPPORTED, "quantize: rows of src and q must be 16-byte aligned");
        if (src == q || src == scale || q == scale) return fail(CMOE_ERR_INVALID_ARG, "quantize: an output has the place of src or the other output");
    }
    int device = 0;
    cmoe_status st = current_device(&device);
    if (st == CMOE_OK) st = check_stream(static_cast<hipStream_t>(stream), device);
    if (st != CMOE_OK || rows == 0 || cols == 0) return st;
    const cmoe::QuantizeArgs a{dtype == CMOE_BF16, src, rows, cols, src_stride, q, q_stride, scale, scale_stride};
    const hipError_t err = cmoe::launch_quantize(a, static_cast<hipStream_t>(stream));
    return err == hipSuccess ? CMOE_OK : hip_fail(err, "quantize");
}

cmoe_status cmoe_moe_query(const cmoe_moe_config* cfg, size_t* workspace_bytes) {
    const cmoe_status st = check_moe(cfg);
    if (st != CMOE_OK) return st;
    if (!workspace_bytes) return fail(CMOE_ERR_INVALID_ARG, "size output is NULL");
    *workspace_bytes = moe_parts(cfg).total;
    return CMOE_OK;
}

cmoe_status cmoe_moe_init(const cmoe_moe_config* cfg, const cmoe_moe_weights* w, void* workspace, void* stream, cmoe_moe** out) {
    if (out) *out = nullptr;
    cmoe_status st = check_moe(cfg);
    if (st != CMOE_OK) return st;
    if (!w || !out) return fail(CMOE_ERR_INVALID_ARG, "weights and output handle are required");
    if (!w->w_router || !w->experts) return fail(CMOE_ERR_INVALID_ARG, "w_router and experts are required");
    if (cfg->weights == CMOE_FORMAT_MX8 && !w->expert_scales)
        return fail(CMOE_ERR_INVALID_ARG, "expert_scales is required with 8-bit weights");
    if (!workspace || !aligned_to(workspace, 256)) return fail(CMOE_ERR_INVALID_ARG, "a workspace is required, 256-byte aligned");
    if (!aligned_to(w->w_router, 16) || !aligned_to(w->experts, 16) || !aligned_to(w->logit_bias, 4) ||
        (cfg->weights == CMOE_FORMAT_MX8 && !aligned_to(w->expert_scales, 4)))
        return fail(CMOE_ERR_INVALID_ARG, "w_router and experts must be 16-byte aligned, logit_bias and expert_scales 4-byte");
    int device = 0;
    if ((st = current_device(&device)) != CMOE_OK) return st;
    if ((st = check_stream(static_cast<hipStream_t>(stream), device)) != CMOE_OK) return st;
    // refuse what the device cannot read rather than fault later
    for (const void* p : {w->w_router, w->experts, static_cast<const void*>(w->expert_scales), static_cast<const void*>(w->logit_bias),
                          static_cast<const void*>(workspace)}) {
        if (!p || (p == w->expert_scales && cfg->weights != CMOE_FORMAT_MX8)) continue;
        hipPointerAttribute_t attr;
        if (hipPointerGetAttributes(&attr, p) != hipSuccess || attr.type != hipMemoryTypeDevice || attr.device != device) {
            (void)hipGetLastError();
            return fail(CMOE_ERR_INVALID_ARG, "a weight or the workspace is not memory of the current device");
        }
    }
    cmoe_moe* m = new (std::nothrow) cmoe_moe{};
    if (!m) return fail(CMOE_ERR_UNSUPPORTED, "no host memory for the handle");
    m->cfg = *cfg;
    m->w = *w;
    m->parts = moe_parts(cfg);
    m->ws = static_cast<char*>(workspace);
    m->stream = static_cast<hipStream_t>(stream);
    m->device = device;
    *out = m;
    return CMOE_OK;
}

cmoe_status cmoe_moe_layer(cmoe_moe* m, const cmoe_moe_call* c) {
    cmoe_status st = usable(m);
    if (st == CMOE_OK) st = check_call(m, c);
    if (st != CMOE_OK) return st;
    const cmoe_moe_config& g = m->cfg;
    const bool a8 = g.activations == CMOE_FORMAT_MX8;
    if (c->T == 0) return CMOE_OK;
    if (!c->h) return fail(CMOE_ERR_INVALID_ARG, "h is required");
    if (c->h_stride < g.d) return fail(CMOE_ERR_INVALID_ARG, "the row stride of h is less than d");
    if (!aligned_to(c->h, 16) || c->h_stride * (int64_t)elem(g.dtype) % 16)
        return fail(CMOE_ERR_UNSUPPORTED, "rows of h must be 16-byte aligned");
    if (a8 && (!c->h8 || !c->h8_scale)) return fail(CMOE_ERR_INVALID_ARG, "h8 and h8_scale are required with 8-bit activations");
    if (a8 && (c->h8_stride < g.d || c->h8_scale_stride < g.d / 32))
        return fail(CMOE_ERR_INVALID_ARG, "a row stride of h8 or h8_scale is less than the row");
    if (a8 && (!aligned_to(c->h8, 16) || c->h8_stride % 16)) return fail(CMOE_ERR_UNSUPPORTED, "rows of h8 must be 16-byte aligned");
    if (!a8 && (c->h8 || c->h8_scale)) return fail(CMOE_ERR_INVALID_ARG, "h8 is given, but the configuration's activations are not 8-bit");
    if (!own_places({c->y, c->selected, c->gates}, {c->h, c->h8, c->h8_scale, c->n_tokens}))
        return fail(CMOE_ERR_INVALID_ARG, "an output has the place of an input or another output");
    return run_layer(m, c, c->h, c->h_stride, c->h8, c->h8_stride, c->h8_scale, c->h8_scale_stride);
}

cmoe_status cmoe_moe_block(cmoe_moe* m, const cmoe_norm* n, const cmoe_moe_call* c) {
    cmoe_status st = usable(m);
    if (st == CMOE_OK) st = check_call(m, c);
    if (st != CMOE_OK) return st;
    const cmoe_moe_config& g = m->cfg;
    if (c->h || c->h8 || c->h8_scale) return fail(CMOE_ERR_INVALID_ARG, "h comes from the norm: h, h8 and h8_scale must be NULL");
    if (!n) return fail(CMOE_ERR_INVALID_ARG, "norm: arguments are NULL");
    if (n->rows != c->T || n->d != g.d || n->dtype != g.dtype)
        return fail(CMOE_ERR_INVALID_ARG, "norm: rows, d and dtype must be the layer's");
    if (n->h || n->h8 || n->h8_scale) return fail(CMOE_ERR_INVALID_ARG, "norm: h goes through the workspace: h, h8 and h8_scale must be NULL");
    if (n->n_rows) return fail(CMOE_ERR_INVALID_ARG, "norm: the number of rows is the call's n_tokens");
    if ((st = check_norm(n, false)) != CMOE_OK) return st;
    if (c->T == 0) return CMOE_OK;
    if (!own_places({c->y, c->selected, c->gates, n->residual_out}, {n->weight, c->n_tokens}) ||
        !own_places({c->y, c->selected, c->gates}, {n->residual}) || !own_places({c->selected, c->gates}, {n->delta}))
        return fail(CMOE_ERR_INVALID_ARG, "an output has the place of an input or another output");
    cmoe::NormArgs a = norm_args(n);
    const bool a8 = g.activations == CMOE_FORMAT_MX8;
    a.n_rows = c->n_tokens;
    a.h = m->ws + m->parts.h;
    a.h_stride = g.d;
    if (a8) {
        a.h8 = reinterpret_cast<uint8_t*>(m->ws + m->parts.h8);
        a.h8_stride = g.d;
        a.h8_scale = reinterpret_cast<uint8_t*>(m->ws + m->parts.h8_scale);
        a.h8_scale_stride = g.d / 32;
    }
    const hipError_t e = cmoe::launch_norm(a, norm_aligned(a), m->stream);
    if (e != hipSuccess) return hip_fail(e, "norm");
    return run_layer(m, c, a.h, a.h_stride, a.h8, a.h8_stride, a.h8_scale, a.h8_scale_stride);
}

cmoe_status cmoe_moe_destroy(cmoe_moe* m) {
    delete m;
    return CMOE_OK;
}

}  // extern "C"
