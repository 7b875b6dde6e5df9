// C entry points of the operators in MX4 and of those for experts: argument checks, the weights' handle.
#include <math.h>

#include <new>

#include "nm_mx4_internal.h"
#include "nm_rows_checks.h"

using namespace nm;

namespace {

constexpr int64_t kMaxGather = ((int64_t)1 << 32) - (1 << 16);   // the kernels' offsets into gathered rows have 32 bits

inline int blocks_of(int width) { return (width + 31) / 32; }

// Codes and scales of rows in MX4.
int check_mx4(const char* what, const Span& q, const char* scales_name, const Span& s, bool output)
{
    NM_TRY(check_span(what, q, output));
    NM_TRY(check_span(scales_name, s, output));
    if ((uintptr_t)q.p % 16 || (q.rows > 1 && q.ld % 16)) {
        set_error("rows of %s must start at multiples of 16 bytes", what);
        return NM_ERR_ARG;
    }
    return NM_OK;
}

int rows_call(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, const void* res, int64_t ldr,
              const float* gamma, double eps, bool norm, void* out, int64_t ldo, uint8_t* q, int64_t ldq, uint8_t* scales,
              int64_t lds, void* stream)
{
    if (!float_dtype(dt)) {
        set_error("x must be fp32 or bf16");
        return NM_ERR_ARG;
    }
    NM_TRY(check_rows(rows, width));
    if (!(eps >= 0.0) || isinf(eps)) {
        set_error("eps must be finite and not negative");
        return NM_ERR_ARG;
    }
    if (rows == 0) return NM_OK;
    const size_t es = q8_elem(dt);
    const int nb = blocks_of(width);
    const Span sx{x, es, rows, width, ldx}, sr{res, es, rows, width, ldr}, so{out, es, rows, width, ldo},
        sq{q, 1, rows, nb * 16, ldq}, ss{scales, 1, rows, nb, lds}, sg{gamma, 4, 1, width, width};
    NM_TRY(check_span("x", sx, false));
    if (res) NM_TRY(check_span("residual", sr, false));
    if (gamma) NM_TRY(check_span("gamma", sg, false));
    if (out) NM_TRY(check_span("residual_out", so, true));
    NM_TRY(check_mx4("q", sq, "scales", ss, true));
    const Span* outs[3] = {&so, &sq, &ss};
    const char* names[3] = {"residual_out", "q", "scales"};
    for (int i = 0; i < 3; ++i) {
        NM_TRY(check_apart(names[i], *outs[i], "x", sx, i == 0));
        NM_TRY(check_apart(names[i], *outs[i], "residual", sr, i == 0));
        NM_TRY(check_apart(names[i], *outs[i], "gamma", sg, false));
        for (int j = i + 1; j < 3; ++j) NM_TRY(check_apart(names[i], *outs[i], names[j], *outs[j], false));
    }
    return run_mx4_rows(x, dt, rows, width, ldx, res, ldr, gamma, eps, norm, out, ldo, q, ldq, scales, lds, (hipStream_t)stream);
}

int check_device(const nm_mx4* w)
{
    int dev = -1;
    NM_HIP_CHECK(hipGetDevice(&dev));
    if (dev != w->device) {
        set_error("packed weights live on device %d, current device is %d", w->device, dev);
        return NM_ERR_ARG;
    }
    return NM_OK;
}

void free_mx4(nm_mx4* w)
{
    if (!w) return;
    // A handle may go (by its owner's garbage collection) while a stream is being captured, which hipFree ends unless the thread allows it.
    hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
    const bool changed = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
    (void)hipFree(w->d_w);
    (void)hipFree(w->d_s);
    if (changed) (void)hipThreadExchangeStreamCaptureMode(&mode);
    delete w;
}

int pack_into(nm_mx4* h, const void* w, nm_dtype_t dt, const uint8_t* scales, int64_t lds, int64_t ldw, hipStream_t s)
{
    if (hipMalloc((void**)&h->d_w, h->w_bytes()) != hipSuccess || hipMalloc((void**)&h->d_s, h->s_bytes()) != hipSuccess) {
        (void)hipGetLastError();
        set_error("hipMalloc(%zu) for packed weights failed", h->w_bytes());
        return NM_ERR_ALLOC;
    }
    Temp rounded, rscales, bad;
    NM_TRY(bad.get(sizeof(int)));
    const uint8_t* q = (const uint8_t*)w;
    const int64_t rows = (int64_t)h->experts * h->channels;
    if (dt != NM_MX4) {
        NM_TRY(rounded.get((size_t)rows * h->blocks * 16));
        NM_TRY(rscales.get((size_t)rows * h->blocks));
        NM_TRY(run_mx4_rows(w, dt, rows, h->width, ldw, nullptr, 0, nullptr, 0.0, false, nullptr, 0, (uint8_t*)rounded.p, h->blocks * 16,
                            (uint8_t*)rscales.p, h->blocks, s));
        q = (const uint8_t*)rounded.p;
        scales = (const uint8_t*)rscales.p;
        ldw = h->blocks * 16;
        lds = h->blocks;
    }
    NM_TRY(run_mx4_pack(q, ldw, scales, lds, h, (int*)bad.p, s));
    int host_bad = 0;
    NM_HIP_CHECK(hipMemcpyAsync(&host_bad, bad.p, sizeof(int), hipMemcpyDeviceToHost, s));
    NM_HIP_CHECK(hipStreamSynchronize(s));
    if (host_bad) {
        set_error("a weight is not finite");
        return NM_ERR_ARG;
    }
    return NM_OK;
}

Mx4Product shape_of(const nm_mx4* w, int64_t rows, bool grouped)
{
    Mx4Product p{};
    p.rows = p.sources = (int)rows;
    p.channels = w->channels;
    p.outs = w->gated ? w->channels / 2 : w->channels;
    p.experts = w->experts;
    p.gated = w->gated;
    p.groups = w->groups;
    p.steps = w->steps;
    p.blocks = w->blocks;
    p.grouped = grouped;
    return p;
}

int product_call(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, int64_t sources, int width, const nm_mx4_t* w, bool grouped,
                 const int32_t* offsets, const int32_t* index, int64_t rows, const float* bias, const void* res, int64_t ldr, void* y,
                 nm_dtype_t dt, int64_t ldy, uint8_t* ys, int64_t ldys, void* stream)
{
    if (!w) {
        set_error("null handle");
        return NM_ERR_ARG;
    }
    if (!float_dtype(dt) && dt != NM_MX4) {
        set_error("y must be fp32, bf16 or MX4");
        return NM_ERR_ARG;
    }
    if (width != w->width) {
        set_error("width %d does not match the packed weights (%d)", width, w->width);
        return NM_ERR_ARG;
    }
    NM_TRY(check_rows(sources, width));
    NM_TRY(check_rows(rows, width));
    if (!grouped && w->experts != 1) {
        set_error("the weights are those of %d experts", w->experts);
        return NM_ERR_UNSUPPORTED;
    }
    if (res && (w->gated || dt == NM_MX4)) {
        set_error("gated weights and outputs in MX4 take no residual");
        return NM_ERR_UNSUPPORTED;
    }
    if (grouped && !index && sources != rows) {
        set_error("%lld rows and %lld entries, without an index", (long long)sources, (long long)rows);
        return NM_ERR_ARG;
    }
    NM_TRY(check_device(w));
    if (rows == 0) return NM_OK;
    if (sources == 0) {
        set_error("no rows to take %lld entries from", (long long)rows);
        return NM_ERR_ARG;
    }
    Mx4Product p = shape_of(w, rows, grouped);
    const bool rounded = dt == NM_MX4;
    const int nb = blocks_of(p.outs);
    const size_t es = q8_elem(dt);
    const Span sq{q, 1, sources, w->blocks * 16, ldq}, ss{scales, 1, sources, w->blocks, lds},
        sb{bias, 4, w->experts, w->channels, w->channels}, sr{res, es, rows, p.outs, ldr}, sy{y, es, rows, rounded ? nb * 16 : p.outs, ldy},
        sys{ys, 1, rows, nb, ldys}, so{offsets, 4, 1, w->experts + 1, w->experts + 1}, si{index, 4, rows, 1, 1};
    NM_TRY(check_mx4("q", sq, "scales", ss, false));
    if (grouped) NM_TRY(check_span("offsets", so, false));
    if (index) NM_TRY(check_span("index", si, false));
    if (index && (int64_t)(sq.bytes() > ss.bytes() ? sq.bytes() : ss.bytes()) > kMaxGather) {
        set_error("rows that are taken by an index span 4 GiB or more");
        return NM_ERR_SHAPE;
    }
    if (bias && (uintptr_t)bias % 4) {
        set_error("bias is not aligned to its element");
        return NM_ERR_ARG;
    }
    if (res) NM_TRY(check_span("residual", sr, false));
    if (rounded) NM_TRY(check_mx4("y", sy, "y_scales", sys, true));
    else NM_TRY(check_span("y", sy, true));
    if (!rounded && ys) {
        set_error("scales of an output that is not in MX4");
        return NM_ERR_ARG;
    }
    const Span* ins[6] = {&sq, &ss, &sb, &so, &si, &sr};
    const char* names[6] = {"q", "scales", "bias", "offsets", "index", "residual"};
    for (int i = 0; i < 6; ++i) {
        NM_TRY(check_apart("y", sy, names[i], *ins[i], i == 5));
        NM_TRY(check_apart("y_scales", sys, names[i], *ins[i], false));
    }
    NM_TRY(check_apart("y", sy, "y_scales", sys, false));
    p.q = q;
    p.s = scales;
    p.w = w->d_w;
    p.ws = w->d_s;
    p.bias = bias;
    p.res = res;
    p.y = y;
    p.ys = ys;
    p.offsets = offsets;
    p.index = index;
    p.ldq = ldq;
    p.lds = lds;
    p.ldr = ldr;
    p.ldy = ldy;
    p.ldys = ldys;
    p.sources = (int)sources;
    p.out = dt;
    p.past = sy.rows * sy.width * (int64_t)es > ((int64_t)160 << 20);
    return run_mx4_product(p, (hipStream_t)stream);
}

// The integers of a block are 64 bits wide; one that does not fit an int is out of range for every argument that is one.
inline int narrow(int64_t v) { return v < -1 || v > 0x7fffffff ? -1 : (int)v; }
inline size_t size_of(int64_t v) { return v < 0 ? 0 : (size_t)v; }

int null_block()
{
    set_error("null pointer argument");
    return NM_ERR_ARG;
}

}  // namespace

extern "C" {

int nm_quantize_mx4(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, uint8_t* q, int64_t ldq, uint8_t* scales, int64_t lds,
                    void* stream)
{
    return rows_call(x, dt, rows, width, ldx, nullptr, 0, nullptr, 0.0, false, nullptr, 0, q, ldq, scales, lds, stream);
}

int nm_rmsnorm_mx4(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, const void* res, int64_t ldr, const float* gamma,
                   double eps, void* out, int64_t ldo, uint8_t* q, int64_t ldq, uint8_t* scales, int64_t lds, void* stream)
{
    return rows_call(x, dt, rows, width, ldx, res, ldr, gamma, eps, true, out, ldo, q, ldq, scales, lds, stream);
}

int nm_dequantize_mx4(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, int64_t rows, int width, void* y, nm_dtype_t dt,
                      int64_t ldy, void* stream)
{
    if (!float_dtype(dt)) {
        set_error("y must be fp32 or bf16");
        return NM_ERR_ARG;
    }
    NM_TRY(check_rows(rows, width));
    if (rows == 0) return NM_OK;
    const int nb = blocks_of(width);
    const Span sq{q, 1, rows, nb * 16, ldq}, ss{scales, 1, rows, nb, lds}, sy{y, q8_elem(dt), rows, width, ldy};
    NM_TRY(check_mx4("q", sq, "scales", ss, false));
    NM_TRY(check_span("y", sy, true));
    NM_TRY(check_apart("y", sy, "q", sq, false));
    NM_TRY(check_apart("y", sy, "scales", ss, false));
    return run_mx4_dequantize(q, ldq, scales, lds, rows, width, y, dt, ldy, (hipStream_t)stream);
}

int nm_mx4_pack(const void* w, nm_dtype_t dt, const uint8_t* scales, int64_t lds, int experts, int channels, int width, int64_t ldw, int gated,
                void* stream, nm_mx4_t** out)
{
    if (!out) return null_block();
    *out = nullptr;
    if (dt != NM_MX4 && !float_dtype(dt)) {
        set_error("weights must be fp32, bf16 or MX4");
        return NM_ERR_ARG;
    }
    if (channels < 1 || (gated != 0 && gated != 1) || (gated && channels % 2) || experts < 1) {
        set_error("bad number of channels: %d (gated %d) of %d experts", channels, gated, experts);
        return NM_ERR_ARG;
    }
    const int64_t rows = (int64_t)experts * channels;
    if (channels > (1 << 24) || experts > NM_MX4_MAX_EXPERTS || rows > kMaxRows) {
        set_error("%d channels of %d experts: too many", channels, experts);
        return NM_ERR_SHAPE;
    }
    NM_TRY(check_rows(rows, width));
    if ((dt == NM_MX4) != (scales != nullptr)) {
        set_error("weights in MX4 come with scales, others without");
        return NM_ERR_ARG;
    }
    const int nb = blocks_of(width);
    if (dt == NM_MX4) NM_TRY(check_mx4("w", Span{w, 1, rows, nb * 16, ldw}, "scales", Span{scales, 1, rows, nb, lds}, false));
    else NM_TRY(check_span("w", Span{w, q8_elem(dt), rows, width, ldw}, false));
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    NM_HIP_CHECK(hipStreamIsCapturing((hipStream_t)stream, &cap));
    if (cap != hipStreamCaptureStatusNone) {
        set_error("weights cannot be packed under stream capture");
        return NM_ERR_HIP;
    }
    nm_mx4* h = new (std::nothrow) nm_mx4;
    if (!h) {
        set_error("out of host memory");
        return NM_ERR_ALLOC;
    }
    h->experts = experts;
    h->channels = channels;
    h->width = width;
    h->gated = gated;
    h->blocks = nb;
    h->groups = (channels + 63) / 64;
    h->steps = (nb + 7) / 8;
    const hipError_t e = hipGetDevice(&h->device);
    int rc = NM_OK;
    if (e != hipSuccess) {
        set_error("hipGetDevice failed: %s", hipGetErrorString(e));
        rc = NM_ERR_HIP;
    }
    if (rc == NM_OK) rc = pack_into(h, w, dt, scales, lds, ldw, (hipStream_t)stream);
    if (rc != NM_OK) {
        free_mx4(h);
        return rc;
    }
    *out = h;
    return NM_OK;
}

int nm_mx4_free(nm_mx4_t* w)
{
    free_mx4(w);
    return NM_OK;
}

int nm_mx4_dims(const nm_mx4_t* w, int* experts, int* channels, int* width, int* gated)
{
    if (!w) {
        set_error("null handle");
        return NM_ERR_ARG;
    }
    if (experts) *experts = w->experts;
    if (channels) *channels = w->channels;
    if (width) *width = w->width;
    if (gated) *gated = w->gated;
    return NM_OK;
}

int nm_mx4_export(const nm_mx4_t* w, uint8_t* q_host, uint8_t* scales_host)
{
    if (!w) {
        set_error("null handle");
        return NM_ERR_ARG;
    }
    NM_TRY(check_device(w));
    const size_t rows = (size_t)w->experts * w->channels, wb = rows * w->blocks * 16, sb = rows * w->blocks;
    Temp tw, ts;
    NM_TRY(tw.get(wb));
    NM_TRY(ts.get(sb));
    NM_TRY(run_mx4_unpack(w, (uint8_t*)tw.p, (uint8_t*)ts.p, nullptr));
    NM_HIP_CHECK(hipStreamSynchronize(nullptr));
    if (q_host) NM_HIP_CHECK(hipMemcpy(q_host, tw.p, wb, hipMemcpyDeviceToHost));
    if (scales_host) NM_HIP_CHECK(hipMemcpy(scales_host, ts.p, sb, hipMemcpyDeviceToHost));
    return NM_OK;
}

int nm_linear_mx4(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, int64_t rows, int width, const nm_mx4_t* w,
                  const float* bias, const void* res, int64_t ldr, void* y, nm_dtype_t dt, int64_t ldy, uint8_t* ys, int64_t ldys,
                  void* stream)
{
    return product_call(q, ldq, scales, lds, rows, width, w, false, nullptr, nullptr, rows, bias, res, ldr, y, dt, ldy, ys, ldys, stream);
}

int nm_experts_mx4(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, int64_t rows, int width, const nm_mx4_t* w,
                   const int32_t* offsets, const int32_t* index, int64_t entries, const float* bias, void* y, nm_dtype_t dt, int64_t ldy,
                   uint8_t* ys, int64_t ldys, void* stream)
{
    return product_call(q, ldq, scales, lds, rows, width, w, true, offsets, index, entries, bias, nullptr, 0, y, dt, ldy, ys, ldys, stream);
}

int nm_route_workspace(int64_t tokens, int experts, size_t* bytes)
{
    if (!bytes) return null_block();
    if (tokens < 0 || tokens > kMaxRows || experts < 1 || experts > NM_ROUTE_MAX_EXPERTS) {
        set_error("bad sizes: %lld tokens, %d experts", (long long)tokens, experts);
        return NM_ERR_ARG;
    }
    *bytes = route_workspace(tokens, experts);
    return NM_OK;
}

int nm_route(const void* logits, nm_dtype_t dt, int64_t tokens, int experts, int64_t ld, int choices, int normalise, int32_t* ids,
             float* weights, int32_t* offsets, int32_t* rows, int32_t* slots, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!float_dtype(dt)) {
        set_error("logits must be fp32 or bf16");
        return NM_ERR_ARG;
    }
    if (tokens < 0 || experts < 1 || choices < 1 || choices > experts || (normalise != 0 && normalise != 1)) {
        set_error("bad sizes: %lld tokens, %d of %d experts (normalise %d)", (long long)tokens, choices, experts, normalise);
        return NM_ERR_ARG;
    }
    if (experts > NM_ROUTE_MAX_EXPERTS || choices > NM_ROUTE_MAX_CHOICES || tokens > kMaxRows || tokens * choices > 0x7fffffff) {
        set_error("%lld tokens, %d of %d experts: too many", (long long)tokens, choices, experts);
        return NM_ERR_SHAPE;
    }
    const Span sl{logits, q8_elem(dt), tokens, experts, ld}, so{offsets, 4, 1, experts + 1, experts + 1}, si{ids, 4, tokens, choices, choices},
        sw{weights, 4, tokens, choices, choices}, sr{rows, 4, tokens, choices, choices}, ss{slots, 4, tokens, choices, choices};
    NM_TRY(check_span("offsets", so, true));
    const Span* outs[5] = {&so, &si, &sw, &sr, &ss};
    const char* names[5] = {"offsets", "ids", "weights", "rows", "slots"};
    if (tokens > 0) {
        NM_TRY(check_span("logits", sl, false));
        for (int i = 1; i < 5; ++i) NM_TRY(check_span(names[i], *outs[i], true));
        for (int i = 0; i < 5; ++i) {
            NM_TRY(check_apart(names[i], *outs[i], "logits", sl, false));
            for (int j = i + 1; j < 5; ++j) NM_TRY(check_apart(names[i], *outs[i], names[j], *outs[j], false));
        }
    }
    const size_t need = route_workspace(tokens, experts);
    if (need) {
        if (!workspace || workspace_bytes < need || (uintptr_t)workspace % 16) {
            set_error("this call needs %zu bytes of workspace, 16-byte aligned; %zu were given", need,
                      workspace ? workspace_bytes : (size_t)0);
            return NM_ERR_ARG;
        }
        const Span sp{workspace, 1, 1, (int64_t)need, (int64_t)need};
        NM_TRY(check_apart("workspace", sp, "logits", sl, false));
        for (int i = 0; i < 5; ++i) NM_TRY(check_apart("workspace", sp, names[i], *outs[i], false));
    }
    const Route r{logits, tokens, ld, dt == NM_BF16, experts, choices, normalise, ids, weights, offsets, rows, slots};
    return run_route(r, workspace, (hipStream_t)stream);
}

int nm_combine(const void* y, nm_dtype_t y_dt, int64_t entries, int64_t ldy, const int32_t* slots, const float* weights, int64_t tokens,
               int choices, int width, const void* res, int64_t ldr, void* out, nm_dtype_t dt, int64_t ldo, void* stream)
{
    if (!float_dtype(y_dt) || !float_dtype(dt)) {
        set_error("y and out must be fp32 or bf16");
        return NM_ERR_ARG;
    }
    NM_TRY(check_rows(tokens, width));
    NM_TRY(check_rows(entries, width));
    if (choices < 1) {
        set_error("bad number of choices: %d", choices);
        return NM_ERR_ARG;
    }
    if (choices > NM_ROUTE_MAX_CHOICES) {
        set_error("%d choices: too many", choices);
        return NM_ERR_SHAPE;
    }
    if (tokens == 0) return NM_OK;
    const size_t es = q8_elem(dt);
    const Span sy{y, q8_elem(y_dt), entries, width, ldy}, ss{slots, 4, tokens, choices, choices}, sw{weights, 4, tokens, choices, choices},
        sr{res, es, tokens, width, ldr}, so{out, es, tokens, width, ldo};
    if (entries) NM_TRY(check_span("y", sy, false));
    NM_TRY(check_span("slots", ss, false));
    NM_TRY(check_span("weights", sw, false));
    if (res) NM_TRY(check_span("residual", sr, false));
    NM_TRY(check_span("out", so, true));
    NM_TRY(check_apart("out", so, "y", sy, false));
    NM_TRY(check_apart("out", so, "slots", ss, false));
    NM_TRY(check_apart("out", so, "weights", sw, false));
    NM_TRY(check_apart("out", so, "residual", sr, true));
    const Combine c{y, slots, weights, res, out, entries, tokens, ldy, ldr, ldo, choices, width, y_dt == NM_BF16, dt == NM_BF16};
    return run_combine(c, (hipStream_t)stream);
}

int nm_rows_mx4_args(const nm_rows_mx4_args_t* a)
{
    if (!a) return null_block();
    if (a->norm)
        return nm_rmsnorm_mx4(a->x_dev, narrow(a->dtype), a->rows, narrow(a->width), a->ldx, a->residual_dev, a->ldr, a->gamma_dev, a->eps,
                              a->residual_out_dev, a->ldo, a->q_dev, a->ldq, a->scales_dev, a->lds, a->hip_stream);
    return nm_quantize_mx4(a->x_dev, narrow(a->dtype), a->rows, narrow(a->width), a->ldx, a->q_dev, a->ldq, a->scales_dev, a->lds, a->hip_stream);
}

int nm_dequantize_mx4_args(const nm_dequantize_mx4_args_t* a)
{
    if (!a) return null_block();
    return nm_dequantize_mx4(a->q_dev, a->ldq, a->scales_dev, a->lds, a->rows, narrow(a->width), a->y_dev, narrow(a->dtype), a->ldy, a->hip_stream);
}

int nm_product_mx4_args(const nm_product_mx4_args_t* a)
{
    if (!a) return null_block();
    if (a->offsets_dev)
        return nm_experts_mx4(a->q_dev, a->ldq, a->scales_dev, a->lds, a->rows, narrow(a->width), a->w, a->offsets_dev, a->index_dev, a->entries,
                              a->bias_dev, a->y_dev, narrow(a->dtype), a->ldy, a->y_scales_dev, a->ldys, a->hip_stream);
    return nm_linear_mx4(a->q_dev, a->ldq, a->scales_dev, a->lds, a->rows, narrow(a->width), a->w, a->bias_dev, a->residual_dev, a->ldr, a->y_dev,
                         narrow(a->dtype), a->ldy, a->y_scales_dev, a->ldys, a->hip_stream);
}

int nm_route_args(const nm_route_args_t* a)
{
    if (!a) return null_block();
    return nm_route(a->logits_dev, narrow(a->dtype), a->tokens, narrow(a->experts), a->ld, narrow(a->choices), narrow(a->normalise), a->ids_dev,
                    a->weights_dev, a->offsets_dev, a->rows_dev, a->slots_dev, a->workspace_dev, size_of(a->workspace_bytes), a->hip_stream);
}

int nm_combine_args(const nm_combine_args_t* a)
{
    if (!a) return null_block();
    return nm_combine(a->y_dev, narrow(a->y_dtype), a->entries, a->ldy, a->slots_dev, a->weights_dev, a->tokens, narrow(a->choices),
                      narrow(a->width), a->residual_dev, a->ldr, a->out_dev, narrow(a->dtype), a->ldo, a->hip_stream);
}

}  // extern "C"
