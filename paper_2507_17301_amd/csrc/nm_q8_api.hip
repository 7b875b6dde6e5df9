// C entry points of the 8-bit feed-forward operators: argument checks, the weights' handle.
#include <math.h>

#include <new>

#include "nm_q8_internal.h"

using namespace nm;

namespace {

constexpr int64_t kMaxRows = 1 << 30, kMaxStride = 1 << 24;

inline size_t q8_elem(nm_dtype_t dt) { return dt == NM_F32 ? 4 : dt == NM_BF16 ? 2 : 1; }
inline bool float_dtype(nm_dtype_t dt) { return dt == NM_F32 || dt == NM_BF16; }

// A tensor of rows as the checks see it.
struct Span {
    const void* p;
    size_t elem;
    int64_t rows, width, ld;
    size_t bytes() const { return ((size_t)(rows - 1) * (size_t)ld + (size_t)width) * elem; }
};

int check_rows(int64_t rows, int width)
{
    if (rows < 0 || rows > kMaxRows || width < 1) {
        set_error("bad sizes: %lld rows of %d", (long long)rows, width);
        return NM_ERR_ARG;
    }
    if (width > NM_Q8_MAX_WIDTH) {
        set_error("width %d exceeds %d", width, (int)NM_Q8_MAX_WIDTH);
        return NM_ERR_SHAPE;
    }
    return NM_OK;
}

int check_span(const char* what, const Span& t, bool output)
{
    if (!t.p) {
        set_error("%s is null", what);
        return NM_ERR_ARG;
    }
    if ((uintptr_t)t.p % t.elem) {
        set_error("%s is not aligned to its element", what);
        return NM_ERR_ARG;
    }
    if (t.ld < 0 || t.ld > kMaxStride || (output && t.rows > 1 && t.ld < t.width)) {
        set_error("row stride %lld of %s (width %lld) is out of range", (long long)t.ld, what, (long long)t.width);
        return NM_ERR_ARG;
    }
    return NM_OK;
}

// Whether an output may share bytes with another tensor.  Two column ranges of one wider tensor (same
// stride in bytes) do not, although their extents overlap.
bool overlap(const Span& a, const Span& b)
{
    if (!a.p || !b.p || a.rows < 1 || b.rows < 1) return false;
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    if (a0 + a.bytes() <= b0 || b0 + b.bytes() <= a0) return false;
    const size_t la = (size_t)a.ld * a.elem, lb = (size_t)b.ld * b.elem;
    if (la == lb && la > 0) {
        const size_t wa = (size_t)a.width * a.elem, wb = (size_t)b.width * b.elem;
        const size_t d = b0 >= a0 ? (b0 - a0) % la : (la - (a0 - b0) % la) % la;   // b's first column within a's rows
        if (d >= wa && d + wb <= la) return false;
    }
    return true;
}

int check_apart(const char* what, const Span& out, const char* other, const Span& in, bool same_allowed)
{
    if (!overlap(out, in)) return NM_OK;
    if (same_allowed && out.p == in.p && (out.ld == in.ld || out.rows <= 1) && out.elem == in.elem) return NM_OK;
    set_error("%s overlaps %s", what, other);
    return NM_ERR_ARG;
}

#define NM_TRY(expr)                        \
    do {                                    \
        const int rc__ = (expr);            \
        if (rc__ != NM_OK) return rc__;     \
    } while (0)

int rows_call(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, const void* res, int64_t ldr,
              const float* gamma, float eps, bool norm, void* out, int64_t ldo, int8_t* q, int64_t ldq, float* scales,
              void* stream)
{
    if (!float_dtype(dt)) {
        set_error("x must be fp32 or bf16");
        return NM_ERR_ARG;
    }
    NM_TRY(check_rows(rows, width));
    if (!(eps >= 0.0f) || isinf(eps)) {
        set_error("eps must be finite and not negative");
        return NM_ERR_ARG;
    }
    if (rows == 0) return NM_OK;
    const size_t es = q8_elem(dt);
    const Span sx{x, es, rows, width, ldx}, sr{res, es, rows, width, ldr}, so{out, es, rows, width, ldo},
        sq{q, 1, rows, width, ldq}, ss{scales, 4, rows, 1, 1}, sg{gamma, 4, 1, width, width};
    NM_TRY(check_span("x", sx, false));
    if (res) NM_TRY(check_span("residual", sr, false));
    if (gamma) NM_TRY(check_span("gamma", sg, false));
    if (out) NM_TRY(check_span("residual_out", so, true));
    NM_TRY(check_span("q", sq, true));
    NM_TRY(check_span("scales", ss, true));
    const Span* outs[3] = {&so, &sq, &ss};
    const char* names[3] = {"residual_out", "q", "scales"};
    for (int i = 0; i < 3; ++i) {
        NM_TRY(check_apart(names[i], *outs[i], "x", sx, i == 0));
        NM_TRY(check_apart(names[i], *outs[i], "residual", sr, i == 0));
        NM_TRY(check_apart(names[i], *outs[i], "gamma", sg, false));
        for (int j = i + 1; j < 3; ++j) NM_TRY(check_apart(names[i], *outs[i], names[j], *outs[j], false));
    }
    return run_q8_rows(x, dt, rows, width, ldx, res, ldr, gamma, eps, norm, out, ldo, q, ldq, scales, (hipStream_t)stream);
}

int check_device(const nm_q8* w)
{
    int dev = -1;
    NM_HIP_CHECK(hipGetDevice(&dev));
    if (dev != w->device) {
        set_error("packed weights live on device %d, current device is %d", w->device, dev);
        return NM_ERR_ARG;
    }
    return NM_OK;
}

void free_q8(nm_q8* w)
{
    if (!w) return;
    (void)hipFree(w->d_w);
    (void)hipFree(w->d_scales);
    delete w;
}

// Device memory for the length of one call.
struct Temp {
    void* p = nullptr;
    ~Temp() { if (p) (void)hipFree(p); }
    int get(size_t bytes)
    {
        if (hipMalloc(&p, bytes) == hipSuccess) return NM_OK;
        p = nullptr;
        (void)hipGetLastError();
        set_error("hipMalloc(%zu) failed", bytes);
        return NM_ERR_ALLOC;
    }
};

int pack_into(nm_q8* h, const void* w, nm_dtype_t dt, const float* scales, int64_t ldw, hipStream_t s)
{
    const size_t wbytes = (size_t)h->groups * h->kblocks * 4096, sbytes = (size_t)h->groups * 64 * sizeof(float);
    if (hipMalloc((void**)&h->d_w, wbytes) != hipSuccess || hipMalloc((void**)&h->d_scales, sbytes) != hipSuccess) {
        (void)hipGetLastError();
        set_error("hipMalloc(%zu) for packed weights failed", wbytes);
        return NM_ERR_ALLOC;
    }
    Temp rounded, rscales, bad;
    NM_TRY(bad.get(sizeof(int)));
    const int8_t* w8 = (const int8_t*)w;
    if (dt != NM_I8) {
        NM_TRY(rounded.get((size_t)h->channels * h->width));
        NM_TRY(rscales.get((size_t)h->channels * sizeof(float)));
        NM_TRY(run_q8_rows(w, dt, h->channels, h->width, ldw, nullptr, 0, nullptr, 0.0f, false, nullptr, 0,
                           (int8_t*)rounded.p, h->width, (float*)rscales.p, s));
        w8 = (const int8_t*)rounded.p;
        scales = (const float*)rscales.p;
        ldw = h->width;
    }
    NM_TRY(run_q8_pack(w8, ldw, scales, h, (int*)bad.p, s));
    int host_bad = 0;
    NM_HIP_CHECK(hipMemcpyAsync(&host_bad, bad.p, sizeof(int), hipMemcpyDeviceToHost, s));
    NM_HIP_CHECK(hipStreamSynchronize(s));
    if (host_bad) {
        set_error(dt == NM_I8 ? "a scale is not finite" : "a weight is not finite");
        return NM_ERR_ARG;
    }
    return NM_OK;
}

}  // namespace

extern "C" {

int nm_quantize_q8(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, int8_t* q, int64_t ldq,
                   float* scales, void* stream)
{
    return rows_call(x, dt, rows, width, ldx, nullptr, 0, nullptr, 0.0f, false, nullptr, 0, q, ldq, scales, stream);
}

int nm_rmsnorm_q8(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, const void* res, int64_t ldr,
                  const float* gamma, float eps, void* out, int64_t ldo, int8_t* q, int64_t ldq, float* scales, void* stream)
{
    return rows_call(x, dt, rows, width, ldx, res, ldr, gamma, eps, true, out, ldo, q, ldq, scales, stream);
}

int nm_dequantize_q8(const int8_t* q, int64_t ldq, const float* scales, int64_t rows, int width, void* y, nm_dtype_t dt,
                     int64_t ldy, void* stream)
{
    if (!float_dtype(dt)) {
        set_error("y must be fp32 or bf16");
        return NM_ERR_ARG;
    }
    NM_TRY(check_rows(rows, width));
    if (rows == 0) return NM_OK;
    const Span sq{q, 1, rows, width, ldq}, ss{scales, 4, rows, 1, 1}, sy{y, q8_elem(dt), rows, width, ldy};
    NM_TRY(check_span("q", sq, false));
    NM_TRY(check_span("scales", ss, false));
    NM_TRY(check_span("y", sy, true));
    NM_TRY(check_apart("y", sy, "q", sq, false));
    NM_TRY(check_apart("y", sy, "scales", ss, false));
    return run_q8_dequantize(q, ldq, scales, rows, width, y, dt, ldy, (hipStream_t)stream);
}

int nm_q8_pack(const void* w, nm_dtype_t dt, const float* scales, int channels, int width, int64_t ldw, int gated,
               void* stream, nm_q8_t** out)
{
    if (!out) {
        set_error("null pointer argument");
        return NM_ERR_ARG;
    }
    *out = nullptr;
    if (dt != NM_I8 && !float_dtype(dt)) {
        set_error("weights must be fp32, bf16 or 8-bit integers");
        return NM_ERR_ARG;
    }
    if (channels < 1 || (gated != 0 && gated != 1) || (gated && channels % 2)) {
        set_error("bad number of channels: %d (gated %d)", channels, gated);
        return NM_ERR_ARG;
    }
    if (channels > (1 << 24)) {
        set_error("%d channels: too many", channels);
        return NM_ERR_SHAPE;
    }
    NM_TRY(check_rows(channels, width));
    if ((dt == NM_I8) != (scales != nullptr)) {
        set_error("8-bit weights come with scales, others without");
        return NM_ERR_ARG;
    }
    NM_TRY(check_span("w", Span{w, q8_elem(dt), channels, width, ldw}, false));
    if (scales) NM_TRY(check_span("scales", Span{scales, 4, channels, 1, 1}, false));
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    NM_HIP_CHECK(hipStreamIsCapturing((hipStream_t)stream, &cap));
    if (cap != hipStreamCaptureStatusNone) {
        set_error("weights cannot be packed under stream capture");
        return NM_ERR_HIP;
    }
    nm_q8* h = new (std::nothrow) nm_q8;
    if (!h) {
        set_error("out of host memory");
        return NM_ERR_ALLOC;
    }
    h->channels = channels;
    h->width = width;
    h->gated = gated;
    h->groups = (channels + 63) / 64;
    h->kblocks = (width + 127) / 128 * 2;
    const hipError_t e = hipGetDevice(&h->device);
    int rc = NM_OK;
    if (e != hipSuccess) {
        set_error("hipGetDevice failed: %s", hipGetErrorString(e));
        rc = NM_ERR_HIP;
    }
    if (rc == NM_OK) rc = pack_into(h, w, dt, scales, ldw, (hipStream_t)stream);
    if (rc != NM_OK) {
        free_q8(h);
        return rc;
    }
    *out = h;
    return NM_OK;
}

int nm_q8_free(nm_q8_t* w)
{
    free_q8(w);
    return NM_OK;
}

int nm_q8_dims(const nm_q8_t* w, int* channels, int* width, int* gated)
{
    if (!w) {
        set_error("null handle");
        return NM_ERR_ARG;
    }
    if (channels) *channels = w->channels;
    if (width) *width = w->width;
    if (gated) *gated = w->gated;
    return NM_OK;
}

int nm_q8_export(const nm_q8_t* w, int8_t* w_host, float* scales_host)
{
    if (!w) {
        set_error("null handle");
        return NM_ERR_ARG;
    }
    NM_TRY(check_device(w));
    const size_t wb = (size_t)w->channels * w->width, sb = (size_t)w->channels * sizeof(float);
    Temp tw, ts;
    NM_TRY(tw.get(wb));
    NM_TRY(ts.get(sb));
    NM_TRY(run_q8_unpack(w, (int8_t*)tw.p, (float*)ts.p, nullptr));
    NM_HIP_CHECK(hipStreamSynchronize(nullptr));
    if (w_host) NM_HIP_CHECK(hipMemcpy(w_host, tw.p, wb, hipMemcpyDeviceToHost));
    if (scales_host) NM_HIP_CHECK(hipMemcpy(scales_host, ts.p, sb, hipMemcpyDeviceToHost));
    return NM_OK;
}

int nm_linear_q8_workspace(const int8_t* q, int64_t rows, int64_t ldq, const nm_q8_t* w, size_t* bytes)
{
    if (!w || !bytes) {
        set_error("null pointer argument");
        return NM_ERR_ARG;
    }
    NM_TRY(check_rows(rows, w->width));
    Q8Linear p{};
    p.q = q;
    p.ldq = ldq;
    p.rows = (int)rows;
    p.width = w->width;
    p.channels = w->channels;
    p.gated = w->gated;
    p.groups = w->groups;
    p.kblocks = w->kblocks;
    const Q8Plan plan = rows ? q8_plan(p) : Q8Plan{};
    *bytes = plan.rows_bytes + plan.part_bytes;
    return NM_OK;
}

int nm_linear_q8(const int8_t* q, int64_t rows, int width, int64_t ldq, const float* scales, const nm_q8_t* w,
                 const float* bias, const void* res, int64_t ldr, void* y, nm_dtype_t dt, int64_t ldy,
                 void* workspace, size_t workspace_bytes, void* stream)
{
    if (!w) {
        set_error("null handle");
        return NM_ERR_ARG;
    }
    if (!float_dtype(dt)) {
        set_error("y must be fp32 or bf16");
        return NM_ERR_ARG;
    }
    if (width != w->width) {
        set_error("width %d does not match the packed weights (%d)", width, w->width);
        return NM_ERR_ARG;
    }
    NM_TRY(check_rows(rows, width));
    if (w->gated && res) {
        set_error("gated weights take no residual");
        return NM_ERR_UNSUPPORTED;
    }
    NM_TRY(check_device(w));
    if (rows == 0) return NM_OK;
    const int outs = w->gated ? w->channels / 2 : w->channels;
    const size_t es = q8_elem(dt);
    const Span sq{q, 1, rows, width, ldq}, ss{scales, 4, rows, 1, 1}, sb{bias, 4, 1, w->channels, w->channels},
        sr{res, es, rows, outs, ldr}, sy{y, es, rows, outs, ldy};
    NM_TRY(check_span("q", sq, false));
    NM_TRY(check_span("scales", ss, false));
    if (bias) NM_TRY(check_span("bias", sb, false));
    if (res) NM_TRY(check_span("residual", sr, false));
    NM_TRY(check_span("y", sy, true));
    NM_TRY(check_apart("y", sy, "q", sq, false));
    NM_TRY(check_apart("y", sy, "scales", ss, false));
    NM_TRY(check_apart("y", sy, "bias", sb, false));
    NM_TRY(check_apart("y", sy, "residual", sr, true));
    Q8Linear p{};
    p.q = q;
    p.qs = scales;
    p.w = w->d_w;
    p.ws = w->d_scales;
    p.bias = bias;
    p.res = res;
    p.y = y;
    p.ldq = ldq;
    p.ldr = ldr;
    p.ldy = ldy;
    p.rows = (int)rows;
    p.width = width;
    p.channels = w->channels;
    p.outs = outs;
    p.gated = w->gated;
    p.groups = w->groups;
    p.kblocks = w->kblocks;
    p.y_bf16 = dt == NM_BF16;
    // In turn on one card: 8192 x 4096 -> 16384 (268 MB) 422 us past the cache and 455 through it, 4096 x 4096 -> 24576 (201 MB) 323 and 340;
    // 16384 x 1024 -> 4096 (134 MB) 89 and 83
    p.past = (size_t)rows * outs * es > ((size_t)160 << 20);
    const Q8Plan plan = q8_plan(p);
    const size_t need = plan.rows_bytes + plan.part_bytes;
    if (need) {
        if (!workspace || workspace_bytes < need || (uintptr_t)workspace % 16) {
            set_error("this call needs %zu bytes of workspace, 16-byte aligned; %zu were given", need,
                      workspace ? workspace_bytes : (size_t)0);
            return NM_ERR_ARG;
        }
        const Span sw{workspace, 1, 1, (int64_t)need, (int64_t)need};
        NM_TRY(check_apart("workspace", sw, "q", sq, false));
        NM_TRY(check_apart("workspace", sw, "scales", ss, false));
        NM_TRY(check_apart("workspace", sw, "bias", sb, false));
        NM_TRY(check_apart("workspace", sw, "residual", sr, false));
        NM_TRY(check_apart("workspace", sw, "y", sy, false));
    }
    return run_q8_linear(p, plan, workspace, (hipStream_t)stream);
}

// The integers of a block are 64 bits wide; one that does not fit an int is out of range for every argument that is one.
static inline int narrow(int64_t v) { return v < -1 || v > 0x7fffffff ? -1 : (int)v; }

int nm_rows_q8_args(const nm_rows_q8_args_t* a)
{
    if (!a) {
        set_error("null pointer argument");
        return NM_ERR_ARG;
    }
    if (a->norm)
        return nm_rmsnorm_q8(a->x_dev, narrow(a->dtype), a->rows, narrow(a->width), a->ldx, a->residual_dev, a->ldr, a->gamma_dev, (float)a->eps,
                             a->residual_out_dev, a->ldo, a->q_dev, a->ldq, a->scales_dev, a->hip_stream);
    return nm_quantize_q8(a->x_dev, narrow(a->dtype), a->rows, narrow(a->width), a->ldx, a->q_dev, a->ldq, a->scales_dev, a->hip_stream);
}

int nm_dequantize_q8_args(const nm_dequantize_q8_args_t* a)
{
    if (!a) {
        set_error("null pointer argument");
        return NM_ERR_ARG;
    }
    return nm_dequantize_q8(a->q_dev, a->ldq, a->scales_dev, a->rows, narrow(a->width), a->y_dev, narrow(a->dtype), a->ldy, a->hip_stream);
}

int nm_linear_q8_args(const nm_linear_q8_args_t* a)
{
    if (!a) {
        set_error("null pointer argument");
        return NM_ERR_ARG;
    }
    return nm_linear_q8(a->q_dev, a->rows, narrow(a->width), a->ldq, a->scales_dev, a->w, a->bias_dev, a->residual_dev, a->ldr, a->y_dev,
                        narrow(a->dtype), a->ldy, a->workspace_dev, a->workspace_bytes < 0 ? 0 : (size_t)a->workspace_bytes, a->hip_stream);
}

}  // extern "C"
