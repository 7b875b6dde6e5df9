// Address- and undefined-behaviour-sanitizer run of the host layer of the 8-bit operators (csrc/nm_q8_api.hip: argument
// checks, overlap of tensors, the weights' handle) with no GPU.  Built by tests/test_q8_host.py from nm_q8_api.hip compiled
// host-only and this file, which stands in for the HIP runtime ("device" memory is host memory) and for the launchers; those
// record what they are handed.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <map>
#include <random>
#include <set>
#include <string>
#include <vector>

#include "nm_q8_internal.h"

#define CHECK(c)                                                            \
    do {                                                                    \
        if (!(c)) {                                                         \
            fprintf(stderr, "check failed at line %d: %s (last error: %s)\n", __LINE__, #c, g_error.c_str()); \
            exit(1);                                                        \
        }                                                                   \
    } while (0)

static std::string g_error;
static std::map<void*, size_t> g_allocs;
static int g_fail_at = -1, g_mallocs = 0, g_launches = 0, g_device = 0;
static bool g_no_device = false, g_capturing = false, g_fail_pack = false, g_bad_scale = false;
static size_t g_workspace = 0;
static nm::Q8Linear g_linear;
static float g_eps = -1;
static void* g_given_workspace = nullptr;

extern "C" {
hipError_t hipGetDevice(int* d) { *d = g_device; return g_no_device ? hipErrorNoDevice : hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "fake HIP error"; }
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipMalloc(void** p, size_t n)
{
    if (g_mallocs++ == g_fail_at) { *p = nullptr; return hipErrorOutOfMemory; }
    *p = malloc(n ? n : 1);
    g_allocs[*p] = n;
    return hipSuccess;
}
hipError_t hipFree(void* p)
{
    if (!p) return hipSuccess;
    CHECK(g_allocs.erase(p) == 1);
    free(p);
    return hipSuccess;
}
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { memcpy(d, s, n); return hipSuccess; }
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind, hipStream_t) { memcpy(d, s, n); return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s)
{
    *s = g_capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return g_no_device ? hipErrorNoDevice : hipSuccess;
}
}

namespace nm {
void set_error(const char* fmt, ...)
{
    char b[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(b, sizeof(b), fmt, ap);
    va_end(ap);
    g_error = b;
}
int run_q8_rows(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, const void*, int64_t, const float*, float eps, bool, void*,
                int64_t, int8_t* q, int64_t ldq, float* scales, hipStream_t)
{
    ++g_launches;
    g_eps = eps;
    if (g_allocs.count(q)) {   // (the rounded weights of nm_q8_pack: written as the kernel does)
        CHECK(g_allocs[q] >= (size_t)rows * width && g_allocs[scales] >= (size_t)rows * 4);
        for (int64_t r = 0; r < rows; ++r) {
            for (int c = 0; c < width; ++c) q[r * ldq + c] = (int8_t)(dt == NM_F32 ? ((const float*)x)[r * ldx + c] : 1);
            scales[r] = g_bad_scale ? NAN : 1.0f;
        }
    }
    return NM_OK;
}
int run_q8_dequantize(const int8_t*, int64_t, const float*, int64_t, int, void*, nm_dtype_t, int64_t, hipStream_t) { ++g_launches; return NM_OK; }
int run_q8_pack(const int8_t* w, int64_t ldw, const float* scales, const nm_q8* h, int* d_bad, hipStream_t)
{
    ++g_launches;
    if (g_fail_pack) { set_error("fake launch failure"); return NM_ERR_HIP; }
    CHECK(g_allocs[h->d_w] == (size_t)h->groups * h->kblocks * 4096 && g_allocs[h->d_scales] == (size_t)h->groups * 64 * 4);
    CHECK(h->groups * 64 >= h->channels && h->kblocks * 64 >= h->width && h->kblocks % 2 == 0);
    *d_bad = 0;
    // the whole packed array, through the map of rows: every channel exactly once
    std::vector<int> seen(h->channels, 0);
    for (int p = 0; p < h->groups * 64; ++p) {
        const int c = q8_row_of(p, h->channels, h->gated);
        if (c >= 0) {
            CHECK(c < h->channels);
            ++seen[c];
            if (!(fabsf(scales[c]) < INFINITY)) *d_bad = 1;
        }
        for (int k = 0; k < h->kblocks * 64; ++k)
            h->d_w[((size_t)(p >> 6) * h->kblocks + k / 64) * 4096 + ((p >> 4) & 3) * 1024 + ((p & 15) + 16 * ((k % 64) / 16)) * 16 + k % 16] =
                c >= 0 && k < h->width ? w[c * ldw + k] : 0;
        h->d_scales[p] = c >= 0 ? scales[c] : 0.0f;
    }
    for (int s : seen) CHECK(s == 1);
    return NM_OK;
}
int run_q8_unpack(const nm_q8* h, int8_t* w, float* scales, hipStream_t)
{
    for (int p = 0; p < h->groups * 64; ++p) {
        const int c = q8_row_of(p, h->channels, h->gated);
        if (c < 0) continue;
        for (int k = 0; k < h->width; ++k)
            w[(size_t)c * h->width + k] = h->d_w[((size_t)(p >> 6) * h->kblocks + k / 64) * 4096 + ((p >> 4) & 3) * 1024 + ((p & 15) + 16 * ((k % 64) / 16)) * 16 + k % 16];
        scales[c] = h->d_scales[p];
    }
    return NM_OK;
}
Q8Plan q8_plan(const Q8Linear&)
{
    Q8Plan p;
    p.rows_bytes = g_workspace / 2;
    p.part_bytes = g_workspace - p.rows_bytes;
    return p;
}
int run_q8_linear(const Q8Linear& p, const Q8Plan&, void* ws, hipStream_t)
{
    ++g_launches;
    g_linear = p;
    g_given_workspace = ws;
    return NM_OK;
}
}  // namespace nm

struct S {
    uintptr_t at;
    int elem, rows, width, ld;
    std::set<uintptr_t> bytes() const
    {
        std::set<uintptr_t> b;
        for (int r = 0; r < rows; ++r)
            for (int i = 0; i < width * elem; ++i) b.insert(at + (uintptr_t)r * ld * elem + i);
        return b;
    }
};
static bool meet(const S& a, const S& b)
{
    const auto x = a.bytes(), y = b.bytes();
    for (uintptr_t v : x)
        if (y.count(v)) return true;
    return false;
}

// Random pairs of tensors: whatever shares a byte is refused; columns of one wide tensor that share none are taken.
static void overlaps()
{
    std::mt19937 g(7);
    auto in = [&](int lo, int hi) { return lo + (int)(g() % (unsigned)(hi - lo + 1)); };
    const uintptr_t far = 0x40000000;
    int shared = 0, apart = 0, columns = 0;
    for (int t = 0; t < 40000; ++t) {
        const int rows = in(1, 4), width = in(1, 12), es = g() % 2 ? 4 : 2;
        const S q{far + (uintptr_t)in(0, 200), 1, rows, width, in(0, 40)};
        const int ldy = g() % 2 && (q.ld % es) == 0 ? q.ld / es : in(width, width + 8);
        const S y{far + (uintptr_t)in(0, 60) * es, es, rows, width, ldy};
        const int rc = nm_dequantize_q8((const int8_t*)q.at, q.ld, (const float*)0x1000, rows, width, (void*)y.at, es == 4 ? NM_F32 : NM_BF16, ldy, nullptr);
        const bool m = meet(q, y);
        if (ldy < width && rows > 1) { CHECK(rc == NM_ERR_ARG); continue; }
        if (m) { CHECK(rc == NM_ERR_ARG); ++shared; }
        else if (rc == NM_OK) ++apart;
        // the stream as columns of the tensor that x is columns of
        const S x{far + (uintptr_t)in(0, 40) * es, es, rows, width, in(width, 40)};
        const S o{far + (uintptr_t)in(0, 40) * es, es, rows, width, x.ld};
        const int rc2 = nm_rmsnorm_q8((const void*)x.at, es == 4 ? NM_F32 : NM_BF16, rows, width, x.ld, nullptr, 0, nullptr, 0.0f, (void*)o.at, o.ld,
                                      (int8_t*)0x2000, width, (float*)0x1000, nullptr);
        if (x.at == o.at) CHECK(rc2 == NM_OK);
        else if (meet(x, o)) CHECK(rc2 == NM_ERR_ARG);
        else {
            const uintptr_t lo = x.at < o.at ? x.at : o.at, hi = x.at < o.at ? o.at : x.at;
            if ((hi - lo) % ((uintptr_t)x.ld * es) + (uintptr_t)width * es <= (uintptr_t)x.ld * es) { CHECK(rc2 == NM_OK); ++columns; }
        }
    }
    CHECK(shared > 1000 && apart > 1000 && columns > 1000);
}

static void refusals()
{
    float x[64] = {}, s[8] = {}, y[64] = {};
    int8_t q[64] = {};
    const int64_t big = ((int64_t)1 << 24) + 1;
    CHECK(nm_quantize_q8(x, NM_F32, 4, 16, 16, q, 16, s, nullptr) == NM_OK);
    CHECK(nm_quantize_q8(x, NM_I8, 4, 16, 16, q, 16, s, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_q8(x, 77, 4, 16, 16, q, 16, s, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_q8(nullptr, NM_F32, 4, 16, 16, q, 16, s, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_q8(x, NM_F32, 4, 16, 16, nullptr, 16, s, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_q8(x, NM_F32, 4, 16, 16, q, 16, nullptr, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_q8(x, NM_F32, -1, 16, 16, q, 16, s, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_q8(x, NM_F32, ((int64_t)1 << 30) + 1, 16, 16, q, 16, s, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_q8(x, NM_F32, 4, 0, 16, q, 16, s, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_q8(x, NM_F32, 1, NM_Q8_MAX_WIDTH + 1, 16, q, 16, s, nullptr) == NM_ERR_SHAPE);
    CHECK(nm_quantize_q8(x, NM_F32, 4, 16, -1, q, 16, s, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_q8(x, NM_F32, 4, 16, big, q, 16, s, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_q8(x, NM_F32, 4, 16, 16, q, 15, s, nullptr) == NM_ERR_ARG);       // rows of an output on one another
    CHECK(nm_quantize_q8((char*)x + 2, NM_F32, 1, 8, 8, q, 16, s, nullptr) == NM_ERR_ARG);   // not aligned to an element
    CHECK(nm_quantize_q8((char*)x + 2, NM_BF16, 1, 8, 8, q, 16, s, nullptr) == NM_OK);
    CHECK(nm_quantize_q8(nullptr, NM_F32, 0, 16, 16, nullptr, 16, nullptr, nullptr) == NM_OK);   // no rows
    for (float eps : {-1.0f, NAN, INFINITY})
        CHECK(nm_rmsnorm_q8(x, NM_F32, 4, 16, 16, nullptr, 0, nullptr, eps, nullptr, 0, q, 16, s, nullptr) == NM_ERR_ARG);
    CHECK(nm_rmsnorm_q8(x, NM_F32, 4, 16, 16, x, 16, nullptr, 0.5f, x, 16, q, 16, s, nullptr) == NM_OK && g_eps == 0.5f);
    CHECK(nm_rmsnorm_q8(x, NM_F32, 4, 16, 16, y, 16, s, 0.5f, nullptr, 0, q, 16, s, nullptr) == NM_ERR_ARG);   // the gains are written over
    CHECK(nm_dequantize_q8(q, 16, s, 4, 16, y, NM_I8, 16, nullptr) == NM_ERR_ARG);
    CHECK(nm_dequantize_q8(q, 16, s, 4, 16, y, NM_BF16, 16, nullptr) == NM_OK);
    CHECK(nm_dequantize_q8(q, 16, y, 4, 16, y, NM_BF16, 16, nullptr) == NM_ERR_ARG);

    const nm_rows_q8_args_t ra{x, nullptr, nullptr, nullptr, q, s, nullptr, NM_F32, 4, 16, 16, 0, 16, 16, 1, 0.25};
    CHECK(nm_rows_q8_args(&ra) == NM_OK && g_eps == 0.25f);
    nm_rows_q8_args_t rb = ra;
    rb.width = ((int64_t)1 << 32) + 16;   // not 16
    CHECK(nm_rows_q8_args(&rb) == NM_ERR_ARG);
    rb = ra;
    rb.dtype = ((int64_t)1 << 32);        // not NM_F32
    CHECK(nm_rows_q8_args(&rb) == NM_ERR_ARG);
    rb = ra;
    rb.norm = 0;
    rb.eps = -1;
    CHECK(nm_rows_q8_args(&rb) == NM_OK && g_eps == 0.0f);
    CHECK(nm_rows_q8_args(nullptr) == NM_ERR_ARG && nm_dequantize_q8_args(nullptr) == NM_ERR_ARG && nm_linear_q8_args(nullptr) == NM_ERR_ARG);
    const nm_dequantize_q8_args_t da{q, s, y, nullptr, NM_F32, 4, 16, 16, 16};
    CHECK(nm_dequantize_q8_args(&da) == NM_OK);
}

static nm_q8_t* pack(int channels, int width, int gated, int8_t seed)
{
    std::vector<int8_t> w((size_t)channels * (width + 3));
    std::vector<float> s(channels);
    for (size_t i = 0; i < w.size(); ++i) w[i] = (int8_t)(i * 31 + seed);
    for (int c = 0; c < channels; ++c) s[c] = c + 0.5f;
    nm_q8_t* h = nullptr;
    CHECK(nm_q8_pack(w.data(), NM_I8, s.data(), channels, width, width + 3, gated, nullptr, &h) == NM_OK && h);
    std::vector<int8_t> e((size_t)channels * width);
    std::vector<float> t(channels);
    CHECK(nm_q8_export(h, e.data(), t.data()) == NM_OK && t == s);
    for (int c = 0; c < channels; ++c) CHECK(!memcmp(&e[(size_t)c * width], &w[(size_t)c * (width + 3)], width));
    CHECK(nm_q8_export(h, nullptr, nullptr) == NM_OK);
    int a, b, d;
    CHECK(nm_q8_dims(h, &a, &b, &d) == NM_OK && a == channels && b == width && d == gated && nm_q8_dims(h, nullptr, nullptr, nullptr) == NM_OK);
    return h;
}

static void weights()
{
    for (int channels : {2, 4, 62, 64, 66, 128, 130})
        for (int width : {1, 15, 64, 65, 128, 129, 300})
            for (int gated : {0, 1}) CHECK(nm_q8_free(pack(channels, width, gated, 3)) == NM_OK);
    CHECK(nm_q8_free(nullptr) == NM_OK && nm_q8_dims(nullptr, nullptr, nullptr, nullptr) == NM_ERR_ARG && nm_q8_export(nullptr, nullptr, nullptr) == NM_ERR_ARG);
    CHECK(g_allocs.empty());
    float w[40] = {1, 2, 3}, s[8] = {1, 1, 1, 1, 1, 1, 1, 1};
    int8_t w8[40] = {};
    nm_q8_t* h = nullptr;
    CHECK(nm_q8_pack(w, NM_F32, nullptr, 4, 10, 10, 0, nullptr, nullptr) == NM_ERR_ARG);
    CHECK(nm_q8_pack(nullptr, NM_F32, nullptr, 4, 10, 10, 0, nullptr, &h) == NM_ERR_ARG);
    CHECK(nm_q8_pack(w, NM_F32, s, 4, 10, 10, 0, nullptr, &h) == NM_ERR_ARG);
    CHECK(nm_q8_pack(w8, NM_I8, nullptr, 4, 10, 10, 0, nullptr, &h) == NM_ERR_ARG);
    CHECK(nm_q8_pack(w, NM_F8E4M3, nullptr, 4, 10, 10, 0, nullptr, &h) == NM_ERR_ARG);
    CHECK(nm_q8_pack(w, NM_F32, nullptr, 3, 10, 10, 1, nullptr, &h) == NM_ERR_ARG);
    CHECK(nm_q8_pack(w, NM_F32, nullptr, 4, 10, 10, 2, nullptr, &h) == NM_ERR_ARG);
    CHECK(nm_q8_pack(w, NM_F32, nullptr, 0, 10, 10, 0, nullptr, &h) == NM_ERR_ARG);
    CHECK(nm_q8_pack(w, NM_F32, nullptr, (1 << 24) + 1, 10, 10, 0, nullptr, &h) == NM_ERR_SHAPE);
    CHECK(nm_q8_pack(w, NM_F32, nullptr, 4, NM_Q8_MAX_WIDTH + 1, 10, 0, nullptr, &h) == NM_ERR_SHAPE);
    g_capturing = true;
    CHECK(nm_q8_pack(w, NM_F32, nullptr, 4, 10, 10, 0, nullptr, &h) == NM_ERR_HIP && g_error.find("capture") != std::string::npos);
    g_capturing = false;
    g_no_device = true;
    CHECK(nm_q8_pack(w, NM_F32, nullptr, 4, 10, 10, 0, nullptr, &h) == NM_ERR_HIP);
    g_no_device = false;
    g_fail_pack = true;
    CHECK(nm_q8_pack(w, NM_F32, nullptr, 4, 10, 10, 0, nullptr, &h) == NM_ERR_HIP && !h);
    g_fail_pack = false;
    g_bad_scale = true;
    CHECK(nm_q8_pack(w, NM_F32, nullptr, 4, 10, 10, 0, nullptr, &h) == NM_ERR_ARG && g_error.find("finite") != std::string::npos);
    g_bad_scale = false;
    s[2] = INFINITY;
    CHECK(nm_q8_pack(w8, NM_I8, s, 4, 10, 10, 0, nullptr, &h) == NM_ERR_ARG && g_error.find("scale") != std::string::npos);
    CHECK(g_allocs.empty());
    // every allocation failing once, in the order they are made: an error, and nothing kept
    for (int dt : {(int)NM_F32, (int)NM_I8}) {
        s[2] = 1;
        int failed = 0;
        for (int at = 0; at < 8; ++at) {
            g_mallocs = 0;
            g_fail_at = at;
            const int rc = nm_q8_pack(dt == NM_F32 ? (void*)w : (void*)w8, dt, dt == NM_F32 ? nullptr : s, 4, 10, 10, 0, nullptr, &h);
            g_fail_at = -1;
            if (rc == NM_OK) { nm_q8_free(h); break; }
            CHECK(rc == NM_ERR_ALLOC && !h && g_allocs.empty());
            ++failed;
        }
        CHECK(failed == (dt == NM_F32 ? 5 : 3));
        CHECK(g_allocs.empty());
    }
    h = pack(4, 10, 0, 1);
    for (int at = 0; at < 2; ++at) {
        g_mallocs = 0;
        g_fail_at = at;
        int8_t e[40];
        CHECK(nm_q8_export(h, e, nullptr) == NM_ERR_ALLOC);
        g_fail_at = -1;
    }
    nm_q8_free(h);
}

static void products()
{
    nm_q8_t *h = pack(8, 16, 0, 1), *hg = pack(8, 16, 1, 1);
    int8_t q[64] = {};
    float s[4] = {}, b[8] = {}, y[32] = {}, r[32] = {};
    char ws[64];
    auto call = [&](const nm_q8_t* w, int width, const float* bias, const void* res, int64_t ldr, void* out, int dt, int64_t ldy, void* p, size_t n) {
        return nm_linear_q8(q, 4, width, 16, s, w, bias, res, ldr, out, dt, ldy, p, n, nullptr);
    };
    CHECK(call(h, 16, b, r, 8, y, NM_F32, 8, nullptr, 0) == NM_OK && g_linear.outs == 8 && g_linear.rows == 4 && !g_linear.gated && !g_linear.y_bf16);
    CHECK(call(hg, 16, b, nullptr, 0, y, NM_BF16, 4, nullptr, 0) == NM_OK && g_linear.outs == 4 && g_linear.gated && g_linear.y_bf16);
    CHECK(call(h, 16, b, y, 8, y, NM_F32, 8, nullptr, 0) == NM_OK);                  // the stream in place
    CHECK(call(h, 16, b, y + 1, 7, y, NM_F32, 8, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(nullptr, 16, b, nullptr, 0, y, NM_F32, 8, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(h, 15, b, nullptr, 0, y, NM_F32, 8, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(h, 16, b, nullptr, 0, y, NM_I8, 8, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(h, 16, b, nullptr, 0, y, NM_F32, 7, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(h, 16, b, nullptr, 0, nullptr, NM_F32, 8, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(h, 16, y, nullptr, 0, y, NM_F32, 8, nullptr, 0) == NM_ERR_ARG);       // the bias is written over
    CHECK(call(hg, 16, b, r, 4, y, NM_F32, 4, nullptr, 0) == NM_ERR_UNSUPPORTED);
    CHECK(nm_linear_q8(nullptr, 0, 16, 16, nullptr, h, nullptr, nullptr, 0, nullptr, NM_F32, 8, nullptr, 0, nullptr) == NM_OK);   // no rows
    g_device = 1;
    CHECK(call(h, 16, b, nullptr, 0, y, NM_F32, 8, nullptr, 0) == NM_ERR_ARG && nm_q8_export(h, q, nullptr) == NM_ERR_ARG);
    g_device = 0;
    g_workspace = 32;
    size_t n = 1;
    CHECK(nm_linear_q8_workspace(q, 4, 16, h, &n) == NM_OK && n == 32);
    CHECK(nm_linear_q8_workspace(q, 0, 16, h, &n) == NM_OK && n == 0);
    CHECK(nm_linear_q8_workspace(q, 4, 16, nullptr, &n) == NM_ERR_ARG && nm_linear_q8_workspace(q, 4, 16, h, nullptr) == NM_ERR_ARG);
    char* aligned = ws + (16 - (uintptr_t)ws % 16) % 16;
    CHECK(call(h, 16, b, nullptr, 0, y, NM_F32, 8, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(h, 16, b, nullptr, 0, y, NM_F32, 8, aligned, 31) == NM_ERR_ARG);
    CHECK(call(h, 16, b, nullptr, 0, y, NM_F32, 8, aligned + 1, 40) == NM_ERR_ARG);
    CHECK(call(h, 16, b, nullptr, 0, y, NM_F32, 8, aligned, 32) == NM_OK && g_given_workspace == aligned);
    char* inside = (char*)y + (16 - (uintptr_t)y % 16) % 16;
    CHECK(call(h, 16, b, nullptr, 0, y, NM_F32, 8, inside, 64) == NM_ERR_ARG);       // the workspace in the output
    g_workspace = 0;
    const nm_linear_q8_args_t la{q, s, h, b, r, y, nullptr, nullptr, NM_F32, 4, 16, 16, 8, 8, 0};
    CHECK(nm_linear_q8_args(&la) == NM_OK && g_linear.res == r && g_linear.bias == b && g_linear.ldr == 8);
    nm_linear_q8_args_t lb = la;
    lb.width = -5;
    CHECK(nm_linear_q8_args(&lb) == NM_ERR_ARG);
    nm_q8_free(h);
    nm_q8_free(hg);
    CHECK(g_allocs.empty());
}

int main()
{
    static_assert(sizeof(nm_rows_q8_args_t) == 128 && sizeof(nm_dequantize_q8_args_t) == 72 && sizeof(nm_linear_q8_args_t) == 120,
                  "the binding packs these blocks itself");
    refusals();
    weights();
    products();
    overlaps();
    printf("8-bit host-layer sanitizer run: ok (%d launches)\n", g_launches);
    return 0;
}
