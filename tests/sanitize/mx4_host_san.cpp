// Address- and undefined-behaviour-sanitizer run of the host layer of the operators in MX4 and of those for experts
// (csrc/nm_mx4_api.hip: argument checks, overlap of tensors, the weights' handle) with no GPU.  Built by tests/test_mx4_host.py from
// nm_mx4_api.hip compiled host-only and this file, which stands in for the HIP runtime ("device" memory is host memory) and for the
// launchers; those record what they are handed.
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

#include "nm_mx4_internal.h"

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
static bool g_no_device = false, g_capturing = false, g_fail_pack = false, g_bad = false;
static hipStreamCaptureMode g_mode = hipStreamCaptureModeGlobal;
static nm::Mx4Product g_product;
static nm::Route g_route;
static nm::Combine g_combine;
static double g_eps = -1;

extern "C" {
hipError_t hipGetDevice(int* d) { *d = g_device; return g_no_device ? hipErrorNoDevice : hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "fake HIP error"; }
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipThreadExchangeStreamCaptureMode(hipStreamCaptureMode* m) { std::swap(*m, g_mode); return hipSuccess; }
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
int run_mx4_rows(const void*, nm_dtype_t, int64_t rows, int width, int64_t, const void*, int64_t, const float*, double eps, bool, void*, int64_t,
                 uint8_t* q, int64_t ldq, uint8_t* scales, int64_t lds, hipStream_t)
{
    ++g_launches;
    g_eps = eps;
    const int nb = (width + 31) / 32;
    if (g_allocs.count(q)) {   // (the rounded weights of nm_mx4_pack)
        CHECK(g_allocs[q] >= (size_t)rows * nb * 16 && g_allocs[scales] >= (size_t)rows * nb);
        for (int64_t r = 0; r < rows; ++r) {
            memset(q + r * ldq, 0x21, nb * 16);
            memset(scales + r * lds, 127, nb);
        }
    }
    return NM_OK;
}
int run_mx4_dequantize(const uint8_t*, int64_t, const uint8_t*, int64_t, int64_t, int, void*, nm_dtype_t, int64_t, hipStream_t) { ++g_launches; return NM_OK; }
// The packed array of a handle, as its description in nm_mx4_internal.h has it.
static uint8_t* unit(const nm_mx4* h, int e, int packed, int kb)
{
    const size_t step = ((size_t)e * h->groups + packed / 64) * h->steps + kb / 8;
    return h->d_w + ((step * 2 + kb / 4 % 2) * 4 + packed / 16 % 4) * 1024 + (packed % 16 + 16 * (kb % 4)) * 16;
}
static uint8_t* scale(const nm_mx4* h, int e, int packed, int kb)
{
    const size_t step = ((size_t)e * h->groups + packed / 64) * h->steps + kb / 8;
    return (uint8_t*)(h->d_s + (step * 2 + kb / 4 % 2) * 64 + packed % 16 + 16 * (kb % 4)) + packed / 16 % 4;
}
int run_mx4_pack(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, const nm_mx4* h, int* d_bad, hipStream_t)
{
    ++g_launches;
    if (g_fail_pack) { set_error("fake launch failure"); return NM_ERR_HIP; }
    CHECK(g_allocs[h->d_w] == h->w_bytes() && g_allocs[h->d_s] == h->s_bytes());
    CHECK(h->groups * 64 >= h->channels && h->steps * 8 >= h->blocks && h->blocks * 32 >= h->width);
    *d_bad = g_bad;
    for (int e = 0; e < h->experts; ++e)
        for (int p = 0; p < h->groups * 64; ++p) {
            const int c = q8_row_of(p, h->channels, h->gated);
            for (int kb = 0; kb < h->steps * 8; ++kb) {
                const bool in = c >= 0 && kb < h->blocks;
                const int64_t row = (int64_t)e * h->channels + c;
                if (in) memcpy(unit(h, e, p, kb), q + row * ldq + kb * 16, 16);
                else memset(unit(h, e, p, kb), 0, 16);
                *scale(h, e, p, kb) = in ? scales[row * lds + kb] : 127;
            }
        }
    return NM_OK;
}
int run_mx4_unpack(const nm_mx4* h, uint8_t* q, uint8_t* scales, hipStream_t)
{
    for (int e = 0; e < h->experts; ++e)
        for (int p = 0; p < h->groups * 64; ++p) {
            const int c = q8_row_of(p, h->channels, h->gated);
            if (c < 0) continue;
            for (int kb = 0; kb < h->blocks; ++kb) {
                const size_t at = ((size_t)e * h->channels + c) * h->blocks + kb;
                memcpy(q + at * 16, unit(h, e, p, kb), 16);
                scales[at] = *scale(h, e, p, kb);
            }
        }
    return NM_OK;
}
int run_mx4_product(const Mx4Product& p, hipStream_t) { ++g_launches; g_product = p; return NM_OK; }
size_t route_workspace(int64_t tokens, int experts) { return tokens <= 64 ? 0 : (size_t)experts * 4; }
int run_route(const Route& r, void*, hipStream_t) { ++g_launches; g_route = r; return NM_OK; }
int run_combine(const Combine& c, hipStream_t) { ++g_launches; g_combine = c; return NM_OK; }
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

// Random places of the outputs: whatever shares a byte with another tensor is refused.
static void overlaps()
{
    std::mt19937 g(7);
    auto in = [&](int lo, int hi) { return lo + (int)(g() % (unsigned)(hi - lo + 1)); };
    const uintptr_t far = 0x40000000;
    int shared = 0, apart = 0;
    for (int t = 0; t < 20000; ++t) {
        const int rows = in(1, 3), width = in(1, 40), nb = (width + 31) / 32, es = g() % 2 ? 4 : 2;
        const nm_dtype_t dt = es == 4 ? NM_F32 : NM_BF16;
        const S x{far + (uintptr_t)in(0, 60) * es, es, rows, width, in(width, width + 4)};
        const S q{far + (uintptr_t)in(0, 40) * 16, 1, rows, nb * 16, in(nb, nb + 1) * 16}, s{far + (uintptr_t)in(0, 600), 1, rows, nb, in(nb, nb + 3)};
        const int rc = nm_quantize_mx4((void*)x.at, dt, rows, width, x.ld, (uint8_t*)q.at, q.ld, (uint8_t*)s.at, s.ld, nullptr);
        const bool m = meet(x, q) || meet(x, s) || meet(q, s);
        if (m) { CHECK(rc == NM_ERR_ARG); ++shared; }
        else if (rc == NM_OK) ++apart;
        const int rc2 = nm_dequantize_mx4((uint8_t*)q.at, q.ld, (uint8_t*)s.at, s.ld, rows, width, (void*)x.at, dt, x.ld, nullptr);
        if (meet(x, q) || meet(x, s)) CHECK(rc2 == NM_ERR_ARG);
        // the answer of a combination and its inputs
        const int entries = in(1, 4), choices = in(1, 3);
        const S y{far + (uintptr_t)in(0, 60) * 2, 2, entries, width, in(width, width + 4)}, o{far + (uintptr_t)in(0, 60) * es, es, rows, width, in(width, width + 4)};
        const S sl{far + (uintptr_t)in(0, 100) * 4, 4, rows, choices, choices}, w{far + (uintptr_t)in(0, 100) * 4, 4, rows, choices, choices};
        const int rc3 = nm_combine((void*)y.at, NM_BF16, entries, y.ld, (int*)sl.at, (float*)w.at, rows, choices, width, nullptr, 0, (void*)o.at, dt, o.ld, nullptr);
        if (meet(o, y) || meet(o, sl) || meet(o, w)) CHECK(rc3 == NM_ERR_ARG);
        CHECK(nm_combine((void*)0x1000, NM_BF16, entries, y.ld, (int*)0x8000, (float*)0x9000, rows, choices, width, (void*)o.at, o.ld, (void*)o.at, dt, o.ld, nullptr) == NM_OK);
    }
    CHECK(shared > 1000 && apart > 1000);
}

static void rows()
{
    float x[128] = {}, y[128] = {};
    alignas(16) uint8_t q[256] = {}, s[16] = {};
    const int64_t big = ((int64_t)1 << 24) + 16;
    CHECK(nm_quantize_mx4(x, NM_F32, 2, 40, 40, q, 32, s, 2, nullptr) == NM_OK);
    CHECK(nm_quantize_mx4(x, NM_MX4, 2, 40, 40, q, 32, s, 2, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_mx4(x, NM_F32, 2, 40, 40, q, 31, s, 2, nullptr) == NM_ERR_ARG);   // rows on one another
    CHECK(nm_quantize_mx4(x, NM_F32, 2, 40, 40, q, 40, s, 2, nullptr) == NM_ERR_ARG);   // not at multiples of 16 bytes
    CHECK(nm_quantize_mx4(x, NM_F32, 2, 40, 40, q + 8, 32, s, 2, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_mx4(x, NM_F32, 1, 40, 40, q, 40, s, 2, nullptr) == NM_OK);        // (one row has no stride)
    CHECK(nm_quantize_mx4(x, NM_F32, 2, 40, 40, q, 32, s, 1, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_mx4(x, NM_F32, 2, 40, big, q, 32, s, 2, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_mx4(x, NM_F32, -1, 40, 40, q, 32, s, 2, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_mx4(x, NM_F32, 2, 0, 40, q, 32, s, 2, nullptr) == NM_ERR_ARG);
    CHECK(nm_quantize_mx4(x, NM_F32, 1, NM_MX4_MAX_WIDTH + 1, 40, q, 32, s, 2, nullptr) == NM_ERR_SHAPE);
    CHECK(nm_quantize_mx4(nullptr, NM_F32, 0, 40, 40, nullptr, 32, nullptr, 2, nullptr) == NM_OK);
    for (double eps : {-1.0, (double)NAN, (double)INFINITY})
        CHECK(nm_rmsnorm_mx4(x, NM_F32, 2, 40, 40, nullptr, 0, nullptr, eps, nullptr, 0, q, 32, s, 2, nullptr) == NM_ERR_ARG);
    CHECK(nm_rmsnorm_mx4(x, NM_F32, 2, 40, 40, x, 40, nullptr, 0.5, x, 40, q, 32, s, 2, nullptr) == NM_OK && g_eps == 0.5);
    CHECK(nm_rmsnorm_mx4(x, NM_F32, 2, 40, 40, y, 40, y, 0.5, y, 40, q, 32, s, 2, nullptr) == NM_ERR_ARG);   // the gains are written over
    CHECK(nm_rmsnorm_mx4(x, NM_F32, 2, 40, 40, y + 1, 40, nullptr, 0.5, y, 40, q, 32, s, 2, nullptr) == NM_ERR_ARG);
    CHECK(nm_dequantize_mx4(q, 32, s, 2, 2, 40, y, NM_MX4, 40, nullptr) == NM_ERR_ARG);
    CHECK(nm_dequantize_mx4(q, 32, s, 2, 2, 40, y, NM_BF16, 40, nullptr) == NM_OK);
    CHECK(nm_dequantize_mx4(q, 0, s, 0, 2, 40, y, NM_F32, 40, nullptr) == NM_OK);       // an input's rows may be one
    CHECK(nm_dequantize_mx4(q, 32, s, 2, 2, 40, y, NM_F32, 39, nullptr) == NM_ERR_ARG);

    const nm_rows_mx4_args_t ra{x, nullptr, nullptr, nullptr, q, s, nullptr, NM_F32, 2, 40, 40, 0, 40, 32, 2, 1, 0.25};
    CHECK(nm_rows_mx4_args(&ra) == NM_OK && g_eps == 0.25);
    nm_rows_mx4_args_t rb = ra;
    rb.width = ((int64_t)1 << 32) + 40;   // not 40
    CHECK(nm_rows_mx4_args(&rb) == NM_ERR_ARG);
    rb = ra;
    rb.norm = 0;
    rb.eps = -1;
    CHECK(nm_rows_mx4_args(&rb) == NM_OK && g_eps == 0.0);
    const nm_dequantize_mx4_args_t da{q, s, y, nullptr, NM_F32, 2, 40, 32, 2, 40};
    CHECK(nm_dequantize_mx4_args(&da) == NM_OK);
    CHECK(nm_rows_mx4_args(nullptr) == NM_ERR_ARG && nm_dequantize_mx4_args(nullptr) == NM_ERR_ARG && nm_product_mx4_args(nullptr) == NM_ERR_ARG);
    CHECK(nm_route_args(nullptr) == NM_ERR_ARG && nm_combine_args(nullptr) == NM_ERR_ARG);
}

static nm_mx4_t* pack(int experts, int channels, int width, int gated)
{
    const int nb = (width + 31) / 32, rows = experts * channels, ldq = nb * 16 + 16, lds = nb + 3;
    uint8_t* w = (uint8_t*)aligned_alloc(16, (size_t)rows * ldq);
    std::vector<uint8_t> s((size_t)rows * lds);
    for (int i = 0; i < rows * ldq; ++i) w[i] = (uint8_t)(i * 37 + i / 251);
    for (size_t i = 0; i < s.size(); ++i) s[i] = (uint8_t)(i % 255);
    nm_mx4_t* h = nullptr;
    CHECK(nm_mx4_pack(w, NM_MX4, s.data(), lds, experts, channels, width, ldq, gated, nullptr, &h) == NM_OK && h);
    std::vector<uint8_t> e((size_t)rows * nb * 16), t((size_t)rows * nb);
    CHECK(nm_mx4_export(h, e.data(), t.data()) == NM_OK);
    for (int r = 0; r < rows; ++r) CHECK(!memcmp(&e[(size_t)r * nb * 16], w + (size_t)r * ldq, nb * 16) && !memcmp(&t[(size_t)r * nb], &s[(size_t)r * lds], nb));
    CHECK(nm_mx4_export(h, nullptr, nullptr) == NM_OK);
    int a, b, c, d;
    CHECK(nm_mx4_dims(h, &a, &b, &c, &d) == NM_OK && a == experts && b == channels && c == width && d == gated);
    CHECK(nm_mx4_dims(h, nullptr, nullptr, nullptr, nullptr) == NM_OK);
    free(w);
    return h;
}

static void weights()
{
    for (int experts : {1, 3})
        for (int channels : {2, 62, 64, 66, 130})
            for (int width : {1, 32, 33, 255, 256, 300})
                for (int gated : {0, 1}) CHECK(nm_mx4_free(pack(experts, channels, width, gated)) == NM_OK);
    CHECK(nm_mx4_free(nullptr) == NM_OK && nm_mx4_dims(nullptr, nullptr, nullptr, nullptr, nullptr) == NM_ERR_ARG);
    CHECK(nm_mx4_export(nullptr, nullptr, nullptr) == NM_ERR_ARG && g_allocs.empty() && g_mode == hipStreamCaptureModeGlobal);
    float w[160] = {1, 2, 3};
    alignas(16) uint8_t q[128] = {}, s[16] = {};
    nm_mx4_t* h = nullptr;
    auto call = [&](const void* p, int dt, const uint8_t* sc, int experts, int channels, int width, int64_t ld, int gated) {
        return nm_mx4_pack(p, dt, sc, 2, experts, channels, width, ld, gated, nullptr, &h);
    };
    CHECK(nm_mx4_pack(w, NM_F32, nullptr, 0, 1, 4, 40, 40, 0, nullptr, nullptr) == NM_ERR_ARG);
    CHECK(call(nullptr, NM_F32, nullptr, 1, 4, 40, 40, 0) == NM_ERR_ARG);
    CHECK(call(w, NM_F32, s, 1, 4, 40, 40, 0) == NM_ERR_ARG);
    CHECK(call(q, NM_MX4, nullptr, 1, 4, 40, 32, 0) == NM_ERR_ARG);
    CHECK(call(q, NM_MX4, s, 1, 4, 40, 24, 0) == NM_ERR_ARG);
    CHECK(call(q + 4, NM_MX4, s, 1, 1, 40, 32, 0) == NM_ERR_ARG);
    CHECK(call(w, NM_I8, nullptr, 1, 4, 40, 40, 0) == NM_ERR_ARG);
    CHECK(call(w, NM_F32, nullptr, 1, 3, 40, 40, 1) == NM_ERR_ARG);
    CHECK(call(w, NM_F32, nullptr, 1, 4, 40, 40, 2) == NM_ERR_ARG);
    CHECK(call(w, NM_F32, nullptr, 0, 4, 40, 40, 0) == NM_ERR_ARG);
    CHECK(call(w, NM_F32, nullptr, NM_MX4_MAX_EXPERTS + 1, 4, 40, 40, 0) == NM_ERR_SHAPE);
    CHECK(call(w, NM_F32, nullptr, 1, (1 << 24) + 1, 40, 40, 0) == NM_ERR_SHAPE);
    CHECK(call(w, NM_F32, nullptr, 1024, 1 << 24, 40, 40, 0) == NM_ERR_SHAPE);
    CHECK(call(w, NM_F32, nullptr, 1, 4, NM_MX4_MAX_WIDTH + 1, 40, 0) == NM_ERR_SHAPE);
    g_capturing = true;
    CHECK(call(w, NM_F32, nullptr, 1, 4, 40, 40, 0) == NM_ERR_HIP && g_error.find("capture") != std::string::npos);
    g_capturing = false;
    g_no_device = true;
    CHECK(call(w, NM_F32, nullptr, 1, 4, 40, 40, 0) == NM_ERR_HIP);
    g_no_device = false;
    g_fail_pack = true;
    CHECK(call(w, NM_F32, nullptr, 1, 4, 40, 40, 0) == NM_ERR_HIP && !h);
    g_fail_pack = false;
    g_bad = true;
    CHECK(call(w, NM_F32, nullptr, 1, 4, 40, 40, 0) == NM_ERR_ARG && !h && g_error.find("finite") != std::string::npos);
    g_bad = false;
    CHECK(g_allocs.empty());
    // every allocation failing once, in the order they are made: an error, and nothing kept
    for (int dt : {(int)NM_F32, (int)NM_MX4}) {
        int failed = 0;
        for (int at = 0; at < 8; ++at) {
            g_mallocs = 0;
            g_fail_at = at;
            const int rc = call(dt == NM_F32 ? (void*)w : (void*)q, dt, dt == NM_F32 ? nullptr : s, 1, 4, 40, dt == NM_F32 ? 40 : 32, 0);
            g_fail_at = -1;
            if (rc == NM_OK) { nm_mx4_free(h); break; }
            CHECK(rc == NM_ERR_ALLOC && !h && g_allocs.empty());
            ++failed;
        }
        CHECK(failed == (dt == NM_F32 ? 5 : 3) && g_allocs.empty());
    }
    h = pack(1, 4, 40, 0);
    for (int at = 0; at < 2; ++at) {
        g_mallocs = 0;
        g_fail_at = at;
        CHECK(nm_mx4_export(h, q, nullptr) == NM_ERR_ALLOC);
        g_fail_at = -1;
    }
    nm_mx4_free(h);
    CHECK(g_allocs.empty());
}

static void products()
{
    nm_mx4_t *h = pack(1, 8, 40, 0), *hg = pack(1, 8, 40, 1), *he = pack(3, 8, 40, 0);
    alignas(16) uint8_t q[128] = {}, s[8] = {}, yq[256] = {}, ys[16] = {};
    float b[24] = {}, y[40] = {}, r[40] = {};
    int32_t off[4] = {}, idx[4] = {};
    auto linear = [&](const nm_mx4_t* w, int width, const float* bias, const void* res, int64_t ldr, void* out, int dt, int64_t ldy, uint8_t* sc) {
        return nm_linear_mx4(q, 32, s, 2, 4, width, w, bias, res, ldr, out, dt, ldy, sc, 1, nullptr);
    };
    CHECK(linear(h, 40, b, r, 8, y, NM_F32, 8, nullptr) == NM_OK && g_product.outs == 8 && g_product.rows == 4 && !g_product.gated && !g_product.grouped);
    CHECK(linear(hg, 40, b, nullptr, 0, y, NM_BF16, 4, nullptr) == NM_OK && g_product.outs == 4 && g_product.gated);
    CHECK(linear(h, 40, b, nullptr, 0, yq, NM_MX4, 16, ys) == NM_OK && g_product.out == NM_MX4 && g_product.ys == ys);
    CHECK(linear(h, 40, b, y, 8, y, NM_F32, 8, nullptr) == NM_OK);                  // the stream in place
    CHECK(linear(h, 40, b, y + 1, 8, y, NM_F32, 8, nullptr) == NM_ERR_ARG);
    CHECK(linear(h, 40, b, y, 7, y, NM_F32, 8, nullptr) == NM_ERR_ARG);
    CHECK(linear(nullptr, 40, b, nullptr, 0, y, NM_F32, 8, nullptr) == NM_ERR_ARG);
    CHECK(linear(h, 64, b, nullptr, 0, y, NM_F32, 8, nullptr) == NM_ERR_ARG);       // not the weights' width
    CHECK(linear(h, 40, b, nullptr, 0, y, NM_I8, 8, nullptr) == NM_ERR_ARG);
    CHECK(linear(h, 40, b, nullptr, 0, y, NM_F32, 7, nullptr) == NM_ERR_ARG);
    CHECK(linear(h, 40, b, nullptr, 0, y, NM_F32, 8, ys) == NM_ERR_ARG);            // scales of fp32
    CHECK(linear(h, 40, b, nullptr, 0, yq, NM_MX4, 16, nullptr) == NM_ERR_ARG);
    CHECK(linear(h, 40, b, nullptr, 0, yq, NM_MX4, 8, ys) == NM_ERR_ARG);
    CHECK(linear(h, 40, b, nullptr, 0, yq, NM_MX4, 16, yq + 16) == NM_ERR_ARG);     // scales among the codes
    CHECK(linear(h, 40, b, nullptr, 0, q, NM_MX4, 16, ys) == NM_ERR_ARG);
    CHECK(linear(h, 40, (float*)((char*)b + 2), nullptr, 0, y, NM_F32, 8, nullptr) == NM_ERR_ARG);
    CHECK(linear(hg, 40, b, r, 4, y, NM_F32, 4, nullptr) == NM_ERR_UNSUPPORTED);
    CHECK(linear(h, 40, b, yq, 16, yq, NM_MX4, 16, ys) == NM_ERR_UNSUPPORTED);
    CHECK(linear(he, 40, b, nullptr, 0, y, NM_F32, 8, nullptr) == NM_ERR_UNSUPPORTED);
    g_device = 1;
    CHECK(linear(h, 40, b, nullptr, 0, y, NM_F32, 8, nullptr) == NM_ERR_ARG && g_error.find("device") != std::string::npos);
    g_device = 0;
    const int before = g_launches;
    CHECK(nm_linear_mx4(nullptr, 32, nullptr, 2, 0, 40, h, nullptr, nullptr, 0, nullptr, NM_F32, 8, nullptr, 0, nullptr) == NM_OK && g_launches == before);

    auto experts = [&](int64_t rows, const int32_t* o, const int32_t* index, int64_t entries, void* out, int64_t ldy) {
        return nm_experts_mx4(q, 32, s, 2, rows, 40, he, o, index, entries, b, out, NM_F32, ldy, nullptr, 0, nullptr);
    };
    CHECK(experts(4, off, nullptr, 4, y, 8) == NM_OK && g_product.grouped && g_product.experts == 3 && g_product.rows == 4 && g_product.sources == 4);
    CHECK(experts(2, off, idx, 4, y, 8) == NM_OK && g_product.sources == 2 && g_product.index == idx);
    CHECK(experts(4, nullptr, nullptr, 4, y, 8) == NM_ERR_ARG);
    CHECK(experts(3, off, nullptr, 4, y, 8) == NM_ERR_ARG);       // without an index the rows are the entries
    CHECK(experts(0, off, idx, 4, y, 8) == NM_ERR_ARG);
    CHECK(experts(4, off, idx, -1, y, 8) == NM_ERR_ARG);
    CHECK(experts(4, off, idx, 0, y, 8) == NM_OK);
    CHECK(experts(4, off, idx, 4, idx, 8) == NM_ERR_ARG);
    CHECK(experts(4, off, idx, 4, off, 8) == NM_ERR_ARG);
    CHECK(nm_experts_mx4(q, (int64_t)1 << 24, s, 2, 300, 40, he, off, idx, 4, b, y, NM_F32, 8, nullptr, 0, nullptr) == NM_ERR_SHAPE);   // 4 GiB

    const nm_product_mx4_args_t pa{q, s, h, b, r, nullptr, nullptr, y, nullptr, nullptr, NM_F32, 4, 40, 32, 2, 8, 0, 8, 0};
    CHECK(nm_product_mx4_args(&pa) == NM_OK && g_product.res == r && !g_product.grouped);
    nm_product_mx4_args_t pb = pa;
    pb.dtype = (int64_t)1 << 32;          // not NM_F32
    CHECK(nm_product_mx4_args(&pb) == NM_ERR_ARG);
    pb = pa;
    pb.w = he;
    pb.offsets_dev = off;
    pb.index_dev = idx;
    pb.entries = 3;
    CHECK(nm_product_mx4_args(&pb) == NM_OK && g_product.rows == 3 && g_product.res == nullptr);
    for (nm_mx4_t* w : {h, hg, he}) nm_mx4_free(w);
    CHECK(g_allocs.empty());
}

static void routing()
{
    std::vector<float> l(100 * 8), w(200);
    std::vector<int32_t> ids(200), off(9), rows(200), slots(200);
    alignas(16) char ws[64];
    auto call = [&](const void* logits, int dt, int64_t tokens, int experts, int choices, int normalise, void* p, size_t n) {
        return nm_route(logits, dt, tokens, experts, 8, choices, normalise, ids.data(), w.data(), off.data(), rows.data(), slots.data(), p, n, nullptr);
    };
    CHECK(call(l.data(), NM_F32, 64, 8, 2, 1, nullptr, 0) == NM_OK && g_route.tokens == 64 && g_route.choices == 2 && !g_route.bf16);
    CHECK(call(l.data(), NM_F32, 65, 8, 2, 1, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(l.data(), NM_F32, 65, 8, 2, 1, ws, 31) == NM_ERR_ARG);
    CHECK(call(l.data(), NM_F32, 65, 8, 2, 1, ws + 4, 60) == NM_ERR_ARG);
    CHECK(call(l.data(), NM_F32, 65, 8, 2, 1, ws, 32) == NM_OK);
    CHECK(call(l.data(), NM_F32, 65, 8, 2, 1, l.data(), 32) == NM_ERR_ARG);
    CHECK(call(l.data(), NM_I8, 4, 8, 2, 1, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(l.data(), NM_BF16, 4, 8, 9, 1, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(l.data(), NM_BF16, 4, 8, 0, 1, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(l.data(), NM_BF16, 4, 8, 2, 2, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(l.data(), NM_BF16, -1, 8, 2, 1, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(l.data(), NM_F32, 4, NM_ROUTE_MAX_EXPERTS + 1, 2, 1, nullptr, 0) == NM_ERR_SHAPE);
    CHECK(call(l.data(), NM_F32, 4, 100, NM_ROUTE_MAX_CHOICES + 1, 1, nullptr, 0) == NM_ERR_SHAPE);
    CHECK(call(l.data(), NM_F32, (int64_t)1 << 30, 8, 2, 1, ws, 64) == NM_ERR_SHAPE);   // 2^31 entries
    CHECK(call(nullptr, NM_F32, 4, 8, 2, 1, nullptr, 0) == NM_ERR_ARG);
    CHECK(call(nullptr, NM_F32, 0, 8, 2, 1, nullptr, 0) == NM_OK);
    CHECK(call(ids.data(), NM_F32, 4, 8, 2, 1, nullptr, 0) == NM_ERR_ARG);
    CHECK(nm_route(l.data(), NM_F32, 4, 8, 8, 2, 1, ids.data(), w.data(), off.data(), rows.data(), ids.data() + 7, nullptr, 0, nullptr) == NM_ERR_ARG);
    CHECK(nm_route(l.data(), NM_F32, 4, 8, 8, 2, 1, ids.data(), w.data(), off.data(), rows.data(), ids.data() + 8, nullptr, 0, nullptr) == NM_OK);
    size_t n = 7;
    CHECK(nm_route_workspace(65, 8, &n) == NM_OK && n == 32 && nm_route_workspace(64, 8, &n) == NM_OK && n == 0);
    CHECK(nm_route_workspace(-1, 8, &n) == NM_ERR_ARG && nm_route_workspace(1, 0, &n) == NM_ERR_ARG && nm_route_workspace(1, 8, nullptr) == NM_ERR_ARG);
    const nm_route_args_t ra{l.data(), ids.data(), w.data(), off.data(), rows.data(), slots.data(), nullptr, nullptr, NM_F32, 4, 8, 8, 2, 1, 0};
    CHECK(nm_route_args(&ra) == NM_OK && g_route.normalise == 1);

    std::vector<float> y(64), out(64), res(64);
    auto combine = [&](const void* from, int64_t entries, int64_t tokens, int choices, const void* r, int64_t ldr, void* o, int64_t ldo) {
        return nm_combine(from, NM_F32, entries, 8, slots.data(), w.data(), tokens, choices, 8, r, ldr, o, NM_F32, ldo, nullptr);
    };
    CHECK(combine(y.data(), 8, 4, 2, res.data(), 8, out.data(), 8) == NM_OK && g_combine.entries == 8 && g_combine.res == res.data());
    CHECK(combine(y.data(), 8, 4, 2, out.data(), 8, out.data(), 8) == NM_OK);      // in place
    CHECK(combine(y.data(), 8, 4, 2, out.data() + 1, 8, out.data(), 8) == NM_ERR_ARG);
    CHECK(combine(y.data(), 8, 4, 2, nullptr, 8, y.data(), 8) == NM_ERR_ARG);
    CHECK(combine(nullptr, 0, 4, 2, nullptr, 8, out.data(), 8) == NM_OK);          // (no entries: only -1 is in range)
    CHECK(combine(nullptr, 1, 4, 2, nullptr, 8, out.data(), 8) == NM_ERR_ARG);
    CHECK(combine(y.data(), 8, 4, 0, nullptr, 8, out.data(), 8) == NM_ERR_ARG);
    CHECK(combine(y.data(), 8, 4, NM_ROUTE_MAX_CHOICES + 1, nullptr, 8, out.data(), 8) == NM_ERR_SHAPE);
    CHECK(combine(y.data(), 8, 4, 2, nullptr, 8, out.data(), 7) == NM_ERR_ARG);
    CHECK(combine(nullptr, 8, 0, 2, nullptr, 8, nullptr, 8) == NM_OK);
    const nm_combine_args_t ca{y.data(), slots.data(), w.data(), nullptr, out.data(), nullptr, NM_F32, 8, 8, 4, 2, 8, 0, NM_F32, 8};
    CHECK(nm_combine_args(&ca) == NM_OK && g_combine.choices == 2);
}

static_assert(sizeof(nm_rows_mx4_args_t) == 136 && sizeof(nm_dequantize_mx4_args_t) == 80 && sizeof(nm_product_mx4_args_t) == 152, "the binding packs these");
static_assert(sizeof(nm_route_args_t) == 120 && sizeof(nm_combine_args_t) == 120, "the binding packs these");

int main()
{
    overlaps();
    rows();
    weights();
    products();
    routing();
    printf("sanitizer run: ok\n");
    return 0;
}
