// Checks of arguments that the entry points of the row operators and products share (host code).
#pragma once

#include "nm_q8_internal.h"

namespace nm {

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

inline int check_rows(int64_t rows, int width)
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

inline int check_span(const char* what, const Span& t, bool output)
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
inline bool overlap(const Span& a, const Span& b)
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

inline int check_apart(const char* what, const Span& out, const char* other, const Span& in, bool same_allowed)
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

}  // namespace nm
