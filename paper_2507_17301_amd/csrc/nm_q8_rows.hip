// Row operators in 8 bits: residual addition + root-mean-square norm + rounding, rounding alone, reading back.
//
//   h = x + r;  v = gamma * h / sqrt(mean(h^2) + eps);  s = max|v| / 127;  q = rint(v * 127 / max|v|)
//
// Bound by HBM: a value is read once (twice with a residual), kept in registers over both reductions (sum of
// squares, largest magnitude), and written once.  NT threads share a row, 8 adjacent values a thread at a time,
// so that a wavefront reads 1 KiB (bf16) or 2 KiB (fp32) of adjacent bytes an instruction and writes 512 bytes
// of q.  One wavefront a row up to 1024 values (no barrier), a workgroup beyond (pick_rows).
// Rows of odd widths and strides run the same code (global memory takes a 16-byte access at any address); only what a
// width leaves past its last group of 8 is taken value by value, one value a thread.
// Sums, norm and products are fp32; the one rounding to fewer bits is that to q, of the unrounded h.
// 16384 rows of 8192 in bf16 with a residual: 185 us, 940 MB, 5.1 TB/s (a copy of 1 GiB reaches as much); in fp32, 16384 of 5001 with a
// residual 226 us, 4.7 TB/s, and without one 112 us, 3.7: 512 x 2 groups leave 39 % of the slots empty there.
#include "nm_q8_device.h"

namespace nm {
namespace {

struct RowArgs {
    const char* x;
    const char* res;
    const float* gamma;
    char* out;
    int8_t* q;
    float* scales;
    int64_t rows, ldx, ldr, ldo, ldq;
    int width;
    float eps;
};

// Sum (or largest) over the NT threads of a row; `part` holds one slot for each wavefront of the row.
template <int NT>
__device__ inline float row_sum(float v, float* part)
{
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
        for (int i = 0; i < NT / 64; ++i) v += part[i];
    }
    return v;
}
template <int NT>
__device__ inline unsigned row_max(unsigned v, unsigned* part)
{
    for (int m = 1; m < 64; m <<= 1) v = max(v, (unsigned)__shfl_xor((int)v, m));
    if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        for (int i = 0; i < NT / 64; ++i) v = max(v, part[i]);
    }
    return v;
}

// x * 127 / a rounded once to fp32, so that a quotient half way between two whole numbers goes to the even one.  (x times 127 / a rounded is
// off a half step by up to 2^-17: 63.5 became 63 under half of all bf16 magnitudes a.)
// bf16: 127 / a in two parts, the first of 16 bits, whose product with x is exact.
// fp32: the product with 127 / a rounded, then its rounding and that of 127 / a added.
template <bool BF16> struct Quotient {
    float inv, rest;
    __device__ inline explicit Quotient(float a) : inv(127.0f / a)
    {
        if constexpr (BF16) {
            inv = __uint_as_float(__float_as_uint(inv) & 0xffffff00u);
            rest = fmaf(-inv, a, 127.0f) / a;
        } else {
            rest = fmaf(-inv, a, 127.0f) * (1.0f / 127.0f);
        }
    }
    __device__ inline float operator()(float x) const
    {
#pragma clang fp contract(off)
        const float y = x * inv;
        if constexpr (BF16) return fmaf(x, rest, y);
        else return y + fmaf(y, rest, fmaf(x, inv, -y));
    }
};

template <bool BF16, int NT, int VPT, bool NORM>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void q8_rows_kernel(RowArgs p)
{
    constexpr int ES = Elem<BF16>::kBytes, BLOCK = NT < 256 ? 256 : NT, RPB = BLOCK / NT;
    constexpr bool EARLY = VPT <= 2;
    __shared__ float psum[NORM ? 2 : 1][NT / 64];   // (the second sum of a row whose first is too small)
    __shared__ unsigned pmax[2][NT / 64];   // in turn: a wavefront may still read one row's when another writes the next row's
    int turn = 0;
    const int t = threadIdx.x % NT;
    const int whole = p.width & ~7, over = p.width & 7;   // the values past the last group of 8: one each for the first threads
    // (with several rows a workgroup there is no barrier, and its wavefronts may leave the loop apart)
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / NT; row < p.rows; row += (int64_t)gridDim.x * RPB) {
        const char* px = p.x + row * p.ldx * ES;
        const char* pr = NORM && p.res ? p.res + row * p.ldr * ES : nullptr;
        char* po = NORM && p.out ? p.out + row * p.ldo * ES : nullptr;
        float h[VPT][8], hx = 0.0f;   // values past the end are 0: they change neither the sum nor the largest magnitude
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = (v * NT + t) * 8;
            if (c < whole)
                Elem<BF16>::load8(px + (size_t)c * ES, h[v]);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) h[v][e] = 0.0f;
        }
        if (t < over) hx = Elem<BF16>::load1(px + (size_t)(whole + t) * ES);
        if (NORM && pr) {
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                const int c = (v * NT + t) * 8;
                if (c < whole) {
                    float r[8];
                    Elem<BF16>::load8(pr + (size_t)c * ES, r);
#pragma unroll
                    for (int e = 0; e < 8; ++e) h[v][e] += r[e];
                }
            }
            if (t < over) hx += Elem<BF16>::load1(pr + (size_t)(whole + t) * ES);
        }
        if (NORM && po) {
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                const int c = (v * NT + t) * 8;
                if (c < whole) Elem<BF16>::store8(po + (size_t)c * ES, h[v]);
            }
            if (t < over) Elem<BF16>::store1(po + (size_t)(whole + t) * ES, hx);
        }
        bool bad = false;
        if constexpr (NORM) {
            float gain[EARLY ? VPT : 1][8], gx = 1.0f;   // (read ahead of the reductions, while the registers last)
            if (EARLY && p.gamma) {
#pragma unroll
                for (int v = 0; v < VPT; ++v) {
                    const int c = (v * NT + t) * 8;
                    if (c < whole) Elem<false>::load8((const char*)(p.gamma + c), gain[v]);
                }
                if (t < over) gx = p.gamma[whole + t];
            }
            auto squares = [&] {
                float sum = hx * hx;
#pragma unroll
                for (int v = 0; v < VPT; ++v)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum = fmaf(h[v][e], h[v][e], sum);
                return sum;
            };
            const float sum = row_sum<NT>(squares(), psum[0]);
            bad = (__float_as_uint(sum) & 0x7fffffffu) >= 0x7f800000u;
            float mean = sum / (float)p.width + p.eps;
            // Squares (and an eps) that fp32 holds in few bits or not at all: the same of h * 2^64, exact.  All threads of a row come here
            // or none.  Partial sums are off by 2^-150 each at most where fp32 no longer holds them in full: a share of 2^-70 at this limit.
            if (mean < 0x1p-80f) {
                constexpr float kUp = 0x1p64f;
#pragma unroll
                for (int v = 0; v < VPT; ++v)
#pragma unroll
                    for (int e = 0; e < 8; ++e) h[v][e] *= kUp;
                hx *= kUp;
                mean = row_sum<NT>(squares(), psum[1]) / (float)p.width + p.eps * kUp * kUp;
                bad = mean < 0x1p-110f;   // a root mean square below 2^-119
            }
            const float r = 1.0f / sqrtf(mean);
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) h[v][e] *= r;
            hx *= r;
            if (p.gamma) {
#pragma unroll
                for (int v = 0; v < VPT; ++v) {
                    const int c = (v * NT + t) * 8;
                    if (c < whole) {
                        if constexpr (!EARLY) Elem<false>::load8((const char*)(p.gamma + c), gain[0]);
#pragma unroll
                        for (int e = 0; e < 8; ++e) h[v][e] *= gain[EARLY ? v : 0][e];
                    }
                }
                if constexpr (!EARLY) {
                    if (t < over) gx = p.gamma[whole + t];
                }
                hx *= gx;
            }
        }
        // the largest magnitude as bits: a NaN is larger than infinity, which is larger than any number
        unsigned most = __float_as_uint(hx) & 0x7fffffffu;
#pragma unroll
        for (int v = 0; v < VPT; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(h[v][e]) & 0x7fffffffu);
        most = row_max<NT>(most, pmax[turn]);
        turn ^= 1;
        bad = bad || most >= 0x7f800000u;
        const float a = __uint_as_float(most);
        const bool none = !(a >= 127.0f * 1.17549435e-38f);
        const float inv = 127.0f / a;
        if (t == 0) p.scales[row] = bad ? __uint_as_float(0x7fc00000u) : none ? 0.0f : a / 127.0f;
        int8_t* pq = p.q + row * p.ldq;
        const bool zero = bad || none;
        // 1.5 * 2^23 + n holds n, rounded to nearest even by the addition, in its low bits.  (A norm's values are themselves rounded ones.)
        const Quotient<BF16> quotient(a);
        auto round8 = [&](float f) {
            if constexpr (NORM) return zero ? 0u : __float_as_uint(fmaf(f, inv, 12582912.0f)) & 0xffu;
            else return zero ? 0u : __float_as_uint(quotient(f) + 12582912.0f) & 0xffu;
        };
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = (v * NT + t) * 8;
            if (c < whole) {
                u32x2 w;
                w[0] = round8(h[v][0]) | round8(h[v][1]) << 8 | round8(h[v][2]) << 16 | round8(h[v][3]) << 24;
                w[1] = round8(h[v][4]) | round8(h[v][5]) << 8 | round8(h[v][6]) << 16 | round8(h[v][7]) << 24;
                __builtin_memcpy(pq + c, &w, 8);
            }
        }
        if (t < over) pq[whole + t] = (int8_t)round8(hx);
    }
}

// The values that 8-bit rows stand for: 8 adjacent ones a thread.  Bound by HBM: 134 million values to bf16 in 66 us, 6.1 TB/s.
template <bool BF16>
__global__ __launch_bounds__(256) void q8_dequantize_kernel(const int8_t* q, int64_t ldq, const float* scales, char* y,
                                                            int64_t ldy, int64_t rows, int width, int units)
{
    constexpr int ES = Elem<BF16>::kBytes;
    const int64_t total = rows * units;   // of 8 values
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = total <= 0xffffffffll ? (int64_t)((unsigned)i / (unsigned)units) : i / units;
        const int c = (int)(i - row * units) * 8;
        const int8_t* pq = q + row * ldq + c;
        char* py = y + (row * ldy + c) * ES;
        const float s = scales[row];
        if (c + 8 <= width) {
            u32x2 w;
            __builtin_memcpy(&w, pq, 8);
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)(w[e / 4] >> (8 * (e % 4))) * s;
            Elem<BF16>::store8(py, v);
        } else {
            for (int e = 0; c + e < width; ++e) Elem<BF16>::store1(py + (size_t)e * ES, (float)pq[e] * s);
        }
    }
}

template <bool BF16, int NT, int VPT, bool NORM>
int launch_rows(const RowArgs& p, hipStream_t s)
{
    constexpr int BLOCK = NT < 256 ? 256 : NT, RPB = BLOCK / NT;
    const int64_t blocks = (p.rows + RPB - 1) / RPB;
    const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20));
    hipLaunchKernelGGL((q8_rows_kernel<BF16, NT, VPT, NORM>), dim3(grid), dim3(BLOCK), 0, s, p);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

// Threads of a row.  us, bf16, threads x groups of 8 a thread, 1 row and 16384:
//   norm      4096   512 x 1  3.2   91     256 x 2  3.6   92     256 x 4  4.1  126    1024 x 1  3.5  134
//             8192  1024 x 1  4.0  189     512 x 2  3.8  195     256 x 4  5.1  224     512 x 4  4.4  345
//            16384  1024 x 2  4.9  342     256 x 8  7.1  392     512 x 4  5.5  566
//   rounding  4096   256 x 2  2.6   37     512 x 1  2.6   39    1024 x 1  2.7   65
//             8192   512 x 2  2.6   69     256 x 4  2.9   73    1024 x 1  2.7   84
//            16384  1024 x 2  3.0  134     256 x 8  3.9  144     512 x 4  3.1  145
// (16384 rows: 5.0 to 5.4 TB/s for the norm, 5.5 to 6.0 for the rounding, whose rows partly come from the last-level cache.  The rounding's
// figures are with one multiplication a value; Quotient's adds 0 to 3 %, 4 % at 512 values a row.)
template <bool BF16, bool NORM>
int pick_rows(const RowArgs& p, hipStream_t s)
{
    const int w = p.width;
    if (w <= 512) return launch_rows<BF16, 64, 1, NORM>(p, s);
    if (w <= 1024) return launch_rows<BF16, 64, 2, NORM>(p, s);
    if (w <= 2048) return launch_rows<BF16, 256, 1, NORM>(p, s);
    if (w <= 4096) return launch_rows<BF16, NORM ? 512 : 256, NORM ? 1 : 2, NORM>(p, s);
    if (w <= 6144 || (w <= 8192 && !NORM)) return launch_rows<BF16, 512, 2, NORM>(p, s);   // (1024 threads would not all have work)
    if (w <= 8192) return launch_rows<BF16, 1024, 1, NORM>(p, s);
    if (w <= 16384) return launch_rows<BF16, 1024, 2, NORM>(p, s);
    if (w <= 32768) return launch_rows<BF16, 1024, 4, NORM>(p, s);
    return launch_rows<BF16, 1024, 8, NORM>(p, s);
}

}  // namespace

int run_q8_rows(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, const void* res, int64_t ldr,
                const float* gamma, float eps, bool norm, void* out, int64_t ldo, int8_t* q, int64_t ldq, float* scales,
                hipStream_t s)
{
    RowArgs p{(const char*)x, (const char*)res, gamma, (char*)out, q, scales, rows, ldx, ldr, ldo, ldq, width, eps};
    if (dt == NM_F32) return norm ? pick_rows<false, true>(p, s) : pick_rows<false, false>(p, s);
    return norm ? pick_rows<true, true>(p, s) : pick_rows<true, false>(p, s);
}

int run_q8_dequantize(const int8_t* q, int64_t ldq, const float* scales, int64_t rows, int width, void* y, nm_dtype_t dt,
                      int64_t ldy, hipStream_t s)
{
    const int units = (width + 7) / 8;
    const int64_t blocks = (rows * units + 255) / 256;
    const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20));
    if (dt == NM_F32)
        hipLaunchKernelGGL((q8_dequantize_kernel<false>), dim3(grid), dim3(256), 0, s, q, ldq, scales, (char*)y, ldy, rows, width, units);
    else
        hipLaunchKernelGGL((q8_dequantize_kernel<true>), dim3(grid), dim3(256), 0, s, q, ldq, scales, (char*)y, ldy, rows, width, units);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

}  // namespace nm
