// Row operators in MX4: residual addition + root-mean-square norm + rounding, rounding alone, reading back.
//
//   h = x + r;  n = 1 / sqrt(mean(h^2) + eps);  v = (h n) gamma;  of 32 values a = max|v|, e = floor(log2 a) - 2, codes of v 2^-e
//
// Eight adjacent values a thread, four threads a block, whose largest magnitude goes round them in two exchanges of registers.
// Bound by HBM: a value is read once (twice with a residual) and written in 17/32 of a byte.  16384 x 8192 in bf16: norm with a residual 164 us
// (5.3 TB/s), reading back 69 to 77 (4.4 to 4.9 TB/s); 4096 x 2048 rounded 7.0.
// The norm's sum is in 64 bits: its order then decides about n, and through n about a code on a border, once in some 10^8 rows.  (Sums in 32
// bits differ by their order in most rows.)
#include "nm_mx4_device.h"

namespace nm {
namespace {

struct Mx4Rows {
    const char* x;
    const char* res;
    const float* gamma;
    char* out;
    uint8_t* q;
    uint8_t* scales;
    int64_t rows, ldx, ldr, ldo, ldq, lds;
    int width, units;   // units: of 8 values, whole blocks
    double eps, each;   // each: 1 / width
};

template <int CTRL> __device__ inline unsigned dpp(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }

// The largest over the four threads of a block (all four active).
__device__ inline unsigned block_max(unsigned m)
{
    m = max(m, dpp<0xb1>(m));    // lanes 1 0 3 2
    return max(m, dpp<0x4e>(m)); // lanes 2 3 0 1
}

// The eight values at c of a row of at least 8; where it ends before them, the last eight: settle_unit puts that right.
template <bool BF16> __device__ inline void load_unit(const char* row, int c, int width, float (&v)[8])
{
    Elem<BF16>::load8(row + (unsigned)(min(c, width - 8) * Elem<BF16>::kBytes), v);
}

// Zeros for what lies past the end, as straight code: a branch a value would wait for each load by itself.
__device__ inline void settle_unit(int c, int width, float (&v)[8])
{
    const int over = c - (width - 8);
    if (over > 0) {
#pragma unroll
        for (int step = 1; step < 8; step <<= 1)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = over & step ? (e + step < 8 ? v[e + step < 8 ? e + step : 0] : 0.0f) : v[e];
        if (over >= 8)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    }
}

// A row of fewer than 8 values: its first unit has them all.
template <bool BF16> __device__ inline void load_short(const char* row, int c, int width, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < width ? Elem<BF16>::load1(row + (size_t)(c + e) * Elem<BF16>::kBytes) : 0.0f;
}

// Writes a thread's eight values; unit u of the row, whose scale's byte the first of a block's four threads writes.
__device__ inline void store_unit(uint8_t* q, uint8_t* scales, int u, const float (&v)[8])
{
    unsigned most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, magnitude(v[e]));
    const unsigned b = mx4_scale(block_max(most)), w = mx4_codes(v, b);
    *reinterpret_cast<unsigned*>(q + (size_t)u * 4) = w;   // (rows start at 16 bytes)
    if ((u & 3) == 0) scales[u >> 2] = (uint8_t)b;
}

// Blocks do not know of each other: a thread takes units 256 apart.
template <bool BF16, bool SHORT>
__global__ __launch_bounds__(256) void mx4_round_kernel(Mx4Rows p)
{
    constexpr int ES = Elem<BF16>::kBytes;
    const int64_t total = p.rows * p.units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {   // (total is a multiple of 4)
        const int64_t row = total <= 0xffffffffll ? (int64_t)((unsigned)i / (unsigned)p.units) : i / p.units;
        const int u = (int)(i - row * p.units);
        float v[8];
        if constexpr (SHORT) {
            load_short<BF16>(p.x + row * p.ldx * ES, u * 8, p.width, v);
        } else {
            load_unit<BF16>(p.x + row * p.ldx * ES, u * 8, p.width, v);
            settle_unit(u * 8, p.width, v);
        }
        store_unit(p.q + row * p.ldq, p.scales + row * p.lds, u, v);
    }
}

template <int CTRL> __device__ inline double dpp(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)dpp<CTRL>((unsigned)(u >> 32)) << 32 | dpp<CTRL>((unsigned)u));
}

// The sum over groups of N lanes (up to 64), the same bits in all of them.
template <int N> __device__ inline double lanes_total(double v)
{
    v += dpp<0xb1>(v);    // lane ^ 1
    v += dpp<0x4e>(v);    // lane ^ 2
    if constexpr (N > 4) v += dpp<0x141>(v);   // mirrored in eight
    if constexpr (N > 8) v += dpp<0x140>(v);   // mirrored in sixteen
    if constexpr (N > 16) {
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
    }
    return v;
}

template <int NT> __device__ inline double row_total(double v, double* part)
{
    v = lanes_total<64>(v);
    if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lanes_total<NT / 64>(part[threadIdx.x & (NT / 64 - 1)]);
    }
    return v;
}

// 1 / sqrt(a), to some bits of the last of 64: the instruction's 2^-26 or so, and a step of third order.  As it is for 0 and infinity.
__device__ inline double inverse_root(double a)
{
    const double y = __builtin_amdgcn_rsq(a), e = fma(-a * y, y, 1.0), z = fma(y * e, fma(e, 0.375, 0.5), y);
    return z == z ? z : y;
}

// NT threads a row, VPT units a thread, held in registers over the sum.  Loads go out in groups of units: all of them, or as many as 1024 threads'
// registers have room for (8192 x 16384 values, 512 x 4: 160 us, in twos 163, one by one 186).
template <bool BF16, int NT, int VPT, bool SHORT>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void mx4_norm_kernel(Mx4Rows p)
{
#pragma clang fp contract(off)
    constexpr int ES = Elem<BF16>::kBytes, BLOCK = NT < 256 ? 256 : NT, RPB = BLOCK / NT;
    constexpr int GROUP = VPT == 8 ? 1 : VPT == 4 && NT == 1024 ? 2 : VPT, AHEAD = VPT < 2 ? VPT : 2;   // AHEAD: units of gamma
    __shared__ double part[2][BLOCK / 64];   // in turn: a wavefront may still read one row's when another writes the next row's
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * RPB + (RPB > 1 ? threadIdx.x / NT : 0); row < p.rows; row += (int64_t)gridDim.x * RPB) {
        int t = RPB > 1 ? threadIdx.x % NT : threadIdx.x;
        if constexpr (VPT > 2) asm volatile("" : "+v"(t));   // (offsets made from it outside the loop would take all registers)
        const char *px = p.x + row * p.ldx * ES, *pr = p.res ? p.res + row * p.ldr * ES : nullptr;
        float h[VPT][8];
#pragma unroll
        for (int i0 = 0; i0 < VPT; i0 += GROUP) {
            float r[GROUP][8];
            if constexpr (SHORT) {
                load_short<BF16>(px, t * 8, p.width, h[0]);
                if (pr) load_short<BF16>(pr, t * 8, p.width, r[0]);
            } else {
#pragma unroll
                for (int i = 0; i < GROUP; ++i) load_unit<BF16>(px, ((i0 + i) * NT + t) * 8, p.width, h[i0 + i]);
                if (pr)
#pragma unroll
                    for (int i = 0; i < GROUP; ++i) load_unit<BF16>(pr, ((i0 + i) * NT + t) * 8, p.width, r[i]);
            }
            if (pr)
#pragma unroll
                for (int i = 0; i < GROUP; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) h[i0 + i][e] += r[i][e];
            if (!SHORT && (i0 + GROUP) * NT * 8 > p.width)
#pragma unroll
                for (int i = 0; i < GROUP; ++i) settle_unit(((i0 + i) * NT + t) * 8, p.width, h[i0 + i]);
        }
        if (p.out) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int c = (i * NT + t) * 8;
                char* po = p.out + (row * p.ldo + c) * ES;
                if (c + 8 <= p.width) Elem<BF16>::store8(po, h[i]);
                else
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (c + e < p.width) Elem<BF16>::store1(po + e * ES, h[i][e]);
            }
        }
        float g[AHEAD][8];
        auto gain = [&](int i) {   // (the last one of a row is settled below)
            if constexpr (SHORT) load_short<false>((const char*)p.gamma, t * 8, p.width, g[0]);
            else load_unit<false>((const char*)p.gamma, (i * NT + t) * 8, p.width, g[i % AHEAD]);
        };
        if (p.gamma)
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) gain(i);
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fma((double)h[i][e], (double)h[i][e], sum);
        const float n = (float)inverse_root(row_total<NT>(sum, part[turn]) * p.each + p.eps);
        turn ^= 1;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int u = i * NT + t;
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] = h[i][e] * n;
            if (p.gamma) {
                if (!SHORT && (i + 1) * NT * 8 > p.width) settle_unit(u * 8, p.width, g[i % AHEAD]);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[i][e] = h[i][e] * g[i % AHEAD][e];
                if (i + AHEAD < VPT) gain(i + AHEAD);
            }
            if (u < p.units) {   // (whole blocks: the four threads of one agree)
                if (u * 8 + 8 > p.width) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (u * 8 + e >= p.width) h[i][e] = 0.0f;   // (0 * infinity in a row without a norm)
                }
                store_unit(p.q + row * p.ldq, p.scales + row * p.lds, u, h[i]);
            }
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, char* y,
                                                             int64_t ldy, int64_t rows, int width, int units)
{
    constexpr int ES = Elem<BF16>::kBytes;
    const int64_t total = rows * units;   // of 8 values
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = total <= 0xffffffffll ? (int64_t)((unsigned)i / (unsigned)units) : i / units;
        const int u = (int)(i - row * units), c = u * 8;
        float v[8];
        mx4_values(*reinterpret_cast<const unsigned*>(q + row * ldq + (size_t)u * 4), scales[row * lds + (u >> 2)], v);
        char* py = y + (row * ldy + c) * ES;
        if (c + 8 <= width) Elem<BF16>::store8(py, v);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < width) Elem<BF16>::store1(py + e * ES, v[e]);
    }
}

inline unsigned grid_of(int64_t blocks) { return (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)); }

template <bool BF16, int NT, int VPT, bool SHORT = false>
int launch_norm(const Mx4Rows& p, hipStream_t s)
{
    constexpr int BLOCK = NT < 256 ? 256 : NT, RPB = BLOCK / NT;
    hipLaunchKernelGGL((mx4_norm_kernel<BF16, NT, VPT, SHORT>), dim3(grid_of((p.rows + RPB - 1) / RPB)), dim3(BLOCK), 0, s, p);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

// Threads of a row.  us, bf16 with a residual and h stored, threads x units a thread, 1 row, 256, and 16384 (8192 of 16384 values):
//    4096   512 x 1  2.9   -    86     256 x 2  3.4   -    92     256 x 4  5.1   -   108
//    8192  1024 x 1  3.7  6.2  202     512 x 2  3.9  6.4  188     256 x 4  4.4  6.6  160
//   16384  1024 x 2   -   8.0  183     512 x 4   -   7.6  163
//   32768  1024 x 4   -    -   177     512 x 8   -    -   190   (4096 rows)
// The many rows move 4.7 to 5.5 TB/s.
template <bool BF16>
int pick_norm(const Mx4Rows& p, hipStream_t s)
{
    const int w = p.width;
    if (w < 8) return launch_norm<BF16, 64, 1, true>(p, s);
    if (w <= 512) return launch_norm<BF16, 64, 1>(p, s);
    if (w <= 1024) return launch_norm<BF16, 64, 2>(p, s);
    if (w <= 2048) return launch_norm<BF16, 256, 1>(p, s);
    if (w <= 4096) return launch_norm<BF16, 512, 1>(p, s);
    const bool few = p.rows < 256;
    if (w <= 8192) return few ? launch_norm<BF16, 1024, 1>(p, s) : launch_norm<BF16, 256, 4>(p, s);
    if (w <= 16384) return few ? launch_norm<BF16, 1024, 2>(p, s) : launch_norm<BF16, 512, 4>(p, s);
    if (w <= 32768) return launch_norm<BF16, 1024, 4>(p, s);
    return launch_norm<BF16, 1024, 8>(p, s);
}

}  // namespace

int run_mx4_rows(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, const void* res, int64_t ldr,
                 const float* gamma, double eps, bool norm, void* out, int64_t ldo, uint8_t* q, int64_t ldq, uint8_t* scales,
                 int64_t lds, hipStream_t s)
{
    const int units = (width + 31) / 32 * 4;
    Mx4Rows p{(const char*)x, (const char*)res, gamma, (char*)out, q, scales, rows, ldx, ldr, ldo, ldq, lds, width, units, eps, 1.0 / width};
    if (norm) return dt == NM_F32 ? pick_norm<false>(p, s) : pick_norm<true>(p, s);
    const dim3 grid(grid_of((rows * units + 255) / 256));
    const bool f32 = dt == NM_F32;
    if (f32 && width < 8) hipLaunchKernelGGL((mx4_round_kernel<false, true>), grid, dim3(256), 0, s, p);
    else if (f32) hipLaunchKernelGGL((mx4_round_kernel<false, false>), grid, dim3(256), 0, s, p);
    else if (width < 8) hipLaunchKernelGGL((mx4_round_kernel<true, true>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((mx4_round_kernel<true, false>), grid, dim3(256), 0, s, p);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

int run_mx4_dequantize(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, int64_t rows, int width, void* y,
                       nm_dtype_t dt, int64_t ldy, hipStream_t s)
{
    const int units = (width + 7) / 8;
    const dim3 grid(grid_of((rows * units + 255) / 256));
    if (dt == NM_F32) hipLaunchKernelGGL((mx4_dequantize_kernel<false>), grid, dim3(256), 0, s, q, ldq, scales, lds, (char*)y, ldy, rows, width, units);
    else hipLaunchKernelGGL((mx4_dequantize_kernel<true>), grid, dim3(256), 0, s, q, ldq, scales, lds, (char*)y, ldy, rows, width, units);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

}  // namespace nm
