// Row operators in MX4: residual addition + root-mean-square norm + rounding, rounding alone, reading back.
//
//   h = x + r;  n = 1 / sqrt(mean(h^2) + eps);  v = (h n) gamma;  of 32 values a = max|v|, e = floor(log2 a) - 2, codes of v 2^-e
//
// Eight adjacent values a thread, four threads a block, whose largest magnitude goes round them in two exchanges of registers.
// Bound by HBM: a value is read once (twice with a residual) and written in 17/32 of a byte.
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
    double eps;
};

template <int CTRL> __device__ inline unsigned dpp(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }

// The largest over the four threads of a block (all four active).
__device__ inline unsigned block_max(unsigned m)
{
    m = max(m, dpp<0xb1>(m));    // lanes 1 0 3 2
    return max(m, dpp<0x4e>(m)); // lanes 2 3 0 1
}

template <bool BF16> __device__ inline void load_unit(const char* row, int c, int width, float (&v)[8])
{
    constexpr int ES = Elem<BF16>::kBytes;
    if (c + 8 <= width) {
        Elem<BF16>::load8(row + (size_t)c * ES, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < width ? Elem<BF16>::load1(row + (size_t)(c + e) * ES) : 0.0f;
    }
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
template <bool BF16>
__global__ __launch_bounds__(256) void mx4_round_kernel(Mx4Rows p)
{
    constexpr int ES = Elem<BF16>::kBytes;
    const int64_t total = p.rows * p.units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {   // (total is a multiple of 4)
        const int64_t row = total <= 0xffffffffll ? (int64_t)((unsigned)i / (unsigned)p.units) : i / p.units;
        const int u = (int)(i - row * p.units);
        float v[8];
        load_unit<BF16>(p.x + row * p.ldx * ES, u * 8, p.width, v);
        store_unit(p.q + row * p.ldq, p.scales + row * p.lds, u, v);
    }
}

template <int NT> __device__ inline double row_total(double v, double* part)
{
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    if constexpr (NT > 64) {
        __syncthreads();   // (the row before has been read)
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0;
        for (int i = 0; i < NT / 64; ++i) v += part[i];
    }
    return v;
}

// NT threads a row, VPT units a thread, held in registers over the sum.
template <bool BF16, int NT, int VPT>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void mx4_norm_kernel(Mx4Rows p)
{
#pragma clang fp contract(off)
    constexpr int ES = Elem<BF16>::kBytes, BLOCK = NT < 256 ? 256 : NT, RPB = BLOCK / NT;
    __shared__ double part[BLOCK / 64];
    const int t = threadIdx.x % NT;
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / NT; row < p.rows; row += (int64_t)gridDim.x * RPB) {
        float h[VPT][8];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (i * NT + t) * 8;
            load_unit<BF16>(p.x + row * p.ldx * ES, c, p.width, h[i]);
            if (p.res) {
                float r[8];
                load_unit<BF16>(p.res + row * p.ldr * ES, c, p.width, r);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[i][e] += r[e];
            }
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
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fma((double)h[i][e], (double)h[i][e], sum);
        const float n = (float)(1.0 / sqrt(row_total<NT>(sum, part) / (double)p.width + p.eps));
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int u = i * NT + t;
            if (u < p.units) {   // (whole blocks: the four threads of one agree)
                float g[8];
                if (p.gamma) load_unit<false>((const char*)p.gamma, u * 8, p.width, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    h[i][e] = h[i][e] * n;
                    if (p.gamma) h[i][e] = h[i][e] * g[e];
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

template <bool BF16, int NT, int VPT>
int launch_norm(const Mx4Rows& p, hipStream_t s)
{
    constexpr int BLOCK = NT < 256 ? 256 : NT, RPB = BLOCK / NT;
    hipLaunchKernelGGL((mx4_norm_kernel<BF16, NT, VPT>), dim3(grid_of((p.rows + RPB - 1) / RPB)), dim3(BLOCK), 0, s, p);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

template <bool BF16>
int pick_norm(const Mx4Rows& p, hipStream_t s)
{
    const int w = p.width;
    if (w <= 512) return launch_norm<BF16, 64, 1>(p, s);
    if (w <= 1024) return launch_norm<BF16, 64, 2>(p, s);
    if (w <= 2048) return launch_norm<BF16, 256, 1>(p, s);
    if (w <= 4096) return launch_norm<BF16, 512, 1>(p, s);
    if (w <= 6144) return launch_norm<BF16, 512, 2>(p, s);
    if (w <= 8192) return launch_norm<BF16, 1024, 1>(p, s);
    if (w <= 16384) return launch_norm<BF16, 1024, 2>(p, s);
    if (w <= 32768) return launch_norm<BF16, 1024, 4>(p, s);
    return launch_norm<BF16, 1024, 8>(p, s);
}

}  // namespace

int run_mx4_rows(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, const void* res, int64_t ldr,
                 const float* gamma, double eps, bool norm, void* out, int64_t ldo, uint8_t* q, int64_t ldq, uint8_t* scales,
                 int64_t lds, hipStream_t s)
{
    const int units = (width + 31) / 32 * 4;
    Mx4Rows p{(const char*)x, (const char*)res, gamma, (char*)out, q, scales, rows, ldx, ldr, ldo, ldq, lds, width, units, eps};
    if (norm) return dt == NM_F32 ? pick_norm<false>(p, s) : pick_norm<true>(p, s);
    const dim3 grid(grid_of((rows * units + 255) / 256));
    if (dt == NM_F32) hipLaunchKernelGGL((mx4_round_kernel<false>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((mx4_round_kernel<true>), grid, dim3(256), 0, s, p);
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
