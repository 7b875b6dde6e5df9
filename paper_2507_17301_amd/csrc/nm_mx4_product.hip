// Products of rows in MX4 with weights in MX4, of one matrix or grouped by expert.
//
//   z[r][c] = sum_k x[r][k] * w[c][k] + bias[c];   y = z (+ residual),  or  silu(gate) * up;   out in fp32, bf16 or MX4
//
// The matrix instruction takes codes and scales as they are; its sums of 128 products and their addition to the accumulators are in fp32
// (measured against 64 bits: within 2^-23 of the sum of the products' magnitudes).  Weights are its first operand, rows of x the second: lane l of
// a wavefront then holds packed weight rows 4 (l / 16) .. + 3 of a 16-row block for row l % 16 of x, and the packing deals channels so that
// the four blocks of a 64-row group give it twice 8 adjacent channels (gated: 8 adjacent outputs, gate and value in the same registers).
// (Out of registers, on normally distributed values, this form does 7.0 PFLOP/s and the 32x32x64 one 6.3; on zeros 9.7 and 8.9.)
#include "nm_mx4_product.h"

namespace nm {
namespace {

// ---------------------------------------------------------------- few rows
// Tiles of up to 16 * TB rows.  A workgroup owns RB blocks of 16 packed channels; its NW wavefronts take the steps of 256 k in turn, U of them
// in flight each, and add their sums through LDS at the end, in the order of the wavefronts.  Weights go from memory into registers: a
// weight is used once, there is nothing to share.  Rows of x go through LDS, a part of it for each wavefront, so that 8 lanes read the 128
// adjacent bytes of a row.
template <int TB, int RB, int NW, int U> constexpr int few4_lds()
{
    const int rows = NW * U * TB * 2048, sums = NW * RB * TB * 1024;
    return rows > sums ? rows : sums;
}

template <int TB, int RB, int NW, int U>
__global__ __launch_bounds__(NW * 64) void mx4_few_kernel(Mx4Product p, int parts)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int tile = blockIdx.x / parts, b0 = (blockIdx.x - tile * parts) * RB;   // (RB divides 4: a workgroup stays within its row group)
    const RowTile t = row_tile(p, tile, 16 * TB);
    if (t.count == 0) return;
    const size_t group = (size_t)t.expert * p.groups + (b0 >> 2);
    const __amdgpu_buffer_rsrc_t wsr = q8_rsrc(p.w + group * p.steps * 8192, (unsigned)p.steps * 8192);
    const __amdgpu_buffer_rsrc_t ssr = q8_rsrc(p.ws + group * p.steps * 128, (unsigned)p.steps * 512);
    const RowBuffers from(p, t);
    const unsigned woff = (b0 & 3) * 1024 + lane * 16, soff = ((b0 >> 1) & 1) * 256 + lane * 4;
    const unsigned mine = wave * (U * TB * 2048), lds0 = (unsigned)(uintptr_t)(lds_ptr_t)smem + mine;
    const unsigned at = mine + (lane & 15) * 128;
    unsigned qoff[TB][2];   // 8 rows an instruction, block c of a row at c ^ (row & 7)
    int source[TB];
    const int chunk = (lane & 7) ^ (lane >> 3);
#pragma unroll
    for (int i = 0; i < TB; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int src = source_of(p, t, i * 16 + h * 8 + (lane >> 3));
            qoff[i][h] = src < 0 ? kPast : (unsigned)(src * p.ldq) + chunk * 16;
        }
        source[i] = source_of(p, t, i * 16 + (lane & 15));
    }
    f32x4 acc[RB][TB] = {};
    for (int k0 = wave; k0 < p.steps; k0 += NW * U) {
        i32x4 wf[U][2][RB];
        unsigned wsc[U][RB == 4 ? 2 : 1], xsc[U][TB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u * NW;
            const bool in = k < p.steps;   // past the last step nothing is read and zeros are multiplied
            const bool row_in = k * 8 + chunk < p.blocks;
#pragma unroll
            for (int i = 0; i < TB; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    load_to_lds(from.q, row_in && qoff[i][h] != kPast ? qoff[i][h] + k * 128 : kPast, lds0 + u * TB * 2048 + i * 2048 + h * 1024);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < RB; ++i)
                    wf[u][h][i] = __builtin_bit_cast(
                        i32x4, __builtin_amdgcn_raw_buffer_load_b128(wsr, in ? woff + i * 1024 + (k * 2 + h) * 4096 : kPast, 0, 2));
#pragma unroll
            for (int i = 0; i < (RB == 4 ? 2 : 1); ++i) wsc[u][i] = __builtin_amdgcn_raw_buffer_load_b32(ssr, in ? soff + i * 256 + k * 512 : kPast, 0, 0);
#pragma unroll
            for (int i = 0; i < TB; ++i) xsc[u][i] = row_scales(p, from.s, source[i], k * 8 + 2 * (lane >> 4));
        }
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (RB == 1) wsc[u][0] >>= 16 * (b0 & 1);
            auto half = [&](auto hh) {
                constexpr int h = decltype(hh)::value;
                i32x4 xf[TB];
#pragma unroll
                for (int j = 0; j < TB; ++j)
                    xf[j] = *reinterpret_cast<const i32x4*>(smem + at + u * TB * 2048 + j * 2048 + (((2 * (lane >> 4) + h) ^ (lane & 7)) << 4));
#pragma unroll
                for (int j = 0; j < TB; ++j) {
                    acc[0][j] = mma4<h, h>(wf[u][h][0], xf[j], acc[0][j], wsc[u][0], xsc[u][j]);
                    if constexpr (RB >= 2) acc[1][j] = mma4<2 + h, h>(wf[u][h][1], xf[j], acc[1][j], wsc[u][0], xsc[u][j]);
                    if constexpr (RB == 4) {
                        acc[2][j] = mma4<h, h>(wf[u][h][2], xf[j], acc[2][j], wsc[u][1], xsc[u][j]);
                        acc[3][j] = mma4<2 + h, h>(wf[u][h][3], xf[j], acc[3][j], wsc[u][1], xsc[u][j]);
                    }
                }
            };
            half(std::integral_constant<int, 0>{});
            half(std::integral_constant<int, 1>{});
        }
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // read, before the next loads land there
    }
    __syncthreads();
    f32x4* part = reinterpret_cast<f32x4*>(smem);   // [NW][TB][RB][64]
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int i = 0; i < RB; ++i) part[((wave * TB + j) * RB + i) * 64 + lane] = acc[i][j];
    __syncthreads();
    // NB blocks of channels at a time: one, or as many as make the 32 outputs of a block in MX4
    auto finish = [&](auto gated, auto nb) {
        constexpr bool GATED = decltype(gated)::value;
        constexpr int NB = decltype(nb)::value;
        for (int u = wave; u < RB / NB * TB; u += NW) {
            const int i = u % (RB / NB) * NB, j = u / (RB / NB), rb = b0 + i;
            const int row = j * 16 + (lane & 15);
            Channels4<GATED, NB> ch;
            ch.load(p, t.expert, rb >> 2, rb & 3, lane);
            f32x4 sum[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                sum[b] = part[(j * RB + i + b) * 64 + lane];
#pragma unroll
                for (int n = 1; n < NW; ++n) sum[b] += part[((n * TB + j) * RB + i + b) * 64 + lane];
            }
            emit4<GATED, NB>(p, ch, sum, t.row0 + row, row < t.count);
        }
    };
    using One = std::integral_constant<int, 1>;
    if (p.out != NM_MX4) {
        if (p.gated) finish(std::true_type{}, One{});
        else finish(std::false_type{}, One{});
    } else {
        if constexpr (RB == 4) {
            if (p.gated) finish(std::true_type{}, std::integral_constant<int, 4>{});
        }
        if constexpr (RB >= 2) {
            if (!p.gated) finish(std::false_type{}, std::integral_constant<int, 2>{});
        }
    }
}

// ---------------------------------------------------------------- weights
// Codes of block kb of a row without those past the width.
__device__ inline i32x4 block_codes(const uint8_t* row, int kb, int width)
{
    i32x4 v = *reinterpret_cast<const i32x4*>(row + (size_t)kb * 16);
    const int n = width - kb * 32;   // values that the block has
    if (n < 32)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const int m = n - d * 8;
            if (m < 8) v[d] = m <= 0 ? 0 : v[d] & ((1 << (4 * m)) - 1);
        }
    return v;
}

// One 16-byte unit of the packed weights a thread, and a word of scales for every 16 of them.
__global__ __launch_bounds__(256) void mx4_pack_kernel(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, uint8_t* to,
                                                       unsigned* to_scales, int experts, int channels, int width, int gated, int groups,
                                                       int steps, int blocks, int* bad)
{
    const int64_t total = (int64_t)experts * groups * steps * 512;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int lane = (int)(i & 63), b = (int)(i >> 6) & 3, h = (int)(i >> 8) & 1;
        const int64_t gk = i >> 9;
        const int step = (int)(gk % steps), group = (int)(gk / steps % groups);
        const int64_t expert = gk / steps / groups;
        const int c = q8_row_of(group * 64 + b * 16 + (lane & 15), channels, gated), kb = step * 8 + 2 * (lane >> 4) + h;
        i32x4 v = {0, 0, 0, 0};
        if (c >= 0 && kb < blocks) v = block_codes(q + (expert * channels + c) * ldq, kb, width);
        *reinterpret_cast<i32x4*>(to + i * 16) = v;
        if (h == 0 && (b & 1) == 0) {
            unsigned word = 0;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int cn = q8_row_of(group * 64 + (b + (n >> 1)) * 16 + (lane & 15), channels, gated), kn = step * 8 + 2 * (lane >> 4) + (n & 1);
                unsigned s = 127;
                if (cn >= 0 && kn < blocks) s = scales[(expert * channels + cn) * lds + kn];
                if (s == 255) atomicOr(bad, 1);
                word |= s << (8 * n);
            }
            to_scales[(gk * 2 + (b >> 1)) * 64 + lane] = word;
        }
    }
}

__global__ __launch_bounds__(256) void mx4_unpack_kernel(const uint8_t* from, const unsigned* from_scales, uint8_t* q, uint8_t* scales, int experts,
                                                         int channels, int gated, int groups, int steps, int blocks)
{
    const int64_t total = (int64_t)experts * groups * steps * 512;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int lane = (int)(i & 63), b = (int)(i >> 6) & 3, h = (int)(i >> 8) & 1;
        const int64_t gk = i >> 9;
        const int step = (int)(gk % steps), group = (int)(gk / steps % groups);
        const int64_t expert = gk / steps / groups;
        const int c = q8_row_of(group * 64 + b * 16 + (lane & 15), channels, gated), kb = step * 8 + 2 * (lane >> 4) + h;
        if (c < 0 || kb >= blocks) continue;
        const int64_t row = expert * channels + c;
        *reinterpret_cast<i32x4*>(q + (row * blocks + kb) * 16) = *reinterpret_cast<const i32x4*>(from + i * 16);
        scales[row * blocks + kb] = (uint8_t)(from_scales[(gk * 2 + (b >> 1)) * 64 + lane] >> (8 * (2 * (b & 1) + h)));
    }
}

__global__ void mx4_clear_kernel(int* p) { *p = 0; }

// ---------------------------------------------------------------- launches
// Tiles of `per` rows that a call can have at most (the groups' sizes are known on the device only).
inline int64_t tiles_of(const Mx4Product& p, int per)
{
    if (!p.grouped) return ((int64_t)p.rows + per - 1) / per;
    return p.rows / per + (p.experts < p.rows ? p.experts : p.rows);
}

template <int TB, int RB, int NW, int U>
int launch_few4(const Mx4Product& p, hipStream_t s)
{
    constexpr int LDS = few4_lds<TB, RB, NW, U>();
    static_assert(LDS <= 64 * 1024, "more needs allow_lds");
    const int parts = p.groups * 4 / RB;
    const int64_t grid = tiles_of(p, 16 * TB) * parts;
    if (grid > 0x7fffffff) {
        set_error("%lld workgroups: too many", (long long)grid);
        return NM_ERR_SHAPE;
    }
    hipLaunchKernelGGL((mx4_few_kernel<TB, RB, NW, U>), dim3((unsigned)grid), dim3(NW * 64), LDS, s, p, parts);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

template <int TB>
int pick_few4(const Mx4Product& p, hipStream_t s)
{
    constexpr int U = TB == 4 ? 1 : 2;
    const int64_t groups = p.groups * (p.grouped ? (p.rows < p.experts ? p.rows : p.experts) : 1);
    if (groups >= 192 || (p.out == NM_MX4 && p.gated)) return launch_few4<TB, 4, 4, U>(p, s);
    if (groups >= 128 || p.out == NM_MX4) return launch_few4<TB, 2, 8, U>(p, s);
    return launch_few4<TB, 1, 8, U>(p, s);
}

}  // namespace

size_t mx4_workspace(const Mx4Product&) { return 0; }

int run_mx4_product(const Mx4Product& p, void*, hipStream_t s)
{
    const int64_t each = p.grouped ? (p.rows + p.experts - 1) / p.experts : p.rows;
    if (each <= 16) return pick_few4<1>(p, s);
    if (each <= 32) return pick_few4<2>(p, s);
    return pick_few4<4>(p, s);
}

int run_mx4_pack(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, const nm_mx4* h, int* d_bad, hipStream_t s)
{
    hipLaunchKernelGGL(mx4_clear_kernel, dim3(1), dim3(1), 0, s, d_bad);
    NM_HIP_CHECK(hipGetLastError());
    const int64_t blocks = (int64_t)h->experts * h->groups * h->steps * 2;
    hipLaunchKernelGGL(mx4_pack_kernel, dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), dim3(256), 0, s, q, ldq, scales, lds, h->d_w,
                       h->d_s, h->experts, h->channels, h->width, h->gated, h->groups, h->steps, h->blocks, d_bad);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

int run_mx4_unpack(const nm_mx4* h, uint8_t* q, uint8_t* scales, hipStream_t s)
{
    const int64_t blocks = (int64_t)h->experts * h->groups * h->steps * 2;
    hipLaunchKernelGGL(mx4_unpack_kernel, dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), dim3(256), 0, s, h->d_w, h->d_s, q, scales,
                       h->experts, h->channels, h->gated, h->groups, h->steps, h->blocks);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

}  // namespace nm
