// Product of 8-bit rows with 8-bit weights, a scale for each row and each channel.
//
//   y[r][c] = (sum_k q[r][k] * w[c][k]) * (s[r] * t[c]) + bias[c] (+ residual[r][c]),  or  silu(gate) * up
//
// The sum is in 32-bit integers and exact, so no split of K changes a result.  Weights are the first operand of the
// 16x16x64 integer matrix instruction, rows of q the second: lane l of a wavefront then holds packed weight rows
// 4 (l / 16) .. + 3 of a 16-row block for row l % 16 of q, and the packing deals channels so that the four blocks of
// a 64-row group give it 16 adjacent channels (gated: 8 adjacent outputs, gate and value in the same registers).
#include "nm_q8_device.h"

namespace nm {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr_t;

__device__ inline __amdgpu_buffer_rsrc_t q8_rsrc(const void* p, unsigned bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

__device__ inline i32x4 mma(i32x4 w, i32x4 q, i32x4 acc) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, q, acc, 0, 0, 0); }

// ---------------------------------------------------------------- epilogue
// What a lane needs of the channels it holds over NB blocks (from block b0 on) of one row group.
template <bool GATED, int NB> struct Channels {
    static constexpr int kOuts = GATED ? 2 * NB : 4 * NB;   // adjacent outputs of a lane
    int c0;                                                 // the first of them
    f32x4 t[NB], bias[NB];

    __device__ inline void load(const Q8Linear& p, int group, int b0, int lane)
    {
        const int g = lane >> 4, half = p.channels / 2;
        c0 = GATED ? group * 32 + g * 8 + b0 * 2 : group * 64 + g * 16 + b0 * 4;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            t[b] = *reinterpret_cast<const f32x4*>(p.ws + group * 64 + (b0 + b) * 16 + g * 4);
            bias[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (p.bias) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if constexpr (GATED) {
                        const int o = c0 + 2 * b + (r & 1);
                        if (o < half) bias[b][r] = p.bias[r < 2 ? o : half + o];
                    } else {
                        const int c = c0 + 4 * b + r;
                        if (c < p.channels) bias[b][r] = p.bias[c];
                    }
                }
            }
        }
    }
};

__device__ inline float silu_times(float gate, float up) { return gate / (1.0f + __expf(-gate)) * up; }

// Scales the sums of one row of q and stores its outputs.
template <bool GATED, bool BF16, int NB>
__device__ inline void emit(const Q8Linear& p, const Channels<GATED, NB>& ch, const i32x4 (&acc)[NB], int64_t row, float s)
{
    constexpr int N = Channels<GATED, NB>::kOuts, ES = Elem<BF16>::kBytes;
    float y[N];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        float z[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) z[r] = fmaf((float)acc[b][r], s * ch.t[b][r], ch.bias[b][r]);
        if constexpr (GATED) {
            y[2 * b] = silu_times(z[0], z[2]);
            y[2 * b + 1] = silu_times(z[1], z[3]);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) y[4 * b + r] = z[r];
        }
    }
    char* py = (char*)p.y + (row * p.ldy + ch.c0) * ES;
    const char* pr = p.res ? (const char*)p.res + (row * p.ldr + ch.c0) * ES : nullptr;
    if (N % 8 == 0 && ch.c0 + N <= p.outs) {
#pragma unroll
        for (int i = 0; i < N; i += 8) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = y[i + e];
            if (!GATED && pr) {
                float r[8];
                Elem<BF16>::load8(pr + i * ES, r);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += r[e];
            }
            Elem<BF16>::store8(py + i * ES, v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (ch.c0 + i < p.outs) {
                float v = y[i];
                if (!GATED && pr) v += Elem<BF16>::load1(pr + i * ES);
                Elem<BF16>::store1(py + i * ES, v);
            }
        }
    }
}

// ---------------------------------------------------------------- few rows
// Up to 16 * TB rows of q.  A workgroup owns RB blocks of 16 packed channels; its NW wavefronts take the 64-k blocks in
// turn, straight from memory into registers (a weight is used once, there is nothing to share), and add their sums
// through LDS.  Bound by the weights' bytes.
template <int TB, int RB, int NW, bool GATED, bool BF16>
__global__ __launch_bounds__(NW * 64) void q8_few_kernel(Q8Linear p)
{
    constexpr int U = TB * RB >= 4 ? 2 : 4;   // k blocks in flight
    __shared__ i32x4 part[NW][RB * TB][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row0 = (int64_t)blockIdx.y * (16 * TB);
    const int8_t* w[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        const int rb = blockIdx.x * RB + i;   // (RB divides 4: a workgroup stays within its row group)
        w[i] = p.w + ((size_t)(rb >> 2) * p.kblocks * 4 + (rb & 3)) * 1024 + lane * 16;
    }
    const int8_t* q[TB];
    bool there[TB];
#pragma unroll
    for (int i = 0; i < TB; ++i) {
        const int64_t row = row0 + i * 16 + (lane & 15);
        there[i] = row < p.rows;
        q[i] = p.q + (there[i] ? row : 0) * p.ldq + (lane >> 4) * 16;
    }
    const int kq = p.width - (lane >> 4) * 16;   // values of the row from this lane's first one on
    i32x4 acc[RB][TB] = {};
    for (int kb = wave; kb < p.kblocks; kb += NW * U) {
        i32x4 wf[U][RB], qf[U][TB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = kb + u * NW;
            const bool in = k < p.kblocks;   // (the same for the whole wavefront)
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                wf[u][i] = i32x4{0, 0, 0, 0};
                if (in) wf[u][i] = *reinterpret_cast<const i32x4*>(w[i] + (size_t)k * 4096);
            }
#pragma unroll
            for (int i = 0; i < TB; ++i) {
                qf[u][i] = i32x4{0, 0, 0, 0};
                if (there[i] && k * 64 + 16 <= kq) {
                    __builtin_memcpy(&qf[u][i], q[i] + (size_t)k * 64, 16);
                } else if (there[i] && k * 64 < kq) {
                    for (int e = 0; e < kq - k * 64; ++e) {   // the row's end
                        const int b = (int)(unsigned char)q[i][(size_t)k * 64 + e] << (8 * (e & 3));
#pragma unroll
                        for (int d = 0; d < 4; ++d) qf[u][i][d] |= (e >> 2) == d ? b : 0;
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < RB; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) acc[i][j] = mma(wf[u][i], qf[u][j], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) part[wave][i * TB + j][lane] = acc[i][j];
    __syncthreads();
    for (int u = wave; u < RB * TB; u += NW) {
        const int i = u / TB, j = u % TB, rb = blockIdx.x * RB + i;
        i32x4 sum[1] = {part[0][u][lane]};
#pragma unroll
        for (int n = 1; n < NW; ++n) sum[0] += part[n][u][lane];
        const int64_t row = row0 + j * 16 + (lane & 15);
        if (row < p.rows) {
            Channels<GATED, 1> ch;
            ch.load(p, rb >> 2, rb & 3, lane);
            emit<GATED, BF16, 1>(p, ch, sum, row, p.qs[row]);
        }
    }
}

// ---------------------------------------------------------------- many rows
// A workgroup of WR x WT wavefronts owns 64 * WR packed channels x 16 * TB * WT rows of q; a wavefront 64 x 16 TB of them.
// K goes by in steps of 128: both operands' next step is loaded straight into LDS while the present one is multiplied.
// Weights lie in LDS as in memory (a wavefront's operand is 1 KiB of adjacent bytes); a row's 128 bytes are 8 chunks of 16,
// chunk c stored at c ^ (row & 7), so that the 8 rows that an LDS cycle reads lie in 8 different places.
// Needs q 16-byte aligned in address, stride and width.  What lies past a row's end meets zero weights; past the tensor's
// end the buffer's bounds give zeros.
template <int WR, int WT, int TB> struct Tile {
    static constexpr int kWaves = WR * WT, kChannels = 64 * WR, kRows = 16 * TB * WT;
    static constexpr int kWBytes = WR * 8192, kQBytes = kRows * 128, kStage = kWBytes + kQBytes, kLds = 2 * kStage;
    static constexpr int kLoads = kStage / 1024 / kWaves;   // of 1 KiB, a wavefront and step
    static_assert(kStage % (1024 * kWaves) == 0, "every wavefront issues the same number of loads");
};

// 16 bytes a lane from memory to LDS at `lds` + 16 * lane.  In asm, so that the compiler does not put a wait for it in front of
// every read of LDS; the kernel waits for it itself.  (m0 is not one of the registers that the compiler hands out.)
__device__ inline void load_to_lds(__amdgpu_buffer_rsrc_t r, unsigned voff, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds), "v"(voff), "s"(r) : "memory");
}

template <int WR, int WT, int TB, bool GATED, bool BF16>
__global__ __launch_bounds__(WR * WT * 64) void q8_tile_kernel(Q8Linear p, int tiles_c, int tiles_r)
{
    using T = Tile<WR, WT, TB>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wr = wave % WR, wt = wave / WR;
    const int tc = blockIdx.x % tiles_c, tr = blockIdx.x / tiles_c;
    const int g0 = tc * WR;
    const int64_t row0 = (int64_t)tr * T::kRows;
    const int nrow = (int)(p.rows - row0 < T::kRows ? p.rows - row0 : T::kRows);
    const int ngrp = p.groups - g0 < WR ? p.groups - g0 : WR;
    const __amdgpu_buffer_rsrc_t wsr = q8_rsrc(p.w + (size_t)g0 * p.kblocks * 4096, (unsigned)ngrp * p.kblocks * 4096);
    const __amdgpu_buffer_rsrc_t qsr = q8_rsrc(p.q + row0 * p.ldq, (unsigned)((nrow - 1) * p.ldq + p.width));
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_ptr_t)smem;
    unsigned voff[T::kLoads];
#pragma unroll
    for (int i = 0; i < T::kLoads; ++i) {
        const int c = wave + i * T::kWaves;   // 1 KiB of the stage
        if (c < T::kWBytes / 1024) {
            voff[i] = (unsigned)(c >> 3) * p.kblocks * 4096 + (c & 7) * 1024 + lane * 16;
        } else {
            const int row = (c - T::kWBytes / 1024) * 8 + (lane >> 3);
            voff[i] = (unsigned)(row * p.ldq) + (((lane & 7) ^ (row & 7)) << 4);
        }
    }
    auto fetch = [&](int stage) {
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) {
            const int c = wave + i * T::kWaves;
            const bool weights = c < T::kWBytes / 1024;
            load_to_lds(weights ? wsr : qsr, voff[i], lds0 + stage * T::kStage + c * 1024);
            voff[i] += weights ? 8192 : 128;
        }
    };
    i32x4 acc[TB][4] = {};
    const int steps = p.kblocks / 2;
    fetch(0);
    const int wlane = wr * 8192 + lane * 16;
    const int qlane = T::kWBytes + (wt * TB * 16 + (lane & 15)) * 128 + (((lane >> 4) ^ (lane & 7)) << 4);
    for (int k = 0; k < steps; ++k) {
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" : : : "memory");
        if (k + 1 < steps) fetch((k + 1) & 1);
        const char* st = smem + (k & 1) * T::kStage;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 wf[4], qf[TB];
#pragma unroll
            for (int b = 0; b < 4; ++b) wf[b] = *reinterpret_cast<const i32x4*>(st + wlane + h * 4096 + b * 1024);
#pragma unroll
            for (int j = 0; j < TB; ++j) qf[j] = *reinterpret_cast<const i32x4*>(st + (qlane ^ (h * 64)) + j * 2048);
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[j][b] = mma(wf[b], qf[j], acc[j][b]);
        }
    }
    if (g0 + wr >= p.groups) return;
    Channels<GATED, 4> ch;
    ch.load(p, g0 + wr, 0, lane);
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int64_t row = row0 + (wt * TB + j) * 16 + (lane & 15);
        if (row < p.rows) emit<GATED, BF16, 4>(p, ch, acc[j], row, p.qs[row]);
    }
}

// Rows copied to 16-byte aligned ones of `pitch` bytes (the bytes past a row's end are zero).
__global__ __launch_bounds__(256) void q8_align_kernel(const int8_t* q, int64_t ldq, int8_t* to, int pitch, int64_t rows, int width)
{
    const int units = pitch / 16;
    const int64_t total = rows * units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / units;
        const int c = (int)(i - row * units) * 16;
        const int8_t* src = q + row * ldq + c;
        i32x4 v = {0, 0, 0, 0};
        if (c + 16 <= width) {
            __builtin_memcpy(&v, src, 16);
        } else {
            for (int e = 0; c + e < width; ++e) {
                const int b = (int)(unsigned char)src[e] << (8 * (e & 3));
#pragma unroll
                for (int d = 0; d < 4; ++d) v[d] |= (e >> 2) == d ? b : 0;
            }
        }
        *reinterpret_cast<i32x4*>(to + row * pitch + c) = v;
    }
}

// ---------------------------------------------------------------- weights
// One 16-byte unit of the packed weights a thread.
__global__ __launch_bounds__(256) void q8_pack_kernel(const int8_t* w, int64_t ldw, const float* scales, int8_t* to, float* to_scales,
                                                      int channels, int width, int gated, int groups, int kblocks, int* bad)
{
    const int64_t total = (int64_t)groups * kblocks * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int lane = (int)(i & 63), b = (int)(i >> 6) & 3;
        const int64_t gk = i >> 8;
        const int kb = (int)(gk % kblocks), group = (int)(gk / kblocks);
        const int c = q8_row_of(group * 64 + b * 16 + (lane & 15), channels, gated);
        const int k = kb * 64 + (lane >> 4) * 16;
        i32x4 v = {0, 0, 0, 0};
        if (c >= 0 && k < width) {
            const int8_t* src = w + c * ldw + k;
            if (k + 16 <= width) {
                __builtin_memcpy(&v, src, 16);
            } else {
                for (int e = 0; k + e < width; ++e) {
                    const int byte = (int)(unsigned char)src[e] << (8 * (e & 3));
#pragma unroll
                    for (int d = 0; d < 4; ++d) v[d] |= (e >> 2) == d ? byte : 0;
                }
            }
        }
        *reinterpret_cast<i32x4*>(to + i * 16) = v;
        if (kb == 0 && (lane >> 4) == 0) {
            const float s = c >= 0 ? scales[c] : 0.0f;
            if (!(fabsf(s) < INFINITY)) atomicOr(bad, 1);
            to_scales[group * 64 + b * 16 + lane] = s;
        }
    }
}

__global__ __launch_bounds__(256) void q8_unpack_kernel(const int8_t* from, const float* from_scales, int8_t* w, float* scales, int channels,
                                                        int width, int gated, int groups, int kblocks)
{
    const int64_t total = (int64_t)groups * kblocks * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int lane = (int)(i & 63), b = (int)(i >> 6) & 3;
        const int64_t gk = i >> 8;
        const int kb = (int)(gk % kblocks), group = (int)(gk / kblocks);
        const int c = q8_row_of(group * 64 + b * 16 + (lane & 15), channels, gated);
        const int k = kb * 64 + (lane >> 4) * 16;
        if (c < 0) continue;
        for (int e = 0; e < 16 && k + e < width; ++e) w[(int64_t)c * width + k + e] = from[i * 16 + e];
        if (kb == 0 && (lane >> 4) == 0) scales[c] = from_scales[group * 64 + b * 16 + lane];
    }
}

__global__ void q8_clear_kernel(int* p) { *p = 0; }

// ---------------------------------------------------------------- launches
constexpr int kFewRows = 64;

inline bool aligned16(const Q8Linear& p) { return (uintptr_t)p.q % 16 == 0 && p.ldq % 16 == 0 && p.width % 16 == 0; }
inline int padded(int width) { return (width + 127) / 128 * 128; }

template <int TB, int RB, int NW, bool GATED, bool BF16>
int launch_few(const Q8Linear& p, hipStream_t s)
{
    const dim3 grid((unsigned)(p.groups * 4 / RB), (unsigned)((p.rows + 16 * TB - 1) / (16 * TB)));
    hipLaunchKernelGGL((q8_few_kernel<TB, RB, NW, GATED, BF16>), grid, dim3(NW * 64), 0, s, p);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

template <int WR, int WT, int TB, bool GATED, bool BF16>
int launch_tile(const Q8Linear& p, hipStream_t s)
{
    using T = Tile<WR, WT, TB>;
    static unsigned long long done = 0;
    const int rc = allow_lds((const void*)q8_tile_kernel<WR, WT, TB, GATED, BF16>, T::kLds, &done);
    if (rc != NM_OK) return rc;
    const int tiles_c = (p.groups + WR - 1) / WR, tiles_r = (int)(((int64_t)p.rows + T::kRows - 1) / T::kRows);
    hipLaunchKernelGGL((q8_tile_kernel<WR, WT, TB, GATED, BF16>), dim3((unsigned)tiles_c * tiles_r), dim3(T::kWaves * 64), T::kLds, s, p,
                       tiles_c, tiles_r);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

template <bool GATED, bool BF16>
int pick_linear(const Q8Linear& p, hipStream_t s)
{
    if (p.rows <= 16) return launch_few<1, 1, 8, GATED, BF16>(p, s);
    if (p.rows <= 32) return launch_few<2, 1, 8, GATED, BF16>(p, s);
    if (p.rows <= kFewRows) return launch_few<4, 1, 8, GATED, BF16>(p, s);
    const int64_t big = (int64_t)((p.groups + 3) / 4) * ((p.rows + 255) / 256);
    if (big >= 192) return launch_tile<4, 2, 8, GATED, BF16>(p, s);
    return launch_tile<2, 2, 4, GATED, BF16>(p, s);
}

}  // namespace

size_t q8_linear_workspace(const Q8Linear& p)
{
    if (p.rows <= kFewRows || aligned16(p)) return 0;
    return (size_t)p.rows * padded(p.width);
}

int run_q8_linear(const Q8Linear& call, void* workspace, hipStream_t s)
{
    Q8Linear p = call;
    if (q8_linear_workspace(p)) {
        const int pitch = padded(p.width);
        const int64_t blocks = ((int64_t)p.rows * (pitch / 16) + 255) / 256;
        hipLaunchKernelGGL(q8_align_kernel, dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), dim3(256), 0, s, p.q, p.ldq,
                           (int8_t*)workspace, pitch, (int64_t)p.rows, p.width);
        NM_HIP_CHECK(hipGetLastError());
        p.q = (const int8_t*)workspace;
        p.ldq = pitch;
        p.width = pitch;
    }
    if (p.gated) return p.y_bf16 ? pick_linear<true, true>(p, s) : pick_linear<true, false>(p, s);
    return p.y_bf16 ? pick_linear<false, true>(p, s) : pick_linear<false, false>(p, s);
}

int run_q8_pack(const int8_t* w, int64_t ldw, const float* scales, const nm_q8* h, int* d_bad, hipStream_t s)
{
    hipLaunchKernelGGL(q8_clear_kernel, dim3(1), dim3(1), 0, s, d_bad);
    NM_HIP_CHECK(hipGetLastError());
    const int64_t blocks = (int64_t)h->groups * h->kblocks;
    hipLaunchKernelGGL(q8_pack_kernel, dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), dim3(256), 0, s, w, ldw, scales, h->d_w,
                       h->d_scales, h->channels, h->width, h->gated, h->groups, h->kblocks, d_bad);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

int run_q8_unpack(const nm_q8* h, int8_t* w, float* scales, hipStream_t s)
{
    const int64_t blocks = (int64_t)h->groups * h->kblocks;
    hipLaunchKernelGGL(q8_unpack_kernel, dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), dim3(256), 0, s, h->d_w, h->d_scales, w,
                       scales, h->channels, h->width, h->gated, h->groups, h->kblocks);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

}  // namespace nm
