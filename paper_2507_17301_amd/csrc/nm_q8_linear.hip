// Product of 8-bit rows with 8-bit weights, a scale for each row and each channel.
//
//   y[r][c] = (sum_k q[r][k] * w[c][k]) * (s[r] * t[c]) + bias[c] (+ residual[r][c]),  or  silu(gate) * up
//
// The sum is in 32-bit integers and exact, so no split of K changes a result.  Weights are the first operand of the
// 16x16x64 integer matrix instruction, rows of q the second: lane l of a wavefront then holds packed weight rows
// 4 (l / 16) .. + 3 of a 16-row block for row l % 16 of q, and the packing deals channels so that the four blocks of
// a 64-row group give it twice 8 adjacent channels (gated: 8 adjacent outputs, gate and value in the same registers).
// (The 32x32x32 form is as fast on zeros, 4.9 POP/s out of registers, but takes more power: 3.4 POP/s on normally distributed
// values, this one 4.0.)
#include "nm_q8_product.h"

namespace nm {
namespace {

// ---------------------------------------------------------------- few rows
// Up to 16 * TB rows of q.  A workgroup owns RB blocks of 16 packed channels; its NW wavefronts take the steps of 128 k in turn,
// U of them in flight each, and add their sums through LDS at the end.  Weights go from memory into registers: a weight is used
// once, there is nothing to share.  Rows of q go through LDS, a part of it for each wavefront, so that 8 lanes read the 128
// adjacent bytes of a row: read straight into operand registers, 16 rows with 64 bytes each an instruction, they come at a third
// of the rate (38 instead of 120 bytes a ns and CU out of the L2), and 64 rows x 4096 x 4096 took 11.4 us instead of 8.7.
// Bound by the weights' bytes: 16 rows x 4096 -> 24576 in 19 us, 5.3 TB/s of them (pick_few has more).
template <int TB, int RB, int NW, int U> constexpr int few_lds()
{
    const int rows = NW * U * TB * 2048, sums = NW * RB * TB * 1024;
    return rows > sums ? rows : sums;
}

template <int TB, int RB, int NW, int U, bool GATED, bool BF16>
__global__ __launch_bounds__(NW * 64) void q8_few_kernel(Q8Linear p)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int b0 = blockIdx.x * RB;   // (RB divides 4: a workgroup stays within its row group)
    const __amdgpu_buffer_rsrc_t wsr = q8_rsrc(p.w + (size_t)(b0 >> 2) * p.kblocks * 4096, (unsigned)p.kblocks * 4096);
    const __amdgpu_buffer_rsrc_t qsr = q8_rsrc(p.q, rows_extent(p, p.rows));
    const unsigned woff = (b0 & 3) * 1024 + lane * 16;
    const unsigned mine = wave * (U * TB * 2048), lds0 = (unsigned)(uintptr_t)(lds_ptr_t)smem + mine;
    const unsigned from = mine + (lane & 15) * 128 + (((lane >> 4) ^ (lane & 7)) << 4);
    unsigned qoff[TB][2];   // 8 rows an instruction, chunk c of a row at c ^ (row & 7)
    bool there[TB][2];
#pragma unroll
    for (int i = 0; i < TB; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = i * 16 + h * 8 + (lane >> 3);
            there[i][h] = row < p.rows;
            qoff[i][h] = (unsigned)(row * p.ldq) + (((lane & 7) ^ (lane >> 3)) << 4);
        }
    i32x4 acc[RB][TB] = {};
    const int steps = p.kblocks / 2;
    for (int k0 = wave; k0 < steps; k0 += NW * U) {
        i32x4 wf[U][2][RB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u * NW;
            const bool in = k < steps;   // past the last step nothing is read and zeros are multiplied
#pragma unroll
            for (int i = 0; i < TB; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    load_to_lds(qsr, in && there[i][h] ? qoff[i][h] + k * 128 : kPast, lds0 + u * TB * 2048 + i * 2048 + h * 1024);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < RB; ++i)   // (nontemporal: no other workgroup reads them; 8 % faster)
                    wf[u][h][i] = __builtin_bit_cast(
                        i32x4, __builtin_amdgcn_raw_buffer_load_b128(wsr, in ? woff + i * 1024 + (k * 2 + h) * 4096 : kPast, 0, 2));
        }
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                i32x4 qf[TB];
#pragma unroll
                for (int j = 0; j < TB; ++j) qf[j] = *reinterpret_cast<const i32x4*>(smem + (from ^ (h * 64)) + u * TB * 2048 + j * 2048);
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int j = 0; j < TB; ++j) acc[i][j] = mma(wf[u][h][i], qf[j], acc[i][j]);
            }
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // read, before the next loads land there
    }
    __syncthreads();
    i32x4* part = reinterpret_cast<i32x4*>(smem);   // [NW][RB * TB][64]
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) part[(wave * RB * TB + i * TB + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int u = wave; u < RB * TB; u += NW) {
        const int i = u / TB, j = u % TB, rb = b0 + i;
        const int row = j * 16 + (lane & 15);
        if (row < p.rows) {
            Channels<GATED, 1> ch;
            ch.load(p, rb >> 2, rb & 3, lane);
            const float s = p.qs[row];
            i32x4 sum[1] = {part[u * 64 + lane]};
#pragma unroll
            for (int n = 1; n < NW; ++n) sum[0] += part[(n * RB * TB + u) * 64 + lane];
            emit<GATED, BF16, 1>(p, ch, sum, row, s);
        }
    }
}

// ---------------------------------------------------------------- many rows
// A workgroup of WR x WT wavefronts owns 64 * WR packed channels x 16 * TB * WT rows of q; a wavefront 64 x 16 TB of them.
// K goes by in steps of 128.  LDS holds NSW steps' weights and NSQ steps' rows, loaded straight into it: while a step is multiplied, the
// next one's lie there and later ones' are on their way.  Operands are read from LDS half a step ahead, into the other half of
// the operand registers, so one barrier a step is enough.  Three stages of each where they fit a CU's LDS; where they do not, two of
// the rows and three of the weights (8192 x 4096 -> 16384 with two of each 1.6 % slower, with a third of the rows 0.5 %).
// Bound by the power limit on large products, and by the starts and ends of their rounds: 8192 x 4096 -> 16384 takes 422 us, 2.6 POP/s (405 to
// 450 by the card), at 1.87 GHz with the matrix units busy 64 % of the cycles.  The 256 x 256 loop without any load or barrier takes 1.16 us a
// step on such values (0.91 on zeros, 0.85 at 2.4 GHz by the instruction's 16 cycles), with them 1.38 (0.98): 32 steps of 8 rounds are
// 353 us of it.  The rest is what 8 rounds take to fill the first stages and to store, with one workgroup a CU and nothing beside it.
// Weights lie in LDS as in memory (a wavefront's operand is 1 KiB of adjacent bytes); a row's 128 bytes are 8 chunks of 16,
// chunk c stored at c ^ (row & 7), so that the 8 rows that an LDS cycle reads lie in 8 different places.
// SPLIT: a workgroup takes `per` of the K steps and stores its integer sums as they lie in the registers,
//   part[split][tile][wave][16-row block][4 blocks][64 lanes], for q8_join_kernel to add and scale.
template <int WR, int WT, int TB, int NSW, int NSQ> struct Tile {
    static constexpr int kWaves = WR * WT, kRows = 16 * TB * WT;
    static constexpr int kWBytes = WR * 8192, kQBytes = kRows * 128, kQAt = NSW * kWBytes, kLds = kQAt + NSQ * kQBytes;
    static constexpr int kWLoads = kWBytes / 1024 / kWaves, kQLoads = kQBytes / 1024 / kWaves;   // of 1 KiB, a wavefront and step
    static_assert(kWBytes % (1024 * kWaves) == 0 && kQBytes % (1024 * kWaves) == 0, "every wavefront issues the same loads");
    // Loads that may be out while a step waits for the stages of the next: those of later steps.  The operand with fewer stages is
    // loaded first, so the other's stage that goes with it may be out too.
    static constexpr int kFew = NSW < NSQ ? NSW : NSQ;
    static constexpr int kOut = (kFew - 2) * (kWLoads + kQLoads) + (NSW < NSQ ? kQLoads : NSQ < NSW ? kWLoads : 0);
};

constexpr int largest_divisor(int n, int most) { return most >= n ? n : n % most == 0 ? most : largest_divisor(n, most - 1); }

template <int WR, int WT, int TB, int NSW, int NSQ, bool SPLIT, bool GATED, bool BF16>
__global__ __launch_bounds__(WR * WT * 64) void q8_tile_kernel(Q8Linear p, TileOrder order, int per, i32x4* part)
{
    using T = Tile<WR, WT, TB, NSW, NSQ>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wr = wave % WR, wt = wave / WR;
    int tc, tr, tile, split;
    order.at(blockIdx.x, tc, tr, tile, split);
    const int g0 = tc * WR;
    const int64_t row0 = (int64_t)tr * T::kRows;
    const int nrow = (int)(p.rows - row0 < T::kRows ? p.rows - row0 : T::kRows);
    const int ngrp = p.groups - g0 < WR ? p.groups - g0 : WR;
    const int first = SPLIT ? split * per : 0;
    const int steps = SPLIT ? (p.kblocks / 2 - first < per ? p.kblocks / 2 - first : per) : p.kblocks / 2;
    const __amdgpu_buffer_rsrc_t wsr = q8_rsrc(p.w + (size_t)g0 * p.kblocks * 4096, (unsigned)ngrp * p.kblocks * 4096);
    const __amdgpu_buffer_rsrc_t qsr = q8_rsrc(p.q + row0 * p.ldq, rows_extent(p, nrow));
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_ptr_t)smem;
    unsigned wvoff[T::kWLoads], qvoff[T::kQLoads];
#pragma unroll
    for (int i = 0; i < T::kWLoads; ++i) {
        const int c = wave + i * T::kWaves;   // 1 KiB of the stage
        wvoff[i] = ((unsigned)(c >> 3) * p.kblocks + first * 2) * 4096 + (c & 7) * 1024 + lane * 16;
    }
#pragma unroll
    for (int i = 0; i < T::kQLoads; ++i) {
        const int row = (wave + i * T::kWaves) * 8 + (lane >> 3);
        qvoff[i] = (unsigned)(row * p.ldq) + first * 128 + (((lane & 7) ^ (row & 7)) << 4);
    }
    // load i of a step's stages, weights at `wat`, rows at `qat`; past the last step nothing is read, so that the count of loads holds
    constexpr bool WFIRST = NSW <= NSQ;
    auto fetch = [&](int i, unsigned wat, bool wthere, unsigned qat, bool qthere) {
        if (WFIRST ? i < T::kWLoads : i >= T::kQLoads) {
            const int n = WFIRST ? i : i - T::kQLoads;
            load_to_lds(wsr, wthere ? wvoff[n] : kPast, lds0 + wat + (wave + n * T::kWaves) * 1024);
            wvoff[n] += 8192;
        } else {
            const int n = WFIRST ? i - T::kWLoads : i;
            load_to_lds(qsr, qthere ? qvoff[n] : kPast, lds0 + T::kQAt + qat + (wave + n * T::kWaves) * 1024);
            qvoff[n] += 128;
        }
    };
    const int wlane = wr * 8192 + lane * 16;
    const int qlane = T::kQAt + (wt * TB * 16 + (lane & 15)) * 128 + (((lane >> 4) ^ (lane & 7)) << 4);
    i32x4 f[2][4 + TB];   // operands of the two halves of a step: 4 blocks of weights, TB of rows
    auto read = [&](int h, int i, unsigned wat, unsigned qat) {
        f[h][i] = *reinterpret_cast<const i32x4*>(smem + (i < 4 ? wat + wlane + h * 4096 + i * 1024 : qat + (qlane ^ (h * 64)) + (i - 4) * 2048));
    };
    constexpr bool EARLY = !SPLIT && TB < 8;   // the scales come with the first stages where the registers last for it
    Channels<GATED, 4> ch;
    const int group = g0 + wr < p.groups ? g0 + wr : p.groups - 1;   // (what a wavefront past the last group has is not stored)
    float early[EARLY ? TB : 1];
    auto scale_of = [&](int j) {
        const int64_t row = row0 + (wt * TB + j) * 16 + (lane & 15);
        return row < p.rows ? p.qs[row] : 0.0f;
    };
    if constexpr (EARLY) {
        ch.load(p, group, 0, lane);
#pragma unroll
        for (int j = 0; j < TB; ++j) early[j] = scale_of(j);
    }
    auto scale = [&](int j) {
        if constexpr (EARLY) return early[j];
        else return scale_of(j);
    };
    i32x4 acc[TB][4] = {};
    constexpr int LOADS = T::kWLoads + T::kQLoads, FEW = T::kFew, MORE = NSW + NSQ - FEW;
#pragma unroll
    for (int s = 0; s < FEW; ++s)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) fetch(i, s * T::kWBytes, s < steps, s * T::kQBytes, s < steps);
#pragma unroll
    for (int s = FEW; s < MORE; ++s)   // the operand with more stages: the second part of a step's loads
#pragma unroll
        for (int i = WFIRST ? T::kWLoads : T::kQLoads; i < LOADS; ++i) fetch(i, s * T::kWBytes, s < steps, s * T::kQBytes, s < steps);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((FEW - 1) * LOADS + (MORE - FEW) * (WFIRST ? T::kQLoads : T::kWLoads)) : "memory");
#pragma unroll
    for (int i = 0; i < 4 + TB; ++i) read(0, i, 0, 0);
    unsigned wnow = 0, qnow = 0;   // the stages that are multiplied
    for (int k = 0; k < steps; ++k) {
        const unsigned wnext = wnow + T::kWBytes == NSW * T::kWBytes ? 0 : wnow + T::kWBytes;
        const unsigned qnext = qnow + T::kQBytes == NSQ * T::kQBytes ? 0 : qnow + T::kQBytes;
        // first half: its operands are in registers; the second half's are read meanwhile
#pragma unroll
        for (int j = 0; j < TB; ++j) {
#pragma unroll
            for (int i = j * (4 + TB) / TB; i < (j + 1) * (4 + TB) / TB; ++i) read(1, i, wnow, qnow);
#pragma unroll
            for (int b = 0; b < 4; ++b) acc[j][b] = mma(f[0][b], f[0][4 + j], acc[j][b]);
            __builtin_amdgcn_sched_barrier(0);
        }
        // these stages have been read, the next ones have landed
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(T::kOut) : "memory");
        // second half: the next step's first operands are read, and what comes after the last stages in LDS is loaded in these ones' place
#pragma unroll
        for (int j = 0; j < TB; ++j) {
#pragma unroll
            for (int i = j * (4 + TB) / TB; i < (j + 1) * (4 + TB) / TB; ++i) read(0, i, wnext, qnext);
#pragma unroll
            for (int i = j * LOADS / TB; i < (j + 1) * LOADS / TB; ++i) fetch(i, wnow, k + NSW < steps, qnow, k + NSQ < steps);
#pragma unroll
            for (int b = 0; b < 4; ++b) acc[j][b] = mma(f[1][b], f[1][4 + j], acc[j][b]);
            __builtin_amdgcn_sched_barrier(0);
        }
        wnow = wnext;
        qnow = qnext;
    }
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");   // no load into LDS outlives the workgroup
    if constexpr (SPLIT) {
        if (g0 + wr >= p.groups) return;
        i32x4* to = part + ((size_t)((size_t)split * order.tiles() + tile) * T::kWaves + wave) * TB * 256 + lane;
#pragma unroll
        for (int j = 0; j < TB; ++j)
            if (wt * TB * 16 + j * 16 < nrow)
#pragma unroll
                for (int b = 0; b < 4; ++b) to[(j * 4 + b) * 64] = acc[j][b];
    } else {
        if constexpr (!EARLY) ch.load(p, group, 0, lane);
        constexpr int kFit = T::kLds / (16 * WT * 64 * WR * 4 / (GATED ? 2 : 1));   // blocks of rows that fit LDS in fp32
        constexpr int JP4 = largest_divisor(TB, kFit), JP2 = largest_divisor(TB, 2 * kFit);
        static_assert(kFit >= 1, "the tile's outputs go through LDS");
        if (!BF16 || p.res) store_tile<WR, WT, TB, JP4, true, GATED, BF16>(p, ch, scale, acc, smem, wr, wt, lane, g0, row0);
        else store_tile<WR, WT, TB, JP2, false, GATED, BF16>(p, ch, scale, acc, smem, wr, wt, lane, g0, row0);
    }
}

// Adds the sums of a tile's parts and stores the results: a wavefront takes 16 rows x 64 packed channels, so that few tiles still
// make many wavefronts.  Bound by the parts' bytes, which the last-level cache holds: 128 x 12288 -> 4096 in 4 to 8 parts takes
// 21 to 23 us with it, 58 undivided.
template <int WR, int WT, int TB, int NSW, int NSQ, bool GATED, bool BF16>
__global__ __launch_bounds__(256) void q8_join_kernel(Q8Linear p, TileOrder order, const i32x4* part)
{
    using T = Tile<WR, WT, TB, NSW, NSQ>;
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = (int)(unit / (T::kWaves * TB)), wave = (int)(unit / TB) % T::kWaves, j = (int)(unit % TB);
    int tc, tr;
    order.place(tile, tc, tr);
    const int group = tc * WR + wave % WR;
    const int64_t row = (int64_t)tr * T::kRows + ((wave / WR) * TB + j) * 16 + (lane & 15);
    if (group >= p.groups || row >= p.rows) return;
    const i32x4* from = part + (((size_t)tile * T::kWaves + wave) * TB + j) * 256 + lane;
    const size_t next = (size_t)order.tiles() * T::kWaves * TB * 256;
    Channels<GATED, 4> ch;
    ch.load(p, group, 0, lane);
    const float s = p.qs[row];
    i32x4 acc[4] = {};
#pragma unroll 4
    for (int i = 0; i < order.splits; ++i)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[b] += from[i * next + b * 64];
    emit<GATED, BF16, 4>(p, ch, acc, row, s);
}

// Rows copied to ones at a stride of `pitch` bytes, a multiple of 16 (the bytes past a row's end are zero).  333 x 1037: 2.7 us, the
// time of a small launch.
__global__ __launch_bounds__(256) void q8_align_kernel(const int8_t* q, int64_t ldq, int8_t* to, int pitch, int rows, int width)
{
    const int c = (blockIdx.x * 256 + threadIdx.x) * 16;
    if (c >= pitch) return;
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y)
        *reinterpret_cast<i32x4*>(to + row * pitch + c) = load16(q + row * ldq, c, width);
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
        *reinterpret_cast<i32x4*>(to + i * 16) = load16(w + (int64_t)(c < 0 ? 0 : c) * ldw, k, c < 0 ? 0 : width);
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
constexpr int kFewRows = NM_Q8_FEW_ROWS;

// Whether the kernels can read q where it lies.
inline bool aligned16(const Q8Linear& p) { return (uintptr_t)p.q % 16 == 0 && (p.rows == 1 || p.ldq % 16 == 0); }

template <int TB, int RB, int NW, int U, bool GATED, bool BF16>
int launch_few(const Q8Linear& p, hipStream_t s)
{
    constexpr int LDS = few_lds<TB, RB, NW, U>();
    static_assert(LDS <= 64 * 1024, "more needs allow_lds");
    hipLaunchKernelGGL((q8_few_kernel<TB, RB, NW, U, GATED, BF16>), dim3((unsigned)(p.groups * 4 / RB)), dim3(NW * 64), LDS, s, p);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

// More channels a workgroup read q less often, fewer make more workgroups: 256 of them at 4096 and at 8192 channels, 192 at 12288, one a CU;
// fewer than 4096 channels leave CUs without one (K is not divided over workgroups here).  us at width 4096, one row,
// 16, 32, 64 rows, with 1 / 2 / 4 blocks of channels a workgroup:
//    4096 channels   5.7 / 5.8 /  7.8    5.7 / 6.5 /  8.5     6.5 /  7.8 / 10.1     8.7 / 10.0 / 12.9
//    8192            8.8 / 8.8 /  8.4    8.9 / 8.8 /  8.9    10.4 /  9.3 / 10.4    14.7 / 10.8 / 13.3
//   12288           11.4 / 11.2 / 10.0  12.0 / 12.0 / 10.2   14.8 / 13.7 / 11.5    20.4 / 17.7 / 14.3
//   24576           20.0 / 19.4 / 17.9  22.1 / 19.6 / 18.6   27.8 / 21.3 / 20.1    38.5 / 26.5 / 24.2
// (16.8, 33.6, 50.3 and 100.7 MB of weights, out of HBM.)
template <int TB, bool GATED, bool BF16>
int pick_few(const Q8Linear& p, hipStream_t s)
{
    constexpr int U = TB == 4 ? 1 : 2;
    if (p.groups >= 192) return launch_few<TB, 4, 4, U, GATED, BF16>(p, s);
    if (p.groups >= 128) return launch_few<TB, 2, 8, U, GATED, BF16>(p, s);
    return launch_few<TB, 1, 8, U, GATED, BF16>(p, s);
}

// The tile kernels' shapes.  More rows or channels a workgroup take less from the L2 for a product; few of either leave CUs without
// work or tiles half empty: over 400 products the best of these seven was 8 % faster than the best of 256 x 256, 128 x 128 and
// 128 x 64 (300 x 4096 -> 2 x 8192 35 -> 28 us, 700 x 4096 -> 2 x 12288 97 -> 76, 2048 x 12288 -> 4096 96 -> 85); leaving any one out
// costs 0.5 to 2 %, and 256 x 64, 128 x 256, 128 x 96 and 128 x 128 twice a CU would add 0.3 % together.
struct Shape {
    int waves, wr, rows, tb;
    int per_cu;                  // workgroups that a CU holds (by LDS)
    float fixed, step, more;     // us: of a round; of a K step; what that takes more where all CUs are full, by the share that is
};
constexpr Shape kShapes[] = {{8, 4, 256, 8, 1, 10.4f, 0.87f, 0.54f},    // 256 channels x 256 rows
                             {8, 4, 192, 6, 1, 7.9f, 0.71f, 0.36f},
                             {8, 4, 128, 4, 1, 7.2f, 0.58f, 0.20f},
                             {4, 2, 192, 6, 1, 5.6f, 0.48f, 0.21f},     // 128 channels
                             {4, 2, 160, 5, 1, 5.6f, 0.38f, 0.20f},
                             {4, 2, 128, 4, 1, 5.7f, 0.32f, 0.20f},
                             {2, 2, 64, 4, 2, 6.0f, 0.18f, 0.46f}};
inline TileOrder order_of(const Q8Linear& p, int shape, int splits)
{
    TileOrder o;
    o.splits = splits;
    o.tiles_c = (p.groups + kShapes[shape].wr - 1) / kShapes[shape].wr;
    o.tiles_r = (int)(((int64_t)p.rows + kShapes[shape].rows - 1) / kShapes[shape].rows);
    return o;
}

// The shape and split with the least estimated time: rounds of workgroups over the 256 CUs, each a fixed part and its K steps; for a
// split the second kernel and its traffic.  The figures are fitted to timings of 65 to 8192 rows on 300 to 24576 channels of 512 to
// 16000 values; of 400 such products the choice was within 5 % of the best of all shapes and splits for 365, within 19 % for all.
Q8Plan plan_linear(const Q8Linear& p)
{
    Q8Plan best;
    if (p.rows <= kFewRows) return best;
    const int steps = p.kblocks / 2;
    const float from_memory = ((float)p.groups * p.kblocks * 4096 + (float)p.rows * p.width) / 7.8e6f;   // us that the operands take at least
    float least = 1e30f;
    for (int sh = 0; sh < (int)(sizeof(kShapes) / sizeof(Shape)); ++sh) {
        const Shape& k = kShapes[sh];
        const TileOrder o = order_of(p, sh, 1);
        const int64_t tiles = (int64_t)o.tiles_c * o.tiles_r, room = 256 * k.per_cu;
        for (int splits = 1; splits <= 16; ++splits) {
            const int per = (steps + splits - 1) / splits;
            if (splits > 1 && (tiles * splits > 512 || per < 3)) break;
            if ((splits - 1) * per >= steps) continue;   // (an empty part)
            const int64_t rounds = tiles * splits / room, rest = tiles * splits % room;
            float us = rounds * per * (k.step + k.more);
            if (rest) us += per * (k.step + k.more * rest / room);
            us = (rounds + (rest > 0)) * k.fixed + (us > from_memory ? us : from_memory);
            if (splits > 1) us += 2.5f + splits * (0.09f + 0.8e-6f * p.rows * p.groups * 64);   // (a fifth of a us for a MB of parts)
            if (us < least) {
                least = us;
                best.shape = sh;
                best.splits = splits;
                best.per = per;
            }
        }
    }
    return best;
}

inline size_t part_bytes(const Q8Linear& p, const Q8Plan& pl)
{
    const TileOrder o = order_of(p, pl.shape, pl.splits);
    return (size_t)pl.splits * o.tiles() * kShapes[pl.shape].waves * kShapes[pl.shape].tb * 4096;
}

template <int SHAPE, int WT, int NSW, int NSQ, bool GATED, bool BF16>
int launch_tile(const Q8Linear& p, const Q8Plan& pl, void* part, hipStream_t s)
{
    constexpr int WR = kShapes[SHAPE].wr, TB = kShapes[SHAPE].tb;
    using T = Tile<WR, WT, TB, NSW, NSQ>;
    static_assert(T::kWaves == kShapes[SHAPE].waves && T::kRows == kShapes[SHAPE].rows, "kShapes describes the kernels");
    const TileOrder o = order_of(p, SHAPE, pl.splits);
    const dim3 grid((unsigned)o.tiles() * pl.splits);
    if (pl.splits == 1) {
        static unsigned long long done = 0;
        const int rc = allow_lds((const void*)q8_tile_kernel<WR, WT, TB, NSW, NSQ, false, GATED, BF16>, T::kLds, &done);
        if (rc != NM_OK) return rc;
        hipLaunchKernelGGL((q8_tile_kernel<WR, WT, TB, NSW, NSQ, false, GATED, BF16>), grid, dim3(T::kWaves * 64), T::kLds, s, p, o, 0, (i32x4*)nullptr);
        NM_HIP_CHECK(hipGetLastError());
        return NM_OK;
    }
    static unsigned long long done = 0;
    const int rc = allow_lds((const void*)q8_tile_kernel<WR, WT, TB, NSW, NSQ, true, false, false>, T::kLds, &done);
    if (rc != NM_OK) return rc;
    hipLaunchKernelGGL((q8_tile_kernel<WR, WT, TB, NSW, NSQ, true, false, false>), grid, dim3(T::kWaves * 64), T::kLds, s, p, o, pl.per, (i32x4*)part);
    NM_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL((q8_join_kernel<WR, WT, TB, NSW, NSQ, GATED, BF16>), dim3((unsigned)o.tiles() * T::kWaves * TB / 4), dim3(256), 0, s, p, o,
                       (const i32x4*)part);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

template <bool GATED, bool BF16>
int pick_linear(const Q8Linear& p, const Q8Plan& pl, void* part, hipStream_t s)
{
    switch (pl.shape) {
    case 0: return launch_tile<0, 2, 3, 2, GATED, BF16>(p, pl, part, s);
    case 1: return launch_tile<1, 2, 3, 2, GATED, BF16>(p, pl, part, s);
    case 2: return launch_tile<2, 2, 3, 3, GATED, BF16>(p, pl, part, s);
    case 3: return launch_tile<3, 2, 3, 3, GATED, BF16>(p, pl, part, s);
    case 4: return launch_tile<4, 2, 3, 3, GATED, BF16>(p, pl, part, s);
    case 5: return launch_tile<5, 2, 3, 3, GATED, BF16>(p, pl, part, s);
    case 6: return launch_tile<6, 1, 3, 3, GATED, BF16>(p, pl, part, s);
    default: break;
    }
    if (p.rows <= 16) return pick_few<1, GATED, BF16>(p, s);
    if (p.rows <= 32) return pick_few<2, GATED, BF16>(p, s);
    return pick_few<4, GATED, BF16>(p, s);
}

}  // namespace

Q8Plan q8_plan(const Q8Linear& p)
{
    Q8Plan pl = plan_linear(p);
    if (!aligned16(p)) pl.rows_bytes = (size_t)p.rows * ((p.width + 15) / 16 * 16);
    if (pl.splits > 1) pl.part_bytes = part_bytes(p, pl);
    return pl;
}

int run_q8_linear(const Q8Linear& call, const Q8Plan& pl, void* workspace, hipStream_t s)
{
    Q8Linear p = call;
    if (pl.rows_bytes) {
        const int pitch = (p.width + 15) / 16 * 16;
        const dim3 grid((unsigned)(pitch / 16 + 255) / 256, (unsigned)(p.rows < 4096 ? p.rows : 4096));
        hipLaunchKernelGGL(q8_align_kernel, grid, dim3(256), 0, s, p.q, p.ldq, (int8_t*)workspace, pitch, p.rows, p.width);
        NM_HIP_CHECK(hipGetLastError());
        p.q = (const int8_t*)workspace;
        p.ldq = pitch;
    }
    void* part = (char*)workspace + pl.rows_bytes;
    if (p.gated) return p.y_bf16 ? pick_linear<true, true>(p, pl, part, s) : pick_linear<true, false>(p, pl, part, s);
    return p.y_bf16 ? pick_linear<false, true>(p, pl, part, s) : pick_linear<false, false>(p, pl, part, s);
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
