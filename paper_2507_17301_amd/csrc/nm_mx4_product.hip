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
    const unsigned woff = (b0 & 3) * 1024 + lane * 16, soff = lane * 4;
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
        unsigned wsc[U][2], xsc[U][TB];
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
            for (int h = 0; h < 2; ++h) wsc[u][h] = __builtin_amdgcn_raw_buffer_load_b32(ssr, in ? soff + (k * 2 + h) * 256 : kPast, 0, 0);
#pragma unroll
            for (int i = 0; i < TB; ++i) xsc[u][i] = row_scales(p, from.s, source[i], k * 8 + (lane >> 4));
        }
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
#pragma unroll
        for (int u = 0; u < U; ++u) {
            auto half = [&](auto hh) {
                constexpr int h = decltype(hh)::value;
                i32x4 xf[TB];
#pragma unroll
                for (int j = 0; j < TB; ++j)
                    xf[j] = *reinterpret_cast<const i32x4*>(smem + at + u * TB * 2048 + j * 2048 + (((4 * h + (lane >> 4)) ^ (lane & 7)) << 4));
                const unsigned ws = RB == 4 ? wsc[u][h] : wsc[u][h] >> (8 * (b0 & 3));
#pragma unroll
                for (int j = 0; j < TB; ++j) {
                    acc[0][j] = mma4<0, h>(wf[u][h][0], xf[j], acc[0][j], ws, xsc[u][j]);
                    if constexpr (RB >= 2) acc[1][j] = mma4<1, h>(wf[u][h][1], xf[j], acc[1][j], ws, xsc[u][j]);
                    if constexpr (RB == 4) {
                        acc[2][j] = mma4<2, h>(wf[u][h][2], xf[j], acc[2][j], ws, xsc[u][j]);
                        acc[3][j] = mma4<3, h>(wf[u][h][3], xf[j], acc[3][j], ws, xsc[u][j]);
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

// ---------------------------------------------------------------- many rows
// A workgroup of WR x WT wavefronts owns 64 * WR packed channels x 16 * TB * WT rows; a wavefront 64 x 16 TB of them.  K goes by in steps
// of 256, each two halves of one matrix instruction's 128.
// Rows go through LDS, NS steps of them, loaded straight into it: while a step is multiplied the next one's lie there and later ones' are on
// their way; a wavefront reads the operand of 16 rows three before it is multiplied.
// Weights go from memory into registers, three halves ahead: their layout in memory is the operands', and the wavefronts that share them read them
// at the same time.  Through LDS as well, LDS is what bounds the loop (192 + 68 KiB a step of 256 x 256, 2080 cycles at 128 bytes, beside
// 2048 of the matrix units).
// A row's 128 bytes are 8 blocks of 16, block c stored at c ^ (row & 7), so that what an LDS cycle reads lies in different banks.
template <int WR, int WT, int TB, int NS> struct Tile4 {
    static constexpr int kWaves = WR * WT, kRows = 16 * TB * WT;
    static constexpr int kXBytes = kRows * 128, kXLoads = kXBytes / 1024 / kWaves;              // of 1 KiB, a wavefront and step
    static constexpr int kSUnits = kRows / 32, kSLoads = (kSUnits + kWaves - 1) / kWaves;       // of 256 bytes: the rows' scales
    static constexpr int kStage = kXBytes + kSUnits * 256, kNowhere = NS * kStage, kLds = kNowhere + 256;   // (where loads of nothing land)
    static constexpr int kLoads = kXLoads + kSLoads;
    static_assert(TB % 4 == 0 && kXBytes % (1024 * kWaves) == 0, "every wavefront issues the same loads");
    static_assert(NS >= 3 && kLds <= 160 * 1024, "");
};

// The rows' scales of a tile and step as the kernel's lanes read them: [2 halves][rows / 64][64 lanes] words, byte j that of row block
// 4 (rows / 64) + j.
struct TileHead {
    int tiles, pad[3];   // of rows
};
struct TileRows {
    int expert, count;
    int64_t row0;
};

// 64 rows of a tile a workgroup.
__global__ __launch_bounds__(256) void mx4_scales_kernel(Mx4Product p, int per, TileHead* head, TileRows* tiles, unsigned* to)
{
    __shared__ int sources[64];
    const int parts = per / 64, tile = blockIdx.x / parts, part = blockIdx.x - tile * parts;   // (blockIdx.y: of the steps)
    int all = 0;
    const RowTile t = row_tile(p, tile, per, blockIdx.x == 0, &all);
    if (part == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
        tiles[tile] = {t.expert, t.count, t.row0};
        if (tile == 0) head->tiles = all;
    }
    if (t.count == 0) return;
    if (threadIdx.x < 64) sources[threadIdx.x] = source_of(p, t, part * 64 + threadIdx.x);
    __syncthreads();
    const int lane = threadIdx.x & 63;
    int src[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) src[j] = sources[j * 16 + (lane & 15)];
    const uint8_t* from = p.s + (p.index ? 0 : t.row0) * p.lds;
    unsigned* put = to + (int64_t)tile * p.steps * per * 2 + part * 64 + lane;
    for (int sh = blockIdx.y * 4 + (threadIdx.x >> 6); sh < p.steps * 2; sh += gridDim.y * 4) {   // step and half
        const int kb = sh * 4 + (lane >> 4);
        unsigned word = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            unsigned s = 127;   // past the row's blocks codes of 0 are multiplied
            if (src[j] == -2) s = 255;
            else if (src[j] >= 0 && kb < p.blocks) s = from[src[j] * p.lds + kb];
            word |= s << (8 * j);
        }
        put[(int64_t)sh * per] = word;
    }
}

// 4 bytes a lane from memory to LDS at `lds` + 4 * lane, as load_to_lds.
__device__ inline void load_to_lds4(__amdgpu_buffer_rsrc_t r, unsigned voff, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : :
                 "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voff), "s"(r));
}

// Values that are the same in all lanes, as the loads into LDS want them.
__device__ inline int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ inline TileRows tile_rows(const TileRows* tiles, int i)
{
    const TileRows t = tiles[i];
    const unsigned lo = (unsigned)scalar((int)t.row0), hi = (unsigned)scalar((int)(t.row0 >> 32));
    return {scalar(t.expert), scalar(t.count), (int64_t)((unsigned long long)hi << 32 | lo)};
}

constexpr int largest_divisor4(int n, int most) { return most >= n ? n : n % most == 0 ? most : largest_divisor4(n, most - 1); }

// A workgroup's outputs through LDS, so that whole rows of its tile are stored, 16 bytes a thread and adjacent threads adjacent.  JP of
// the TB blocks of rows at a time, STAGE32 in fp32 (fp32 outputs, and for a residual, so that it rounds once), or as what is stored.  The
// 16-byte pieces of a row lie at piece ^ (row & 7) (fewer bits for rows of fewer pieces).
template <int WR, int WT, int TB, int JP, bool STAGE32, bool GATED, int OUT>
__device__ inline void store_tile4(const Mx4Product& p, const Channels4<GATED, 4>& ch, const f32x4 (&acc)[TB][4], char* smem,
                                   int wr, int wt, int lane, int group0, const TileRows& t)
{
    constexpr bool MX = OUT == NM_MX4, BF16 = OUT == NM_BF16;
    constexpr int C = Channels4<GATED, 4>::kRuns * 8;   // outputs of a group and lane
    constexpr int kOuts = WR * C * 4, kThreads = WR * WT * 64, kRows = WT * JP * 16;
    constexpr int kPitch = MX ? kOuts / 2 : kOuts * (STAGE32 ? 4 : 2), kHas = kPitch / 16, kMask = kHas >= 8 ? 7 : kHas - 1;
    constexpr int kPieces = MX ? kHas : kOuts * (BF16 ? 2 : 4) / 16, kPer = kOuts / kPieces;   // 16-byte pieces of a stored row; values in one
    constexpr int ES = BF16 ? 2 : 4;
    const int col0 = group0 * C * 4;
    const bool past = p.past;
#pragma unroll
    for (int j0 = 0; j0 < TB; j0 += JP) {
        __syncthreads();   // the stages, or the outputs before, have been read
#pragma unroll
        for (int jj = 0; jj < JP; ++jj) {
            const int lrow = (wt * JP + jj) * 16 + (lane & 15);
            char* to = smem + lrow * kPitch;
#pragma unroll
            for (int run = 0; run < Channels4<GATED, 4>::kRuns; ++run) {
                float y[8];
                outputs4<GATED, 4>(ch, acc[j0 + jj], run, y);
                const int c = wr * C * 4 + run * 32 + (lane >> 4) * 8;   // column in the tile
                if constexpr (MX) {
                    unsigned scale;
                    const unsigned codes = rounded8(y, scale);
                    *reinterpret_cast<unsigned*>(to + ((c >> 5) ^ (lrow & kMask)) * 16 + (lane >> 4) * 4) = codes;
                    const int row = (wt * TB + j0 + jj) * 16 + (lane & 15), block = (col0 + c) >> 5;
                    if ((lane >> 4) == 0 && row < t.count && block * 32 < p.outs) p.ys[(t.row0 + row) * p.ldys + block] = (uint8_t)scale;
                } else if constexpr (STAGE32) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        *reinterpret_cast<f32x4*>(to + (((c >> 2) + h) ^ (lrow & 7)) * 16) = f32x4{y[4 * h], y[4 * h + 1], y[4 * h + 2], y[4 * h + 3]};
                } else {
                    u32x4 v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = bf16_pair(y[2 * i], y[2 * i + 1]);
                    *reinterpret_cast<u32x4*>(to + ((c >> 3) ^ (lrow & 7)) * 16) = v;
                }
            }
        }
        __syncthreads();
#pragma unroll 4
        for (int u = threadIdx.x; u < kRows * kPieces; u += kThreads) {
            const int lrow = u / kPieces, piece = u % kPieces;
            const int trow = (lrow / (JP * 16)) * TB * 16 + j0 * 16 + lrow % (JP * 16), col = col0 + piece * kPer;
            if (trow >= t.count || col >= p.outs) continue;
            const int64_t row = t.row0 + trow;
            const char* from = smem + lrow * kPitch;
            if constexpr (MX) {
                store16((char*)p.y + row * p.ldy + (size_t)(col >> 5) * 16, *reinterpret_cast<const u32x4*>(from + (piece ^ (lrow & kMask)) * 16), past);
            } else {
                char* py = (char*)p.y + (row * p.ldy + col) * ES;
                u32x4 v;
                if constexpr (STAGE32 && BF16) {
                    const f32x4 a = *reinterpret_cast<const f32x4*>(from + ((2 * piece) ^ (lrow & 7)) * 16);
                    const f32x4 b = *reinterpret_cast<const f32x4*>(from + ((2 * piece + 1) ^ (lrow & 7)) * 16);
                    float y[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
                    if (p.res) {
                        const char* pr = (const char*)p.res + (row * p.ldr + col) * ES;
                        if (col + 8 <= p.outs) {
                            float r[8];
                            Elem<true>::load8(pr, r);
#pragma unroll
                            for (int e = 0; e < 8; ++e) y[e] += r[e];
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (col + e < p.outs) y[e] += Elem<true>::load1(pr + e * 2);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = bf16_pair(y[2 * i], y[2 * i + 1]);
                } else {
                    v = *reinterpret_cast<const u32x4*>(from + (piece ^ (lrow & 7)) * 16);
                    if (!BF16 && p.res) {
                        const char* pr = (const char*)p.res + (row * p.ldr + col) * 4;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (col + e < p.outs) v[e] = __float_as_uint(__uint_as_float(v[e]) + Elem<false>::load1(pr + e * 4));
                    }
                }
                if (col + kPer <= p.outs) {
                    store16(py, v, past);
                } else {
#pragma unroll
                    for (int e = 0; e < kPer; ++e)
                        if (col + e < p.outs) {
                            if constexpr (BF16) { const unsigned short h = (unsigned short)(v[e / 2] >> (16 * (e & 1))); __builtin_memcpy(py + e * 2, &h, 2); }
                            else { const unsigned w = v[e]; __builtin_memcpy(py + e * 4, &w, 4); }
                        }
                }
            }
        }
    }
}

template <int WR, int WT, int TB, int NS, int PER_CU, bool GATED, int OUT>
__global__ __launch_bounds__(WR * WT * 64, PER_CU * WR * WT / 4) void mx4_tile_kernel(Mx4Product p, TileOrder order, const TileHead* head,
                                                                                      const TileRows* tiles, const unsigned* scales)
{
    using T = Tile4<WR, WT, TB, NS>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wr = wave % WR, wt = wave / WR;
    int tc, tr, tile, split;
    if (p.grouped) {   // (tiles past those that there are end here, so that the others are dealt to all XCDs)
        order.tiles_r = head->tiles;
        if ((int)blockIdx.x >= order.tiles()) return;
    }
    order.at(blockIdx.x, tc, tr, tile, split);
    tc = scalar(tc);
    tr = scalar(tr);
    const TileRows t = tile_rows(tiles, tr);
    const int g0 = tc * WR, steps = p.steps, halves = steps * 2;
    const bool own = g0 + wr < p.groups;   // (a wavefront past the last group multiplies zeros)
    const size_t group = (size_t)t.expert * p.groups + (own ? g0 + wr : 0);
    const RowTile rt{t.expert, t.count, t.row0};
    const __amdgpu_buffer_rsrc_t wsr = q8_rsrc(p.w + group * halves * 4096, own ? (unsigned)halves * 4096 : 0);
    const __amdgpu_buffer_rsrc_t gsr = q8_rsrc(p.ws + group * halves * 64, own ? (unsigned)halves * 256 : 0);
    const __amdgpu_buffer_rsrc_t xsr = RowBuffers(p, rt).q;
    const __amdgpu_buffer_rsrc_t ssr = q8_rsrc(scales + (size_t)tr * halves * T::kRows, (unsigned)halves * T::kRows * 4);
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_ptr_t)smem;
    constexpr unsigned kNone = 0xc0000000u;   // (and what a lane adds: past the end of weights and scales)
    // Rows past the tile's last read its first: what comes of them is not stored.  (The scale of a row for an index outside x is NaN.)
    const int chunk = (lane & 7) ^ (lane >> 3);   // the block of a step that the lane loads, of a row with row & 7 = lane / 8
    unsigned xvoff[T::kXLoads];
#pragma unroll
    for (int i = 0; i < T::kXLoads; ++i) {
        const int src = source_of(p, rt, (wave + i * T::kWaves) * 8 + (lane >> 3));
        xvoff[i] = (unsigned)((src < 0 ? 0 : src) * p.ldq) + chunk * 16;
    }
    const int xsteps = (p.blocks + 7 - chunk) >> 3;   // steps that have it
    const unsigned lane16 = lane * 16, lane4 = lane * 4;
    // load i of step s into the stage at `at`; past the last step nothing is read, so that the count of loads holds
    auto fetch = [&](int i, int s, unsigned at) {
        if (i < T::kXLoads) {
            load_to_lds(xsr, s < xsteps ? xvoff[i] + (unsigned)s * 128 : kPast, lds0 + at + (wave + i * T::kWaves) * 1024);
        } else {
            const int u = wave + (i - T::kXLoads) * T::kWaves;
            const bool in = T::kSUnits % T::kWaves == 0 || u < T::kSUnits;
            load_to_lds4(ssr, (s < steps && in ? (unsigned)s * (T::kRows * 8) + u * 256 : kNone) + lane4, lds0 + (in ? at + T::kXBytes + u * 256 : (unsigned)T::kNowhere));
        }
    };
    i32x4 w[4][4], x[4];            // weights of four halves; rows of four blocks
    unsigned ws[4], xs[2][TB / 4];  // their scales
    auto weights = [&](int set, int i, int half) {   // load i of a half's
        const unsigned from = half < halves ? (unsigned)half : kNone >> 12;
        if (i < 4) w[set][i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(wsr, from * 4096 + i * 1024 + lane16, 0, 0));
        else ws[set] = __builtin_amdgcn_raw_buffer_load_b32(gsr, from * 256 + lane4, 0, 0);
    };
    const int xlane = (wt * TB * 16 + (lane & 15)) * 128 + (((lane >> 4) ^ (lane & 7)) << 4), slane = T::kXBytes + wt * TB * 64 + lane * 4;
    auto rows = [&](int h, int j, unsigned at) { x[j & 3] = *reinterpret_cast<const i32x4*>(smem + at + (xlane ^ (h * 64)) + j * 2048); };
    auto row_words = [&](int h, int i, unsigned at) { xs[h][i] = *reinterpret_cast<const unsigned*>(smem + at + slane + h * (T::kRows * 4) + i * 256); };
    f32x4 acc[TB][4] = {};
#pragma unroll
    for (int s = 0; s < NS; ++s) {
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) fetch(i, s, s * T::kStage);
        asm volatile("" : : : "memory");   // (the first step's rows are the oldest loads)
        if (s < 3)
#pragma unroll
            for (int i = 0; i < 5; ++i) weights(s, i, s);
    }
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((NS - 1) * T::kLoads + 15) : "memory");
#pragma unroll
    for (int j = 0; j < 3; ++j) rows(0, j, 0);
#pragma unroll
    for (int i = 0; i < TB / 4; ++i) row_words(0, i, 0);
    auto multiply = [&](int set, int h, int j) {
        auto four = [&](auto ox) {
            constexpr int OX = decltype(ox)::value;
            acc[j][0] = mma4<0, OX>(w[set][0], x[j & 3], acc[j][0], ws[set], xs[h][j / 4]);
            acc[j][1] = mma4<1, OX>(w[set][1], x[j & 3], acc[j][1], ws[set], xs[h][j / 4]);
            acc[j][2] = mma4<2, OX>(w[set][2], x[j & 3], acc[j][2], ws[set], xs[h][j / 4]);
            acc[j][3] = mma4<3, OX>(w[set][3], x[j & 3], acc[j][3], ws[set], xs[h][j / 4]);
        };
        if (j % 4 == 0) four(std::integral_constant<int, 0>{});
        else if (j % 4 == 1) four(std::integral_constant<int, 1>{});
        else if (j % 4 == 2) four(std::integral_constant<int, 2>{});
        else four(std::integral_constant<int, 3>{});
    };
    unsigned now = 0;   // the stage that is multiplied
    // two steps a turn, for the four sets of weights; past the last step zeros are multiplied
    for (int k = 0; k < halves; k += 4) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int h = q & 1;
            const unsigned then = now + T::kStage == T::kNowhere ? 0 : now + T::kStage;
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                // In a step's second half, once all of its rows are read: all wavefronts have read this stage, and the next one has landed.  Younger
                // than its loads are those of NS - 2 steps and of the weights of four halves.
                if (h == 1 && j == TB - 3)
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((NS - 2) * T::kLoads + 15) : "memory");
                if (j + 3 < TB) rows(h, j + 3, now);
                else rows(1 - h, j + 3 - TB, h == 0 ? now : then);
                if (j >= TB - 3 && j - (TB - 3) < TB / 4) row_words(1 - h, j - (TB - 3), h == 0 ? now : then);
                if constexpr (TB == 4) {
                    weights((q + 3) & 3, j, k + q + 3);
                    if (j == 3) weights((q + 3) & 3, 4, k + q + 3);
                } else {
                    if (j < 5) weights((q + 3) & 3, j, k + q + 3);
                }
                if (h == 1 && j >= TB - 3)
#pragma unroll
                    for (int i = (j - TB + 3) * T::kLoads / 3; i < (j - TB + 4) * T::kLoads / 3; ++i) fetch(i, (k + q) / 2 + NS, now);
                multiply(q, h, j);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (h == 1) now = then;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");   // no load into LDS outlives the workgroup
    Channels4<GATED, 4> ch;
    ch.load(p, t.expert, own ? g0 + wr : p.groups - 1, 0, lane);   // (what a wavefront past the last group has is not stored)
    constexpr int kOuts = WR * Channels4<GATED, 4>::kRuns * 32;
    constexpr int JP4 = largest_divisor4(TB, T::kLds / (16 * WT * kOuts * 4)), JP2 = largest_divisor4(TB, T::kLds / (16 * WT * kOuts * 2)),
                  JPM = largest_divisor4(TB, T::kLds / (16 * WT * kOuts / 2));
    if constexpr (OUT == NM_MX4) store_tile4<WR, WT, TB, JPM, false, GATED, OUT>(p, ch, acc, smem, wr, wt, lane, g0, t);
    else if constexpr (OUT == NM_F32) store_tile4<WR, WT, TB, JP4, true, GATED, OUT>(p, ch, acc, smem, wr, wt, lane, g0, t);
    else if (p.res) store_tile4<WR, WT, TB, JP4, true, GATED, OUT>(p, ch, acc, smem, wr, wt, lane, g0, t);
    else store_tile4<WR, WT, TB, JP2, false, GATED, OUT>(p, ch, acc, smem, wr, wt, lane, g0, t);
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

// One 16-byte unit of the packed weights a thread; those of the first row block also the words of scales.
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
        const int c = q8_row_of(group * 64 + b * 16 + (lane & 15), channels, gated), kb = step * 8 + 4 * h + (lane >> 4);
        i32x4 v = {0, 0, 0, 0};
        if (c >= 0 && kb < blocks) v = block_codes(q + (expert * channels + c) * ldq, kb, width);
        *reinterpret_cast<i32x4*>(to + i * 16) = v;
        if (b == 0) {
            unsigned word = 0;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int cn = q8_row_of(group * 64 + n * 16 + (lane & 15), channels, gated);
                unsigned scale = 127;
                if (cn >= 0 && kb < blocks) scale = scales[(expert * channels + cn) * lds + kb];
                if (scale == 255) atomicOr(bad, 1);
                word |= scale << (8 * n);
            }
            to_scales[(gk * 2 + h) * 64 + lane] = word;
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
        const int c = q8_row_of(group * 64 + b * 16 + (lane & 15), channels, gated), kb = step * 8 + 4 * h + (lane >> 4);
        if (c < 0 || kb >= blocks) continue;
        const int64_t row = expert * channels + c;
        *reinterpret_cast<i32x4*>(q + (row * blocks + kb) * 16) = *reinterpret_cast<const i32x4*>(from + i * 16);
        scales[row * blocks + kb] = (uint8_t)(from_scales[(gk * 2 + h) * 64 + lane] >> (8 * b));
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

// The tile kernels' shapes.
struct Shape4 {
    int wr, rows, waves, per_cu;   // per_cu: workgroups that a CU holds (by LDS)
};
constexpr Shape4 kShapes4[] = {{4, 256, 8, 1},    // 256 packed channels x 256 rows
                               {4, 128, 4, 2},
                               {4, 64, 4, 2}};

template <int SHAPE, int WT, int TB, int NS, bool GATED, int OUT>
int launch_tile4(const Mx4Product& p, const Mx4Plan& pl, char* workspace, hipStream_t s)
{
    constexpr int WR = kShapes4[SHAPE].wr;
    using T = Tile4<WR, WT, TB, NS>;
    static_assert(T::kWaves == kShapes4[SHAPE].waves && T::kRows == kShapes4[SHAPE].rows, "kShapes4 describes the kernels");
    TileOrder o;
    o.splits = 1;
    o.tiles_c = (p.groups + WR - 1) / WR;
    o.tiles_r = (int)pl.tiles;
    const int64_t grid = pl.tiles * o.tiles_c, parts = T::kRows / 64;
    if (grid > 0x7fffffff || pl.tiles * parts > 0x7fffffff) {
        set_error("%lld tiles: too many", (long long)grid);
        return NM_ERR_SHAPE;
    }
    TileHead* head = (TileHead*)workspace;
    TileRows* tiles = (TileRows*)(head + 1);
    unsigned* scales = (unsigned*)(workspace + pl.tile_bytes);
    hipLaunchKernelGGL(mx4_scales_kernel, dim3((unsigned)(pl.tiles * parts), (unsigned)(p.steps < 32 ? (p.steps + 1) / 2 : 16)), dim3(256), 0, s, p, T::kRows, head, tiles, scales);
    NM_HIP_CHECK(hipGetLastError());
    static unsigned long long done = 0;
    const int rc = allow_lds((const void*)mx4_tile_kernel<WR, WT, TB, NS, kShapes4[SHAPE].per_cu, GATED, OUT>, T::kLds, &done);
    if (rc != NM_OK) return rc;
    hipLaunchKernelGGL((mx4_tile_kernel<WR, WT, TB, NS, kShapes4[SHAPE].per_cu, GATED, OUT>), dim3((unsigned)grid), dim3(T::kWaves * 64), T::kLds, s, p, o,
                       (const TileHead*)head, (const TileRows*)tiles, (const unsigned*)scales);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

template <bool GATED, int OUT>
int pick_tile4(const Mx4Product& p, const Mx4Plan& pl, char* workspace, hipStream_t s)
{
    switch (pl.shape) {
    case 0: return launch_tile4<0, 2, 8, 3, GATED, OUT>(p, pl, workspace, s);
    case 1: return launch_tile4<1, 1, 8, 3, GATED, OUT>(p, pl, workspace, s);
    default: return launch_tile4<2, 1, 4, 4, GATED, OUT>(p, pl, workspace, s);
    }
}

}  // namespace

Mx4Plan mx4_plan(const Mx4Product& p)
{
    Mx4Plan pl;
    const int64_t each = p.grouped ? (p.rows + p.experts - 1) / p.experts : p.rows;
    if (each <= NM_MX4_FEW_ROWS) return pl;
    pl.shape = each >= 256 ? 0 : 2;
    if (pl.shape < 0) return pl;
    const int per = kShapes4[pl.shape].rows;
    pl.tiles = tiles_of(p, per);
    pl.tile_bytes = (sizeof(TileHead) + (size_t)pl.tiles * sizeof(TileRows) + 255) / 256 * 256;
    pl.scale_bytes = (size_t)pl.tiles * per * p.steps * 8;
    return pl;
}

int run_mx4_product(const Mx4Product& p, const Mx4Plan& pl, void* workspace, hipStream_t s)
{
    if (pl.shape >= 0) {
        char* ws = (char*)workspace;
        if (p.out == NM_MX4) return p.gated ? pick_tile4<true, NM_MX4>(p, pl, ws, s) : pick_tile4<false, NM_MX4>(p, pl, ws, s);
        if (p.out == NM_BF16) return p.gated ? pick_tile4<true, NM_BF16>(p, pl, ws, s) : pick_tile4<false, NM_BF16>(p, pl, ws, s);
        return p.gated ? pick_tile4<true, NM_F32>(p, pl, ws, s) : pick_tile4<false, NM_F32>(p, pl, ws, s);
    }
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
