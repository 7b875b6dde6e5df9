// Products of rows in MX4 with weights in MX4, of one matrix or grouped by expert.
//
//   z[r][c] = sum_k x[r][k] * w[c][k] + bias[c];   y = z (+ residual),  or  silu(gate) * up;   out in fp32, bf16 or MX4
//
// The matrix instruction takes codes and scales as they are; its sums of 128 products and their addition to the accumulators are in fp32
// (measured against 64 bits: within 2^-23 of the sum of the products' magnitudes).  Weights are its first operand, rows of x the second: lane l of
// a wavefront then holds packed weight rows 4 (l / 16) .. + 3 of a 16-row block for row l % 16 of x, and the packing deals channels so that
// the four blocks of a 64-row group give it twice 8 adjacent channels (gated: 8 adjacent outputs, gate and value in the same registers).
// (Out of registers, on normally distributed values, this form does 7.0 to 7.3 PFLOP/s and the 32x32x64 one 6.2; on zeros 9.7 and 8.9.)
#include "nm_mx4_product.h"

namespace nm {
namespace {

// ---------------------------------------------------------------- few rows
// Tiles of up to 16 * TB rows.  A workgroup owns RB blocks of 16 packed channels; its NW wavefronts take the steps of 256 k in turn, and add
// their sums through LDS at the end, in the order of the wavefronts.  Weights go from memory into registers: a
// weight is used once, there is nothing to share.  Rows of x go through LDS, a part of it for each wavefront, so that 8 lanes read the 128
// adjacent bytes of a row.
template <int TB, int RB, int NW> constexpr int few4_lds()
{
    const int rows = NW * TB * 2048, sums = NW * RB * TB * 1024;
    return rows > sums ? rows : sums;
}

template <int TB, int RB, int NW>
__global__ __launch_bounds__(NW * 64) void mx4_few_kernel(Mx4Product p, int parts, int tile0)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int in = blockIdx.x / parts, b0 = (blockIdx.x - in * parts) * RB;   // (RB divides 4: a workgroup stays within its row group)
    const RowTile t = GroupTiles(p, 16 * TB).at(p, tile0 + in);
    if (t.count == 0) return;
    const size_t group = (size_t)t.expert * p.groups + (b0 >> 2);
    const __amdgpu_buffer_rsrc_t wsr = q8_rsrc(p.w + group * p.steps * 8192, (unsigned)p.steps * 8192);
    const __amdgpu_buffer_rsrc_t ssr = q8_rsrc(p.ws + group * p.steps * 128, (unsigned)p.steps * 512);
    const __amdgpu_buffer_rsrc_t qsr = row_buffer(p, t);
    const unsigned woff = (b0 & 3) * 1024 + lane * 16, soff = lane * 4;
    const unsigned mine = wave * (TB * 2048), lds0 = (unsigned)(uintptr_t)(lds_ptr_t)smem + mine;
    const unsigned at = mine + (lane & 15) * 128;
    unsigned qoff[TB][2];   // 8 rows an instruction, block c of a row at c ^ (row & 7)
    // A step's eight scales of a row: one load of a lane for each of the tile's rows, dealt out among the lanes.
    const int source = source_of(p, t, lane & (16 * TB - 1));
    const uint8_t* scales = p.s + (p.index ? 0 : (int64_t)t.row0 * p.lds) + (source < 0 ? 0 : source) * p.lds;
    const unsigned pick = 0x0c0c0400u + (lane >> 4) * 0x0101u;   // of two words the byte of the lane's block each
    const int chunk = (lane & 7) ^ (lane >> 3);
#pragma unroll
    for (int i = 0; i < TB; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int src = source_of(p, t, i * 16 + h * 8 + (lane >> 3));
            qoff[i][h] = src < 0 ? kPast : (unsigned)(src * p.ldq) + chunk * 16;
        }
    }
    f32x4 acc[RB][TB] = {};
    for (int k = wave; k < p.steps; k += NW) {
        i32x4 wf[2][RB];
        unsigned wsc[2], xsc[TB];
        const bool row_in = k * 8 + chunk < p.blocks;
#pragma unroll
        for (int i = 0; i < TB; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                load_to_lds(qsr, row_in && qoff[i][h] != kPast ? qoff[i][h] + k * 128 : kPast, lds0 + i * 2048 + h * 1024);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < RB; ++i)
                wf[h][i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(wsr, woff + i * 1024 + (k * 2 + h) * 4096, 0, 2));
#pragma unroll
        for (int h = 0; h < 2; ++h) wsc[h] = __builtin_amdgcn_raw_buffer_load_b32(ssr, soff + (k * 2 + h) * 256, 0, 0);
        u32x2 s8;
        if (k * 8 + 8 <= p.blocks) __builtin_memcpy(&s8, scales + k * 8, 8);
        else s8 = last_scales(scales + k * 8, p.blocks - k * 8);
        if (source == -2) s8 = u32x2{0xffffffffu, 0xffffffffu};
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
#pragma unroll
        for (int i = 0; i < TB; ++i) {
            const unsigned lo = TB == 1 ? s8[0] : __shfl(s8[0], i * 16 + (lane & 15)), hi = TB == 1 ? s8[1] : __shfl(s8[1], i * 16 + (lane & 15));
            xsc[i] = __builtin_amdgcn_perm(hi, lo, pick);
        }
        auto half = [&](auto hh) {
            constexpr int h = decltype(hh)::value;
            i32x4 xf[TB];
#pragma unroll
            for (int j = 0; j < TB; ++j)
                xf[j] = *reinterpret_cast<const i32x4*>(smem + at + j * 2048 + (((4 * h + (lane >> 4)) ^ (lane & 7)) << 4));
            const unsigned ws = RB == 4 ? wsc[h] : wsc[h] >> (8 * (b0 & 3));
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                acc[0][j] = mma4<0, h>(wf[h][0], xf[j], acc[0][j], ws, xsc[j]);
                if constexpr (RB >= 2) acc[1][j] = mma4<1, h>(wf[h][1], xf[j], acc[1][j], ws, xsc[j]);
                if constexpr (RB == 4) {
                    acc[2][j] = mma4<2, h>(wf[h][2], xf[j], acc[2][j], ws, xsc[j]);
                    acc[3][j] = mma4<3, h>(wf[h][3], xf[j], acc[3][j], ws, xsc[j]);
                }
            }
        };
        half(std::integral_constant<int, 0>{});
        half(std::integral_constant<int, 1>{});
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
            emit4<GATED, NB>(p, ch, sum, (int64_t)t.row0 + row, row < t.count);
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
// A workgroup of WR wavefronts owns 64 * WR packed channels x 16 * TB rows; a wavefront 64 x 16 TB of them.  K goes by in steps
// of 256, each two halves of one matrix instruction's 128.
// Rows go through LDS, NS steps of them, loaded straight into it: while a step is multiplied the next one's lie there and later ones' are on
// their way; a wavefront reads the operand of 16 rows three before it is multiplied.
// Weights go from memory into registers, three halves ahead: their layout in memory is the operands', and no other wavefront of the workgroup
// wants them.  Through LDS as well, LDS is what bounds the loop.
// The rows' scales are dealt out in LDS for kSteps steps at once, as the lanes read them: a word has those of four blocks of 16 rows.
// (Read byte by byte in the loop they made large products 3 to 8 % slower, dealt out by a kernel in front small ones 2 to 5 us.)
// Where all of the chip multiplies the matrix units work 61 % of the cycles, at a clock that power decides (8192 x 4096 -> 16384 249 us at 1.7 GHz on
// normally distributed values, 182 at 2.2 on zeros, as many cycles; the instruction alone 1.34 times as fast on zeros; by the card 240 to 300).
// Where K is short a tile's start and end decide: of the 18.9 us of a tile of eight steps, gated and rounded, the loop takes 8.5, silu, rounding and
// stores 5.0, the first loads 2.75.
// A row's 128 bytes are 8 blocks of 16, block c stored at c ^ (row & 7), so that what an LDS cycle reads lies in different banks.
template <int WR, int TB, int NS> struct Tile4 {
    static constexpr int kWaves = WR, kThreads = 64 * kWaves, kRows = 16 * TB;
    static constexpr int kXBytes = kRows * 128, kXLoads = kXBytes / 1024 / kWaves;       // of 1 KiB, a wavefront and step
    static constexpr int kSteps = 24, kWords = kRows / 64;                               // words of scales of a half and lane
    static constexpr int kHalf = kWords * 256 + 4;                                       // (so that a row's words go to different banks)
    static constexpr int kSAt = NS * kXBytes, kFromAt = kSAt + (kSteps * 2 + 1) * kHalf; // (a half past the last is read)
    static constexpr int kLds = kFromAt + kRows * 4;                                     // where the tile's rows lie in x, for an index
    static_assert(TB % 4 == 0 && kXBytes % (1024 * kWaves) == 0 && kThreads % 32 == 0 && 16 * kWords % (kThreads / 32) == 0, "every wavefront issues the same loads");
    static_assert(NS >= 3 && kLds <= 160 * 1024, "");
};

// A value that is the same in all lanes, as the loads into LDS want it.
__device__ inline int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }

constexpr int largest_divisor4(int n, int most) { return most >= n ? n : n % most == 0 ? most : largest_divisor4(n, most - 1); }

// A workgroup's outputs through LDS, so that whole rows of its tile are stored, 16 bytes a thread and adjacent threads adjacent.  JP of
// the TB blocks of rows at a time, STAGE32 in fp32 (fp32 outputs, and for a residual, so that it rounds once), or as what is stored.  The
// 16-byte pieces of a row lie at piece ^ (row & 7) (fewer bits for rows of fewer pieces).  (Codes in MX4 stored straight from the registers,
// 16 bytes of a row an instruction, made 4096 x 4096 -> 2 x 12288 8 % slower.)
template <int WR, int TB, int JP, bool STAGE32, bool GATED, int OUT>
__device__ inline void store_tile4(const Mx4Product& p, const Channels4<GATED, 4>& ch, const f32x4 (&acc)[TB][4], char* smem, int wave,
                                   int lane, int group0, const RowTile& t)
{
    constexpr bool MX = OUT == NM_MX4, BF16 = OUT == NM_BF16;
    constexpr int C = Channels4<GATED, 4>::kRuns * 8;   // outputs of a group and lane
    constexpr int kOuts = WR * C * 4, kThreads = WR * 64, kRows = JP * 16;
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
            const int lrow = jj * 16 + (lane & 15);
            char* to = smem + lrow * kPitch;
#pragma unroll
            for (int run = 0; run < Channels4<GATED, 4>::kRuns; ++run) {
                float y[8];
                outputs4<GATED, 4>(ch, acc[j0 + jj], run, y);
                const int c = wave * C * 4 + run * 32 + (lane >> 4) * 8;   // column in the tile
                if constexpr (MX) {
                    unsigned scale;
                    const unsigned codes = rounded8(y, scale);
                    *reinterpret_cast<unsigned*>(to + ((c >> 5) ^ (lrow & kMask)) * 16 + (lane >> 4) * 4) = codes;
                    const int row = (j0 + jj) * 16 + (lane & 15), block = (col0 + c) >> 5;
                    if ((lane >> 4) == 0 && row < t.count && block * 32 < p.outs) p.ys[((int64_t)t.row0 + row) * p.ldys + block] = (uint8_t)scale;
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
            const int trow = j0 * 16 + lrow, col = col0 + piece * kPer;
            if (trow >= t.count || col >= p.outs) continue;
            const int64_t row = (int64_t)t.row0 + trow;
            const char* from = smem + lrow * kPitch;
            if constexpr (MX) {
                store16((char*)p.y + row * p.ldy + (size_t)(col >> 5) * 16, *reinterpret_cast<const u32x4*>(from + (piece ^ (lrow & kMask)) * 16), past);
                continue;
            }
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

template <int WR, int TB, int NS, int PER_CU, bool GATED, int OUT>
__global__ __launch_bounds__(WR * 64, PER_CU * WR / 4) void mx4_tile_kernel(Mx4Product p, TileBands order, int block0)
{
    using T = Tile4<WR, TB, NS>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = scalar(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const GroupTiles groups(p, T::kRows);
    order.tiles_r = groups.all;   // (of experts, those that there are, so that they are dealt to all XCDs)
    const int block = block0 + blockIdx.x;
    if (block >= order.tiles()) return;
    int tc, tr;
    order.at(block, tc, tr);
    tc = scalar(tc);
    tr = scalar(tr);
    const RowTile t = groups.at(p, tr);
    const int g0 = tc * WR, steps = p.steps, halves = steps * 2;
    const bool own = g0 + wave < p.groups;   // (a wavefront past the last group multiplies zeros)
    const size_t group = (size_t)t.expert * p.groups + (own ? g0 + wave : 0);
    const __amdgpu_buffer_rsrc_t wsr = q8_rsrc(p.w + group * halves * 4096, own ? (unsigned)halves * 4096 : 0);
    const __amdgpu_buffer_rsrc_t gsr = q8_rsrc(p.ws + group * halves * 64, own ? (unsigned)halves * 256 : 0);
    const __amdgpu_buffer_rsrc_t qsr = row_buffer(p, t);
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_ptr_t)smem;
    constexpr unsigned kNone = 0xc0000000u;   // (and what a lane adds: past the end of weights and scales)
    // Rows past the tile's last read its first: what comes of them is not stored.
    if (p.index) {
        for (int i = threadIdx.x; i < T::kRows; i += T::kThreads) *reinterpret_cast<int*>(smem + T::kFromAt + i * 4) = source_of(p, t, i);
        __syncthreads();
    }
    auto source = [&](int row) { return p.index ? *reinterpret_cast<const int*>(smem + T::kFromAt + row * 4) : row < t.count ? row : -1; };
    const int chunk = (lane & 7) ^ (lane >> 3);   // the block of a step that the lane loads, of a row with row & 7 = lane / 8
    unsigned xvoff[T::kXLoads];
#pragma unroll
    for (int i = 0; i < T::kXLoads; ++i) {
        const int src = source((wave + i * T::kWaves) * 8 + (lane >> 3));
        xvoff[i] = (unsigned)((src < 0 ? 0 : src) * p.ldq) + chunk * 16;
    }
    const int xsteps = (p.blocks + 7 - chunk) >> 3;   // steps that have it
    const unsigned lane16 = lane * 16, lane4 = lane * 4;
    // load i of step s into the stage at `at`; past the last step nothing is read, so that the count of loads holds
    auto fetch = [&](int i, int s, unsigned at) {
        load_to_lds(qsr, s < xsteps ? xvoff[i] + (unsigned)s * 128 : kPast, lds0 + at + (wave + i * T::kWaves) * 1024);
    };
    i32x4 w[4][4], x[4];                 // weights of four halves; rows of four blocks
    unsigned ws[4], xs[2][T::kWords];    // their scales
    auto weights = [&](int set, int i, int half) {   // load i of a half's
        const unsigned at = half < halves ? (unsigned)half : kNone >> 12;
        if (i < 4) w[set][i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(wsr, at * 4096 + i * 1024 + lane16, 0, 0));
        else ws[set] = __builtin_amdgcn_raw_buffer_load_b32(gsr, at * 256 + lane4, 0, 0);
    };
    // The scales of 32 halves at a time: a thread takes one half of them, and in turn PASSES times four rows, 16 apart; their words of four blocks
    // each become for each of those blocks the word of the four rows.
    constexpr int ROWS = T::kThreads / 32, PASSES = 16 * T::kWords / ROWS;
    struct Scales {
        unsigned v[4];
        bool lost[4];   // (of a row for an index outside x they are NaN)
    };
    const uint8_t* scales_of = p.s + (p.index ? 0 : (int64_t)t.row0 * p.lds);
    auto load_scales = [&](int half, int pass, Scales& s) {
        const int at = pass * ROWS + (threadIdx.x >> 5), kb = half * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int src = source(((at >> 4) * 4 + j) * 16 + (at & 15));
            const uint8_t* row = scales_of + (src < 0 ? 0 : src) * p.lds;
            s.lost[j] = src == -2;
            // the row's last word, moved down to where its end is, and 1 past that: codes of 0 are multiplied (without branches, so that the
            // loads of all passes are out together)
            const int at_kb = kb < p.blocks - 4 ? kb : p.blocks - 4, less = kb - at_kb;
            unsigned word;
            __builtin_memcpy(&word, row + at_kb, 4);
            word = __builtin_amdgcn_alignbyte(0x7f7f7f7fu, word, less & 3);
            s.v[j] = less < 4 ? word : 0x7f7f7f7fu;
        }
    };
    auto put_scales = [&](int half, int pass, Scales& s) {   // `half`: among those in LDS
        const int at = pass * ROWS + (threadIdx.x >> 5);
#pragma unroll
        for (int j = 0; j < 4; ++j) s.v[j] = s.lost[j] ? 0xffffffffu : s.v[j];
        // byte b of word j becomes byte j of word b
        const unsigned a0 = __builtin_amdgcn_perm(s.v[1], s.v[0], 0x05010400), a1 = __builtin_amdgcn_perm(s.v[1], s.v[0], 0x07030602);
        const unsigned c0 = __builtin_amdgcn_perm(s.v[3], s.v[2], 0x05010400), c1 = __builtin_amdgcn_perm(s.v[3], s.v[2], 0x07030602);
        const unsigned out[4] = {(a0 & 0xffffu) | c0 << 16, a0 >> 16 | (c0 & 0xffff0000u), (a1 & 0xffffu) | c1 << 16, a1 >> 16 | (c1 & 0xffff0000u)};
        if (half < T::kSteps * 2)
#pragma unroll
            for (int b = 0; b < 4; ++b) *reinterpret_cast<unsigned*>(smem + T::kSAt + half * T::kHalf + (at >> 4) * 256 + b * 64 + (at & 15) * 4) = out[b];
    };
    auto deal = [&](int first, int done) {   // those of halves first .., but for the first `done`
        const int rest = (halves - first + 3) & ~3, end = rest < T::kSteps * 2 ? rest : T::kSteps * 2;
        for (int h = done; h < end; h += 32)
#pragma unroll 2
            for (int i = 0; i < PASSES; ++i) {
                Scales s;
                load_scales(first + h + (threadIdx.x & 31), i, s);
                put_scales(h + (threadIdx.x & 31), i, s);
            }
    };
    const int xlane = (lane & 15) * 128 + (((lane >> 4) ^ (lane & 7)) << 4), slane = T::kSAt + lane * 4;
    auto rows = [&](int h, int j, unsigned at) { x[j & 3] = *reinterpret_cast<const i32x4*>(smem + at + (xlane ^ (h * 64)) + j * 2048); };
    auto words = [&](int h, int i, unsigned at) { xs[h][i] = *reinterpret_cast<const unsigned*>(smem + slane + at + i * 256); };
    f32x4 acc[TB][4];
    // The first scales are asked for before all else: what is asked for later is waited for with them.
    Scales first[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) load_scales(threadIdx.x & 31, i, first[i]);
    asm volatile("" : : : "memory");
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < T::kXLoads; ++i) fetch(i, s, s * T::kXBytes);
    asm volatile("" : : : "memory");   // (rows first, so that the weights may still be out when they have landed)
#pragma unroll
    for (int s = 0; s < 3; ++s)
#pragma unroll
        for (int i = 0; i < 5; ++i) weights(s, i, s);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) put_scales(threadIdx.x & 31, i, first[i]);
    deal(0, 32);
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[j][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    asm volatile("s_waitcnt vmcnt(15) lgkmcnt(0)\n\ts_barrier" : : : "memory");
#pragma unroll
    for (int j = 0; j < 3; ++j) rows(0, j, 0);
#pragma unroll
    for (int i = 0; i < T::kWords; ++i) words(0, i, 0);
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
    unsigned now = 0, scales = 0;   // the stage that is multiplied; the words of its half
    int left = T::kSteps;           // steps whose scales lie in LDS
    // two steps a turn, for the four sets of weights; past the last step zeros are multiplied
    for (int k = 0; k < halves; k += 4) {
        if (left == 0) {
            __syncthreads();   // (the scales have been read)
            deal(k, 0);
            __syncthreads();
            scales = 0;
            left = T::kSteps;
#pragma unroll
            for (int i = 0; i < T::kWords; ++i) words(0, i, 0);
        }
        left -= 2;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int h = q & 1;
            const unsigned then = now + T::kXBytes == T::kSAt ? 0 : now + T::kXBytes;
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                // In a step's second half, once all of its rows are read: all wavefronts have read this stage, and the next one has landed.  Younger
                // than its loads are those of NS - 2 steps and of the weights of three halves at least.
                if (h == 1 && j == TB - 3)
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((NS - 2) * T::kXLoads + 15) : "memory");
                if (j + 3 < TB) rows(h, j + 3, now);
                else rows(1 - h, j + 3 - TB, h == 0 ? now : then);
                if (j >= TB - 3 && j - (TB - 3) < T::kWords) words(1 - h, j - (TB - 3), scales + (q + 1) * T::kHalf);
                if constexpr (TB == 4) {
                    weights((q + 3) & 3, j, k + q + 3);
                    if (j == 3) weights((q + 3) & 3, 4, k + q + 3);
                } else {
                    if (j < 5) weights((q + 3) & 3, j, k + q + 3);
                }
                if (h == 1 && j >= TB - 3)
#pragma unroll
                    for (int i = (j - TB + 3) * T::kXLoads / 3; i < (j - TB + 4) * T::kXLoads / 3; ++i) fetch(i, (k + q) / 2 + NS, now);
                multiply(q, h, j);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (h == 1) now = then;
        }
        scales += 4 * T::kHalf;
    }
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");   // no load into LDS outlives the workgroup
    Channels4<GATED, 4> ch;
    ch.load(p, t.expert, own ? g0 + wave : p.groups - 1, 0, lane);   // (what a wavefront past the last group has is not stored)
    constexpr int kOuts = WR * Channels4<GATED, 4>::kRuns * 32;
    constexpr int JP4 = largest_divisor4(TB, T::kLds / (16 * kOuts * 4)), JP2 = largest_divisor4(TB, T::kLds / (16 * kOuts * 2)),
                  JPM = largest_divisor4(TB, T::kLds / (16 * kOuts / 2));
    if constexpr (OUT == NM_MX4) store_tile4<WR, TB, JPM, false, GATED, OUT>(p, ch, acc, smem, wave, lane, g0, t);
    else if constexpr (OUT == NM_F32) store_tile4<WR, TB, JP4, true, GATED, OUT>(p, ch, acc, smem, wave, lane, g0, t);
    else if (p.res) store_tile4<WR, TB, JP4, true, GATED, OUT>(p, ch, acc, smem, wave, lane, g0, t);
    else store_tile4<WR, TB, JP2, false, GATED, OUT>(p, ch, acc, smem, wave, lane, g0, t);
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

// Work-items of a launch.  A call that wants more is several launches.
constexpr int64_t kMaxItems = 0xffffffffll;

template <int TB, int RB, int NW>
int launch_few4(const Mx4Product& p, hipStream_t s)
{
    constexpr int LDS = few4_lds<TB, RB, NW>();
    if constexpr (LDS > 64 * 1024) {
        static unsigned long long done = 0;
        const int rc = allow_lds((const void*)mx4_few_kernel<TB, RB, NW>, LDS, &done);
        if (rc != NM_OK) return rc;
    }
    const int parts = p.groups * 4 / RB;   // (at most 2^20, of channels up to 2^24)
    const int64_t tiles = tiles_of(p, 16 * TB), each = kMaxItems / (NW * 64) / parts;
    for (int64_t at = 0; at < tiles; at += each) {
        const int64_t n = tiles - at < each ? tiles - at : each;
        hipLaunchKernelGGL((mx4_few_kernel<TB, RB, NW>), dim3((unsigned)(n * parts)), dim3(NW * 64), LDS, s, p, parts, (int)at);
        NM_HIP_CHECK(hipGetLastError());
    }
    return NM_OK;
}

// Groups of 64 packed channels times tiles of `per` rows, were the rows dealt evenly.
inline int64_t places(const Mx4Product& p, int per)
{
    const int groups = !p.grouped ? 1 : p.experts < p.rows ? p.experts : p.rows;
    const int each = (p.rows + groups - 1) / groups;
    return (int64_t)groups * ((each + per - 1) / per) * p.groups;
}

// Up to 16 rows bound by HBM: 12288 -> 4096 takes 9.0 us, of which 3.5 are a call's that reads next to nothing and 5.9 the weights' at a copy's rate.  Of
// more rows by the vector memory unit of a CU, through which a workgroup's rows of x go as its weights do (64 rows of 12288 -> 4096: 16.0; with
// each scale of a row loaded by itself 22.3).  So as many channels a workgroup as leave one for most CUs.  us, row blocks x wavefronts:
//   rows     weights          places    1 x 8   2 x 8   4 x 8   4 x 4
//     16    4096 ->  4096        64       5.6     6.0
//     16   12288 ->  4096        64       8.9    11.1    14.5    14.6
//     64   12288 ->  4096        64      16.1    18.5    23.8    25.1
//     64    8192 ->  8192       128      19.9    14.9    18.1    18.8
//    128   12288 ->  4096       128      27.1    17.9    22.7    23.9
//     16    4096 -> 12288       192              10.7     8.4     9.1
//    200   12288 ->  4096       256      44.9    31.3    22.5    23.1
//     64    4096 -> 32768       512              27.3    25.1    22.2
//   64 experts, 1024 -> 2048, 256 entries                17.7    14.8
// (Two or four steps in flight a wavefront: the same, but where k has too few for that.  Wavefronts of different workgroups at different steps at a time:
// the same.)
template <int TB>
int pick_few4(const Mx4Product& p, hipStream_t s)
{
    const int64_t n = places(p, 16 * TB);
    if (n >= 192 || (p.out == NM_MX4 && p.gated)) return n <= 256 ? launch_few4<TB, 4, 8>(p, s) : launch_few4<TB, 4, 4>(p, s);
    if (n >= 128 || p.out == NM_MX4) return launch_few4<TB, 2, 8>(p, s);
    return launch_few4<TB, 1, 8>(p, s);
}

// What runs a call: a tile shape, or the few-row kernels (-1).
struct Mx4Plan {
    int shape = -1;
    int64_t tiles = 0;   // of rows, at most
};

// The tile kernels' shapes.  More rows a workgroup read weights less often and keep the matrix units busier; fewer make more workgroups, and
// leave less of a group's last tile empty.
struct Shape4 {
    int wr, rows, waves, per_cu;      // per_cu: workgroups that a CU holds (by registers)
    float fixed, alone, shared;       // us: of a tile; of a step with one workgroup a CU, with two
};
constexpr Shape4 kShapes4[] = {{4, 128, 4, 2, 5.5f, 0.70f, 1.80f},    // 256 packed channels x 128 rows
                               {4, 64, 4, 2, 5.0f, 0.49f, 1.15f}};

template <int SHAPE, int TB, int NS, bool GATED, int OUT>
int launch_tile4(const Mx4Product& p, const Mx4Plan& pl, hipStream_t s)
{
    constexpr int WR = kShapes4[SHAPE].wr, PER_CU = kShapes4[SHAPE].per_cu;
    using T = Tile4<WR, TB, NS>;
    static_assert(T::kWaves == kShapes4[SHAPE].waves && T::kRows == kShapes4[SHAPE].rows, "kShapes4 describes the kernels");
    const TileBands o{(p.groups + WR - 1) / WR, (int)pl.tiles, 8};
    const int64_t grid = pl.tiles * o.tiles_c;
    if (grid > 0x7fffffff) {
        set_error("%lld tiles: too many", (long long)grid);
        return NM_ERR_SHAPE;
    }
    static unsigned long long done = 0;
    const int rc = allow_lds((const void*)mx4_tile_kernel<WR, TB, NS, PER_CU, GATED, OUT>, T::kLds, &done);
    if (rc != NM_OK) return rc;
    constexpr int64_t kEach = kMaxItems / T::kThreads & ~7;   // (a multiple of the XCDs')
    for (int64_t at = 0; at < grid; at += kEach) {
        const unsigned n = (unsigned)(grid - at < kEach ? grid - at : kEach);
        hipLaunchKernelGGL((mx4_tile_kernel<WR, TB, NS, PER_CU, GATED, OUT>), dim3(n), dim3(T::kThreads), T::kLds, s, p, o, (int)at);
        NM_HIP_CHECK(hipGetLastError());
    }
    return NM_OK;
}

template <bool GATED, int OUT>
int pick_tile4(const Mx4Product& p, const Mx4Plan& pl, hipStream_t s)
{
    if (pl.shape == 0) return launch_tile4<0, 8, 3, GATED, OUT>(p, pl, s);
    return launch_tile4<1, 4, 4, GATED, OUT>(p, pl, s);
}

}  // namespace

// Which kernel, by the rows (of a group, on average) and by the places that there are for workgroups.
// The few-row kernels up to one workgroup a CU (whatever the rows: the tile kernels' few workgroups would take all of K one after another), of one matrix
// also up to 32 rows and, of 640 places at most, 64; of experts up to 10 rows (whose numbers are uneven).  us, few-row and tile kernel:
//   128 x 12288 -> 4096 17.9 and 46, 200 x 4096 -> 4096 11.0 and 12.9, 333 x 4096 -> 4096 17 and 13, 128 x 8192 -> 8192 17.9 and 32, 128 x 4096
//   -> 10240 18.5 and 18.8, 32 x 4096 -> 65536 30 and 31, 48 rows 37 and 32, 64 x 4096 -> 32768 22 and 25; 64 experts, 2048 -> 2 x 1024, of 8 rows each
//   28 and 32, 16 rows 34 and 32, 1024 -> 2048 15.8 and 15.7, 22 and 15.9; 60 experts, 1440 -> 1111, of 9 rows 13.9 and 15.4.
// Of the tile kernels that with the least estimated time: rounds of workgroups over 256 CUs, two a CU; a group leaves five eighths of a tile empty (half,
// but for those of fewer rows than a tile).
// us, 128 rows and 64, weights out of HBM: 512 x 4096 -> 4096 17.2 and 13.3, 2048 x 4096 -> 8192 39 and 55; 64 experts, 2048 -> 2 x 1024, of 64 rows each
// 44 and 41, 128 rows 50 and 53, 256 rows 69 and 77, 512 rows 115 and 129; 256 experts, 2048 -> 2 x 512, of 32 rows 68 and 63; 60 experts, 1440 ->
// 1111, of 200 rows 44 and 43.  8192 x 4096 -> 16384 270 and 330.
// (Dropped: one workgroup after another on a CU's slots, the next tile asked for before the last is stored, 0 to 16 % slower; three workgroups of 64 rows a
// CU, weights one half step ahead, 8 to 11 % faster at 128 to 256 rows of an expert whose weights lie in the last-level cache, 0 to 11 % slower
// out of HBM.)
static Mx4Plan mx4_plan(const Mx4Product& p)
{
    Mx4Plan pl;
    const int groups = !p.grouped ? 1 : p.experts < p.rows ? p.experts : p.rows;
    const int each = (p.rows + groups - 1) / groups;
    const int64_t n = places(p, 64);
    if (p.blocks < 4) return pl;   // (the tile kernels read scales by fours)
    if (n <= 256 || each <= (p.grouped ? 10 : 32) || (!p.grouped && each <= 64 && n <= 640)) return pl;
    float least = 1e30f;
    for (int sh = 0; sh < (int)(sizeof(kShapes4) / sizeof(Shape4)); ++sh) {
        const Shape4& k = kShapes4[sh];
        const int64_t tall = !p.grouped ? (p.rows + k.rows - 1) / k.rows : p.rows / k.rows + (groups * (int64_t)5 + 7) / 8;
        const int64_t tiles = (tall < groups ? groups : tall) * ((p.groups + k.wr - 1) / k.wr);
        const int64_t rounds = tiles / 512, rest = tiles % 512;
        const float us = rounds * (k.fixed + p.steps * k.shared) + (rest ? k.fixed + p.steps * (rest > 256 ? k.shared : k.alone) : 0.0f);
        if (us < least) {
            least = us;
            pl.shape = sh;
        }
    }
    pl.tiles = tiles_of(p, kShapes4[pl.shape].rows);
    return pl;
}

int run_mx4_product(const Mx4Product& p, hipStream_t s)
{
    const Mx4Plan pl = mx4_plan(p);
    if (pl.shape >= 0) {
        if (p.out == NM_MX4) return p.gated ? pick_tile4<true, NM_MX4>(p, pl, s) : pick_tile4<false, NM_MX4>(p, pl, s);
        if (p.out == NM_BF16) return p.gated ? pick_tile4<true, NM_BF16>(p, pl, s) : pick_tile4<false, NM_BF16>(p, pl, s);
        return p.gated ? pick_tile4<true, NM_F32>(p, pl, s) : pick_tile4<false, NM_F32>(p, pl, s);
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
