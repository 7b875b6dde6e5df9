// Device code that the product kernels in 8 bits share: the matrix instruction, loads into LDS, the order of tiles, the epilogue.
#pragma once

#include <type_traits>

#include "nm_q8_device.h"

namespace nm {

constexpr unsigned kPast = 0xfffffff0u;   // an offset past the end of every buffer here

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr_t;

__device__ inline __amdgpu_buffer_rsrc_t q8_rsrc(const void* p, unsigned bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

__device__ inline i32x4 mma(i32x4 w, i32x4 q, i32x4 acc) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, q, acc, 0, 0, 0); }

// Bytes from the first of `rows` rows of q to the end of the last 16-byte unit that holds a value of them.  Kernels read q (16-byte
// aligned in address and stride) through a buffer of this size: past it, zeros come back.  What a row's loads bring from past its end
// meets zero weights, whatever it is: the gap to the next row, that row, or up to 15 bytes after the tensor that share the aligned 16
// of its last value, and so its page.
__device__ inline unsigned rows_extent(const Q8Linear& p, int rows) { return (unsigned)((rows - 1) * p.ldq + ((p.width + 15) & ~15)); }

// 16 bytes of a row from byte c on, zeros past its end; the row may begin at any address.
__device__ inline i32x4 load16(const int8_t* row, int c, int width)
{
    i32x4 v = {0, 0, 0, 0};
    if (c + 16 <= width) {
        __builtin_memcpy(&v, row + c, 16);
    } else if (c < width && width >= 16) {   // the row's last 16, moved down to where its end is
        unsigned __int128 u;
        __builtin_memcpy(&u, row + width - 16, 16);
        u >>= 8 * (c + 16 - width);
        __builtin_memcpy(&v, &u, 16);
    } else {
        for (int e = 0; c + e < width; ++e) {
            const int b = (int)(unsigned char)row[c + e] << (8 * (e & 3));
#pragma unroll
            for (int d = 0; d < 4; ++d) v[d] |= (e >> 2) == d ? b : 0;
        }
    }
    return v;
}

// What a lane needs of the channels it holds over NB blocks (from block b0 on) of one row group: one run of adjacent outputs, or two.
template <bool GATED, int NB> struct Channels {
    static constexpr int kRun = GATED ? 2 * NB : NB < 2 ? 4 * NB : 8, kRuns = (GATED ? 2 : 4) * NB / kRun;
    int c0;   // first output of the first run; the second is 32 further on
    f32x4 t[NB], bias[NB];

    __device__ inline void load(const Q8Linear& p, int group, int b0, int lane)
    {
        const int g = lane >> 4, half = p.channels / 2;
        c0 = GATED ? group * 32 + g * 8 + b0 * 2 : group * 64 + (b0 >> 1) * 32 + g * 8 + (b0 & 1) * 4;
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
                        const int c = c0 + (b >> 1) * 32 + (b & 1) * 4 + r;
                        if (c < p.channels) bias[b][r] = p.bias[c];
                    }
                }
            }
        }
    }
};

// __expf's relative error, 2 |gate| u with u = 2^-24, is that of a gate moved by two roundings; the gate itself carries the three of its product,
// sum and bias.  expf, within 2 u, would cost 3 to 6 % of a product (300 x 4096 -> 2 x 8192 22.3 us and 23.8, 4096 x 4096 -> 2 x 12288 323 and 338).
__device__ inline float silu_times(float gate, float up) { return gate / (1.0f + __expf(-gate)) * up; }

// 16 bytes of the output, through the L2 as they come (agent scope: at a kernel's end each XCD's L2 would have to write back what it
// still holds), or past the 256 MB last-level cache too where that would not hold the output until it is read.
typedef u32x4 __attribute__((aligned(2))) u32x4_anywhere;
__device__ inline void store16(char* p, u32x4 v, bool past)
{
    if (past) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_anywhere*>(p));
    else __builtin_amdgcn_global_store_b128((__attribute__((address_space(1))) u32x4*)p, v, "agent");
}

// The outputs of run `run` of a lane's sums for one row of q with scale s, in fp32.
template <bool GATED, int NB>
__device__ inline void outputs(const Channels<GATED, NB>& ch, const i32x4 (&acc)[NB], float s, int run, float (&y)[Channels<GATED, NB>::kRun])
{
    constexpr int PER = NB / Channels<GATED, NB>::kRuns;   // blocks of a run
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = run * PER + i;
        float z[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) z[r] = fmaf((float)acc[b][r], s * ch.t[b][r], ch.bias[b][r]);
        if constexpr (GATED) {
            y[2 * i] = silu_times(z[0], z[2]);
            y[2 * i + 1] = silu_times(z[1], z[3]);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) y[4 * i + r] = z[r];
        }
    }
}

// Stores them straight from the registers: 64 adjacent bytes of a row at a time at best.
template <bool GATED, bool BF16, int NB>
__device__ inline void emit(const Q8Linear& p, const Channels<GATED, NB>& ch, const i32x4 (&acc)[NB], int64_t row, float s)
{
    using C = Channels<GATED, NB>;
    constexpr int N = C::kRun, ES = Elem<BF16>::kBytes;
    char* py = (char*)p.y + row * p.ldy * ES;
    const char* pr = !GATED && p.res ? (const char*)p.res + row * p.ldr * ES : nullptr;
#pragma unroll
    for (int run = 0; run < C::kRuns; ++run) {
        const int c0 = ch.c0 + run * 32;
        float y[N];
        outputs<GATED, NB>(ch, acc, s, run, y);
        bool whole = false;
        if constexpr (N == 8) {
            whole = c0 + 8 <= p.outs;
            if (whole) {
                if (pr) {
                    float r[8];
                    Elem<BF16>::load8(pr + (int64_t)c0 * ES, r);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] += r[e];
                }
                Elem<BF16>::store8(py + (int64_t)c0 * ES, y);
            }
        }
        if (!whole) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (c0 + i < p.outs) {
                    if (pr) y[i] += Elem<BF16>::load1(pr + (int64_t)(c0 + i) * ES);
                    Elem<BF16>::store1(py + (int64_t)(c0 + i) * ES, y[i]);
                }
            }
        }
    }
}

// A workgroup's outputs through LDS, so that whole rows of its tile are stored, 16 bytes a thread and adjacent threads adjacent:
// straight from the registers (above) a store instruction reaches 16 rows with 64 bytes each, and 8192 x 4096 -> 16384 took 2.6 %
// longer, 8000 x 2000 -> 5000 (rows that begin in the middle of a line) 7 % (in turn, 433 us and 422, 99 and 92).  JP of the TB blocks of rows
// at a time, STAGE32 in fp32 (for a residual, so that it rounds once).  The 16-byte pieces of a row lie at piece ^ (row & 7).
template <int WR, int WT, int TB, int JP, bool STAGE32, bool GATED, bool BF16, typename Scale>
__device__ inline void store_tile(const Q8Linear& p, const Channels<GATED, 4>& ch, Scale scale, const i32x4 (&acc)[TB][4], char* smem,
                                  int wr, int wt, int lane, int group0, int64_t row0)
{
    constexpr int SB = STAGE32 ? 4 : 2, ES = Elem<BF16>::kBytes, C = Channels<GATED, 4>::kRuns * 8;   // outputs of a group and lane
    constexpr int kOuts = WR * C * 4, kPitch = kOuts * SB, kThreads = WR * WT * 64, kRows = WT * JP * 16;
    const int64_t col0 = (int64_t)group0 * C * 4;
    const bool past = p.past;
#pragma unroll
    for (int j0 = 0; j0 < TB; j0 += JP) {
        __syncthreads();   // the stages, or the outputs before, have been read
#pragma unroll
        for (int jj = 0; jj < JP; ++jj) {
            const int lrow = (wt * JP + jj) * 16 + (lane & 15);
            const float s = scale(j0 + jj);
#pragma unroll
            for (int run = 0; run < Channels<GATED, 4>::kRuns; ++run) {
                float y[8];
                outputs<GATED, 4>(ch, acc[j0 + jj], s, run, y);
                const int c = wr * C * 4 + run * 32 + (lane >> 4) * 8;   // column in the tile
                char* to = smem + lrow * kPitch;
                if constexpr (STAGE32) {
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
        constexpr int kPieces = kOuts * ES / 16;   // of a row, as it is stored
#pragma unroll 4
        for (int u = threadIdx.x; u < kRows * kPieces; u += kThreads) {
            const int lrow = u / kPieces, piece = u % kPieces;
            const int64_t row = row0 + (lrow / (JP * 16)) * TB * 16 + j0 * 16 + lrow % (JP * 16);
            const int64_t col = col0 + piece * (16 / ES);
            if (row >= p.rows || col >= p.outs) continue;
            char* py = (char*)p.y + (row * p.ldy + col) * ES;
            const char* from = smem + lrow * kPitch;
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
            if (col + 16 / ES <= p.outs) {
                store16(py, v, past);
            } else {
#pragma unroll
                for (int e = 0; e < 16 / ES; ++e)
                    if (col + e < p.outs) {
                        if constexpr (BF16) { const unsigned short h = (unsigned short)(v[e / 2] >> (16 * (e & 1))); __builtin_memcpy(py + e * 2, &h, 2); }
                        else { const unsigned w = v[e]; __builtin_memcpy(py + e * 4, &w, 4); }
                    }
            }
        }
    }
}

// Tile of a workgroup.  Workgroups go to the eight XCDs, each with an L2 of its own, in turn by their number: every XCD gets
// a run of adjacent tiles, in bands of up to 4 tiles of rows, so that the 32 of a round share few strips of either operand.
// With `splits` parts of K, a part's tiles follow the part's before.
struct TileOrder {
    int tiles_c, tiles_r, splits;
    __host__ __device__ inline int tiles() const { return tiles_c * tiles_r; }
    __device__ inline void at(int block, int& tc, int& tr, int& tile, int& split) const
    {
        const int n = tiles() * splits, xcd = block & 7, more = n & 7;
        const int unit = xcd * (n >> 3) + (xcd < more ? xcd : more) + (block >> 3);
        split = splits > 1 ? unit / tiles() : 0;
        tile = unit - split * tiles();
        place(tile, tc, tr);
    }
    __device__ inline void place(int tile, int& tc, int& tr) const
    {
        const int band = tile / (4 * tiles_c), in = tile - band * 4 * tiles_c;
        const int h = tiles_r - band * 4 < 4 ? tiles_r - band * 4 : 4;
        tc = in / h;
        tr = band * 4 + in % h;
    }
};

// 16 bytes a lane from memory to LDS at `lds` + 16 * lane.  In asm, so that the compiler does not put a wait for it in front of
// every read of LDS; the kernel waits for it itself.  (m0 is a reserved register: the compiler hands it out to nothing, has no use of its
// own for it in these kernels, and warns of a list of clobbers that names it.)
__device__ inline void load_to_lds(__amdgpu_buffer_rsrc_t r, unsigned voff, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : :
                 "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voff), "s"(r));
}

}  // namespace nm
