// Device code that the product kernels in MX4 share: the matrix instruction, which rows a tile has, the epilogue.
#pragma once

#include "nm_mx4_device.h"
#include "nm_q8_product.h"

namespace nm {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// 16 rows of weights times 16 rows of x over 128 k.  OW and OX: the byte of the scales' words that this instruction takes.
template <int OW, int OX>
__device__ inline f32x4 mma4(i32x4 w, i32x4 x, f32x4 acc, unsigned ws, unsigned xs)
{
    const i32x8 a = __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1), b = __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, OW, (int)ws, OX, (int)xs);
}

// Rows of y that a workgroup has, and whose weights they meet.
struct RowTile {
    int expert, count, row0;
};

// The tiles of `per` rows that the groups have, one group's after another's.  A lane looks at (experts + 63) / 64 adjacent groups; every
// wavefront for itself.
struct GroupTiles {
    int per, each, mine, upto;   // groups of a lane; tiles of its groups, and of those and all before
    int all;
    int first, count;            // row and rows of the lane's first group

    // (values outside the rows of y count as the nearer end)
    static __device__ inline void range(const Mx4Product& p, int e, int& begin, int& n)
    {
        const int in = e < p.experts ? e : p.experts - 1;
        begin = min(max(p.offsets[in], 0), p.rows);
        const int end = min(max(p.offsets[in + 1], 0), p.rows);
        n = e < p.experts ? max(end - begin, 0) : 0;
    }
    // the sum of a lane's v and of all lanes' before it
    static __device__ inline int scan(int v)
    {
        v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // within sixteen lanes: the one 1 below,
        v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);   // 2,
        v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);   // 4
        v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);   // and 8 below
        v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // the last of lanes 0 - 15 and 32 - 47 to the sixteen after
        v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // lane 31 to the upper half
        return v;
    }
    __device__ inline GroupTiles(const Mx4Product& p, int tile_rows) : per(tile_rows), each((p.experts + 63) >> 6)
    {
        const int lane = threadIdx.x & 63;
        int m = 0, to = 0, n = (int)((p.rows + (int64_t)tile_rows - 1) / tile_rows), b0 = 0, n0 = 0;
        if (p.grouped) {
            range(p, lane * each, b0, n0);
            m = (n0 + tile_rows - 1) / tile_rows;
#pragma unroll 4
            for (int i = 1; i < each; ++i) {
                int b, k;
                range(p, lane * each + i, b, k);
                m += (k + tile_rows - 1) / tile_rows;
            }
            to = scan(m);
            n = __builtin_amdgcn_readlane(to, 63);
        }
        mine = m;
        upto = to;
        all = n;
        first = b0;
        count = n0;
    }
    // Tile number `tile`; count is 0 past the last one.
    __device__ inline RowTile at(const Mx4Product& p, int tile) const
    {
        if (!p.grouped) return {0, __builtin_amdgcn_readfirstlane(max(min(p.rows - tile * per, per), 0)), __builtin_amdgcn_readfirstlane(tile * per)};
        int expert = 0, row0 = 0, n = 0, before = upto - mine;
        for (int i = 0; i < each; ++i) {   // (every lane as if the tile were of its groups)
            const int e = (threadIdx.x & 63) * each + i, in = tile - before;
            int b = first, k = count;
            if (i) range(p, e, b, k);
            const bool here = in >= 0 && in * (int64_t)per < k;
            expert = here ? e : expert;
            row0 = here ? b + in * per : row0;
            n = here ? min(k - in * per, per) : n;
            before += (k + per - 1) / per;
        }
        const int l = tile < all ? __ffsll(__ballot(upto > tile)) - 1 : 0;
        return {__builtin_amdgcn_readlane(expert, l), tile < all ? __builtin_amdgcn_readlane(n, l) : 0, __builtin_amdgcn_readlane(row0, l)};
    }
};

// Where row `row` of a tile comes from: rows of x from `base` on that the kernels' buffers begin with.  -1: nowhere.
__device__ inline int source_of(const Mx4Product& p, const RowTile& t, int row)
{
    if (row >= t.count) return -1;
    if (!p.index) return row;
    const int at = p.index[(int64_t)t.row0 + row];
    return (unsigned)at < (unsigned)p.sources ? at : -2;   // -2: an index outside x
}

// The buffer of the codes of a tile's rows.
__device__ inline __amdgpu_buffer_rsrc_t row_buffer(const Mx4Product& p, const RowTile& t)
{
    const int64_t first = p.index ? 0 : t.row0, rows = p.index ? p.sources : t.count;
    return q8_rsrc(p.q + first * p.ldq, (unsigned)((rows - 1) * p.ldq + p.blocks * 16));
}

// The scales of a row's last step, of which `have` < 8 are there; the others are 1 (the codes there meet zeros).
__device__ inline u32x2 last_scales(const uint8_t* from, int have)
{
    u32x2 v = {0x7f7f7f7fu, 0x7f7f7f7fu};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < have) v[i >> 2] = (v[i >> 2] & ~(0xffu << (8 * (i & 3)))) | (unsigned)from[i] << (8 * (i & 3));
    return v;
}

// What a lane needs of the channels it holds over NB blocks (from block b0 on) of one row group: one run of adjacent outputs, or two.
template <bool GATED, int NB> struct Channels4 {
    static constexpr int kRun = GATED ? 2 * NB : NB < 2 ? 4 * NB : 8, kRuns = (GATED ? 2 : 4) * NB / kRun;
    int c0;   // first output of the first run; the second is 32 further on
    f32x4 bias[NB];

    __device__ inline void load(const Mx4Product& p, int expert, int group, int b0, int lane)
    {
        const int g = lane >> 4, half = p.channels / 2;
        c0 = GATED ? group * 32 + g * 8 + b0 * 2 : group * 64 + (b0 >> 1) * 32 + g * 8 + (b0 & 1) * 4;
        const float* from = p.bias ? p.bias + (int64_t)expert * p.channels : nullptr;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            bias[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (from) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if constexpr (GATED) {
                        const int o = c0 + 2 * b + (r & 1);
                        if (o < half) bias[b][r] = from[r < 2 ? o : half + o];
                    } else {
                        const int c = c0 + (b >> 1) * 32 + (b & 1) * 4 + r;
                        if (c < p.channels) bias[b][r] = from[c];
                    }
                }
            }
        }
    }
};

// silu(gate) * up, with s = exp(-|gate| / 2): gate / (1 + s^2) for gates that are not negative, otherwise gate s / (1 + s^2) times s up.  Nothing
// on the way leaves fp32's range before the result does, down to gates of -174 (s^2 as one number would at -87, and the reciprocal of
// 1 + exp(-gate) is 0 there).  Under -174.7 s is 0, and so is the result.
// u = 2^-24: s is within (|gate| + 2) u (its argument's constant and rounding, then 2 u of the instruction), the reciprocal within 2 u, the
// sum and the four products round once each, and s counts twice at most: (2 |gate| + 12) u in all.  The gate itself is a sum of 128
// products and more in fp32, of whose roundings silu takes over |gate| times as much: a quotient to the last bit would not show.
__device__ inline float silu4(float gate, float up)
{
    const float s = __builtin_amdgcn_exp2f(fabsf(gate) * -0.72134752f), r = __builtin_amdgcn_rcpf(fmaf(s, s, 1.0f));   // log2(e) / 2
    const float t = gate < 0.0f ? s : 1.0f;
    return gate * r * t * (up * t);
}

// The outputs of run `run` of a lane's sums for one row, in fp32.
template <bool GATED, int NB>
__device__ inline void outputs4(const Channels4<GATED, NB>& ch, const f32x4 (&acc)[NB], int run, float (&y)[Channels4<GATED, NB>::kRun])
{
    constexpr int PER = NB / Channels4<GATED, NB>::kRuns;   // blocks of a run
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = run * PER + i;
        const f32x4 z = acc[b] + ch.bias[b];
        if constexpr (GATED) {
            y[2 * i] = silu4(z[0], z[2]);
            y[2 * i + 1] = silu4(z[1], z[3]);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) y[4 * i + r] = z[r];
        }
    }
}

// The largest over the lanes l, l ^ 16, l ^ 32, l ^ 48 (all four active): a block of 32 outputs of one row.
__device__ inline unsigned column_max(unsigned m)
{
    const u32x2 a = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    m = max(a[0], a[1]);
    const u32x2 b = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    return max(b[0], b[1]);
}

// Eight adjacent outputs of a lane, whose block of 32 the lanes l ^ 16, l ^ 32 and l ^ 48 share, as codes and the block's scale.  (Outputs
// past the last channel are zeros.)
__device__ inline unsigned rounded8(const float (&y)[8], unsigned& scale)
{
    unsigned most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, magnitude(y[e]));
    scale = mx4_scale(column_max(most));
    return mx4_codes(y, scale);
}

// Stores a lane's outputs of one row straight from the registers.  All lanes of a wavefront come here, also for rows that are not stored.
template <bool GATED, int NB>
__device__ inline void emit4(const Mx4Product& p, const Channels4<GATED, NB>& ch, const f32x4 (&acc)[NB], int64_t row, bool there)
{
    using C = Channels4<GATED, NB>;
    constexpr int N = C::kRun;
#pragma unroll
    for (int run = 0; run < C::kRuns; ++run) {
        const int c0 = ch.c0 + run * 32;
        float y[N];
        outputs4<GATED, NB>(ch, acc, run, y);
        if constexpr (N == 8) {
            if (p.out == NM_MX4) {
                unsigned scale;
                const unsigned codes = rounded8(y, scale);
                const int block = c0 >> 5;
                if (there && block * 32 < p.outs) {
                    *reinterpret_cast<unsigned*>((uint8_t*)p.y + row * p.ldy + (size_t)(c0 >> 3) * 4) = codes;
                    if ((c0 & 31) == 0) p.ys[row * p.ldys + block] = (uint8_t)scale;
                }
                continue;
            }
        }
        if (!there) continue;
        auto store = [&](auto bf16) {
            constexpr bool BF16 = decltype(bf16)::value;
            constexpr int ES = Elem<BF16>::kBytes;
            char* py = (char*)p.y + row * p.ldy * ES;
            const char* pr = !GATED && p.res ? (const char*)p.res + row * p.ldr * ES : nullptr;
            if constexpr (N == 8) {
                if (c0 + 8 <= p.outs) {
                    if (pr) {
                        float r[8];
                        Elem<BF16>::load8(pr + (int64_t)c0 * ES, r);
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] += r[e];
                    }
                    Elem<BF16>::store8(py + (int64_t)c0 * ES, y);
                    return;
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (c0 + i < p.outs) {
                    if (pr) y[i] += Elem<BF16>::load1(pr + (int64_t)(c0 + i) * ES);
                    Elem<BF16>::store1(py + (int64_t)(c0 + i) * ES, y[i]);
                }
            }
        };
        if (p.out == NM_BF16) store(std::true_type{});
        else store(std::false_type{});
    }
}

// Tile of a workgroup.  Workgroups go to the eight XCDs, each with an L2 of its own, in turn by their number: every XCD gets a run of
// adjacent tiles, in bands of `band` tiles of rows, whose weights it reads once.
struct TileBands {
    int tiles_c, tiles_r, band;
    __host__ __device__ inline int tiles() const { return tiles_c * tiles_r; }
    __device__ inline void at(int block, int& tc, int& tr) const
    {
        const int n = tiles(), xcd = block & 7, more = n & 7;
        const int tile = xcd * (n >> 3) + (xcd < more ? xcd : more) + (block >> 3);
        const int b = tile / (band * tiles_c), in = tile - b * band * tiles_c;
        const int h = tiles_r - b * band < band ? tiles_r - b * band : band;
        tc = in / h;
        tr = b * band + in % h;
    }
};

}  // namespace nm
