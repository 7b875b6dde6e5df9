// Shared by the translation units of the 8-bit feed-forward operators.
#pragma once

#include <string.h>

#include "nm_internal.h"
#include "nm_q8.h"

// Packed weights.  A packed row group is 64 channels; its rows lie as the 16x16x64 integer matrix
// instruction reads them, so that a wavefront's load of 16 channels x 64 k is 1 KiB of adjacent bytes:
//   d_w [groups][kblocks][4 blocks][64 lanes][16 bytes]
//       lane l of block b holds packed row 16 b + l % 16, k = 64 kblock + 16 (l / 16) .. + 15
// The instruction gives lane l the rows 4 (l / 16) .. + 3 of a block, so the channels are dealt to packed
// rows in the order that leaves a lane with adjacent channels over the four blocks (q8_row_of).
// Rows and k past the ends are zero: whatever finite bytes meet them add nothing.
struct nm_q8 {
    int device = -1;
    int channels = 0, width = 0, gated = 0;
    int groups = 0;        // of 64 packed rows
    int kblocks = 0;       // of 64 k, an even number
    int8_t* d_w = nullptr;
    float* d_scales = nullptr;   // [groups * 64] in packed-row order, 0 in padding rows
};

namespace nm {

// Channel (row of the caller's weight matrix) of packed row p, or -1 for padding.
//   plain: block b, row 4 g + r of group G <-> channel 64 G + 32 (b / 2) + 8 g + 4 (b & 1) + r  (twice 8 adjacent ones a lane)
//   gated: r < 2 the gate, r >= 2 the value of output 32 G + 8 g + 2 b + (r & 1)                (8 adjacent outputs a lane)
// Eight bf16 are the 16 bytes that a lane stores at once, and the four g of a row then store 64 adjacent bytes.
__host__ __device__ inline int q8_row_of(int p, int channels, int gated)
{
    const int G = p >> 6, b = (p >> 4) & 3, g = (p >> 2) & 3, r = p & 3;
    if (!gated) {
        const int c = G * 64 + (b >> 1) * 32 + g * 8 + (b & 1) * 4 + r;
        return c < channels ? c : -1;
    }
    const int o = G * 32 + g * 8 + b * 2 + (r & 1), half = channels / 2;
    return o < half ? (r < 2 ? o : half + o) : -1;
}

// row operators (nm_q8_rows.hip)
int run_q8_rows(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, const void* res, int64_t ldr,
                const float* gamma, float eps, bool norm, void* out, int64_t ldo, int8_t* q, int64_t ldq, float* scales,
                hipStream_t s);
int run_q8_dequantize(const int8_t* q, int64_t ldq, const float* scales, int64_t rows, int width, void* y, nm_dtype_t dt,
                      int64_t ldy, hipStream_t s);

// weights and products (nm_q8_linear.hip)
int run_q8_pack(const int8_t* w, int64_t ldw, const float* scales, const nm_q8* h, int* d_bad, hipStream_t s);
int run_q8_unpack(const nm_q8* h, int8_t* w, float* scales, hipStream_t s);

struct Q8Linear {
    const int8_t* q;
    const float* qs;
    const int8_t* w;
    const float* ws;
    const float* bias;
    const void* res;
    void* y;
    int64_t ldq, ldr, ldy;
    int rows, width, channels, outs;   // outs: channels of y
    int gated, groups, kblocks, y_bf16;
    int past;   // y is stored past the last-level cache
};
// What runs a call: a tile shape and the parts that K is cut into; and the workspace: rows of q at a stride that the kernels can read,
// if theirs is none, then the parts of a divided sum.
struct Q8Plan {
    int shape = -1;    // -1: the few-row kernels
    int splits = 1;
    int per = 0;       // K steps of a part
    size_t rows_bytes = 0, part_bytes = 0;
};
Q8Plan q8_plan(const Q8Linear& p);
int run_q8_linear(const Q8Linear& p, const Q8Plan& plan, void* workspace, hipStream_t s);

}  // namespace nm
