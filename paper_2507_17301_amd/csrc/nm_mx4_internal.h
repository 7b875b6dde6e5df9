// Shared by the translation units of the operators in MX4 and of those for experts.
#pragma once

#include "nm_experts.h"
#include "nm_q8_internal.h"

// Packed weights.  Channels are dealt to packed rows as in 8 bits (q8_row_of), 64 of them a row group.  A step is 256 k, 8 blocks; in a
// 16x16x128 matrix instruction, half a step, lane l holds one block of one row.
//   d_w [experts][groups][steps][2 halves][4 blocks of rows][64 lanes][16 bytes]
//       lane l of row block b holds packed row 16 b + l % 16, block of k 8 step + 4 half + l / 16
//   d_s [experts][groups][steps][2 halves][64 lanes] words of four scales, byte b that of row block b
// Rows and blocks past the ends are zeros with the scale 1: whatever numbers meet them add nothing.
struct nm_mx4 {
    int device = -1;
    int experts = 0, channels = 0, width = 0, gated = 0;
    int blocks = 0;        // of 32 k
    int groups = 0;        // of 64 packed rows, of one expert
    int steps = 0;         // of 8 blocks
    uint8_t* d_w = nullptr;
    unsigned* d_s = nullptr;
    size_t w_bytes() const { return (size_t)experts * groups * steps * 8192; }
    size_t s_bytes() const { return (size_t)experts * groups * steps * 512; }
};

namespace nm {

// row operators (nm_mx4_rows.hip)
int run_mx4_rows(const void* x, nm_dtype_t dt, int64_t rows, int width, int64_t ldx, const void* res, int64_t ldr,
                 const float* gamma, double eps, bool norm, void* out, int64_t ldo, uint8_t* q, int64_t ldq, uint8_t* scales,
                 int64_t lds, hipStream_t s);
int run_mx4_dequantize(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, int64_t rows, int width, void* y,
                       nm_dtype_t dt, int64_t ldy, hipStream_t s);

// weights and products (nm_mx4_product.hip)
int run_mx4_pack(const uint8_t* q, int64_t ldq, const uint8_t* scales, int64_t lds, const nm_mx4* h, int* d_bad, hipStream_t s);
int run_mx4_unpack(const nm_mx4* h, uint8_t* q, uint8_t* scales, hipStream_t s);

struct Mx4Product {
    const uint8_t* q;
    const uint8_t* s;
    const uint8_t* w;
    const unsigned* ws;
    const float* bias;
    const void* res;
    void* y;
    uint8_t* ys;
    const int* offsets;   // grouped: of the experts' rows
    const int* index;
    int64_t ldq, lds, ldr, ldy, ldys;
    int rows, sources;    // rows of y, of q
    int channels, outs;   // outs: channels of y
    int grouped, experts, gated, groups, steps, blocks;
    nm_dtype_t out;       // NM_F32, NM_BF16 or NM_MX4
    int past;             // y is stored past the last-level cache
};
int run_mx4_product(const Mx4Product& p, hipStream_t s);

// routing (nm_experts.hip)
struct Route {
    const void* logits;
    int64_t tokens, ld;
    int bf16, experts, choices, normalise;
    int* ids;
    float* weights;
    int* offsets;
    int* rows;
    int* slots;
};
size_t route_workspace(int64_t tokens, int experts);
int run_route(const Route& r, void* workspace, hipStream_t s);

struct Combine {
    const void* y;
    const int* slots;
    const float* weights;
    const void* res;
    void* out;
    int64_t entries, tokens, ldy, ldr, ldo;
    int choices, width, y_bf16, bf16;
};
int run_combine(const Combine& c, hipStream_t s);

}  // namespace nm
