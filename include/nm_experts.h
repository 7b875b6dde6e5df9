/*
 * nm_experts.h -- C ABI of libnmconv: routing of tokens to experts and the sum of what the experts answer.
 *
 * Conventions are those of nm_q8.h: calls enqueue on `hip_stream` of the current device, allocate nothing and never wait, and
 * may be captured into a graph; no output may overlap an input but where that is said.
 */
#ifndef NM_EXPERTS_H
#define NM_EXPERTS_H

#include "nm_mx4.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { NM_ROUTE_MAX_EXPERTS = 1024, NM_ROUTE_MAX_CHOICES = 64, NM_ROUTE_ONE_LAUNCH = 64 };

/*
 * nm_route -- each token's `choices` largest logits and the order of the tokens by expert:
 *   ids      int32 [tokens][choices]  the experts, largest logit first, of equal logits the lowest expert first
 *   weights  fp32 [tokens][choices]   exp(l_j - l_0) / sum, the sum over the token's choices (normalise = 1) or over all
 *                                     its experts (normalise = 0)
 *   offsets  int32 [experts + 1]      expert e has the entries offsets[e] .. offsets[e + 1] - 1
 *   rows     int32 [tokens * choices] the token of an entry; an expert's entries go by token.  -1 past the last entry
 *   slots    int32 [tokens][choices]  the entry of a choice
 * An expert whose logit is minus infinity is closed to the token: where fewer than `choices` are open the last ids and slots are
 * -1, their weights 0.  A token with no open expert (padding) makes no entry.  A NaN counts as the largest logit; the weights of a
 * token that has one, or a logit of plus infinity, are NaN.
 *   logits_dev   rows of dtype (NM_F32 or NM_BF16) at stride ld
 *   1 <= experts <= NM_ROUTE_MAX_EXPERTS, 1 <= choices <= min(experts, NM_ROUTE_MAX_CHOICES), 0 <= tokens * choices < 2^31
 *   (no tokens: offsets are still written)
 *   workspace_dev  at least nm_route_workspace() bytes, 16-byte aligned (none for up to NM_ROUTE_ONE_LAUNCH tokens)
 */
int nm_route(const void* logits_dev, nm_dtype_t dtype, int64_t tokens, int experts, int64_t ld, int choices, int normalise,
             int32_t* ids_dev, float* weights_dev, int32_t* offsets_dev, int32_t* rows_dev, int32_t* slots_dev,
             void* workspace_dev, size_t workspace_bytes, void* hip_stream);

int nm_route_workspace(int64_t tokens, int experts, size_t* bytes);

/*
 * nm_combine -- out_t = residual_t + sum_j weights_tj * y_(slots_tj), summed in fp32 in the order of j, rounded once.
 *   y_dev         rows of y_dtype (NM_F32 or NM_BF16) at stride ldy; entries of them
 *   slots_dev     int32 [tokens][choices]; -1 adds nothing, another value outside [0, entries) makes the row NaN
 *   weights_dev   fp32 [tokens][choices]
 *   residual_dev  rows of dtype at stride ldr, or NULL.  It may be out_dev itself (same stride).
 *   out_dev       rows of dtype (NM_F32 or NM_BF16) at stride ldo >= width
 *   1 <= width <= NM_Q8_MAX_WIDTH, 1 <= choices <= NM_ROUTE_MAX_CHOICES
 */
int nm_combine(const void* y_dev, nm_dtype_t y_dtype, int64_t entries, int64_t ldy, const int32_t* slots_dev,
               const float* weights_dev, int64_t tokens, int choices, int width, const void* residual_dev, int64_t ldr,
               void* out_dev, nm_dtype_t dtype, int64_t ldo, void* hip_stream);

/* The calls above with their arguments in one block. */
typedef struct nm_route_args {
    const void* logits_dev;
    int32_t* ids_dev;
    float* weights_dev;
    int32_t* offsets_dev;
    int32_t* rows_dev;
    int32_t* slots_dev;
    void* workspace_dev;
    void* hip_stream;
    int64_t dtype, tokens, experts, ld, choices, normalise, workspace_bytes;
} nm_route_args_t;
int nm_route_args(const nm_route_args_t* args);

typedef struct nm_combine_args {
    const void* y_dev;
    const int32_t* slots_dev;
    const float* weights_dev;
    const void* residual_dev;
    void* out_dev;
    void* hip_stream;
    int64_t y_dtype, entries, ldy, tokens, choices, width, ldr, dtype, ldo;
} nm_combine_args_t;
int nm_combine_args(const nm_combine_args_t* args);

#ifdef __cplusplus
}
#endif
#endif /* NM_EXPERTS_H */
