// Internal launchers of the join with the residual stream (join.hip) and of the
// token log probabilities (logprobs.hip); arguments are validated by
// api_block.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rmm {

// ------------------------------------------------------------------ join
// h = rs * r + gate * (post ? y * inv_rms(y) * gpost : y), stored to H; x = h *
// inv_rms(h) * gpre.  Rows are numbered over the units (units are M * ld apart).
struct JoinArgs {
    const void *y, *r;               // either may be null
    void *h, *x;                     // either may be null
    const void *gpost, *gpre, *gate; // null: ones
    int64_t ldy, ldr, ldh, ldx;
    int64_t gate_unit, gate_row;     // strides of the gate (0: shared)
    int64_t M, rows;                 // rows per unit, rows over all units
    int K, post;
    float rs, eps;
    float *rscale;                   // [rows] 1 / rms of the stored h, or null
};
constexpr int64_t kJoinMaxK = 65536;
// y_bf16: type of y, the gains, the gate and x; stream_bf16: of r and h
hipError_t launch_join_rows(const JoinArgs &a, bool y_bf16, bool stream_bf16, hipStream_t stream);
// Xt[b][j][m] = bf16(H[b][m][j] * rscale[b][m] * gpre[j]) and the column energies
// of Xt; out: energy itself when splits == 1, else [B][splits][K] partials
int64_t join_splits(int64_t B, int64_t M, int64_t K);
hipError_t launch_join_kmajor(const void *H, bool stream_bf16, int64_t ldh, const float *rscale, const uint16_t *gpre,
                              int64_t B, int64_t M, int64_t K, uint16_t *Xt, int64_t ldxt, double *partials,
                              double *energy, hipStream_t stream);

// -------------------------------------------------------------- logprobs
struct LogprobArgs {
    const void *z;                   // [T] rows of V logits
    int64_t ld, T;
    int V, pieces, given, top;
    float c;                         // scale * log2(e)
    const int32_t *tokens;           // [T][given]
    float *logp, *entropy;           // [T][given], [T] or null
    int32_t *top_idx;                // [T][top] or null
    float *top_logp;
    void *part;                      // pieces > 1: partial results
};
constexpr int kMaxTop = 64;
int logprob_pieces(int64_t T, int64_t V);
size_t logprob_workspace_bytes(int64_t T, int64_t V, int64_t top);
hipError_t launch_logprobs(const LogprobArgs &a, bool bf16, hipStream_t stream);

}  // namespace rmm
