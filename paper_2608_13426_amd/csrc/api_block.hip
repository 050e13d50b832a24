// C-ABI of the products with an epilogue, the join with the residual stream and
// the token log probabilities: host-side validation and dispatch.  Every check
// happens before the first HIP call.
#include <cmath>
#include <cstdint>

#include "../../include/rmm.h"
#include "block.h"
#include "epilogue.h"
#include "kernels.h"

namespace {

constexpr int64_t kInt32Max = 2147483647;
constexpr int64_t kGridYZMax = 65535;
constexpr int64_t kMaxRows = int64_t(1) << 22;     // a launch holds fewer than 2^32 threads

constexpr int64_t kMaxVocab = int64_t(1) << 30;    // a row's indices and its last chunk's end in 32 bits
constexpr int64_t kMaxGiven = int64_t(1) << 30;    // so are a row's given tokens and a thread's step past them

inline size_t align256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }
inline bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline rmm_status_t from_hip(hipError_t e) { return e == hipSuccess ? RMM_OK : RMM_ERR_HIP; }
inline bool valid_dtype(rmm_dtype_t dt) { return dt == RMM_F32 || dt == RMM_BF16; }

// e may be null: no bias, no activation, no residual
rmm_status_t check_epilogue(const rmm_epilogue_t *e, rmm_dtype_t dt, int64_t N, const void *Y, int64_t ldy,
                            rmm::Epilogue *out) {
    *out = {};
    if (!e) return RMM_OK;
    if (e->act < RMM_ACT_NONE || e->act > RMM_ACT_GELU_TANH) return RMM_ERR_INVALID_ARGUMENT;
    if (e->residual && (e->ldr < N || !std::isfinite(e->residual_scale))) return RMM_ERR_INVALID_ARGUMENT;
    if (e->residual == Y && e->ldr != ldy) return RMM_ERR_INVALID_ARGUMENT;
    const size_t size = dt == RMM_BF16 ? 2 : 4;
    if (!aligned(e->bias, size) || !aligned(e->residual, size)) return RMM_ERR_INVALID_ARGUMENT;
    out->bias = e->bias;
    out->res = e->residual;
    out->ldr = e->ldr;
    out->rs = e->residual_scale;
    out->act = e->act;
    return RMM_OK;
}

rmm_status_t check_product(const void *X, const void *W, const int32_t *idx, int64_t B, int64_t M, int64_t N, int64_t K,
                           int64_t k, int64_t ldw, const void *Y, int64_t ldy) {
    if (!X || !W || !idx || !Y) return RMM_ERR_INVALID_ARGUMENT;
    if (B < 1 || M < 1 || N < 1 || K < 1 || k < 1 || k > K) return RMM_ERR_INVALID_ARGUMENT;
    if (ldw < N || ldy < N) return RMM_ERR_INVALID_ARGUMENT;
    if (K > kInt32Max || M > kInt32Max || N > kInt32Max) return RMM_ERR_INVALID_ARGUMENT;
    if (B > kGridYZMax || N > rmm::kMaxStepped || k > rmm::kMaxStepped) return RMM_ERR_UNSUPPORTED;
    return RMM_OK;
}

}  // namespace

extern "C" {

rmm_status_t rmm_reduced_gemm_epilogue(const void *X, const void *W, const int32_t *idx, rmm_dtype_t dtype, int64_t B,
                                       int64_t M, int64_t N, int64_t K, int64_t k, int64_t ldx, int64_t ldw, void *Y,
                                       int64_t ldy, const rmm_epilogue_t *epilogue, hipStream_t stream) {
    if (!valid_dtype(dtype)) return RMM_ERR_INVALID_ARGUMENT;
    rmm_status_t st = check_product(X, W, idx, B, M, N, K, k, ldw, Y, ldy);
    if (st != RMM_OK) return st;
    if (ldx < K) return RMM_ERR_INVALID_ARGUMENT;
    rmm::Epilogue ep;
    st = check_epilogue(epilogue, dtype, N, Y, ldy, &ep);
    if (st != RMM_OK) return st;
    if (M > kGridYZMax * 32) return RMM_ERR_UNSUPPORTED;
    if (dtype == RMM_BF16)
        return from_hip(rmm::launch_gemm_bf16(static_cast<const uint16_t *>(X), static_cast<const uint16_t *>(W), idx, B,
                                              M, N, K, k, ldx, ldw, static_cast<uint16_t *>(Y), ldy, &ep, stream));
    return from_hip(rmm::launch_gemm_f32(static_cast<const float *>(X), static_cast<const float *>(W), idx, B, M, N, K, k,
                                         ldx, ldw, static_cast<float *>(Y), ldy, &ep, stream));
}

rmm_status_t rmm_reduced_gemm_kmajor_epilogue(const void *Xt, const void *W, const int32_t *idx, int64_t B, int64_t M,
                                              int64_t N, int64_t K, int64_t k, int64_t ldxt, int64_t ldw, void *Y,
                                              int64_t ldy, const rmm_epilogue_t *epilogue, hipStream_t stream) {
    rmm_status_t st = check_product(Xt, W, idx, B, M, N, K, k, ldw, Y, ldy);
    if (st != RMM_OK) return st;
    if (ldxt < M) return RMM_ERR_INVALID_ARGUMENT;
    rmm::Epilogue ep;
    st = check_epilogue(epilogue, RMM_BF16, N, Y, ldy, &ep);
    if (st != RMM_OK) return st;
    // 16-byte vectors through descriptors whose byte offsets stay below 2^31
    const int64_t lim = int64_t(1) << 31;
    if (!aligned(Xt, 16) || !aligned(W, 16) || ldxt % 8 || ldw % 8 || K * ldxt * 2 + ldxt * 2 >= lim ||
        K * ldw * 2 + ldw * 2 >= lim)
        return RMM_ERR_UNSUPPORTED;
    return from_hip(rmm::launch_gemm_kmajor_bf16(static_cast<const uint16_t *>(Xt), static_cast<const uint16_t *>(W), idx,
                                                 B, M, N, K, k, ldxt, ldw, static_cast<uint16_t *>(Y), ldy, &ep, stream));
}

rmm_status_t rmm_reduced_gemv_epilogue(const void *X, const void *W, const int32_t *idx, int64_t B, int64_t M, int64_t N,
                                       int64_t K, int64_t k, int64_t ldx, int64_t ldw, void *Y, int64_t ldy,
                                       const rmm_epilogue_t *epilogue, void *workspace, size_t workspace_bytes,
                                       hipStream_t stream) {
    rmm_status_t st = check_product(X, W, idx, B, M, N, K, k, ldw, Y, ldy);
    if (st != RMM_OK) return st;
    if (ldx < K) return RMM_ERR_INVALID_ARGUMENT;
    rmm::Epilogue ep;
    st = check_epilogue(epilogue, RMM_BF16, N, Y, ldy, &ep);
    if (st != RMM_OK) return st;
    if (M > 8 || K * ldw * 2 >= (int64_t(1) << 31)) return RMM_ERR_UNSUPPORTED;
    const size_t need = rmm::gemv_workspace_bytes(B, M, N, k);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return RMM_ERR_WORKSPACE_TOO_SMALL;
        if (!aligned(workspace, 16)) return RMM_ERR_INVALID_ARGUMENT;
    }
    return from_hip(rmm::launch_gemv_bf16(static_cast<const uint16_t *>(X), static_cast<const uint16_t *>(W), idx, B, M, N,
                                          K, k, ldx, ldw, static_cast<uint16_t *>(Y), ldy, workspace, &ep, stream));
}

size_t rmm_block_join_workspace_size(int64_t B, int64_t M, int64_t K) {
    if (B < 1 || M < 1 || K < 1 || K > rmm::kJoinMaxK || B > kGridYZMax || M >= kMaxRows / B) return 0;
    const int64_t S = rmm::join_splits(B, M, K);
    return align256(static_cast<size_t>(B * M) * sizeof(float)) +
           (S == 1 ? 0 : align256(static_cast<size_t>(B * S * K) * sizeof(double)));
}

rmm_status_t rmm_block_join(const rmm_join_t *j, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!j || !valid_dtype(j->dtype) || !valid_dtype(j->stream_dtype)) return RMM_ERR_INVALID_ARGUMENT;
    const int64_t B = j->B, M = j->M, K = j->K;
    if (B < 1 || M < 1 || K < 1) return RMM_ERR_INVALID_ARGUMENT;
    if ((!j->Y && !j->R) || (!j->H && !j->X && !j->Xt) || !j->Xt != !j->energy) return RMM_ERR_INVALID_ARGUMENT;
    if (!j->Y && (j->post_norm || j->gate)) return RMM_ERR_INVALID_ARGUMENT;
    if ((j->Y && j->ldy < K) || (j->R && j->ldr < K) || (j->H && j->ldh < K) || (j->X && j->ldx < K) ||
        (j->Xt && j->ldxt < M))
        return RMM_ERR_INVALID_ARGUMENT;
    if (j->gate && (j->gate_unit_stride < 0 || j->gate_row_stride < 0)) return RMM_ERR_INVALID_ARGUMENT;
    if (!(j->eps >= 0.f) || std::isinf(j->eps) || (j->R && !std::isfinite(j->residual_scale))) return RMM_ERR_INVALID_ARGUMENT;
    // in place only row for row
    if ((j->H && j->H == j->R && j->ldh != j->ldr) || (j->X && j->X == j->Y && j->ldx != j->ldy)) return RMM_ERR_INVALID_ARGUMENT;
    const size_t size = j->dtype == RMM_BF16 ? 2 : 4, ssize = j->stream_dtype == RMM_BF16 ? 2 : 4;
    if (!aligned(j->Y, size) || !aligned(j->X, size) || !aligned(j->post_gamma, size) || !aligned(j->pre_gamma, size) ||
        !aligned(j->gate, size) || !aligned(j->R, ssize) || !aligned(j->H, ssize) || !aligned(j->energy, 8))
        return RMM_ERR_INVALID_ARGUMENT;
    if ((j->X && j->Xt) || (j->dtype == RMM_F32 && j->stream_dtype != RMM_F32)) return RMM_ERR_UNSUPPORTED;
    if (K > rmm::kJoinMaxK || B > kGridYZMax || M >= kMaxRows / B) return RMM_ERR_UNSUPPORTED;
    if (j->Xt) {
        if (!j->H) return RMM_ERR_INVALID_ARGUMENT;
        if (j->dtype != RMM_BF16 || K % 8 || j->ldxt % 8 || !aligned(j->Xt, 16) || !aligned(j->H, 16) ||
            j->ldh * ssize % 16 || !aligned(j->pre_gamma, 16))
            return RMM_ERR_UNSUPPORTED;
    }
    rmm::JoinArgs a = {};
    a.y = j->Y;
    a.r = j->R;
    a.h = j->H;
    a.x = j->X;
    a.gpost = j->post_gamma;
    a.gpre = j->pre_gamma;
    a.gate = j->gate;
    a.ldy = j->ldy;
    a.ldr = j->ldr;
    a.ldh = j->ldh;
    a.ldx = j->ldx;
    a.gate_unit = j->gate ? j->gate_unit_stride : 0;
    a.gate_row = j->gate ? j->gate_row_stride : 0;
    a.M = M;
    a.rows = B * M;
    a.K = static_cast<int>(K);
    a.post = j->post_norm != 0;
    a.rs = j->residual_scale;
    a.eps = j->eps;
    const bool bf16 = j->dtype == RMM_BF16, stream_bf16 = j->stream_dtype == RMM_BF16;
    if (!j->Xt) return from_hip(rmm::launch_join_rows(a, bf16, stream_bf16, stream));
    const size_t need = rmm_block_join_workspace_size(B, M, K);
    if (!workspace || workspace_bytes < need) return RMM_ERR_WORKSPACE_TOO_SMALL;
    if (!aligned(workspace, 256)) return RMM_ERR_INVALID_ARGUMENT;
    a.rscale = static_cast<float *>(workspace);
    double *partials = reinterpret_cast<double *>(static_cast<char *>(workspace) +
                                                  align256(static_cast<size_t>(B * M) * sizeof(float)));
    const hipError_t e = rmm::launch_join_rows(a, bf16, stream_bf16, stream);
    if (e != hipSuccess) return RMM_ERR_HIP;
    return from_hip(rmm::launch_join_kmajor(a.h, stream_bf16, a.ldh, a.rscale, static_cast<const uint16_t *>(a.gpre), B, M,
                                            K, static_cast<uint16_t *>(j->Xt), j->ldxt, partials, j->energy, stream));
}

size_t rmm_token_logprobs_workspace_size(int64_t T, int64_t V, int64_t top) {
    if (T < 1 || V < 1 || T >= kMaxRows || V >= kMaxVocab || top < 0 || top > rmm::kMaxTop) return 0;
    return align256(rmm::logprob_workspace_bytes(T, V, top));
}

rmm_status_t rmm_token_logprobs(const void *logits, rmm_dtype_t dtype, int64_t T, int64_t V, int64_t ldl, float scale,
                                const int32_t *tokens, int64_t given, float *logp, float *entropy, int64_t top,
                                int32_t *top_idx, float *top_logp, void *workspace, size_t workspace_bytes,
                                hipStream_t stream) {
    if (!logits || !valid_dtype(dtype)) return RMM_ERR_INVALID_ARGUMENT;
    if (T < 1 || V < 1 || V > kInt32Max || ldl < V) return RMM_ERR_INVALID_ARGUMENT;
    if (!(scale > 0.f) || std::isinf(scale * 1.44269504f)) return RMM_ERR_INVALID_ARGUMENT;     // also NaN
    if (given < 0 || top < 0 || top > V || (given == 0 && top == 0 && !entropy)) return RMM_ERR_INVALID_ARGUMENT;
    if (given > 0 && (!tokens || !logp)) return RMM_ERR_INVALID_ARGUMENT;
    if (top > 0 && (!top_idx || !top_logp)) return RMM_ERR_INVALID_ARGUMENT;
    const size_t size = dtype == RMM_BF16 ? 2 : 4;
    if (!aligned(logits, size) || !aligned(tokens, 4) || !aligned(logp, 4) || !aligned(entropy, 4) ||
        !aligned(top_idx, 4) || !aligned(top_logp, 4))
        return RMM_ERR_INVALID_ARGUMENT;
    if (top > rmm::kMaxTop || T >= kMaxRows || V >= kMaxVocab || given >= kMaxGiven) return RMM_ERR_UNSUPPORTED;
    const size_t need = rmm_token_logprobs_workspace_size(T, V, top);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return RMM_ERR_WORKSPACE_TOO_SMALL;
        if (!aligned(workspace, 8)) return RMM_ERR_INVALID_ARGUMENT;
    }
    rmm::LogprobArgs a = {};
    a.z = logits;
    a.ld = ldl;
    a.T = T;
    a.V = static_cast<int>(V);
    a.pieces = rmm::logprob_pieces(T, V);
    a.given = static_cast<int>(given);
    a.top = static_cast<int>(top);
    a.c = scale * 1.44269504f;
    a.tokens = tokens;
    a.logp = logp;
    a.entropy = entropy;
    a.top_idx = top_idx;
    a.top_logp = top_logp;
    a.part = workspace;
    return from_hip(rmm::launch_logprobs(a, dtype == RMM_BF16, stream));
}

}  // extern "C"
