// C-ABI of the rotation, paged-cache and cache-attention entry points: host-side
// validation and dispatch.  Every check happens before the first HIP call.
#include <cmath>
#include <cstdint>

#include "../../include/rmm.h"
#include "kernels.h"
#include "kv_cache.h"

namespace {

constexpr int64_t kInt32Max = 2147483647;
constexpr int64_t kMaxHeads = 65535;

inline size_t align256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }
inline bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline rmm_status_t from_hip(hipError_t e) { return e == hipSuccess ? RMM_OK : RMM_ERR_HIP; }

// heads of 16-byte aligned rows; esz: bytes per element
rmm_status_t check_heads(const rmm_heads_t *h, int64_t esz, rmm::Heads *out) {
    if (!h->data || h->n < 1 || h->batch_stride < 0 || h->token_stride < 0 || h->head_stride < 0)
        return RMM_ERR_INVALID_ARGUMENT;
    const int64_t step = 16 / esz;
    if (!aligned(h->data, 16) || h->batch_stride % step || h->token_stride % step || h->head_stride % step ||
        h->n > kMaxHeads)
        return RMM_ERR_UNSUPPORTED;
    *out = {h->data, static_cast<int>(h->n), h->batch_stride, h->token_stride, h->head_stride};
    return RMM_OK;
}

rmm_status_t check_rope(const rmm_rope_t *rope, const int32_t *positions, int64_t D, rmm::RotateArgs *a) {
    if (!rope || rope->rot == 0) return RMM_OK;
    if (!rope->cos || !rope->sin || !positions || rope->rot < 0 || rope->rot > D || rope->n_pos < 1)
        return RMM_ERR_INVALID_ARGUMENT;
    if (rope->rot % 16 || !aligned(rope->cos, 16) || !aligned(rope->sin, 16) || !aligned(positions, 4) ||
        rope->n_pos > kInt32Max)
        return RMM_ERR_UNSUPPORTED;
    a->cs = rope->cos;
    a->sn = rope->sin;
    a->n_pos = static_cast<int>(rope->n_pos);
    a->rot = static_cast<int>(rope->rot);
    a->interleaved = rope->interleaved != 0;
    a->pos = positions;
    return RMM_OK;
}

rmm_status_t check_cache(const rmm_kv_cache_t *c, rmm::KvPages *kv) {
    if (!c || !c->k || !c->v || c->n_pages < 1 || c->page_size < 1 || c->Hkv < 1 || c->D < 1) return RMM_ERR_INVALID_ARGUMENT;
    if (c->type != RMM_CACHE_BF && c->type != RMM_CACHE_MX) return RMM_ERR_INVALID_ARGUMENT;
    const bool mx = c->type == RMM_CACHE_MX;
    if (mx && (!c->k_scale || !c->v_scale)) return RMM_ERR_INVALID_ARGUMENT;
    if ((c->D != 64 && c->D != 128) || c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) ||
        c->Hkv > kMaxHeads || c->n_pages > kInt32Max / c->page_size)
        return RMM_ERR_UNSUPPORTED;
    const int64_t rows = c->Hkv * c->page_size, row = mx ? c->D / 2 : c->D * 2, srow = c->D / 32;
    const bool many = c->n_pages > 1;                      // one page has no stride
    if (many && (c->k_stride < rows * row || c->v_stride < rows * row)) return RMM_ERR_INVALID_ARGUMENT;
    if (many && mx && (c->k_scale_stride < rows * srow || c->v_scale_stride < rows * srow)) return RMM_ERR_INVALID_ARGUMENT;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || (many && (c->k_stride % 16 || c->v_stride % 16))) return RMM_ERR_UNSUPPORTED;
    if (mx && (!aligned(c->k_scale, 16) || !aligned(c->v_scale, 16) ||
               (many && (c->k_scale_stride % 16 || c->v_scale_stride % 16))))
        return RMM_ERR_UNSUPPORTED;
    kv->k = static_cast<uint8_t *>(c->k);
    kv->v = static_cast<uint8_t *>(c->v);
    kv->ks = mx ? static_cast<uint8_t *>(c->k_scale) : nullptr;
    kv->vs = mx ? static_cast<uint8_t *>(c->v_scale) : nullptr;
    kv->k_page = many ? c->k_stride : 0;
    kv->v_page = many ? c->v_stride : 0;
    kv->ks_page = many && mx ? c->k_scale_stride : 0;
    kv->vs_page = many && mx ? c->v_scale_stride : 0;
    kv->n_pages = static_cast<int>(c->n_pages);
    kv->lg_page = 0;
    while ((int64_t(1) << kv->lg_page) < c->page_size) ++kv->lg_page;
    kv->Hkv = static_cast<int>(c->Hkv);
    kv->mx = mx;
    return RMM_OK;
}

}  // namespace

extern "C" {

size_t rmm_qk_norm_rope_workspace_size(int64_t batch, int64_t H, int64_t L, int64_t D) {
    if (batch < 1 || H < 1 || L < 1 || (D != 64 && D != 128) || L > kInt32Max / batch || H > kMaxHeads) return 0;
    const int64_t blocks = rmm::rotate_blocks(batch, L, H, static_cast<int>(D));
    return blocks < 2 ? 0 : align256(static_cast<size_t>(batch * blocks * H * D) * sizeof(double));
}

rmm_status_t rmm_qk_norm_rope(rmm_dtype_t dtype, int64_t batch, int64_t L, int64_t D, const rmm_heads_t *q,
                              const rmm_heads_t *q_out, const rmm_heads_t *k, const rmm_heads_t *k_out,
                              const void *gamma_q, const void *gamma_k, float eps, const rmm_rope_t *rope,
                              const int32_t *positions, double *energy, void *workspace,
                              size_t workspace_bytes, hipStream_t stream) {
    if ((dtype != RMM_BF16 && dtype != RMM_F32) || batch < 1 || L < 1 || D < 1) return RMM_ERR_INVALID_ARGUMENT;
    if ((!q && !k) || !q != !q_out || !k != !k_out || (energy && !q)) return RMM_ERR_INVALID_ARGUMENT;
    if (!(eps >= 0.f) || std::isinf(eps)) return RMM_ERR_INVALID_ARGUMENT;
    const int64_t esz = dtype == RMM_BF16 ? 2 : 4;
    rmm::RotateArgs a = {};
    rmm_status_t st = RMM_OK;
    if (q && st == RMM_OK) st = check_heads(q, esz, &a.q);
    if (q && st == RMM_OK) st = check_heads(q_out, esz, &a.qo);
    if (k && st == RMM_OK) st = check_heads(k, esz, &a.k);
    if (k && st == RMM_OK) st = check_heads(k_out, esz, &a.ko);
    if (st != RMM_OK) return st;
    if (a.q.n != a.qo.n || a.k.n != a.ko.n) return RMM_ERR_INVALID_ARGUMENT;
    if ((D != 64 && D != 128) || batch > kInt32Max / L || a.q.n + a.k.n > kMaxHeads) return RMM_ERR_UNSUPPORTED;
    if (!aligned(gamma_q, 16) || !aligned(gamma_k, 16) || !aligned(energy, 8)) return RMM_ERR_UNSUPPORTED;
    st = check_rope(rope, positions, D, &a);
    if (st != RMM_OK) return st;
    a.gq = gamma_q;
    a.gk = gamma_k;
    a.eps = eps;
    a.T = batch * L;
    a.L = L;
    if (!energy) return from_hip(rmm::launch_rotate(a, dtype == RMM_BF16, static_cast<int>(D), stream));
    const int64_t blocks = rmm::rotate_blocks(batch, L, a.q.n, static_cast<int>(D));
    const size_t need = rmm_qk_norm_rope_workspace_size(batch, a.q.n, L, D);
    a.partials = energy;
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return RMM_ERR_WORKSPACE_TOO_SMALL;
        if (!aligned(workspace, 8)) return RMM_ERR_INVALID_ARGUMENT;
        a.partials = static_cast<double *>(workspace);
    }
    const hipError_t e = rmm::launch_rotate(a, dtype == RMM_BF16, static_cast<int>(D), stream);
    if (e != hipSuccess || need == 0) return from_hip(e);
    // sixteen threads per column's partial sums (1 x 8192 tokens, 128 of them: 5 us, 6
    // with one thread; 1000 tokens: 4, 8; 65 tokens: 3, 3), by batch in the grid's y
    if (batch > kMaxHeads)
        return from_hip(rmm::launch_score_finalize(a.partials, batch, blocks, a.q.n * D, energy, stream));
    return from_hip(rmm::launch_score_finalize_grouped(a.partials, batch, blocks, a.q.n * D, energy, stream));
}

rmm_status_t rmm_kv_append(int64_t T, const rmm_heads_t *k, const rmm_heads_t *v, const int32_t *slots,
                           const rmm_kv_cache_t *cache, const void *gamma_k, const rmm_heads_t *q,
                           const rmm_heads_t *q_out, const void *gamma_q, float eps, const rmm_rope_t *rope,
                           const int32_t *positions, hipStream_t stream) {
    if (T < 1 || !k || !v || !slots || !q != !q_out) return RMM_ERR_INVALID_ARGUMENT;
    if (!(eps >= 0.f) || std::isinf(eps)) return RMM_ERR_INVALID_ARGUMENT;
    rmm::RotateArgs a = {};
    rmm_status_t st = check_cache(cache, &a.kv);
    if (st == RMM_OK) st = check_heads(k, 2, &a.k);
    if (st == RMM_OK) st = check_heads(v, 2, &a.v);
    if (q && st == RMM_OK) st = check_heads(q, 2, &a.q);
    if (q && st == RMM_OK) st = check_heads(q_out, 2, &a.qo);
    if (st != RMM_OK) return st;
    if (a.k.n != a.kv.Hkv || a.v.n != a.kv.Hkv || a.q.n != a.qo.n) return RMM_ERR_INVALID_ARGUMENT;
    if (T > kInt32Max || a.q.n + 2 * a.kv.Hkv > kMaxHeads || !aligned(gamma_q, 16) || !aligned(gamma_k, 16) || !aligned(slots, 4))
        return RMM_ERR_UNSUPPORTED;
    st = check_rope(rope, positions, cache->D, &a);
    if (st != RMM_OK) return st;
    a.gq = gamma_q;
    a.gk = gamma_k;
    a.eps = eps;
    a.slots = slots;
    a.T = a.L = T;
    return from_hip(rmm::launch_kv_append(a, static_cast<int>(cache->D), stream));
}

rmm_status_t rmm_kv_gather(const rmm_kv_cache_t *cache, const int32_t *slots, int64_t T, const rmm_heads_t *k,
                           const rmm_heads_t *v, hipStream_t stream) {
    if (T < 1 || !slots || !k || !v) return RMM_ERR_INVALID_ARGUMENT;
    rmm::KvPages kv = {};
    rmm::Heads ko = {}, vo = {};
    rmm_status_t st = check_cache(cache, &kv);
    if (st == RMM_OK) st = check_heads(k, 2, &ko);
    if (st == RMM_OK) st = check_heads(v, 2, &vo);
    if (st != RMM_OK) return st;
    if (ko.n != kv.Hkv || vo.n != kv.Hkv) return RMM_ERR_INVALID_ARGUMENT;
    // a thread takes 8 elements of four rows, a launch holds fewer than 2^32 threads
    if (T > (int64_t(1) << 37) / (2 * kv.Hkv * cache->D) - 1 || T > kInt32Max / kv.Hkv || !aligned(slots, 4)) return RMM_ERR_UNSUPPORTED;
    return from_hip(rmm::launch_kv_gather(kv, slots, T, ko, vo, static_cast<int>(cache->D), stream));
}

size_t rmm_paged_attention_workspace_size(int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D) {
    if (T < 1 || B < 1 || H < 1 || Hkv < 1 || H % Hkv || (D != 64 && D != 128) || T > kInt32Max / H) return 0;
    return align256(rmm::paged_workspace_bytes(T, B, H, Hkv, static_cast<int>(D)));
}

rmm_status_t rmm_paged_attention(int64_t T, const rmm_heads_t *q, const rmm_kv_cache_t *cache,
                                 const int32_t *page_table, int64_t table_stride, int64_t max_pages,
                                 const int32_t *lengths, int64_t B, const int32_t *q_start,
                                 const int32_t *idx, int64_t k, float scale, int causal, const rmm_heads_t *o,
                                 void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!q || !o || !page_table || !lengths || T < 1 || B < 1 || max_pages < 1 || table_stride < max_pages)
        return RMM_ERR_INVALID_ARGUMENT;
    if (!q_start && T != B) return RMM_ERR_INVALID_ARGUMENT;
    rmm::PagedArgs a = {};
    a.c = scale * 1.4426950408889634f;
    if (!std::isfinite(a.c)) return RMM_ERR_INVALID_ARGUMENT;
    rmm_status_t st = check_cache(cache, &a.kv);
    if (st == RMM_OK) st = check_heads(q, 2, &a.q);
    if (st == RMM_OK) st = check_heads(o, 2, &a.o);
    if (st != RMM_OK) return st;
    if (a.q.n % a.kv.Hkv || a.o.n != a.q.n) return RMM_ERR_INVALID_ARGUMENT;
    if (idx && (k < 1 || k > cache->D)) return RMM_ERR_INVALID_ARGUMENT;
    if (T > kInt32Max / a.q.n || B > kInt32Max - 64 || max_pages > (int64_t(1) << 30) / cache->page_size ||
        !rmm::paged_line_fits(T, B, a.q.n, a.kv.Hkv, a.kv.mx != 0, static_cast<int>(cache->D),
                              max_pages * cache->page_size) ||
        !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(q_start, 4) || !aligned(idx, 4))
        return RMM_ERR_UNSUPPORTED;
    const size_t need = rmm_paged_attention_workspace_size(T, B, a.q.n, a.kv.Hkv, cache->D);
    if (!workspace || workspace_bytes < need) return RMM_ERR_WORKSPACE_TOO_SMALL;
    if (!aligned(workspace, 256)) return RMM_ERR_INVALID_ARGUMENT;
    a.table = page_table;
    a.lens = lengths;
    a.q_start = q_start;
    a.idx = idx;
    a.table_ld = table_stride;
    a.width = static_cast<int>(max_pages);
    a.B = static_cast<int>(B);
    a.k = static_cast<int>(k);
    a.T = T;
    a.causal = causal != 0;
    return from_hip(rmm::launch_paged_attn(a, static_cast<int>(cache->D), workspace, stream));
}

}  // extern "C"
