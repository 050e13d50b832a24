// Arguments of the rotation, cache and cache-attention kernels (kv_cache.hip,
// paged_attn.hip), validated by the C-ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rmm {

// n heads of D contiguous elements each: batch b, token t, head h at
// p + b * sb + t * st + h * sh elements
struct Heads {
    void *p;
    int n;
    int64_t sb, st, sh;
};

// a paged cache; page strides in bytes, inside a page [Hkv][page_size][row]
struct KvPages {
    uint8_t *k, *v, *ks, *vs;              // ks, vs: scale bytes (4-bit caches)
    int64_t k_page, v_page, ks_page, vs_page;
    int n_pages, lg_page, Hkv, mx;         // page_size = 1 << lg_page
};

struct RotateArgs {
    Heads q, k, v, qo, ko;                 // n = 0: absent (k: written to ko, or with v to the cache)
    const void *gq, *gk;                   // norm weights [D], or null
    float eps;
    const float *cs, *sn;                  // cos and sin [n_pos][rot / 2]; rot = 0: no rotation
    int n_pos, rot, interleaved;
    const int32_t *pos, *slots;            // [T]
    KvPages kv;
    double *partials;                      // energies: [batch][blocks][q.n * D]
    int64_t T, L;                          // tokens in all, per batch entry
};

// Rotation (and norm) of q and k; with partials, the per-block column sums of
// squares of qo, rotate_blocks(batch, L, heads) blocks per batch entry
int64_t rotate_blocks(int64_t batch, int64_t L, int64_t heads, int D);
hipError_t launch_rotate(const RotateArgs &a, bool bf16, int D, hipStream_t stream);
// The same pass with k and v going to the cache's slots
hipError_t launch_kv_append(const RotateArgs &a, int D, hipStream_t stream);
hipError_t launch_kv_gather(const KvPages &kv, const int32_t *slots, int64_t T, const Heads &k, const Heads &v, int D,
                            hipStream_t stream);

struct PagedArgs {
    Heads q, o;
    KvPages kv;
    const int32_t *table, *lens, *q_start, *idx;
    int64_t table_ld;
    int width, B, k;                       // pages per table row, sequences, list length
    int64_t T;
    float c;                               // scale * log2(e)
    int causal;
    void *pieces;                          // what joins the pieces of cut units
    float *part_o, *part_ml;               // their outputs, their (max, sum)
    int nw, whole;                         // workgroups; whether no unit is cut
};
bool paged_line_fits(int64_t T, int64_t B, int64_t H, int64_t Hkv, bool mx, int D, int64_t keys);
size_t paged_workspace_bytes(int64_t T, int64_t B, int64_t H, int64_t Hkv, int D);
hipError_t launch_paged_attn(PagedArgs a, int D, void *workspace, hipStream_t stream);

}  // namespace rmm
