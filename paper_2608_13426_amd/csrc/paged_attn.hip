// Attention of new tokens over a paged key/value cache (bf16, or MXFP4: 4-bit
// codes with one power-of-two scale per 32 dims):
//   O[t][h] = softmax(scale * Q[t][h][I] . K[s][g][I]) V[s][g],  s the positions the
//   token sees, I all dims or the (token, head)'s retained ones
//
// A unit is one (sequence, kv head, tile of 16 * R query rows); a query row is
// one (new token, query head of the kv head), so the heads of a group share
// every key read.  The 32-key chunks of all units lie on one line that is cut
// into equal runs, one per workgroup: lengths are only known on the device, and
// a batch with one long sequence still loads from every CU.  A unit inside one
// workgroup is written at once; the pieces of a cut one go to the workspace as
// (maximum, sum, unnormalised output) and a second launch joins them in order.
//
// Inside a workgroup the four waves take chunks in turn and meet only at the
// end of a unit.  Keys and values go from memory to registers to the matrix
// cores without LDS: S^T = K Q^T takes 16 key rows as loaded (v_mfma_f32_16x16x32,
// a lane holds 8 dims of one key), its result has a query row per lane and,
// with key 8 g + 4 tb + i at row 4 g + i of tile tb, exactly the eight keys per lane group
// that O^T = V^T P^T takes as its contraction, so the weights stay in place; the value rows are
// turned 8 x 8 in registers (v_perm).  4-bit codes become bf16 with
// v_cvt_scalef32_pk_bf16_fp4 (exact, the scale included).
#include <algorithm>

#include "device_common.h"
#include "kernels.h"
#include "kv_cache.h"

namespace rmm {

namespace {

namespace pg {
constexpr int kThreads = 256, kWaves = 4, TK = 32;
constexpr float kTau = 8.f;               // lazy-rescale threshold, log2 units
constexpr int kMinChunks = 8;             // chunks per workgroup at least
constexpr int kMaxGroups = 512;           // workgroups: two per CU

// f over the four lanes l, l ^ 16, l ^ 32, l ^ 48 (all of them get the result)
template <typename F>
__device__ __forceinline__ float across_rows(float x, F f) {
#if defined(__HIP_DEVICE_COMPILE__)
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(b[0]), __uint_as_float(b[1]));
#endif
    return x;
}

__device__ __forceinline__ f32x4_t mfma(const uint4 a, const uint4 b, const f32x4_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
#else
    return c;
#endif
}
// two codes (byte B of w) as packed bf16
template <int B>
__device__ __forceinline__ uint32_t unpack_mx(uint32_t w, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
#else
    return 0;
#endif
}
__device__ __forceinline__ float exp_two(float x) { return __builtin_amdgcn_exp2f(x); }

// One sequence's share of the line of chunks
struct Seq {
    int q0, n, len, tiles, chunks;        // first token, new tokens, keys, row tiles, chunks per unit (0: no work)
    bool bad;                             // longer than its row of the page table
};
__device__ __forceinline__ Seq seq_of(const PagedArgs &a, int b, int grp, int rows) {
    Seq s;
    int q1;
    if (a.q_start) {
        s.q0 = min(max(a.q_start[b], 0), static_cast<int>(a.T));
        q1 = min(a.q_start[b + 1], static_cast<int>(a.T));
    } else {
        s.q0 = b;
        q1 = b + 1;
    }
    s.n = max(q1 - s.q0, 0);
    const int64_t cap = static_cast<int64_t>(a.width) << a.kv.lg_page;
    s.len = max(a.lens[b], 0);
    s.bad = s.len > cap;
    if (s.bad) s.len = static_cast<int>(cap);
    s.tiles = static_cast<int>((static_cast<int64_t>(s.n) * grp + rows - 1) / rows);
    s.chunks = s.n > 0 ? max((s.len + TK - 1) / TK, 1) : 0;
    return s;
}
__device__ __forceinline__ int64_t seq_work(const PagedArgs &a, const Seq &s) {
    return static_cast<int64_t>(s.tiles) * s.chunks * a.kv.Hkv;
}

__device__ __forceinline__ int64_t shfl_up64(int64_t x, int d) { return __shfl_up(static_cast<long long>(x), d, 64); }

// Sum of all sequences' work, the same in every lane
__device__ __forceinline__ int64_t total_work(const PagedArgs &a, int grp, int rows) {
    int64_t w = 0;
    for (int b = threadIdx.x & 63; b < a.B; b += 64) w += seq_work(a, seq_of(a, b, grp, rows));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) w += __shfl_xor(static_cast<long long>(w), d, 64);
    return w;
}
// The sequence whose chunks hold position x of the line, and where they begin
__device__ __forceinline__ int find_seq(const PagedArgs &a, int grp, int rows, int64_t x, int64_t *start) {
    int64_t base = 0;
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int b = b0 + lane;
        const int64_t w = b < a.B ? seq_work(a, seq_of(a, b, grp, rows)) : 0;
        int64_t s = w;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t y = shfl_up64(s, d);
            if (lane >= d) s += y;
        }
        const uint64_t past = __ballot(base + s > x);
        if (past) {
            const int l = __builtin_ctzll(past);
            *start = base + __shfl(static_cast<long long>(s - w), l, 64);
            return b0 + l;
        }
        base += __shfl(static_cast<long long>(s), 63, 64);
    }
    *start = base;
    return a.B;
}
__device__ __forceinline__ int64_t uniform64(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(static_cast<uint64_t>(x) >> 32));
    return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}
// chunks per workgroup: a whole number of rounds of the four waves
__device__ __forceinline__ int64_t run_length(int64_t total, int nw) {
    const int64_t per = (total + nw - 1) / nw;
    return max((per + kWaves - 1) / kWaves * kWaves, static_cast<int64_t>(kMinChunks));
}
}  // namespace pg

}  // namespace

// MX: 4-bit cache; IDX: scores over retained dims
template <int D, bool MX, int R, bool IDX>
__global__ __launch_bounds__(pg::kThreads, R == 1 ? 2 : 1) void paged_attn_kernel(PagedArgs a) {
    using namespace pg;
    constexpr int KS = D / 32, DM = D / 16;               // contraction steps of S^T, MFMA rows of O^T
    constexpr int ROWB = MX ? D / 2 : D * 2, SROWB = D / 32;    // bytes per cached row, scale bytes per row
    constexpr int OLD = D + 4;                            // row stride of the joining buffer, floats
    __shared__ __attribute__((aligned(16))) float oj[kWaves][16][OLD];
    __shared__ float ml[kWaves][16][2];
    __shared__ uint32_t keep[IDX ? 16 * R : 1][KS];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int H = a.q.n, Hkv = a.kv.Hkv, grp = H / Hkv;

    const int64_t total = uniform64(total_work(a, grp, 16 * R));
    const int64_t run = run_length(total, a.nw);
    int64_t x = blockIdx.x * run;
    const int64_t x_end = min(total, x + run);
    if (x >= x_end) return;
    int64_t f = 0;
    int b = __builtin_amdgcn_readfirstlane(find_seq(a, grp, 16 * R, x, &f));
    f = uniform64(f);
    const int64_t x_begin = x;
    const int lg = a.kv.lg_page, ps = 1 << lg;

    while (x < x_end) {
        const Seq sq = seq_of(a, b, grp, 16 * R);
        const int64_t end_b = f + seq_work(a, sq);
        if (x >= end_b) {                                  // next sequence (an empty one has no chunks)
            f = end_b;
            ++b;
            continue;
        }
        const int unit = __builtin_amdgcn_readfirstlane(static_cast<int>((x - f) / sq.chunks));
        const int64_t u0 = f + static_cast<int64_t>(unit) * sq.chunks;
        const int c0 = static_cast<int>(x - u0);
        const int64_t u_end = u0 + sq.chunks;
        const int c1 = static_cast<int>(min(x_end, u_end) - u0);
        const int kvh = unit / sq.tiles, tile = unit % sq.tiles;
        const int row0 = tile * 16 * R, n_rows = min(16 * R, sq.n * grp - row0);
        const int64_t ubegin = u0;

        // ---- the unit's query rows
        if constexpr (IDX) {
            for (int i = tid; i < 16 * R * KS; i += kThreads) (&keep[0][0])[i] = 0;
            __syncthreads();
            for (int i = tid; i < n_rows * a.k; i += kThreads) {
                const int r = i / a.k, u = i - r * a.k, rho = row0 + r;
                const int d = a.idx[(static_cast<int64_t>(sq.q0 + rho / grp) * H + kvh * grp + rho % grp) * a.k + u];
                if (d >= 0 && d < D) atomicOr(&keep[r][d >> 5], 1u << (d & 31));
            }
            __syncthreads();
        }
        // dims that lane (col, g) holds at contraction step s
        auto dim_of = [&](int s) { return MX ? (D / 4) * g + 8 * s : 32 * s + 8 * g; };
        uint4 qf[R][KS];
        int lim[R];                                        // last key the lane's row sees
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int rr = 16 * r + col, rho = row0 + rr;
            const bool on = rr < n_rows;
            const int tok = on ? rho / grp : 0, hd = on ? kvh * grp + rho % grp : 0;
            lim[r] = !on ? -1 : a.causal ? sq.len - sq.n + tok : sq.len - 1;
            const uint16_t *qp = static_cast<const uint16_t *>(a.q.p) + (sq.q0 + tok) * a.q.st + hd * a.q.sh;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                uint4 w = make_uint4(0, 0, 0, 0);
                if (on) w = *reinterpret_cast<const uint4 *>(qp + dim_of(s));
                if constexpr (IDX) {
                    const uint32_t m = keep[rr][dim_of(s) >> 5] >> (dim_of(s) & 31);
                    w.x &= (m & 1 ? 0xffffu : 0u) | (m & 2 ? 0xffff0000u : 0u);
                    w.y &= (m & 4 ? 0xffffu : 0u) | (m & 8 ? 0xffff0000u : 0u);
                    w.z &= (m & 16 ? 0xffffu : 0u) | (m & 32 ? 0xffff0000u : 0u);
                    w.w &= (m & 64 ? 0xffffu : 0u) | (m & 128 ? 0xffff0000u : 0u);
                }
                qf[r][s] = w;
            }
        }
        // keys seen by every row / by no row past it
        const int first_tok = row0 / grp, last_tok = (row0 + n_rows - 1) / grp;
        const int lo_lim = a.causal ? sq.len - sq.n + first_tok : sq.len - 1;
        const int hi_lim = a.causal ? sq.len - sq.n + last_tok : sq.len - 1;
        const int c_stop = min(c1, hi_lim < 0 ? 0 : hi_lim / TK + 1);

        f32x4_t o[R][DM];
        float m_run[R], l_run[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m_run[r] = -__builtin_inff();
            l_run[r] = 0.f;
#pragma unroll
            for (int i = 0; i < DM; ++i) o[r][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        bool bad = sq.bad;

        // ---- the wave's chunks c0 + wave, + 4, ...; lane l holds the pages of the
        // l-th of them (two where a page has 16 keys)
        const int32_t *trow = a.table + b * a.table_ld;
        int pid_a = 0, pid_b = 0;
        struct Chunk {
            uint4 k[2][MX ? 1 : KS];
            uint32_t ks[2];
            uint4 v[MX ? 1 : 8];                           // bf16: DM elements of 8 value rows
            uint32_t vc[8];                                // MX: DM codes of 8 value rows
            uint4 vs[MX ? 2 : 1];
        };
        auto fetch_pages = [&](int c) __attribute__((always_inline)) {
            const int key = (c + kWaves * lane) * TK;      // this lane's chunk
            const bool on = c + kWaves * lane < c_stop;
            const int p0 = on ? key >> lg : 0, p1 = on && key + 16 < sq.len ? (key + 16) >> lg : p0;
            pid_a = on ? trow[p0] : 0;
            pid_b = on ? trow[p1] : 0;
            const bool oka = pid_a >= 0 && pid_a < a.kv.n_pages, okb = pid_b >= 0 && pid_b < a.kv.n_pages;
            if (__ballot(!oka || !okb)) bad = true;
            if (!oka) pid_a = 0;
            if (!okb) pid_b = 0;
        };
        // rows of the chunk at keys 8 (col / 4) + 4 tb + col % 4 (K), 8 g + kk (V)
        auto load = [&](Chunk &ck, int c, int nth) __attribute__((always_inline)) {
            const int64_t pa = __builtin_amdgcn_readlane(pid_a, nth), pb = __builtin_amdgcn_readlane(pid_b, nth);
            const int key = c * TK, oa = key & (ps - 1), ob = (key + 16) & (ps - 1);
            const int64_t hrow = static_cast<int64_t>(kvh) << lg;
            const int krow = 8 * (col >> 2) + (col & 3), vrow = 8 * g;
            const bool k2 = col >= 8, v2 = g >= 2;
            const int64_t ra = hrow + oa, rb = hrow + ob - 16;
            const uint8_t *kp = (k2 ? a.kv.k + pb * a.kv.k_page + rb * ROWB : a.kv.k + pa * a.kv.k_page + ra * ROWB) + krow * ROWB;
            const uint8_t *vp = (v2 ? a.kv.v + pb * a.kv.v_page + rb * ROWB : a.kv.v + pa * a.kv.v_page + ra * ROWB) + vrow * ROWB;
            if constexpr (!MX) {
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        ck.k[tb][s] = *reinterpret_cast<const uint4 *>(kp + tb * 4 * ROWB + 64 * s + 16 * g);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    if constexpr (D == 128) {
                        ck.v[kk] = *reinterpret_cast<const uint4 *>(vp + kk * ROWB + 16 * col);
                    } else {
                        const uint2 w = *reinterpret_cast<const uint2 *>(vp + kk * ROWB + 8 * col);
                        ck.v[kk] = make_uint4(w.x, w.y, 0, 0);
                    }
                }
            } else {
                const uint8_t *ksp = (k2 ? a.kv.ks + pb * a.kv.ks_page + rb * SROWB : a.kv.ks + pa * a.kv.ks_page + ra * SROWB) + krow * SROWB;
                const uint8_t *vsp = (v2 ? a.kv.vs + pb * a.kv.vs_page + rb * SROWB : a.kv.vs + pa * a.kv.vs_page + ra * SROWB) + vrow * SROWB;
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) {
                    if constexpr (D == 128) {
                        ck.k[tb][0] = *reinterpret_cast<const uint4 *>(kp + tb * 4 * ROWB + 16 * g);
                        ck.ks[tb] = ksp[tb * 4 * SROWB + g];
                    } else {
                        const uint2 w = *reinterpret_cast<const uint2 *>(kp + tb * 4 * ROWB + 8 * g);
                        ck.k[tb][0] = make_uint4(w.x, w.y, 0, 0);
                        ck.ks[tb] = ksp[tb * 4 * SROWB + (g >> 1)];
                    }
                }
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    if constexpr (D == 128) ck.vc[kk] = *reinterpret_cast<const uint32_t *>(vp + kk * ROWB + 4 * col);
                    else ck.vc[kk] = *reinterpret_cast<const uint16_t *>(vp + kk * ROWB + 2 * col);
                }
                ck.vs[0] = reinterpret_cast<const uint4 *>(vsp)[0];
                if constexpr (D == 128) ck.vs[1] = reinterpret_cast<const uint4 *>(vsp)[1];
            }
        };

        auto compute = [&](const Chunk &ck, int c) __attribute__((always_inline)) {
            const int key = c * TK;
            const bool edge = key + TK - 1 > lo_lim;       // wave-uniform: some row does not see every key
            // ---- key fragments, and the value rows as pairs of dims
            uint4 kf[2][KS];
            uint32_t vr[8][DM / 2];
            if constexpr (!MX) {
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int s = 0; s < KS; ++s) kf[tb][s] = ck.k[tb][s];
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    const uint32_t w[4] = {ck.v[kk].x, ck.v[kk].y, ck.v[kk].z, ck.v[kk].w};
#pragma unroll
                    for (int p = 0; p < DM / 2; ++p) vr[kk][p] = w[p];
                }
            } else {
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) {
                    const float sc = __uint_as_float(ck.ks[tb] << 23);
                    const uint32_t w[4] = {ck.k[tb][0].x, ck.k[tb][0].y, ck.k[tb][0].z, ck.k[tb][0].w};
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        kf[tb][s] = make_uint4(unpack_mx<0>(w[s], sc), unpack_mx<1>(w[s], sc), unpack_mx<2>(w[s], sc),
                                               unpack_mx<3>(w[s], sc));
                }
                const uint32_t sw[8] = {ck.vs[0].x, ck.vs[0].y, ck.vs[0].z, ck.vs[0].w,
                                        ck.vs[MX ? 1 : 0].x, ck.vs[MX ? 1 : 0].y, ck.vs[MX ? 1 : 0].z, ck.vs[MX ? 1 : 0].w};
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    // D = 128: four scale bytes per row; D = 64: two
                    const uint32_t sb = D == 128 ? (sw[kk] >> (8 * (col >> 2))) & 0xffu
                                                 : (sw[kk >> 1] >> (16 * (kk & 1) + 8 * (col >> 3))) & 0xffu;
                    const float sc = __uint_as_float(sb << 23);
                    vr[kk][0] = unpack_mx<0>(ck.vc[kk], sc);
                    vr[kk][1] = unpack_mx<1>(ck.vc[kk], sc);
                    if constexpr (D == 128) {
                        vr[kk][2] = unpack_mx<2>(ck.vc[kk], sc);
                        vr[kk][3] = unpack_mx<3>(ck.vc[kk], sc);
                    }
                }
            }
            // ---- scores of the row tiles and their weights
            uint4 pf[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                f32x4_t sc[2];
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) {
                    sc[tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < KS; ++s) sc[tb] = mfma(kf[tb][s], qf[r][s], sc[tb]);
                }
                if constexpr (IDX) {
                    // an infinite or NaN key value in a dim that a row drops must not
                    // reach it: then each row multiplies keys cleared by its own set
                    bool fin = true;
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) fin = fin && __builtin_fabsf(sc[tb][i]) < __builtin_inff();
                    if (__ballot(!fin)) {
                        for (int cc = 0; cc < 16; ++cc) {
#pragma unroll
                            for (int tb = 0; tb < 2; ++tb) {
                                f32x4_t t = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                                for (int s = 0; s < KS; ++s) {
                                    const uint32_t m = keep[16 * r + cc][dim_of(s) >> 5] >> (dim_of(s) & 31);
                                    uint4 w = kf[tb][s];
                                    w.x &= (m & 1 ? 0xffffu : 0u) | (m & 2 ? 0xffff0000u : 0u);
                                    w.y &= (m & 4 ? 0xffffu : 0u) | (m & 8 ? 0xffff0000u : 0u);
                                    w.z &= (m & 16 ? 0xffffu : 0u) | (m & 32 ? 0xffff0000u : 0u);
                                    w.w &= (m & 64 ? 0xffffu : 0u) | (m & 128 ? 0xffff0000u : 0u);
                                    t = mfma(w, qf[r][s], t);
                                }
#pragma unroll
                                for (int i = 0; i < 4; ++i) sc[tb][i] = col == cc ? t[i] : sc[tb][i];
                            }
                        }
                    }
                }
                float p[2][4], mx = -__builtin_inff();
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[tb][i] = sc[tb][i] * a.c;
                        if (edge && key + 8 * g + 4 * tb + i > lim[r]) p[tb][i] = -__builtin_inff();
                        mx = fmaxf(mx, p[tb][i]);
                    }
                mx = across_rows(mx, [](float u, float v) { return fmaxf(u, v); });
                if (__ballot(mx > m_run[r] + kTau)) {
                    const float m_new = fmaxf(m_run[r], mx);
                    const float al = m_new == -__builtin_inff() ? 1.f : exp_two(m_run[r] - m_new);
                    l_run[r] *= al;
#pragma unroll
                    for (int i = 0; i < DM; ++i) o[r][i] *= al;
                    m_run[r] = m_new;
                }
                const float m_use = m_run[r] == -__builtin_inff() ? 0.f : m_run[r];
                float ls = 0.f;
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[tb][i] = exp_two(p[tb][i] - m_use);
                        ls += p[tb][i];
                    }
                l_run[r] += ls;
                pf[r] = make_uint4(pack_bf16x2(p[0][0], p[0][1]), pack_bf16x2(p[0][2], p[0][3]),
                                   pack_bf16x2(p[1][0], p[1][1]), pack_bf16x2(p[1][2], p[1][3]));
            }
            // ---- O^T += V^T P^T: dim DM * col + i of the value rows at MFMA i
            auto value_frag = [&](const uint32_t(&v)[8][DM / 2], int i) __attribute__((always_inline)) {
                const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;
                uint4 w;
                w.x = __builtin_amdgcn_perm(v[1][i >> 1], v[0][i >> 1], sel);
                w.y = __builtin_amdgcn_perm(v[3][i >> 1], v[2][i >> 1], sel);
                w.z = __builtin_amdgcn_perm(v[5][i >> 1], v[4][i >> 1], sel);
                w.w = __builtin_amdgcn_perm(v[7][i >> 1], v[6][i >> 1], sel);
                return w;
            };
            if (!edge) {
#pragma unroll
                for (int i = 0; i < DM; ++i) {
                    const uint4 w = value_frag(vr, i);
#pragma unroll
                    for (int r = 0; r < R; ++r) o[r][i] = mfma(w, pf[r], o[r][i]);
                }
            } else {
                // A weight of zero does not silence an infinite or NaN value, so the
                // rows of each token multiply values cleared past what it sees
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int ra = row0 + 16 * r, rb = min(ra + 15, row0 + n_rows - 1);
                    if (ra > rb) continue;
                    const int t0 = a.causal ? ra / grp : 0, t1 = a.causal ? rb / grp : 0;
                    for (int tok = t0; tok <= t1; ++tok) {
                        const int last = a.causal ? sq.len - sq.n + tok : sq.len - 1;
                        uint32_t vm[8][DM / 2];
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk)
#pragma unroll
                            for (int p = 0; p < DM / 2; ++p) vm[kk][p] = key + 8 * g + kk <= last ? vr[kk][p] : 0u;
                        const bool mine = lim[r] == last;
#pragma unroll
                        for (int i = 0; i < DM; ++i) {
                            const f32x4_t t = mfma(value_frag(vm, i), pf[r], o[r][i]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[r][i][e] = mine ? t[e] : o[r][i][e];
                        }
                    }
                }
            }
        };

        {
            Chunk ca, cb;
            int c = c0 + wave;
            while (c < c_stop) {                           // up to 64 chunks per fetch of page numbers
                fetch_pages(c);
                const int n = min(64, (c_stop - c + kWaves - 1) / kWaves);
                load(ca, c, 0);
                for (int i = 0; i < n; i += 2) {
                    if (i + 1 < n) load(cb, c + kWaves * (i + 1), i + 1);
                    compute(ca, c + kWaves * i);
                    if (i + 1 < n) {
                        if (i + 2 < n) load(ca, c + kWaves * (i + 2), i + 2);
                        compute(cb, c + kWaves * (i + 1));
                    }
                }
                c += kWaves * n;
            }
        }

        // ---- the four waves join, 16 rows at a time
        const bool whole = ubegin >= x_begin && u_end <= x_end;
        const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (ubegin >= x_begin ? 1 : 0);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float l = across_rows(l_run[r], [](float u, float v) { return u + v; });
            __syncthreads();
            if (g == 0) {
                ml[wave][col][0] = m_run[r];
                ml[wave][col][1] = bad ? __builtin_nanf("") : l;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < DM; i += 4)
                    *reinterpret_cast<float4 *>(&oj[wave][col][DM * (4 * g + e) + i]) =
                        make_float4(o[r][i][e], o[r][i + 1][e], o[r][i + 2][e], o[r][i + 3][e]);
            __syncthreads();
            const int rr = tid >> 4, d0 = (tid & 15) * DM;
            if (16 * r + rr < n_rows) {
                float m = -__builtin_inff(), ls = 0.f, acc[DM];
#pragma unroll
                for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml[w][rr][0]);
#pragma unroll
                for (int i = 0; i < DM; ++i) acc[i] = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float mw = ml[w][rr][0], al = mw == -__builtin_inff() ? 0.f : exp_two(mw - m);
                    const float lw = ml[w][rr][1];
                    ls += lw == lw ? lw * al : lw;
#pragma unroll
                    for (int i = 0; i < DM; ++i) acc[i] += al == 0.f ? 0.f : al * oj[w][rr][d0 + i];
                }
                if (whole) {
                    const int rho = row0 + 16 * r + rr;
                    const float inv = ls == 0.f ? 0.f : 1.f / ls;
                    uint16_t *op = static_cast<uint16_t *>(a.o.p) + (sq.q0 + rho / grp) * a.o.st +
                                   (kvh * grp + rho % grp) * a.o.sh + d0;
                    uint32_t w[DM / 2];
#pragma unroll
                    for (int i = 0; i < DM / 2; ++i) w[i] = pack_bf16x2(acc[2 * i] * inv, acc[2 * i + 1] * inv);
                    if constexpr (D == 128) *reinterpret_cast<uint4 *>(op) = make_uint4(w[0], w[1], w[2], w[3]);
                    else *reinterpret_cast<uint2 *>(op) = make_uint2(w[0], w[1]);
                } else {
                    const int64_t prow = slot * (16 * R) + 16 * r + rr;
                    if ((tid & 15) == 0) {
                        a.part_ml[2 * prow] = m;
                        a.part_ml[2 * prow + 1] = ls;
                    }
#pragma unroll
                    for (int i = 0; i < DM; i += 4)
                        *reinterpret_cast<float4 *>(a.part_o + prow * D + d0 + i) =
                            make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
                }
            }
        }
        x = f + static_cast<int64_t>(unit) * sq.chunks + c1;
    }
}

// Joins the pieces of the cut unit that workgroup blockIdx.x ends inside of or
// continues: the unit's pieces are those of workgroups i0 .. i1, and workgroup
// i0 + q of them takes its rows q, q + (i1 - i0 + 1), ...
template <int D, int R>
__global__ __launch_bounds__(pg::kThreads) void paged_merge_kernel(PagedArgs a) {
    using namespace pg;
    constexpr int LD = D / 4, PW = kThreads / LD;          // lanes per row, pieces taken at once
    __shared__ float4 acc_s[PW][LD];
    __shared__ float2 ml_s[PW];
    const int H = a.q.n, grp = H / a.kv.Hkv, tid = threadIdx.x;
    const int64_t total = uniform64(total_work(a, grp, 16 * R));
    const int64_t run = run_length(total, a.nw);
    // the unit that a workgroup's first chunk lies in, or the one that its run
    // ends inside of: the latter also covers the former of the next workgroup,
    // so a unit that continues is looked at from its first chunk here
    for (int part = 0; part < 2; ++part) {
        const int64_t x = blockIdx.x * run, x_end = min(total, x + run);
        if (x >= x_end) return;
        const int64_t at = part == 0 ? x : x_end - 1;
        int64_t f = 0;
        const int b = __builtin_amdgcn_readfirstlane(find_seq(a, grp, 16 * R, at, &f));
        f = uniform64(f);
        const Seq sq = seq_of(a, b, grp, 16 * R);
        const int unit = __builtin_amdgcn_readfirstlane(static_cast<int>((at - f) / sq.chunks));
        const int64_t u0 = f + static_cast<int64_t>(unit) * sq.chunks, u1 = u0 + sq.chunks;
        if (part == 0 && u0 >= x) continue;                // not a continued unit
        if (part == 1 && (u0 < x || u1 <= x_end)) continue;    // seen as part 0, or whole
        const int i0 = static_cast<int>(u0 / run), i1 = static_cast<int>((u1 - 1) / run), n = i1 - i0 + 1;
        const int kvh = unit / sq.tiles, row0 = unit % sq.tiles * 16 * R;
        const int n_rows = min(16 * R, sq.n * grp - row0);
        for (int r = static_cast<int>(blockIdx.x) - i0; r < n_rows; r += n) {
            const int pw = tid / LD, l = tid % LD;
            float m = -__builtin_inff(), ls = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int p = pw; p < n; p += PW) {
                // a piece is its workgroup's first one (continued) unless the unit starts there
                const int64_t slot = 2 * static_cast<int64_t>(i0 + p) + (u0 >= (i0 + p) * run ? 1 : 0);
                const int64_t row = slot * (16 * R) + r;
                const float mp = a.part_ml[2 * row], lp = a.part_ml[2 * row + 1];
                const float4 v = *reinterpret_cast<const float4 *>(a.part_o + row * D + 4 * l);
                const float mn = fmaxf(m, mp);
                const float a0 = m == -__builtin_inff() ? 0.f : exp_two(m - mn);
                const float a1 = mp == -__builtin_inff() ? 0.f : exp_two(mp - mn);
                ls = ls * (ls == ls ? a0 : 1.f) + (lp == lp ? lp * a1 : lp);
                o.x = (a0 == 0.f ? 0.f : o.x * a0) + (a1 == 0.f ? 0.f : v.x * a1);
                o.y = (a0 == 0.f ? 0.f : o.y * a0) + (a1 == 0.f ? 0.f : v.y * a1);
                o.z = (a0 == 0.f ? 0.f : o.z * a0) + (a1 == 0.f ? 0.f : v.z * a1);
                o.w = (a0 == 0.f ? 0.f : o.w * a0) + (a1 == 0.f ? 0.f : v.w * a1);
                m = mn;
            }
            __syncthreads();
            acc_s[pw][l] = o;
            if (l == 0) ml_s[pw] = make_float2(m, ls);
            __syncthreads();
            if (pw == 0) {
#pragma unroll
                for (int p = 1; p < PW; ++p) m = fmaxf(m, ml_s[p].x);
                float lt = 0.f;
                float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int p = 0; p < PW; ++p) {
                    const float mp = ml_s[p].x, al = mp == -__builtin_inff() ? 0.f : exp_two(mp - m), lp = ml_s[p].y;
                    lt += lp == lp ? lp * al : lp;
                    const float4 v = acc_s[p][l];
                    t.x += al == 0.f ? 0.f : v.x * al;
                    t.y += al == 0.f ? 0.f : v.y * al;
                    t.z += al == 0.f ? 0.f : v.z * al;
                    t.w += al == 0.f ? 0.f : v.w * al;
                }
                const float inv = lt == 0.f ? 0.f : 1.f / lt;
                const int rho = row0 + r;
                uint16_t *op = static_cast<uint16_t *>(a.o.p) + (sq.q0 + rho / grp) * a.o.st +
                               (kvh * grp + rho % grp) * a.o.sh + 4 * l;
                *reinterpret_cast<uint2 *>(op) = make_uint2(pack_bf16x2(t.x * inv, t.y * inv), pack_bf16x2(t.z * inv, t.w * inv));
            }
        }
    }
}

namespace {

// 16-row tiles per wave: as many as an average sequence's query rows fill
int row_tiles(int64_t T, int64_t B, int64_t grp) {
    const int64_t rows = (T * grp + B - 1) / B;
    return rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
}

template <int D, bool MX, int R>
hipError_t launch(const PagedArgs &a, hipStream_t stream) {
    if (a.idx) paged_attn_kernel<D, MX, R, true><<<a.nw, pg::kThreads, 0, stream>>>(a);
    else paged_attn_kernel<D, MX, R, false><<<a.nw, pg::kThreads, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    paged_merge_kernel<D, R><<<a.nw, pg::kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

template <int D, bool MX>
hipError_t launch_rows(const PagedArgs &a, int R, hipStream_t stream) {
    if (R == 1) return launch<D, MX, 1>(a, stream);
    if (R == 2) return launch<D, MX, 2>(a, stream);
    return launch<D, MX, 4>(a, stream);
}

}  // namespace

size_t paged_workspace_bytes(int64_t T, int64_t B, int64_t H, int64_t Hkv, int D) {
    const int64_t rows = 2 * pg::kMaxGroups * 16 * row_tiles(T, B, H / Hkv);
    return static_cast<size_t>(rows) * (D + 2) * sizeof(float);
}

hipError_t launch_paged_attn(PagedArgs a, int D, void *workspace, hipStream_t stream) {
    const int R = row_tiles(a.T, a.B, a.q.n / a.kv.Hkv);
    a.nw = pg::kMaxGroups;
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = a.part_o + static_cast<int64_t>(2 * pg::kMaxGroups * 16 * R) * D;
    if (a.kv.mx) return D == 128 ? launch_rows<128, true>(a, R, stream) : launch_rows<64, true>(a, R, stream);
    return D == 128 ? launch_rows<128, false>(a, R, stream) : launch_rows<64, false>(a, R, stream);
}

}  // namespace rmm
