// Attention of new tokens over a paged key/value cache (bf16, or MXFP4: 4-bit
// codes with one power-of-two scale per 32 dims):
//   O[t][h] = softmax(scale * Q[t][h][I] . K[s][g][I]) V[s][g],  s the positions the
//   token sees, I all dims or the (token, head)'s retained ones
//
// A query row is one (new token, query head of a kv head): the heads of a group
// share every key read.  A unit is one (sequence, kv head, tile of query rows).
//
//   few rows (a decode step, drafted tokens): paged_few_kernel, units of 16 to 64
//   rows.  The four waves of a workgroup take 32-key chunks in turn; keys and values
//   go from memory to registers to the matrix cores without LDS.  Bound by reading
//   the cache.
//   more rows (prompt chunks): paged_rows_kernel, units of 256 rows, 32 per wave,
//   over 64-key tiles staged once per workgroup in an LDS ring.  Bound by the matrix
//   cores and the exponentials beside them.
// unit_rows says which, with what both measured.
//
// Lengths are known on the device only, and a batch may hold one long sequence
// among short ones, so the work is cut there: the key blocks of all units lie on
// one line, which is cut into equal runs, one per workgroup.  A unit inside one
// run is written at once; the pieces of a cut one go to the workspace as (maximum,
// sum, unnormalised output) and a second launch joins them in order.  Where whole
// units spread over the workgroups as well, but for less than what the pieces cost,
// the line is cut between units instead.
//
// With the causal mask a unit ends at the last key that any of its rows sees.
// Row tiles are laid on the line in pairs of one early and one late tile, which
// have the same number of blocks (to within the two that the pair's length allows).
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "kernels.h"
#include "kv_cache.h"
#include "paged_plan.h"

namespace rmm {

namespace {

namespace pg {
// A row's reference lies this far above its maximum (log2 units): weights are 2^-32 at
// most, so that sums over 2^30 keys of values up to the type's largest stay in fp32.
// They are powers of two times what they would be otherwise, and bf16 has fp32's exponents;
// values below 2^-94 lose bits to it.  The reference follows every new maximum: the largest
// weight is then a power of two, which bf16 holds exactly.  Following only a maximum 2^8
// above the last one gave that weight the others' rounding (two chunks of 1024 tokens
// 0.0020 off float64 for 0.0017, the output's own rounding being 0.0016; 5 drafted tokens
// 0.0018 for 0.0016; single tokens 0.0017 for 0.00165) and saved up to 3 % (the chunks
// 250 us for 254, heads of 64 176 for 182; single tokens nothing).
constexpr float kLift = 32.f;

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
// f over the lanes l, l ^ 32
template <typename F>
__device__ __forceinline__ float across_halves(float x, F f) {
#if defined(__HIP_DEVICE_COMPILE__)
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(b[0]), __uint_as_float(b[1]));
#endif
    return x;
}
__device__ __forceinline__ float fmax2(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float add2(float a, float b) { return a + b; }

__device__ __forceinline__ f32x4_t mfma(const uint4 a, const uint4 b, const f32x4_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
#else
    return c;
#endif
}
__device__ __forceinline__ f32x16_t mfma(const uint4 a, const uint4 b, const f32x16_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
#else
    return c;
#endif
}
// two codes (byte B of w) as packed bf16, exact
template <int B>
__device__ __forceinline__ uint32_t unpack_mx(uint32_t w, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
#else
    return 0;
#endif
}
__device__ __forceinline__ uint4 unpack_mx8(uint32_t w, float scale) {
    return make_uint4(unpack_mx<0>(w, scale), unpack_mx<1>(w, scale), unpack_mx<2>(w, scale), unpack_mx<3>(w, scale));
}
// s + the two bf16 values of w
__device__ __forceinline__ float add_pair(uint32_t w, float s) {
#if defined(__HIP_DEVICE_COMPILE__)
    const bf16x2_t one = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), one, s, false);
#else
    return s;
#endif
}
__device__ __forceinline__ float exp_two(float x) { return __builtin_amdgcn_exp2f(x); }
// what a row's weighted sum is multiplied with; lim: the last key that the row sees.
// A sum of zero is a softmax of nothing but -inf (NaN), or of no key (0).
__device__ __forceinline__ float row_scale(float sum, int lim) {
    return sum == 0.f ? (lim < 0 ? 0.f : __builtin_nanf("")) : 1.f / sum;
}
// of 8 bf16 values (w), those at the set bits of m
__device__ __forceinline__ uint4 keep8(uint4 w, uint32_t m) {
    w.x &= (m & 1 ? 0xffffu : 0u) | (m & 2 ? 0xffff0000u : 0u);
    w.y &= (m & 4 ? 0xffffu : 0u) | (m & 8 ? 0xffff0000u : 0u);
    w.z &= (m & 16 ? 0xffffu : 0u) | (m & 32 ? 0xffff0000u : 0u);
    w.w &= (m & 64 ? 0xffffu : 0u) | (m & 128 ? 0xffff0000u : 0u);
    return w;
}

// x, in a form that keeps what depends on it inside the branch it is used in (a
// rarely taken one would be turned into selects that every pass pays for)
__device__ __forceinline__ int in_branch(int x) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+v"(x));
#endif
    return x;
}

__device__ __forceinline__ int64_t uniform(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(static_cast<uint64_t>(x) >> 32));
    return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}
// x or that of the lane that the DPP control CTRL names; every lane must be active
template <int CTRL>
__device__ __forceinline__ uint32_t or_row(uint32_t x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return x | static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, 0xF, 0xF, false));
#else
    return x;
#endif
}
// inclusive prefix sum over the wave's lanes
__device__ __forceinline__ int prefix_sum(int x) {
#if defined(__HIP_DEVICE_COMPILE__)
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);      // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);     // lane 15 of a row to the next row
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);     // lane 31 to the upper half
#endif
    return x;
}

// The workgroup's run
template <int TK, int ROWS>
__device__ __forceinline__ bool Walk<TK, ROWS>::init(const PagedArgs &a, int min_run, int cut_cost) {
    const int lane = threadIdx.x & 63;
    pl.grp = a.q.n / a.kv.Hkv;
    pl.causal = a.causal;
    pl.Hkv = a.kv.Hkv;
    pl.whole = false;
    // the line's length in blocks and in units, the longest unit: lane l looks
    // at sequences l, l + 64, ...
    Seq mine = {0, 0, 0, 0};
    if (lane < a.B) mine = pl.load(a, lane);
    int64_t tokens = mine.n;
    int most = pl.longest(mine), most2 = pl.longest_pair(mine);
    int w0 = pl.work(mine), blocks = w0, units = pl.units(mine);
    for (int i = lane + 64; i < a.B; i += 64) {
        const Seq q = pl.load(a, i);
        most = max(most, pl.longest(q));
        most2 = max(most2, pl.longest_pair(q));
        blocks += pl.work(q);
        units += pl.units(q);
        tokens = min(tokens + q.n, a.T + 1);
    }
    wg = static_cast<int>(blockIdx.x);
    over = false;
    if (a.q_start) {                      // a lane's share is at most 2^31
        const int lo = prefix_sum(static_cast<int>(tokens & 0xffff)), hi = prefix_sum(static_cast<int>(tokens >> 16));
        over = (static_cast<int64_t>(__builtin_amdgcn_readlane(hi, 63)) << 16) + __builtin_amdgcn_readlane(lo, 63) > a.T;
        if (over) return false;
    }
    int sum0 = prefix_sum(blocks);
    int total = __builtin_amdgcn_readlane(sum0, 63);
    if (a.whole) {
        pl.whole = true;
    } else {
        const int nu = __builtin_amdgcn_readlane(prefix_sum(units), 63);
        const int rounds = quot(nu + a.nw - 1, a.nw), room = quot(total, a.nw) + cut_cost;
        pl.whole = __ballot((rounds >> 1) * most2 + (rounds & 1) * most > room) == 0;
    }
    if (pl.whole) {
        w0 = pl.units(mine);
        sum0 = prefix_sum(units);
        total = __builtin_amdgcn_readlane(sum0, 63);
    }
    if (a.B > 64) sum0 = prefix_sum(w0);
    run = quot(total + a.nw - 1, a.nw);
    run = pl.whole ? max(run, 1) : (max(run, min_run) + 3) / 4 * 4;
    // consecutive runs on one XCD (workgroups are dealt to the 8 XCDs in turn),
    // where units that share keys share its L2, the XCDs evenly used
    const int i0 = static_cast<int>(blockIdx.x), runs = quot(total + run - 1, run), per = (runs + 7) >> 3;
    wg = i0;                          // idle workgroups keep the places behind the runs
    if ((i0 >> 3) < per) wg = (i0 & 7) * per + (i0 >> 3);
    if ((i0 >> 3) >= per || wg >= runs) return false;
    begin = x = wg * run;
    end = min(total - x, run) + x;
    // the sequence at x
    int base = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        Seq q = mine;
        int w = w0, sum = sum0;
        if (b0 > 0) {
            q = b0 + lane < a.B ? pl.load(a, b0 + lane) : Seq{0, 0, 0, 0};
            w = pl.work(q);
            sum = prefix_sum(w);
        }
        const uint64_t past = __ballot(base + sum > x);
        if (past) {
            const int l = __builtin_ctzll(past);
            b = b0 + l;
            f = base + __builtin_amdgcn_readlane(sum - w, l);
            s.q0 = __builtin_amdgcn_readlane(q.q0, l);
            s.n = __builtin_amdgcn_readlane(q.n, l);
            s.len = __builtin_amdgcn_readlane(q.len, l);
            s.bad = __builtin_amdgcn_readlane(q.bad, l);
            break;
        }
        base += __builtin_amdgcn_readlane(sum, 63);
    }
    return true;
}

// What the joining launch needs to know of a workgroup's piece of a cut unit:
// the unit's workgroups first .. first + n - 1 (n = 0: no piece), its rows
struct PieceOf {
    int n, first, rows, q0, kvh, row0, lim0, pad;         // lim0: last key that the sequence's first token sees
};
// A workgroup has at most two pieces: of the unit its run begins inside of
// (slot 0) and of the one it ends inside of (slot 1)
template <int TK, int ROWS>
__device__ __forceinline__ PieceOf piece_of(const Walk<TK, ROWS> &w, int rows) {
    const int first = quot(w.u0, w.run), last = quot(w.u1 - 1, w.run);
    return {last - first + 1, first, rows, w.s.q0, w.kvh, w.tile * ROWS, w.pl.causal ? w.s.len - w.s.n : w.s.len - 1, 0};
}

// NaN for every output: what a q_start gives whose sequences overlap
template <int D>
__device__ __forceinline__ void all_nan(const PagedArgs &a) {
    const int64_t n = a.T * a.o.n * (D / 8);
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        const int64_t row = i / (D / 8);
        uint16_t *op = static_cast<uint16_t *>(a.o.p) + row / a.o.n * a.o.st + row % a.o.n * a.o.sh + 8 * (i % (D / 8));
        *reinterpret_cast<uint4 *>(op) = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
    }
}

// dims d, d + 1 of a cached row
template <int D, bool MX>
__device__ __forceinline__ float2 cached_pair(const uint8_t *rows, const uint8_t *scales, int64_t row, int d) {
    uint32_t w;
    if constexpr (MX) w = unpack_mx<0>(rows[row * (D / 2) + d / 2], __uint_as_float(static_cast<uint32_t>(scales[row * (D / 32) + d / 32]) << 23));
    else w = *reinterpret_cast<const uint32_t *>(rows + (row * D + d) * 2);
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// whether a value of keys [k0, k1) of kv head kvh is infinite or NaN (whole waves,
// the same answer in each)
template <int D, bool MX>
__device__ __forceinline__ bool odd_values(const PagedArgs &a, int b, int kvh, int k0, int k1) {
    const int lg = a.kv.lg_page;
    const int32_t *trow = a.table + b * a.table_ld;
    bool odd = false;
#pragma unroll 1
    for (int i = threadIdx.x & 63; i < (k1 - k0) * (D / 2); i += 64) {
        const int key = k0 + i / (D / 2), pid = trow[key >> lg], page = pid >= 0 && pid < a.kv.n_pages ? pid : 0;
        const int64_t row = (static_cast<int64_t>(kvh) << lg) + (key & ((1 << lg) - 1));
        const float2 v = cached_pair<D, MX>(a.kv.v + page * a.kv.v_page, a.kv.vs + page * a.kv.vs_page, row, 2 * (i % (D / 2)));
        odd = odd || !(__builtin_fabsf(v.x) < __builtin_inff()) || !(__builtin_fabsf(v.y) < __builtin_inff());
    }
    return __ballot(odd) != 0;
}

// The query rows r of a unit for which wants(r) holds over its keys [k0, k1), one row
// per wave (the first of `step`) with nothing shared between rows: what a unit's rows are
// redone with whose result is not finite, where a weight or a query of zero may not have
// silenced a key or value that the row does not see.  A row with a NaN weight is NaN: the
// rest of its keys are left out.  put(row, m, l,
// d, o): reference, sum and two dims of a row's output, called by every lane that holds some.
template <int D, bool MX, bool IDX, typename Wants, typename Put>
__device__ __forceinline__ void careful_rows(const PagedArgs &a, const Seq &sq, int b, int kvh, int row0, int n_rows,
                                             int first, int step, int k0, int k1, const uint32_t (*keep)[D / 32],
                                             Wants wants, Put put) {
    const int lane = threadIdx.x & 63, grp = a.q.n / a.kv.Hkv, lg = a.kv.lg_page;
    const int32_t *trow = a.table + b * a.table_ld;
    const int d2 = 2 * lane;                               // the lane's output dims (D / 2 lanes)
    int nth = 0;
#pragma unroll 1
    for (int r = 0; r < n_rows; ++r) {                     // wave-uniform
        if (!wants(r) || nth++ % step != first) continue;
        const int tok = (row0 + r) / grp, hd = kvh * grp + (row0 + r) % grp;
        const int see = min(k1, a.causal ? sq.len - sq.n + tok + 1 : sq.len);
        const uint16_t *qp = static_cast<const uint16_t *>(a.q.p) + (sq.q0 + tok) * a.q.st + hd * a.q.sh;
        float m = -__builtin_inff(), l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll 1
        for (int key0 = k0; key0 < see; key0 += 64) {
            const int key = key0 + lane, pid = key < see ? trow[key >> lg] : 0;
            const int page = pid >= 0 && pid < a.kv.n_pages ? pid : 0;
            const int64_t row = (static_cast<int64_t>(kvh) << lg) + (key & ((1 << lg) - 1));
            float sc = -__builtin_inff();
            if (key < see) {
                const uint8_t *kp = a.kv.k + page * a.kv.k_page, *sp = a.kv.ks + page * a.kv.ks_page;
                float x = 0.f;
#pragma unroll 1
                for (int d = 0; d < D; d += 2) {
                    const float2 k = cached_pair<D, MX>(kp, sp, row, d);
                    const uint32_t bits = IDX ? keep[r][d >> 5] >> (d & 31) : 3u;
                    if (bits & 1) x += bf16_to_f32(qp[d]) * k.x;
                    if (bits & 2) x += bf16_to_f32(qp[d + 1]) * k.y;
                }
                sc = x * a.c;
            }
            float mx = sc;
#pragma unroll
            for (int i = 32; i > 0; i >>= 1) mx = fmaxf(mx, __shfl_xor(mx, i, 64));
            const float mn = fmaxf(m, mx + kLift), use = mn == -__builtin_inff() ? 0.f : mn;
            const float al = exp_two((m == -__builtin_inff() ? use : m) - use);
            const float p = bf16_to_f32(f32_to_bf16(exp_two(sc - use)));
            l *= al;
            o0 *= al;
            o1 *= al;
            m = mn;
            float ps = p;
#pragma unroll
            for (int i = 32; i > 0; i >>= 1) ps += __shfl_xor(ps, i, 64);
            l += ps;
            if (l != l) break;                             // the same in every lane
#pragma unroll 1
            for (int i = 0; i < min(64, see - key0); ++i) {
                const float w = __shfl(p, i, 64);
                const int64_t pg = __shfl(page, i, 64);
                const int64_t vrow = (static_cast<int64_t>(kvh) << lg) + ((key0 + i) & ((1 << lg) - 1));
                if (d2 < D) {
                    const float2 v = cached_pair<D, MX>(a.kv.v + pg * a.kv.v_page, a.kv.vs + pg * a.kv.vs_page, vrow, d2);
                    o0 += w * v.x;
                    o1 += w * v.y;
                }
            }
        }
        if (d2 < D) put(r, m, l, d2, o0, o1);
    }
}

// The retained dims of a unit's rows as bits; dims outside [0, D) are ignored.  16
// lanes per row, each with up to D / 16 entries of its list, up to four rows' lists
// per lane asked for at once (whole waves together).
template <int D, int NT, int ROWS>
__device__ __forceinline__ void read_lists(const PagedArgs &a, const Seq &sq, int kvh, int row0, int n_rows, uint32_t (*keep)[D / 32]) {
    constexpr int E = D / 16, W = D / 32, STEP = NT / 16;
    constexpr int M = ROWS <= STEP ? 1 : ROWS <= 2 * STEP ? 2 : 4;
    const int H = a.q.n, grp = H / a.kv.Hkv, u0 = threadIdx.x & 15, n4 = (n_rows + 3) / 4 * 4;
    for (int r = threadIdx.x >> 4; r < n4; r += M * STEP) {
        int d[M][E];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            if (r + m * STEP >= n4) break;
            const int q = row0 + min(r + m * STEP, n_rows - 1);
            const int32_t *list = a.idx + (static_cast<int64_t>(sq.q0 + q / grp) * H + kvh * grp + q % grp) * a.k;
#pragma unroll
            for (int i = 0; i < E; ++i) d[m][i] = u0 + 16 * i < a.k ? list[u0 + 16 * i] : -1;
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            if (r + m * STEP >= n4) break;
            uint32_t w[W];
#pragma unroll
            for (int j = 0; j < W; ++j) {
                w[j] = 0;
#pragma unroll
                for (int i = 0; i < E; ++i) w[j] |= (d[m][i] >> 5) == j ? 1u << (d[m][i] & 31) : 0u;
                w[j] = or_row<0xB1>(w[j]);                 // over the 16 lanes: l ^ 1, l ^ 2, mirrored in 8, in 16
                w[j] = or_row<0x4E>(w[j]);
                w[j] = or_row<0x141>(w[j]);
                w[j] = or_row<0x140>(w[j]);
            }
            if (r + m * STEP < n_rows && u0 == 0) {
#pragma unroll
                for (int j = 0; j < W; ++j) keep[r + m * STEP][j] = w[j];
            }
        }
    }
}

template <int N>
__device__ __forceinline__ void wait_vmcnt_le() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}
}  // namespace pg

}  // namespace

// ------------------------------------------------------------- few rows
// S^T = K Q^T takes 16 key rows as they are loaded (v_mfma_f32_16x16x32: a lane
// holds 8 dims of one key).  In its result a lane holds one query row, and with
// key 8 g + 4 tb + i at row 4 g + i of key tile tb exactly the eight keys that
// its lane group contributes to O^T = V^T P^T: the weights stay where they are.
// The value rows, loaded as rows, are turned 8 x 8 in registers (v_perm).  4-bit
// codes become bf16 with v_cvt_scalef32_pk_bf16_fp4 (exact, the scale included).
// Bound by reading the cache, 16 bytes per lane and load, a wave's next chunk on
// its way while one is used.  32 heads of 128 on 8, one token per sequence: 16
// sequences of up to 8000 keys (318 MB) 65 us, 4.9 TB/s, and 6 joining; two of
// 131000 in 4 bits (285 MB) 62 us, 4.6 TB/s, and 6; one of 200 8.6 us, all latency.
// R: 16-row tiles per wave, which share each key and value fragment (their queries
// are then kept in LDS); RG: groups of waves with rows of their own, which walk the
// same chunks side by side, so that all but the first read them from a cache;
// MX: 4-bit cache; IDX: scores over retained dims
template <int D, bool MX, int R, int RG, bool IDX>
__global__ __launch_bounds__(few::kThreads, 2) void paged_few_kernel(PagedArgs a) {
    using namespace pg;
    using namespace few;
    constexpr int WROWS = 16 * R, ROWS = WROWS * RG, KG = kWaves / RG;       // rows per wave, per unit; chunk streams
    constexpr int KS = D / 32, DM = D / 16;               // contraction steps of S^T, MFMA rows of O^T
    constexpr int ROWB = MX ? D / 2 : D * 2, SROWB = D / 32;    // bytes per cached row, scale bytes per row
    constexpr int OLD = D + 4;                            // row stride of the joining buffer, floats
    constexpr int NBUF = MX && R == 1 ? 2 : 1;            // chunks held
    __shared__ __attribute__((aligned(16))) float oj[kWaves][16][OLD];
    __shared__ float ml[kWaves][16][2];
    __shared__ int bad_of[kWaves];                        // a page or length out of range
    __shared__ uint64_t odd_of[kWaves];                   // rows whose result is not finite
    __shared__ uint32_t keep[IDX ? ROWS : 1][KS];
    __shared__ uint4 qs[R > 1 ? R * RG : 1][KS][R > 1 ? 64 : 1];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rg = wave % RG, kg = wave / RG;
    const int col = lane & 15, g = lane >> 4;
    const int H = a.q.n, grp = H / a.kv.Hkv;
    const int lg = a.kv.lg_page, ps = 1 << lg;

    int held = 0;                                          // which of the two pieces there are
    Walk<TK, ROWS> w;
    bool more = w.init(a, kMinRun, kCutCost);
    const int wg = w.wg;
    if (w.over) all_nan<D>(a);
    while (more) {
        if (!w.locate(a)) {
            more = w.x < w.end;
            continue;
        }
        const Seq sq = w.s;
        const int kvh = w.kvh, row0 = w.tile * ROWS, n_rows = min(ROWS, sq.n * grp - row0);

        // last key of the lane's rows; the first limit and the last of the unit's rows
        int lim[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int rr = rg * WROWS + 16 * r + col;
            lim[r] = rr >= n_rows ? -1 : a.causal ? sq.len - sq.n + (row0 + rr) / grp : sq.len - 1;
        }
        const int lo_lim = a.causal ? sq.len - sq.n + quot(row0, grp) : sq.len - 1;
        const int hi_lim = a.causal ? sq.len - sq.n + quot(row0 + n_rows - 1, grp) : sq.len - 1;
        // a wave without rows has no chunks
        const int c_stop = rg * WROWS < n_rows ? min(w.c1, hi_lim < 0 ? 0 : hi_lim / TK + 1) : 0;

        bool bad = sq.bad;

        // ---- the wave's chunks c0 + kg, + KG, ...; lane l holds the pages of the
        // l-th of them (two where a page has 16 keys)
        const int32_t *trow = a.table + w.b * a.table_ld;
        int pid_a = 0, pid_b = 0;
        auto fetch_pages = [&](int c) __attribute__((always_inline)) {
            const bool in = c + KG * lane < c_stop;
            const int key = in ? (c + KG * lane) * TK : 0;
            const int p0 = key >> lg, p1 = in && key + 16 < sq.len ? (key + 16) >> lg : p0;
            pid_a = in ? trow[p0] : 0;
            pid_b = in ? trow[p1] : 0;
            const bool oka = pid_a >= 0 && pid_a < a.kv.n_pages, okb = pid_b >= 0 && pid_b < a.kv.n_pages;
            if (__ballot(!oka || !okb)) bad = true;
            if (!oka) pid_a = 0;
            if (!okb) pid_b = 0;
        };
        // keys 8 (col / 4) + 4 tb + col % 4 of the chunk (K), 8 g + kk (V): the
        // lane's first row, among the second 16 keys for `second` lanes
        auto row_at = [&](const uint8_t *base, int64_t page_bytes, int row_bytes, int c, int nth, bool second,
                          int row) __attribute__((always_inline)) {
            const int64_t pa = __builtin_amdgcn_readlane(pid_a, nth), pb = __builtin_amdgcn_readlane(pid_b, nth);
            const int key = c * TK, oa = key & (ps - 1), ob = ((key + 16) & (ps - 1)) - 16;
            const int64_t hrow = static_cast<int64_t>(kvh) << lg;
            const uint8_t *ra = base + pa * page_bytes + (hrow + oa) * row_bytes;
            const uint8_t *rb = base + pb * page_bytes + (hrow + ob) * row_bytes;
            return (second ? rb : ra) + row * row_bytes;
        };
        struct Raw {
            uint4 k[2][MX ? 1 : KS], v[MX ? 1 : 8], vs[MX ? 2 : 1];
            uint32_t ks[2], vc[8];
        };
        auto load_k = [&](Raw &x, int c, int nth) __attribute__((always_inline)) {
            const int krow = 8 * (col >> 2) + (col & 3);
            const uint8_t *kp = row_at(a.kv.k, a.kv.k_page, ROWB, c, nth, col >= 8, krow);
            if constexpr (!MX) {
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        x.k[tb][s] = *reinterpret_cast<const uint4 *>(kp + tb * 4 * ROWB + 64 * s + 16 * g);
            } else {
                const uint8_t *sp = row_at(a.kv.ks, a.kv.ks_page, SROWB, c, nth, col >= 8, krow);
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) {
                    if constexpr (D == 128) {
                        x.k[tb][0] = *reinterpret_cast<const uint4 *>(kp + tb * 4 * ROWB + 16 * g);
                        x.ks[tb] = sp[tb * 4 * SROWB + g];
                    } else {
                        const uint2 y = *reinterpret_cast<const uint2 *>(kp + tb * 4 * ROWB + 8 * g);
                        x.k[tb][0] = make_uint4(y.x, y.y, 0, 0);
                        x.ks[tb] = sp[tb * 4 * SROWB + (g >> 1)];
                    }
                }
            }
        };
        auto load_v = [&](Raw &x, int c, int nth) __attribute__((always_inline)) {
            const uint8_t *vp = row_at(a.kv.v, a.kv.v_page, ROWB, c, nth, g >= 2, 8 * g);
            if constexpr (!MX) {
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    if constexpr (D == 128) {
                        x.v[kk] = *reinterpret_cast<const uint4 *>(vp + kk * ROWB + 16 * col);
                    } else {
                        const uint2 y = *reinterpret_cast<const uint2 *>(vp + kk * ROWB + 8 * col);
                        x.v[kk] = make_uint4(y.x, y.y, 0, 0);
                    }
                }
            } else {
                const uint8_t *sp = row_at(a.kv.vs, a.kv.vs_page, SROWB, c, nth, g >= 2, 8 * g);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    if constexpr (D == 128) x.vc[kk] = *reinterpret_cast<const uint32_t *>(vp + kk * ROWB + 4 * col);
                    else x.vc[kk] = *reinterpret_cast<const uint16_t *>(vp + kk * ROWB + 2 * col);
                }
                x.vs[0] = reinterpret_cast<const uint4 *>(sp)[0];
                if constexpr (D == 128) x.vs[MX ? 1 : 0] = reinterpret_cast<const uint4 *>(sp)[1];
            }
        };

        // the first chunks are on their way while the lists and queries are read
        Raw raw[NBUF];
        int c = w.c0 + kg;
        auto first = [&]() __attribute__((always_inline)) {    // up to 64 chunks per fetch of page numbers
            fetch_pages(c);
            load_k(raw[0], c, 0);
            load_v(raw[0], c, 0);
            if constexpr (NBUF == 2) {
                if (c + KG < c_stop) {
                    load_k(raw[NBUF - 1], c + KG, 1);
                    load_v(raw[NBUF - 1], c + KG, 1);
                }
            }
        };
        if (c < c_stop) first();

        // ---- the unit's query rows
        // dims that lane (col, g) holds at contraction step s
        auto dim_of = [&](int s) { return MX ? (D / 4) * g + 8 * s : 32 * s + 8 * g; };
        auto query = [&](int r, int s) __attribute__((always_inline)) {
            const int rr = 16 * r + col;
            if (rr >= n_rows) return make_uint4(0, 0, 0, 0);
            const int rho = row0 + rr, tok = rho / grp;
            const uint16_t *qp = static_cast<const uint16_t *>(a.q.p) + (sq.q0 + tok) * a.q.st + (kvh * grp + rho - tok * grp) * a.q.sh;
            return *reinterpret_cast<const uint4 *>(qp + dim_of(s));
        };
        auto kept = [&](int r, int s, uint4 x) __attribute__((always_inline)) {
            if constexpr (IDX) return keep8(x, keep[16 * r + col][dim_of(s) >> 5] >> (dim_of(s) & 31));
            return x;
        };
        // the queries that this wave reads: all of its rows' (R = 1), or its share of the unit's
        constexpr int NQ = R > 1 ? R * RG * KS / kWaves : KS;
        uint4 qf[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) qf[i] = R > 1 ? query((wave + kWaves * i) / KS, (wave + kWaves * i) % KS) : query(0, i);
        if constexpr (IDX) {
            read_lists<D, kThreads, ROWS>(a, sq, kvh, row0, n_rows, keep);
            lds_barrier();
        }
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if constexpr (R == 1) qf[i] = kept(0, i, qf[i]);
            else {
                const int r = (wave + kWaves * i) / KS, s = (wave + kWaves * i) % KS;
                qs[r][s][lane] = kept(r, s, qf[i]);
            }
        }
        if constexpr (R > 1) lds_barrier();
        f32x4_t o[R][DM];
        float m_run[R], l_run[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m_run[r] = -__builtin_inff();
            l_run[r] = 0.f;
#pragma unroll
            for (int i = 0; i < DM; ++i) o[r][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        // chunk c, held in x; the keys and then the values of the chunk that takes its
        // place are asked for as soon as its own are used up
        auto chunk = [&](Raw &x, int c, int nth, bool next) __attribute__((always_inline)) {
            const int key = c * TK;
            const bool edge = key + TK - 1 > lo_lim;       // wave-uniform: some row does not see every key
            uint4 kf[2][KS];
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                const uint32_t cw[4] = {x.k[tb][0].x, x.k[tb][0].y, x.k[tb][0].z, x.k[tb][0].w};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    if constexpr (MX) kf[tb][s] = unpack_mx8(cw[s], __uint_as_float(x.ks[tb] << 23));
                    else kf[tb][s] = x.k[tb][s];
                }
            }
            uint4 pf[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                f32x4_t sc[2];
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) sc[tb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    uint4 q;
                    if constexpr (R == 1) q = qf[s];
                    else q = qs[rg * R + r][s][lane];
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb) sc[tb] = mfma(kf[tb][s], q, sc[tb]);
                }
                // the next keys as soon as these are used up
                if (r == R - 1 && next) load_k(x, c + KG * NBUF, nth + NBUF);
                // ---- weights
                float p[2][4], mx = -__builtin_inff();
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[tb][i] = sc[tb][i] * a.c;
                if (edge) {
                    const int rel = in_branch(lim[r] - key - 8 * g);
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (4 * tb + i > rel) p[tb][i] = -__builtin_inff();
                }
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, p[tb][i]);
                mx = across_rows(mx, fmax2);
                if (__ballot(mx > m_run[r] - kLift)) {
                    const float m_new = fmaxf(m_run[r], mx + kLift);
                    const float al = m_new == -__builtin_inff() ? 1.f : exp_two(m_run[r] - m_new);
                    l_run[r] *= al;
#pragma unroll
                    for (int i = 0; i < DM; ++i) o[r][i] *= al;
                    m_run[r] = m_new;
                }
                // a row with nothing kept yet has only masked (-inf) scores here
                const float m_use = m_run[r] == -__builtin_inff() ? 0.f : m_run[r];
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[tb][i] = exp_two(p[tb][i] - m_use);
                pf[r] = make_uint4(pack_bf16x2(p[0][0], p[0][1]), pack_bf16x2(p[0][2], p[0][3]),
                                   pack_bf16x2(p[1][0], p[1][1]), pack_bf16x2(p[1][2], p[1][3]));
                // the sum is of the rounded weights: they then sum to one, and a weight's
                // rounding moves the output only by its key's distance from it
                l_run[r] = add_pair(pf[r].w, add_pair(pf[r].z, add_pair(pf[r].y, add_pair(pf[r].x, l_run[r]))));
                // one row tile after the other: their scores together do not fit the registers
                if constexpr (R > 1) __builtin_amdgcn_sched_barrier(0);
            }
            // ---- O^T += V^T P^T: dim DM * col + i of the value rows at MFMA i
            uint32_t vr[8][DM / 2];
            if constexpr (!MX) {
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    const uint32_t y[4] = {x.v[kk].x, x.v[kk].y, x.v[kk].z, x.v[kk].w};
#pragma unroll
                    for (int q = 0; q < DM / 2; ++q) vr[kk][q] = y[q];
                }
            } else {
                const uint4 s2 = x.vs[MX ? 1 : 0];
                const uint32_t sw[8] = {x.vs[0].x, x.vs[0].y, x.vs[0].z, x.vs[0].w, s2.x, s2.y, s2.z, s2.w};
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    // D = 128: four scale bytes per row; D = 64: two
                    const uint32_t sb = D == 128 ? (sw[kk] >> (8 * (col >> 2))) & 0xffu
                                                 : (sw[kk >> 1] >> (16 * (kk & 1) + 8 * (col >> 3))) & 0xffu;
                    const uint4 y = unpack_mx8(x.vc[kk], __uint_as_float(sb << 23));
                    vr[kk][0] = y.x;
                    vr[kk][1] = y.y;
                    if constexpr (D == 128) {
                        vr[kk][2] = y.z;
                        vr[kk][3] = y.w;
                    }
                }
            }
            // a weight of zero does not silence what lies past the last key that some row sees
            if (key + TK - 1 > hi_lim) {
                const int rel = in_branch(hi_lim - key - 8 * g);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
#pragma unroll
                    for (int q = 0; q < DM / 2; ++q) vr[kk][q] = kk <= rel ? vr[kk][q] : 0u;
            }
#pragma unroll
            for (int i = 0; i < DM; ++i) {
                const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;
                const uint4 f = make_uint4(__builtin_amdgcn_perm(vr[1][i >> 1], vr[0][i >> 1], sel),
                                           __builtin_amdgcn_perm(vr[3][i >> 1], vr[2][i >> 1], sel),
                                           __builtin_amdgcn_perm(vr[5][i >> 1], vr[4][i >> 1], sel),
                                           __builtin_amdgcn_perm(vr[7][i >> 1], vr[6][i >> 1], sel));
#pragma unroll
                for (int r = 0; r < R; ++r) o[r][i] = mfma(f, pf[r], o[r][i]);
            }
            if (next) load_v(x, c + KG * NBUF, nth + NBUF);
        };
        while (c < c_stop) {
            const int n = min(64, (c_stop - c + KG - 1) / KG);
            for (int i = 0; i < n; i += NBUF) {
                chunk(raw[0], c + KG * i, i, i + NBUF < n);
                if constexpr (NBUF == 2) {
                    if (i + 1 < n) chunk(raw[NBUF - 1], c + KG * (i + 1), i + 1, i + 3 < n);
                }
            }
            c += KG * n;
            if (c < c_stop) first();
        }

        // ---- the waves of a row group join, 16 rows at a time
        const bool complete = w.complete();
        const int part = w.part();
        uint64_t odd = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            l_run[r] = across_rows(l_run[r], add2);
            bool fin = l_run[r] < __builtin_inff();
#pragma unroll
            for (int i = 0; i < DM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) fin = fin && __builtin_fabsf(o[r][i][e]) < __builtin_inff();
            uint64_t m = __ballot(!fin && rg * WROWS + 16 * r + col < n_rows);      // row col in four lanes
            m |= m >> 32;
            odd |= ((m | m >> 16) & 0xffff) << (rg * WROWS + 16 * r);
        }
        // row r of the unit: N dims from d on
        auto put = [&](int r, float m, float ls, int d, const auto &acc) __attribute__((always_inline)) {
            constexpr int N = sizeof(acc) / sizeof(float);
            if (complete) {
                const int q = row0 + r;
                const float inv = row_scale(ls, a.causal ? sq.len - sq.n + q / grp : sq.len - 1);
                uint16_t *op = static_cast<uint16_t *>(a.o.p) + (sq.q0 + q / grp) * a.o.st + (kvh * grp + q % grp) * a.o.sh + d;
                uint32_t y[N / 2];
#pragma unroll
                for (int i = 0; i < N / 2; ++i) y[i] = pack_bf16x2(acc[2 * i] * inv, acc[2 * i + 1] * inv);
                if constexpr (N == 8) *reinterpret_cast<uint4 *>(op) = make_uint4(y[0], y[1], y[2], y[3]);
                else if constexpr (N == 4) *reinterpret_cast<uint2 *>(op) = make_uint2(y[0], y[1]);
                else *reinterpret_cast<uint32_t *>(op) = y[0];
            } else {
                const int64_t prow = (2 * static_cast<int64_t>(wg) + part) * ROWS + r;
                if (d == 0) *reinterpret_cast<float2 *>(a.part_ml + 2 * prow) = make_float2(m, ls);
#pragma unroll
                for (int i = 0; i < N; i += N >= 4 ? 4 : 2) {
                    float *po = a.part_o + prow * D + d + i;
                    if constexpr (N >= 4) *reinterpret_cast<float4 *>(po) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
                    else *reinterpret_cast<float2 *>(po) = make_float2(acc[0], acc[1]);
                }
            }
        };
        bool none = false;                                 // no row of the unit has an answer
        uint64_t redo = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            __syncthreads();
            if (r == 0 && lane == 0) {
                bad_of[wave] = bad;
                odd_of[wave] = odd;
            }
            if (g == 0) {
                ml[wave][col][0] = m_run[r];
                ml[wave][col][1] = l_run[r];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < DM; i += 4)
                    *reinterpret_cast<float4 *>(&oj[wave][col][DM * (4 * g + e) + i]) =
                        make_float4(o[r][i][e], o[r][i + 1][e], o[r][i + 2][e], o[r][i + 3][e]);
            __syncthreads();
            if (r == 0) {
                none = (bad_of[0] | bad_of[1] | bad_of[2] | bad_of[3]) != 0;
                redo = odd_of[0] | odd_of[1] | odd_of[2] | odd_of[3];
                // an infinite or NaN key (outside a list) or value (of a key that only some rows
                // see) that should not count has made these NaN, as zero times it; without one
                // they are what they should be
                if (__builtin_expect(redo != 0, 0)) {
                    if (none || (!IDX && !odd_values<D, MX>(a, w.b, kvh, max(lo_lim + 1, w.c0 * TK), min(hi_lim + 1, w.c1 * TK))))
                        redo = 0;
                }
            }
            const int rr = tid >> 4, d0 = (tid & 15) * DM;
#pragma unroll
            for (int q = 0; q < RG; ++q) {                 // row group q is held by the waves q, q + RG, ...
                const int row = q * WROWS + 16 * r + rr;
                if (row >= n_rows || (redo >> row & 1)) continue;
                float m = -__builtin_inff(), ls = 0.f, acc[DM];
#pragma unroll
                for (int v = 0; v < KG; ++v) m = fmaxf(m, ml[q + RG * v][rr][0]);
#pragma unroll
                for (int i = 0; i < DM; ++i) acc[i] = 0.f;
#pragma unroll
                for (int v = 0; v < KG; ++v) {
                    const float mw = ml[q + RG * v][rr][0], al = mw == -__builtin_inff() ? 0.f : exp_two(mw - m);
                    ls += ml[q + RG * v][rr][1] * al;
#pragma unroll
                    for (int i = 0; i < DM; ++i) acc[i] += al * oj[q + RG * v][rr][d0 + i];
                }
                put(row, m, none ? __builtin_nanf("") : ls, d0, acc);
            }
        }
        if (__builtin_expect(redo != 0, 0))
            careful_rows<D, MX, IDX>(a, sq, w.b, kvh, row0, n_rows, wave, kWaves, w.c0 * TK, w.c1 * TK, keep,
                                     [&](int r) { return (redo >> r & 1) != 0; },
                                     [&](int r, float m, float ls, int d, float y, float z) {
                                         const float acc[2] = {y, z};
                                         put(r, m, ls, d, acc);
                                     });
        if (!complete) {
            if (tid == 0) reinterpret_cast<PieceOf *>(a.pieces)[2 * wg + part] = piece_of(w, n_rows);
            held |= 1 << part;
        }
        w.advance();
        more = w.x < w.end;
        if constexpr (IDX || R > 1) __syncthreads();       // the lists and queries are free for the next unit
    }
    if (tid < 2 && !(held >> tid & 1)) reinterpret_cast<PieceOf *>(a.pieces)[2 * wg + tid].n = 0;
}


// ------------------------------------------------------------ many rows
// Eight waves of 32 query rows over a ring of 64-key tiles in LDS, each filled two
// steps (bf16, by LDS DMA) or one step (4-bit, through registers, as bf16) ahead:
// S^T = K Q^T with v_mfma_f32_32x32x16 (a lane holds 16 keys of one row), online softmax in log2
// units, O^T += V^T P^T with V^T by the transposing LDS read.  Step i multiplies
// the keys of tile i and the values of tile i - 1; the two halves of the
// workgroup take the softmax at opposite ends of a step, so that one's
// exponentials meet the other's matrix instructions.
// Two prompts' chunks of 1024 tokens behind 7000 cached ones, 32 heads of 128 on 8
// (239 GFLOP): 247 to 260 us a call over several cards, 920 to 970 TFLOP/s of the 1103 that a
// large product reaches, 5 us of it joining; from a 4-bit cache 300 to 308, since the tiles
// then pass through registers; heads of 64 175 to 182 (660 to 680 TFLOP/s: the
// exponentials of as many scores beside half the matrix work).  At 256 registers per lane
// a larger tile of either kind spills.
template <int D, bool MX, bool IDX>
__global__ __launch_bounds__(rowsk::NT, 1) void paged_rows_kernel(PagedArgs a) {
    using namespace pg;
    using namespace rowsk;
    constexpr int KS = D / 16, DB = D / 32;               // contraction steps of S^T, 32-dim blocks of O^T
    constexpr int RB = D * 2, KB = TK * RB;               // bytes per staged row, of the keys of a slot
    constexpr int CH = RB / 16;                           // 16-byte chunks per row
    __shared__ __attribute__((aligned(1024))) char slot0[2 * KB], slot1[2 * KB], slot2[2 * KB], slot3[2 * KB];
    __shared__ uint32_t keep[IDX ? ROWS : 1][D / 32];
    __shared__ int state;                                 // a page or length out of range
    __shared__ uint32_t odd_of[NW];                       // rows whose result is not finite

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 31, lh = lane >> 5;
    const int H = a.q.n, grp = H / a.kv.Hkv;
    const int lg = a.kv.lg_page, ps = 1 << lg;
    // scale: a negative one is taken into the queries; zero as the smallest normal
    // float, which leaves the weights of finite scores exactly 1 and of masked ones 0
    const float c = fmaxf(__builtin_fabsf(a.c), 1.17549435e-38f);
    const uint32_t flip = a.c < 0.f ? 0x80008000u : 0u;

    // chunk p of staged row r sits at p ^ swizzle(r): rows that are read together at
    // one chunk fall on distinct banks
    auto kswz = [](int r) { return D == 128 ? r & 15 : (r >> 1) & 7; };
    auto vswz = [](int r) { return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); };
    // K fragment (A of S^T): key row 32 tb + lr, chunk 2 ks + lh: kaddr ^ 32 ks
    const int kaddr = lr * RB + 16 * (lh ^ kswz(lr));
    // V^T fragment (A of O^T): 16-lane group gr reads keys 16 st + 4 (gr / 2) + s16 / 4 (and
    // + 8) of dims 32 db + 16 (gr % 2) + 4 (s16 % 4) .. + 3 (transposing read): vaddr ^ 64 db
    int vaddr;
    {
        const int gr = lane >> 4, s16 = lane & 15, vv = s16 >> 2, qq = s16 & 3, r = 4 * (gr >> 1) + vv;
        vaddr = r * RB + 16 * ((2 * (gr & 1) + (qq >> 1)) ^ vswz(r)) + 8 * (qq & 1);
    }

    int held = 0;                                          // which of the two pieces there are
    Walk<TK, ROWS> w;
    bool more = w.init(a, kMinRun, kCutCost);
    const int wg = w.wg;
    if (w.over) all_nan<D>(a);
    while (more) {
        if (!w.locate(a)) {
            more = w.x < w.end;
            continue;
        }
        const Seq sq = w.s;
        const int kvh = w.kvh, row0 = w.tile * ROWS, n_rows = min(ROWS, sq.n * grp - row0);
        const int hi_lim = a.causal ? sq.len - sq.n + quot(row0 + n_rows - 1, grp) : sq.len - 1;
        const int kend = max(hi_lim + 1, 0);               // keys that some row sees
        const int c_end = kend == 0 ? w.c0 : w.c1;
        const int n_tiles = c_end - w.c0;
        if (tid == 0) state = sq.bad;

        // ---- the wave's rows
        const int rr = wave * 32 + lr, rho = row0 + rr;
        const bool on = rr < n_rows;
        const int tok = on ? rho / grp : 0;
        const int hd = on ? kvh * grp + rho % grp : 0;
        const int lim = !on ? -1 : a.causal ? sq.len - sq.n + tok : sq.len - 1;
        const int wa = row0 + wave * 32, wb = min(wa + 31, row0 + n_rows - 1);      // the wave's rows (none: wb < wa)
        const int tok_a = quot(wa, grp), tok_b = quot(max(wb, wa), grp);
        const int lim_lo = a.causal ? sq.len - sq.n + tok_a : sq.len - 1;      // every row of the wave sees these
        const int lim_hi = wb < wa ? -1 : a.causal ? sq.len - sq.n + tok_b : sq.len - 1;

        // ---- staging
        const int32_t *trow = a.table + w.b * a.table_ld;
        bool bad = false;
        auto page_at = [&](int key, bool in) __attribute__((always_inline)) {
            int pid = in ? trow[key >> lg] : 0;
            const bool ok = pid >= 0 && pid < a.kv.n_pages;
            if (__ballot(!ok)) bad = true;
            return ok ? pid : 0;
        };
        const int64_t hrow = static_cast<int64_t>(kvh) << lg;
        // bf16: the wave stages 8 rows of keys and of values, which lie in one page;
        // lane l holds the page of tile pbase + l
        constexpr int RPW = TK / NW, RPI = 1024 / RB, PER = 2 * (RPW / RPI);     // rows per wave, per DMA instruction
        int pid = 0, pbase = 0;
        auto fetch = [&](int kt) __attribute__((always_inline)) {
            pbase = kt;
            const int key = (kt + lane) * TK + wave * RPW;
            pid = page_at(key, kt + lane < c_end && key < kend);
        };
        auto dma = [&](char *slot, int kt) __attribute__((always_inline)) {
            if (kt - pbase >= 64) fetch(kt);
            const int r = lane / CH, ch = lane % CH;
            const int key = kt * TK + wave * RPW;
            // rows past the last key that some row sees are staged as zeros
            const int rows = uniform(kt < c_end ? max(0, min(RPW, kend - key)) : 0);
            const int64_t page = __builtin_amdgcn_readlane(pid, (kt - pbase) & 63);
            const int64_t at = (hrow + (key & (ps - 1))) * RB;
            // (scalar by construction; said so, since a descriptor that may differ between lanes
            // is loaded from in a loop over its values)
            const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(
                a.kv.k + uniform(page * a.kv.k_page + at), 0, static_cast<uint32_t>(rows * RB), 0x00020000);
            const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(
                a.kv.v + uniform(page * a.kv.v_page + at), 0, static_cast<uint32_t>(rows * RB), 0x00020000);
#pragma unroll
            for (int u = 0; u < RPW / RPI; ++u) {
                const int row = wave * RPW + u * RPI;      // first row of the instruction in the tile
                lds_load16(kr, slot + row * RB, static_cast<uint32_t>((u * RPI + r) * RB + 16 * (ch ^ kswz(row + r))));
                lds_load16(vr, slot + KB + row * RB, static_cast<uint32_t>((u * RPI + r) * RB + 16 * (ch ^ vswz(row + r))));
            }
        };
        // 4-bit: a thread takes groups of 32 dims (16 bytes of codes, a scale byte);
        // lane l holds the page of key block l % 4 (16 keys) of tile pbase + l / 4
        constexpr int GPR = D / 32, UNITS = TK * GPR;      // groups per row, per tile of keys (of values)
        const int mid = tid % UNITS, mrow = mid / GPR, mgrp = mid % GPR;
        const bool mval = tid >= UNITS, mon = tid < 2 * UNITS;
        uint4 codes = make_uint4(0, 0, 0, 0);
        uint32_t scale = 0;
        int pcur = 0, pnext = 0;
        auto mx_pages = [&](int kt) __attribute__((always_inline)) {
            const int key = (kt + (lane >> 2)) * TK + 16 * (lane & 3);
            return page_at(key, kt + (lane >> 2) < c_end && key < kend);
        };
        auto mx_load = [&](int kt) __attribute__((always_inline)) {
            if (kt - pbase >= 16) {
                pcur = pnext;
                pbase += 16;
                pnext = mx_pages(pbase + 16);
            }
            const int key = kt * TK + mrow;
            const int64_t page = __shfl(pcur, (4 * (kt - pbase) + (mrow >> 4)) & 63, 64);
            codes = make_uint4(0, 0, 0, 0);
            scale = 0;
            if (mon && kt < c_end && key < kend) {
                const int64_t row = hrow + (key & (ps - 1));
                const uint8_t *cp = (mval ? a.kv.v + page * a.kv.v_page : a.kv.k + page * a.kv.k_page) + row * (D / 2);
                const uint8_t *sp = (mval ? a.kv.vs + page * a.kv.vs_page : a.kv.ks + page * a.kv.ks_page) + row * GPR;
                codes = reinterpret_cast<const uint4 *>(cp)[mgrp];
                scale = sp[mgrp];
            }
        };
        auto mx_store = [&](char *slot) __attribute__((always_inline)) {
            if (!mon) return;
            char *row = slot + (mval ? KB : 0) + mrow * RB;
            const int swz = mval ? vswz(mrow) : kswz(mrow);
            const uint32_t cw[4] = {codes.x, codes.y, codes.z, codes.w};
            const float sc = __uint_as_float(scale << 23);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<uint4 *>(row + 16 * ((4 * mgrp + j) ^ swz)) = unpack_mx8(cw[j], sc);
        };

        // the first tiles are on their way while the lists and queries are read
        const int t0 = w.c0;
        if constexpr (!MX) {
            fetch(t0);
            dma(slot0, t0);
            dma(slot1, t0 + 1);
        } else {
            pbase = t0;
            pcur = mx_pages(t0);
            pnext = mx_pages(t0 + 16);
            mx_load(t0);
        }

        uint4 qf[KS];
        {
            const uint16_t *qp = static_cast<const uint16_t *>(a.q.p) + (sq.q0 + tok) * a.q.st + hd * a.q.sh;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                qf[ks] = make_uint4(0, 0, 0, 0);
                if (on) qf[ks] = *reinterpret_cast<const uint4 *>(qp + 16 * ks + 8 * lh);
            }
            if constexpr (IDX) {
                read_lists<D, NT, ROWS>(a, sq, kvh, row0, n_rows, keep);
                lds_barrier();
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if constexpr (IDX) qf[ks] = keep8(qf[ks], keep[rr][ks >> 1] >> (16 * (ks & 1) + 8 * lh));
                qf[ks].x ^= flip; qf[ks].y ^= flip; qf[ks].z ^= flip; qf[ks].w ^= flip;
            }
        }

        // ---- one tile's work
        f32x16_t o[DB];
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
        float m_run = -__builtin_inff(), l_run = 0.f;
        // the sum is of the rounded weights where that costs nothing (two chunks of 1024
        // tokens, heads of 64: 182 us, 184 unrounded; heads of 128: 268 against 254, for the same
        // error of 0.0017, so of the unrounded)
        constexpr bool ROUNDED = D == 64;
        f32x16_t s[2];
        uint4 pf[TK / 16];
        // s[tb][v] is key kt * TK + 32 tb + 8 (v / 4) + 4 lh + v % 4 of row lr
        auto qk = [&](const char *slot) __attribute__((always_inline)) {
            uint4 kf[KS][2];                               // all fragments first, so the MFMAs wait once
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) kf[ks][tb] = *reinterpret_cast<const uint4 *>(slot + (kaddr ^ (32 * ks)) + 32 * tb * RB);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int v = 0; v < 16; ++v) s[tb][v] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) s[tb] = mfma(kf[ks][tb], qf[ks], s[tb]);
        };
        auto softmax = [&](int kt) __attribute__((always_inline)) {
            const int t0 = kt * TK;
            if (__builtin_expect(a.c == 0.f, 0)) {         // 0 times an infinite score is NaN
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int v = 0; v < 16; ++v) s[tb][v] *= a.c;
            }
            if (t0 + TK - 1 > lim_lo) {                    // the tile crosses some row's limit
                const int rel = in_branch(lim - t0 - 4 * lh);
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (32 * tb + 8 * (v >> 2) + (v & 3) > rel) s[tb][v] = -__builtin_inff();
            }
            float m4[4] = {-__builtin_inff(), -__builtin_inff(), -__builtin_inff(), -__builtin_inff()};
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int v = 0; v < 16; ++v) m4[v & 3] = fmaxf(m4[v & 3], s[tb][v]);
            const float mx = across_halves(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), fmax2);
            const float mt = mx == -__builtin_inff() ? mx : mx * c;
            const bool need = mt > m_run - kLift;
            if (__ballot(need)) {
                const float m_new = need ? mt + kLift : m_run;
                const float al = need ? exp_two(m_run - m_new) : 1.f;
                l_run *= al;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int v = 0; v < 16; ++v) o[db][v] *= al;
                m_run = m_new;
            }
            const float mu = m_run == -__builtin_inff() ? 0.f : m_run;
            float l4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float p = exp_two(__builtin_fmaf(s[tb][v], c, -mu));
                    s[tb][v] = p;
                    if constexpr (!ROUNDED) l4[v & 3] += p;
                }
            if constexpr (!ROUNDED) l_run += (l4[0] + l4[1]) + (l4[2] + l4[3]);
            // weights of keys 16 st + 8 (e / 4) + 4 lh + e % 4: the order of the V^T fragments
#pragma unroll
            for (int st = 0; st < TK / 16; ++st) {
                const int tb = st >> 1, v0 = 8 * (st & 1);
                pf[st] = make_uint4(pack_bf16x2(s[tb][v0], s[tb][v0 + 1]), pack_bf16x2(s[tb][v0 + 2], s[tb][v0 + 3]),
                                    pack_bf16x2(s[tb][v0 + 4], s[tb][v0 + 5]), pack_bf16x2(s[tb][v0 + 6], s[tb][v0 + 7]));
            }
        };
        auto pv = [&](const char *slot) __attribute__((always_inline)) {
            uint4 vf[TK / 16][DB];                         // all fragments first, so the MFMAs wait once
#pragma unroll
            for (int st = 0; st < TK / 16; ++st)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const char *p = slot + KB + (vaddr ^ (64 * db)) + 16 * st * RB;
                    const s16x4_t lo = lds_read_tr16(p);
                    const s16x4_t hi = lds_read_tr16(p + 8 * RB);
                    vf[st][db] = __builtin_bit_cast(uint4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int st = 0; st < TK / 16; ++st)
#pragma unroll
                for (int db = 0; db < DB; ++db) o[db] = mfma(vf[st][db], pf[st], o[db]);
            if constexpr (ROUNDED) {
                float l4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int st = 0; st < TK / 16; ++st) {
                    l4[0] = add_pair(pf[st].x, l4[0]);
                    l4[1] = add_pair(pf[st].y, l4[1]);
                    l4[2] = add_pair(pf[st].z, l4[2]);
                    l4[3] = add_pair(pf[st].w, l4[3]);
                }
                l_run += (l4[0] + l4[1]) + (l4[2] + l4[3]);
            }
        };

        // ---- the ring: tile c0 + i lives in slot i % 4
        if constexpr (!MX) {
            wait_vmcnt_le<PER>();
        } else {
            mx_store(slot0);
            mx_load(t0 + 1);
        }
        lds_barrier();
        auto slot_at = [&](auto S) -> char * {
            constexpr int sl = decltype(S)::value;
            if constexpr (sl == 0) return slot0;
            else if constexpr (sl == 1) return slot1;
            else if constexpr (sl == 2) return slot2;
            else return slot3;
        };
        const bool late = wave >= NW / 2;
        auto active = [&](int i) { return i >= 0 && i < n_tiles && (t0 + i) * TK <= lim_hi; };
        auto step = [&](auto S, int i) __attribute__((always_inline)) {
            constexpr int sl = decltype(S)::value;
            if constexpr (!MX) {
                dma(slot_at(std::integral_constant<int, (sl + 2) % NS>{}), t0 + i + 2);
            } else {
                mx_store(slot_at(std::integral_constant<int, (sl + 1) % NS>{}));
                mx_load(t0 + i + 2);
            }
            const bool prev = active(i - 1), cur = active(i);
            if (late && prev) softmax(t0 + i - 1);
            if (prev) pv(slot_at(std::integral_constant<int, (sl + 3) % NS>{}));
            if (cur) qk(slot_at(S));
            if (!late && cur) softmax(t0 + i);
            if constexpr (!MX) wait_vmcnt_le<PER>();
            lds_barrier();
        };
        for (int i = 0; i <= n_tiles; i += NS) {
            step(std::integral_constant<int, 0>{}, i);
            if (i + 1 <= n_tiles) step(std::integral_constant<int, 1>{}, i + 1);
            if (i + 2 <= n_tiles) step(std::integral_constant<int, 2>{}, i + 2);
            if (i + 3 <= n_tiles) step(std::integral_constant<int, 3>{}, i + 3);
        }
        wait_vmcnt_le<0>();                                // the trailing loads

        // ---- the unit's rows out
        const bool complete = w.complete();
        const int part = w.part();
        const float l = across_halves(l_run, add2);
        bool odd = !(l < __builtin_inff());
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) odd = odd || !(__builtin_fabsf(o[db][v]) < __builtin_inff());
        const uint64_t odd_lanes = __ballot(on && odd);    // row lr in two of them
        if (lane == 0) {
            odd_of[wave] = static_cast<uint32_t>(odd_lanes | odd_lanes >> 32);
            if (bad) atomicOr(&state, 1);
        }
        __syncthreads();
        const bool none = state != 0;                      // no row of the unit has an answer
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) any |= odd_of[i];
        // an infinite or NaN key (outside a list) or value (of a key that only some rows see)
        // that should not count has made these NaN, as zero times it; without one they are
        // what they should be
        const int lo = a.causal ? sq.len - sq.n + quot(row0, grp) : sq.len - 1;
        const bool redo = !none && __builtin_expect(uniform(static_cast<int>(any)) != 0, 0) &&
                          (IDX || odd_values<D, MX>(a, w.b, kvh, max(lo + 1, w.c0 * TK), min(kend, w.c1 * TK)));
        if (__builtin_expect(redo, 0)) {
            careful_rows<D, MX, IDX>(a, sq, w.b, kvh, row0, n_rows, wave, NW, w.c0 * TK, w.c1 * TK, keep,
                                     [&](int r) { return uniform(static_cast<int>(odd_of[r >> 5] >> (r & 31) & 1)) != 0; },
                                     [&](int r, float m, float ls, int d, float x, float y) {
                if (complete) {
                    const int q = row0 + r;
                    const float inv = row_scale(ls, a.causal ? sq.len - sq.n + q / grp : sq.len - 1);
                    *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(a.o.p) + (sq.q0 + q / grp) * a.o.st +
                                                  (kvh * grp + q % grp) * a.o.sh + d) = pack_bf16x2(x * inv, y * inv);
                } else {
                    const int64_t prow = (2 * static_cast<int64_t>(wg) + part) * ROWS + r;
                    if (d == 0) *reinterpret_cast<float2 *>(a.part_ml + 2 * prow) = make_float2(m, ls);
                    *reinterpret_cast<float2 *>(a.part_o + prow * D + d) = make_float2(x, y);
                }
            });
        }
        if (on && !(redo && (odd_lanes >> lr | odd_lanes >> (lr + 32)) & 1)) {
            const float ls = none ? __builtin_nanf("") : l;
            if (complete) {
                const float inv = row_scale(ls, lim);
                uint16_t *op = static_cast<uint16_t *>(a.o.p) + (sq.q0 + tok) * a.o.st + hd * a.o.sh + 4 * lh;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<uint2 *>(op + 32 * db + 8 * q) =
                            make_uint2(pack_bf16x2(o[db][4 * q] * inv, o[db][4 * q + 1] * inv),
                                       pack_bf16x2(o[db][4 * q + 2] * inv, o[db][4 * q + 3] * inv));
            } else {
                const int64_t prow = (2 * static_cast<int64_t>(wg) + part) * ROWS + rr;
                if (lh == 0) *reinterpret_cast<float2 *>(a.part_ml + 2 * prow) = make_float2(m_run, ls);
                float *po = a.part_o + prow * D + 4 * lh;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<float4 *>(po + 32 * db + 8 * q) =
                            make_float4(o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]);
            }
        }
        if (!complete) {
            if (tid == 0) reinterpret_cast<PieceOf *>(a.pieces)[2 * wg + part] = piece_of(w, n_rows);
            held |= 1 << part;
        }
        w.advance();
        more = w.x < w.end;
        // the ring and the state are free for the next unit, no store is on its way
        wait_vmcnt_le<0>();
        __syncthreads();
    }
    if (tid < 2 && !(held >> tid & 1)) reinterpret_cast<PieceOf *>(a.pieces)[2 * wg + tid].n = 0;
}

constexpr int joins(int rows) { return (rows + 31) / 32; }

// Joins the pieces of the cut units: workgroup i looks at its own two, and of a
// unit cut over workgroups first .. first + n - 1 takes the rows i - first, + n, ...,
// of which the YS workgroups (i, y) take every YS-th (a 256-row unit has too many for one).
// D / 4 lanes take a row's dims; RP rows are joined at once, each by SP of the
// workgroup's groups of lanes (which take every SP-th piece).
// Bound by latency (descriptors, then maxima and sums, then outputs): 4 us where
// nothing was cut, 6 for 16 sequences of one token, up to 20 for 256-row units all cut.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a) {
    using namespace pg;
    constexpr int LD = D / 4, PW = 256 / LD, YS = joins(ROWS);
    __shared__ float4 acc_s[PW][LD];
    __shared__ float2 ml_s[PW];
    const int tid = threadIdx.x, pw = tid / LD, l = tid % LD;
    const int H = a.q.n, grp = H / a.kv.Hkv, wg = static_cast<int>(blockIdx.x);
    for (int part = 0; part < 2; ++part) {
        const PieceOf pc = reinterpret_cast<const PieceOf *>(a.pieces)[2 * wg + part];
        if (pc.n == 0) continue;
        // as many rows at once as this workgroup has
        const int step = pc.n * YS, r0 = wg - pc.first + static_cast<int>(blockIdx.y) * pc.n;
        const int mine = (pc.rows - r0 + step - 1) / step;
        int RP = 1;
        while (RP < PW && RP < mine) RP *= 2;
        const int SP = PW / RP, ri = pw % RP, si = pw / RP;
        for (int i0 = 0; i0 < mine; i0 += RP) {
            const int r = r0 + (i0 + ri) * step;
            float m = -__builtin_inff(), ls = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
            auto add = [&](float mp, float lp, const float4 v) __attribute__((always_inline)) {
                const float mn = fmaxf(m, mp);
                const float a0 = m == -__builtin_inff() ? 0.f : exp_two(m - mn);
                const float a1 = mp == -__builtin_inff() ? 0.f : exp_two(mp - mn);
                // a NaN sum stays one whatever its maximum, and so does an output that is not
                // finite: a visible value was infinite or NaN, and no weight makes 0 of it
                ls = (ls == ls ? ls * a0 : ls) + (lp == lp ? lp * a1 : lp);
                o.x = o.x * a0 + v.x * a1;
                o.y = o.y * a0 + v.y * a1;
                o.z = o.z * a0 + v.z * a1;
                o.w = o.w * a0 + v.w * a1;
                m = mn;
            };
            if (r < pc.rows) {
#pragma unroll 4
                for (int p = si; p < pc.n; p += SP) {
                    // the unit's first piece is its workgroup's last one, the others begin a run
                    const int64_t row = (2 * static_cast<int64_t>(pc.first + p) + (p == 0 ? 1 : 0)) * ROWS + r;
                    const float2 x = *reinterpret_cast<const float2 *>(a.part_ml + 2 * row);
                    add(x.x, x.y, *reinterpret_cast<const float4 *>(a.part_o + row * D + 4 * l));
                }
            }
            if (SP > 1) {
                __syncthreads();
                acc_s[pw][l] = o;
                if (l == 0) ml_s[pw] = make_float2(m, ls);
                __syncthreads();
                if (si == 0) {
                    for (int q = 1; q < SP; ++q) m = fmaxf(m, ml_s[ri + q * RP].x);
                    ls = 0.f;
                    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                    for (int q = 0; q < SP; ++q) {
                        const float2 x = ml_s[ri + q * RP];
                        const float4 v = acc_s[ri + q * RP][l];
                        const float al = x.x == -__builtin_inff() ? 0.f : exp_two(x.x - m);
                        ls += x.y == x.y ? x.y * al : x.y;
                        o.x += v.x * al;
                        o.y += v.y * al;
                        o.z += v.z * al;
                        o.w += v.w * al;
                    }
                }
            }
            if (si == 0 && r < pc.rows) {
                const int rho = pc.row0 + r;
                const float inv = row_scale(ls, a.causal ? pc.lim0 + rho / grp : pc.lim0);
                uint16_t *op = static_cast<uint16_t *>(a.o.p) + (pc.q0 + rho / grp) * a.o.st + (pc.kvh * grp + rho % grp) * a.o.sh + 4 * l;
                *reinterpret_cast<uint2 *>(op) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
            }
        }
    }
}

namespace {

template <int D, bool MX, int ROWS>
hipError_t launch(const PagedArgs &a, hipStream_t stream) {
    if constexpr (ROWS <= 64) {
        constexpr int R = ROWS == 16 ? 1 : 2, RG = ROWS / (16 * R);
        if (a.idx) paged_few_kernel<D, MX, R, RG, true><<<a.nw, few::kThreads, 0, stream>>>(a);
        else paged_few_kernel<D, MX, R, RG, false><<<a.nw, few::kThreads, 0, stream>>>(a);
    } else {
        if (a.idx) paged_rows_kernel<D, MX, true><<<a.nw, rowsk::NT, 0, stream>>>(a);
        else paged_rows_kernel<D, MX, false><<<a.nw, rowsk::NT, 0, stream>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.whole) return e;
    paged_join_kernel<D, ROWS><<<dim3(a.nw, joins(ROWS)), 256, 0, stream>>>(a);
    return hipGetLastError();
}

template <int D, bool MX>
hipError_t launch_rows(const PagedArgs &a, int rows, hipStream_t stream) {
    if (rows == 16) return launch<D, MX, 16>(a, stream);
    if (rows == 32) return launch<D, MX, 32>(a, stream);
    if constexpr (MX) {
        if (rows == 64) return launch<D, MX, 64>(a, stream);
    }
    return launch<D, MX, rowsk::ROWS>(a, stream);
}

}  // namespace

// whether the line is shorter than 2^30 whatever the lengths (keys: what a page
// table row can hold; a unit's share of its pair's length is at most four blocks
// more than the keys')
bool paged_line_fits(int64_t T, int64_t B, int64_t H, int64_t Hkv, bool mx, int D, int64_t keys) {
    const int rows = unit_rows(T, B, H / Hkv, mx, D);
    return (most_units(T, B, H, Hkv, rows) + 1) * (keys / block_keys(rows) + 5) < (int64_t(1) << 30);
}

// two pieces per workgroup: what joins them, their maxima and sums, their outputs
// (the same size for both types of cache)
size_t paged_workspace_bytes(int64_t T, int64_t B, int64_t H, int64_t Hkv, int D) {
    size_t bytes = 0;
    for (bool mx : {false, true}) {
        const int rows = unit_rows(T, B, H / Hkv, mx, D);
        const size_t n = 2 * static_cast<size_t>(workgroups(rows));
        bytes = std::max(bytes, n * (sizeof(pg::PieceOf) + static_cast<size_t>(rows) * (D + 2) * sizeof(float)));
    }
    return bytes;
}

hipError_t launch_paged_attn(PagedArgs a, int D, void *workspace, hipStream_t stream) {
    const int rows = unit_rows(a.T, a.B, a.q.n / a.kv.Hkv, a.kv.mx, D);
    a.nw = workgroups(rows);
    a.whole = never_cut(a, rows);
    a.pieces = workspace;
    a.part_o = reinterpret_cast<float *>(static_cast<char *>(workspace) + 2 * a.nw * sizeof(pg::PieceOf));
    a.part_ml = a.part_o + static_cast<int64_t>(2 * a.nw) * rows * D;
    if (a.kv.mx) return D == 128 ? launch_rows<128, true>(a, rows, stream) : launch_rows<64, true>(a, rows, stream);
    return D == 128 ? launch_rows<128, false>(a, rows, stream) : launch_rows<64, false>(a, rows, stream);
}

}  // namespace rmm
